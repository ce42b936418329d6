// gsd_verify_attn_q8, warp-level back end for few stacked rows: attention of the draft nodes over a cache held in 8
// bits (e4m3 or int8 codes, a power-of-two scale 2^e for each block of tokens and kv head) and a bf16 draft block.
//
//   s_j = scale <q, c_j> 2^(ek_j),   p_j = 2^(s_j log2(e) - m),   out = sum_j p_j 2^(ev_j) w_j / sum_j p_j
//
// with K_j = c_j 2^(ek_j) and V_j = w_j 2^(ev_j).  The codes go to the tensor cores as they are, widened to fp16 (exact:
// four and eight significant bits): ek is one factor of a tile's scores, ev one of its weights, so nothing is
// multiplied per cache element.  fp16 holds a query row exactly once a power of two has brought its maximum to 2^14
// (what falls below 2^-24 then is under 2^-38 of the maximum), and a weight p 2^(8 + ev - e_ref) to 11 bits, e_ref the
// largest ev met so far; the accumulators are in units of 2^(e_ref - 8).  That holds while the scales of V that a warp has
// met lie within 2^12: what is below 2^-14 in fp16, p < 2^-10 at most, is then off by 2^-21 of the row's largest p.  A
// scale that is further away, of a block that a row may give no weight, would take the bits of all others; from such a tile on
// the accumulators are in units of 1 and weights p 2^ev and codes go to the product as bf16, which has the exponents of
// fp32.  Blocks at the least exponent, as the writers give zeros, do not count for the distance.
//
// Every warp has tiles of 16 keys of its own, a ring of them in shared memory filled by asynchronous copies and nothing to
// wait for but its own; the warps meet once, at the end.  What bounds it is instructions: 16 keys (4 KB) of eight rows
// took 522 with rows as the 16 rows of a product (half of them empty); here both products are transposed, S^T = K Q^T and
// O^T = V^T P^T, with 16 keys or columns and 8 rows each, weights turned round by a movmatrix.  A tile's maximum is looked
// at row by row only when a score exceeds the running one by more than 2^7.
//
// Measured (device time, inputs from DRAM): 32 x 64/8 heads, N 1, L 4096 47.9 us, 85% of the copy rate, int8 48.3; 8 x 64/8, N 1, L
// 500-4000 14.9 us (22.1 over a bf16 cache); 4 x 32/8 heads of 64, N 12, L 1000-4000 16.6 us (15.4); 1 x 32 heads, N 64, L 2048 22.6 us
// (14.9).  With half of the blocks 2^14 below the others, on the bf16 products, such calls take 0 to 6% more.  With 32 rows latency bounds it:
// an instruction in 29% of the cycles of two warps a scheduler, the tensor pipe 21% busy, most of the waiting for instructions
// to be fetched (the loop is unrolled over rows and columns) and for fixed latencies; with 24 rows of 64 43% and 18%.  48 rows as 24 and 24, not 32 and 16, two CTAs an SM there and
// draft rows asked for ahead of time took the heads of 64 from 19.6 to 16.4 us; two CTAs with 32 rows spill (4 x 32/8 heads
// of 64, N 8, L 4000: 21.6 instead of 17.3 us, as both were then).
//
// A lane takes its operands from whole 16-byte pieces of a row: the order of the head dimension inside a product
// is free (queries are loaded in the same order), and so is the order of the output columns.
#include "gsd_internal.cuh"
#include "gsd_kv8.cuh"
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

namespace gsd {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kKeys = 16;                    // keys of a warp's tile
constexpr int kWeightBits = 8;               // what weights are brought up by in fp16
constexpr int kSpread = 12;                  // log2 of how far the scales of V may lie apart for weights in fp16
constexpr float kLag = 7.f;                  // the running maximum of a row may lag behind by this much (log2 units): weights stay below 2^15

struct Q8Params {
    const __nv_bfloat16 *q, *draft_k, *draft_v;
    const uint8_t *k_cache, *v_cache;
    const int8_t *k_exp, *v_exp;
    const uint32_t* mask;
    const int32_t* seq_lens;
    __nv_bfloat16* out;
    float* part_o;   // [slot][D / 4][64] float4
    float* part_ml;  // [slot][64][2]
    PlanDev plan;
    int32_t* status;
    int B, N, Hq, Hkv, Lmax, G, W, R;
    int NB, block_log2;                      // scale blocks of a sequence, log2 of their tokens
    int slots;
    float scale_log2;
};

template <int D, int NT>
struct Q8Geo {
    static constexpr int ROWS = 8 * NT;                         // stacked rows of an item
    static constexpr int TILE = kKeys * D;                      // bytes of a K or V tile
    static constexpr int BLOCKS = NT <= 2 || (NT == 3 && D == 64) ? 2 : 1;   // CTAs an SM, as their registers allow
    static constexpr int STAGES = BLOCKS == 2 && D == 128 ? 3 : 5;
    static constexpr int RING = kWarps * STAGES * 2 * TILE;
    static constexpr int MTILES = D / 16;                       // output tiles of 16 columns
    static constexpr int VALUES = NT * (MTILES * 4 + 4);        // of a thread, when the warps' results are brought together
    static constexpr int MEET = kWarps * VALUES * 32 * 4;
    static constexpr int Q_AT = RING > MEET ? RING : MEET;      // query fragments: [row group][k-step][lane] pairs of registers
    static constexpr int SMEM = Q_AT + NT * (D / 16) * 32 * 8;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16-byte async copy; src_bytes == 0 writes zeros and reads nothing
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int src_bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Pairs in place, an instruction for both.
__device__ __forceinline__ void mul2(float& a0, float& a1, float b0, float b1) {
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}" : "+f"(a0), "+f"(a1) : "f"(b0), "f"(b1));
}
__device__ __forceinline__ void add2(float& a0, float& a1, float b0, float b1) {
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}" : "+f"(a0), "+f"(a1) : "f"(b0), "f"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// Two fp16 values of up to eight significant bits as bf16.
__device__ __forceinline__ uint32_t bf16_from_f16(uint32_t v) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
    return pack_bf16(f.x, f.y);
}
// 8x8 fp16 or bf16 values, a row a quarter of lanes -> their transpose.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}

template <int D, int NT, bool INT8>
__global__ void __launch_bounds__(kThreads, Q8Geo<D, NT>::BLOCKS) attn_q8_mma_kernel(Q8Params p) {
    using T = Q8Geo<D, NT>;
    constexpr int KS = D / 16;              // k-steps of the product with K
    constexpr int MTL = T::MTILES;          // output tiles
    constexpr int ST = T::STAGES;
    extern __shared__ __align__(128) unsigned char smem[];

    if (p.slots > 0) let_successor_start();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int i8 = lane >> 2, j4 = lane & 3;
    int item, split, nsplit, slot;
    plan_decode(p.plan, blockIdx.x, item, split, nsplit, slot);
    const int unit = item / p.plan.tiles_per_unit;   // b * Hkv + c
    const int row0 = (item % p.plan.tiles_per_unit) * T::ROWS;
    const int b = unit / p.Hkv, c = unit % p.Hkv;
    const int N = p.N, G = p.G, R = p.R;

    wait_for_predecessor();
    int L = p.seq_lens[b];
    if (L < 0 || L > p.Lmax) {
        if (tid == 0 && p.status) atomicOr((unsigned*)p.status, GSD_DEV_BAD_SEQ_LEN);
        L = L < 0 ? 0 : p.Lmax;
    }
    // Key tiles of 16: the prefix, then the draft block.  The CTA has [t_begin, t_end) of them, the warp every eighth.
    const int nPT = (L + kKeys - 1) / kKeys, nT = nPT + (N + kKeys - 1) / kKeys;
    const int per = (nT + nsplit - 1) / nsplit;
    const int t_begin = min(split * per, nT), t_end = min(t_begin + per, nT);
    const int first = t_begin + warp;
    const int n_prefix = max(0, (min(t_end, nPT) - first + kWarps - 1) / kWarps);       // prefix tiles of this warp

    // ---- the ring: K and V tiles of 16 rows, 16-byte pieces swizzled for the reads below
    const uint32_t ring = smem_u32(smem) + warp * (ST * 2 * T::TILE);
    const size_t row_bytes = (size_t)p.Hkv * D;
    constexpr int PIECES = D / 16, LANE_ROWS = 32 / PIECES;                              // of a row; rows a copy of the warp takes
    auto k_off = [](int r, int ch) -> uint32_t {
        if (D == 128) return (uint32_t)(r * 128 + ((ch ^ ((r & 1) << 2)) << 4));
        return (uint32_t)((r >> 1) * 128 + ((((r & 1) << 2) + ch) << 4));
    };
    auto v_off = [](int r, int ch) -> uint32_t {
        if (D == 128) return (uint32_t)(r * 128 + ((ch ^ (r & 6)) << 4));
        return (uint32_t)((r >> 1) * 128 + (((((r & 1) << 2) + ch) ^ (((r >> 1) & 3) << 1)) << 4));
    };
    // where the lane's pieces of the next tile to be copied come from
    const int my_row = lane / PIECES, my_piece = lane % PIECES;
    int copy_key = first * kKeys + my_row;
    const uint8_t* copy_k = p.k_cache + ((size_t)b * p.Lmax * p.Hkv + c) * D + (size_t)copy_key * row_bytes + my_piece * 16;
    const ptrdiff_t k_to_v = p.v_cache - p.k_cache;
    auto issue = [&](uint32_t stage) {
#pragma unroll
        for (int x = 0; x < kKeys / LANE_ROWS; ++x) {
            const int r = x * LANE_ROWS + my_row;
            const bool ok = copy_key + x * LANE_ROWS < L && GSD_IN_BOUNDS(copy_key + x * LANE_ROWS < p.Lmax && b < p.B && c < p.Hkv, p.status);
            const uint8_t* src = ok ? copy_k + (size_t)(x * LANE_ROWS) * row_bytes : p.k_cache;
            cp_async16(stage + k_off(r, my_piece), src, ok ? 16 : 0);
            cp_async16(stage + T::TILE + v_off(r, my_piece), src + k_to_v, ok ? 16 : 0);
        }
        copy_key += kWarps * kKeys;
        copy_k += (size_t)(kWarps * kKeys) * row_bytes;
    };
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) {
        if (s < n_prefix) issue(ring + s * (2 * T::TILE));
        cp_async_commit();
    }
    // The draft tiles come last, as a chain of mask, keys and values: asked for from DRAM now.
    for (int t = first + n_prefix * kWarps; t < t_end; t += kWarps) {
        const int row = (t - nPT) * kKeys + (lane & 15);
        if (row < N) {
            const size_t at = (((size_t)b * N + row) * p.Hkv + c) * D;
            const __nv_bfloat16* src = lane < 16 ? p.draft_k + at : p.draft_v + at;
#pragma unroll
            for (int x = 0; x < D; x += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(src + x) : "memory");
        }
        for (int node = row0 / G + lane; node <= min(row0 + T::ROWS - 1, R - 1) / G; node += 32)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p.mask + ((size_t)b * N + node) * p.W + ((t - nPT) * kKeys >> 5)) : "memory");
    }
    // The exponents of the warp's next 32 tiles, a tile a lane (a tile lies in one block: 16 divides a block).
    auto load_exps = [&](int i0) -> int {
        const int i = i0 + lane;
        if (i >= n_prefix) return 0;
        const int blk = ((first + i * kWarps) * kKeys) >> p.block_log2;
        if (!GSD_IN_BOUNDS(blk < p.NB, p.status)) return 0;
        const size_t at = ((size_t)b * p.NB + blk) * p.Hkv + c;
        return (int)(uint8_t)p.k_exp[at] | (int)p.v_exp[at] << 8;
    };
    int exps = 0, exps_next = load_exps(0);

    // ---- the query rows as fp16 fragments (rows are columns of the products), each lifted by a power of two: a warp for
    // every eight rows puts them where all warps find them
    __shared__ float s_mult[NT * 8];
    const uint32_t q_at = smem_u32(smem) + T::Q_AT + lane * 8;
    if (warp < NT) {
        const int row = row0 + warp * 8 + i8;
        const bool in = row < R;
        const int rr = in ? row : 0;
        const __nv_bfloat16* q = p.q + (((size_t)b * N + rr / G) * p.Hq + c * G + rr % G) * D + j4 * 16;
        uint32_t w[D / 8];
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
            const uint4 v = in ? *reinterpret_cast<const uint4*>(q + (x >> 1) * 64 + (x & 1) * 8) : make_uint4(0, 0, 0, 0);
            w[x * 4] = v.x; w[x * 4 + 1] = v.y; w[x * 4 + 2] = v.z; w[x * 4 + 3] = v.w;
        }
        uint32_t top = 0;
#pragma unroll
        for (int x = 0; x < D / 8; ++x) top = max(top, max((w[x] & 0x7FFFu), (w[x] >> 16) & 0x7FFFu));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const int ex = lift_exp(top);
        const float lift = two(kLiftBits - ex);
        if (j4 == 0) s_mult[warp * 8 + i8] = p.scale_log2 * two(ex - kLiftBits);
        auto half2 = [&](uint32_t v) { return pack_f16(__uint_as_float(v << 16) * lift, __uint_as_float(v & 0xFFFF0000u) * lift); };
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(q_at + (warp * KS + ks) * 256), "r"(half2(w[ks * 2])), "r"(half2(w[ks * 2 + 1])) : "memory");
    }
    __syncthreads();
    uint2 qf[NT == 1 ? KS : 1];
    if (NT == 1) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[NT == 1 ? ks : 0] = lds64(q_at + ks * 256);
    }
    float row_mult[NT][2];                  // of the rows whose scores the thread holds: 8 nt + 2 j4 + {0, 1}
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        row_mult[nt][0] = s_mult[nt * 8 + 2 * j4];
        row_mult[nt][1] = s_mult[nt * 8 + 2 * j4 + 1];
    }

    float o[NT][MTL][4];                    // columns (D / 8) i8 + 2 mt and the one behind it, of the thread's two rows
    float m_run[NT][2], l_run[NT][2];       // l: the lane's own keys
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int mt = 0; mt < MTL; ++mt) o[nt][mt][0] = o[nt][mt][1] = o[nt][mt][2] = o[nt][mt][3] = 0.f;
        m_run[nt][0] = m_run[nt][1] = -CUDART_INF_F;
        l_run[nt][0] = l_run[nt][1] = 0.f;
    }
    int e_ref = -126;                                                                    // accumulators: units of 2^(e_ref - kWeightBits)
    int e_low = 127;                                                                     // the least scale of V met, GSD_KV8_EXP_MIN aside
    bool apart = false;                                                                  // the scales are too far apart for fp16
    auto back_from = [](int from, int to) { return from - to < -126 ? 0.f : two(from - to); };

    // Products s (times mult[.][.]: log2 units; hidden ones -inf) -> weights 2^(s - m) in place.  The running maximum is
    // raised when a score exceeds it by more than kLag; the accumulators then follow, as they do a larger unit.
    // (The maximum is taken off rounded scores, not off the products in one step: the largest product differs from the maximum
    // by what that was rounded by, 2^6 where scores are 2^30, and its weight was then beyond fp16.)
    auto softmax = [&](float (&s)[NT][4], const float (&mult)[NT][2], float unit_back) {
        bool raise = unit_back != 1.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mul2(s[nt][0], s[nt][1], mult[nt][0], mult[nt][1]);
            mul2(s[nt][2], s[nt][3], mult[nt][0], mult[nt][1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) raise |= fmaxf(s[nt][e], s[nt][e + 2]) - m_run[nt][e] > kLag;
        }
        if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float a[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float mx = fmaxf(s[nt][e], s[nt][e + 2]);
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, x));
                    const float m_new = fmaxf(m_run[nt][e], mx), m_use = m_new == -CUDART_INF_F ? 0.f : m_new;   // (nothing visible yet)
                    a[e] = fast_exp2(m_run[nt][e] - m_use);
                    m_run[nt][e] = m_new;
                    l_run[nt][e] *= a[e];
                    a[e] *= unit_back;
                }
#pragma unroll
                for (int mt = 0; mt < MTL; ++mt) {
                    o[nt][mt][0] *= a[0]; o[nt][mt][2] *= a[0];
                    o[nt][mt][1] *= a[1]; o[nt][mt][3] *= a[1];
                }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float off[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) off[e] = m_run[nt][e] == -CUDART_INF_F ? 0.f : -m_run[nt][e];
            add2(s[nt][0], s[nt][1], off[0], off[1]);
            add2(s[nt][2], s[nt][3], off[0], off[1]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[nt][e] = fast_exp2(s[nt][e]);
#pragma unroll
            for (int e = 0; e < 2; ++e) l_run[nt][e] += s[nt][e] + s[nt][e + 2];
        }
    };

    uint32_t stage = ring, fill = ring + (ST - 1) * (2 * T::TILE);
    const uint32_t ring_end = ring + ST * (2 * T::TILE);
#pragma unroll 1
    for (int i = 0; i < n_prefix; ++i) {
        if (i + ST - 1 < n_prefix) issue(fill);
        cp_async_commit();
        fill = stage;
        if ((i & 31) == 0) {
            exps = exps_next;
            exps_next = load_exps(i + 32);
        }
        const int ex = __shfl_sync(0xFFFFFFFFu, exps, i & 31);
        const int ek = max((int)(int8_t)(ex & 255), -126), ev = max(ex >> 8, -126);
        cp_async_wait<ST - 1>();
        __syncwarp();
        const uint32_t sk = stage, sv = stage + T::TILE;
        stage += 2 * T::TILE;
        if (stage == ring_end) stage = ring;

        // S^T = K Q^T: 16 keys (i8, i8 + 8) x 8 rows; two chains at least
        constexpr int CHAINS = NT == 1 ? 2 : 1;
        float s[NT][4], s1[CHAINS][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[nt][e] = s1[0][e] = 0.f;
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
            const uint4 k0 = lds128(sk + k_off(i8, x * 4 + j4)), k1 = lds128(sk + k_off(8 + i8, x * 4 + j4));
            const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                uint32_t a[4];
                widen<INT8>(w0[y], a[0], a[2]);
                widen<INT8>(w1[y], a[1], a[3]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint2 q = NT == 1 ? qf[NT == 1 ? x * 4 + y : 0] : lds64(q_at + (nt * KS + x * 4 + y) * 256);
                    mma_f16(NT == 1 && (y & 1) ? s1[0] : s[nt], a, q.x, q.y);
                }
            }
        }
        float mult[NT][2];
        const float sk2 = two(ek);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mult[nt][0] = row_mult[nt][0] * sk2;
            mult[nt][1] = row_mult[nt][1] * sk2;
            if (NT == 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nt][e] += s1[0][e];
            }
        }
        const int key = (first + i * kWarps) * kKeys + i8;
        if (key - i8 + kKeys > L) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    mult[nt][e] = fmaxf(mult[nt][e], 1.2e-38f);                          // (0 times -inf)
                    if (key >= L) s[nt][e] = -CUDART_INF_F;
                    if (key + 8 >= L) s[nt][e + 2] = -CUDART_INF_F;
                }
        }
        float back = 1.f;
        if (!apart && (ev > e_ref || (ev < e_low && ev > GSD_KV8_EXP_MIN))) {
            if (ev > GSD_KV8_EXP_MIN) e_low = min(e_low, ev);
            const int top = max(ev, e_ref);
            apart = top - e_low > kSpread;
            const int to = apart ? kWeightBits : top;
            back = back_from(e_ref, to);
            e_ref = to;
        }
        softmax(s, mult, back);
        // (zeros far below the unit: their weights vanish in fp16)
        const float unit = two(apart ? ev : max(ev - e_ref + kWeightBits, -40));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mul2(s[nt][0], s[nt][1], unit, unit);
            mul2(s[nt][2], s[nt][3], unit, unit);
        }
        // O^T += V^T P^T: the lane's keys are 2 j4, 2 j4 + 1, and these + 8; its columns (D / 8) i8 + 2 mt and the one behind
        uint32_t vw[4][D / 32];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int r = 2 * j4 + (x & 1) + (x >> 1) * 8;
            if constexpr (D == 128) {
                const uint4 v = lds128(sv + v_off(r, i8));
                vw[x][0] = v.x; vw[x][1] = v.y; vw[x][2] = v.z; vw[x][3] = v.w;
            } else {
                const uint2 v = lds64(sv + v_off(r, i8 >> 1) + (i8 & 1) * 8);
                vw[x][0] = v.x; vw[x][1] = v.y;
            }
        }
        uint32_t pf[NT][2];
        if (!apart) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                pf[nt][0] = transpose8(pack_f16(s[nt][0], s[nt][1]));
                pf[nt][1] = transpose8(pack_f16(s[nt][2], s[nt][3]));
            }
#pragma unroll
            for (int y = 0; y < D / 32; ++y)
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    uint32_t a[4];
                    widen<INT8>(__byte_perm(vw[0][y], vw[1][y], z ? 0x7362 : 0x5140), a[0], a[1]);
                    widen<INT8>(__byte_perm(vw[2][y], vw[3][y], z ? 0x7362 : 0x5140), a[2], a[3]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][y * 2 + z], a, pf[nt][0], pf[nt][1]);
                }
        } else {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                pf[nt][0] = transpose8(pack_bf16(s[nt][0], s[nt][1]));
                pf[nt][1] = transpose8(pack_bf16(s[nt][2], s[nt][3]));
            }
#pragma unroll
            for (int y = 0; y < D / 32; ++y)
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    uint32_t a[4];
                    widen<INT8>(__byte_perm(vw[0][y], vw[1][y], z ? 0x7362 : 0x5140), a[0], a[1]);
                    widen<INT8>(__byte_perm(vw[2][y], vw[3][y], z ? 0x7362 : 0x5140), a[2], a[3]);
#pragma unroll
                    for (int x = 0; x < 4; ++x) a[x] = bf16_from_f16(a[x]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_bf16(o[nt][y * 2 + z], a, pf[nt][0], pf[nt][1]);
                }
        }
        __syncwarp();                       // the stage has been read: a copy may take its place
    }
    cp_async_wait<0>();

    // ---- draft tiles: bf16 rows straight from global memory, by bf16 products
    if (n_prefix * kWarps + first < t_end) {
        // in units of 1: the rows are not scaled, and weights have the exponents of fp32
        const float back = back_from(e_ref, kWeightBits);
        e_ref = kWeightBits;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][mt][e] *= back;
        const __nv_bfloat16* dk = p.draft_k + ((size_t)b * N * p.Hkv + c) * D;
        const __nv_bfloat16* dv = p.draft_v + ((size_t)b * N * p.Hkv + c) * D;
#pragma unroll 1
        for (int t = first + n_prefix * kWarps; t < t_end; t += kWarps) {
            const int key0 = (t - nPT) * kKeys;
            uint32_t bits[NT][2], any = 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = row0 + nt * 8 + 2 * j4 + e;
                    uint32_t w = 0;
                    if (row < R) w = p.mask[((size_t)b * N + row / G) * p.W + (key0 >> 5)] >> (key0 & 16);
                    if (N - key0 < kKeys) w &= (1u << (N - key0)) - 1u;
                    any |= bits[nt][e] = w & 0xFFFFu;
                }
            const uint32_t seen = __reduce_or_sync(0xFFFFFFFFu, any);     // keys that any row sees: others are not read
            if (!seen) continue;
            float s[NT][4], mult[NT][2];
            uint32_t kw[2][D / 8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = h * 8 + i8;
                const bool ok = (seen >> at) & 1u;
                const __nv_bfloat16* src = dk + (size_t)(ok ? key0 + at : 0) * row_bytes + j4 * 16;
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    const uint4 v = ok ? *reinterpret_cast<const uint4*>(src + (x >> 1) * 64 + (x & 1) * 8) : make_uint4(0, 0, 0, 0);
                    kw[h][x * 4] = v.x; kw[h][x * 4 + 1] = v.y; kw[h][x * 4 + 2] = v.z; kw[h][x * 4 + 3] = v.w;
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int row = row0 + nt * 8 + i8;
                const bool in = row < R;
                const __nv_bfloat16* q = p.q + (((size_t)b * N + (in ? row / G : 0)) * p.Hq + c * G + (in ? row % G : 0)) * D + j4 * 16;
                s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
                mult[nt][0] = mult[nt][1] = p.scale_log2;
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {               // two k-steps: eight elements of a row
                    const uint4 v = in ? *reinterpret_cast<const uint4*>(q + (x >> 1) * 64 + (x & 1) * 8) : make_uint4(0, 0, 0, 0);
                    const uint32_t a0[4] = {kw[0][x * 4], kw[1][x * 4], kw[0][x * 4 + 1], kw[1][x * 4 + 1]};
                    const uint32_t a1[4] = {kw[0][x * 4 + 2], kw[1][x * 4 + 2], kw[0][x * 4 + 3], kw[1][x * 4 + 3]};
                    mma_bf16(s[nt], a0, v.x, v.y);
                    mma_bf16(s[nt], a1, v.z, v.w);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!((bits[nt][e & 1] >> (i8 + (e >> 1) * 8)) & 1u)) s[nt][e] = -CUDART_INF_F;
            }
            softmax(s, mult, 1.f);
            uint32_t pf[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                pf[nt][0] = transpose8(pack_bf16(s[nt][0], s[nt][1]));
                pf[nt][1] = transpose8(pack_bf16(s[nt][2], s[nt][3]));
            }
#pragma unroll
            for (int y = 0; y < D / 64; ++y) {                   // eight columns of a lane at a time
                uint32_t w[4][4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int at = 2 * j4 + (x & 1) + (x >> 1) * 8;
                    const bool ok = (seen >> at) & 1u;
                    const uint4 v = ok ? *reinterpret_cast<const uint4*>(dv + (size_t)(key0 + at) * row_bytes + i8 * (D / 8) + y * 8) : make_uint4(0, 0, 0, 0);
                    w[x][0] = v.x; w[x][1] = v.y; w[x][2] = v.z; w[x][3] = v.w;
                }
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const uint32_t a[4] = {__byte_perm(w[0][z], w[1][z], 0x5410), __byte_perm(w[0][z], w[1][z], 0x7632),
                                           __byte_perm(w[2][z], w[3][z], 0x5410), __byte_perm(w[2][z], w[3][z], 0x7632)};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_bf16(o[nt][y * 4 + z], a, pf[nt][0], pf[nt][1]);
                }
            }
        }
    }

    // ---- the warps' results meet in the memory of the rings, each warp brings a share of the columns together
    const float in_units = back_from(e_ref, kWeightBits);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) l_run[nt][e] += __shfl_xor_sync(0xFFFFFFFFu, l_run[nt][e], x);
    float* const part = reinterpret_cast<float*>(smem) + lane;
    auto part_of = [&](int w, int nt) { return part + (w * NT + nt) * (T::VALUES / NT * 32); };
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float* at = part_of(warp, nt);
#pragma unroll
        for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e) at[(mt * 4 + e) * 32] = o[nt][mt][e] * in_units;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            at[(MTL * 4 + e) * 32] = m_run[nt][e];
            at[(MTL * 4 + 2 + e) * 32] = l_run[nt][e];
        }
    }
    __syncthreads();
    // (D = 64: half as many output tiles as warps; the row groups are shared out too)
    constexpr int SHARERS = kWarps / MTL;
    const int mt = warp % MTL;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        if (SHARERS > 1 && nt % SHARERS != warp / MTL) continue;
        float w[kWarps][2], m[2], l[2], r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            m[e] = -CUDART_INF_F;
            l[e] = 0.f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                w[k][e] = part_of(k, nt)[(MTL * 4 + e) * 32];
                m[e] = fmaxf(m[e], w[k][e]);
            }
            const float m_use = m[e] == -CUDART_INF_F ? 0.f : m[e];
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                w[k][e] = fast_exp2(w[k][e] - m_use);
                l[e] += w[k][e] * part_of(k, nt)[(MTL * 4 + 2 + e) * 32];
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int k = 0; k < kWarps; ++k) r[e] += w[k][e & 1] * part_of(k, nt)[(mt * 4 + e) * 32];
        const int col = i8 * (D / 8) + 2 * mt;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int rloc = nt * 8 + 2 * j4 + e, row = row0 + rloc;
            if (row >= R) continue;
            if (nsplit == 1) {
                if (!GSD_IN_BOUNDS(b < p.B && c < p.Hkv && row < p.R, p.status)) continue;
                const float inv = l[e] > 0.f ? 1.f / l[e] : 0.f;
                *reinterpret_cast<uint32_t*>(p.out + (((size_t)b * N + row / G) * p.Hq + c * G + row % G) * D + col) = pack_bf16(r[e] * inv, r[e + 2] * inv);
            } else {
                if (!GSD_IN_BOUNDS(slot >= 0 && slot < p.slots, p.status)) continue;
                *reinterpret_cast<float2*>(p.part_o + (((size_t)slot * (D / 4) + col / 4) * 64 + rloc) * 4 + col % 4) = make_float2(r[e], r[e + 2]);
                if (mt == 0 && i8 == 0) *reinterpret_cast<float2*>(p.part_ml + ((size_t)slot * 64 + rloc) * 2) = make_float2(m[e], l[e]);
            }
        }
    }
}

template <int D, int NT, bool INT8>
int launch_t(const AttnArgs& a) {
    Q8Params p;
    p.q = (const __nv_bfloat16*)a.q; p.draft_k = (const __nv_bfloat16*)a.draft_k; p.draft_v = (const __nv_bfloat16*)a.draft_v;
    p.k_cache = (const uint8_t*)a.k_cache; p.v_cache = (const uint8_t*)a.v_cache;
    p.k_exp = a.kv8.k_exp; p.v_exp = a.kv8.v_exp; p.NB = a.kv8.blocks; p.block_log2 = a.kv8.block_log2;
    p.mask = a.mask; p.seq_lens = a.seq_lens; p.out = (__nv_bfloat16*)a.out; p.status = a.status;
    p.B = a.B; p.N = a.N; p.Hq = a.Hq; p.Hkv = a.Hkv; p.Lmax = a.Lmax; p.G = a.G; p.W = a.W; p.R = a.N * a.G;
    p.scale_log2 = a.scale_log2; p.plan = a.plan.dev; p.slots = a.plan.slots;
    p.part_o = (float*)a.workspace;
    p.part_ml = (float*)((char*)a.workspace + plan_part_o_bytes(a.plan, a.D));
    constexpr int smem = Q8Geo<D, NT>::SMEM;
    {
        static bool done[64] = {};   // per template instance: the opt-in sticks per device
        int dev = 0;
        GSD_CUDA_TRY(cudaGetDevice(&dev));
        if (dev < 0 || dev >= 64 || !done[dev]) {
            GSD_CUDA_TRY(cudaFuncSetAttribute(attn_q8_mma_kernel<D, NT, INT8>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
            if (dev >= 0 && dev < 64) done[dev] = true;
        }
    }
    GSD_CUDA_TRY(launch_dependent(attn_q8_mma_kernel<D, NT, INT8>, dim3(a.plan.ctas), dim3(kThreads), smem, a.stream, p));
    return GSD_OK;
}
template <int D, int NT>
int launch_fmt(const AttnArgs& a) { return a.kv8.int8 ? launch_t<D, NT, true>(a) : launch_t<D, NT, false>(a); }

}  // namespace

// As few items as 32 rows each allow, with the row groups shared out evenly.
int attn_q8_mma_rows(int R) {
    const int items = (R + 31) / 32, groups = (R + 7) / 8;
    return 8 * ((groups + items - 1) / items);
}
int attn_q8_mma_resident(int R, int D) {
    const int rows = attn_q8_mma_rows(R);
    return rows <= 16 || (rows == 24 && D == 64) ? 2 : 1;
}

template <int D>
static int launch_d(const AttnArgs& a) {
    switch (a.plan.rows_per_item) {
        case 8: return launch_fmt<D, 1>(a);
        case 16: return launch_fmt<D, 2>(a);
        case 24: return launch_fmt<D, 3>(a);
        default: return launch_fmt<D, 4>(a);
    }
}

int launch_attn_q8_mma(const AttnArgs& a) {
    if (a.D == 128) return launch_d<128>(a);
    if (a.D == 64) return launch_d<64>(a);
    return GSD_ERR_BAD_SHAPE;
}

}  // namespace gsd
