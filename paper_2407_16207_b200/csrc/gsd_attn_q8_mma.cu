// gsd_verify_attn_q8, warp-level back end for few stacked rows: attention of the draft nodes over a cache held in 8
// bits (e4m3 or int8 codes, a power-of-two scale 2^e for each block of tokens and kv head) and a bf16 draft block.
//
//   s_j = scale <q, c_j> 2^(ek_j),   p_j = 2^(s_j log2(e) - m),   out = sum_j p_j 2^(ev_j) w_j / sum_j p_j
//
// with K_j = c_j 2^(ek_j) and V_j = w_j 2^(ev_j).  The codes go to the tensor cores as they are, widened to fp16 (exact:
// four and eight significant bits): ek is one factor of a tile's scores, ev one of its weights, so nothing is
// multiplied per cache element.  fp16 holds a query row exactly once a power of two has brought its maximum to 2^14
// (what falls below 2^-24 then is under 2^-38 of the maximum), and a weight p 2^(14 + ev - e_ref) to 11 bits, e_ref the
// largest ev met so far; the accumulators are in units of 2^(e_ref - 14).
//
// What bounds it: the one read of the codes.  Every warp has tiles of 16 keys of its own, a ring of them in shared
// memory filled by asynchronous copies and nothing to wait for but its own; the warps meet once, at the end.
// Widening costs one conversion for two e4m3 codes, and five integer or half instructions for four int8 codes.
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

template <int D, int MT>
struct Q8Geo {
    static constexpr int ROWS = 16 * MT;                        // stacked rows of an item
    static constexpr int TILE = kKeys * D;                      // bytes of a K or V tile
    static constexpr int STAGES = MT == 1 ? 3 : D == 128 ? 5 : 6;
    static constexpr int BLOCKS = MT == 1 ? 2 : 1;              // CTAs an SM
    static constexpr int RING = kWarps * STAGES * 2 * TILE;
    static constexpr int VALUES = MT * (D / 8 * 4 + 4);         // of a thread, when the warps' results are brought together
    static constexpr int MEET = kWarps * VALUES * 32 * 4;
    static constexpr int SMEM = RING > MEET ? RING : MEET;
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
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
template <int D, int MT, bool INT8>
__global__ void __launch_bounds__(kThreads, Q8Geo<D, MT>::BLOCKS) attn_q8_mma_kernel(Q8Params p) {
    using T = Q8Geo<D, MT>;
    constexpr int KS = D / 16;              // k-steps of the QK^T product
    constexpr int DT = D / 8;               // output n-tiles
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
    const uint8_t* kbase = p.k_cache + ((size_t)b * p.Lmax * p.Hkv + c) * D;
    const uint8_t* vbase = p.v_cache + ((size_t)b * p.Lmax * p.Hkv + c) * D;
    constexpr int PIECES = D / 16;                                                       // of a row
    auto k_off = [](int r, int ch) -> uint32_t {
        if (D == 128) return (uint32_t)(r * 128 + ((ch ^ ((r & 1) << 2)) << 4));
        return (uint32_t)((r >> 1) * 128 + ((((r & 1) << 2) + ch) << 4));
    };
    auto v_off = [](int r, int ch) -> uint32_t {
        if (D == 128) return (uint32_t)(r * 128 + ((ch ^ (r & 6)) << 4));
        return (uint32_t)((r >> 1) * 128 + (((((r & 1) << 2) + ch) ^ (((r >> 1) & 3) << 1)) << 4));
    };
    auto issue = [&](int i) {
        const int key0 = (first + i * kWarps) * kKeys;
        const uint32_t sk = ring + (i % ST) * (2 * T::TILE), sv = sk + T::TILE;
#pragma unroll
        for (int x = 0; x < kKeys * PIECES / 32; ++x) {
            const int at = x * 32 + lane, r = at / PIECES, ch = at % PIECES;
            const bool ok = key0 + r < L && GSD_IN_BOUNDS(key0 + r < p.Lmax && b < p.B && c < p.Hkv, p.status);
            const size_t off = (size_t)(ok ? key0 + r : 0) * row_bytes + ch * 16;
            cp_async16(sk + k_off(r, ch), kbase + off, ok ? 16 : 0);
            cp_async16(sv + v_off(r, ch), vbase + off, ok ? 16 : 0);
        }
    };
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) {
        if (s < n_prefix) issue(s);
        cp_async_commit();
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

    // ---- the query rows as fp16 fragments, each lifted by a power of two
    uint32_t qf[MT][KS][4];
    float row_mult[MT][2];
    bool rvalid[MT][2];
    const __nv_bfloat16* qrow[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = row0 + mt * 16 + h * 8 + i8;
            rvalid[mt][h] = row < R;
            const int rr = rvalid[mt][h] ? row : 0;
            qrow[mt][h] = p.q + (((size_t)b * N + rr / G) * p.Hq + c * G + rr % G) * D + j4 * 16;
            uint32_t w[D / 8];
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                const uint4 v = rvalid[mt][h] ? *reinterpret_cast<const uint4*>(qrow[mt][h] + (x >> 1) * 64 + (x & 1) * 8) : make_uint4(0, 0, 0, 0);
                w[x * 4] = v.x; w[x * 4 + 1] = v.y; w[x * 4 + 2] = v.z; w[x * 4 + 3] = v.w;
            }
            uint32_t top = 0;
#pragma unroll
            for (int x = 0; x < D / 8; ++x) top = max(top, max((w[x] & 0x7FFFu), (w[x] >> 16) & 0x7FFFu));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const int ex = lift_exp(top);
            const float lift = two(kLiftBits - ex);
            row_mult[mt][h] = p.scale_log2 * two(ex - kLiftBits);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t v = w[ks * 2 + e];
                    qf[mt][ks][h + 2 * e] = pack_f16(__uint_as_float(v << 16) * lift, __uint_as_float(v & 0xFFFF0000u) * lift);
                }
        }

    float o[MT][DT][4];
    float m_run[MT][2], l_run[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[mt][dt][0] = o[mt][dt][1] = o[mt][dt][2] = o[mt][dt][3] = 0.f;
        m_run[mt][0] = m_run[mt][1] = -CUDART_INF_F;
        l_run[mt][0] = l_run[mt][1] = 0.f;
    }
    int e_ref = -126;                                                                    // accumulators: units of 2^(e_ref - kLiftBits)

    // Scores (log2 units, hidden ones -inf) -> weights in place; the accumulators follow a raised maximum or unit.
    auto softmax = [&](float (&s)[MT][2][4], float unit_back) {
        bool raised = unit_back != 1.f;
        float alpha[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float mx = fmaxf(fmaxf(s[mt][0][2 * h], s[mt][0][2 * h + 1]), fmaxf(s[mt][1][2 * h], s[mt][1][2 * h + 1]));
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
                const float m_new = fmaxf(m_run[mt][h], mx);
                const float m_use = m_new == -CUDART_INF_F ? 0.f : m_new;                // nothing visible yet
                alpha[mt][h] = fast_exp2(m_run[mt][h] - m_use);
                raised |= m_new != m_run[mt][h];
                m_run[mt][h] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    s[mt][nt][2 * h] = fast_exp2(s[mt][nt][2 * h] - m_use);
                    s[mt][nt][2 * h + 1] = fast_exp2(s[mt][nt][2 * h + 1] - m_use);
                    sum += s[mt][nt][2 * h] + s[mt][nt][2 * h + 1];
                }
                l_run[mt][h] = l_run[mt][h] * alpha[mt][h] + sum;
            }
        if (__any_sync(0xFFFFFFFFu, raised)) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const float a0 = alpha[mt][0] * unit_back, a1 = alpha[mt][1] * unit_back;
                    o[mt][dt][0] *= a0; o[mt][dt][1] *= a0;
                    o[mt][dt][2] *= a1; o[mt][dt][3] *= a1;
                }
        }
    };

    for (int i = 0; i < n_prefix; ++i) {
        if (i + ST - 1 < n_prefix) issue(i + ST - 1);
        cp_async_commit();
        if ((i & 31) == 0) {
            exps = exps_next;
            exps_next = load_exps(i + 32);
        }
        const int ex = __shfl_sync(0xFFFFFFFFu, exps, i & 31);
        const int ek = max((int)(int8_t)(ex & 255), -126), ev = max(ex >> 8, -126);
        cp_async_wait<ST - 1>();
        __syncwarp();
        const uint32_t sk = ring + (i % ST) * (2 * T::TILE), sv = sk + T::TILE;

        float s[MT][2][4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) s[mt][nt][0] = s[mt][nt][1] = s[mt][nt][2] = s[mt][nt][3] = 0.f;
#pragma unroll
            for (int x = 0; x < D / 64; ++x) {
                const uint4 kw = lds128(sk + k_off(nt * 8 + i8, x * 4 + j4));
                const uint32_t w[4] = {kw.x, kw.y, kw.z, kw.w};
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    uint32_t b0, b1;
                    widen<INT8>(w[y], b0, b1);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) mma_f16(s[mt][nt], qf[mt][x * 4 + y], b0, b1);
                }
            }
        }
        const int key0 = (first + i * kWarps) * kKeys;
        const float sk2 = two(ek);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[mt][nt][e] *= row_mult[mt][e >> 1] * sk2;
        if (key0 + kKeys > L) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (key0 + nt * 8 + j4 * 2 + (e & 1) >= L) s[mt][nt][e] = -CUDART_INF_F;
        }
        float back = 1.f;
        if (ev > e_ref) {
            back = two(max(e_ref - ev, -126));                                           // (below 2^-126 of the unit: nothing is left)
            e_ref = ev;
        }
        softmax(s, back);
        const float lift = two(max(kLiftBits + ev - e_ref, -126));
        uint32_t pf[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                pf[mt][x] = pack_f16(s[mt][x >> 1][(x & 1) * 2] * lift, s[mt][x >> 1][(x & 1) * 2 + 1] * lift);
        // V: the lane's keys are 2 j4, 2 j4 + 1, and these + 8; its column in n-tile dt is i8 * (D / 8) + dt
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
#pragma unroll
        for (int y = 0; y < D / 32; ++y)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                uint32_t a0, a1, c0, c1;
                widen<INT8>(__byte_perm(vw[0][y], vw[1][y], z ? 0x7362 : 0x5140), a0, a1);
                widen<INT8>(__byte_perm(vw[2][y], vw[3][y], z ? 0x7362 : 0x5140), c0, c1);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    mma_f16(o[mt][y * 4 + z * 2], pf[mt], a0, c0);
                    mma_f16(o[mt][y * 4 + z * 2 + 1], pf[mt], a1, c1);
                }
            }
        __syncwarp();                       // the stage has been read: a copy may take its place
    }
    cp_async_wait<0>();

    // ---- draft tiles: bf16 rows straight from global memory, by bf16 products
    if (n_prefix * kWarps + first < t_end) {
        // (the unit of the accumulators: weights 2^(14 - e_ref) must fit bf16)
        float back = 1.f;
        if (e_ref < -100) {
            back = two(max(e_ref + 100, -126));
            e_ref = -100;
        }
        const float lift = two(kLiftBits - e_ref);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[mt][dt][e] *= back;
        const __nv_bfloat16* dk = p.draft_k + ((size_t)b * N * p.Hkv + c) * D;
        const __nv_bfloat16* dv = p.draft_v + ((size_t)b * N * p.Hkv + c) * D;
#pragma unroll 1
        for (int t = first + n_prefix * kWarps; t < t_end; t += kWarps) {
            const int key0 = (t - nPT) * kKeys;
            uint32_t bits[MT][2], any = 0;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = row0 + mt * 16 + h * 8 + i8;
                    uint32_t w = 0;
                    if (rvalid[mt][h]) w = p.mask[((size_t)b * N + row / G) * p.W + (key0 >> 5)] >> (key0 & 16);
                    if (N - key0 < kKeys) w &= (1u << (N - key0)) - 1u;
                    any |= bits[mt][h] = w & 0xFFFFu;
                }
            const uint32_t seen = __reduce_or_sync(0xFFFFFFFFu, any);     // keys that any row sees: others are not read
            if (!seen) continue;
            float s[MT][2][4];
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                const int key = key0 + nt * 8 + i8;
                const bool ok = (seen >> (nt * 8 + i8)) & 1u;
                const __nv_bfloat16* src = dk + (size_t)(ok ? key : 0) * row_bytes + j4 * 16;
                uint32_t kw[D / 8];
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    const uint4 v = ok ? *reinterpret_cast<const uint4*>(src + (x >> 1) * 64 + (x & 1) * 8) : make_uint4(0, 0, 0, 0);
                    kw[x * 4] = v.x; kw[x * 4 + 1] = v.y; kw[x * 4 + 2] = v.z; kw[x * 4 + 3] = v.w;
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    s[mt][nt][0] = s[mt][nt][1] = s[mt][nt][2] = s[mt][nt][3] = 0.f;
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) {           // two k-steps: eight elements of either row
                        uint4 v[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            v[h] = rvalid[mt][h] ? *reinterpret_cast<const uint4*>(qrow[mt][h] + (x >> 1) * 64 + (x & 1) * 8) : make_uint4(0, 0, 0, 0);
                        const uint32_t a0[4] = {v[0].x, v[1].x, v[0].y, v[1].y}, a1[4] = {v[0].z, v[1].z, v[0].w, v[1].w};
                        mma_bf16(s[mt][nt], a0, kw[x * 4], kw[x * 4 + 1]);
                        mma_bf16(s[mt][nt], a1, kw[x * 4 + 2], kw[x * 4 + 3]);
                    }
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[mt][nt][e] = (bits[mt][e >> 1] >> (nt * 8 + j4 * 2 + (e & 1))) & 1u ? s[mt][nt][e] * p.scale_log2 : -CUDART_INF_F;
            softmax(s, 1.f);
            uint32_t pf[MT][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    pf[mt][x] = pack_bf16(s[mt][x >> 1][(x & 1) * 2] * lift, s[mt][x >> 1][(x & 1) * 2 + 1] * lift);
#pragma unroll
            for (int y = 0; y < D / 64; ++y) {                   // eight output n-tiles at a time
                uint32_t w[4][4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int at = 2 * j4 + (x & 1) + (x >> 1) * 8, key = key0 + at;
                    const bool ok = (seen >> at) & 1u;
                    const uint4 v = ok ? *reinterpret_cast<const uint4*>(dv + (size_t)key * row_bytes + i8 * (D / 8) + y * 8) : make_uint4(0, 0, 0, 0);
                    w[x][0] = v.x; w[x][1] = v.y; w[x][2] = v.z; w[x][3] = v.w;
                }
#pragma unroll
                for (int z = 0; z < 4; ++z)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t b0 = __byte_perm(w[0][z], w[1][z], e ? 0x7632 : 0x5410), b1 = __byte_perm(w[2][z], w[3][z], e ? 0x7632 : 0x5410);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) mma_bf16(o[mt][y * 8 + z * 2 + e], pf[mt], b0, b1);
                    }
            }
        }
    }

    // ---- the warps' results meet in the memory of the rings, each warp brings a share of the columns together
    const float in_units = two(e_ref) * two(-kLiftBits);           // (below 2^-126: one product, exact)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l_run[mt][h] += __shfl_xor_sync(0xFFFFFFFFu, l_run[mt][h], 1);
            l_run[mt][h] += __shfl_xor_sync(0xFFFFFFFFu, l_run[mt][h], 2);
        }
    float* const part = reinterpret_cast<float*>(smem) + lane;
    auto part_of = [&](int w, int mt) { return part + (w * MT + mt) * (T::VALUES / MT * 32); };
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        float* at = part_of(warp, mt);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) at[(dt * 4 + e) * 32] = o[mt][dt][e] * in_units;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            at[(DT * 4 + h) * 32] = m_run[mt][h];
            at[(DT * 4 + 2 + h) * 32] = l_run[mt][h];
        }
    }
    __syncthreads();
    constexpr int SHARE = DT / kWarps;                           // n-tiles of a warp: columns i * DT + warp * SHARE + 0..SHARE - 1
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        float w[kWarps][2], m[2], l[2], r[SHARE][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            m[h] = -CUDART_INF_F;
            l[h] = 0.f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                w[k][h] = part_of(k, mt)[(DT * 4 + h) * 32];
                m[h] = fmaxf(m[h], w[k][h]);
            }
            const float m_use = m[h] == -CUDART_INF_F ? 0.f : m[h];
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                w[k][h] = fast_exp2(w[k][h] - m_use);
                l[h] += w[k][h] * part_of(k, mt)[(DT * 4 + 2 + h) * 32];
            }
        }
#pragma unroll
        for (int dt = 0; dt < SHARE; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                r[dt][e] = 0.f;
#pragma unroll
                for (int k = 0; k < kWarps; ++k) r[dt][e] += w[k][e >> 1] * part_of(k, mt)[((warp * SHARE + dt) * 4 + e) * 32];
            }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (!rvalid[mt][h]) continue;
            const int rloc = mt * 16 + h * 8 + i8, row = row0 + rloc;
            if (nsplit == 1) {
                if (!GSD_IN_BOUNDS(b < p.B && c < p.Hkv && row < p.R, p.status)) continue;
                const float inv = l[h] > 0.f ? 1.f / l[h] : 0.f;
                __nv_bfloat16* dst = p.out + (((size_t)b * N + row / G) * p.Hq + c * G + row % G) * D;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int col = (j4 * 2 + e) * DT + warp * SHARE;
                    if constexpr (SHARE == 2) *reinterpret_cast<uint32_t*>(dst + col) = pack_bf16(r[0][h * 2 + e] * inv, r[1][h * 2 + e] * inv);
                    else dst[col] = __float2bfloat16_rn(r[0][h * 2 + e] * inv);
                }
            } else {
                if (!GSD_IN_BOUNDS(slot >= 0 && slot < p.slots, p.status)) continue;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int col = (j4 * 2 + e) * DT + warp * SHARE;
                    float* dst = p.part_o + (((size_t)slot * (D / 4) + col / 4) * 64 + rloc) * 4 + col % 4;
                    if constexpr (SHARE == 2) *reinterpret_cast<float2*>(dst) = make_float2(r[0][h * 2 + e], r[1][h * 2 + e]);
                    else *dst = r[0][h * 2 + e];
                }
                if (warp == 0 && j4 == 0) *reinterpret_cast<float2*>(p.part_ml + ((size_t)slot * 64 + rloc) * 2) = make_float2(m[h], l[h]);
            }
        }
    }
}

template <int D, int MT, bool INT8>
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
    constexpr int smem = Q8Geo<D, MT>::SMEM;
    {
        static bool done[64] = {};   // per template instance: the opt-in sticks per device
        int dev = 0;
        GSD_CUDA_TRY(cudaGetDevice(&dev));
        if (dev < 0 || dev >= 64 || !done[dev]) {
            GSD_CUDA_TRY(cudaFuncSetAttribute(attn_q8_mma_kernel<D, MT, INT8>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
            if (dev >= 0 && dev < 64) done[dev] = true;
        }
    }
    GSD_CUDA_TRY(launch_dependent(attn_q8_mma_kernel<D, MT, INT8>, dim3(a.plan.ctas), dim3(kThreads), smem, a.stream, p));
    return GSD_OK;
}
template <int D, int MT>
int launch_fmt(const AttnArgs& a) { return a.kv8.int8 ? launch_t<D, MT, true>(a) : launch_t<D, MT, false>(a); }

}  // namespace

int attn_q8_mma_rows(int R) { return R <= 16 ? 16 : 32; }
int attn_q8_mma_resident(int R) { return R <= 16 ? 2 : 1; }

int launch_attn_q8_mma(const AttnArgs& a) {
    const bool one = a.plan.rows_per_item == 16;
    if (a.D == 128) return one ? launch_fmt<128, 1>(a) : launch_fmt<128, 2>(a);
    if (a.D == 64) return one ? launch_fmt<64, 1>(a) : launch_fmt<64, 2>(a);
    return GSD_ERR_BAD_SHAPE;
}

}  // namespace gsd
