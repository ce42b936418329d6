// gsd_verify_attn_paged, warp-level back end for few stacked rows (single tokens, small draft graphs): attention over a bf16
// cache held in pages.
//
//   s_j = scale <q, K_j>,   p_j = 2^(s_j log2(e) - m),   out = sum_j p_j V_j / sum_j p_j
//
// A tile is 16 keys: a page holds whole tiles, so each lies in one place and takes one TMA copy each of K and V.  Every warp has
// tiles of its own, a ring of them in shared memory, and nothing to wait for but its own copies; the warps meet once, at the
// end.  Lane l of a warp looks up the page of the l-th of its next 32 tiles.  The tile that holds the end of the sequence is
// copied as the 16 rows up to the end (rows before the page's first come back as zeros), so that nothing behind the end is read.
// Both products are transposed, S^T = K Q^T and O^T = V^T P^T, so that 8 rows fill an instruction (16 keys or 16 columns by 8
// rows); the weights are turned round by a movmatrix.  A row's running maximum is raised when a score exceeds it by more than
// 2^kLag: the weights are rounded to bf16, the type that the product with V takes, whose relative step does not depend on their size,
// and sums stay fp32.
//
// The work is dealt out by length inside the kernel for up to 32 sequences: every item (a group of rows of a sequence and
// kv head) is cut into ranges of at most T rounds of keys, T the least with which all ranges are resident at once; a merge pass brings
// them together.  Where items of eight rows are cut evenly and not too long, a cluster has the ranges of an item and needs no such pass.
//
// Bound by DRAM where keys are many, by dependent trips and the length of a warp's round where they are few.  32 x 64/8 heads of 128,
// N 1, L 4096: 83 us for 537 MB, the rate of a copy; 8 of them, L 500-4000, 17.9 us for 74 MB in clusters of two (by length, with the
// merge launch, 20.1; padded cache 24.0).  4 x 32/8 heads of 64, N 12, L 1000-4000 16.1 us (16.3); 32 x 32/8 of 64, N 1, L 4096 46 us for
// 268 MB.  Four warps and two CTAs an SM, or two and four, took 92 and 97 us for the first; copies by cp.async 84 us; weights in two bf16 terms bring the error from 2.3e-3 to 1.7e-3 for 1-5 % of the time.
#include "gsd_tma.cuh"
#include <cuda_bf16.h>
#include <math_constants.h>

namespace gsd {
namespace {

constexpr int kKeys = 16;                    // keys of a warp's tile
constexpr float kLag = 8.f;                  // log2
constexpr int kTableLines = 16;              // lines of the page table that a CTA asks for ahead of time

struct RowsParams {
    const __nv_bfloat16* q;
    const uint32_t* mask;
    const int32_t* seq_lens;
    __nv_bfloat16* out;
    float* part_o;   // [slot][D / 4][64] float4
    float* part_ml;  // [slot][64][2]
    int* left;       // plan by length: split counts and first units for the merge pass
    int left_off;
    PlanDev plan;
    PageArgs pages;
    int32_t* status;
    int B, N, Hq, Hkv, Lmax, G, W, R;
    int slots;
    int cluster;             // the ranges of an item are brought together by a cluster of as many CTAs; 0: by the merge pass, or whole
    float scale_log2;
    unsigned long long wait_limit_ns;
    int withhold_first_k;    // test hook: every warp leaves out the K copy of its first tile
};

template <int D, int NT>
struct RowsGeo {
    static constexpr int WARPS = 8;
    static constexpr int THREADS = 32 * WARPS;
    static constexpr int ROWS = 8 * NT;                         // stacked rows of an item
    static constexpr int TILE = kKeys * D * 2;                  // bytes of a K or V tile
    static constexpr int BLOCKS = D == 64 && NT <= 3 ? 2 : 1;   // CTAs an SM
    static constexpr int STAGES = D == 128 ? 3 : BLOCKS == 2 ? 3 : 5;
    static constexpr int RING = WARPS * STAGES * 2 * TILE;
    static constexpr int MTILES = D / 16;                       // output tiles of 16 columns
    static constexpr int VALUES = MTILES * 4 + 4;               // of a lane and 8 rows, when the warps' results are brought together
    static constexpr int MEET = WARPS * NT * VALUES * 32 * 4;
    static constexpr int SHARED = NT == 1 ? ROWS * (D + 4) * 4 : 0;     // what a CTA of a cluster has of its item: [row][D + 4], behind MEET
    static constexpr int Q_AT = RING > MEET + SHARED ? RING : MEET + SHARED;    // query fragments: [row group][k-step][lane] pairs of registers
    static constexpr int SMEM = Q_AT + NT * (D / 16) * 32 * 8 + 1024;       // (alignment)
};

__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
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
// 8x8 bf16 values, a row a quarter of lanes -> their transpose.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}

// Bounded wait, by the whole warp; false: it gave up.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, unsigned long long limit_ns) {
    bool ok = mbar_try_wait(bar, parity);
    if (!__all_sync(0xFFFFFFFFu, ok)) {
        const unsigned long long t0 = global_ns();
        while (!ok && global_ns() - t0 <= limit_ns) ok = mbar_try_wait(bar, parity);
        ok = __all_sync(0xFFFFFFFFu, ok);
    }
    return ok;
}

constexpr int kMostCluster = 8;
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
// From the shared memory of CTA k of the cluster, at this CTA's address `at`.
__device__ __forceinline__ uint32_t of_cta(uint32_t at, int k) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(k));
    return r;
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t at, int k) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(of_cta(at, k)) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t at, int k) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(of_cta(at, k)) : "memory");
    return v;
}

// What a CTA works on: rows of (sequence b, kv head c), keys of one of `nsplit` ranges.
struct Unit {
    int b, c, row0, split, nsplit, slot, L;
};

__device__ __forceinline__ int visible_len(const RowsParams& p, int b) {
    const int L = p.seq_lens[b];
    return L < 0 ? 0 : (L > p.Lmax ? p.Lmax : L);
}

// n / d for n >= 0, d >= 1 and a quotient below 2^16, `inv` = 1 / d to a few ulp: the estimate is off by less than one.  A third of an
// integer division, of which the plan takes a chain.
__device__ __forceinline__ int div_by(int n, int d, float inv) {
    int q = (int)((float)n * inv);
    const int r = n - q * d;
    if (r < 0) --q;
    if (r >= d) ++q;
    return q;
}
__device__ __forceinline__ int div_by(int n, int d) { return div_by(n, d, __fdividef(1.f, (float)d)); }

// Plan by length, made by every warp for itself, a lane per sequence: the cut of each sequence's items into ranges of at most T
// rounds (a tile for each warp); unit w is this CTA's, if there are that many.  `leave`: the merge pass's tables are written.
template <int kRound>
__device__ __forceinline__ bool unit_by_length(const RowsParams& p, int w, int lane, bool leave, Unit& u) {
    const unsigned all = 0xFFFFFFFFu;
    const bool in = lane < p.B;
    const int per_seq = p.Hkv * p.plan.tiles_per_unit, resident = (int)gridDim.x;
    const int L = in ? visible_len(p, lane) : 0;
    const int t = in ? ((L + kKeys - 1) / kKeys + (p.N + kKeys - 1) / kKeys + kRound - 1) / kRound : 0;    // rounds
    const int total = __reduce_add_sync(all, t), longest = __reduce_max_sync(all, t);
    // lane k tries the k-th candidate for T, from the lower bound on (two rounds, 64 parts an item); the longest sequence
    // whole always fits, as there are no more items than CTAs
    const int bound = max(max((int)((float)total * __fdividef((float)per_seq, (float)resident)) + 1, (longest + 63) / 64), 2);
    const int T = bound + lane * max(1, bound / 16);
    const float inv = __fdividef(1.f, (float)T);
    int units = 0;
    for (int j0 = 0; j0 < p.B; j0 += 4)                     // (lanes behind the last sequence have no rounds)
#pragma unroll
        for (int j = 0; j < 4; ++j) units += div_by(__shfl_sync(all, t, j0 + j) + T - 1, T, inv);
    const int best = min(longest, (int)__reduce_min_sync(all, units * per_seq <= resident ? T : 0x7FFFFFFF));
    const int n = in ? div_by(t + best - 1, best) : 0;
    int end = n;                                            // ranges up to and with this sequence, per item
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int before = __shfl_up_sync(all, end, o);
        if (lane >= o) end += before;
    }
    if (leave && in) {
        p.left[lane] = n;
        p.left[p.left_off + lane] = (end - n) * per_seq;
    }
    u.b = min(__popc(__ballot_sync(all, in && end * per_seq <= w)), p.B - 1);
    u.L = __shfl_sync(all, L, u.b);
    u.nsplit = __shfl_sync(all, n, u.b);
    const int r = w - __shfl_sync(all, end - n, u.b) * per_seq;
    u.split = div_by(max(r, 0), per_seq);
    const int item = r - u.split * per_seq;
    u.c = div_by(max(item, 0), p.plan.tiles_per_unit);
    u.row0 = item - u.c * p.plan.tiles_per_unit;
    u.slot = w;
    return w < __shfl_sync(all, end, 31) * per_seq;
}

template <int D, int NT>
__global__ void __launch_bounds__(RowsGeo<D, NT>::THREADS, RowsGeo<D, NT>::BLOCKS) attn_paged_rows_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_dk,
                       const __grid_constant__ CUtensorMap tm_dv, const RowsParams p) {
    using T = RowsGeo<D, NT>;
    constexpr int KS = D / 16;              // k-steps of the product with K
    constexpr int MTL = T::MTILES, WARPS = T::WARPS, ST = T::STAGES;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long s_full[WARPS * ST];
    unsigned char* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);

    // (Where an SM holds two CTAs, the next call's would take places beside this one's: 11.3 -> 19.3 us for 4 x 32/8 heads of 64, N 8, L
    // 1000-2000.  With one they do not fit, and a chain of short calls is a seventh faster: 1 x 32/8 of 128, L 60-120 4.5 -> 3.8.)
    if (p.slots > 0 || T::BLOCKS == 1) let_successor_start();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int i8 = lane >> 2, j4 = lane & 3;
    const int N = p.N, G = p.G, R = p.R;
    const uint32_t full = smem_u32(s_full) + warp * (ST * 8);      // the warp's barriers, one a stage
    if (lane == 0) {
        for (int s = 0; s < ST; ++s) mbar_init(full + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (warp == 0) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_k) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_v) : "memory");
        }
    }
    __syncwarp();
    Unit u;
    const bool by_length = p.plan.balanced == 3;
    if (!by_length) {
        // (no need to wait for what precedes the call)
        int item;
        plan_decode(p.plan, blockIdx.x, item, u.split, u.nsplit, u.slot);
        const int pair = item / p.plan.tiles_per_unit;   // b * Hkv + c
        u.row0 = item - pair * p.plan.tiles_per_unit;
        u.b = pair / p.Hkv;
        u.c = pair - u.b * p.Hkv;
    }
    wait_for_predecessor();
    if (tid < kTableLines) {
        // the table's first lines, a few a CTA, while the lengths come: its look-ups are the next trip
        const int lines = (p.Lmax >> p.pages.page_log2) / 32 + 1, i = blockIdx.x * kTableLines + tid;      // of a row, 128 bytes each
        const int row = i / lines, at = (i - row * lines) * 32;
        if (row < p.B && at < p.pages.max_pages)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p.pages.table + (size_t)row * p.pages.max_pages + at) : "memory");
    }
    if (by_length && !unit_by_length<WARPS>(p, blockIdx.x, lane, blockIdx.x == 0 && warp == 0, u)) return;
    u.row0 *= T::ROWS;
    const int b = u.b, c = u.c, row0 = u.row0;
    // Key tiles of 16: the prefix, then the draft block.  By length the CTA has a run of them, a warp every WARPS-th of the run; else
    // the warps of all ranges take them in turns, so that which tiles a warp begins with does not hang on the length.
    const int step = by_length ? WARPS : WARPS * u.nsplit;
    const int32_t* table = p.pages.table + (size_t)b * p.pages.max_pages;
    const int given = by_length ? 0 : p.seq_lens[b];
    // What the table has for the warp's tiles `lane`, and the query rows (a warp for every eight), are asked for beside the length, a
    // trip to memory less.  Queries before keys: behind 128 KB of them an SM they took 2.5 us.
    const int entry = by_length ? 0 : table[min((u.split * WARPS + warp + lane * step) * kKeys >> p.pages.page_log2, p.pages.max_pages - 1)];
    static_assert(NT <= WARPS, "a row group a warp");
    uint32_t qw[KS][2];
    if (warp < NT) {
        const int row = row0 + warp * 8 + i8;
        const bool in = row < R;
        const int rr = in ? row : 0;
        const __nv_bfloat16* q = p.q + (((size_t)b * N + rr / G) * p.Hq + c * G + rr % G) * D + 2 * j4;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qw[ks][0] = in ? *reinterpret_cast<const uint32_t*>(q + ks * 16) : 0u;
            qw[ks][1] = in ? *reinterpret_cast<const uint32_t*>(q + ks * 16 + 8) : 0u;
        }
    }
    const int L = by_length ? u.L : min(max(given, 0), p.Lmax);
    if (tid == 0 && p.status) {
        const int len = by_length ? p.seq_lens[b] : given;
        if (len < 0 || len > p.Lmax) atomicOr((unsigned*)p.status, GSD_DEV_BAD_SEQ_LEN);
    }
    const int nPT = (L + kKeys - 1) / kKeys, nT = nPT + (N + kKeys - 1) / kKeys;
    const int per = by_length ? ((nT + WARPS - 1) / WARPS + u.nsplit - 1) / u.nsplit * WARPS : WARPS;
    const int first = u.split * per + warp, t_end = by_length ? min(u.split * per + per, nT) : nT;
    const int all_tiles = max(0, t_end - first + step - 1), n_tiles = step == WARPS ? all_tiles / WARPS : all_tiles / step;    // (a shift)

    // ---- the ring: K and V tiles of 16 rows, blocks of 64 columns
    const uint32_t ring = smem_u32(smem) + warp * (ST * 2 * T::TILE);
    // the pages of the warp's tiles i0 + lane; -1: none (draft tiles, no such tile, no such page)
    auto find_pages = [&](int i0) -> int {
        const int key = (first + (i0 + lane) * step) * kKeys;
        if (i0 + lane >= n_tiles || key >= L || !GSD_IN_BOUNDS(key >> p.pages.page_log2 < p.pages.max_pages, p.status)) return -1;
        const int page = i0 == 0 && !by_length ? entry : table[key >> p.pages.page_log2];
        if ((unsigned)page < (unsigned)p.pages.num_pages) return page;
        if (p.status) atomicOr((unsigned*)p.status, GSD_DEV_BAD_PAGE);
        return -1;
    };
    auto issue = [&](int i, int stage, int pages) {
        const int t = first + i * step;
        const int page = __shfl_sync(0xFFFFFFFFu, pages, i & 31);
        if (lane == 0) {
            const uint32_t dst = ring + stage * (2 * T::TILE), bar = full + 8 * stage;
            mbar_expect_tx(bar, 2 * T::TILE);
            if (t >= nPT) {
                if (!(p.withhold_first_k && i == 0)) tma_load_4d(dst, &tm_dk, bar, 0, (t - nPT) * kKeys, c * (D / 64), b);
                tma_load_4d(dst + T::TILE, &tm_dv, bar, 0, (t - nPT) * kKeys, c * (D / 64), b);
            } else {
                const int key0 = t * kKeys;
                // (no such page: from behind the pool, zeros)
                const int row = (key0 & ((1 << p.pages.page_log2) - 1)) + min(0, L - key0 - kKeys), at = page < 0 ? p.pages.num_pages : page;
                if (!(p.withhold_first_k && i == 0)) tma_load_4d(dst, &tm_k, bar, 0, row, c * (D / 64), at);
                tma_load_4d(dst + T::TILE, &tm_v, bar, 0, row, c * (D / 64), at);
            }
        }
        __syncwarp();
    };
    int pages = find_pages(0);
    for (int s = 0; s < min(ST, n_tiles); ++s) issue(s, s, pages);
    int pages_next = find_pages(32);

    // the mask words of the draft tiles, which come last, as a trip of their own
    for (int t = first + (n_tiles - 1) * step; t >= max(first, nPT); t -= step)
        for (int node = row0 / G + lane; node <= min(row0 + T::ROWS - 1, R - 1) / G; node += 32)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p.mask + ((size_t)b * N + node) * p.W + ((t - nPT) * kKeys >> 5)) : "memory");
    // ---- the query rows as fragments (rows are columns of the products), where all warps find them
    const uint32_t q_at = smem_u32(smem) + T::Q_AT + lane * 8;
    if (warp < NT) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(q_at + (warp * KS + ks) * 256), "r"(qw[ks][0]), "r"(qw[ks][1]) : "memory");
    }
    __syncthreads();
    uint2 qf[NT == 1 ? KS : 1];
    if (NT == 1) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[NT == 1 ? ks : 0] = lds64(q_at + ks * 256);
    }

    float o[NT][MTL][4];                    // columns 16 mt + i8 and the one 8 behind it, of rows 8 nt + 2 j4 + {0, 1}
    float m_run[NT][2], l_run[NT][2];       // l: the lane's own keys
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int mt = 0; mt < MTL; ++mt) o[nt][mt][0] = o[nt][mt][1] = o[nt][mt][2] = o[nt][mt][3] = 0.f;
        m_run[nt][0] = m_run[nt][1] = -CUDART_INF_F;
        l_run[nt][0] = l_run[nt][1] = 0.f;
    }
    // where the lane's rows of the matrices start: K keys (lane & 15), pieces + (lane >> 4); V keys (lane & 7) + 8 (lane >> 4).  A
    // piece of 16 bytes sits at its number exclusive-or'ed with the low bits of its row's (the copies' swizzle).
    const int k_row = lane & 15, v_row = (lane & 7) + ((lane >> 4) << 3);
    const uint32_t k_at = k_row * 128 + (((lane >> 4) ^ (k_row & 7)) << 4), v_at = v_row * 128 + ((((lane >> 3) & 1) ^ (v_row & 7)) << 4);
    auto piece_pair = [](uint32_t at, int x) -> uint32_t { return (at ^ ((x & 3) << 5)) + (x >> 2) * (kKeys * 128); };   // pieces 2 x and 2 x + 1
    int stage = 0;
    uint32_t parity = 0;
    bool ok = true;
    int done = 0;                           // tiles that have landed
#pragma unroll 1
    for (int i = 0; i < n_tiles; ++i) {
        ok = wait_warp(full + 8 * stage, parity, p.wait_limit_ns);
        if (!ok) break;
        ++done;
        const uint32_t sk = ring + stage * (2 * T::TILE), sv = sk + T::TILE;

        // S^T = K Q^T: 16 keys (i8, i8 + 8) x 8 rows; two chains at least
        constexpr int CHAINS = NT == 1 ? 2 : 1;
        float s[NT][4], s1[CHAINS][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[nt][e] = s1[0][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint32_t a[4];
            ldmatrix_x4(a, sk + piece_pair(k_at, ks));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint2 q = NT == 1 ? qf[NT == 1 ? ks : 0] : lds64(q_at + (nt * KS + ks) * 256);
                mma_bf16(NT == 1 && (ks & 1) ? s1[0] : s[nt], a, q.x, q.y);
            }
        }
        if (NT == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[0][e] += s1[0][e];
        }
        // ---- in log2 units, hidden ones -inf
        const int t = first + i * step;
        bool raise = false;
        if (t >= nPT) {
            const int key0 = (t - nPT) * kKeys;
            uint32_t seen = 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = row0 + nt * 8 + 2 * j4 + e;
                    uint32_t w = row < R ? p.mask[((size_t)b * N + row / G) * p.W + (key0 >> 5)] >> (key0 & 16) : 0u;
                    if (N - key0 < kKeys) w &= (1u << (N - key0)) - 1u;
                    seen |= w;
                    s[nt][e] = (w >> i8) & 1u ? s[nt][e] * p.scale_log2 : -CUDART_INF_F;
                    s[nt][e + 2] = (w >> (i8 + 8)) & 1u ? s[nt][e + 2] * p.scale_log2 : -CUDART_INF_F;
                }
            // zeros in the rows of V that no row here sees: their weight is 0, and 0 times an infinity is not
            uint32_t hide = ~__reduce_or_sync(0xFFFFFFFFu, seen) & (N - key0 < kKeys ? (1u << (N - key0)) - 1u : 0xFFFFu);
            if (hide != 0) {
                for (; hide != 0; hide &= hide - 1)
                    if (lane < D / 8)
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(sv + (lane >> 3) * (kKeys * 128) + (__ffs((int)hide) - 1) * 128 + (lane & 7) * 16), "r"(0) : "memory");
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // (before a copy takes the stage again)
                __syncwarp();
            }
        } else {
            const int before = t * kKeys + kKeys - L;       // keys of the last tile that the tile before it has covered, or zeros
            const bool lo = i8 >= before, hi = i8 + 8 >= before;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    s[nt][e] = lo ? s[nt][e] * p.scale_log2 : -CUDART_INF_F;
                    s[nt][e + 2] = hi ? s[nt][e + 2] * p.scale_log2 : -CUDART_INF_F;
                }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) raise |= fmaxf(s[nt][e], s[nt][e + 2]) > m_run[nt][e] + kLag;
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
                }
#pragma unroll
                for (int mt = 0; mt < MTL; ++mt) {
                    o[nt][mt][0] *= a[0]; o[nt][mt][2] *= a[0];
                    o[nt][mt][1] *= a[1]; o[nt][mt][3] *= a[1];
                }
            }
        }
        uint32_t pf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float m_use = m_run[nt][e] == -CUDART_INF_F ? 0.f : m_run[nt][e];
                s[nt][e] = fast_exp2(s[nt][e] - m_use);
                s[nt][e + 2] = fast_exp2(s[nt][e + 2] - m_use);
                l_run[nt][e] += s[nt][e] + s[nt][e + 2];
            }
            pf[nt][0] = transpose8(pack_bf16(s[nt][0], s[nt][1]));
            pf[nt][1] = transpose8(pack_bf16(s[nt][2], s[nt][3]));
        }
        // O^T += V^T P^T
#pragma unroll
        for (int mt = 0; mt < MTL; ++mt) {
            uint32_t a[4];
            ldmatrix_x4_trans(a, sv + piece_pair(v_at, mt));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_bf16(o[nt][mt], a, pf[nt][0], pf[nt][1]);
        }
        __syncwarp();                       // the stage has been read: a copy may take its place
        const int ahead = i + ST;
        if ((ahead & 31) == 0) {
            pages = pages_next;
            pages_next = find_pages(ahead + 32);
        }
        if (ahead < n_tiles) issue(ahead, stage, pages);
        if (++stage == ST) {
            stage = 0;
            parity ^= 1;
        }
    }
    if (!ok) {
        // gave up: the copies under way have to land before the memory is used again
        if (lane == 0 && p.status) atomicOr((unsigned*)p.status, GSD_DEV_WAIT_EXPIRED);
        for (int i = done; i < min(done + ST, n_tiles); ++i) wait_warp(full + 8 * (i % ST), (uint32_t)(i / ST) & 1u, p.wait_limit_ns);
    }

    // ---- the warps' results meet in the memory of the rings
    float* const shared = reinterpret_cast<float*>(smem + T::MEET);     // for the cluster: a row's sums, then m and l
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) l_run[nt][e] += __shfl_xor_sync(0xFFFFFFFFu, l_run[nt][e], x);
    float* const part = reinterpret_cast<float*>(smem);
    auto part_of = [&](int w, int nt) { return part + (w * NT + nt) * (T::VALUES * 32); };
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float* at = part_of(warp, nt);
        // (swizzled so that neither these stores nor the loads below conflict)
#pragma unroll
        for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e) at[(mt * 4 + e) * 32 + (lane ^ (e << 2))] = o[nt][mt][e];
        if (i8 == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                at[MTL * 128 + 2 * j4 + e] = m_run[nt][e];
                at[MTL * 128 + 8 + 2 * j4 + e] = l_run[nt][e];
            }
        }
    }
    __syncthreads();
    // a thread takes four columns of a row
#pragma unroll 2
    for (int x = tid; x < NT * 8 * (D / 4); x += T::THREADS) {
        const int r8 = x & 7, quad = (x >> 3) % (D / 4), nt = (x >> 3) / (D / 4);
        const int row = row0 + nt * 8 + r8;
        if (row >= R) continue;
        float w[WARPS], m = -CUDART_INF_F, l = 0.f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
            w[k] = part_of(k, nt)[MTL * 128 + r8];
            m = fmaxf(m, w[k]);
        }
        const float m_use = m == -CUDART_INF_F ? 0.f : m;
        float r[4] = {0.f, 0.f, 0.f, 0.f};
        const int col = quad * 4, e = ((col >> 3) & 1) * 2 + (r8 & 1), at = ((col >> 4) * 4 + e) * 32;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
            const float wk = fast_exp2(w[k] - m_use);
            l += wk * part_of(k, nt)[MTL * 128 + 8 + r8];
#pragma unroll
            for (int y = 0; y < 4; ++y) r[y] += wk * part_of(k, nt)[at + ((((col & 7) + y) * 4 + (r8 >> 1)) ^ (e << 2))];
        }
        if (u.nsplit == 1) {
            if (!GSD_IN_BOUNDS(b < p.B && c < p.Hkv && row < p.R, p.status)) continue;
            const float inv = l > 0.f ? 1.f / l : 0.f;
            *reinterpret_cast<uint2*>(p.out + (((size_t)b * N + row / G) * p.Hq + c * G + row % G) * D + col) =
                make_uint2(pack_bf16(r[0] * inv, r[1] * inv), pack_bf16(r[2] * inv, r[3] * inv));
        } else if (NT == 1 && p.cluster) {
            float* at = shared + (nt * 8 + r8) * (D + 4);
            *reinterpret_cast<float4*>(at + col) = make_float4(r[0], r[1], r[2], r[3]);
            if (quad == 0) *reinterpret_cast<float2*>(at + D) = make_float2(m, l);
        } else {
            if (!GSD_IN_BOUNDS(u.slot >= 0 && u.slot < p.slots, p.status)) continue;
            *reinterpret_cast<float4*>(p.part_o + (((size_t)u.slot * (D / 4) + quad) * 64 + nt * 8 + r8) * 4) = make_float4(r[0], r[1], r[2], r[3]);
            if (quad == 0) *reinterpret_cast<float2*>(p.part_ml + ((size_t)u.slot * 64 + nt * 8 + r8) * 2) = make_float2(m, l);
        }
    }
    if (NT != 1 || p.cluster == 0) return;
    // ---- the ranges meet: each CTA of the cluster takes a share of the rows' columns
    cluster_meet();
    const uint32_t mine = smem_u32(shared);
    for (int x = u.split * T::THREADS + tid; x < T::ROWS * (D / 4); x += p.cluster * T::THREADS) {
        const int r = x / (D / 4), col = x % (D / 4) * 4, row = row0 + r;
        if (row >= R || !GSD_IN_BOUNDS(b < p.B && c < p.Hkv, p.status)) continue;
        float m = -CUDART_INF_F, l = 0.f;
        float4 o4 = make_float4(0.f, 0.f, 0.f, 0.f);
        float2 ml[kMostCluster];
#pragma unroll
        for (int k = 0; k < kMostCluster; ++k) {
            ml[k] = k < p.cluster ? ld_cluster2(mine + (r * (D + 4) + D) * 4, k) : make_float2(-CUDART_INF_F, 0.f);
            m = fmaxf(m, ml[k].x);
        }
        const float m_use = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll
        for (int k = 0; k < kMostCluster; ++k) {
            if (k >= p.cluster) break;
            const float wk = fast_exp2(ml[k].x - m_use);
            const float4 v = ld_cluster4(mine + (r * (D + 4) + col) * 4, k);
            l += wk * ml[k].y;
            o4.x += wk * v.x; o4.y += wk * v.y; o4.z += wk * v.z; o4.w += wk * v.w;
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        *reinterpret_cast<uint2*>(p.out + (((size_t)b * N + row / G) * p.Hq + c * G + row % G) * D + col) =
            make_uint2(pack_bf16(o4.x * inv, o4.y * inv), pack_bf16(o4.z * inv, o4.w * inv));
    }
    cluster_meet();                         // (no CTA ends while another reads its memory)
}

template <int D, int NT>
int launch_t(const AttnArgs& a) {
    RowsParams p;
    p.q = (const __nv_bfloat16*)a.q;
    p.pages = a.pages;
    CUtensorMap tk, tv, tdk, tdv;
    int rc;
    if ((rc = make_rows_map(&tk, a.k_cache, D, a.Hkv, 1 << a.pages.page_log2, a.pages.num_pages, kKeys)) != GSD_OK) return rc;
    if ((rc = make_rows_map(&tv, a.v_cache, D, a.Hkv, 1 << a.pages.page_log2, a.pages.num_pages, kKeys)) != GSD_OK) return rc;
    if ((rc = make_rows_map(&tdk, a.draft_k, D, a.Hkv, a.N, a.B, kKeys)) != GSD_OK) return rc;
    if ((rc = make_rows_map(&tdv, a.draft_v, D, a.Hkv, a.N, a.B, kKeys)) != GSD_OK) return rc;
    p.wait_limit_ns = g_wait_limit_ns;
    p.withhold_first_k = g_withhold_first_k;
    p.mask = a.mask; p.seq_lens = a.seq_lens; p.out = (__nv_bfloat16*)a.out; p.status = a.status;
    p.B = a.B; p.N = a.N; p.Hq = a.Hq; p.Hkv = a.Hkv; p.Lmax = a.Lmax; p.G = a.G; p.W = a.W; p.R = a.N * a.G;
    p.scale_log2 = a.scale_log2; p.plan = a.plan.dev; p.slots = a.plan.slots; p.cluster = a.plan.cluster;
    p.part_o = (float*)a.workspace;
    p.part_ml = (float*)((char*)a.workspace + plan_part_o_bytes(a.plan, a.D));
    p.left = a.plan.dev.balanced == 3 ? plan_left_table(a.plan, a.D, a.workspace) : nullptr;
    p.left_off = (int)(align_up((size_t)a.B * sizeof(int), 256) / sizeof(int));
    constexpr int smem = RowsGeo<D, NT>::SMEM;
    {
        static bool done[64] = {};   // per template instance: the opt-in sticks per device
        int dev = 0;
        GSD_CUDA_TRY(cudaGetDevice(&dev));
        if (dev < 0 || dev >= 64 || !done[dev]) {
            GSD_CUDA_TRY(cudaFuncSetAttribute(attn_paged_rows_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
            if (dev >= 0 && dev < 64) done[dev] = true;
        }
    }
    cudaLaunchAttribute attr[2];
    dependent_launch_attr(attr);
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.plan.cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.plan.ctas);
    cfg.blockDim = dim3(RowsGeo<D, NT>::THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = a.stream;
    cfg.attrs = attr;
    cfg.numAttrs = a.plan.cluster > 0 ? 2 : 1;
    GSD_CUDA_TRY(cudaLaunchKernelEx(&cfg, attn_paged_rows_kernel<D, NT>, tk, tv, tdk, tdv, p));
    return GSD_OK;
}

}  // namespace

// Stacked rows of an item.  More rows an item read the cache fewer times (the rest comes from L2); fewer rows spread the same
// work over more SMs, and a warp's round is shorter.  So an item gets the fewest rows with which all items, each cut into as many
// ranges as the length asks for (one for 20 rounds of keys), still run side by side: up to 32 rows with a CTA an SM; for D = 64,
// where two fit, up to 24 rows with two; past that the most rows.  us at 8, 16, 24 and 32 rows, D 128: 4 x 32/8 heads, N 8, L
// 250-500 6.7, 8.3, 8.2, 11.0, L 4000-8000 36, 27, 27, 27; 1 x 32/8, N 12, L 500-1000 7.8, 8.6, 9.3, 9.4; 16 x 32/8, N 16, L 500-1000
// 55, 39, 35, 29.  D 64: 4 x 96/24, N 16, L 250-500 20, 15, 11, 17; 48 x 32/8, N 16, L 100-200 55, 35, 31, 41.
int attn_paged_rows(int R, int D, int pairs, int ranges, int sm_count) {
    const int groups = (R + 7) / 8;
    for (int ctas = 1; ctas <= (D == 64 ? 2 : 1); ++ctas)
        for (int per = 1; per <= (ctas == 1 ? 4 : 3); ++per) {
            const int items = (groups + per - 1) / per;
            if ((long long)pairs * items * ranges <= (long long)sm_count * ctas) return 8 * ((groups + items - 1) / items);
        }
    const int most = D == 64 ? 3 : 4, items = (groups + most - 1) / most;
    return 8 * ((groups + items - 1) / items);
}
int attn_paged_rows_resident(int rows, int D) { return D == 64 && rows <= 24 ? 2 : 1; }

int launch_attn_paged_rows(const AttnArgs& a) {
    switch (a.plan.rows_per_item * 1000 + a.D) {
        case 8128: return launch_t<128, 1>(a);
        case 16128: return launch_t<128, 2>(a);
        case 24128: return launch_t<128, 3>(a);
        case 32128: return launch_t<128, 4>(a);
        case 8064: return launch_t<64, 1>(a);
        case 16064: return launch_t<64, 2>(a);
        case 24064: return launch_t<64, 3>(a);
        case 32064: return launch_t<64, 4>(a);
    }
    return GSD_ERR_BAD_SHAPE;
}

}  // namespace gsd
