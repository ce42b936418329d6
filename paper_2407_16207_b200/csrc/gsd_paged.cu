// gsd_append_kv_paged and gsd_commit_kv_paged: bf16 K/V rows into a cache held in pages, behind the old end of every sequence
// (the rows of a prompt, K rotated by position on the way; or the accepted path of a verification step).
//
// A CTA has a run of (row, kv head) places of a sequence, a thread a chunk of 16 columns of K and of V of several of them
// (gsd_rotary.cuh).  While its first pieces come, the CTA looks up its rows' pages and forms their sines and cosines in shared
// memory.  Rows from the first on whose page the table does not name are dropped: every CTA looks through the entries up to
// its own last row's.  Bound by DRAM for prompts, by dependent trips to memory for accepted paths and short chunks, which go to one
// cluster of CTAs per sequence, so that it can move the length on itself.
//
// Measured in captured graphs: 8 prompts of 1000-4096 rows, 8 kv heads of 128, 29.1 us for 167 MB, 89 % of the rate of a copy, and 3 us
// for the launch that moves the lengths on; a chunk of 1031 rows of 4 heads 3.8 us; paths of up to 17 rows, 8 x 8 heads, 3.5 us, of up to
// 10 rows, 32 x 40 heads, 5.8 us.  One launch for all appends, whose last CTA moves the length on, would need a counter that is zero.
#include "gsd_pages.cuh"
#include "gsd_rotary.cuh"
#include <initializer_list>

namespace gsd {
namespace {

constexpr int kThreads = kRotaryThreads;

struct WriteArgs {
    uint16_t *k_pages, *v_pages;
    const int32_t* table;
    const uint16_t *k, *v;
    const int32_t* nodes;        // accepted path [B, Tcap], else nullptr
    const int32_t* count;        // its length, or the rows to append
    int32_t* seq_lens;
    int32_t* status;
    Rotation r;
    long long k_stride, v_stride;
    int B, M, Hkv, Lmax, Tcap;   // M: rows per sequence in k / v
    int page_log2, max_pages, num_pages;
    int batches;                 // of a CTA (not of a path's)
};

enum Mode { APPEND, APPEND_CLUSTER, COMMIT };   // the rows of a grid, of one cluster per sequence; a path, one cluster per sequence

// With a cluster CTA 0 moves the length on once all of it have read the old one.
template <int D, int kBatch, int MODE>
__global__ void __launch_bounds__(kThreads, kRotaryBlocks) paged_write_kernel(const __grid_constant__ WriteArgs a) {
    constexpr int CH = D / 16, SLOTS = kThreads / CH, ROWS = MODE == COMMIT ? GSD_MAX_NODES : rotary_tokens(D);
    __shared__ AngleTable<D> s_angles[MODE == COMMIT ? 1 : ROWS];
    __shared__ int s_page[ROWS];                                  // the pages of the CTA's rows
    __shared__ int s_src[MODE == COMMIT ? GSD_MAX_NODES : 1];     // source row of each new place
    __shared__ int s_tot[kThreads / 32];
    __shared__ int s_bad;                                         // first table entry that names no page
    if (MODE != APPEND) let_successor_start();
    const int b = blockIdx.y, tid = threadIdx.x;
    if (tid == 0) s_bad = 0x7FFFFFFF;
    __syncthreads();
    wait_for_predecessor();
    if (MODE == APPEND) let_successor_start();      // (paged_advance_kernel, which reads the call's inputs before it waits)
    unsigned flags = 0;
    int L = a.seq_lens[b];
    if (L < 0 || L > a.Lmax) {
        flags |= GSD_DEV_BAD_SEQ_LEN;
        L = L < 0 ? 0 : a.Lmax;
    }
    int n = a.count[b];
    if (MODE == COMMIT) {
        // the valid nodes of the path, in its order
        const int len = min(min(n, a.Tcap), GSD_MAX_NODES);
        const int lane = tid & 31, warp = tid >> 5;
        n = 0;
        for (int i0 = 0; i0 < len; i0 += kThreads) {
            const int i = i0 + tid;
            const int node = i < len ? a.nodes[(size_t)b * a.Tcap + i] : -1;
            const bool valid = node >= 0 && node < a.M;
            if (i < len && !valid) flags |= GSD_DEV_BAD_CSR;
            const unsigned vote = __ballot_sync(0xFFFFFFFFu, valid);
            if (lane == 0) s_tot[warp] = __popc(vote);
            __syncthreads();
            int at = n + __popc(vote & ((1u << lane) - 1u));
            for (int w = 0; w < kThreads / 32; ++w) {
                if (w < warp) at += s_tot[w];
                n += s_tot[w];
            }
            if (valid) s_src[at] = node;
            __syncthreads();
        }
    } else {
        if (n < 0 || n > a.M) flags |= GSD_DEV_BAD_SEQ_LEN;
        n = min(max(n, 0), a.M);
    }
    if (n > a.Lmax - L) flags |= GSD_DEV_CACHE_FULL;
    n = min(n, a.Lmax - L);

    const int32_t* table = a.table + (size_t)b * a.max_pages;
    const int places = n * a.Hkv;
    const int run = MODE == COMMIT ? ((places + (int)gridDim.x - 1) / (int)gridDim.x + SLOTS - 1) / SLOTS * SLOTS : SLOTS * a.batches;
    const int begin = (int)blockIdx.x * run, end = min(begin + run, places);
    const int row0 = begin / a.Hkv, row1 = (end - 1) / a.Hkv;
    const int j = tid % CH, slot = tid / CH;
    const int2 col = chunk_columns(a.r, j);
    const bool turned = MODE != COMMIT && j < a.r.chunks;
    for (int at0 = begin; at0 < end; at0 += SLOTS * kBatch) {
        uint4 x[kBatch][4];
        int t[kBatch], h[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int at = min(at0 + i * SLOTS + slot, end - 1);        // (the last place again, for those behind it)
            t[i] = at / a.Hkv;
            h[i] = at - t[i] * a.Hkv;
            const size_t tok = (size_t)b * a.M + (MODE == COMMIT ? s_src[t[i]] : t[i]);
            const uint16_t *k = a.k + tok * a.k_stride + h[i] * D, *v = a.v + tok * a.v_stride + h[i] * D;
            x[i][0] = *reinterpret_cast<const uint4*>(k + col.x);
            x[i][1] = *reinterpret_cast<const uint4*>(k + col.y);
            x[i][2] = *reinterpret_cast<const uint4*>(v + col.x);
            x[i][3] = *reinterpret_cast<const uint4*>(v + col.y);
        }
        if (at0 == begin) {
            // (a cluster's CTAs all look as far as the last row: CTA 0 needs to know what was written)
            const int entries = ((L + (MODE == APPEND ? row1 : n - 1)) >> a.page_log2) + 1;
            const int bad = first_bad_page(table, L >> a.page_log2, entries, a.num_pages, tid, kThreads);
            if (bad < entries) atomicMin(&s_bad, bad);
            for (int i = tid; i <= row1 - row0; i += kThreads) s_page[i] = table[(L + row0 + i) >> a.page_log2];
            if (MODE != COMMIT)
                form_angles(a.r, s_angles, row1 - row0 + 1, a.B, a.M, [&](int m, int& seq, int& t, int& place) {
                    seq = b;
                    t = row0 + m;
                    place = L + t;
                });
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int place = L + t[i];
            if (at0 + i * SLOTS + slot >= end || (place >> a.page_log2) >= s_bad) continue;
            if (turned) turn_chunk<D>(a.r.neighbours != 0, s_angles[t[i] - row0], j, x[i][0], x[i][1]);
            const size_t row = ((size_t)s_page[t[i] - row0] << a.page_log2) + (place & ((1 << a.page_log2) - 1));
            if (!GSD_IN_BOUNDS(place < a.Lmax && row < (size_t)a.num_pages << a.page_log2, a.status)) continue;
            uint16_t *k = a.k_pages + (row * a.Hkv + h[i]) * D, *v = a.v_pages + (row * a.Hkv + h[i]) * D;
            *reinterpret_cast<uint4*>(k + col.x) = x[i][0];
            *reinterpret_cast<uint4*>(k + col.y) = x[i][1];
            *reinterpret_cast<uint4*>(v + col.x) = x[i][2];
            *reinterpret_cast<uint4*>(v + col.y) = x[i][3];
        }
    }
    if (begin < end && s_bad != 0x7FFFFFFF) flags |= GSD_DEV_BAD_PAGE;
    if (flags && a.status) atomicOr((unsigned*)a.status, flags);
    if (MODE != APPEND) {
        // (not the aligned forms: the warps come here by way of branches that their threads took apart)
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (blockIdx.x == 0 && tid == 0) {
            const int bad = s_bad;
            a.seq_lens[b] = bad == 0x7FFFFFFF ? L + n : max(L, min(L + n, bad << a.page_log2));
        }
    }
}

// The lengths behind an append whose CTAs are too many to meet: a warp per sequence.  It starts when every CTA of the append has
// passed its own wait - all that precedes the call is over then - works the new length out, and stores it once the append,
// whose CTAs read the old one, is over.
__global__ void __launch_bounds__(kThreads) paged_advance_kernel(WriteArgs a) {
    let_successor_start();
    const int b = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    int moved = 0;
    if (b < a.B) {
        const int L = min(max(a.seq_lens[b], 0), a.Lmax);
        const int n = min(min(max(a.count[b], 0), a.M), a.Lmax - L);
        moved = L + n;
        if (n > 0) {
            const int first = L >> a.page_log2, end = ((L + n - 1) >> a.page_log2) + 1;
            const int bad = __reduce_min_sync(0xFFFFFFFFu, first_bad_page(a.table + (size_t)b * a.max_pages, first, end, a.num_pages, lane, 32));
            if (bad != end) moved = max(L, bad << a.page_log2);
        }
    }
    wait_for_predecessor();
    if (b < a.B && lane == 0) a.seq_lens[b] = moved;
}

constexpr int kCluster = 8;         // CTAs of a sequence that meet

template <int D>
int launch_write(WriteArgs& a, cudaStream_t stream) {
    DeviceInfo di;
    if (device_info(&di) != 0) return GSD_ERR_CUDA;
    const int slots = kThreads / (D / 16);
    const long long places = (long long)(a.nodes ? (a.Tcap < a.M ? a.Tcap : a.M) : a.M) * a.Hkv;
    a.batches = a.nodes ? 1 : rotary_batches(places * a.B, a.Hkv, D, di.sm_count);
    const long long ctas = (places + slots * a.batches - 1) / (slots * a.batches);
    if (!a.nodes && ctas > kCluster) {
        const dim3 grid((unsigned)ctas, a.B);
        if (a.batches == 1) GSD_CUDA_TRY(launch_dependent(paged_write_kernel<D, 1, APPEND>, grid, dim3(kThreads), 0, stream, a));
        else GSD_CUDA_TRY(launch_dependent(paged_write_kernel<D, 2, APPEND>, grid, dim3(kThreads), 0, stream, a));
        GSD_CUDA_TRY(launch_dependent(paged_advance_kernel, dim3((a.B + kThreads / 32 - 1) / (kThreads / 32)), dim3(kThreads), 0, stream, a));
        return GSD_OK;
    }
    int cluster = 1;
    while (cluster < kCluster && cluster < ctas) cluster <<= 1;
    cudaLaunchAttribute attr[2];
    dependent_launch_attr(attr);
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cluster, a.B);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    GSD_CUDA_TRY(cudaLaunchKernelEx(&cfg, a.nodes ? paged_write_kernel<D, 2, COMMIT> : paged_write_kernel<D, 2, APPEND_CLUSTER>, a));
    return GSD_OK;
}

int write_rows(WriteArgs& a, const gsd_page_params* c, int D, cudaStream_t stream) {
    a.page_log2 = page_rows_log2(c, a.Lmax);
    a.max_pages = c->max_pages;
    a.num_pages = c->num_pages;
    return D == 128 ? launch_write<128>(a, stream) : launch_write<64>(a, stream);
}

int misaligned(std::initializer_list<const void*> ptrs, unsigned bytes) {
    for (const void* ptr : ptrs)
        if (((uintptr_t)ptr & (bytes - 1)) != 0) return 1;
    return 0;
}

}  // namespace
}  // namespace gsd

extern "C" int gsd_commit_kv_paged(void* k_pages, void* v_pages, const int32_t* page_table, const void* draft_k, const void* draft_v,
                                   const int32_t* accepted_nodes, const int32_t* accepted_len, int32_t* seq_lens,
                                   const gsd_commit_params* p, const gsd_page_params* c, int32_t* status, void* stream) {
    using namespace gsd;
    if (!p || !c || !k_pages || !v_pages || !page_table || !draft_k || !draft_v || !accepted_nodes || !accepted_len || !seq_lens)
        return GSD_ERR_NULL_POINTER;
    if (p->B < 1 || p->N < 1 || p->N > GSD_MAX_NODES || p->Hkv < 1 || (p->D != 64 && p->D != 128) || p->Lmax < 1 ||
        p->Tcap < 1 || p->B > 65535 || p->Hkv > 65535 || page_rows_log2(c, p->Lmax) < 0)
        return GSD_ERR_BAD_SHAPE;
    if (misaligned({k_pages, v_pages, draft_k, draft_v}, 16) || misaligned({page_table, accepted_nodes, accepted_len, seq_lens}, 4))
        return GSD_ERR_MISALIGNED;
    WriteArgs a = {};
    a.k_pages = (uint16_t*)k_pages; a.v_pages = (uint16_t*)v_pages; a.table = page_table;
    a.k = (const uint16_t*)draft_k; a.v = (const uint16_t*)draft_v; a.nodes = accepted_nodes; a.count = accepted_len;
    a.seq_lens = seq_lens; a.status = status;
    a.k_stride = a.v_stride = (long long)p->Hkv * p->D;
    a.B = p->B; a.M = p->N; a.Hkv = p->Hkv; a.Lmax = p->Lmax; a.Tcap = p->Tcap;
    return write_rows(a, c, p->D, (cudaStream_t)stream);
}

extern "C" int gsd_append_kv_paged(void* k_pages, void* v_pages, const int32_t* page_table, const void* k, const void* v,
                                   const int32_t* counts, int32_t* seq_lens, const float* freqs, const int32_t* positions,
                                   const int32_t* offsets, const gsd_append_paged_params* p, const gsd_page_params* c,
                                   const gsd_rotation* r, int32_t* status, void* stream) {
    using namespace gsd;
    if (!p || !c || !k_pages || !v_pages || !page_table || !k || !v || !counts || !seq_lens || !r != !freqs) return GSD_ERR_NULL_POINTER;
    if (p->B < 1 || p->T < 1 || p->Hkv < 1 || (p->D != 64 && p->D != 128) || p->Lmax < 1 || p->B > 65535 || p->Hkv > 65535 ||
        (long long)p->T * p->Hkv > (1 << 30) || page_rows_log2(c, p->Lmax) < 0)
        return GSD_ERR_BAD_SHAPE;
    if (p->k_stride < (long long)p->Hkv * p->D || p->v_stride < (long long)p->Hkv * p->D) return GSD_ERR_BAD_SHAPE;
    WriteArgs a = {};
    if (r && !rotation_of(r, p->D, &a.r)) return GSD_ERR_BAD_SHAPE;
    if (misaligned({k_pages, v_pages, k, v}, 16) || misaligned({page_table, counts, seq_lens, freqs, positions, offsets}, 4) ||
        p->k_stride % 8 != 0 || p->v_stride % 8 != 0)
        return GSD_ERR_MISALIGNED;
    a.k_pages = (uint16_t*)k_pages; a.v_pages = (uint16_t*)v_pages; a.table = page_table;
    a.k = (const uint16_t*)k; a.v = (const uint16_t*)v; a.count = counts;
    a.seq_lens = seq_lens; a.status = status;
    a.r.freqs = freqs; a.r.positions = positions; a.r.offsets = offsets;
    a.k_stride = p->k_stride; a.v_stride = p->v_stride;
    a.B = p->B; a.M = p->T; a.Hkv = p->Hkv; a.Lmax = p->Lmax; a.Tcap = 0;
    return write_rows(a, c, p->D, (cudaStream_t)stream);
}
