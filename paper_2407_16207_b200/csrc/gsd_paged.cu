// gsd_append_kv_paged and gsd_commit_kv_paged: bf16 K/V rows into a cache held in pages, behind the old end of every sequence
// (the rows of a prompt, K rotated by position on the way; or the accepted path of a verification step).
//
// A thread has a chunk of 16 columns (gsd_rotary.cuh) of a row, of kHeads heads of K and the same of V; it asks for its pieces
// of all of them and looks up the page and forms its sines and cosines while they come.  Rows from the first on whose page the
// table does not name are dropped: every CTA looks through the entries up to its own last row's.
#include "gsd_pages.cuh"
#include "gsd_rotary.cuh"
#include <initializer_list>

namespace gsd {
namespace {

constexpr int kThreads = 256;

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
    int splits;                  // threads that share the heads of a row
};

enum Mode { APPEND, APPEND_CLUSTER, COMMIT };   // the rows of a grid, of one cluster per sequence; a path, one cluster per sequence

// One CTA of a sequence's, or all of them together, take the rows; with a cluster CTA 0 moves the length on once all have
// read the old one.
template <int D, int kHeads, int MODE>
__global__ void __launch_bounds__(kThreads) paged_write_kernel(WriteArgs a) {
    constexpr int CH = D / 16, SLOTS = kThreads / CH;
    __shared__ int s_src[MODE == COMMIT ? GSD_MAX_NODES : 1];     // source row of each new place
    __shared__ int s_tot[kThreads / 32];
    __shared__ int s_bad;                                         // first table entry that names no page
    let_successor_start();
    const int b = blockIdx.y, tid = threadIdx.x;
    const bool leader = blockIdx.x == 0;
    if (tid == 0) s_bad = 0x7FFFFFFF;
    wait_for_predecessor();
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

    const int32_t* row = a.table + (size_t)b * a.max_pages;
    const int page = 1 << a.page_log2, first_entry = L >> a.page_log2;
    const int stride = (int)gridDim.x * SLOTS, begin = (int)blockIdx.x * SLOTS, items = n * a.splits;
    const int last_item = MODE == APPEND ? min(begin + SLOTS, items) - 1 : items - 1;     // whose page the CTA has to know
    if (begin < items || (MODE != APPEND && leader)) __syncthreads();
    for (int i0 = begin; i0 < items; i0 += stride) {
        const int item = i0 + tid / CH, j = tid % CH;
        const int t = item / a.splits, part = item - t * a.splits;
        const bool in = item < items;
        const int2 col = chunk_columns(a.r, j);
        uint4 x[2 * kHeads][2];
        if (in) {
            const int from = MODE == COMMIT ? s_src[t] : t;
            const size_t tok = (size_t)b * a.M + from;
#pragma unroll
            for (int i = 0; i < 2 * kHeads; ++i) {
                const int h = part + (i >> 1) * a.splits;
                if (h < a.Hkv) {
                    const uint16_t* src = (i & 1 ? a.v + tok * a.v_stride : a.k + tok * a.k_stride) + h * D;
                    x[i][0] = *reinterpret_cast<const uint4*>(src + col.x);
                    x[i][1] = *reinterpret_cast<const uint4*>(src + col.y);
                }
            }
        }
        if (i0 == begin) {
            const int end = ((L + last_item / a.splits) >> a.page_log2) + 1;
            const int bad = first_bad_page(row, first_entry, end, a.num_pages, tid, kThreads);
            if (bad < end) atomicMin(&s_bad, bad);
            __syncthreads();
        }
        const int place = L + t, entry = place >> a.page_log2;
        float2 cs[8];
        const bool turned = MODE != COMMIT && j < a.r.chunks;
        if (MODE != COMMIT && in && turned) chunk_angles(a.r, j, token_pos(a.r, b, t, a.B, a.M, place), cs);
        if (!in || entry >= s_bad) continue;
        const size_t dst_row = (size_t)row[entry] * page + (place & (page - 1));
        if (!GSD_IN_BOUNDS(place < a.Lmax && dst_row < (size_t)a.num_pages * page, a.status)) continue;
#pragma unroll
        for (int i = 0; i < 2 * kHeads; ++i) {
            const int h = part + (i >> 1) * a.splits;
            if (h < a.Hkv) {
                if (!(i & 1) && turned) turn_chunk(a.r.neighbours != 0, cs, x[i][0], x[i][1]);
                uint16_t* dst = (i & 1 ? a.v_pages : a.k_pages) + (dst_row * a.Hkv + h) * D;
                *reinterpret_cast<uint4*>(dst + col.x) = x[i][0];
                *reinterpret_cast<uint4*>(dst + col.y) = x[i][1];
            }
        }
    }
    if (begin < items && s_bad != 0x7FFFFFFF) flags |= GSD_DEV_BAD_PAGE;
    if (flags && a.status) atomicOr((unsigned*)a.status, flags);
    if (MODE != APPEND) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (leader && tid == 0) {
            const int bad = s_bad;
            a.seq_lens[b] = bad == 0x7FFFFFFF ? L + n : max(L, min(L + n, bad << a.page_log2));
        }
    }
}

// The lengths behind an append whose CTAs are too many to meet: a warp per sequence.
__global__ void __launch_bounds__(kThreads) paged_advance_kernel(WriteArgs a) {
    let_successor_start();
    const int b = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    wait_for_predecessor();
    if (b >= a.B) return;
    const int L = min(max(a.seq_lens[b], 0), a.Lmax);
    const int n = min(min(max(a.count[b], 0), a.M), a.Lmax - L);
    if (n == 0) {
        if (lane == 0) a.seq_lens[b] = L;
        return;
    }
    const int first = L >> a.page_log2, end = ((L + n - 1) >> a.page_log2) + 1;
    const int bad = __reduce_min_sync(0xFFFFFFFFu, first_bad_page(a.table + (size_t)b * a.max_pages, first, end, a.num_pages, lane, 32));
    if (lane == 0) a.seq_lens[b] = bad == end ? L + n : max(L, bad << a.page_log2);
}

constexpr int kCluster = 8;         // CTAs of a sequence that meet

template <int D, int kHeads>
int launch_write(WriteArgs& a, cudaStream_t stream) {
    a.splits = (a.Hkv + kHeads - 1) / kHeads;
    const int slots = kThreads / (D / 16);
    const long long items = (long long)(a.nodes ? (a.Tcap < a.M ? a.Tcap : a.M) : a.M) * a.splits;
    const long long ctas = (items + slots - 1) / slots;
    if (!a.nodes && ctas > kCluster) {
        GSD_CUDA_TRY(launch_dependent(paged_write_kernel<D, kHeads, APPEND>, dim3((unsigned)ctas, a.B), dim3(kThreads), 0, stream, a));
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
    GSD_CUDA_TRY(cudaLaunchKernelEx(&cfg, a.nodes ? paged_write_kernel<D, kHeads, COMMIT> : paged_write_kernel<D, kHeads, APPEND_CLUSTER>, a));
    return GSD_OK;
}

int write_rows(WriteArgs& a, const gsd_page_params* c, int D, cudaStream_t stream) {
    a.page_log2 = page_rows_log2(c, a.Lmax);
    a.max_pages = c->max_pages;
    a.num_pages = c->num_pages;
    return D == 128 ? launch_write<128, 4>(a, stream) : launch_write<64, 4>(a, stream);
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
