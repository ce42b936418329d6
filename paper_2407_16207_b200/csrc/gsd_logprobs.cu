// gsd_token_logprobs: log probabilities of given tokens, entropy of the rows they came from, and the rows' best entries.
//
//   with m = max x, y_j = (x_j - m) log2(e), s = sum 2^y_j, u = sum y_j 2^y_j:
//   log p_t = (x_t - m) - ln s,   entropy = ln s - ln(2) u / s
//
// Two launches, one read of the logits.  The first cuts a row into slices of at most 8192 entries, which a CTA holds in
// registers: so the sums are formed at the slice's own maximum without rescaling, and the k best are found by a
// threshold instead of lists that every entry is compared with.  The k-th largest of the 256 threads' maxima is
// reached by at least k entries, and hardly more (20 of 8192 random ones: 21 on average); what reaches it is collected and
// sorted by one warp.  Runs of equal logits that overflow the collection take k rounds of a block-wide maximum instead.
// A slice leaves (m, s, u) and k sorted 64-bit keys (value, then lowest index first); the second launch, a CTA per
// token and a programmatic dependent, puts the slices together.
// Entries at -inf are never collected; if fewer than k are left, the lowest indices that are not among them follow.
#include "gsd_internal.cuh"
#include <math_constants.h>

namespace gsd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kVecs = 8;                            // 16-byte loads of a thread
constexpr int kSliceVecs = kThreads * kVecs;        // of a slice, at most
constexpr int kCollect = 128;
constexpr int kCtasPerSm = 3;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr unsigned kAll = 0xFFFFFFFFu;

struct SliceStats {
    float m, s, u, pad;
};
struct LogprobArgs {
    const float* logits;
    const int32_t *nodes, *tokens, *lens;
    float *logprobs, *entropy;
    int32_t* top_tokens;
    float* top_logprobs;
    SliceStats* stats;              // [B * T][slices]
    unsigned long long* keys;       // [B * T][slices][k]
    int32_t* status;
    int N, V, T, k, slices;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float4 load_stream(const float4* p) {
    float4 v;
    asm volatile("ld.global.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
    return v;
}
// Larger key = better entry: the value, then the lower index.  0 is no entry.
__device__ __forceinline__ unsigned long long key_of(float x, int i) {
    const unsigned b = __float_as_uint(x + 0.f);                       // (-0 counts as 0)
    return (unsigned long long)(b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u)) << 32 | (0xFFFFFFFFu - (unsigned)i);
}
__device__ __forceinline__ int key_index(unsigned long long k) { return (int)(0xFFFFFFFFu - (unsigned)k); }
__device__ __forceinline__ float key_value(unsigned long long k) {
    const unsigned b = (unsigned)(k >> 32);
    return __uint_as_float(b ^ ((b >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ float pick(float a, float b, bool larger) { return larger ? fmaxf(a, b) : fminf(a, b); }
__device__ __forceinline__ unsigned long long pick(unsigned long long a, unsigned long long b, bool larger) { return (a > b) == larger ? a : b; }
// A value a lane, brought into descending order (bitonic).
template <class X>
__device__ __forceinline__ X sort32(X v, int lane) {
#pragma unroll
    for (int n = 2; n <= 32; n <<= 1)
#pragma unroll
        for (int j = n >> 1; j > 0; j >>= 1) v = pick(v, __shfl_xor_sync(kAll, v, j), ((lane & n) == 0) == ((lane & j) == 0));
    return v;
}
// The 32 largest of two descending lists, descending; `b_reversed`: the other list from its end.
template <class X>
__device__ __forceinline__ X merge32(X a, X b_reversed, int lane) {
    X v = pick(a, b_reversed, true);
#pragma unroll
    for (int j = 16; j > 0; j >>= 1) v = pick(v, __shfl_xor_sync(kAll, v, j), (lane & j) == 0);
    return v;
}

__global__ void __launch_bounds__(kThreads, kCtasPerSm) logprobs_scan_kernel(LogprobArgs a) {
    __shared__ float s_sorted[kWarps][32];          // the lanes' maxima of every warp, descending
    __shared__ float2 s_sums[kWarps];
    __shared__ unsigned long long s_found[kCollect];
    __shared__ unsigned long long s_best[kWarps];
    __shared__ int s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.y;
    wait_for_predecessor();
    let_successor_start();
    const int len = min(max(a.lens[b], 0), a.T);
    for (int w = blockIdx.x; w < len * a.slices; w += gridDim.x) {
        const int i = w / a.slices, slice = w - i * a.slices;
        const int node = a.nodes[(size_t)b * a.T + i];
        if (node < 0 || node >= a.N) continue;                       // (the second launch says so)
        const float* row = a.logits + ((size_t)b * a.N + node) * a.V;
        const RowSpan span = row_span(row, a.V);
        const int per = (span.nvec + a.slices - 1) / a.slices;
        const int v0 = min(slice * per, span.nvec), n = min(per, span.nvec - v0);
        const float4* vec = reinterpret_cast<const float4*>(row + span.head) + v0;
        float4 x[kVecs];
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int at = j * kThreads + tid;
            x[j] = at < n ? load_stream(vec + at) : make_float4(-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F);
        }
        // the entries before the first boundary go with the first slice, those behind the last group with the last
        float odd = -CUDART_INF_F;
        int odd_at = -1;
        const int behind = span.head + 4 * span.nvec;
        if (slice == 0 && tid < span.head) odd_at = tid;
        if (slice == a.slices - 1 && tid >= 32 && behind + tid - 32 < a.V) odd_at = behind + tid - 32;
        if (odd_at >= 0) odd = row[odd_at];
        if (tid == 0) s_count = 0;

        float g[kVecs], top = odd;
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            g[j] = fmaxf(fmaxf(x[j].x, x[j].y), fmaxf(x[j].z, x[j].w));
            top = fmaxf(top, g[j]);
        }
        s_sorted[warp][lane] = sort32(top, lane);
        __syncthreads();
        float m = s_sorted[0][0];
#pragma unroll
        for (int k = 1; k < kWarps; ++k) m = fmaxf(m, s_sorted[k][0]);
        if (a.k > 0) {
            float l[kWarps];
#pragma unroll
            for (int k = 0; k < kWarps; ++k) l[k] = s_sorted[k][k & 1 ? 31 - lane : lane];
#pragma unroll
            for (int n2 = 1; n2 < kWarps; n2 <<= 1)
#pragma unroll
                for (int k = 0; k < kWarps; k += 2 * n2) {
                    const float up = merge32(l[k], l[k + n2], lane);
                    l[k] = (k / (2 * n2)) & 1 ? __shfl_sync(kAll, up, 31 - lane) : up;
                }
            const float least = __shfl_sync(kAll, l[0], a.k - 1);
            auto collect = [&](float v, int at) {
                if (v >= least && v > -CUDART_INF_F) {
                    const int pos = atomicAdd(&s_count, 1);
                    if (pos < kCollect) s_found[pos] = key_of(v, at);
                }
            };
#pragma unroll
            for (int j = 0; j < kVecs; ++j)
                if (g[j] >= least && g[j] > -CUDART_INF_F) {
                    const int at = span.head + 4 * (v0 + j * kThreads + tid);
                    collect(x[j].x, at); collect(x[j].y, at + 1); collect(x[j].z, at + 2); collect(x[j].w, at + 3);
                }
            collect(odd, odd_at);
        }
        const float m_use = m == -CUDART_INF_F ? 0.f : m;
        float s = 0.f, u = 0.f;
        auto add = [&](float v) {
            const float y = (v - m_use) * kLog2e, e = ex2(y);
            s += e;                                                  // (a NaN stays in s)
            u = fmaf(e, fmaxf(y, -200.f), u);
        };
#pragma unroll
        for (int j = 0; j < kVecs; ++j) { add(x[j].x); add(x[j].y); add(x[j].z); add(x[j].w); }
        add(odd);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s += __shfl_xor_sync(kAll, s, o);
            u += __shfl_xor_sync(kAll, u, o);
        }
        if (lane == 0) s_sums[warp] = make_float2(s, u);
        __syncthreads();
        const size_t out = ((size_t)b * a.T + i) * a.slices + slice;
        if (tid == 32) {
            SliceStats st{m, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kWarps; ++k) { st.s += s_sums[k].x; st.u += s_sums[k].y; }
            a.stats[out] = st;
        }
        if (a.k > 0) {
            const int count = s_count;
            if (count <= kCollect) {
                if (warp == 0) {
                    unsigned long long best = sort32(lane < count ? s_found[lane] : 0ull, lane);
                    for (int at = 32; at < count; at += 32) {
                        const unsigned long long next = sort32(at + lane < count ? s_found[at + lane] : 0ull, lane);
                        best = merge32(best, __shfl_sync(kAll, next, 31 - lane), lane);
                    }
                    if (lane < a.k) a.keys[out * a.k + lane] = best;
                }
            } else {
                unsigned long long last = ~0ull;
                for (int r = 0; r < a.k; ++r) {
                    unsigned long long best = 0;
                    auto offer = [&](float v, int at) {
                        const unsigned long long key = key_of(v, at);
                        if (v > -CUDART_INF_F && key < last && key > best) best = key;
                    };
#pragma unroll
                    for (int j = 0; j < kVecs; ++j) {
                        const int at = span.head + 4 * (v0 + j * kThreads + tid);
                        offer(x[j].x, at); offer(x[j].y, at + 1); offer(x[j].z, at + 2); offer(x[j].w, at + 3);
                    }
                    if (odd_at >= 0) offer(odd, odd_at);
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) best = pick(best, __shfl_xor_sync(kAll, best, o), true);
                    if (lane == 0) s_best[warp] = best;
                    __syncthreads();
#pragma unroll
                    for (int k = 0; k < kWarps; ++k) best = pick(best, s_best[k], true);
                    if (tid == 0) a.keys[out * a.k + r] = best;
                    last = best;
                    __syncthreads();
                }
            }
        }
        __syncthreads();                                             // (s_count, s_found and s_sums have been read)
    }
}

__global__ void __launch_bounds__(kThreads) logprobs_join_kernel(LogprobArgs a) {
    __shared__ unsigned long long s_list[kWarps][32];
    __shared__ float s_stat[2][kWarps];
    __shared__ float s_m[kWarps];
    let_successor_start();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.y;
    // (the inputs are older than the first launch, which let this one start after its own wait)
    const int len = min(max(a.lens[b], 0), a.T);
    wait_for_predecessor();
    const float nan = CUDART_NAN_F;
    for (int i = blockIdx.x; i < len; i += gridDim.x) {
        const size_t at = (size_t)b * a.T + i;
        const int node = a.nodes[at], token = a.tokens[at];
        const bool row_ok = node >= 0 && node < a.N, token_ok = token >= 0 && token < a.V;
        const SliceStats* st = a.stats + at * a.slices;
        // every warp has the sums of a share of the slices at their common maximum, and their best keys
        float m = -CUDART_INF_F;
        if (row_ok)
            for (int k = tid; k < a.slices; k += kThreads) m = fmaxf(m, st[k].m);
        m = fmaxf(m, __shfl_xor_sync(kAll, m, 16)); m = fmaxf(m, __shfl_xor_sync(kAll, m, 8)); m = fmaxf(m, __shfl_xor_sync(kAll, m, 4));
        m = fmaxf(m, __shfl_xor_sync(kAll, m, 2)); m = fmaxf(m, __shfl_xor_sync(kAll, m, 1));
        if (lane == 0) s_m[warp] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kWarps; ++k) m = fmaxf(m, s_m[k]);
        const float m_use = m == -CUDART_INF_F ? 0.f : m;
        float s = 0.f, u = 0.f;
        if (row_ok)
            for (int k = tid; k < a.slices; k += kThreads) {
                const SliceStats v = st[k];
                const float d = fmaxf((v.m - m_use) * kLog2e, -200.f), f = ex2(d);
                s += f * v.s;
                u += f * (v.u + v.s * d);
            }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s += __shfl_xor_sync(kAll, s, o);
            u += __shfl_xor_sync(kAll, u, o);
        }
        if (lane == 0) { s_stat[0][warp] = s; s_stat[1][warp] = u; }
        unsigned long long best = 0;
        if (a.k > 0 && row_ok) {
            const unsigned long long* keys = a.keys + at * a.slices * a.k;
            if (warp < a.slices && lane < a.k) best = keys[(size_t)warp * a.k + lane];
            for (int k = warp + kWarps; k < a.slices; k += kWarps)
                best = merge32(best, 31 - lane < a.k ? keys[(size_t)k * a.k + 31 - lane] : 0ull, lane);
            s_list[warp][lane] = best;
        }
        __syncthreads();
        if (warp == 0) {
            s = u = 0.f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) { s += s_stat[0][k]; u += s_stat[1][k]; }
            // (a row with a NaN or +inf has a NaN sum, one without a finite entry an empty one)
            const bool ok = row_ok && s > 0.f && m < CUDART_INF_F;
            const float ln_s = logf(s);
            if (lane == 0) {
                a.logprobs[at] = !ok || !token_ok ? nan : a.logits[((size_t)b * a.N + node) * a.V + token] - m - ln_s;
                if (a.entropy) a.entropy[at] = ok ? fmaxf(ln_s - kLn2 * (u / s), 0.f) : nan;
                const unsigned flags = (row_ok ? 0u : GSD_DEV_BAD_CSR) | (row_ok && !ok ? GSD_DEV_BAD_LOGITS : 0u) | (token_ok ? 0u : GSD_DEV_BAD_TOKEN);
                if (flags && a.status) atomicOr((unsigned*)a.status, flags);
            }
            if (a.k > 0) {
                if (row_ok)
                    for (int k = 1; k < min(kWarps, a.slices); ++k) best = merge32(best, s_list[k][31 - lane], lane);
                const int have = __popc(__ballot_sync(kAll, best != 0ull));
                int index = best ? key_index(best) : -1;
                float value = best ? key_value(best) : -CUDART_INF_F;
                if (ok && have < a.k) {
                    // entries at -inf: the lowest indices that are not among the others
                    int next = 0;
                    for (int r = have; r < a.k; ++r) {
                        while (__any_sync(kAll, lane < have && index == next)) ++next;
                        if (lane == r) index = next;
                        ++next;
                    }
                }
                if (lane < a.k) {
                    a.top_tokens[at * a.k + lane] = ok ? index : -1;
                    a.top_logprobs[at * a.k + lane] = ok ? value - m - ln_s : nan;
                }
            }
        }
        __syncthreads();                                             // (the shared words have been read)
    }
    // what lies behind the last token of the sequence
    const int step = (int)gridDim.x * kThreads, from = (int)blockIdx.x * kThreads + tid;
    for (int i = len + from; i < a.T; i += step) {
        a.logprobs[(size_t)b * a.T + i] = 0.f;
        if (a.entropy) a.entropy[(size_t)b * a.T + i] = 0.f;
    }
    for (int i = len * a.k + from; i < a.T * a.k; i += step) {
        a.top_tokens[(size_t)b * a.T * a.k + i] = -1;
        a.top_logprobs[(size_t)b * a.T * a.k + i] = 0.f;
    }
}

int params_ok(const gsd_logprobs_params* p) {
    if (!p) return GSD_ERR_NULL_POINTER;
    if (p->B < 1 || p->B > 65535 || p->N < 1 || p->N > GSD_MAX_NODES || p->V < 1 || p->T < 1 || p->T > GSD_MAX_NODES || p->k < 0 ||
        p->k > GSD_LOGPROBS_MAX_K || p->k > p->V)
        return GSD_ERR_BAD_SHAPE;
    return GSD_OK;
}
// Slices of a row: as many as their size asks for, more where there are few rows to go round.
int slices_of(const gsd_logprobs_params* p, int sm_count) {
    const int vecs = p->V / 4 + 1;
    const int need = (vecs + kSliceVecs - 1) / kSliceVecs;
    const long long rows = (long long)p->B * p->T;
    const int spread = (int)((2ll * sm_count + rows - 1) / rows), most = (vecs + kThreads - 1) / kThreads;
    const int want = spread < most ? spread : most;
    return need > want ? need : want;
}

}  // namespace
}  // namespace gsd

extern "C" size_t gsd_token_logprobs_workspace_bytes(const gsd_logprobs_params* p) {
    using namespace gsd;
    DeviceInfo di;
    if (params_ok(p) != GSD_OK || device_info(&di) != 0) return 0;
    return align_up((size_t)p->B * p->T * slices_of(p, di.sm_count) * (sizeof(SliceStats) + 8 * (size_t)p->k), 256);
}

extern "C" int gsd_token_logprobs(const float* logits, const int32_t* nodes, const int32_t* tokens, const int32_t* lens,
                                  float* logprobs, float* entropy, int32_t* top_tokens, float* top_logprobs,
                                  const gsd_logprobs_params* p, void* workspace, size_t workspace_bytes, int32_t* status,
                                  void* stream) {
    using namespace gsd;
    if (!p || !logits || !nodes || !tokens || !lens || !logprobs) return GSD_ERR_NULL_POINTER;
    const int ok = params_ok(p);
    if (ok != GSD_OK) return ok;
    if (p->k > 0 && (!top_tokens || !top_logprobs)) return GSD_ERR_NULL_POINTER;
    if (((uintptr_t)logits & 3u) != 0) return GSD_ERR_MISALIGNED;
    DeviceInfo di;
    if (device_info(&di) != 0) return GSD_ERR_CUDA;
    LogprobArgs a;
    a.logits = logits; a.nodes = nodes; a.tokens = tokens; a.lens = lens; a.logprobs = logprobs; a.entropy = entropy;
    a.top_tokens = top_tokens; a.top_logprobs = top_logprobs; a.status = status;
    a.N = p->N; a.V = p->V; a.T = p->T; a.k = p->k; a.slices = slices_of(p, di.sm_count);
    const size_t places = (size_t)p->B * p->T * a.slices;
    if (!workspace || workspace_bytes < places * (sizeof(SliceStats) + 8 * (size_t)p->k)) return GSD_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 7u) != 0) return GSD_ERR_MISALIGNED;
    a.stats = (SliceStats*)workspace;
    a.keys = (unsigned long long*)((char*)workspace + places * sizeof(SliceStats));
    const long long share = ((long long)kCtasPerSm * di.sm_count + p->B - 1) / p->B;
    const long long work = (long long)p->T * a.slices;
    GSD_CUDA_TRY(launch_dependent(logprobs_scan_kernel, dim3((unsigned)(work < share ? work : share), p->B), dim3(kThreads), 0, (cudaStream_t)stream, a));
    const long long join = 2 * share < p->T ? 2 * share : p->T;
    GSD_CUDA_TRY(launch_dependent(logprobs_join_kernel, dim3((unsigned)join, p->B), dim3(kThreads), 0, (cudaStream_t)stream, a));
    return GSD_OK;
}
