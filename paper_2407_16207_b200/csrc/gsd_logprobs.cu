// gsd_token_logprobs: log probabilities of given tokens, entropy of the rows they came from, and the rows' best entries.
//
//   with m = max x, y_j = (x_j - m) log2(e), s = sum 2^y_j, u = sum y_j 2^y_j:
//   log p_t = (x_t - m) - ln s,   entropy = ln s - ln(2) u / s
//
// Two launches, one read of the logits, which bound it where the call is large; where it is small the latency of both does.
//
// The first shares the rows of all sequences out in loads of 4 KB, as many in a row to each warp that fits, wherever a row
// ends: with a grid per sequence, or with slices of equal length, a last and partly filled wave cost up to a third.
// A lane keeps sums at its own maximum, so that warps never wait for one another; the load that follows is asked for
// from DRAM before a warp turns to the one it has (6 rows x 128 of 50257: 29.0 -> 27.2 us).
// The best entries: lanes' maxima over a load, sorted into a list of 32, bound from below what the k best reach, as every
// one of them is an entry; groups of four that reach the bound are put by as they are, and only when a slice is done,
// or the place for them full, are their entries sorted.  In random rows some k (1 + ln n) of n loads' entries come so far.
// A slice, what a warp has of a row, leaves (m, s, u) and k sorted 64-bit keys (value, then lowest index first).  The
// second launch, a warp per token and a programmatic dependent, puts the slices together, in 3 to 6 us.
// Entries at -inf are never put by; if fewer than k are left, the lowest indices that are not among them follow.
//
// Measured, of the time a copy of the same bytes takes: 6 rows x 128 of 50257, k 0: 27.2 us (87%), k 5: 38.4 us, k 20:
// 42.0 us; 8 x 256 rows of 32000, k 5: 54.6 us (73%); 9 rows of 50257, k 20: 9.6 us.  What the k best add is latency: sorts
// of 15 steps, one behind the other, while a warp's next load has come.  A CTA per slice in registers with a
// block-wide threshold took 42.9, 64.4, 68.3, 144.5 and 9.0 us; 4 CTAs per SM (64 registers, spills) 27.7, 46.0 and
// 51.8 us, a load of 2 KB 26.9, 48.4 and 56.5 us, of 8 KB 27.4, 61.0 and 59.9 us.
#include "gsd_internal.cuh"
#include <math_constants.h>

namespace gsd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kJoinWarps = 4;
constexpr int kVecs = 8;                            // 16-byte loads of a thread
constexpr int kCtasPerSm = 3;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kGroup = 1024;                        // sequences whose rows are shared out together, at most

struct SliceStats {
    float m, s, u, pad;
};
struct LogprobArgs {
    const float* logits;
    const int32_t *nodes, *tokens, *lens;
    float *logprobs, *entropy;
    int32_t* top_tokens;
    float* top_logprobs;
    SliceStats* stats;              // [groups][places]
    unsigned long long* keys;       // [groups][places][k]
    int32_t* status;
    int B, N, V, T, k;
    int loads, warps;               // of a row; of a group of sequences
    int per_group;                  // sequences
    // Warp w has the loads from w * per_warp on, in the order of the rows, and its slice of row r the place r + w: from one
    // slice to the next either goes up by one.
    __device__ __forceinline__ long long per_warp(int rows) const { return ((long long)rows * loads + warps - 1) / warps; }
    __device__ __forceinline__ size_t place0(int group) const { return (size_t)group * (warps + (size_t)per_group * T); }
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
__device__ __forceinline__ unsigned pick(unsigned a, unsigned b, bool larger) { return larger ? max(a, b) : min(a, b); }
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

// packed fp32 pairs
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
    return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    unsigned long long d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
    return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d)
        : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)), "l"(*reinterpret_cast<unsigned long long*>(&c)));
    return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ void prefetch(const float4* p, int vecs) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" :: "l"(p), "r"(vecs * 16) : "memory");
}
// sum 2^y and sum y 2^y at the maximum m
struct Sums {
    float m, s, u;
    __device__ __forceinline__ float raise(float to) {               // to a larger maximum; returns what entries are taken relative to
        const float m_use = to == -CUDART_INF_F ? 0.f : to;
        const float d = fmaxf((m - m_use) * kLog2e, -200.f), f = ex2(d);
        u = f * fmaf(s, d, u);
        s *= f;
        m = to;
        return m_use;
    }
};
// A warp's sums, in every lane.
__device__ __forceinline__ void reduce(Sums& v) {
    float m = v.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, o));
    v.raise(m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.s += __shfl_xor_sync(kAll, v.s, o);
        v.u += __shfl_xor_sync(kAll, v.u, o);
    }
}
// Keys that wait to be sorted into a warp's list of the 32 best, which lies in its lanes in descending order.
constexpr int kKeys = 160;
struct Best {
    unsigned long long list;
    unsigned long long* keys;       // [kKeys]
    int count;
    bool any;                       // in the list
    __device__ __forceinline__ void add(bool is, unsigned long long key, int lane) {
        const unsigned who = __ballot_sync(kAll, is);
        if (is) keys[count + __popc(who & ((1u << lane) - 1))] = key;
        count += __popc(who);
    }
    __device__ __forceinline__ void sort(int lane) {
        __syncwarp();
        for (int at = 0; at < count; at += 32) {
            const unsigned long long next = sort32(at + lane < count ? keys[at + lane] : 0ull, lane);
            list = any ? merge32(list, __shfl_sync(kAll, next, 31 - lane), lane) : next;
            any = true;
        }
        count = 0;
        __syncwarp();
    }
};
// The groups of four entries that may hold one of the best.
constexpr int kPool = 128;
struct Pool {
    float4* vec;                    // [kPool]
    int* at;                        // their first entries' indices
    int count;
    float least;                    // k entries of lower index than any to come reach it
    float tops;                     // the 32 largest maxima of a lane over a batch, descending
    bool any;                       // in tops
    __device__ __forceinline__ void add(unsigned who, const float4& v, int index, int lane) {
        if (who >> lane & 1) {
            const int to = count + __popc(who & ((1u << lane) - 1));
            vec[to] = v;
            at[to] = index;
        }
        count += __popc(who);
    }
    __device__ __forceinline__ void sort(Best& best, float bound, int k, int lane) {
        __syncwarp();
        for (int first = 0; first < count; first += 32) {
            const bool is = first + lane < count;
            const float4 x = is ? vec[first + lane] : make_float4(-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F);
            const int index = is ? at[first + lane] : 0;
            const float v[4] = {x.x, x.y, x.z, x.w};
            if (best.count > kKeys - 128) best.sort(lane);
#pragma unroll
            for (int h = 0; h < 4; ++h) best.add(v[h] >= bound && v[h] > -CUDART_INF_F, key_of(v[h], index + h), lane);
        }
        count = 0;
        best.sort(lane);
        const unsigned long long last = __shfl_sync(kAll, best.list, k - 1);
        if (last) least = fmaxf(least, key_value(last));
    }
};

// Rows of a group's sequences before each of them, and of all.
__device__ __forceinline__ void rows_before(const LogprobArgs& a, int b0, int nb, int (&from)[kGroup + 1]) {
    __shared__ int s_sum[kWarps];
    constexpr int kEach = kGroup / kThreads;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int n[kEach], sum = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        n[j] = tid * kEach + j < nb ? min(max(a.lens[b0 + tid * kEach + j], 0), a.T) : 0;
        sum += n[j];
    }
    int before = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(kAll, before, o);
        if (lane >= o) before += up;
    }
    if (lane == 31) s_sum[warp] = before;
    __syncthreads();
    before -= sum;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) before += w < warp ? s_sum[w] : 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if (tid * kEach + j <= nb) from[tid * kEach + j] = before;
        before += n[j];
    }
    if (nb == kGroup && tid == kThreads - 1) from[nb] = before;
    __syncthreads();
}

template <bool TOP>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) logprobs_scan_kernel(LogprobArgs a) {
    __shared__ int s_from[kGroup + 1];
    __shared__ float4 s_vec[TOP ? kWarps : 1][TOP ? kPool : 1];
    __shared__ int s_at[TOP ? kWarps : 1][TOP ? kPool : 1];
    __shared__ unsigned long long s_keys[TOP ? kWarps : 1][TOP ? kKeys : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b0 = blockIdx.y * a.per_group, nb = min(a.per_group, a.B - b0);
    wait_for_predecessor();
    let_successor_start();
    rows_before(a, b0, nb, s_from);
    const int rows = s_from[nb], me = warp * gridDim.x + blockIdx.x;
    const long long per = a.per_warp(rows), first = me * per;
    int left = (int)max(min(per, (long long)rows * a.loads - first), 0ll);
    if (left == 0) return;
    int r = (int)(first / a.loads), col = (int)(first - (long long)r * a.loads), seq = 0;
    for (int step = kGroup / 2; step > 0; step >>= 1)                // the last sequence that begins at or before row r: not empty
        if (seq + step < nb && s_from[seq + step] <= r) seq += step;
    int node = a.nodes[(size_t)(b0 + seq) * a.T + r - s_from[seq]];
    for (int n, here; left > 0; left -= n, ++r, col = 0) {
        n = min(left, a.loads - col);
        here = node;
        const int b = b0 + seq;
        if (left > n) {
            while (s_from[seq + 1] <= r + 1) ++seq;
            node = a.nodes[(size_t)(b0 + seq) * a.T + r + 1 - s_from[seq]];
        }
        if (here < 0 || here >= a.N) continue;                       // (the second launch says so)
        const float* row = a.logits + ((size_t)b * a.N + here) * a.V;
        const RowSpan span = row_span(row, a.V);
        const bool last = col + n == a.loads;
        const int v0 = col * 32 * kVecs, v1 = last ? span.nvec : (col + n) * 32 * kVecs;
        const float4* vec = reinterpret_cast<const float4*>(row + span.head);
        Sums sums{-CUDART_INF_F, 0.f, 0.f};
        Best best{0ull, s_keys[TOP ? warp : 0], 0, false};
        Pool pool{s_vec[TOP ? warp : 0], s_at[TOP ? warp : 0], 0, -CUDART_INF_F, -CUDART_INF_F, false};
        // the entries before the first boundary go with the first slice, those behind the last group with the last
        auto odd = [&](int first, int n) {
            const float v = lane < n ? row[first + lane] : -CUDART_INF_F;
            const float y = fmaxf((v - sums.raise(fmaxf(sums.m, v))) * kLog2e, -200.f), e = ex2(y);
            sums.s += v != v ? v : e;
            sums.u = fmaf(e, y, sums.u);
            if (TOP) pool.add(__ballot_sync(kAll, v > pool.least), make_float4(v, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F), first + lane, lane);
        };
        if (col == 0 && span.head) odd(0, span.head);
        for (int at = v0; at < v1; at += 32 * kVecs) {
            float4 x[kVecs];
#pragma unroll
            for (int j = 0; j < kVecs; ++j)
                x[j] = at + j * 32 + lane < v1 ? load_stream(vec + at + j * 32 + lane) : make_float4(-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F);
            if (lane == 0 && at + 32 * kVecs < v1) prefetch(vec + at + 32 * kVecs, min(32 * kVecs, v1 - at - 32 * kVecs));
            float top = -CUDART_INF_F;
#pragma unroll
            for (int j = 0; j < kVecs; ++j) top = max3(max3(x[j].x, x[j].y, top), x[j].z, x[j].w);
            if (TOP && __any_sync(kAll, top > pool.least)) {
                const float now = sort32(top, lane);
                pool.tops = pool.any ? merge32(pool.tops, __shfl_sync(kAll, now, 31 - lane), lane) : now;
                pool.any = true;
                const float bound = __shfl_sync(kAll, pool.tops, a.k - 1);
                unsigned in[kVecs];
                int all = pool.count;
#pragma unroll
                for (int j = 0; j < kVecs; ++j) {
                    const float g = fmaxf(max3(x[j].x, x[j].y, x[j].z), x[j].w);
                    in[j] = __ballot_sync(kAll, g > pool.least && g >= bound);
                    all += __popc(in[j]);
                }
                if (all <= kPool) {
#pragma unroll
                    for (int j = 0; j < kVecs; ++j) pool.add(in[j], x[j], span.head + 4 * (at + j * 32 + lane), lane);
                } else {
#pragma unroll
                    for (int j = 0; j < kVecs; ++j) {
                        if (pool.count > kPool - 32) pool.sort(best, fmaxf(bound, pool.least), a.k, lane);
                        const float g = fmaxf(max3(x[j].x, x[j].y, x[j].z), x[j].w);
                        pool.add(__ballot_sync(kAll, g > pool.least && g >= bound), x[j], span.head + 4 * (at + j * 32 + lane), lane);
                    }
                }
                pool.least = fmaxf(pool.least, bound);
            }
            const float m_use = sums.raise(fmaxf(sums.m, top));
            const float2 off = make_float2(-m_use, -m_use), scale = make_float2(kLog2e, kLog2e);
            float2 s2 = make_float2(0.f, 0.f), u2 = s2;
#pragma unroll
            for (int j = 0; j < kVecs; ++j) {
                const float2 p[2] = {make_float2(x[j].x, x[j].y), make_float2(x[j].z, x[j].w)};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float2 y = mul2(add2(p[h], off), scale);
                    const float2 e = make_float2(ex2(y.x), ex2(y.y));
                    s2 = add2(s2, e);                                // (a NaN stays in s)
                    y = make_float2(fmaxf(y.x, -200.f), fmaxf(y.y, -200.f));
                    u2 = fma2(e, y, u2);
                }
            }
            sums.s += s2.x + s2.y;
            sums.u += u2.x + u2.y;
        }
        const int behind = span.head + 4 * span.nvec;
        if (last && behind < a.V) {
            if (TOP && pool.count > kPool - 32) pool.sort(best, pool.least, a.k, lane);
            odd(behind, a.V - behind);
        }
        reduce(sums);
        const size_t out = a.place0(blockIdx.y) + r + me;
        if (lane == 0) a.stats[out] = SliceStats{sums.m, sums.s, sums.u, 0.f};
        if (TOP) {
            pool.sort(best, pool.least, a.k, lane);
            if (lane < a.k) a.keys[out * a.k + lane] = best.list;
        }
    }
}

__device__ __forceinline__ void finish(const LogprobArgs& a, size_t at, bool row_ok, bool token_ok, float given, float m, float s, float u, unsigned long long best, int lane) {
    const float nan = CUDART_NAN_F;
    // (a row with a NaN or +inf has a NaN sum, one without a finite entry an empty one)
    const bool ok = row_ok && s > 0.f && m < CUDART_INF_F;
    const float ln_s = logf(s);
    if (lane == 0) {
        a.logprobs[at] = !ok || !token_ok ? nan : given - m - ln_s;
        if (a.entropy) a.entropy[at] = ok ? fmaxf(ln_s - kLn2 * (u / s), 0.f) : nan;
        const unsigned flags = (row_ok ? 0u : GSD_DEV_BAD_CSR) | (row_ok && !ok ? GSD_DEV_BAD_LOGITS : 0u) | (token_ok ? 0u : GSD_DEV_BAD_TOKEN);
        if (flags && a.status) atomicOr((unsigned*)a.status, flags);
    }
    if (a.k == 0) return;
    const int have = __popc(__ballot_sync(kAll, best != 0ull));
    int index = best ? key_index(best) : -1;
    const float value = best ? key_value(best) : -CUDART_INF_F;
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
// What lies behind the last token of the sequence.
__device__ __forceinline__ void clear_behind(const LogprobArgs& a, int b, int len) {
    const int step = (int)(gridDim.x * blockDim.x), from = (int)(blockIdx.x * blockDim.x + threadIdx.x);
    for (int i = len + from; i < a.T; i += step) {
        a.logprobs[(size_t)b * a.T + i] = 0.f;
        if (a.entropy) a.entropy[(size_t)b * a.T + i] = 0.f;
    }
    for (int i = len * a.k + from; i < a.T * a.k; i += step) {
        a.top_tokens[(size_t)b * a.T * a.k + i] = -1;
        a.top_logprobs[(size_t)b * a.T * a.k + i] = 0.f;
    }
}

constexpr int kFetch = 4;                            // keys of a lane at a time
// A warp puts the slices of a token together.
template <bool TOP>
__global__ void __launch_bounds__(kJoinWarps * 32) logprobs_join_kernel(LogprobArgs a) {
    __shared__ unsigned long long s_keys[TOP ? kJoinWarps : 1][TOP ? 32 + 32 * kFetch : 1];
    let_successor_start();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.y;
    // (the inputs are older than the first launch, which let this one start after its own wait)
    const int len = min(max(a.lens[b], 0), a.T);
    const int group = b / a.per_group, b0 = group * a.per_group, nb = min(a.per_group, a.B - b0);
    int from = 0, rows = 0;
    for (int k = lane; k < nb; k += 32) {
        const int n = min(max(a.lens[b0 + k], 0), a.T);
        rows += n;
        from += b0 + k < b ? n : 0;
    }
    from = __reduce_add_sync(kAll, from);
    rows = __reduce_add_sync(kAll, rows);
    const long long per = max(a.per_warp(rows), 1ll);
    int i = blockIdx.x * kJoinWarps + warp;
    bool row_ok = false, token_ok = false;
    float given = 0.f;
    auto look = [&] {
        if (i >= len) return;
        const int node = a.nodes[(size_t)b * a.T + i], token = a.tokens[(size_t)b * a.T + i];
        row_ok = node >= 0 && node < a.N;
        token_ok = token >= 0 && token < a.V;
        if (row_ok && token_ok) given = a.logits[((size_t)b * a.N + node) * a.V + token];
    };
    look();
    wait_for_predecessor();
    for (; i < len; i += gridDim.x * kJoinWarps, look()) {
        const size_t at = (size_t)b * a.T + i;
        const long long first = (long long)(from + i) * a.loads;
        const int w0 = (int)(first / per), slices = (int)((first + a.loads - 1) / per) - w0 + 1;
        const size_t place = a.place0(group) + from + i + w0;
        Sums sums{-CUDART_INF_F, 0.f, 0.f};
        Best best{0ull, s_keys[TOP ? warp : 0], 0, false};
        if (row_ok) {
            const unsigned long long* keys = a.keys + place * a.k;
            const unsigned n = a.k * slices;
            unsigned long long key[kFetch], top;
            auto fetch = [&](unsigned p) {
#pragma unroll
                for (int h = 0; h < kFetch; ++h, p += 32) {
                    key[h] = 0ull;
                    if (p - lane >= n) continue;                     // (of the whole warp)
                    const unsigned rank = p / (unsigned)slices;
                    if (p < n) key[h] = keys[(size_t)(p - rank * slices) * a.k + rank];
                }
            };
            if (TOP) fetch(lane);
            for (int k = lane; k < slices; k += 128) {
                SliceStats v[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) v[h] = k + h * 32 < slices ? a.stats[place + k + h * 32] : SliceStats{-CUDART_INF_F, 0.f, 0.f, 0.f};
                const float m_use = sums.raise(max3(max3(v[0].m, v[1].m, sums.m), v[2].m, v[3].m));
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const float d = fmaxf((v[h].m - m_use) * kLog2e, -200.f), f = ex2(d);
                    sums.s = fmaf(f, v[h].s, sums.s);
                    sums.u = fmaf(f, fmaf(v[h].s, d, v[h].u), sums.u);
                }
            }
            reduce(sums);
            if (TOP) {
                // k lanes' best values among the slices' first keys bound what is looked at
                auto best_of = [&] {
                    top = key[0];
#pragma unroll
                    for (int h = 1; h < kFetch; ++h) top = max(top, key[h]);
                };
                best_of();
                const unsigned bound = __shfl_sync(kAll, sort32((unsigned)(top >> 32), lane), a.k - 1);
                unsigned long long least = bound ? (unsigned long long)bound << 32 : 1ull;
                // the slices' keys descend: as many in a row as there are slices, all less, are less than those behind them
                for (unsigned p = 0, without = 0; p < n && without < slices; p += 32 * kFetch) {
                    if (p) { fetch(p + lane); best_of(); }
                    if (!__any_sync(kAll, top >= least)) { without += 32 * kFetch; continue; }
                    without = 0;
                    if (best.count > 32) {
                        best.sort(lane);
                        const unsigned long long last = __shfl_sync(kAll, best.list, a.k - 1);
                        least = last > least ? last : least;
                    }
#pragma unroll
                    for (int h = 0; h < kFetch; ++h)
                        if (p + h * 32 < n) best.add(key[h] >= least, key[h], lane);
                }
                best.sort(lane);
            }
        }
        finish(a, at, row_ok, token_ok, given, sums.m, sums.s, sums.u, best.list, lane);
    }
    clear_behind(a, b, len);
}

int params_ok(const gsd_logprobs_params* p) {
    if (!p) return GSD_ERR_NULL_POINTER;
    if (p->B < 1 || p->B > 65535 || p->N < 1 || p->N > GSD_MAX_NODES || p->V < 1 || p->T < 1 || p->T > GSD_MAX_NODES || p->k < 0 ||
        p->k > GSD_LOGPROBS_MAX_K || p->k > p->V)
        return GSD_ERR_BAD_SHAPE;
    return GSD_OK;
}
// Loads of a warp that a row takes.
int loads_of(const gsd_logprobs_params* p) {
    const int n = (int)(((long long)p->V / 4 + 32 * kVecs - 1) / (32 * kVecs));
    return n > 0 ? n : 1;
}
// Groups of as equal numbers of sequences as can be; the CTAs and the places in scratch of each.
struct Groups {
    int sequences, groups, blocks;
    size_t places;
};
Groups groups_of(const gsd_logprobs_params* p, int sm_count) {
    Groups g;
    g.groups = (p->B + kGroup - 1) / kGroup;
    g.sequences = (p->B + g.groups - 1) / g.groups;
    g.groups = (p->B + g.sequences - 1) / g.sequences;
    const long long most = (kCtasPerSm * sm_count + g.groups - 1) / g.groups, work = (long long)g.sequences * p->T * loads_of(p);
    g.blocks = (int)(work < most ? work : most);
    g.places = (size_t)g.groups * ((size_t)g.blocks * kWarps + (size_t)g.sequences * p->T);
    return g;
}
}  // namespace
}  // namespace gsd

extern "C" size_t gsd_token_logprobs_workspace_bytes(const gsd_logprobs_params* p) {
    using namespace gsd;
    DeviceInfo di;
    if (params_ok(p) != GSD_OK || device_info(&di) != 0) return 0;
    return align_up(groups_of(p, di.sm_count).places * (sizeof(SliceStats) + 8 * (size_t)p->k), 256);
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
    const Groups g = groups_of(p, di.sm_count);
    a.B = p->B; a.N = p->N; a.V = p->V; a.T = p->T; a.k = p->k; a.loads = loads_of(p); a.warps = g.blocks * kWarps; a.per_group = g.sequences;
    const size_t places = g.places;
    if (!workspace || workspace_bytes < places * (sizeof(SliceStats) + 8 * (size_t)p->k)) return GSD_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 7u) != 0) return GSD_ERR_MISALIGNED;
    a.stats = (SliceStats*)workspace;
    a.keys = (unsigned long long*)((char*)workspace + places * sizeof(SliceStats));
    GSD_CUDA_TRY(launch_dependent(p->k > 0 ? logprobs_scan_kernel<true> : logprobs_scan_kernel<false>, dim3(g.blocks, g.groups), dim3(kThreads), 0, (cudaStream_t)stream, a));
    const long long most = (16ll * di.sm_count + p->B - 1) / p->B, join = (p->T + kJoinWarps - 1) / kJoinWarps;
    GSD_CUDA_TRY(launch_dependent(p->k > 0 ? logprobs_join_kernel<true> : logprobs_join_kernel<false>, dim3((unsigned)(join < most ? join : most), p->B), dim3(kJoinWarps * 32), 0, (cudaStream_t)stream, a));
    return GSD_OK;
}
