// gsd_commit_kv_q8 and gsd_append_kv_q8: bf16 K/V rows rounded into a cache held in 8 bits, behind the old end of every
// sequence (the accepted path of a verification step, or the rows of a prompt).
//
// For every block of `block` tokens and kv head that gets new rows x:
//   e(x)  = the least e with max |x| <= QMAX 2^e (QMAX 448 for e4m3, 127 for int8), within [-117, 119]
//   e'    = max(e, e(x)) where the block holds earlier rows with exponent e, else e(x)
//   codes = round(x 2^-e'), and of the earlier rows round(code 2^(e - e')), half to even, saturating
// The scales are powers of two: the quotients are exact in fp32 (of a normal result), so a code is the correctly rounded one
// on any machine, a row that is rounded again loses nothing to the quotient, and a reader may widen the codes and
// apply the scale without a rounding of its own.
//
// An item is one block of one head of K or V; a group of 32 to 256 threads, as many as its rows need at eight
// 16-byte pieces a thread, holds the item in registers: one read of the rows, the maximum by shuffles and shared memory, one
// write.  Heads follow one another, so that groups side by side read whole rows.  Bound by DRAM for prompts, by two
// dependent trips to memory (length and path, then the rows) for accepted paths; those go to one cluster of CTAs per
// sequence, which may advance seq_lens itself once every CTA of it has read the old length.  Where the exponent of a block
// grows, its earlier rows take another trip, or several: a group has room for kPieces pieces of each thread at a time.
// Measured: 8 x 4096 tokens of 8 heads, e4m3: blocks of 16 38.1 us (80% of the copy rate), of 128 42.0 us, int8 40.2 and 44.5;
// 8 paths of up to 17 tokens 4.6 us, 32 of up to 10 tokens of 40 heads 7.3 us.  3 to 64 CTAs an SM, 64 instead of 80
// registers: the same within 3%, but 34 and 49 us for two of the appends with one wave of CTAs.
// Paths behind blocks of 16, 64 and 128 tokens that hold all but one, no exponent growing and all of them (calls of a captured
// graph, which add 0.5 to 1.2 us): the 8 paths 5.1, 6.4, 6.2 and 5.6, 8.7, 11.8 us, the 32 paths 9.8, 9.7, 10.1 and 14.0, 22.0, 35.3 us; one
// row of 32 heads behind blocks of 128 4.1 and 12.8 us.  With the earlier rows read and written one piece after the other all
// growing took 8.7, 21.8, 38.1; 22.0, 57.6, 105.5; and 45.3 us.
#include "gsd_internal.cuh"
#include "gsd_kv8.cuh"
#include <initializer_list>

namespace gsd {
namespace {

constexpr int kThreads = 256;
constexpr int kPieces = 8;          // 16-byte pieces of a thread

struct WriteArgs {
    uint8_t *k_cache, *v_cache;
    int8_t *k_exp, *v_exp;
    const uint4 *k, *v;             // new rows [B, M, Hkv, D] bf16
    const int32_t* nodes;           // [B, Tcap] rows to take, or nullptr: the first ones
    const int32_t* count;
    int32_t* seq_lens;
    int32_t* status;
    int M, Hkv, Lmax, Tcap, NB, block_log2;
    int B;
};

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// Two values times f, as fp32 pairs (one instruction).
__device__ __forceinline__ float2 scaled(float a, float b, float f) {
    const float2 v = make_float2(a, b), s = make_float2(f, f);
    unsigned long long d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<const unsigned long long*>(&v)), "l"(*reinterpret_cast<const unsigned long long*>(&s)));
    return *reinterpret_cast<float2*>(&d);
}
// Four values in units of the scale, of at most 11 significant bits -> four codes.
// int8: the values are exact in fp16 (what is below its normal numbers becomes 0), and 1536 + x has x's nearest integer in its
// lowest bits, ties to even.  A conversion to an integer per value, at a quarter of the rate, took 51.2 instead of
// 44.4 us where 8 x 4096 tokens of 8 heads are appended.
template <bool INT8>
__device__ __forceinline__ uint32_t round4(float2 a, float2 b) {
    uint32_t w;
    if constexpr (INT8) {
        uint32_t p[2];
        const float2 v[2] = {a, b};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm("{\n .reg .b32 h;\n cvt.rn.satfinite.f16x2.f32 h, %2, %1;\n min.xorsign.abs.f16x2 h, h, %3;\n add.rn.f16x2 %0, h, %4;\n}"
                : "=r"(p[i]) : "f"(v[i].x), "f"(v[i].y), "r"(0x57F057F0u), "r"(0x66006600u));      // 127, 1536
        w = __byte_perm(p[0], p[1], 0x6420);
    } else {
        asm("{\n .reg .b16 l, h;\n cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n mov.b32 %0, {l, h};\n}"
            : "=r"(w) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    }
    return w;
}
// Four codes in units of another scale.
template <bool INT8>
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
    float x[4];
    if constexpr (INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
    } else {
        uint32_t p[2];
        asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(p[0]), "=r"(p[1]) : "r"(w));
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}" : "=f"(x[2 * i]), "=f"(x[2 * i + 1]) : "r"(p[i]));
    }
    return round4<INT8>(scaled(x[0], x[1], f), scaled(x[2], x[3], f));
}
// The exponent that a largest magnitude (bf16 bits) asks for.
template <bool INT8>
__device__ __forceinline__ int least_exp(uint32_t top) {
    const int e = INT8 ? (int)(top >> 7) - 133 + ((top & 127u) > 126u) : (int)(top >> 7) - 135 + ((top & 127u) > 96u);
    return min(max(e, GSD_KV8_EXP_MIN), GSD_KV8_EXP_MAX);
}

// What a call appends to sequence b: `n` rows behind position L, those that fit.
struct Span {
    int L, n;
};

template <int D, bool INT8, bool CLUSTER>
__global__ void __launch_bounds__(kThreads) kv8_write_kernel(WriteArgs a) {
    constexpr int ROW_PIECES = D / 8;
    __shared__ int s_src[GSD_MAX_NODES];
    __shared__ int s_tot[kThreads / 32];
    __shared__ uint32_t s_top[2][kThreads / 32];
    let_successor_start();
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    wait_for_predecessor();
    Span s;
    unsigned flags = 0;
    s.L = a.seq_lens[b];
    int want = a.count[b];
    if (s.L < 0 || s.L > a.Lmax) {
        flags |= GSD_DEV_BAD_SEQ_LEN;
        s.L = s.L < 0 ? 0 : a.Lmax;
    }
    // (only now may another CTA of the cluster write the length)
    if (CLUSTER) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    if (a.nodes) {
        // the valid node ids of the path, in order: a ballot a warp, a scan over the warps
        want = min(min(want, a.Tcap), GSD_MAX_NODES);
        int base = 0;
        for (int i0 = 0; i0 < want; i0 += kThreads) {
            const int i = i0 + tid;
            int node = -1;
            if (i < want) {
                node = a.nodes[(size_t)b * a.Tcap + i];
                if (node < 0 || node >= a.M) { node = -1; flags |= GSD_DEV_BAD_CSR; }
            }
            const unsigned vote = __ballot_sync(0xFFFFFFFFu, node >= 0);
            if (lane == 0) s_tot[warp] = __popc(vote);
            __syncthreads();
            int at = base;
            for (int w = 0; w < kThreads / 32; ++w) {
                if (w < warp) at += s_tot[w];
                base += s_tot[w];
            }
            if (node >= 0) s_src[at + __popc(vote & ((1u << lane) - 1u))] = node;
            __syncthreads();
        }
        want = base;
    } else if (want < 0 || want > a.M) {
        flags |= GSD_DEV_BAD_SEQ_LEN;
        want = want < 0 ? 0 : a.M;
    }
    s.n = min(want, a.Lmax - s.L);
    if (s.n < want) flags |= GSD_DEV_CACHE_FULL;

    if (s.n > 0) {
        const int block = 1 << a.block_log2, first = s.L >> a.block_log2, blocks = ((s.L + s.n - 1) >> a.block_log2) - first + 1;
        const int pieces = min(block, s.n) * ROW_PIECES;                   // of an item, at most
        int group = 32;
        while (group < kThreads && group * kPieces < pieces) group <<= 1;
        const int per_cta = kThreads / group, mine = tid / group, t = tid % group;
        const int items = 2 * blocks * a.Hkv, step = (int)gridDim.x * per_cta;
        int parity = 0;
        for (int i0 = (int)blockIdx.x * per_cta; i0 < items; i0 += step, parity ^= 1) {
            const int item = i0 + mine;
            const bool in = item < items;
            const int head = item % a.Hkv, blk = first + item / a.Hkv % blocks, is_v = item / a.Hkv / blocks;
            const int lo = blk << a.block_log2;
            const int r0 = max(lo, s.L), r1 = in ? min(lo + block, s.L + s.n) : r0;      // positions of the new rows
            const uint4* src = (is_v ? a.v : a.k) + ((size_t)b * a.M * a.Hkv + head) * ROW_PIECES;
            uint8_t* dst = (is_v ? a.v_cache : a.k_cache) + ((size_t)b * a.Lmax * a.Hkv + head) * D;
            int8_t* ex = (is_v ? a.v_exp : a.k_exp) + ((size_t)b * a.NB + blk) * a.Hkv + head;
            const bool held = in && lo < s.L;
            const int e_old = held && GSD_IN_BOUNDS(blk < a.NB, a.status) ? *ex : GSD_KV8_EXP_MIN;
            uint4 x[kPieces];
            uint32_t top2 = 0;
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                const int at = k * group + t, pos = r0 + at / ROW_PIECES;
                x[k] = make_uint4(0, 0, 0, 0);
                if (pos < r1) {
                    const int row = a.nodes ? s_src[pos - s.L] : pos - s.L;
                    if (GSD_IN_BOUNDS(row >= 0 && row < a.M, a.status)) x[k] = src[(size_t)row * a.Hkv * ROW_PIECES + at % ROW_PIECES];
                }
            }
            auto largest = [&]() {
                top2 = 0;
#pragma unroll
                for (int k = 0; k < kPieces; ++k)
                    top2 = max_u16x2(top2, max_u16x2(max_u16x2(x[k].x & 0x7FFF7FFFu, x[k].y & 0x7FFF7FFFu), max_u16x2(x[k].z & 0x7FFF7FFFu, x[k].w & 0x7FFF7FFFu)));
                return max(top2 & 0xFFFFu, top2 >> 16);
            };
            uint32_t top = largest();
            if (top >= 0x7F80u) {
                flags |= GSD_DEV_BAD_KV;
                if (top > 0x7F80u) {                                       // a NaN is stored as zero
                    auto clean = [](uint32_t& w) {
                        if ((w & 0x7FFFu) > 0x7F80u) w &= 0xFFFF0000u;
                        if ((w >> 16 & 0x7FFFu) > 0x7F80u) w &= 0xFFFFu;
                    };
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) { clean(x[k].x); clean(x[k].y); clean(x[k].z); clean(x[k].w); }
                    top = largest();
                }
            }
            top = __reduce_max_sync(0xFFFFFFFFu, top);
            if (group > 32) {
                // (two sets of words by turns: the next item's cannot overtake the reads of this one's)
                if (lane == 0) s_top[parity][warp] = top;
                __syncthreads();
                const int w0 = mine * (group / 32);
                for (int w = 0; w < group / 32; ++w) top = max(top, s_top[parity][w0 + w]);
            }
            if (!in) continue;
            const int e = max(least_exp<INT8>(top), e_old);
            const float f = two(-e);
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                const int at = k * group + t, pos = r0 + at / ROW_PIECES;
                if (pos >= r1 || !GSD_IN_BOUNDS(pos >= 0 && pos < a.Lmax, a.status)) continue;
                auto both = [&](uint32_t w) { return scaled(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u), f); };
                const uint2 c = make_uint2(round4<INT8>(both(x[k].x), both(x[k].y)), round4<INT8>(both(x[k].z), both(x[k].w)));
                *reinterpret_cast<uint2*>(dst + (size_t)pos * a.Hkv * D + at % ROW_PIECES * 8) = c;
            }
            if (held && e > e_old) {
                // the earlier rows of the block in the new scale, eight 16-byte pieces of a thread on their way
                const float g = e - e_old > 126 ? 0.f : two(e_old - e);
                constexpr int PIECES = D / 16;
                const int held_pieces = (s.L - lo) * PIECES;
                for (int at0 = t; at0 < held_pieces; at0 += kPieces * group) {
                    auto where = [&](int at) { return reinterpret_cast<uint4*>(dst + (size_t)(lo + at / PIECES) * a.Hkv * D + at % PIECES * 16); };
#pragma unroll
                    for (int k = 0; k < kPieces; ++k)
                        if (at0 + k * group < held_pieces) x[k] = *where(at0 + k * group);
#pragma unroll
                    for (int k = 0; k < kPieces; ++k)
                        if (at0 + k * group < held_pieces)
                            *where(at0 + k * group) = make_uint4(rescale4<INT8>(x[k].x, g), rescale4<INT8>(x[k].y, g), rescale4<INT8>(x[k].z, g), rescale4<INT8>(x[k].w, g));
                }
            }
            if (t == 0 && GSD_IN_BOUNDS(blk < a.NB, a.status)) *ex = (int8_t)e;
        }
    }
    if (flags && a.status) atomicOr((unsigned*)a.status, flags);
    if (CLUSTER) {
        // (not the aligned form: the threads come from branches of their own)
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (blockIdx.x == 0 && tid == 0) a.seq_lens[b] = s.L + s.n;
    }
}

// The lengths behind a call whose CTAs are too many to meet.
__global__ void __launch_bounds__(kThreads) kv8_advance_kernel(const int32_t* count, int32_t* seq_lens, int B, int M, int Lmax) {
    let_successor_start();
    wait_for_predecessor();
    const int b = blockIdx.x * kThreads + threadIdx.x;
    if (b >= B) return;
    const int L = min(max(seq_lens[b], 0), Lmax);
    seq_lens[b] = L + min(min(max(count[b], 0), M), Lmax - L);
}

constexpr int kCluster = 8;         // CTAs of a sequence that commits a path

template <int D, bool INT8>
int launch_write(const WriteArgs& a, cudaStream_t stream) {
    DeviceInfo di;
    if (device_info(&di) != 0) return GSD_ERR_CUDA;
    if (a.nodes) {
        // a warp's worth of rows an item, and at most two blocks for a path shorter than a block
        const int items = 2 * a.Hkv * 2;
        int ctas = 1;
        while (ctas < kCluster && ctas * (kThreads / 32) < items) ctas <<= 1;
        cudaLaunchAttribute attr[2];
        dependent_launch_attr(attr);
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = ctas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(ctas, a.B);
        cfg.blockDim = dim3(kThreads);
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        GSD_CUDA_TRY(cudaLaunchKernelEx(&cfg, kv8_write_kernel<D, INT8, true>, a));
        return GSD_OK;
    }
    const int block = 1 << a.block_log2, pieces = (block < a.M ? block : a.M) * (D / 8);
    int group = 32;
    while (group < kThreads && group * kPieces < pieces) group <<= 1;
    const int blocks = (a.M + block - 2) / block + 1;       // that M rows can touch
    const long long items = 2ll * a.Hkv * blocks, per_cta = kThreads / group;
    long long ctas = (items + per_cta - 1) / per_cta;
    const long long most = ((long long)di.sm_count * 8 + a.B - 1) / a.B;
    if (ctas > most) ctas = most;
    GSD_CUDA_TRY(launch_dependent(kv8_write_kernel<D, INT8, false>, dim3((unsigned)ctas, a.B), dim3(kThreads), 0, stream, a));
    GSD_CUDA_TRY(launch_dependent(kv8_advance_kernel, dim3((a.B + kThreads - 1) / kThreads), dim3(kThreads), 0, stream,
                                  a.count, a.seq_lens, a.B, a.M, a.Lmax));
    return GSD_OK;
}

int write_rows(WriteArgs& a, const gsd_kv8_params* c, int D, cudaStream_t stream) {
    a.block_log2 = kv8_block_log2(c);
    a.NB = (a.Lmax + c->block - 1) / c->block;
    if (c->format == GSD_KV8_INT8) return D == 128 ? launch_write<128, true>(a, stream) : launch_write<64, true>(a, stream);
    return D == 128 ? launch_write<128, false>(a, stream) : launch_write<64, false>(a, stream);
}

int misaligned(std::initializer_list<const void*> by16) {
    for (const void* ptr : by16)
        if (((uintptr_t)ptr & 15u) != 0) return 1;
    return 0;
}

}  // namespace
}  // namespace gsd

extern "C" int gsd_commit_kv_q8(void* k_cache, void* v_cache, int8_t* k_exp, int8_t* v_exp, const void* draft_k, const void* draft_v,
                                const int32_t* accepted_nodes, const int32_t* accepted_len, int32_t* seq_lens,
                                const gsd_commit_params* p, const gsd_kv8_params* c, int32_t* status, void* stream) {
    using namespace gsd;
    if (!p || !c || !k_cache || !v_cache || !k_exp || !v_exp || !draft_k || !draft_v || !accepted_nodes || !accepted_len || !seq_lens)
        return GSD_ERR_NULL_POINTER;
    if (p->B < 1 || p->N < 1 || p->N > GSD_MAX_NODES || p->Hkv < 1 || (p->D != 64 && p->D != 128) || p->Lmax < 1 ||
        p->Tcap < 1 || p->B > 65535 || p->Hkv > 65535 || kv8_block_log2(c) < 0)
        return GSD_ERR_BAD_SHAPE;
    if (misaligned({k_cache, v_cache, draft_k, draft_v})) return GSD_ERR_MISALIGNED;
    WriteArgs a;
    a.k_cache = (uint8_t*)k_cache; a.v_cache = (uint8_t*)v_cache; a.k_exp = k_exp; a.v_exp = v_exp;
    a.k = (const uint4*)draft_k; a.v = (const uint4*)draft_v; a.nodes = accepted_nodes; a.count = accepted_len;
    a.seq_lens = seq_lens; a.status = status;
    a.B = p->B; a.M = p->N; a.Hkv = p->Hkv; a.Lmax = p->Lmax; a.Tcap = p->Tcap;
    return write_rows(a, c, p->D, (cudaStream_t)stream);
}

extern "C" int gsd_append_kv_q8(void* k_cache, void* v_cache, int8_t* k_exp, int8_t* v_exp, const void* k, const void* v,
                                const int32_t* counts, int32_t* seq_lens, const gsd_append_params* p, const gsd_kv8_params* c,
                                int32_t* status, void* stream) {
    using namespace gsd;
    if (!p || !c || !k_cache || !v_cache || !k_exp || !v_exp || !k || !v || !counts || !seq_lens) return GSD_ERR_NULL_POINTER;
    if (p->B < 1 || p->T < 1 || p->Hkv < 1 || (p->D != 64 && p->D != 128) || p->Lmax < 1 || p->B > 65535 || p->Hkv > 65535 ||
        kv8_block_log2(c) < 0 || ((long long)p->T / c->block + 2) * 2 * p->Hkv > (1 << 30))
        return GSD_ERR_BAD_SHAPE;
    if (misaligned({k_cache, v_cache, k, v})) return GSD_ERR_MISALIGNED;
    WriteArgs a;
    a.k_cache = (uint8_t*)k_cache; a.v_cache = (uint8_t*)v_cache; a.k_exp = k_exp; a.v_exp = v_exp;
    a.k = (const uint4*)k; a.v = (const uint4*)v; a.nodes = nullptr; a.count = counts;
    a.seq_lens = seq_lens; a.status = status;
    a.B = p->B; a.M = p->T; a.Hkv = p->Hkv; a.Lmax = p->Lmax; a.Tcap = 0;
    return write_rows(a, c, p->D, (cudaStream_t)stream);
}
