// gsd_verify_attn_q8 with many stacked rows, first pass: the visible rows of an 8-bit cache as bf16 rows in scratch, over
// which the tcgen05 attention of a bf16 cache then runs.
//
//   out[b,j,c,:] = code[b,j,c,:] * 2^exp[b, j / block, c]   for j < seq_lens[b]: exact, bf16 holds every such value
//
// With many rows a key is used by many CTAs, and widening it once here (one read and two bytes written an element, at the
// rate of DRAM or, for caches of up to some 40 MB, of the L2; conversions take 65% of what their pipe has) costs less than widening it in every one of them: the tensor
// cores take no 8-bit operand beside a 16-bit one, and inside the attention kernel the widening warps, beside softmax
// warps that are almost always ready, get an instruction in every 10 to 20 cycles and add to the code that the instruction
// cache has to hold.  8 x 64/8 heads, N 256, L 4096: 432 to 790 us with four forms of that, the bf16 kernel alone 223; smaller row
// counts, whose softmax warps have more room, were not measured.
//
// A thread widens 16 codes at a time, four pieces on their way.  Blocks of their own copy the draft block's V with zeros for
// rows that no node of the sequence sees: the attention kernel multiplies every row of a tile, with a weight of 0 where it
// is hidden, and 0 times an infinity or NaN would reach the result.
#include "gsd_internal.cuh"
#include "gsd_kv8.cuh"

namespace gsd {
namespace {

constexpr int kThreads = 256, kBatch = 4;

struct ExpandArgs {
    const uint8_t *k_codes, *v_codes;
    const int8_t *k_exp, *v_exp;
    const int32_t* seq_lens;
    uint4 *k_out, *v_out;
    const uint4* draft_v;
    uint4* draft_v_out;
    const uint32_t* mask;
    int32_t* status;
    int B, N, W, Lmax, Hkv, NB, block_log2;
};

// Four rows of the draft block's V, eight pieces of a thread on their way.
constexpr int kDraftRows = 4;
template <int D>
__device__ __forceinline__ void copy_draft(const ExpandArgs& a, int b, int row0) {
    __shared__ uint32_t s_seen;
    if (threadIdx.x == 0) s_seen = 0;
    __syncthreads();
    uint32_t seen = 0;
    for (int n = threadIdx.x; n < a.N; n += kThreads) seen |= a.mask[((size_t)b * a.N + n) * a.W + (row0 >> 5)];
    seen = __reduce_or_sync(0xFFFFFFFFu, seen);
    if ((threadIdx.x & 31) == 0 && seen) atomicOr(&s_seen, seen);
    __syncthreads();
    seen = s_seen >> (row0 & 31);
    const int row_pieces = a.Hkv * (D / 8), total = min(kDraftRows, a.N - row0) * row_pieces;
    const size_t first = ((size_t)b * a.N + row0) * row_pieces;
    for (int at0 = threadIdx.x; at0 < total; at0 += 8 * kThreads) {
        uint4 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int at = at0 + k * kThreads;
            x[k] = at < total && (seen >> (at / row_pieces)) & 1u ? a.draft_v[first + at] : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (at0 + k * kThreads < total) a.draft_v_out[first + at0 + k * kThreads] = x[k];
    }
}

template <int D, bool INT8>
__global__ void __launch_bounds__(kThreads) kv8_expand_kernel(ExpandArgs a) {
    constexpr int PIECES = D / 16;                      // 16-byte pieces of a row of codes
    wait_for_predecessor();
    let_successor_start();
    const int b = blockIdx.y;
    if (blockIdx.z == 2) {
        for (int row0 = (int)blockIdx.x * kDraftRows; row0 < a.N; row0 += (int)gridDim.x * kDraftRows) {
            copy_draft<D>(a, b, row0);
            __syncthreads();
        }
        return;
    }
    const int L = min(max(a.seq_lens[b], 0), a.Lmax);
    const unsigned row_pieces = (unsigned)a.Hkv * PIECES;
    const long long total = (long long)L * row_pieces;
    const size_t first = (size_t)b * a.Lmax * row_pieces;
    const bool is_v = blockIdx.z != 0;
    const uint4* src = reinterpret_cast<const uint4*>(is_v ? a.v_codes : a.k_codes) + first;
    const int8_t* exps = (is_v ? a.v_exp : a.k_exp) + (size_t)b * a.NB * a.Hkv;
    uint4* dst = (is_v ? a.v_out : a.k_out) + first * 2;
    const long long step = (long long)gridDim.x * kThreads * kBatch;
    for (long long at0 = ((long long)blockIdx.x * kBatch) * kThreads + threadIdx.x; at0 < total; at0 += step) {
        uint4 x[kBatch];
        int e[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const long long at = at0 + k * kThreads;
            x[k] = make_uint4(0, 0, 0, 0);
            e[k] = 0;
            if (at < total) {
                x[k] = src[at];
                const int row = at < (1ll << 32) ? (int)((unsigned)at / row_pieces) : (int)(at / row_pieces);
                const int head = (int)(at - (long long)row * row_pieces) / PIECES;
                if (GSD_IN_BOUNDS((row >> a.block_log2) < a.NB, a.status)) e[k] = exps[(size_t)(row >> a.block_log2) * a.Hkv + head];
            }
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const long long at = at0 + k * kThreads;
            if (at >= total) continue;
            const float f = two(max(e[k], -126));
            const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
            uint32_t o[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[4];
                // (int8 through fp16 or bf16 arithmetic instead of a conversion per code: 1 x 64/8 heads, N 32, L 32768 76.8 us instead
                // of 70.4, e4m3 by bf16 arithmetic the same)
                if constexpr (INT8) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = (float)(int8_t)(w[i] >> (8 * j));
                } else {
                    uint32_t p[2];
                    widen<false>(w[i], p[0], p[1]);
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}" : "=f"(v[2 * j]), "=f"(v[2 * j + 1]) : "r"(p[j]));
                }
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[2 * i]) : "f"(v[1] * f), "f"(v[0] * f));
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[2 * i + 1]) : "f"(v[3] * f), "f"(v[2] * f));
            }
            // (32 bytes a store: with halves of a sector written one after the other the whole call of 8 x 64/8 heads, L 4096, took 275 us, 264 so)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"(dst + 2 * at), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]) : "memory");
        }
    }
}

template <int D, bool INT8>
int launch_t(const AttnArgs& a, void* k_out, void* v_out, void* draft_v_out) {
    ExpandArgs p;
    p.k_codes = (const uint8_t*)a.k_cache; p.v_codes = (const uint8_t*)a.v_cache;
    p.k_exp = a.kv8.k_exp; p.v_exp = a.kv8.v_exp; p.seq_lens = a.seq_lens; p.status = a.status;
    p.k_out = (uint4*)k_out; p.v_out = (uint4*)v_out;
    p.draft_v = (const uint4*)a.draft_v; p.draft_v_out = (uint4*)draft_v_out; p.mask = a.mask; p.N = a.N; p.W = a.W;
    p.B = a.B; p.Lmax = a.Lmax; p.Hkv = a.Hkv; p.NB = a.kv8.blocks; p.block_log2 = a.kv8.block_log2;
    DeviceInfo di;
    if (device_info(&di) != 0) return GSD_ERR_CUDA;
    const long long pieces = (long long)a.Lmax * a.Hkv * (D / 16), blocks = (pieces + kThreads * kBatch - 1) / (kThreads * kBatch);
    // (more blocks than fit: the sequences' lengths differ.  32 ragged sequences, the whole call: 142.3 us with 8 an SM, 139.9 with 16)
    const long long share = (32ll * di.sm_count + 2 * a.B - 1) / (2 * a.B);
    const long long grid = blocks < share ? blocks : share;
    GSD_CUDA_TRY(launch_dependent(kv8_expand_kernel<D, INT8>, dim3((unsigned)grid, a.B, 3), dim3(kThreads), 0, a.stream, p));
    return GSD_OK;
}

}  // namespace

int launch_kv8_expand(const AttnArgs& a, void* k_out, void* v_out, void* draft_v_out) {
    if (a.D == 128) return a.kv8.int8 ? launch_t<128, true>(a, k_out, v_out, draft_v_out) : launch_t<128, false>(a, k_out, v_out, draft_v_out);
    return a.kv8.int8 ? launch_t<64, true>(a, k_out, v_out, draft_v_out) : launch_t<64, false>(a, k_out, v_out, draft_v_out);
}

}  // namespace gsd
