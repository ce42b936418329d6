// gsd_rotary: rotary positions of Q and K rows, with one position axis (text) or several (images, video).
//
//   angle_i = (positions[axis[i]][b][t] + offsets[b]) * freqs[i],   (x, y) -> (x cos - y sin, x sin + y cos)
//
// A thread has a chunk of 16 columns (gsd_rotary.cuh) of a token and kHeads heads of it, Q's heads and K's counted in one
// line; it asks for its pieces of all of them, forms its 8 sines and cosines while they come, and turns them.  The heads of a
// thread lie `splits` apart, so that neighbours read neighbouring heads.
#include "gsd_rotary.cuh"

namespace gsd {
namespace {

constexpr int kThreads = 256;

struct RotaryArgs {
    const uint16_t *q, *k;
    uint16_t *q_out, *k_out;
    Rotation r;
    int B, T, Hq, heads;         // heads of q and k together
    int splits;                  // threads that share the heads of a token
    int items;                   // tokens * splits
    long long q_stride, k_stride;
};

template <int D, int kHeads>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs p) {
    constexpr int CH = D / 16;
    let_successor_start();
    wait_for_predecessor();
    const int j = threadIdx.x % CH, item = blockIdx.x * (kThreads / CH) + threadIdx.x / CH;
    if (item >= p.items) return;
    const int tok = item / p.splits, part = item - tok * p.splits, b = tok / p.T, t = tok - b * p.T;
    const int2 col = chunk_columns(p.r, j);
    uint4 x[kHeads][2];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int h = part + i * p.splits;
        if (h < p.heads) {
            const uint16_t* src = h < p.Hq ? p.q + tok * p.q_stride + h * D : p.k + tok * p.k_stride + (h - p.Hq) * D;
            x[i][0] = *reinterpret_cast<const uint4*>(src + col.x);
            x[i][1] = *reinterpret_cast<const uint4*>(src + col.y);
        }
    }
    float2 cs[8];
    const bool turned = j < p.r.chunks;
    if (turned) chunk_angles(p.r, j, token_pos(p.r, b, t, p.B, p.T, 0), cs);
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int h = part + i * p.splits;
        if (h < p.heads) {
            if (turned) turn_chunk(p.r.neighbours != 0, cs, x[i][0], x[i][1]);
            uint16_t* dst = h < p.Hq ? p.q_out + ((size_t)tok * p.Hq + h) * D : p.k_out + ((size_t)tok * (p.heads - p.Hq) + h - p.Hq) * D;
            *reinterpret_cast<uint4*>(dst + col.x) = x[i][0];
            *reinterpret_cast<uint4*>(dst + col.y) = x[i][1];
        }
    }
}

template <int D>
int launch_rotary(RotaryArgs& a, cudaStream_t stream) {
    const long long tokens = (long long)a.B * a.T;
    auto go = [&](auto kernel, int heads) -> int {
        a.splits = (a.heads + heads - 1) / heads;
        a.items = (int)(tokens * a.splits);
        const int per_cta = kThreads / (D / 16);
        GSD_CUDA_TRY(launch_dependent(kernel, dim3((unsigned)((a.items + (long long)per_cta - 1) / per_cta)), dim3(kThreads), 0, stream, a));
        return GSD_OK;
    };
    return go(rotary_kernel<D, 4>, 4);
}

}  // namespace
}  // namespace gsd

extern "C" int gsd_rotary(const void* q, const void* k, const float* freqs, const int32_t* positions, const int32_t* offsets,
                          void* q_out, void* k_out, const gsd_rotary_params* p, const gsd_rotation* r, void* stream) {
    using namespace gsd;
    if (!p || !r || !q || !q_out || !freqs || !positions || !k != !k_out) return GSD_ERR_NULL_POINTER;
    const int Hkv = k ? p->Hkv : 0;
    if (p->B < 1 || p->T < 1 || p->Hq < 1 || (k && Hkv < 1) || (p->D != 64 && p->D != 128)) return GSD_ERR_BAD_SHAPE;
    // (a token's head is counted in 32 bits: 550 GB of them)
    const long long heads = (long long)p->Hq + Hkv;
    if (heads > (1 << 20) || (long long)p->B * p->T > 0x7FFFFFFFll / heads) return GSD_ERR_BAD_SHAPE;
    if (p->q_stride < (long long)p->Hq * p->D || (k && p->k_stride < (long long)Hkv * p->D)) return GSD_ERR_BAD_SHAPE;
    RotaryArgs a;
    if (!rotation_of(r, p->D, &a.r)) return GSD_ERR_BAD_SHAPE;
    for (const void* ptr : {q, k, (const void*)q_out, (const void*)k_out})
        if (((uintptr_t)ptr & 15u) != 0) return GSD_ERR_MISALIGNED;
    for (const void* ptr : {(const void*)freqs, (const void*)positions, (const void*)offsets})
        if (((uintptr_t)ptr & 3u) != 0) return GSD_ERR_MISALIGNED;
    if (p->q_stride % 8 != 0 || (k && p->k_stride % 8 != 0)) return GSD_ERR_MISALIGNED;
    a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.q_out = (uint16_t*)q_out; a.k_out = (uint16_t*)k_out;
    a.r.freqs = freqs; a.r.positions = positions; a.r.offsets = offsets;
    a.B = p->B; a.T = p->T; a.Hq = p->Hq; a.heads = (int)heads;
    a.q_stride = p->q_stride; a.k_stride = p->k_stride;
    return p->D == 128 ? launch_rotary<128>(a, (cudaStream_t)stream) : launch_rotary<64>(a, (cudaStream_t)stream);
}
