// gsd_rotary: rotary positions of Q and K rows, with one position axis (text) or several (images, video).
//
//   angle_i = (positions[axis[i]][b][t] + offsets[b]) * freqs[i],   (x, y) -> (x cos - y sin, x sin + y cos)
//
// A CTA has a run of (token, head) places, Q's heads and K's of a token counted in one line, and forms the sines and cosines of its
// tokens in shared memory while its first pieces come (gsd_rotary.cuh).  Bound by DRAM for large calls: 8 x 256 tokens of 64 + 8 heads of 128 13.3 us for 75 MB, 88 % of the rate
// of a copy; single tokens 2.4 us.
#include "gsd_rotary.cuh"

namespace gsd {
namespace {

constexpr int kThreads = kRotaryThreads;

struct RotaryArgs {
    const uint16_t *q, *k;
    uint16_t *q_out, *k_out;
    Rotation r;
    int B, T, Hq, heads;         // heads of q and k together
    int places;                  // tokens * heads
    int batches;                 // of a CTA
    long long q_stride, k_stride;
};

template <int D, int kBatch>
__global__ void __launch_bounds__(kThreads, kRotaryBlocks) rotary_kernel(const __grid_constant__ RotaryArgs p) {
    constexpr int CH = D / 16, SLOTS = kThreads / CH;
    __shared__ AngleTable<D> s_angles[rotary_tokens(D)];
    let_successor_start();
    wait_for_predecessor();
    const int j = threadIdx.x % CH, slot = threadIdx.x / CH;
    const int begin = blockIdx.x * (SLOTS * p.batches), end = min(begin + SLOTS * p.batches, p.places);
    const int tok0 = begin / p.heads;
    const int2 col = chunk_columns(p.r, j);
    const bool turned = j < p.r.chunks;
    for (int at0 = begin; at0 < end; at0 += SLOTS * kBatch) {
        uint4 x[kBatch][2];
        int tok[kBatch], head[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int at = min(at0 + i * SLOTS + slot, end - 1);        // (the last place again, for those behind it)
            tok[i] = at / p.heads;
            head[i] = at - tok[i] * p.heads;
            const uint16_t* src = head[i] < p.Hq ? p.q + tok[i] * p.q_stride + head[i] * D : p.k + tok[i] * p.k_stride + (head[i] - p.Hq) * D;
            x[i][0] = *reinterpret_cast<const uint4*>(src + col.x);
            x[i][1] = *reinterpret_cast<const uint4*>(src + col.y);
        }
        if (at0 == begin) {
            form_angles(p.r, s_angles, (end - 1) / p.heads - tok0 + 1, p.B, p.T, [&](int m, int& b, int& t, int& place) {
                b = (tok0 + m) / p.T;
                t = tok0 + m - b * p.T;
                place = 0;
            });
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (at0 + i * SLOTS + slot >= end) continue;
            if (turned) turn_chunk<D>(p.r.neighbours != 0, s_angles[tok[i] - tok0], j, x[i][0], x[i][1]);
            uint16_t* dst = head[i] < p.Hq ? p.q_out + ((size_t)tok[i] * p.Hq + head[i]) * D
                                           : p.k_out + ((size_t)tok[i] * (p.heads - p.Hq) + head[i] - p.Hq) * D;
            *reinterpret_cast<uint4*>(dst + col.x) = x[i][0];
            *reinterpret_cast<uint4*>(dst + col.y) = x[i][1];
        }
    }
}

template <int D>
int launch_rotary(RotaryArgs& a, cudaStream_t stream) {
    DeviceInfo di;
    if (device_info(&di) != 0) return GSD_ERR_CUDA;
    a.batches = rotary_batches(a.places, a.heads, D, di.sm_count);
    const int run = kThreads / (D / 16) * a.batches;
    const dim3 grid((unsigned)((a.places + (long long)run - 1) / run));
    if (a.batches == 1) GSD_CUDA_TRY(launch_dependent(rotary_kernel<D, 1>, grid, dim3(kThreads), 0, stream, a));
    else GSD_CUDA_TRY(launch_dependent(rotary_kernel<D, 2>, grid, dim3(kThreads), 0, stream, a));
    return GSD_OK;
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
    if (heads > (1 << 20) || (long long)p->B * p->T > 0x7F000000ll / heads) return GSD_ERR_BAD_SHAPE;
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
    a.B = p->B; a.T = p->T; a.Hq = p->Hq; a.heads = (int)heads; a.places = (int)(heads * p->B * p->T);
    a.q_stride = p->q_stride; a.k_stride = p->k_stride;
    return p->D == 128 ? launch_rotary<128>(a, (cudaStream_t)stream) : launch_rotary<64>(a, (cudaStream_t)stream);
}
