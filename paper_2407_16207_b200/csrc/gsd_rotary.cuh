// Rotary positions: what gsd_rotary and gsd_append_kv_paged share.
//
// Of the D columns of a head the first 2 * pairs are rotated, pair i by angle_i = position[axis[i]] * freqs[i].  The work is cut
// into chunks of 16 columns, 8 pairs: two 16-byte pieces of a head that one thread holds, so that a pair is read, turned and written
// in one place and a rotation in place is safe.  The thread's 8 sines and cosines serve all heads it takes.
//
// The angle is formed in turns and reduced in 64 bits: pos * freq / 2 pi, less the nearest whole number.  In 32 bits a
// position of 10^6 would leave an angle 2^-4 off.  What is left, at most half a turn, goes to sincospif (2 ulp).
#pragma once
#include "gsd_internal.cuh"

namespace gsd {

struct Rotation {
    const float* freqs;
    const int32_t* positions;    // [axes][B][T], or nullptr: the caller says the position
    const int32_t* offsets;      // [B], or nullptr
    int chunks;                  // chunks that are rotated, pairs / 8; 0: none
    int axes;
    int neighbours;              // pairs are columns 2 i and 2 i + 1, else i and pairs + i
    uint32_t axis_bits[4];       // two bits for each pair
};

// The rotation of the caller's parameters; false if they are not those of one for heads of D columns.
inline bool rotation_of(const gsd_rotation* r, int D, Rotation* out) {
    if (r->pairs < 8 || r->pairs % 8 != 0 || 2 * r->pairs > D || r->axes < 1 || r->axes > GSD_ROTARY_MAX_AXES ||
        (r->layout != GSD_ROTARY_HALVES && r->layout != GSD_ROTARY_NEIGHBOURS))
        return false;
    out->chunks = r->pairs / 8;
    out->axes = r->axes;
    out->neighbours = r->layout == GSD_ROTARY_NEIGHBOURS;
    for (uint32_t& w : out->axis_bits) w = 0;
    for (int i = 0; i < r->pairs; ++i) {
        if (r->axis[i] >= r->axes) return false;
        out->axis_bits[i >> 4] |= (uint32_t)r->axis[i] << (2 * (i & 15));
    }
    return true;
}

#ifdef __CUDACC__
// The two 16-byte pieces of chunk j of a head, as element offsets.
__device__ __forceinline__ int2 chunk_columns(const Rotation& r, int j) {
    if (j < r.chunks && !r.neighbours) return make_int2(8 * j, 8 * (r.chunks + j));
    return make_int2(16 * j, 16 * j + 8);
}

// The positions of a token on every axis.
struct TokenPos {
    long long at[GSD_ROTARY_MAX_AXES];
};
__device__ __forceinline__ TokenPos token_pos(const Rotation& r, int b, int t, int B, int T, int place) {
    TokenPos p;
    const long long off = r.offsets ? r.offsets[b] : 0;
#pragma unroll
    for (int a = 0; a < GSD_ROTARY_MAX_AXES; ++a) {
        if (a == 0 || a < r.axes) p.at[a] = (r.positions ? r.positions[((size_t)a * B + b) * T + t] : place) + off;
        else p.at[a] = 0;
    }
    return p;
}

// (cos, sin) of the 8 pairs of chunk j.
__device__ __forceinline__ void chunk_angles(const Rotation& r, int j, const TokenPos& pos, float2 (&cs)[8]) {
    const uint32_t bits = r.axis_bits[j >> 1] >> (16 * (j & 1));
    const float4 f0 = make_float4(r.freqs[8 * j], r.freqs[8 * j + 1], r.freqs[8 * j + 2], r.freqs[8 * j + 3]);
    const float4 f1 = make_float4(r.freqs[8 * j + 4], r.freqs[8 * j + 5], r.freqs[8 * j + 6], r.freqs[8 * j + 7]);
    const float f[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int a = (bits >> (2 * i)) & 3;
        const long long at = a == 0 ? pos.at[0] : a == 1 ? pos.at[1] : a == 2 ? pos.at[2] : pos.at[3];
        double turns = (double)at * ((double)f[i] * 0.15915494309189533577);     // 1 / (2 pi)
        turns -= rint(turns);
        sincospif((float)(2.0 * turns), &cs[i].y, &cs[i].x);
    }
}

__device__ __forceinline__ uint32_t rotary_pack(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// The two pieces of a rotated chunk, turned.
__device__ __forceinline__ void turn_chunk(bool neighbours, const float2 (&cs)[8], uint4& a, uint4& b) {
    uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
    if (neighbours) {
        auto turn = [](uint32_t w, const float2& c) {
            const float u = bf16_lo(w), v = bf16_hi(w);
            return rotary_pack(u * c.x - v * c.y, u * c.y + v * c.x);
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = turn(x[i], cs[i]);
            y[i] = turn(y[i], cs[4 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 c0 = cs[2 * i], c1 = cs[2 * i + 1];
            const float u0 = bf16_lo(x[i]), u1 = bf16_hi(x[i]), v0 = bf16_lo(y[i]), v1 = bf16_hi(y[i]);
            x[i] = rotary_pack(u0 * c0.x - v0 * c0.y, u1 * c1.x - v1 * c1.y);
            y[i] = rotary_pack(u0 * c0.y + v0 * c0.x, u1 * c1.y + v1 * c1.x);
        }
    }
    a = make_uint4(x[0], x[1], x[2], x[3]);
    b = make_uint4(y[0], y[1], y[2], y[3]);
}
#endif

}  // namespace gsd
