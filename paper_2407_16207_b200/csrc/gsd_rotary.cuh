// Rotary positions: what gsd_rotary and gsd_append_kv_paged share.
//
// Of the D columns of a head the first 2 * pairs are rotated, pair i by angle_i = position[axis[i]] * freqs[i].  The work is cut
// into chunks of 16 columns, 8 pairs: two 16-byte pieces of a head that one thread holds, so that a pair is read, turned and written
// in one place and a rotation in place is safe.  A CTA has a run of (token, head) places; it forms the sines and cosines of its
// tokens once, in shared memory, for all heads.
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

constexpr int kRotaryThreads = 256, kRotaryBlocks = 4;

// Places (token, head) of a CTA: kRotaryThreads / (D / 16) at a time, `batches` times.  More of them share their tokens' angles, as
// long as every SM has four CTAs; and a CTA has at most rotary_tokens(D) tokens.  A thread has two of them on their way, four CTAs an
// SM (us; 8 x 256 nodes of 64 + 8 heads and 8 x 3000 nodes of 16 + 4 heads of 64: so 12.6 and 7.8; four on their way and
// eight batches, three CTAs an SM, 15.5 and 9.7; one and two, six CTAs 15.6 and 9.1; two and four, six CTAs, spilling, 16.0 and 11.8).
__host__ __device__ constexpr int rotary_tokens(int D) { return kRotaryThreads / (D / 16) + 2; }
inline int rotary_batches(long long places, int heads, int D, int sm_count) {
    const int slots = kRotaryThreads / (D / 16);
    int n = 1;
    while (n < 4 && places > 4ll * sm_count * slots * n && 2 * n * slots / heads + 2 <= rotary_tokens(D)) n *= 2;
    return n;
}

#ifdef __CUDACC__
// The two 16-byte pieces of chunk j of a head, as element offsets.
__device__ __forceinline__ int2 chunk_columns(const Rotation& r, int j) {
    if (j < r.chunks && !r.neighbours) return make_int2(8 * j, 8 * (r.chunks + j));
    return make_int2(16 * j, 16 * j + 8);
}

// Sines and cosines of a token: [quarter of a chunk][chunk] of (cos, sin) of two pairs, so that the threads of a token's chunks
// read without conflicts.
template <int D>
struct AngleTable {
    float4 at[4][D / 16];
    __device__ __forceinline__ float2& pair(int i) { return reinterpret_cast<float2*>(&at[(i & 7) >> 1][i >> 3])[i & 1]; }
};

// The angles of `n` tokens, by the whole CTA: token(m, b, t, place) says which the m-th is; its position is `place` where there are
// no positions.  A thread has one pair of every few tokens.
template <int D, class Token>
__device__ __forceinline__ void form_angles(const Rotation& r, AngleTable<D>* angles, int n, int B, int T, Token token) {
    constexpr int PAIRS = D / 2, STEP = kRotaryThreads / PAIRS;
    const int i = threadIdx.x % PAIRS;
    if (i >= r.chunks * 8) return;
    const int32_t* positions = r.positions + (r.positions ? (size_t)((r.axis_bits[i >> 4] >> (2 * (i & 15))) & 3) * B * T : 0);
    const double turns_per = (double)r.freqs[i] * 0.15915494309189533577;          // 1 / (2 pi)
#pragma unroll 4
    for (int m = threadIdx.x / PAIRS; m < n; m += STEP) {
        int b, t, place;
        token(m, b, t, place);
        const long long pos = (long long)(r.positions ? positions[(size_t)b * T + t] : place) + (r.offsets ? r.offsets[b] : 0);
        double turns = (double)pos * turns_per;
        turns -= rint(turns);
        float2 cs;
        sincospif((float)(2.0 * turns), &cs.y, &cs.x);
        angles[m].pair(i) = cs;
    }
}

__device__ __forceinline__ uint32_t rotary_pack(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// (x, y) turned.  The order of the roundings is fixed, so that a row gets the same bits wherever it is turned.
__device__ __forceinline__ float turned_x(float x, float y, float c, float s) { return __fmaf_rn(x, c, -__fmul_rn(y, s)); }
__device__ __forceinline__ float turned_y(float x, float y, float c, float s) { return __fmaf_rn(x, s, __fmul_rn(y, c)); }

// The two pieces of a rotated chunk j, turned.
template <int D>
__device__ __forceinline__ void turn_chunk(bool neighbours, const AngleTable<D>& angles, int j, uint4& a, uint4& b) {
    const float4 c0 = angles.at[0][j], c1 = angles.at[1][j], c2 = angles.at[2][j], c3 = angles.at[3][j];
    if (neighbours) {
        auto turn = [](uint32_t w, float c, float s) {
            const float u = bf16_lo(w), v = bf16_hi(w);
            return rotary_pack(turned_x(u, v, c, s), turned_y(u, v, c, s));
        };
        a = make_uint4(turn(a.x, c0.x, c0.y), turn(a.y, c0.z, c0.w), turn(a.z, c1.x, c1.y), turn(a.w, c1.z, c1.w));
        b = make_uint4(turn(b.x, c2.x, c2.y), turn(b.y, c2.z, c2.w), turn(b.z, c3.x, c3.y), turn(b.w, c3.z, c3.w));
    } else {
        auto turn = [](uint32_t& x, uint32_t& y, const float4& c) {
            const float u0 = bf16_lo(x), u1 = bf16_hi(x), v0 = bf16_lo(y), v1 = bf16_hi(y);
            x = rotary_pack(turned_x(u0, v0, c.x, c.y), turned_x(u1, v1, c.z, c.w));
            y = rotary_pack(turned_y(u0, v0, c.x, c.y), turned_y(u1, v1, c.z, c.w));
        };
        turn(a.x, b.x, c0);
        turn(a.y, b.y, c1);
        turn(a.z, b.z, c2);
        turn(a.w, b.w, c3);
    }
}
#endif

}  // namespace gsd
