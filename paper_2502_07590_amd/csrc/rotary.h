// Rotary positions: pairs of channels turned by angles that grow with the token's coordinates.  Shared by rotary.hip and cache_append.hip.
#pragma once

#include "common.h"
#include "norm_rows.h"

namespace dsv {

struct TurnArgs {
    const int32_t *pos;   // [tokens][axes]
    const double *freq;   // [pairs of all coordinates], radians a position
    int32_t axes, total;  // coordinates; pairs
    int32_t end0, end1;   // pairs before the second, the third coordinate's
    int32_t layout;
    float gain;
};

// (cos, sin) of pair i's angle at a token, times the gain.  The product is formed and brought within half a turn in 64 bits: in
// 32, an angle of 10^6 radians is off by 0.06.  What rounding that to 32 bits leaves, up to 9e-8 radians, turns the result once more (its square is
// nothing): without it cos and sin are 3.3e-8 off in the mean square, with it 1.9e-8, their own rounding 1.5e-8; in no more time.
__device__ __forceinline__ float2 turn_of(const TurnArgs &a, const int (&pos)[3], int i)
{
    if (i >= a.total) return make_float2(0.f, 0.f);  // none: not read
    const int p = i < a.end0 ? pos[0] : i < a.end1 ? pos[1] : pos[2];
    double t = (double)p * a.freq[i] * 0.15915494309189535;
    t -= rint(t);
    const float near = (float)t, off = (float)((t - (double)near) * 6.283185307179586);
    float s, c;
    sincospif(2.f * near, &s, &c);
    return make_float2(fmaf(-s, off, c) * a.gain, fmaf(c, off, s) * a.gain);
}
__device__ __forceinline__ void read_position(const TurnArgs &a, int64_t token, int (&pos)[3])
{
#pragma unroll
    for (int x = 0; x < 3; ++x) pos[x] = x < a.axes ? a.pos[token * a.axes + x] : 0;
}

// Where pair i's channels lie.
__device__ __forceinline__ void pair_channels(const TurnArgs &a, int i, int &lo, int &hi)
{
    if (a.layout == DSV_TURN_INTERLEAVED) {
        lo = 2 * i;
        hi = lo + 1;
    } else if (a.layout == DSV_TURN_HALVES) {
        lo = i;
        hi = i + a.total;
    } else {
        const int begin = i < a.end0 ? 0 : i < a.end1 ? a.end0 : a.end1, end = i < a.end0 ? a.end0 : i < a.end1 ? a.end1 : a.total;
        lo = i + begin;
        hi = lo + end - begin;
    }
}

// The other way round: the pair of channel c, whether c is its second, and its other channel.  c is one of those that are turned.
__device__ __forceinline__ void pair_of(const TurnArgs &a, int c, int &pair, bool &second, int &other)
{
    if (a.layout == DSV_TURN_INTERLEAVED) {
        pair = c >> 1;
        second = c & 1;
        other = c ^ 1;
        return;
    }
    int begin = 0, end = a.total;
    if (a.layout == DSV_TURN_AXIS_HALVES) {
        begin = c < 2 * a.end0 ? 0 : c < 2 * a.end1 ? a.end0 : a.end1;
        end = c < 2 * a.end0 ? a.end0 : c < 2 * a.end1 ? a.end1 : a.total;
    }
    const int n = end - begin;
    second = c - 2 * begin >= n;
    pair = c - begin - (second ? n : 0);
    other = second ? c - n : c + n;
}

// Sixteen channels of a row: two times eight side by side, in eight pairs (2 i, 2 i + 1 of them, or i and 8 + i) or in none.
struct Sixteen {
    int first, second;  // channels
    int pair;           // the first of the eight, or -1
};
// For rows of whole sixteens whose halves' pairs come in eights (`eights` below).
__device__ __forceinline__ Sixteen sixteen_of(const TurnArgs &a, int job)
{
    Sixteen s;
    if (a.layout == DSV_TURN_INTERLEAVED || 8 * job >= a.total) {
        s.first = 16 * job;
        s.second = s.first + 8;
        s.pair = 8 * job < a.total ? 8 * job : -1;
    } else {
        s.pair = 8 * job;
        pair_channels(a, s.pair, s.first, s.second);
    }
    return s;
}
__host__ __forceinline__ bool eights(int layout, int axes, const int32_t *pairs, int d)
{
    if (d % 16) return false;
    if (layout == DSV_TURN_INTERLEAVED) return true;
    int total = 0;
    for (int i = 0; i < axes; ++i) {
        if (layout == DSV_TURN_AXIS_HALVES && pairs[i] % 8) return false;
        total += pairs[i];
    }
    return total % 8 == 0;
}

// The sixteen values, loaded and stored in 16-byte pieces.
__device__ __forceinline__ void load8(const bf16_t *p, float (&f)[8]) { unpack(*reinterpret_cast<const Piece<bf16_t, 8> *>(p), f); }
__device__ __forceinline__ void load8(const float *p, float (&f)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&f)[8]) { put(p, f); }
__device__ __forceinline__ void store8(float *p, const float (&f)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
template <bool BACK> __device__ __forceinline__ void turn(float &x, float &y, float2 t)
{
    const float a = x, b = y, s = BACK ? -t.y : t.y;
    x = a * t.x - b * s;
    y = a * s + b * t.x;
}
// left: how many of the eight are there; the others' channels stay as they are, bit for bit
template <bool BACK> __device__ __forceinline__ void turn_sixteen(bool interleaved, int left, const float2 (&t)[8], float (&f)[8], float (&g)[8])
{
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < left) turn<BACK>(f[2 * i], f[2 * i + 1], t[i]);
            if (4 + i < left) turn<BACK>(g[2 * i], g[2 * i + 1], t[4 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn<BACK>(f[i], g[i], t[i]);
    }
}

struct RotaryArgs {
    TurnArgs t;
    int32_t tokens, heads, d;
    int64_t x_row, x_head, y_row, y_head;  // elements
};
dsv_status launch_rotary(const RotaryArgs &a, int dtype, bool wide, bool back, const void *X, void *Y, hipStream_t st);

}  // namespace dsv
