// Rows spread over lanes, as the kernels of norms hold them.
#pragma once

#include <type_traits>

#include "common.h"

namespace dsv {

// A lane's share of a row: pieces lane, lane + LPR, ... of CH elements.
template <typename T, int CH> struct Piece;
template <> struct Piece<bf16_t, 8> { uint4 w; };
template <> struct Piece<float, 4> { uint4 w; };
template <> struct Piece<bf16_t, 1> { uint16_t w; };
template <> struct Piece<float, 1> { uint32_t w; };
__device__ __forceinline__ void unpack(const Piece<bf16_t, 8> &p, float (&f)[8])
{
    const uint32_t w[4] = {p.w.x, p.w.y, p.w.z, p.w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(const Piece<float, 4> &p, float (&f)[4])
{
    f[0] = __uint_as_float(p.w.x); f[1] = __uint_as_float(p.w.y); f[2] = __uint_as_float(p.w.z); f[3] = __uint_as_float(p.w.w);
}
__device__ __forceinline__ void unpack(const Piece<bf16_t, 1> &p, float (&f)[1]) { f[0] = __uint_as_float((uint32_t)p.w << 16); }
__device__ __forceinline__ void unpack(const Piece<float, 1> &p, float (&f)[1]) { f[0] = __uint_as_float(p.w); }

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const f32x2_t f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}
__device__ __forceinline__ void put(bf16_t *p, const float (&f)[8])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}
__device__ __forceinline__ void put(float *p, const float (&f)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]); }
__device__ __forceinline__ void put(bf16_t *p, const float (&f)[1]) { *p = (bf16_t)(pack2(f[0], 0.f) & 0xFFFFu); }
__device__ __forceinline__ void put(float *p, const float (&f)[1]) { *p = f[0]; }

// Sums of two values over the LPR lanes of a row.  256 and more: the whole block, through LDS.
template <int LPR> __device__ __forceinline__ float2 row_sums(float a, float b, float2 *red)
{
    constexpr int W = LPR < 64 ? LPR : 64;
#pragma unroll
    for (int s = W / 2; s > 0; s >>= 1) {
        a += __shfl_xor(a, s);
        b += __shfl_xor(b, s);
    }
    if constexpr (LPR >= 256) {
        constexpr int N = LPR / 64;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) red[wave] = make_float2(a, b);
        __syncthreads();
        float2 v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = red[i];
#pragma unroll
        for (int s = 1; s < N; s *= 2)
#pragma unroll
            for (int i = 0; i < N; i += 2 * s) v[i] = make_float2(v[i].x + v[i + s].x, v[i].y + v[i + s].y);
        a = v[0].x;
        b = v[0].y;
    }
    return make_float2(a, b);
}

// Lanes to a row and pieces to a lane: a row within a wave, as few lanes as hold it, where that takes at most 32 elements a lane (16
// one-element pieces), else a row to a block.
struct NormShape {
    int lpr, np;
};
inline constexpr int max_wave_np(int ch) { return ch == 1 ? 16 : 32 / ch; }
inline NormShape norm_shape(int n, int ch)
{
    const int pieces = (n + ch - 1) / ch;
    for (int lpr = 8; lpr <= 64; lpr *= 2)
        if (pieces <= lpr) return {lpr, 1};
    for (int np : {2, 3, 4, 6, 8, 16})
        if (np <= max_wave_np(ch) && pieces <= 64 * np) return {64, np};
    int np = 2;
    while (pieces > 256 * np) np *= 2;
    return {256, np};
}

// f(integral constants LPR, NP) for the shape of a row
template <int CH, typename F> dsv_status with_shape(const NormShape &s, F f)
{
#define DSV_SHAPE(L, N) \
    if (s.lpr == L && s.np == N) return f(std::integral_constant<int, L>{}, std::integral_constant<int, N>{});
    DSV_SHAPE(8, 1) DSV_SHAPE(16, 1) DSV_SHAPE(32, 1) DSV_SHAPE(64, 1) DSV_SHAPE(64, 2) DSV_SHAPE(64, 3) DSV_SHAPE(64, 4)
    if constexpr (CH < 8) { DSV_SHAPE(64, 6) DSV_SHAPE(64, 8) }
    if constexpr (CH == 1) { DSV_SHAPE(64, 16) }
    if constexpr (CH == 8) { DSV_SHAPE(256, 2) }
    if constexpr (CH > 1) { DSV_SHAPE(256, 4) }
    if constexpr (CH < 8) { DSV_SHAPE(256, 8) }
    if constexpr (CH == 1) { DSV_SHAPE(256, 16) DSV_SHAPE(256, 32) }
#undef DSV_SHAPE
    return DSV_EUNSUPPORTED;
}

}  // namespace dsv
