// Rotary positions of rows [tokens, heads, d].
//
//   pair i of coordinate p:  t = p freq_i;  lo' = gain (lo cos t - hi sin t), hi' = gain (lo sin t + hi cos t);  back: t -> -t (the transpose)
//
// Bound by memory: 16-byte pieces in and out; the sines are formed once for all heads that a lane walks.  32768 tokens, 32 heads of 128
// inside rows of 48, bf16: 115 us, 4.7 TB/s, where a copy of 1 GiB has 5.1; 1024 tokens, four heads of 64, fp32: 4.8 us.
#include <algorithm>

#include "rotary.h"

namespace dsv {
namespace {

// Lanes take sixteen channels each of one token and of heads h, h + H, ...; the job's places run along channels, then along the axis whose
// stride is smaller.
template <typename T, bool BACK>
__global__ __launch_bounds__(256) void rotary_kernel(const T *X, T *Y, RotaryArgs a, int H, bool tokens_inner)
{
    const int per = a.d >> 4;
    const uint32_t e = blockIdx.x * 256u + threadIdx.x, rest = e / (uint32_t)per;
    const int job = (int)(e - rest * per);
    uint32_t token, h;
    if (tokens_inner) {
        h = rest / (uint32_t)a.tokens;
        token = rest - h * a.tokens;
    } else {
        token = rest / (uint32_t)H;
        h = rest - token * H;
    }
    if (token >= (uint32_t)a.tokens || h >= (uint32_t)H) return;
    const Sixteen s = sixteen_of(a.t, job);
    if (s.pair < 0 && X == Y) return;  // in place: the rest of a row is there
    float2 t[8];
    if (s.pair >= 0) {
        int pos[3];
        read_position(a.t, token, pos);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = turn_of(a.t, pos, s.pair + i);
    }
    const T *x = X + token * a.x_row;
    T *y = Y + token * a.y_row;
    for (int k = (int)h; k < a.heads; k += H) {
        float f[8], g[8];
        load8(x + k * a.x_head + s.first, f);
        load8(x + k * a.x_head + s.second, g);
        if (s.pair >= 0) turn_sixteen<BACK>(a.t.layout == DSV_TURN_INTERLEAVED, a.t.total - s.pair, t, f, g);
        store8(y + k * a.y_head + s.first, f);
        store8(y + k * a.y_head + s.second, g);
    }
}

// Any alignment, any number of pairs: a lane takes one pair, or one channel that is not turned.
template <typename T, bool BACK> __global__ __launch_bounds__(256) void rotary_pairs_kernel(const T *X, T *Y, RotaryArgs a)
{
    const int per = a.d - a.t.total;
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, token = e / per;
    const int job = (int)(e - token * per);
    if (token >= a.tokens) return;
    const T *x = X + token * a.x_row;
    T *y = Y + token * a.y_row;
    if (job >= a.t.total) {
        const int c = job + a.t.total;
        for (int k = 0; k < a.heads && X != Y; ++k) y[k * a.y_head + c] = x[k * a.x_head + c];
        return;
    }
    int pos[3], lo, hi;
    read_position(a.t, token, pos);
    const float2 t = turn_of(a.t, pos, job);
    pair_channels(a.t, job, lo, hi);
    for (int k = 0; k < a.heads; ++k) {
        float f[1] = {to_f32(x[k * a.x_head + lo])}, g[1] = {to_f32(x[k * a.x_head + hi])};
        turn<BACK>(f[0], g[0], t);
        put(y + k * a.y_head + lo, f);
        put(y + k * a.y_head + hi, g);
    }
}

template <typename T, bool BACK> dsv_status launch_t(const RotaryArgs &a, bool wide, const T *X, T *Y, hipStream_t st)
{
    if (wide) {
        // H lanes share a token's heads: four, more where tokens are few.  32768 tokens, 32 heads of 128, forward and backward, us: 4 227, 1 262, 32 286
        // (one pair a lane, below, 255).
        const int64_t lanes = (int64_t)a.tokens * (a.d / 16);
        const int H = (int)std::min<int64_t>(a.heads, std::max<int64_t>(4, ((1 << 18) + lanes - 1) / lanes));
        const int64_t blocks = (lanes * H + 255) / 256;
        rotary_kernel<T, BACK><<<(unsigned)blocks, 256, 0, st>>>(X, Y, a, H, a.heads > 1 && a.x_head > a.x_row);
    } else {
        rotary_pairs_kernel<T, BACK><<<(unsigned)(((int64_t)a.tokens * (a.d - a.t.total) + 255) / 256), 256, 0, st>>>(X, Y, a);
    }
    DSV_LAUNCH_CHECK();
    return DSV_OK;
}
template <typename T> dsv_status launch_d(const RotaryArgs &a, bool wide, bool back, const void *X, void *Y, hipStream_t st)
{
    const T *x = static_cast<const T *>(X);
    T *y = static_cast<T *>(Y);
    return back ? launch_t<T, true>(a, wide, x, y, st) : launch_t<T, false>(a, wide, x, y, st);
}
}  // namespace

dsv_status launch_rotary(const RotaryArgs &a, int dtype, bool wide, bool back, const void *X, void *Y, hipStream_t st)
{
    return dtype == DSV_BF16 ? launch_d<bf16_t>(a, wide, back, X, Y, st) : launch_d<float>(a, wide, back, X, Y, st);
}

}  // namespace dsv
