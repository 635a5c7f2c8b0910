// Layer norm of rows of n elements, forward and backward.
//
//   mu = mean x, r = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) r, y = xh gamma + beta
//   g = dy gamma;  dx = r (g - mean g - xh mean(g xh));  dgamma = sum over rows of dy xh, dbeta = sum over rows of dy
//
// Bound by memory: a row is read once into registers, LPR lanes to a row (8 .. 64 of a wave, or the whole block), CH elements a load, while
// the row before it is worked on.  Of 64 M elements, bytes read and written over time: forward 5.0 .. 6.3 TB/s, backward with the sums of
// dgamma and dbeta 4.0 .. 5.6 TB/s (a copy of 1 GiB: 5.1).  Without the read ahead the backward pass had 3.4 TB/s at n = 2048.
// The variance is formed from the differences in registers, not from sums of squares.
#include <algorithm>

#include "norm.h"
#include "norm_rows.h"

namespace dsv {
namespace {

// Rows first, first + gridDim * RPB, ... of a lane group, as token and head without a division a row.
template <int LPR> struct RowWalk {
    static constexpr int RPB = 256 / LPR;
    int head, step_head;
    int64_t id, step, tok, step_tok;  // past the last token by up to a step
    __device__ __forceinline__ RowWalk(const NormArgs &a)
    {
        id = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR;
        step = (int64_t)gridDim.x * RPB;
        tok = id / a.heads;
        head = (int)(id - tok * a.heads);
        step_tok = step / a.heads;
        step_head = (int)(step - step_tok * a.heads);
    }
    __device__ __forceinline__ void next(const NormArgs &a)
    {
        id += step;
        tok += step_tok;
        head += step_head;
        if (head >= a.heads) {
            head -= a.heads;
            ++tok;
        }
    }
};

template <typename T, int CH, int LPR, int NP>
__global__ __launch_bounds__(256) void norm_fwd_kernel(const T *__restrict__ X, const T *__restrict__ gamma, const T *__restrict__ beta, T *__restrict__ Y,
                                                       float *__restrict__ mean, float *__restrict__ rstd, NormArgs a)
{
    __shared__ float2 red[2][4];
    const int lane = threadIdx.x % LPR;
    const float inv_n = 1.f / (float)a.n;
    Piece<T, CH> gp[NP], bp[NP];
    bool in[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int e = (lane + i * LPR) * CH;
        in[i] = e < a.n;
        if (gamma && in[i]) gp[i] = *reinterpret_cast<const Piece<T, CH> *>(gamma + e);
        if (beta && in[i]) bp[i] = *reinterpret_cast<const Piece<T, CH> *>(beta + e);
    }
    Piece<T, CH> xp[NP];
    auto load = [&](const RowWalk<LPR> &w) __attribute__((always_inline)) {
        const T *x = X + w.tok * a.x_row + w.head * a.x_head;
#pragma unroll
        for (int i = 0; i < NP; ++i)
            if (in[i]) xp[i] = *reinterpret_cast<const Piece<T, CH> *>(x + (lane + i * LPR) * CH);
    };
    RowWalk<LPR> w(a);
    if (w.tok < a.tokens) load(w);
    while (w.tok < a.tokens) {
        float f[NP][CH], s = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            unpack(xp[i], f[i]);
#pragma unroll
            for (int c = 0; c < CH; ++c) s += in[i] ? f[i][c] : 0.f;
        }
        const float mu = row_sums<LPR>(s, 0.f, red[0]).x * inv_n;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                f[i][c] -= mu;
                s += in[i] ? f[i][c] * f[i][c] : 0.f;
            }
        RowWalk<LPR> next = w;
        next.next(a);
        if (next.tok < a.tokens) load(next);  // on its way while this row is finished
        const float r = 1.f / sqrtf(fmaf(row_sums<LPR>(s, 0.f, red[1]).x, inv_n, a.eps));
        T *y = Y + w.tok * a.y_row + w.head * a.y_head;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!in[i]) continue;
            float o[CH], g[CH], b[CH];
            if (gamma) unpack(gp[i], g);
            if (beta) unpack(bp[i], b);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                o[c] = f[i][c] * r;
                if (gamma) o[c] *= g[c];
                if (beta) o[c] += b[c];
            }
            put(y + (lane + i * LPR) * CH, o);
        }
        if (lane == 0) {
            mean[w.id] = mu;
            rstd[w.id] = r;
        }
        w = next;
    }
}

// part [gridDim.x][2][n]: the block's sums of dy xh and of dy (null: not wanted)
template <typename T, int CH, int LPR, int NP>
__global__ __launch_bounds__(256) void norm_bwd_kernel(const T *__restrict__ X, const T *__restrict__ gamma, const float *__restrict__ mean,
                                                       const float *__restrict__ rstd, const T *__restrict__ dY, T *__restrict__ dX, float *__restrict__ part, NormArgs a)
{
    __shared__ float2 red[2][4];
    const int lane = threadIdx.x % LPR;
    const float inv_n = 1.f / (float)a.n;
    Piece<T, CH> gp[NP];
    bool in[NP];
    float dg[NP][CH], db[NP][CH];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int e = (lane + i * LPR) * CH;
        in[i] = e < a.n;
        if (gamma && in[i]) gp[i] = *reinterpret_cast<const Piece<T, CH> *>(gamma + e);
#pragma unroll
        for (int c = 0; c < CH; ++c) dg[i][c] = db[i][c] = 0.f;
    }
    int turn = 0;
    Piece<T, CH> xn[NP], yn[NP];
    float mun = 0.f, rn = 0.f;
    auto load = [&](const RowWalk<LPR> &w) __attribute__((always_inline)) {
        const T *x = X + w.tok * a.x_row + w.head * a.x_head, *dy = dY + w.tok * a.dy_row + w.head * a.dy_head;
#pragma unroll
        for (int i = 0; i < NP; ++i)
            if (in[i]) {
                xn[i] = *reinterpret_cast<const Piece<T, CH> *>(x + (lane + i * LPR) * CH);
                yn[i] = *reinterpret_cast<const Piece<T, CH> *>(dy + (lane + i * LPR) * CH);
            }
        mun = mean[w.id];
        rn = rstd[w.id];
    };
    RowWalk<LPR> w(a);
    if (w.tok < a.tokens) load(w);
    while (w.tok < a.tokens) {
        Piece<T, CH> xp[NP], yp[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            xp[i] = xn[i];
            yp[i] = yn[i];
        }
        const float mu = mun, r = rn;
        RowWalk<LPR> next = w;
        next.next(a);
        if (next.tok < a.tokens) load(next);  // on its way while this row is worked on
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float xf[CH], yf[CH], g[CH];
            unpack(xp[i], xf);
            unpack(yp[i], yf);
            if (gamma) unpack(gp[i], g);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const float xh = in[i] ? (xf[c] - mu) * r : 0.f, y = in[i] ? yf[c] : 0.f, v = gamma ? y * (in[i] ? g[c] : 0.f) : y;
                s1 += v;
                s2 = fmaf(v, xh, s2);
                dg[i][c] = fmaf(y, xh, dg[i][c]);
                db[i][c] += y;
            }
        }
        const float2 s = row_sums<LPR>(s1, s2, red[turn]);
        turn ^= 1;
        const float m1 = s.x * inv_n, m2 = s.y * inv_n;
        T *dx = dX + w.tok * a.dx_row + w.head * a.dx_head;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!in[i]) continue;
            float xf[CH], yf[CH], g[CH], o[CH];
            unpack(xp[i], xf);
            unpack(yp[i], yf);
            if (gamma) unpack(gp[i], g);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const float xh = (xf[c] - mu) * r, v = gamma ? yf[c] * g[c] : yf[c];
                o[c] = r * (v - m1 - xh * m2);
            }
            put(dx + (lane + i * LPR) * CH, o);
        }
        w = next;
    }
    if (!part) return;
    // the block's lane groups joined, a piece of each lane at a time: LPR * CH columns
    constexpr int RPB = 256 / LPR;
    float *const out = part + (int64_t)blockIdx.x * 2 * a.n;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!in[i]) continue;
            const int e = (lane + i * LPR) * CH;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                out[e + c] = dg[i][c];
                out[a.n + e + c] = db[i][c];
            }
        }
    } else {
        __shared__ float acc[RPB][2][LPR * CH];
        const int grp = threadIdx.x / LPR;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                acc[grp][0][lane * CH + c] = dg[i][c];
                acc[grp][1][lane * CH + c] = db[i][c];
            }
            __syncthreads();
            for (int k = threadIdx.x; k < 2 * LPR * CH; k += 256) {
                const int which = k / (LPR * CH), e = k - which * (LPR * CH), col = i * LPR * CH + e;
                float v = 0.f;
#pragma unroll
                for (int g = 0; g < RPB; ++g) v += acc[g][which][e];
                if (col < a.n) out[which * a.n + col] = v;
            }
        }
    }
}

// Columns of part summed over the blocks: eight columns a block, 32 rows at a time.
__global__ __launch_bounds__(256) void norm_sum_kernel(const float *__restrict__ part, int blocks, int n, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    __shared__ float acc[32][9];
    const int c = threadIdx.x & 7, g = threadIdx.x >> 3, col = blockIdx.x * 8 + c;
    float v = 0.f;
    if (col < 2 * n) {
#pragma unroll 8
        for (int b = g; b < blocks; b += 32) v += part[(int64_t)b * 2 * n + col];
    }
    acc[g][c] = v;
    __syncthreads();
    if (g == 0 && col < 2 * n) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) v += acc[i][c];
        (col < n ? dgamma[col] : dbeta[col - n]) = v;
    }
}

int64_t norm_row_blocks(const NormArgs &a, int lpr) { return ((int64_t)a.tokens * a.heads + 256 / lpr - 1) / (256 / lpr); }
// Blocks of the two kernels, which then walk over the rows, each row's loads under way while the one before is worked on.  Backward: the more
// elements a lane has, the more registers and the fewer blocks run at once, and each block leaves 2 n floats to sum.  64 M elements, us with
// the sum, in 256, 512 and 768 blocks: bf16, 8 elements a lane (n 128) 128, 87, 83; 16 (n 1024) 88, 77, 93; 32 (n 2048) 83, 94, 100.
constexpr int kFwdBlocks = 4096;
int bwd_blocks(int per_lane) { return per_lane <= 8 ? 768 : per_lane <= 16 ? 512 : 256; }

template <typename T, int CH, int LPR, int NP>
dsv_status fwd_shape(const NormArgs &a, const T *X, const T *gamma, const T *beta, T *Y, float *mean, float *rstd, hipStream_t st)
{
    norm_fwd_kernel<T, CH, LPR, NP><<<(unsigned)std::min<int64_t>(norm_row_blocks(a, LPR), kFwdBlocks), 256, 0, st>>>(X, gamma, beta, Y, mean, rstd, a);
    DSV_LAUNCH_CHECK();
    return DSV_OK;
}
template <typename T, int CH, int LPR, int NP>
dsv_status bwd_shape(const NormArgs &a, const T *X, const T *gamma, const float *mean, const float *rstd, const T *dY, T *dX, float *dgamma, float *dbeta,
                     float *part, hipStream_t st)
{
    const int blocks = (int)std::min<int64_t>(norm_row_blocks(a, LPR), bwd_blocks(CH * NP));
    if (blocks > 0) {
        norm_bwd_kernel<T, CH, LPR, NP><<<blocks, 256, 0, st>>>(X, gamma, mean, rstd, dY, dX, part, a);
        DSV_LAUNCH_CHECK();
    }
    if (dgamma) {
        norm_sum_kernel<<<(2 * a.n + 7) / 8, 256, 0, st>>>(part, blocks, a.n, dgamma, dbeta);
        DSV_LAUNCH_CHECK();
    }
    return DSV_OK;
}

template <typename T, int CH>
dsv_status fwd_t(const NormArgs &a, const void *X, const void *gamma, const void *beta, void *Y, float *mean, float *rstd, hipStream_t st)
{
    return with_shape<CH>(norm_shape(a.n, CH), [&](auto lpr, auto np) {
        return fwd_shape<T, CH, decltype(lpr)::value, decltype(np)::value>(a, static_cast<const T *>(X), static_cast<const T *>(gamma), static_cast<const T *>(beta),
                                                                          static_cast<T *>(Y), mean, rstd, st);
    });
}
template <typename T, int CH>
dsv_status bwd_t(const NormArgs &a, const void *X, const void *gamma, const float *mean, const float *rstd, const void *dY, void *dX, float *dgamma, float *dbeta,
                 float *part, hipStream_t st)
{
    return with_shape<CH>(norm_shape(a.n, CH), [&](auto lpr, auto np) {
        return bwd_shape<T, CH, decltype(lpr)::value, decltype(np)::value>(a, static_cast<const T *>(X), static_cast<const T *>(gamma), mean, rstd,
                                                                          static_cast<const T *>(dY), static_cast<T *>(dX), dgamma, dbeta, part, st);
    });
}
int chunk_of(int dtype, bool wide) { return !wide ? 1 : dtype == DSV_BF16 ? 8 : 4; }
}  // namespace

dsv_status launch_norm_fwd(const NormArgs &a, int dtype, bool wide, const void *X, const void *gamma, const void *beta, void *Y, float *mean, float *rstd,
                           hipStream_t st)
{
    if (dtype == DSV_BF16)
        return wide ? fwd_t<bf16_t, 8>(a, X, gamma, beta, Y, mean, rstd, st) : fwd_t<bf16_t, 1>(a, X, gamma, beta, Y, mean, rstd, st);
    return wide ? fwd_t<float, 4>(a, X, gamma, beta, Y, mean, rstd, st) : fwd_t<float, 1>(a, X, gamma, beta, Y, mean, rstd, st);
}

int norm_bwd_blocks(const NormArgs &a, int dtype, bool wide)
{
    const int ch = chunk_of(dtype, wide);
    const NormShape s = norm_shape(a.n, ch);
    return (int)std::min<int64_t>(norm_row_blocks(a, s.lpr), bwd_blocks(ch * s.np));
}

dsv_status launch_norm_bwd(const NormArgs &a, int dtype, bool wide, const void *X, const void *gamma, const float *mean, const float *rstd, const void *dY,
                           void *dX, float *dgamma, float *dbeta, float *part, hipStream_t st)
{
    if (dtype == DSV_BF16)
        return wide ? bwd_t<bf16_t, 8>(a, X, gamma, mean, rstd, dY, dX, dgamma, dbeta, part, st)
                    : bwd_t<bf16_t, 1>(a, X, gamma, mean, rstd, dY, dX, dgamma, dbeta, part, st);
    return wide ? bwd_t<float, 4>(a, X, gamma, mean, rstd, dY, dX, dgamma, dbeta, part, st)
                : bwd_t<float, 1>(a, X, gamma, mean, rstd, dY, dX, dgamma, dbeta, part, st);
}

}  // namespace dsv
