// Gate, residual and modulated norm of rows of n elements, forward and backward.
//
//   u = y, or N(y) (post);  h = a x + gate u;  z = N(h) (1 + scale) + shift
//   N(v) = (v - mu) r, r = 1 / sqrt(mean (v - mu)^2 + eps), mu = mean v (rms: 0);  gate, scale, shift: one row a segment
//
//   w = dz (1 + scale), xh = N(h):  dh = dH + r (w - mean w - xh mean(w xh));  dx = a dh;  v = gate dh
//   dy = v, or r_y (v - mean v - u mean(v u)) (post);  over a segment's rows dgate = sum dh u, dscale = sum dz xh, dshift = sum dz
//
// Bound by memory: a row's elements are read once into registers, LPR lanes to a row, the next row's on their way while one is worked on.
// The backward forms h from x and y once more: as many bytes as reading it, and none of the 8 bits that its rounding leaves.
#include <algorithm>

#include "gated_norm.h"
#include "norm_rows.h"
#include "sequences.h"

namespace dsv {
namespace {

// A block's rows: some of one segment's.
struct Span {
    int seg, first, count, row0, len;  // first: the segment's first row of all; row0: the block's first row of the segment
};
__device__ __forceinline__ Span block_rows(const GatedNormArgs &a)
{
    Span s;
    const int slot = blockIdx.x;
    s.seg = __builtin_amdgcn_readfirstlane(find_sequence(a.cu, a.n_seg, a.tokens, 1, a.rows, slot));
    s.first = min(max(a.cu[s.seg], 0), a.tokens);
    s.len = min(max(a.cu[s.seg + 1], s.first), a.tokens) - s.first;
    const int64_t row0 = (int64_t)(slot - first_slot(a.cu[s.seg], a.tokens, 1, a.rows, s.seg)) * a.rows;
    s.row0 = (int)min((int64_t)s.len, max((int64_t)0, row0));
    s.count = row0 < 0 ? 0 : min(a.rows, s.len - s.row0);
    return s;
}

template <typename T, int CH, int LPR, int NP> struct Lane {
    typedef Piece<T, CH> P;
    int lane;
    bool in[NP];
    __device__ __forceinline__ explicit Lane(int n) : lane(threadIdx.x % LPR)
    {
#pragma unroll
        for (int i = 0; i < NP; ++i) in[i] = (lane + i * LPR) * CH < n;
    }
    __device__ __forceinline__ int at(int i) const { return (lane + i * LPR) * CH; }
    __device__ __forceinline__ void load(const T *row, P (&p)[NP]) const
    {
#pragma unroll
        for (int i = 0; i < NP; ++i)
            if (in[i]) p[i] = *reinterpret_cast<const P *>(row + at(i));
    }
};

// Mean and 1 / deviation of a row in registers; mean taken off f.  turn: LDS of the next sum, never that of the one before (a barrier lies between
// a wave's reads of one sum and another's writes of the next but one).
template <int CH, int LPR, int NP>
__device__ __forceinline__ float2 normed(float (&f)[NP][CH], const bool (&in)[NP], float inv_n, float eps, bool rms, float2 (*red)[4], int &turn)
{
    float s = 0.f, mu = 0.f;
    if (!rms) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int c = 0; c < CH; ++c) s += in[i] ? f[i][c] : 0.f;
        mu = row_sums<LPR>(s, 0.f, red[turn ^= 1]).x * inv_n;
        s = 0.f;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            f[i][c] -= mu;
            s += in[i] ? f[i][c] * f[i][c] : 0.f;
        }
    const float r = 1.f / sqrtf(fmaf(row_sums<LPR>(s, 0.f, red[turn ^= 1]).x, inv_n, eps));
    return make_float2(mu, r);
}

template <typename T, int CH, int LPR, int NP>
__global__ __launch_bounds__(256) void gated_fwd_kernel(const T *X, const T *__restrict__ Y, const T *__restrict__ gate, const T *__restrict__ scale,
                                                        const T *__restrict__ shift, T *__restrict__ Z, T *H, float4 *__restrict__ stats, GatedNormArgs a)
{
    typedef Lane<T, CH, LPR, NP> L;
    constexpr int RPB = 256 / LPR;
    __shared__ float2 red[2][4];
    const Span s = block_rows(a);
    if (s.count <= 0) return;
    const L l(a.n);
    const float inv_n = 1.f / (float)a.n;
    typename L::P gp[NP], sp[NP], tp[NP], xp[NP], yp[NP];
    if (gate) l.load(gate + s.seg * a.gate, gp);
    if (scale) l.load(scale + s.seg * a.scale, sp);
    if (shift) l.load(shift + s.seg * a.shift, tp);
    const int64_t base = s.first + s.row0;
    int k = threadIdx.x / LPR, turn = 0;
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        l.load(X + row * a.x, xp);
        if (Y) l.load(Y + row * a.y, yp);
    };
    if (k < s.count) load(base + k);
    for (; k < s.count; k += RPB) {
        const int64_t row = base + k;
        float f[NP][CH];
        float2 ny = make_float2(0.f, 0.f);
        if (Y) {
            float u[NP][CH];
#pragma unroll
            for (int i = 0; i < NP; ++i) unpack(yp[i], u[i]);
            if (a.post) ny = normed<CH, LPR, NP>(u, l.in, inv_n, a.eps, a.rms, red, turn);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float g[CH], x[CH];
                if (gate) unpack(gp[i], g);
                unpack(xp[i], x);
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    float v = u[i][c];
                    if (a.post) v *= ny.y;
                    if (gate) v *= g[c];
                    f[i][c] = fmaf(a.residual, x[c], v);
                }
                if (l.in[i]) put(H + row * a.h + l.at(i), f[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                unpack(xp[i], f[i]);
#pragma unroll
                for (int c = 0; c < CH; ++c) f[i][c] *= a.residual;
            }
        }
        if (k + RPB < s.count) load(row + RPB);  // on its way while this row is finished
        const float2 nh = normed<CH, LPR, NP>(f, l.in, inv_n, a.eps, a.rms, red, turn);
        T *const z = Z + row * a.z;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!l.in[i]) continue;
            float o[CH], m[CH], t[CH];
            if (scale) unpack(sp[i], m);
            if (shift) unpack(tp[i], t);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                o[c] = f[i][c] * nh.y;
                if (scale) o[c] = fmaf(o[c], m[c], o[c]);
                if (shift) o[c] += t[c];
            }
            put(z + l.at(i), o);
        }
        if (l.lane == 0) stats[row] = make_float4(nh.x, nh.y, ny.x, ny.y);
    }
}

// A segment of several blocks leaves its sums in rows of `part` [..][3][n], 2 floor(first row / rows a block) onwards: no two such segments share one.
__device__ __forceinline__ int64_t part_row(const GatedNormArgs &a, int first) { return 2 * (int64_t)(first / a.rows); }

template <typename T, int CH, int LPR, int NP>
__global__ __launch_bounds__(256) void gated_bwd_kernel(const T *__restrict__ X, const T *__restrict__ Y, const T *__restrict__ gate, const T *__restrict__ scale,
                                                        const float4 *__restrict__ stats, const T *__restrict__ dZ, const T *dH, T *dX,
                                                        T *__restrict__ dY, float *dgate, float *dscale, float *dshift, float *__restrict__ part, GatedNormArgs a)
{
    typedef Lane<T, CH, LPR, NP> L;
    constexpr int RPB = 256 / LPR;
    __shared__ float2 red[2][4];
    const Span s = block_rows(a);
    if (s.count <= 0) return;
    const L l(a.n);
    const float inv_n = 1.f / (float)a.n;
    typename L::P gp[NP], sp[NP], xn[NP], yn[NP], zn[NP], hn[NP];
    if (gate) l.load(gate + s.seg * a.gate, gp);
    if (scale) l.load(scale + s.seg * a.scale, sp);
    float dg[NP][CH], ds[NP][CH], dt[NP][CH];
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int c = 0; c < CH; ++c) dg[i][c] = ds[i][c] = dt[i][c] = 0.f;
    const int64_t base = s.first + s.row0;
    int k = threadIdx.x / LPR, turn = 0;
    float4 stn = make_float4(0.f, 0.f, 0.f, 0.f);
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        l.load(X + row * a.x, xn);
        if (Y) l.load(Y + row * a.y, yn);
        l.load(dZ + row * a.dz, zn);
        if (dH) l.load(dH + row * a.dh, hn);
        stn = stats[row];
    };
    if (k < s.count) load(base + k);
    for (; k < s.count; k += RPB) {
        const int64_t row = base + k;
        typename L::P hp[NP];
        const float4 st = stn;  // mean and 1 / deviation of h, of y
        float u[NP][CH], xh[NP][CH], w[NP][CH], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float x[CH], y[CH], dz[CH], g[CH], m[CH];
            unpack(xn[i], x);
            if (Y) unpack(yn[i], y);
            unpack(zn[i], dz);
            hp[i] = hn[i];
            if (gate) unpack(gp[i], g);
            if (scale) unpack(sp[i], m);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float h = a.residual * x[c];
                u[i][c] = 0.f;
                if (Y) {
                    u[i][c] = a.post ? (y[c] - st.z) * st.w : y[c];
                    h += gate ? g[c] * u[i][c] : u[i][c];
                }
                xh[i][c] = l.in[i] ? (h - st.x) * st.y : 0.f;
                const float d = l.in[i] ? dz[c] : 0.f;
                w[i][c] = scale && l.in[i] ? fmaf(d, m[c], d) : d;
                dt[i][c] += d;
                ds[i][c] = fmaf(d, xh[i][c], ds[i][c]);
                s1 += w[i][c];
                s2 = fmaf(w[i][c], xh[i][c], s2);
            }
        }
        if (k + RPB < s.count) load(row + RPB);  // on its way while this row is worked on
        const float2 sums = row_sums<LPR>(s1, s2, red[turn ^= 1]);
        const float m1 = a.rms ? 0.f : sums.x * inv_n, m2 = sums.y * inv_n;
        float t1 = 0.f, t2 = 0.f;
        T *const dx = dX + row * a.dx;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float g[CH], dh[CH], o[CH];
            if (gate) unpack(gp[i], g);
            if (dH) unpack(hp[i], dh);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float d = st.y * (w[i][c] - m1 - xh[i][c] * m2);
                if (dH) d += dh[c];
                d = l.in[i] ? d : 0.f;
                o[c] = a.residual * d;
                dg[i][c] = fmaf(d, l.in[i] ? u[i][c] : 0.f, dg[i][c]);
                const float v = gate && l.in[i] ? g[c] * d : d;
                w[i][c] = v;
                if (a.post) {
                    t1 += v;
                    t2 = fmaf(v, l.in[i] ? u[i][c] : 0.f, t2);
                }
            }
            if (l.in[i]) put(dx + l.at(i), o);
        }
        if (Y) {
            float n1 = 0.f, n2 = 0.f, r = 1.f;
            if (a.post) {
                const float2 t = row_sums<LPR>(t1, t2, red[turn ^= 1]);
                n1 = a.rms ? 0.f : t.x * inv_n;
                n2 = t.y * inv_n;
                r = st.w;
            }
            T *const dy = dY + row * a.dy;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                if (!l.in[i]) continue;
                float o[CH];
#pragma unroll
                for (int c = 0; c < CH; ++c) o[c] = a.post ? r * (w[i][c] - n1 - u[i][c] * n2) : w[i][c];
                put(dy + l.at(i), o);
            }
        }
    }
    if (!dgate && !dscale && !dshift) return;
    // the sums of the block's lane groups, a piece of each lane at a time
    const bool whole = s.len <= a.rows;
    float *const to = part + (whole ? 0 : (part_row(a, s.first) + s.row0 / a.rows) * 3 * a.n);
    auto out = [&](int which, int col, float v) __attribute__((always_inline)) {
        if (!whole) {
            to[(int64_t)which * a.n + col] = v;
            return;
        }
        float *const d = which == 0 ? dgate : which == 1 ? dscale : dshift;
        if (d) d[s.seg * (which == 0 ? a.dgate : which == 1 ? a.dscale : a.dshift) + col] = v;
    };
    if constexpr (RPB == 1) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!l.in[i]) continue;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                out(0, l.at(i) + c, dg[i][c]);
                out(1, l.at(i) + c, ds[i][c]);
                out(2, l.at(i) + c, dt[i][c]);
            }
        }
    } else {
        __shared__ float acc[RPB][3][LPR * CH];
        const int grp = threadIdx.x / LPR;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                acc[grp][0][l.lane * CH + c] = dg[i][c];
                acc[grp][1][l.lane * CH + c] = ds[i][c];
                acc[grp][2][l.lane * CH + c] = dt[i][c];
            }
            __syncthreads();
            for (int e = threadIdx.x; e < 3 * LPR * CH; e += 256) {
                const int which = e / (LPR * CH), off = e - which * (LPR * CH), col = i * LPR * CH + off;
                float v = 0.f;
#pragma unroll
                for (int g = 0; g < RPB; ++g) v += acc[g][which][off];
                if (col < a.n) out(which, col, v);
            }
        }
    }
}

// The blocks' sums of one segment: 32 columns a block, eight rows at a time.
__global__ __launch_bounds__(256) void gated_sum_kernel(const float *__restrict__ part, float *dgate, float *dscale, float *dshift, GatedNormArgs a, int col_blocks)
{
    __shared__ float acc[8][33];
    const int seg = blockIdx.x / col_blocks, c = threadIdx.x & 31, g = threadIdx.x >> 5, col = (blockIdx.x - seg * col_blocks) * 32 + c, which = blockIdx.y;
    float *const d = which == 0 ? dgate : which == 1 ? dscale : dshift;
    if (!d) return;
    const int first = min(max(a.cu[seg], 0), a.tokens), len = min(max(a.cu[seg + 1], first), a.tokens) - first;
    if (len > 0 && len <= a.rows) return;  // written by its one block
    const int blocks = (len + a.rows - 1) / a.rows;
    float v = 0.f;
    if (col < a.n) {
        const float *const p = part + (part_row(a, first) * 3 + which) * a.n + col;
#pragma unroll 4
        for (int b = g; b < blocks; b += 8) v += p[(int64_t)b * 3 * a.n];
    }
    acc[g][c] = v;
    __syncthreads();
    if (g == 0 && col < a.n) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += acc[i][c];
        d[seg * (which == 0 ? a.dgate : which == 1 ? a.dscale : a.dshift) + col] = v;
    }
}

int rows_a_block(int64_t tokens, int lpr, int blocks)
{
    const int rpb = 256 / lpr;
    return (int)std::max<int64_t>(1, (tokens + (int64_t)blocks * rpb - 1) / ((int64_t)blocks * rpb)) * rpb;
}
constexpr int kFwdBlocks = 2048;
constexpr int kBwdBlocks = 512;
int bwd_rows(int64_t tokens, int lpr) { return rows_a_block(tokens, lpr, kBwdBlocks); }
int chunk_of(int dtype, bool wide) { return !wide ? 1 : dtype == DSV_BF16 ? 8 : 4; }

template <typename T, int CH>
dsv_status fwd_t(GatedNormArgs a, const GatedNormIn &in, void *Z, void *H, float4 *stats, hipStream_t st)
{
    const NormShape s = norm_shape(a.n, CH);
    a.rows = rows_a_block(a.tokens, s.lpr, kFwdBlocks);
    return with_shape<CH>(s, [&](auto lpr, auto np) {
        gated_fwd_kernel<T, CH, decltype(lpr)::value, decltype(np)::value><<<(unsigned)tile_slots(a.tokens, 1, a.rows, a.n_seg), 256, 0, st>>>(
            static_cast<const T *>(in.X), static_cast<const T *>(in.Y), static_cast<const T *>(in.gate), static_cast<const T *>(in.scale),
            static_cast<const T *>(in.shift), static_cast<T *>(Z), static_cast<T *>(H), stats, a);
        DSV_LAUNCH_CHECK();
        return DSV_OK;
    });
}
template <typename T, int CH>
dsv_status bwd_t(GatedNormArgs a, const GatedNormIn &in, const float4 *stats, const void *dZ, const void *dH, void *dX, void *dY, float *dgate, float *dscale,
                 float *dshift, float *part, hipStream_t st)
{
    const NormShape s = norm_shape(a.n, CH);
    a.rows = bwd_rows(a.tokens, s.lpr);
    return with_shape<CH>(s, [&](auto lpr, auto np) {
        if (a.tokens > 0) {
            gated_bwd_kernel<T, CH, decltype(lpr)::value, decltype(np)::value><<<(unsigned)tile_slots(a.tokens, 1, a.rows, a.n_seg), 256, 0, st>>>(
                static_cast<const T *>(in.X), static_cast<const T *>(in.Y), static_cast<const T *>(in.gate), static_cast<const T *>(in.scale), stats,
                static_cast<const T *>(dZ), static_cast<const T *>(dH), static_cast<T *>(dX), static_cast<T *>(dY), dgate, dscale, dshift, part, a);
            DSV_LAUNCH_CHECK();
        }
        if (dgate || dscale || dshift) {
            const int col_blocks = (a.n + 31) / 32;
            gated_sum_kernel<<<dim3((unsigned)(a.n_seg * col_blocks), 3), 256, 0, st>>>(part, dgate, dscale, dshift, a, col_blocks);
            DSV_LAUNCH_CHECK();
        }
        return DSV_OK;
    });
}
}  // namespace

dsv_status launch_gated_fwd(GatedNormArgs a, int dtype, bool wide, const GatedNormIn &in, void *Z, void *H, float4 *stats, hipStream_t st)
{
    if (dtype == DSV_BF16) return wide ? fwd_t<bf16_t, 8>(a, in, Z, H, stats, st) : fwd_t<bf16_t, 1>(a, in, Z, H, stats, st);
    return wide ? fwd_t<float, 4>(a, in, Z, H, stats, st) : fwd_t<float, 1>(a, in, Z, H, stats, st);
}

// the pointers do not enter: as many rows as either alignment leaves
size_t gated_bwd_bytes(int64_t tokens, int n, int dtype)
{
    size_t most = 0;
    for (bool wide : {false, true}) {
        const int rows = bwd_rows(tokens, norm_shape(n, chunk_of(dtype, wide)).lpr);
        // one segment of more than `rows` at least; the last one's begins at row 2 floor(first / rows) and has ceil(len / rows)
        most = std::max(most, tokens > rows ? (size_t)(2 * (tokens / rows) + 2) * 3 * n * 4 : (size_t)0);
    }
    return align_up(most, 256);
}

dsv_status launch_gated_bwd(GatedNormArgs a, int dtype, bool wide, const GatedNormIn &in, const float4 *stats, const void *dZ, const void *dH, void *dX, void *dY,
                            float *dgate, float *dscale, float *dshift, float *part, hipStream_t st)
{
    if (dtype == DSV_BF16)
        return wide ? bwd_t<bf16_t, 8>(a, in, stats, dZ, dH, dX, dY, dgate, dscale, dshift, part, st)
                    : bwd_t<bf16_t, 1>(a, in, stats, dZ, dH, dX, dY, dgate, dscale, dshift, part, st);
    return wide ? bwd_t<float, 4>(a, in, stats, dZ, dH, dX, dY, dgate, dscale, dshift, part, st)
                : bwd_t<float, 1>(a, in, stats, dZ, dH, dX, dY, dgate, dscale, dshift, part, st);
}

}  // namespace dsv
