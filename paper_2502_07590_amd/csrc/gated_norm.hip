// Gate, residual and modulated norm of rows of n elements, forward and backward.
//
//   u = y, or N(y) (post);  h = a x + gate u;  z = N(h) (1 + scale) + shift
//   N(v) = (v - mu) r, r = 1 / sqrt(mean (v - mu)^2 + eps), mu = mean v (rms: 0);  gate, scale, shift: one row a segment
//
//   w = dz (1 + scale), xh = N(h):  dh = dH + r (w - mean w - xh mean(w xh));  dx = a dh;  v = gate dh
//   dy = v, or r_y (v - mean v - u mean(v u)) (post);  over a segment's rows dgate = sum dh u, dscale = sum dz xh, dshift = sum dz
//
// Bound by memory: a row's elements are read once into registers, LPR lanes to a row, the next row's on their way while one is worked on.
// The backward forms h from x and y once more: as many bytes as reading it, and none of the 8 bits that its rounding leaves.  32768 rows of 2048, bf16:
// 102 to 107 us forward (5.2 TB/s; a copy of 1 GiB: 5.1), 172 and 7 for the sums backward (4.7); 20280 of 1536, fp32, post: 90 (5.5) and 158 (4.7).
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

// What is not there -- a modulation, Y, dH, elements past the row's end -- is held as zeros (a gate that is not there as ones), so that no element asks.
// Past the end that leaves numbers in no sum but dg, of columns that are not written.
template <typename T, int CH, int LPR, int NP>
__global__ __launch_bounds__(LPR < 256 ? 256 : LPR, LPR == 512 ? 2 : NP * CH <= 8 ? 3 : NP * CH <= 16 ? 2 : 1) void gated_bwd_kernel(
    const T *__restrict__ X, const T *__restrict__ Y, const T *__restrict__ gate, const T *__restrict__ scale, const float4 *__restrict__ stats,
    const T *__restrict__ dZ, const T *dH, T *dX, T *__restrict__ dY, float *dgate, float *dscale, float *dshift, float *__restrict__ part, GatedNormArgs a)
{
    typedef Lane<T, CH, LPR, NP> L;
    constexpr int RPB = LPR < 256 ? 256 / LPR : 1;
    constexpr bool kAhead = NP * CH <= (CH == 8 ? 16 : 8);  // the next row's loads under way: its registers would be others' with more elements
    __shared__ float2 red[2][LPR < 256 ? 4 : LPR / 64];
    const Span s = block_rows(a);
    if (s.count <= 0) return;
    const L l(a.n);
    const float inv_n = 1.f / (float)a.n;
    typename L::P xn[NP] = {}, yn[NP] = {}, zn[NP] = {}, hn[NP] = {};
    float gf[NP][CH], mf[NP][CH], dg[NP][CH], ds[NP][CH], dt[NP][CH];
    {
        typename L::P gp[NP] = {}, sp[NP] = {};
        if (gate) l.load(gate + s.seg * a.gate, gp);
        if (scale) l.load(scale + s.seg * a.scale, sp);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            unpack(gp[i], gf[i]);
            unpack(sp[i], mf[i]);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!gate && l.in[i]) gf[i][c] = 1.f;
                dg[i][c] = ds[i][c] = dt[i][c] = 0.f;
            }
        }
    }
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
    if (kAhead && k < s.count) load(base + k);
    for (; k < s.count; k += RPB) {
        const int64_t row = base + k;
        if (!kAhead) load(row);
        typename L::P hp[NP];
        const float mu = stn.x, r = stn.y, mu_y = a.post ? stn.z : 0.f, r_y = a.post ? stn.w : 1.f;
        float u[NP][CH], xh[NP][CH], w[NP][CH], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float x[CH], y[CH], dz[CH];
            unpack(xn[i], x);
            unpack(yn[i], y);
            unpack(zn[i], dz);
            hp[i] = hn[i];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                u[i][c] = (y[c] - mu_y) * r_y;
                xh[i][c] = (fmaf(gf[i][c], u[i][c], a.residual * x[c]) - mu) * r;
                w[i][c] = fmaf(dz[c], mf[i][c], dz[c]);
                dt[i][c] += dz[c];
                ds[i][c] = fmaf(dz[c], xh[i][c], ds[i][c]);
                s1 += w[i][c];
                s2 = fmaf(w[i][c], xh[i][c], s2);
            }
        }
        if (kAhead && k + RPB < s.count) load(row + RPB);  // on its way while this row is worked on
        const float2 sums = row_sums<LPR>(s1, s2, red[turn ^= 1]);
        const float m1 = a.rms ? 0.f : sums.x * inv_n, m2 = sums.y * inv_n;
        float t1 = 0.f, t2 = 0.f;
        T *const dx = dX + row * a.dx;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float dh[CH], o[CH];
            unpack(hp[i], dh);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const float d = fmaf(r, w[i][c] - m1 - xh[i][c] * m2, dh[c]);
                o[c] = a.residual * d;
                dg[i][c] = fmaf(d, u[i][c], dg[i][c]);
                w[i][c] = gf[i][c] * d;
                t1 += w[i][c];
                t2 = fmaf(w[i][c], u[i][c], t2);
            }
            if (l.in[i]) put(dx + l.at(i), o);
        }
        if (Y) {
            float n1 = 0.f, n2 = 0.f;
            if (a.post) {
                const float2 t = row_sums<LPR>(t1, t2, red[turn ^= 1]);
                n1 = a.rms ? 0.f : t.x * inv_n;
                n2 = t.y * inv_n;
            }
            T *const dy = dY + row * a.dy;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float o[CH];
#pragma unroll
                for (int c = 0; c < CH; ++c) o[c] = r_y * (w[i][c] - n1 - u[i][c] * n2);
                if (l.in[i]) put(dy + l.at(i), o);
            }
        }
    }
    if (!dgate && !dscale && !dshift) return;
    // the sums of the block's lane groups, a piece of each lane at a time
    const bool whole = s.len <= a.rows;
    float *const to = part + (whole ? 0 : (part_row(a, s.first) + s.row0 / a.rows) * 3 * a.n);
    float *const to0 = whole ? dgate + s.seg * a.dgate : to, *const to1 = whole ? dscale + s.seg * a.dscale : to + a.n,
          *const to2 = whole ? dshift + s.seg * a.dshift : to + 2 * a.n;
    const bool w0 = dgate, w1 = dscale, w2 = dshift;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!l.in[i]) continue;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (w0) to0[l.at(i) + c] = dg[i][c];
                if (w1) to1[l.at(i) + c] = ds[i][c];
                if (w2) to2[l.at(i) + c] = dt[i][c];
            }
        }
    } else {
        __shared__ float acc[RPB][LPR * CH];
        const int grp = threadIdx.x / LPR;
        auto join = [&](const float (&v)[NP][CH], float *out) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                __syncthreads();
#pragma unroll
                for (int c = 0; c < CH; ++c) acc[grp][l.lane * CH + c] = v[i][c];
                __syncthreads();
                for (int e = threadIdx.x; e < LPR * CH; e += 256) {
                    const int col = i * LPR * CH + e;
                    float x = 0.f;
#pragma unroll
                    for (int g = 0; g < RPB; ++g) x += acc[g][e];
                    if (col < a.n) out[col] = x;
                }
            }
        };
        if (w0) join(dg, to0);
        if (w1) join(ds, to1);
        if (w2) join(dt, to2);
    }
}

// The blocks' sums of one segment: 32 columns a block, eight rows at a time.
__global__ __launch_bounds__(256) void gated_sum_kernel(const float *__restrict__ part, float *dgate, float *dscale, float *dshift, GatedNormArgs a, int col_blocks)
{
    __shared__ float acc[8][33];
    const int seg = blockIdx.x / col_blocks, c = threadIdx.x & 31, g = threadIdx.x >> 5, col = (blockIdx.x - seg * col_blocks) * 32 + c, which = blockIdx.y;
    float *const d = which == 0 ? dgate : which == 1 ? dscale : dshift;
    const int64_t row = which == 0 ? a.dgate : which == 1 ? a.dscale : a.dshift;
    if (!d) return;
    const int first = min(max(a.cu[seg], 0), a.tokens), len = min(max(a.cu[seg + 1], first), a.tokens) - first;
    if (len > 0 && len <= a.rows) return;  // written by its one block
    const int blocks = (len + a.rows - 1) / a.rows;
    float v = 0.f;
    if (col < a.n) {
        const float *const p = part + (part_row(a, first) * 3 + which) * a.n + col;
#pragma unroll 8
        for (int b = g; b < blocks; b += 8) v += p[(int64_t)b * 3 * a.n];
    }
    acc[g][c] = v;
    __syncthreads();
    if (g == 0 && col < a.n) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += acc[i][c];
        d[seg * row + col] = v;
    }
}

// Lanes to a row and pieces to a lane: few elements a lane, a row to a block where a wave would hold more than two pieces.  (A wave to rows of 2048, four
// pieces a lane: the backward's registers leave one wave a SIMD, 32768 rows in bf16 346 us.)  Past two pieces a lane of 256, 512 lanes, for the same
// reason; us, 256 and 512: 20000 rows of 4480 in bf16 352, 224; 1500 of 8192 100, 46; in fp32 of 2560 362, 252; 1500 of 8192 104, 75.
// (Spilled: 19 and 21 registers of bf16 rows past 2048 in pieces of one element, 4 of fp32 rows past 4096.)
NormShape bwd_shape(int n, int ch)
{
    const int pieces = (n + ch - 1) / ch;
    if (ch == 1) {
        for (int np : {1, 4, 8})
            if (pieces <= 64 * np) return {64, np};
        int np = 4;
        while (pieces > 256 * np) np *= 2;
        return {256, np};
    }
    for (int lpr = 8; lpr <= 64; lpr *= 2)
        if (pieces <= lpr) return {lpr, 1};
    if (pieces <= 128) return {64, 2};
    for (int np : {1, 2})
        if (np * ch <= 16 && pieces <= 256 * np) return {256, np};
    return {512, pieces <= 1024 ? 2 : 4};
}
// f(integral constants LPR, NP) for the shape of a row
template <int CH, typename F> dsv_status with_bwd_shape(const NormShape &s, F f)
{
#define DSV_SHAPE(L, N) \
    if (s.lpr == L && s.np == N) return f(std::integral_constant<int, L>{}, std::integral_constant<int, N>{});
    if constexpr (CH == 1) {
        DSV_SHAPE(64, 1) DSV_SHAPE(64, 4) DSV_SHAPE(64, 8) DSV_SHAPE(256, 4) DSV_SHAPE(256, 8) DSV_SHAPE(256, 16) DSV_SHAPE(256, 32)
    } else {
        DSV_SHAPE(8, 1) DSV_SHAPE(16, 1) DSV_SHAPE(32, 1) DSV_SHAPE(64, 1) DSV_SHAPE(64, 2) DSV_SHAPE(256, 1) DSV_SHAPE(256, 2) DSV_SHAPE(512, 2)
        if constexpr (CH == 4) { DSV_SHAPE(512, 4) }
    }
#undef DSV_SHAPE
    return DSV_EUNSUPPORTED;
}

int rows_a_block(int64_t tokens, int lpr, int blocks)
{
    const int rpb = std::max(1, 256 / lpr);
    return (int)std::max<int64_t>(1, (tokens + (int64_t)blocks * rpb - 1) / ((int64_t)blocks * rpb)) * rpb;
}
// Forward: a block goes on to further rows with the modulation in its registers and the next row under way, or there are more blocks.  us, with 2048, 8192
// and 32768 blocks: 17000 rows of 2048 in bf16 49, 54, 54; 64000 of 512 47, 52, 61; 64000 of 2048 210, 185, 192; 17000 of 5120 144, 144, 162;
// in fp32 17000 of 512 24, 23, 23; 17000 of 2048 127, 108, 107; 64000 of 2048 449, 420, 370; 17000 of 8192 576, 513, 389.
int fwd_blocks(int64_t tokens, int n, bool bf16) { return !bf16 ? 32768 : tokens * n >= (3ll << 24) ? 8192 : 2048; }
// Backward: two blocks of 256 a CU, or one of 512, and no more of them than that by the segments' last ones: a CU that takes a third sets the time.  Each
// leaves 3 n floats to sum.  us, 512 blocks and 768 (three a CU fit up to 8 elements a lane): 32768 rows of 2048 in four segments, bf16, forward and
// backward 276, 282 (512 without regard to the segments: 300); backward alone 1500 rows of 2048 24, 29; 20000 111, 119; in fp32 208, 213.
int bwd_rows(int64_t tokens, int n_seg, const NormShape &s)
{
    const int blocks = s.lpr == 512 ? 256 : 512;
    return rows_a_block(tokens, s.lpr, blocks - std::min(n_seg, blocks / 4));
}
int chunk_of(int dtype, bool wide) { return !wide ? 1 : dtype == DSV_BF16 ? 8 : 4; }

template <typename T, int CH>
dsv_status fwd_t(GatedNormArgs a, const GatedNormIn &in, void *Z, void *H, float4 *stats, hipStream_t st)
{
    const NormShape s = norm_shape(a.n, CH);
    a.rows = rows_a_block(a.tokens, s.lpr, fwd_blocks(a.tokens, a.n, std::is_same<T, bf16_t>::value));
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
    const NormShape s = bwd_shape(a.n, CH);
    a.rows = bwd_rows(a.tokens, a.n_seg, s);
    return with_bwd_shape<CH>(s, [&](auto lpr, auto np) {
        if (a.tokens > 0) {
            gated_bwd_kernel<T, CH, decltype(lpr)::value, decltype(np)::value><<<(unsigned)tile_slots(a.tokens, 1, a.rows, a.n_seg), std::max(256, s.lpr), 0, st>>>(
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
size_t gated_bwd_bytes(int64_t tokens, int n, int n_seg, int dtype)
{
    size_t most = 0;
    for (bool wide : {false, true}) {
        const int rows = bwd_rows(tokens, n_seg, bwd_shape(n, chunk_of(dtype, wide)));
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
