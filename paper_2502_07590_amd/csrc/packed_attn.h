// Attention over packed sequences: what its kernels share (packed_fwd.hip, packed_bwd.hip).
//
// Sequence i holds query tokens cu_q[i] .. cu_q[i+1] - 1 and key tokens cu_k[i] .. cu_k[i+1] - 1.  The `group` query heads that read one
// K/V head are rows of the same tile: row = query * group + head of the group.  A single query of a decoding step then still gives a tile
// `group` rows, and the key-major sums of the backward run over the shared heads by themselves.
#pragma once

#include <type_traits>
#include <utility>

#include "stage2_core.h"

namespace dsv {

constexpr float kNegInf = -__builtin_inff();

// A descriptor as the kernels read it; strides in bytes.
struct PackedArgs {
    const int32_t *cu_q, *cu_k;
    int32_t n_seq, total_q, total_k, max_q, max_k, Hq, Hkv, group;
    uint32_t magic;   // row / group = umulhi(row, magic) for group > 1: magic = floor(2^32 / group) + 1, rows below 2^32 / group
    int32_t causal;
    float scale;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
    int64_t do_row, do_head, dq_row, dq_head, dk_row, dk_head, dv_row, dv_head;
    int32_t splits, chunk;  // the long axis in `splits` pieces of `chunk` rows (0: in one)
};

__device__ __forceinline__ int row_token(const PackedArgs &a, int row) { return a.group == 1 ? row : (int)__umulhi((uint32_t)row, a.magic); }

// One sequence, its ends forced into the tensors: nothing an entry of cu_q or cu_k can say leads out of them.
struct Sequence {
    int q0, k0, nq, nk;
};
__device__ __forceinline__ Sequence read_sequence(const PackedArgs &a, int i)
{
    Sequence s;
    s.q0 = min(max(a.cu_q[i], 0), a.total_q);
    s.k0 = min(max(a.cu_k[i], 0), a.total_k);
    s.nq = min(min(max(a.cu_q[i + 1], s.q0), a.total_q) - s.q0, a.max_q);
    s.nk = min(min(max(a.cu_k[i + 1], s.k0), a.total_k) - s.k0, a.max_k);
    return s;
}

// Pieces of a.chunk keys that query token t of a sequence sees something of.
__device__ __forceinline__ int pieces_seen(const PackedArgs &a, const Sequence &s, int t)
{
    const int seen = a.causal ? min(s.nk, t + s.nk - s.nq + 1) : s.nk;
    return seen > 0 ? (seen + a.chunk - 1) / a.chunk : 0;
}

// Tiles of ROWS rows are numbered without a sum over the sequences before: sequence i's begin at floor(cu[i] * mul / ROWS) + i, which leaves
// ceil(length / ROWS) places at least.  The owner of a place is the last sequence that begins at or before it; 64 candidates a step.
// ROWS = 0: the tokens themselves, no place left empty (the owner of a token).
__device__ __forceinline__ int first_slot(int cu, int total, int mul, int rows, int i)
{
    const int at = min(max(cu, 0), total) * mul;
    return rows ? (int)((uint32_t)at / (uint32_t)rows) + i : at;
}
__device__ __forceinline__ int find_sequence(const int32_t *__restrict__ cu, int n_seq, int total, int mul, int rows, int slot)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n_seq;  // lo begins at or before the slot, hi after it
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, at = lo + (lane + 1) * step;
        const bool before = at < hi && first_slot(cu[at], total, mul, rows, at) <= slot;
        lo += __popcll(__ballot(before)) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}
__host__ __device__ __forceinline__ int64_t tile_slots(int64_t total, int mul, int rows, int n_seq) { return total * mul / rows + n_seq; }

// A tile of rows in LDS, row after row.  Piece p (16 bytes) of row r lies at place p ^ turn(r) of the row, so that what one cycle of the 64
// banks serves lies in different ones: 16 bytes of 16 consecutive rows; for the transposing reads 64 bytes of four rows (bf16); 128 bytes of two rows
// four apart (fp32, element by element).  (With bits of turn that let the halves of a transposing read meet, those took twice as long: a third
// of all LDS cycles of the forward.)
template <typename T, int D> struct RowTile {
    static constexpr int RB = D * (int)sizeof(T), PIECES = RB / 16;
    __device__ __forceinline__ static int turn(int r)
    {
        if constexpr (sizeof(T) == 4) return (((r >> 2) & 1) << 3) | ((r & 3) << 1) | ((r >> 3) & 1);
        else if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
        else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);  // two rows to 256 bytes
    }
    __device__ __forceinline__ static int at(int r, int p) { return r * RB + ((p ^ turn(r)) << 4); }
};

// The loads of one wave for tiles of ROWS rows that WAVES waves bring together, directly into LDS, a kilobyte an instruction.  A lane's
// place in a tile is one offset plus what all lanes add; rows past the end repeat the last one.
template <typename T, int D, int ROWS, int WAVES> struct RowLoads {
    typedef RowTile<T, D> RT;
    static constexpr int N = ROWS * RT::RB / 1024 / WAVES, RPC = 1024 / RT::RB, STEP = WAVES * RPC;  // rows from a load to the next
    static constexpr int NV = STEP % 16 ? 2 : 1;  // turn() has a period of 16 rows
    static_assert(N * WAVES * 1024 == ROWS * RT::RB && (NV == 1 || STEP == 8), "every kilobyte has its wave");
    uint32_t off[NV], piece[NV], step_b;
    int wave;
    __device__ __forceinline__ int row(int i) const { return i * STEP + wave * RPC + (int)(threadIdx.x & 63) / RT::PIECES; }
    __device__ __forceinline__ void set(int wave_, int64_t row_b)  // for keys()
    {
        wave = wave_;
        step_b = (uint32_t)STEP * (uint32_t)row_b;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            piece[v] = (uint32_t)(((int)(threadIdx.x & 63) % RT::PIECES) ^ RT::turn(row(v))) << 4;
            off[v] = (uint32_t)row(0) * (uint32_t)row_b + piece[v];
        }
    }
    __device__ __forceinline__ void set(int wave_, int64_t row_b, const PackedArgs &a, int64_t head_b)  // for rows()
    {
        set(wave_, row_b);
        if (a.group == 1) return;
        step_b = STEP % a.group == 0 ? (uint32_t)(STEP / a.group) * (uint32_t)row_b : 0u;
        const int tok = row_token(a, row(0));
#pragma unroll
        for (int v = 0; v < NV; ++v) off[v] = (uint32_t)tok * (uint32_t)row_b + (uint32_t)(row(0) - tok * a.group) * (uint32_t)head_b + piece[v];
    }
    __device__ __forceinline__ void send(const unsigned char *base, const uint32_t (&at)[N], unsigned char *lds) const
    {
        // by a buffer of all 32-bit offsets: as global loads, which the compiler takes for ones that may read LDS too, they would make every wait for
        // an LDS read one for all of them
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(base), 0, -1, 0x00027000);
#pragma unroll
        for (int i = 0; i < N; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(lds + (i * WAVES + wave) * 1024), 16, (int)at[i], 0, 0, 0);
    }
    // loads step_b apart, none behind the row at `last`
    __device__ __forceinline__ void plain(uint32_t last, uint32_t (&at)[N]) const
    {
        uint32_t o[NV], p[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {  // hidden from the compiler, which would keep all N places in registers that the products need
            o[v] = off[v];
            p[v] = piece[v];
            asm volatile("" : "+v"(o[v]), "+v"(p[v]));
        }
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] = min(o[i % NV] + (uint32_t)i * step_b, last + p[i % NV]);
    }
    // rows k0 .. of n that lie row_b apart
    __device__ __forceinline__ void keys(const unsigned char *first, int64_t row_b, int k0, int n, unsigned char *lds) const
    {
        uint32_t at[N];
        plain((uint32_t)(min(n - k0, ROWS) - 1) * (uint32_t)row_b, at);
        send(first + (int64_t)k0 * row_b, at, lds);
    }
    // rows r0 .. of n, row = token * group + head
    __device__ __forceinline__ void rows(const PackedArgs &a, const unsigned char *first, int64_t row_b, int64_t head_b, int r0, int n, unsigned char *lds) const
    {
        uint32_t at[N];
        const int tok0 = row_token(a, r0);
        if (a.group == 1) {
            plain((uint32_t)(min(n - r0, ROWS) - 1) * (uint32_t)row_b, at);
        } else if (step_b && n - r0 >= ROWS) {  // whole tokens from a load to the next (the divisions and products below: a third of a tile's time)
            uint32_t o[NV];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                o[v] = off[v];
                asm volatile("" : "+v"(o[v]));
            }
#pragma unroll
            for (int i = 0; i < N; ++i) at[i] = o[i % NV] + (uint32_t)i * step_b;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int rho = min(r0 + row(i), n - 1), tok = row_token(a, rho);
                at[i] = (uint32_t)(tok - tok0) * (uint32_t)row_b + (uint32_t)(rho - tok * a.group) * (uint32_t)head_b + piece[i % NV];
            }
        }
        send(first + (int64_t)tok0 * row_b, at, lds);
    }
};

// Operands of the products.  Every product is one of 32 x 32 with the tile's rows (or channels) as A and the wave's own 32 rows as B; a
// lane holds column lane % 32 and, of each eight rows, the four of its half: rows 8 (i / 4) + 4 (lane / 32) + i % 4.
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { bf16x8_t v; };
template <> struct Frag<float> { floatx4_t v; };

__device__ __forceinline__ floatx16_t product(const Frag<bf16_t> &a, const Frag<bf16_t> &b, const floatx16_t &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
// 16 bytes are four channels: half 0 brings channels 0 .. 3 of eight, half 1 channels 4 .. 7; step i contracts over channels i and 4 + i
__device__ __forceinline__ floatx16_t product(const Frag<float> &a, const Frag<float> &b, floatx16_t c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ floatx16_t zero16()
{
    floatx16_t z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}

// Pieces 2 m + half of row r, m = 0 .. NM - 1
template <typename T, int D> __device__ __forceinline__ Frag<T> row_frag(const unsigned char *tile, int r, int m, int half)
{
    return *reinterpret_cast<const Frag<T> *>(tile + RowTile<T, D>::at(r, 2 * m + half));
}

// Operands are read some steps before the products that need them, and the order is pinned: left alone a read sinks to its use, or all of them
// rise and spill.
constexpr int kAhead = 3;  // steps of tile_scores; 2 and 4 are as fast
constexpr int kRing = 6;   // operands of the dkdv kernel; 4 and 8 are as fast
template <typename F, int... K> __device__ __forceinline__ void static_for_(F f, std::integer_sequence<int, K...>) { (f(std::integral_constant<int, K>{}), ...); }
template <int N, typename F> __device__ __forceinline__ void static_for(F f) { static_for_(f, std::make_integer_sequence<int, N>{}); }  // f(0) .. f(N - 1), as constants
__device__ __forceinline__ void pin_order() { __builtin_amdgcn_sched_barrier(0); }

// s[t] = rows r + 32 t of a tile by the own rows
template <typename T, int D, int KT>
__device__ __forceinline__ void tile_scores(const unsigned char *tile, int r, const Frag<T> (&own)[D * sizeof(T) / 32], floatx16_t (&s)[KT])
{
    constexpr int NM = D * (int)sizeof(T) / 32;
    const int half = (threadIdx.x & 63) >> 5;
    Frag<T> f[kAhead][KT];
    auto fetch = [&](int m) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < KT; ++t) f[m % kAhead][t] = row_frag<T, D>(tile, r + 32 * t, m, half);
    };
#pragma unroll
    for (int t = 0; t < KT; ++t) s[t] = zero16();
#pragma unroll
    for (int m = 0; m < kAhead; ++m) fetch(m);
    pin_order();
#pragma unroll
    for (int m = 0; m < NM; ++m) {
#pragma unroll
        for (int t = 0; t < KT; ++t) s[t] = product(f[m % kAhead][t], own[m], s[t]);
        if (m + kAhead < NM) fetch(m + kAhead);
        pin_order();
    }
}
// The same of row r of two tiles, each by own rows of its own
template <typename T, int D>
__device__ __forceinline__ void tile_scores2(const unsigned char *t1, const unsigned char *t2, int r, const Frag<T> (&own1)[D * sizeof(T) / 32],
                                             const Frag<T> (&own2)[D * sizeof(T) / 32], floatx16_t &s1, floatx16_t &s2)
{
    constexpr int NM = D * (int)sizeof(T) / 32;
    const int half = (threadIdx.x & 63) >> 5;
    Frag<T> f[kAhead][2];
    auto fetch = [&](int m) __attribute__((always_inline)) {
        f[m % kAhead][0] = row_frag<T, D>(t1, r, m, half);
        f[m % kAhead][1] = row_frag<T, D>(t2, r, m, half);
    };
    s1 = zero16();
    s2 = zero16();
#pragma unroll
    for (int m = 0; m < kAhead; ++m) fetch(m);
    pin_order();
#pragma unroll
    for (int m = 0; m < NM; ++m) {
        s1 = product(f[m % kAhead][0], own1[m], s1);
        s2 = product(f[m % kAhead][1], own2[m], s2);
        if (m + kAhead < NM) fetch(m + kAhead);
        pin_order();
    }
}

// Weights as the products take them: of 32 tile rows by the own column, results of a product with the tile rows as A.
// bf16: rounded (half a step of 2^-8 each, of one sign as often as the other; the sums are in 32 bits), 16 rows a step.
template <typename T> struct Weights;
template <> struct Weights<bf16_t> {
    bf16x8_t v[2];
    __device__ __forceinline__ void set(const floatx16_t &w)
    {
#pragma unroll
        for (int s = 0; s < 2; ++s)
            v[s] = __builtin_bit_cast(bf16x8_t, make_uint4(pack_bf16x2(w[8 * s], w[8 * s + 1]), pack_bf16x2(w[8 * s + 2], w[8 * s + 3]),
                                                           pack_bf16x2(w[8 * s + 4], w[8 * s + 5]), pack_bf16x2(w[8 * s + 6], w[8 * s + 7])));
    }
    __device__ __forceinline__ float sum(float x) const  // x + all of them, as they were rounded
    {
        const bf16x2_t one = __builtin_bit_cast(bf16x2_t, 0x3F803F80u);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint4 h = __builtin_bit_cast(uint4, v[s]);
            x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, h.x), one, x, false);
            x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, h.y), one, x, false);
            x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, h.z), one, x, false);
            x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, h.w), one, x, false);
        }
        return x;
    }
    // what the rounding of w to *this left
    __device__ __forceinline__ void set_tail(const floatx16_t &w, const Weights &head)
    {
        floatx16_t t;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint4 h = __builtin_bit_cast(uint4, head.v[s]);
            const uint32_t x[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                t[8 * s + 2 * i] = w[8 * s + 2 * i] - __uint_as_float(x[i] << 16);
                t[8 * s + 2 * i + 1] = w[8 * s + 2 * i + 1] - __uint_as_float(x[i] & 0xFFFF0000u);
            }
        }
        set(t);
    }
    __device__ __forceinline__ void set_pair(int i, float a, float b)  // weights i, i + 1
    {
        uint4 x = __builtin_bit_cast(uint4, v[i >> 3]);
        const uint32_t p = pack_bf16x2(a, b);
        if ((i & 6) == 0) x.x = p;
        else if ((i & 6) == 2) x.y = p;
        else if ((i & 6) == 4) x.z = p;
        else x.w = p;
        v[i >> 3] = __builtin_bit_cast(bf16x8_t, x);
    }
};
template <> struct Weights<float> {
    floatx16_t v;
    __device__ __forceinline__ void set(const floatx16_t &w) { v = w; }
};

// acc[nb] (channels 32 nb .. + 31 by own rows) += sum over tile rows r0 .. r0 + 31 of row[channel] * w, in STEPS steps: operands of step i are read
// by fetch(i), at least AHEAD steps before step(i).
template <typename T, int D> struct RowSum;
template <int D> struct RowSum<bf16_t, D> {
    typedef RowTile<bf16_t, D> RT;
    static constexpr int NB = D / 32, STEPS = 2 * NB, AHEAD = 4;
    typedef bf16x8_t Operand;
    __device__ __forceinline__ static Operand fetch(const unsigned char *tile, int r0, int i)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, e = (lane >> 2) & 3, q = lane & 3, b4 = (lane >> 4) & 1;
        const int r = r0 + 4 * half + e + 16 * (i / NB), p = 4 * (i % NB) + 2 * b4 + (q >> 1), sub = (q & 1) * 8;
        return tr_frag(tile + RT::at(r, p) + sub, tile + RT::at(r + 8, p) + sub);
    }
    __device__ __forceinline__ static void step(int i, const Operand &f, const Weights<bf16_t> &w, floatx16_t (&acc)[NB])
    {
        acc[i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, w.v[i / NB], acc[i % NB], 0, 0, 0);
    }
};
template <int D> struct RowSum<float, D> {
    typedef RowTile<float, D> RT;
    static constexpr int NB = D / 32, STEPS = 16, AHEAD = 2;
    struct Operand {
        float v[NB];
    };
    __device__ __forceinline__ static Operand fetch(const unsigned char *tile, int r0, int i)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, n = lane & 31, r = r0 + 8 * (i >> 2) + 4 * half + (i & 3);
        Operand f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) f.v[nb] = *reinterpret_cast<const float *>(tile + RT::at(r, 8 * nb + (n >> 2)) + (n & 3) * 4);
        return f;
    }
    __device__ __forceinline__ static void step(int i, const Operand &f, const Weights<float> &w, floatx16_t (&acc)[NB])
    {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(f.v[nb], w.v[i], acc[nb], 0, 0, 0);
    }
};
template <typename T, int D> __device__ __forceinline__ void weighted_rows(const unsigned char *tile, int r0, const Weights<T> &w, floatx16_t (&acc)[D / 32])
{
    typedef RowSum<T, D> RS;
    typename RS::Operand f[RS::AHEAD];
#pragma unroll
    for (int i = 0; i < RS::AHEAD; ++i) f[i] = RS::fetch(tile, r0, i);
    pin_order();
#pragma unroll
    for (int i = 0; i < RS::STEPS; ++i) {
        RS::step(i, f[i % RS::AHEAD], w, acc);
        if (i + RS::AHEAD < RS::STEPS) f[i % RS::AHEAD] = RS::fetch(tile, r0, i + RS::AHEAD);
        pin_order();
    }
}
template <typename T, int D> __device__ __forceinline__ void weighted_rows(const unsigned char *tile, int r0, const floatx16_t &w, floatx16_t (&acc)[D / 32])
{
    Weights<T> x;
    x.set(w);
    weighted_rows<T, D>(tile, r0, x, acc);
}

// Weights as two bf16 words, 16 significant bits; the operands are read once for both.
template <typename T, int D> __device__ __forceinline__ void precise_weighted_rows(const unsigned char *tile, int r0, const floatx16_t &w, floatx16_t (&acc)[D / 32])
{
    if constexpr (sizeof(T) == 4) {
        weighted_rows<T, D>(tile, r0, w, acc);
    } else {
        typedef RowSum<T, D> RS;
        Weights<T> head, tail;
        head.set(w);
        tail.set_tail(w, head);
        typename RS::Operand f[RS::AHEAD];
#pragma unroll
        for (int i = 0; i < RS::AHEAD; ++i) f[i] = RS::fetch(tile, r0, i);
        pin_order();
#pragma unroll
        for (int i = 0; i < RS::STEPS; ++i) {
            RS::step(i, f[i % RS::AHEAD], tail, acc);
            RS::step(i, f[i % RS::AHEAD], head, acc);
            if (i + RS::AHEAD < RS::STEPS) f[i % RS::AHEAD] = RS::fetch(tile, r0, i + RS::AHEAD);
            pin_order();
        }
    }
}

// Value of the other half's lane with the same column, combined by max or sum.
__device__ __forceinline__ float halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// four channels of a row
__device__ __forceinline__ void store4(bf16_t *p, float a, float b, float c, float d)
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}
__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) { *reinterpret_cast<float4 *>(p) = make_float4(a, b, c, d); }

// O rounded to its type, and what the rounding took (the backward's Delta = dO . O wants more than 8 bits of O: with O alone, queries that see
// few keys get gradients 5e-3 off, with the tail 2.5e-3, the rounding of weights and results).
__device__ __forceinline__ uint32_t tail_of(float a, float b)
{
    const uint32_t w = pack_bf16x2(a, b);
    return pack_bf16x2(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ void store_out(bf16_t *p, bf16_t *tail, float a, float b, float c, float d)
{
    store4(p, a, b, c, d);
    if (tail) *reinterpret_cast<uint2 *>(tail) = make_uint2(tail_of(a, b), tail_of(c, d));
}
__device__ __forceinline__ void store_out(float *p, bf16_t *, float a, float b, float c, float d) { store4(p, a, b, c, d); }

// Kernels that join pieces: LPR lanes to a row (token and head) and piece.  GROUPS = 1: a wave takes 64 / LPR heads of one token; false behind the
// last token (whole waves), heads past the last one are the caller's to leave out.  Else a block takes one row, GROUPS pieces at a time.
template <int LPR, int GROUPS> __device__ __forceinline__ bool merge_row(int total, int heads, int &tok, int &head)
{
    const uint32_t block = blockIdx.z * gridDim.x + blockIdx.x;  // below 2^28: total * heads is below 2^29
    if constexpr (GROUPS > 1) {
        tok = (int)(block / (uint32_t)heads);
        head = (int)(block - (uint32_t)tok * (uint32_t)heads);
    } else {
        constexpr int HPW = 64 / LPR;
        const uint32_t per = ((uint32_t)heads + HPW - 1) / HPW, w = block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        tok = (int)(w / per);
        head = (int)(w - (uint32_t)tok * per) * HPW + (threadIdx.x & 63) / LPR;
    }
    return tok < total;
}
// Their grid, twice for y = 2.  Along x as many blocks as keep their threads below 2^32, the rest along z.
template <int LPR, int GROUPS> __host__ __forceinline__ dim3 merge_grid(int64_t total, int heads, int y = 1)
{
    constexpr int HPW = 64 / LPR;
    const int64_t n = GROUPS > 1 ? total * heads : (total * ((heads + HPW - 1) / HPW) + 3) / 4, most = 1 << 22;
    return dim3((unsigned)(n < most ? n : most), (unsigned)y, (unsigned)((n + most - 1) / most));
}
// A row of many pieces has a block to itself where that is not too many blocks.
__host__ __forceinline__ bool wide_merge(int splits, int64_t rows) { return splits > 8 && rows < 65536; }
// The groups' sums of four channels each; group 0 has them all.
template <int LPR, int GROUPS> __device__ __forceinline__ void join_groups(float (&v)[4])
{
    if constexpr (GROUPS > 1) {
        __shared__ __align__(16) float part[GROUPS][LPR * 4];
        const int lane = threadIdx.x % LPR, grp = threadIdx.x / LPR;
        *reinterpret_cast<float4 *>(&part[grp][4 * lane]) = make_float4(v[0], v[1], v[2], v[3]);
        __syncthreads();
        if (grp == 0) {
            v[0] = v[1] = v[2] = v[3] = 0.f;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const float4 x = *reinterpret_cast<const float4 *>(&part[g][4 * lane]);
                v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
            }
        }
    }
}

// LDS that lanes of one wave write for others of it: keeps the compiler from moving accesses, of whatever types, across the point.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ void wait_loads_and_sync()
{
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): a barrier alone does not wait for loads into LDS
    __syncthreads();
}

// Bytes of the unnormalised sums of a forward in pieces; behind them, two floats a row and piece.
inline size_t packed_fwd_acc_bytes(int64_t total_q, int Hq, int d, int splits) { return splits > 1 ? align_up((size_t)total_q * Hq * splits * d * 4, 256) : 0; }
// few: tiles of 32 rows whose four waves share the long axis, else 128 rows, 32 a wave
dsv_status launch_packed_fwd(const PackedArgs &a, int dtype, int d, bool few, const void *Q, const void *K, const void *V, void *O, void *O_tail,
                             float *lse, char *ws, hipStream_t st);

// The backward's scratch: statistics of every row, and the pieces of dQ or of dK and dV.
struct PackedBwdPlan {
    bool few_q, few_k;        // tiles of 32 rows in the dq step, of 32 keys in the dkdv step
    int splits_q, chunk_q;    // keys of the dq step in pieces
    int splits_k, chunk_k;    // rows of the dkdv step in pieces
};
inline size_t packed_stat_bytes(int64_t total_q, int Hq) { return align_up((size_t)total_q * Hq * 8, 256); }
inline size_t packed_dq_bytes(int64_t total_q, int Hq, int d, int splits) { return splits > 1 ? align_up((size_t)total_q * Hq * splits * d * 4, 256) : 0; }
inline size_t packed_dkdv_bytes(int64_t total_k, int Hkv, int d, int splits) { return splits > 1 ? 2 * align_up((size_t)total_k * Hkv * splits * d * 4, 256) : 0; }
dsv_status launch_packed_bwd(const PackedArgs &a, const PackedBwdPlan &plan, int dtype, int d, const void *Q, const void *K, const void *V, const void *O,
                             const void *O_tail, const float *lse, const void *dO, void *dQ, void *dK, void *dV, char *ws, hipStream_t st);

}  // namespace dsv
