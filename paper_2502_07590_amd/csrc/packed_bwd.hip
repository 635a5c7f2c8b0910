// Softmax attention over packed sequences, backward.
//
//   p_ij = exp(s_ij - lse_i);  Delta_i = dO_i . O_i;  dS_ij = p_ij (dO_i . v_j - Delta_i)
//   dQ_i = scale sum_j dS_ij k_j;   dK_j = scale sum_i dS_ij q_i;   dV_j = sum_i p_ij dO_i   (i over the queries of every head that reads j's)
//
// Three kernels: the rows' statistics; dQ with a wave's 32 rows as columns against tiles of keys, as in the forward; dK and dV with a wave's 32
// keys as columns against tiles of rows.  Scores and dP are formed in both, so that every sum has one owner: no atomics, the same bits from
// run to run.  With dS as two bf16 words in dQ's product that makes eight products of 2 d operations a pair, where five would do.  Formed once, by
// the key-major step, dQ would be a sum over blocks of 128 keys in 32 bits: 32768 tokens, 4 heads, d = 128, 17 GB written and read again, 6.8 ms at a
// copy's rate, for two products of eight, 1.8 ms.
//
// Roundings (bf16): dS is two words in dQ because its errors there meet Delta's: one word leaves 2.5 to 2.7e-3 in norm, two 1.8 to 2.0e-3.  In dK, and
// P in dV, it is one word: 2.4 to 2.5e-3 and 2.0 to 2.3e-3; a second word each would be two products more.
//
// Bound by products under the power limit: 32768 tokens, 4 heads, d = 128, bf16: statistics 0.02 ms, dQ 3.4 (1290 TFLOP/s of its four products),
// dK and dV 3.75 (1170).
#include "packed_attn.h"

namespace dsv {
namespace {

template <typename T, int D> __device__ __forceinline__ float dot16(const T *a, const T *b)  // 16 bytes of each
{
    constexpr int CH = 16 / sizeof(T);
    return dot_chunk<T, CH>(load_chunk<T, CH>(a), load_chunk<T, CH>(b));
}

// stat[hk][token * group + head of the group] = {lse * log2(e), Delta}; rows that saw no key: {inf, 0}, weights of zero
template <typename T, int D>
__global__ __launch_bounds__(256) void packed_stat_kernel(const T *__restrict__ O, const T *__restrict__ tail, const T *__restrict__ dO, const float *__restrict__ lse,
                                                          float2 *__restrict__ stat, PackedArgs a)
{
    constexpr int LPR = D * (int)sizeof(T) / 16, CH = 16 / (int)sizeof(T);
    int tok, head;
    if (!merge_row<LPR, 1>(a.total_q, a.Hq, tok, head)) return;
    const int lane = threadIdx.x % LPR;
    const int hc = min(head, a.Hq - 1);
    const T *go = reinterpret_cast<const T *>(reinterpret_cast<const unsigned char *>(dO) + (int64_t)tok * a.do_row + (int64_t)hc * a.do_head) + lane * CH;
    const T *o = reinterpret_cast<const T *>(reinterpret_cast<const unsigned char *>(O) + (int64_t)tok * a.o_row + (int64_t)hc * a.o_head) + lane * CH;
    float x = dot16<T, D>(go, o);
    if (tail) x += dot16<T, D>(go, tail + ((int64_t)tok * a.Hq + hc) * D + lane * CH);
#pragma unroll
    for (int s = LPR / 2; s > 0; s >>= 1) x += __shfl_xor(x, s);
    if (lane || head >= a.Hq) return;
    const float l = lse[(int64_t)head * a.total_q + tok];
    const int hk = head / a.group;
    stat[(int64_t)hk * a.total_q * a.group + (int64_t)tok * a.group + (head - hk * a.group)] =
        l == kNegInf ? make_float2(-kNegInf, 0.f) : make_float2(l * kLog2e, x);
}

template <typename T, int D, int WK> struct BwdShape {
    static constexpr int OWN = WK == 1 ? 128 : 32, ROWS = WK == 1 ? 64 : 128, RT = ROWS / 32 / WK;  // own rows, rows of a tile, 32s of them a wave
    static constexpr int TILE = ROWS * D * (int)sizeof(T);
    static constexpr int NBUF = 2 * 2 * TILE <= 128 * 1024 ? 2 : 1;
    static_assert(TILE / (NBUF == 2 ? 1 : 2) >= 32 * D * 4, "a wave's sums fit its part of the tiles");
};

// The four waves' sums of the same 32 rows, joined in LDS: thread t's share is channels 4 g .. 4 g + 3 of row t % 32 for g = t / 32, + 8, ...
// area(w): where wave w's 32 rows of D sums go.
template <int D, typename A, typename F> __device__ __forceinline__ void join_waves(A area, const floatx16_t (&acc)[D / 32], int wave, F put)
{
    const int lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
    __syncthreads();
#pragma unroll
    for (int nb = 0; nb < D / 32; ++nb)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4 *>(area(wave) + ((nb * 8 + 2 * g + half) * 32 + n) * 4) =
                make_float4(acc[nb][4 * g], acc[nb][4 * g + 1], acc[nb][4 * g + 2], acc[nb][4 * g + 3]);
    __syncthreads();
    for (int g = wave * 2 + half; g < D / 4; g += 8) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float4 x = *reinterpret_cast<const float4 *>(area(w) + (g * 32 + n) * 4);
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
        }
        put(4 * g, v[0], v[1], v[2], v[3]);
    }
}

template <typename T, int D, int WK>
__global__ __launch_bounds__(256, sizeof(T) == 2 && WK == 1 ? 2 : 1) void packed_dq_kernel(const T *__restrict__ Q, const T *__restrict__ K, const T *__restrict__ V,
                                                                                       const T *__restrict__ dO, const float2 *__restrict__ stat,
                                                                                       T *__restrict__ dQ, float *__restrict__ part, PackedArgs a)
{
    typedef RowTile<T, D> RT;
    typedef BwdShape<T, D, WK> Sh;
    constexpr int NM = RT::RB / 32, NB = D / 32;
    // every tile an array of its own: reads of one then need not wait for the loads into another
    __shared__ __align__(1024) unsigned char ka[Sh::TILE], va[Sh::TILE], kb[Sh::NBUF == 2 ? Sh::TILE : 16], vb[Sh::NBUF == 2 ? Sh::TILE : 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int hk = blockIdx.x % a.Hkv, place = blockIdx.x / a.Hkv, split = blockIdx.y;
    const int slot = a.causal ? (int)(gridDim.x / a.Hkv) - 1 - place : place;
    const int si = __builtin_amdgcn_readfirstlane(find_sequence(a.cu_q, a.n_seq, a.total_q, a.group, Sh::OWN, slot));
    const Sequence sq = read_sequence(a, si);
    const int rows = sq.nq * a.group;
    const int row0 = (slot - first_slot(a.cu_q[si], a.total_q, a.group, Sh::OWN, si)) * Sh::OWN;
    if (row0 < 0 || row0 >= rows) return;
    const int row = row0 + (WK == 1 ? wave * 32 : 0) + n;
    const int rc = min(row, rows - 1), tok = row_token(a, rc), head = hk * a.group + (rc - tok * a.group);
    const int kbeg = split * a.chunk, kcut = a.chunk ? min(sq.nk, kbeg + a.chunk) : sq.nk;
    const int past = sq.nk - sq.nq, seen = a.causal ? min(sq.nk, tok + past + 1) : sq.nk;
    int kend = kcut;
    if (a.causal) kend = min(kend, row_token(a, min(row0 + Sh::OWN, rows) - 1) + past + 1);
    if (a.splits > 1 && kbeg >= kend) return;  // no row of this tile sees the piece: the sum does not read it

    Frag<T> qf[NM], gf[NM];
    {
        const unsigned char *qp = reinterpret_cast<const unsigned char *>(Q) + (int64_t)(sq.q0 + tok) * a.q_row + (int64_t)head * a.q_head;
        const unsigned char *gp = reinterpret_cast<const unsigned char *>(dO) + (int64_t)(sq.q0 + tok) * a.do_row + (int64_t)head * a.do_head;
#pragma unroll
        for (int m = 0; m < NM; ++m) {
            qf[m] = *reinterpret_cast<const Frag<T> *>(qp + (2 * m + half) * 16);
            gf[m] = *reinterpret_cast<const Frag<T> *>(gp + (2 * m + half) * 16);
        }
    }
    const float2 rs = stat[(int64_t)hk * a.total_q * a.group + (int64_t)sq.q0 * a.group + rc];
    const unsigned char *kp = reinterpret_cast<const unsigned char *>(K) + (int64_t)sq.k0 * a.k_row + (int64_t)hk * a.k_head;
    const unsigned char *vp = reinterpret_cast<const unsigned char *>(V) + (int64_t)sq.k0 * a.v_row + (int64_t)hk * a.v_head;
    RowLoads<T, D, Sh::ROWS, 4> kl, vl;
    kl.set(wave, a.k_row);
    vl.set(wave, a.v_row);
    auto request = [&](int k0, unsigned char *kt, unsigned char *vt) __attribute__((always_inline)) {
        kl.keys(kp, a.k_row, k0, sq.nk, kt);
        vl.keys(vp, a.v_row, k0, sq.nk, vt);
    };
    const float c = a.scale * kLog2e;
    floatx16_t acc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[nb] = zero16();
    auto tile = [&](int k0, const unsigned char *kt, const unsigned char *vt) __attribute__((always_inline)) {
        const bool edge = k0 + Sh::ROWS > kcut || (a.causal && k0 + Sh::ROWS > row_token(a, row0) + past + 1);
#pragma unroll
        for (int t = 0; t < Sh::RT; ++t) {
            const int sub = (WK == 1 ? 0 : wave * 32) + 32 * t;
            floatx16_t s, dp;
            tile_scores2<T, D>(kt, vt, sub + n, qf, gf, s, dp);
            if (edge) {
                const int lim = min(seen, kcut) - k0 - sub - 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) < lim ? s[i] : kNegInf;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = fast_exp2(fmaf(s[i], c, -rs.x)) * (dp[i] - rs.y);
            precise_weighted_rows<T, D>(kt, sub, s, acc);
        }
    };
    if (kbeg < kend) {
        if constexpr (Sh::NBUF == 2) {
            request(kbeg, ka, va);
            for (int k0 = kbeg; k0 < kend; k0 += 2 * Sh::ROWS) {
                wait_loads_and_sync();
                if (k0 + Sh::ROWS < kend) request(k0 + Sh::ROWS, kb, vb);
                tile(k0, ka, va);
                if (k0 + Sh::ROWS < kend) {  // (a break here makes the compiler move all sums to other registers and back)
                    wait_loads_and_sync();
                    if (k0 + 2 * Sh::ROWS < kend) request(k0 + 2 * Sh::ROWS, ka, va);
                    tile(k0 + Sh::ROWS, kb, vb);
                }
            }
        } else {
            for (int k0 = kbeg; k0 < kend; k0 += Sh::ROWS) {
                __syncthreads();
                request(k0, ka, va);
                wait_loads_and_sync();
                tile(k0, ka, va);
            }
        }
    }
    T *const op = reinterpret_cast<T *>(reinterpret_cast<unsigned char *>(dQ) + (int64_t)(sq.q0 + tok) * a.dq_row + (int64_t)head * a.dq_head);
    float *const pp = part + (((int64_t)(sq.q0 + tok) * a.Hq + head) * a.splits + split) * D;
    auto put = [&](int ch, float x, float y, float z, float w) __attribute__((always_inline)) {
        if (row >= rows) return;
        if (a.splits > 1) store4(pp + ch, x * a.scale, y * a.scale, z * a.scale, w * a.scale);
        else store4(op + ch, x * a.scale, y * a.scale, z * a.scale, w * a.scale);
    };
    if constexpr (WK > 1) {
        auto area = [&](int w) __attribute__((always_inline)) {
            return reinterpret_cast<float *>(Sh::NBUF == 2 ? (w == 0 ? ka : w == 1 ? va : w == 2 ? kb : vb) : (w < 2 ? ka : va) + (w & 1) * (Sh::TILE / 2));
        };
        join_waves<D>(area, acc, wave, put);
    } else {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int g = 0; g < 4; ++g) put(32 * nb + 8 * g + 4 * half, acc[nb][4 * g], acc[nb][4 * g + 1], acc[nb][4 * g + 2], acc[nb][4 * g + 3]);
    }
}

// Calls of few keys, and fp32: 32 keys a block, the four waves take 32 rows each of a tile of 128.  fp32, 1024 tokens of two heads, d = 64: 18 us, one
// round of blocks of products that take 64 cycles each; 128 keys a block would spill in fp32.
template <typename T, int D>
__global__ __launch_bounds__(256, 1) void packed_dkdv_few_kernel(
    const T *__restrict__ Q, const T *__restrict__ K, const T *__restrict__ V, const T *__restrict__ dO, const float2 *__restrict__ stat, T *__restrict__ dK,
    T *__restrict__ dV, float *__restrict__ part_k, float *__restrict__ part_v, PackedArgs a)
{
    typedef RowTile<T, D> RT;
    typedef BwdShape<T, D, 4> Sh;
    constexpr int NM = RT::RB / 32, NB = D / 32;
    // every tile an array of its own: reads of one then need not wait for the loads into another
    __shared__ __align__(1024) unsigned char qa[Sh::TILE], ga[Sh::TILE], qb[Sh::NBUF == 2 ? Sh::TILE : 16], gb[Sh::NBUF == 2 ? Sh::TILE : 16];
    __shared__ __align__(16) float st[Sh::NBUF][2][Sh::ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int hk = blockIdx.x % a.Hkv, slot = blockIdx.x / a.Hkv, split = blockIdx.y;
    const int si = __builtin_amdgcn_readfirstlane(find_sequence(a.cu_k, a.n_seq, a.total_k, 1, Sh::OWN, slot));
    const Sequence sq = read_sequence(a, si);
    const int key0 = (slot - first_slot(a.cu_k[si], a.total_k, 1, Sh::OWN, si)) * Sh::OWN;
    if (key0 < 0 || key0 >= sq.nk) return;
    const int rows = sq.nq * a.group, past = sq.nk - sq.nq;
    const int key = key0 + n, kc = min(key, sq.nk - 1);
    int rbeg = split * a.chunk;
    const int rend = a.chunk ? min(rows, rbeg + a.chunk) : rows;
    if (a.causal) rbeg = max(rbeg, max(0, key0 - past) * a.group / Sh::ROWS * Sh::ROWS);  // rows before see none of these keys
    if (a.splits > 1 && rbeg >= rend) return;  // no row of the piece sees these keys: the sum does not read it

    Frag<T> kf[NM], vf[NM];
    {
        const unsigned char *kp = reinterpret_cast<const unsigned char *>(K) + (int64_t)(sq.k0 + kc) * a.k_row + (int64_t)hk * a.k_head;
        const unsigned char *vp = reinterpret_cast<const unsigned char *>(V) + (int64_t)(sq.k0 + kc) * a.v_row + (int64_t)hk * a.v_head;
#pragma unroll
        for (int m = 0; m < NM; ++m) {
            kf[m] = *reinterpret_cast<const Frag<T> *>(kp + (2 * m + half) * 16);
            vf[m] = *reinterpret_cast<const Frag<T> *>(vp + (2 * m + half) * 16);
        }
    }
    const unsigned char *qp = reinterpret_cast<const unsigned char *>(Q) + (int64_t)sq.q0 * a.q_row + (int64_t)hk * a.group * a.q_head;
    const unsigned char *gp = reinterpret_cast<const unsigned char *>(dO) + (int64_t)sq.q0 * a.do_row + (int64_t)hk * a.group * a.do_head;
    const float2 *const sp = stat + (int64_t)hk * a.total_q * a.group + (int64_t)sq.q0 * a.group;
    float2 sn = make_float2(-kNegInf, 0.f);
    RowLoads<T, D, Sh::ROWS, 4> ql, gl;
    ql.set(wave, a.q_row, a, a.q_head);
    gl.set(wave, a.do_row, a, a.do_head);
    auto request = [&](int r0, unsigned char *qt, unsigned char *gt) __attribute__((always_inline)) {
        ql.rows(a, qp, a.q_row, a.q_head, r0, rows, qt);
        gl.rows(a, gp, a.do_row, a.do_head, r0, rows, gt);
        if ((int)threadIdx.x < Sh::ROWS) sn = r0 + (int)threadIdx.x < rend ? sp[r0 + threadIdx.x] : make_float2(-kNegInf, 0.f);  // rows past the end: weights of zero
    };
    auto park = [&](int b) __attribute__((always_inline)) {
        if ((int)threadIdx.x < Sh::ROWS) {
            st[b][0][threadIdx.x] = sn.x;
            st[b][1][threadIdx.x] = sn.y;
        }
    };
    const float c = a.scale * kLog2e;
    floatx16_t dk[NB], dv[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) dk[nb] = dv[nb] = zero16();
    const int first_seen = a.causal ? min(max(key - past, 0), sq.nq) * a.group : 0;  // key j is seen by rows from (j - past) * group on
    auto tile = [&](int r0, const unsigned char *qt, const unsigned char *gt, int b) __attribute__((always_inline)) {
        const bool edge = a.causal && key0 + Sh::OWN > row_token(a, r0) + past + 1;
        const int sub = wave * 32;
        {
            floatx16_t s, dp;
            tile_scores2<T, D>(qt, gt, sub + n, kf, vf, s, dp);
            if (edge) {
                const int lim = first_seen - r0 - sub - 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) >= lim ? s[i] : kNegInf;
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 l2 = *reinterpret_cast<const float4 *>(&st[b][0][sub + 8 * g + 4 * half]);
                const float4 dl = *reinterpret_cast<const float4 *>(&st[b][1][sub + 8 * g + 4 * half]);
                const float l[4] = {l2.x, l2.y, l2.z, l2.w}, d[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[4 * g + i] = fast_exp2(fmaf(s[4 * g + i], c, -l[i]));
                    dp[4 * g + i] = s[4 * g + i] * (dp[4 * g + i] - d[i]);
                }
            }
            weighted_rows<T, D>(gt, sub, s, dv);
            weighted_rows<T, D>(qt, sub, dp, dk);
        }
    };
    if (rbeg < rend) {
        if constexpr (Sh::NBUF == 2) {
            request(rbeg, qa, ga);
            park(0);
            for (int r0 = rbeg; r0 < rend; r0 += 2 * Sh::ROWS) {
                wait_loads_and_sync();
                if (r0 + Sh::ROWS < rend) request(r0 + Sh::ROWS, qb, gb);
                tile(r0, qa, ga, 0);
                if (r0 + Sh::ROWS < rend) {
                    park(1);
                    wait_loads_and_sync();
                    if (r0 + 2 * Sh::ROWS < rend) request(r0 + 2 * Sh::ROWS, qa, ga);
                    tile(r0 + Sh::ROWS, qb, gb, 1);
                    if (r0 + 2 * Sh::ROWS < rend) park(0);
                }
            }
        } else {
            for (int r0 = rbeg; r0 < rend; r0 += Sh::ROWS) {
                __syncthreads();
                request(r0, qa, ga);
                park(0);
                wait_loads_and_sync();
                tile(r0, qa, ga, 0);
            }
        }
    }
    T *const kop = reinterpret_cast<T *>(reinterpret_cast<unsigned char *>(dK) + (int64_t)(sq.k0 + kc) * a.dk_row + (int64_t)hk * a.dk_head);
    T *const vop = reinterpret_cast<T *>(reinterpret_cast<unsigned char *>(dV) + (int64_t)(sq.k0 + kc) * a.dv_row + (int64_t)hk * a.dv_head);
    const int64_t pid = (((int64_t)(sq.k0 + kc) * a.Hkv + hk) * a.splits + split) * D;
    auto put_k = [&](int ch, float x, float y, float z, float w) __attribute__((always_inline)) {
        if (key >= sq.nk) return;
        if (a.splits > 1) store4(part_k + pid + ch, x * a.scale, y * a.scale, z * a.scale, w * a.scale);
        else store4(kop + ch, x * a.scale, y * a.scale, z * a.scale, w * a.scale);
    };
    auto put_v = [&](int ch, float x, float y, float z, float w) __attribute__((always_inline)) {
        if (key >= sq.nk) return;
        if (a.splits > 1) store4(part_v + pid + ch, x, y, z, w);
        else store4(vop + ch, x, y, z, w);
    };
    auto area = [&](int w) __attribute__((always_inline)) {
        return reinterpret_cast<float *>(Sh::NBUF == 2 ? (w == 0 ? qa : w == 1 ? ga : w == 2 ? qb : gb) : (w < 2 ? qa : ga) + (w & 1) * (Sh::TILE / 2));
    };
    join_waves<D>(area, dk, wave, put_k);
    join_waves<D>(area, dv, wave, put_v);
}

template <int D, bool CAUSAL>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void packed_dkdv_kernel(
    const bf16_t *__restrict__ Q, const bf16_t *__restrict__ K, const bf16_t *__restrict__ V, const bf16_t *__restrict__ dO, const float2 *__restrict__ stat, bf16_t *__restrict__ dK,
    bf16_t *__restrict__ dV, float *__restrict__ part_k, float *__restrict__ part_v, PackedArgs a)
{
    typedef bf16_t T;
    typedef RowTile<T, D> RT;
    typedef RowSum<T, D> RS;
    typedef BwdShape<T, D, 1> Sh;
    constexpr int RING = D == 128 ? kRing : kRing - 2;  // (6 at d = 64 would spill)
    static_assert(Sh::RT == 2 && Sh::NBUF == 2, "two halves of a tile");
    constexpr int NM = RT::RB / 32, NB = D / 32;
    // every tile an array of its own: reads of one then need not wait for the loads into another
    __shared__ __align__(1024) unsigned char qa[Sh::TILE], ga[Sh::TILE], qb[Sh::NBUF == 2 ? Sh::TILE : 16], gb[Sh::NBUF == 2 ? Sh::TILE : 16];
    __shared__ __align__(16) float st[Sh::NBUF][2][Sh::ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int hk = blockIdx.x % a.Hkv, slot = blockIdx.x / a.Hkv, split = blockIdx.y;
    const int si = __builtin_amdgcn_readfirstlane(find_sequence(a.cu_k, a.n_seq, a.total_k, 1, Sh::OWN, slot));
    const Sequence sq = read_sequence(a, si);
    const int key0 = (slot - first_slot(a.cu_k[si], a.total_k, 1, Sh::OWN, si)) * Sh::OWN;
    if (key0 < 0 || key0 >= sq.nk) return;
    const int rows = sq.nq * a.group, past = sq.nk - sq.nq;
    const int key = key0 + wave * 32 + n, kc = min(key, sq.nk - 1);
    int rbeg = split * a.chunk;
    const int rend = a.chunk ? min(rows, rbeg + a.chunk) : rows;
    if (a.causal) rbeg = max(rbeg, max(0, key0 - past) * a.group / Sh::ROWS * Sh::ROWS);  // rows before see none of these keys
    if (a.splits > 1 && rbeg >= rend) return;  // no row of the piece sees these keys: the sum does not read it

    Frag<T> kf[NM], vf[NM];
    {
        const unsigned char *kp = reinterpret_cast<const unsigned char *>(K) + (int64_t)(sq.k0 + kc) * a.k_row + (int64_t)hk * a.k_head;
        const unsigned char *vp = reinterpret_cast<const unsigned char *>(V) + (int64_t)(sq.k0 + kc) * a.v_row + (int64_t)hk * a.v_head;
#pragma unroll
        for (int m = 0; m < NM; ++m) {
            kf[m] = *reinterpret_cast<const Frag<T> *>(kp + (2 * m + half) * 16);
            vf[m] = *reinterpret_cast<const Frag<T> *>(vp + (2 * m + half) * 16);
        }
        if constexpr (D == 128) {  // to the other half of the registers, where products can take them from
#pragma unroll
            for (int m = 0; m < NM; ++m) asm volatile("" : "+a"(kf[m].v), "+a"(vf[m].v));
        }
    }
    const unsigned char *qp = reinterpret_cast<const unsigned char *>(Q) + (int64_t)sq.q0 * a.q_row + (int64_t)hk * a.group * a.q_head;
    const unsigned char *gp = reinterpret_cast<const unsigned char *>(dO) + (int64_t)sq.q0 * a.do_row + (int64_t)hk * a.group * a.do_head;
    const float2 *const sp = stat + (int64_t)hk * a.total_q * a.group + (int64_t)sq.q0 * a.group;
    float2 sn = make_float2(-kNegInf, 0.f);
    RowLoads<T, D, Sh::ROWS, 4> ql, gl;
    ql.set(wave, a.q_row, a, a.q_head);
    gl.set(wave, a.do_row, a, a.do_head);
    auto request = [&](int r0, unsigned char *qt, unsigned char *gt) __attribute__((always_inline)) {
        ql.rows(a, qp, a.q_row, a.q_head, r0, rows, qt);
        gl.rows(a, gp, a.do_row, a.do_head, r0, rows, gt);
        if ((int)threadIdx.x < Sh::ROWS) sn = r0 + (int)threadIdx.x < rend ? sp[r0 + threadIdx.x] : make_float2(-kNegInf, 0.f);  // rows past the end: weights of zero
    };
    const float c = a.scale * kLog2e;
    auto park = [&](int b) __attribute__((always_inline)) {
        if ((int)threadIdx.x < Sh::ROWS) {
            st[b][0][threadIdx.x] = -sn.x / c;
            st[b][1][threadIdx.x] = -sn.y;
        }
    };
    floatx16_t dk[NB], dv[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) dk[nb] = dv[nb] = zero16();
    // Rows sub .. sub + 31 of a tile: their scores and dP, the statistics they need, the weights made of them
    struct Part {
        floatx16_t s, dp;
        Weights<T> p, ds;
    };
    // key j is seen by rows from (j - past) * group on
    const int first_seen = a.causal ? min(max(key - past, 0), sq.nq) * a.group : 0;
    auto mask = [&](Part &x, int r0, int sub) __attribute__((always_inline)) {
        const int lim = first_seen - r0 - sub - 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i) x.s[i] = 8 * (i >> 2) + (i & 3) >= lim ? x.s[i] : kNegInf;
    };
    auto statistics = [&](Part &x, int sub, int b) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 l = *reinterpret_cast<const float4 *>(&st[b][0][sub + 8 * g + 4 * half]);
            const float4 d = *reinterpret_cast<const float4 *>(&st[b][1][sub + 8 * g + 4 * half]);
            x.s[4 * g] = l.x; x.s[4 * g + 1] = l.y; x.s[4 * g + 2] = l.z; x.s[4 * g + 3] = l.w;
            x.dp[4 * g] = d.x; x.dp[4 * g + 1] = d.y; x.dp[4 * g + 2] = d.z; x.dp[4 * g + 3] = d.w;
        }
    };
    auto weigh = [&](Part &x, int j) __attribute__((always_inline)) {  // rows 2 j, 2 j + 1 of the lane's 16
        const float p0 = fast_exp2(x.s[2 * j] * c), p1 = fast_exp2(x.s[2 * j + 1] * c);
        x.p.set_pair(2 * j, p0, p1);
        x.ds.set_pair(2 * j, p0 * x.dp[2 * j], p1 * x.dp[2 * j + 1]);
    };
    auto tile = [&](int r0, const unsigned char *qt, const unsigned char *gt, int b) __attribute__((always_inline)) {
        // a wave has its SIMD to itself: one row of operands for all products of the tile, read RING steps ahead, and the weights of each half made
        // between products that do not need them
        constexpr int NS = 2 * NM, NW = 2 * RS::STEPS, N = 2 * NS + 2 * NW;
        Part x, y;
        bf16x8_t ring[RING];
        auto fetch = [&](auto at) __attribute__((always_inline)) {
            constexpr int k = decltype(at)::value;
            if constexpr (k < 2 * NS) {
                ring[k % RING] = row_frag<T, D>(k & 1 ? gt : qt, (k / NS) * 32 + n, (k % NS) / 2, half).v;
            } else {
                constexpr int j = k - 2 * NS;
                ring[k % RING] = RS::fetch((j % NW) < RS::STEPS ? gt : qt, (j / NW) * 32, j % RS::STEPS);
            }
        };
        auto use = [&](auto at, Part &z) __attribute__((always_inline)) {
            constexpr int k = decltype(at)::value;
            if constexpr (k < 2 * NS) {
                constexpr int m = (k % NS) / 2;
                if constexpr (k & 1) z.dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[k % RING], vf[m].v, z.dp, 0, 0, 0);
                else z.s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[k % RING], kf[m].v, z.s, 0, 0, 0);
            } else {
                constexpr int j = k - 2 * NS;
                if constexpr ((j % NW) < RS::STEPS) RS::step(j % RS::STEPS, ring[k % RING], z.p, dv);
                else RS::step(j % RS::STEPS, ring[k % RING], z.ds, dk);
            }
        };
        statistics(x, 0, b);
        static_for<RING>(fetch);
        pin_order();
        static_for<N>([&](auto at) __attribute__((always_inline)) {
            constexpr int k = decltype(at)::value;
            if constexpr (k < 2 * NS ? k < NS : k - 2 * NS < NW) use(at, x);
            else use(at, y);
            if constexpr (k + RING < N) fetch(std::integral_constant<int, k + RING>{});
            if constexpr (k == NS - 4) statistics(y, 32, b);
            if constexpr (CAUSAL && k == NS - 1) mask(x, r0, 0);
            if constexpr (CAUSAL && k == 2 * NS - 1) mask(y, r0, 32);
            if constexpr (k >= NS && k < 2 * NS && (k - NS) % (NS / 8) == NS / 8 - 1) weigh(x, (k - NS) / (NS / 8));
            if constexpr (k >= 2 * NS && k < 2 * NS + NW && (k - 2 * NS) % (NW / 8) == NW / 8 - 1) weigh(y, (k - 2 * NS) / (NW / 8));
            pin_order();
        });
    };
    if (rbeg < rend) {
        request(rbeg, qa, ga);
        park(0);
        for (int r0 = rbeg; r0 < rend; r0 += 2 * Sh::ROWS) {
            wait_loads_and_sync();
            if (r0 + Sh::ROWS < rend) request(r0 + Sh::ROWS, qb, gb);
            tile(r0, qa, ga, 0);
            if (r0 + Sh::ROWS < rend) {
                park(1);
                wait_loads_and_sync();
                if (r0 + 2 * Sh::ROWS < rend) request(r0 + 2 * Sh::ROWS, qa, ga);
                tile(r0 + Sh::ROWS, qb, gb, 1);
                if (r0 + 2 * Sh::ROWS < rend) park(0);
            }
        }
    }
    T *const kop = reinterpret_cast<T *>(reinterpret_cast<unsigned char *>(dK) + (int64_t)(sq.k0 + kc) * a.dk_row + (int64_t)hk * a.dk_head);
    T *const vop = reinterpret_cast<T *>(reinterpret_cast<unsigned char *>(dV) + (int64_t)(sq.k0 + kc) * a.dv_row + (int64_t)hk * a.dv_head);
    const int64_t pid = (((int64_t)(sq.k0 + kc) * a.Hkv + hk) * a.splits + split) * D;
    auto put_k = [&](int ch, float x, float y, float z, float w) __attribute__((always_inline)) {
        if (key >= sq.nk) return;
        if (a.splits > 1) store4(part_k + pid + ch, x * a.scale, y * a.scale, z * a.scale, w * a.scale);
        else store4(kop + ch, x * a.scale, y * a.scale, z * a.scale, w * a.scale);
    };
    auto put_v = [&](int ch, float x, float y, float z, float w) __attribute__((always_inline)) {
        if (key >= sq.nk) return;
        if (a.splits > 1) store4(part_v + pid + ch, x, y, z, w);
        else store4(vop + ch, x, y, z, w);
    };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int ch = 32 * nb + 8 * g + 4 * half;
            put_k(ch, dk[nb][4 * g], dk[nb][4 * g + 1], dk[nb][4 * g + 2], dk[nb][4 * g + 3]);
            put_v(ch, dv[nb][4 * g], dv[nb][4 * g + 1], dv[nb][4 * g + 2], dv[nb][4 * g + 3]);
        }
}

// Sums of the pieces.  KEYS: of dK and dV (blockIdx.y), pieces of the rows; else of dQ, pieces of the keys.
template <typename T, int D, bool KEYS, int GROUPS>
__global__ __launch_bounds__(256) void packed_sum_kernel(const float *__restrict__ p0, const float *__restrict__ p1, T *__restrict__ out0, T *__restrict__ out1, PackedArgs a)
{
    constexpr int LPR = D / 4;
    const int heads = KEYS ? a.Hkv : a.Hq, total = KEYS ? a.total_k : a.total_q;
    int tok, head;
    if (!merge_row<LPR, GROUPS>(total, heads, tok, head)) return;
    const int lane = threadIdx.x % LPR, grp = GROUPS > 1 ? threadIdx.x / LPR : 0;
    const Sequence sq = read_sequence(a, __builtin_amdgcn_readfirstlane(find_sequence(KEYS ? a.cu_k : a.cu_q, a.n_seq, total, 1, 0, tok)));
    const int t0 = KEYS ? sq.k0 : sq.q0, nt = KEYS ? sq.nk : sq.nq;
    if (tok < t0 || tok >= t0 + nt || head >= heads) return;
    // of rows that see the key, or of keys that the row sees
    const int first = KEYS && a.causal ? min(max(tok - t0 - (sq.nk - sq.nq), 0), sq.nq) * a.group / a.chunk : 0;
    const int pieces = KEYS ? (sq.nq * a.group + a.chunk - 1) / a.chunk : pieces_seen(a, sq, tok - t0);
    const bool second = KEYS && blockIdx.y;
    const float *p = (second ? p1 : p0) + ((int64_t)tok * heads + head) * a.splits * D + 4 * lane;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = first + grp; s < pieces; s += GROUPS) {
        const float4 x = *reinterpret_cast<const float4 *>(p + (int64_t)s * D);
        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    }
    join_groups<LPR, GROUPS>(v);
    if (grp > 0) return;
    const int64_t rb = KEYS ? (second ? a.dv_row : a.dk_row) : a.dq_row, hb = KEYS ? (second ? a.dv_head : a.dk_head) : a.dq_head;
    T *op = reinterpret_cast<T *>(reinterpret_cast<unsigned char *>(second ? out1 : out0) + (int64_t)tok * rb + (int64_t)head * hb);
    store4(op + 4 * lane, v[0], v[1], v[2], v[3]);
}
template <typename T, int D, bool KEYS> void launch_sum(const PackedArgs &a, const float *p0, const float *p1, T *out0, T *out1, hipStream_t st)
{
    constexpr int LPR = D / 4, G = 256 / LPR;
    const int64_t total = KEYS ? a.total_k : a.total_q;
    const int heads = KEYS ? a.Hkv : a.Hq;
    if (wide_merge(a.splits, total * heads))
        packed_sum_kernel<T, D, KEYS, G><<<merge_grid<LPR, G>(total, heads, KEYS ? 2 : 1), 256, 0, st>>>(p0, p1, out0, out1, a);
    else
        packed_sum_kernel<T, D, KEYS, 1><<<merge_grid<LPR, 1>(total, heads, KEYS ? 2 : 1), 256, 0, st>>>(p0, p1, out0, out1, a);
}

template <typename T, int D, int WK>
dsv_status launch_dq(const PackedArgs &a, const T *Q, const T *K, const T *V, const T *dO, const float2 *stat, T *dQ, float *part, hipStream_t st)
{
    const int64_t slots = tile_slots(a.total_q, a.group, BwdShape<T, D, WK>::OWN, a.n_seq);
    packed_dq_kernel<T, D, WK><<<dim3((unsigned)(slots * a.Hkv), a.splits), 256, 0, st>>>(Q, K, V, dO, stat, dQ, part, a);
    DSV_LAUNCH_CHECK();
    if (a.splits > 1) {
        launch_sum<T, D, false>(a, part, nullptr, dQ, nullptr, st);
        DSV_LAUNCH_CHECK();
    }
    return DSV_OK;
}

template <typename T, int D>
dsv_status launch_dkdv(const PackedArgs &a, bool few, const T *Q, const T *K, const T *V, const T *dO, const float2 *stat, T *dK, T *dV, float *part, hipStream_t st)
{
    few |= sizeof(T) == 4;
    const int64_t slots = tile_slots(a.total_k, 1, few ? BwdShape<T, D, 4>::OWN : BwdShape<T, D, 1>::OWN, a.n_seq);
    const dim3 grid((unsigned)(slots * a.Hkv), a.splits);
    float *const part_v = part + packed_dkdv_bytes(a.total_k, a.Hkv, D, a.splits) / 8;
    if constexpr (sizeof(T) == 2) {
        if (few) packed_dkdv_few_kernel<T, D><<<grid, 256, 0, st>>>(Q, K, V, dO, stat, dK, dV, part, part_v, a);
        else if (a.causal) packed_dkdv_kernel<D, true><<<grid, 256, 0, st>>>(Q, K, V, dO, stat, dK, dV, part, part_v, a);
        else packed_dkdv_kernel<D, false><<<grid, 256, 0, st>>>(Q, K, V, dO, stat, dK, dV, part, part_v, a);
    } else {
        packed_dkdv_few_kernel<T, D><<<grid, 256, 0, st>>>(Q, K, V, dO, stat, dK, dV, part, part_v, a);
    }
    DSV_LAUNCH_CHECK();
    if (a.splits > 1) {
        launch_sum<T, D, true>(a, part, part_v, dK, dV, st);
        DSV_LAUNCH_CHECK();
    }
    return DSV_OK;
}

template <typename T, int D>
dsv_status launch_t(PackedArgs a, const PackedBwdPlan &pl, const void *Qv, const void *Kv, const void *Vv, const void *Ov, const void *tail, const float *lse,
                    const void *dOv, void *dQv, void *dKv, void *dVv, char *ws, hipStream_t st)
{
    const T *Q = static_cast<const T *>(Qv), *K = static_cast<const T *>(Kv), *V = static_cast<const T *>(Vv), *dO = static_cast<const T *>(dOv);
    T *dQ = static_cast<T *>(dQv), *dK = static_cast<T *>(dKv), *dV = static_cast<T *>(dVv);
    float2 *const stat = reinterpret_cast<float2 *>(ws);
    float *const part = reinterpret_cast<float *>(ws + packed_stat_bytes(a.total_q, a.Hq));  // of dQ, then, when that is done, of dK and dV
    dsv_status s = DSV_OK;
    if (a.total_q > 0) {
        packed_stat_kernel<T, D><<<merge_grid<D *(int)sizeof(T) / 16, 1>(a.total_q, a.Hq), 256, 0, st>>>(static_cast<const T *>(Ov), static_cast<const T *>(tail), dO, lse, stat, a);
        DSV_LAUNCH_CHECK();
        a.splits = pl.splits_q;
        a.chunk = pl.chunk_q;
        s = pl.few_q ? launch_dq<T, D, 4>(a, Q, K, V, dO, stat, dQ, part, st) : launch_dq<T, D, 1>(a, Q, K, V, dO, stat, dQ, part, st);
        if (s != DSV_OK) return s;
    }
    if (a.total_k > 0) {
        a.splits = pl.splits_k;
        a.chunk = pl.chunk_k;
        s = launch_dkdv<T, D>(a, pl.few_k, Q, K, V, dO, stat, dK, dV, part, st);
    }
    return s;
}
}  // namespace

dsv_status launch_packed_bwd(const PackedArgs &a, const PackedBwdPlan &plan, int dtype, int d, const void *Q, const void *K, const void *V, const void *O,
                             const void *O_tail, const float *lse, const void *dO, void *dQ, void *dK, void *dV, char *ws, hipStream_t st)
{
    if (dtype == DSV_BF16)
        return d == 128 ? launch_t<bf16_t, 128>(a, plan, Q, K, V, O, O_tail, lse, dO, dQ, dK, dV, ws, st) : launch_t<bf16_t, 64>(a, plan, Q, K, V, O, O_tail, lse, dO, dQ, dK, dV, ws, st);
    return d == 128 ? launch_t<float, 128>(a, plan, Q, K, V, O, nullptr, lse, dO, dQ, dK, dV, ws, st) : launch_t<float, 64>(a, plan, Q, K, V, O, nullptr, lse, dO, dQ, dK, dV, ws, st);
}

}  // namespace dsv
