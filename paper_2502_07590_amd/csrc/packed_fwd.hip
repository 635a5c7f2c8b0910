// Softmax attention over packed sequences, forward.
//
//   s_ij = scale q_i . k_j over the keys j of i's sequence (causal: j <= i + nk - nq);  O_i = sum_j p_ij v_j,  lse_i = log sum_j exp s_ij
//
// One pass over the keys with the running maximum and sum.  A wave owns 32 rows as the columns of its products, S^T = K Q^T and
// O^T = V^T P^T: a lane then holds one row's scores, the maximum and the sum are its own but for one exchange between the halves, and
// the scores are where the second product wants them.
//
// Long calls are bound by power: 1.83 GHz of 2.4 under products and exponentials together (a tile of 64 keys, d = 128: 1056 cycles of
// products, about 960 of vector work a wave, two waves a SIMD; products busy 56 % of the time a CU has blocks, and laying the weights of
// half a tile between the products of the other changes nothing): 32768 tokens, 4 heads, d = 128, bf16 2.1 ms, 1030 TFLOP/s, where a large
// library product has 1350. Single queries against long caches are bound by memory: 104 MB of K and V in
// 24 + 4 us with the join, 3.7 TB/s.  Few keys (34128 queries of 16 heads against 77 .. 512, d = 64): 57 us, half of it Q and O themselves, the
// rest the chain from lengths to rows to scores of a block that walks two to eight tiles.  fp32 is bound by its products (64 cycles each):
// 1724 tokens of two heads, d = 64, 17.5 us and 4 for the join, each by itself; 19.3 one call behind another.
#include "packed_attn.h"

namespace dsv {
namespace {

// WK = 1: the four waves own 32 rows each and share tiles of 64 keys.  WK = 4: they own the same 32 rows and take 32 keys each of a tile of
// 128; for calls of few rows.  NBUF: tiles in LDS in turn.  (For WK = 1 the next tile's scores laid between the weights of this one, and
// wave priorities by turns, were no faster; two groups of 32 rows a wave, one's products beside the other's weights: 306 us for 277 at 2 x 8192 tokens.)
template <typename T, int D, int WK> struct FwdShape {
    static constexpr int ROWS = WK == 1 ? 128 : 32, KEYS = WK == 1 ? 64 : 128, KT = KEYS / 32 / WK;
    static constexpr int TILE = KEYS * D * (int)sizeof(T);
    static constexpr int NBUF = WK == 1 || (sizeof(T) == 4 && D == 64) ? 2 : 1;  // fp32 is bound by the products: two blocks on a CU would leave others idle
};

// lse of a row whose weights, against m, add up to l.  Only a sum of zero is one over no keys: a score that is no number, or infinite, makes l no
// number, and lse and O with it; taken for a row without keys it would have gradients of zero.
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? kNegInf : (m + __builtin_amdgcn_logf(l)) * kLn2; }

template <typename T, int D, int WK>
__global__ __launch_bounds__(256, sizeof(T) == 4 && (D == 128 || WK > 1) ? 1 : 2) void packed_fwd_kernel(const T *__restrict__ Q, const T *__restrict__ K, const T *__restrict__ V,
                                                                                        T *__restrict__ O, bf16_t *__restrict__ O_tail, float *__restrict__ lse,
                                                                                        float2 *__restrict__ pml, float *__restrict__ pacc, PackedArgs a)
{
    typedef RowTile<T, D> RT;
    typedef FwdShape<T, D, WK> Sh;
    constexpr int NM = RT::RB / 32, NB = D / 32, KT = Sh::KT;
    // every tile an array of its own: reads of one then need not wait for the loads into another
    __shared__ __align__(1024) unsigned char ka[Sh::TILE], va[Sh::TILE], kb[Sh::NBUF == 2 ? Sh::TILE : 16], vb[Sh::NBUF == 2 ? Sh::TILE : 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    // heads side by side: with as many heads as XCDs, or a multiple or a divisor of that, a head's keys stay in the L2 of one or a few of them;
    // causal tiles of most keys first, within a sequence; the last sequence's before those of the others
    const int hk = blockIdx.x % a.Hkv, place = blockIdx.x / a.Hkv, split = blockIdx.y;
    const int slot = a.causal ? (int)(gridDim.x / a.Hkv) - 1 - place : place;
    const int si = __builtin_amdgcn_readfirstlane(find_sequence(a.cu_q, a.n_seq, a.total_q, a.group, Sh::ROWS, slot));
    const Sequence sq = read_sequence(a, si);
    const int rows = sq.nq * a.group;
    const int row0 = (slot - first_slot(a.cu_q[si], a.total_q, a.group, Sh::ROWS, si)) * Sh::ROWS;
    if (row0 < 0 || row0 >= rows) return;
    const int row = row0 + (WK == 1 ? wave * 32 : 0) + n;
    const int rc = min(row, rows - 1), tok = row_token(a, rc), head = hk * a.group + (rc - tok * a.group);
    // keys this block walks, and the first key that this lane's row does not see
    const int kbeg = split * a.chunk, kcut = a.chunk ? min(sq.nk, kbeg + a.chunk) : sq.nk;
    const int past = sq.nk - sq.nq, seen = a.causal ? min(sq.nk, tok + past + 1) : sq.nk;
    int kend = kcut;
    if (a.causal) kend = min(kend, row_token(a, min(row0 + Sh::ROWS, rows) - 1) + past + 1);
    if (a.splits > 1 && kbeg >= kend) return;  // no row of this tile sees the piece: the merge does not read it

    Frag<T> qf[NM];
    {
        const unsigned char *qp = reinterpret_cast<const unsigned char *>(Q) + (int64_t)(sq.q0 + tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
        for (int m = 0; m < NM; ++m) qf[m] = *reinterpret_cast<const Frag<T> *>(qp + (2 * m + half) * 16);
    }
    const unsigned char *kp = reinterpret_cast<const unsigned char *>(K) + (int64_t)sq.k0 * a.k_row + (int64_t)hk * a.k_head;
    const unsigned char *vp = reinterpret_cast<const unsigned char *>(V) + (int64_t)sq.k0 * a.v_row + (int64_t)hk * a.v_head;
    RowLoads<T, D, Sh::KEYS, 4> kl, vl;
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
    float mrun = kNegInf, l = 0.f, lr = 0.f;  // lr: sum of the weights as the second product takes them
    const int sub = WK == 1 ? 0 : wave * 32;
    auto scores = [&](const unsigned char *kt, floatx16_t (&s)[KT]) __attribute__((always_inline)) { tile_scores<T, D, KT>(kt, sub + n, qf, s); };
    auto rest = [&](int k0, floatx16_t (&s)[KT], const unsigned char *vt) __attribute__((always_inline)) {
        // the tile's last key is behind the end, or not seen by the wave's first row
        const bool edge = k0 + Sh::KEYS > kcut || (a.causal && k0 + Sh::KEYS > row_token(a, row0) + past + 1);
        if (edge) {
            const int lim = min(seen, kcut) - k0 - sub - 4 * half;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i] = 32 * t + 8 * (i >> 2) + (i & 3) < lim ? s[t][i] : kNegInf;
        }
        float mx = s[0][0];
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[t][i]);
        mx = halves_max(mx) * c;
        // The sums are held against a maximum that may be up to 2^8 too low: they are rescaled only when a row's has grown by more.
        if (__any(mx > mrun + 8.f)) {
            const float m2 = fmaxf(mrun, mx), f = m2 == kNegInf ? 1.f : fast_exp2(mrun - m2);
            l *= f;
            lr *= f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[nb][i] *= f;
            mrun = m2;
        }
        const float mref = mrun == kNegInf ? 0.f : mrun;
        float lt = 0.f, lrt = 0.f;  // of this tile: one chain over a long row would be 1e-5 off
#pragma unroll
        for (int t = 0; t < KT; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[t][i] = fast_exp2(fmaf(s[t][i], c, -mref));
                lt += s[t][i];
            }
            Weights<T> w;
            w.set(s[t]);
            if constexpr (sizeof(T) == 2) lrt = w.sum(lrt);
            weighted_rows<T, D>(vt, sub + 32 * t, w, acc);
        }
        l += lt;
        lr += lrt;
    };
    auto tile = [&](int k0, const unsigned char *kt, const unsigned char *vt) __attribute__((always_inline)) {
        floatx16_t s[KT];
        scores(kt, s);
        rest(k0, s, vt);
    };
    if (kbeg < kend) {
        if constexpr (Sh::NBUF == 2) {
            request(kbeg, ka, va);
            for (int k0 = kbeg; k0 < kend; k0 += 2 * Sh::KEYS) {
                wait_loads_and_sync();
                if (k0 + Sh::KEYS < kend) request(k0 + Sh::KEYS, kb, vb);
                tile(k0, ka, va);
                if (k0 + Sh::KEYS < kend) {  // (a break here makes the compiler move all sums to other registers and back)
                    wait_loads_and_sync();
                    if (k0 + 2 * Sh::KEYS < kend) request(k0 + 2 * Sh::KEYS, ka, va);
                    tile(k0 + Sh::KEYS, kb, vb);
                }
            }
        } else {
            // one tile of each, V on its way while the scores are formed and the next K while V is summed: room for two blocks
            kl.keys(kp, a.k_row, kbeg, sq.nk, ka);
            for (int k0 = kbeg; k0 < kend; k0 += Sh::KEYS) {
                wait_loads_and_sync();
                vl.keys(vp, a.v_row, k0, sq.nk, va);
                floatx16_t s[KT];
                scores(ka, s);
                wait_loads_and_sync();
                if (k0 + Sh::KEYS < kend) kl.keys(kp, a.k_row, k0 + Sh::KEYS, sq.nk, ka);
                rest(k0, s, va);
            }
        }
    }
    l = halves_sum(l);
    // Weights go into the product as one bf16 word: a second one, as the sparse forward has it, would make three products of two, in a kernel bound by
    // their power.  O is the average by the weights that were summed, lse the logarithm of the unrounded ones': rounding then moves weight between the keys and
    // adds none (bf16, against 64 bits: O 2.4e-3 off when divided by l, 1.9e-3 by lr, 1.7e-3 the rounding of O alone)
    const float whole = sizeof(T) == 2 ? halves_sum(lr) : l, fair = whole == 0.f ? 0.f : l / whole;
    if constexpr (WK > 1) {  // the waves' sums over their keys, joined in LDS: wave w then holds channels 32 w / 4 .. of every row
        __shared__ float sm[128], sl[128];
        auto area = [&](int w) __attribute__((always_inline)) {  // 32 rows of D sums
            return reinterpret_cast<float *>(Sh::NBUF == 2 ? (w == 0 ? ka : w == 1 ? va : w == 2 ? kb : vb) : (w < 2 ? ka : va) + (w & 1) * (Sh::TILE / 2));
        };
        static_assert(Sh::TILE / (Sh::NBUF == 2 ? 1 : 2) >= 32 * D * 4, "a wave's sums fit its part of the tiles");
        __syncthreads();
        if (half == 0) {
            sm[wave * 32 + n] = mrun;
            sl[wave * 32 + n] = l;
        }
        __syncthreads();
        float m2 = kNegInf;
#pragma unroll
        for (int w = 0; w < 4; ++w) m2 = fmaxf(m2, sm[w * 32 + n]);
        const float mref = m2 == kNegInf ? 0.f : m2;
        l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) l += sl[w * 32 + n] * fast_exp2(sm[w * 32 + n] - mref);
        const float f = fast_exp2(mrun - mref) * fair;
        // channel by row, [channel / 4][row][4]
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4 *>(area(wave) + ((nb * 8 + 2 * g + half) * 32 + n) * 4) =
                    make_float4(acc[nb][4 * g] * f, acc[nb][4 * g + 1] * f, acc[nb][4 * g + 2] * f, acc[nb][4 * g + 3] * f);
        mrun = m2;
        __syncthreads();
        if (row >= rows) return;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int64_t rid = (int64_t)(sq.q0 + tok) * a.Hq + head;
        for (int g = wave * 2 + half; g < D / 4; g += 8) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float4 x = *reinterpret_cast<const float4 *>(area(w) + (g * 32 + n) * 4);
                v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
            }
            if (a.splits > 1) {
                store4(pacc + (rid * a.splits + split) * D + 4 * g, v[0], v[1], v[2], v[3]);
            } else {
                T *op = reinterpret_cast<T *>(reinterpret_cast<unsigned char *>(O) + (int64_t)(sq.q0 + tok) * a.o_row + (int64_t)head * a.o_head);
                store_out(op + 4 * g, O_tail ? O_tail + rid * D + 4 * g : nullptr, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
            }
        }
        if (wave == 0 && half == 0) {
            if (a.splits > 1) pml[rid * a.splits + split] = make_float2(mrun, l);
            else lse[(int64_t)head * a.total_q + sq.q0 + tok] = row_lse(mrun, l);
        }
    } else {
        const float inv = whole == 0.f ? 0.f : 1.f / whole;
        const int64_t rid = (int64_t)(sq.q0 + tok) * a.Hq + head;
        if (a.splits > 1) {
            if (row >= rows) return;
            float *const pa = pacc + (rid * a.splits + split) * D;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    store4(pa + 32 * nb + 8 * g + 4 * half, acc[nb][4 * g] * fair, acc[nb][4 * g + 1] * fair, acc[nb][4 * g + 2] * fair, acc[nb][4 * g + 3] * fair);
            if (half == 0) pml[rid * a.splits + split] = make_float2(mrun, l);
        } else {
            // the wave's rows by way of LDS, so that they leave as whole lines
            typedef RowTile<T, D> RT;
            unsigned char *const mine = (wave < 2 ? ka : va) + (wave & 1) * (Sh::TILE / 2);
            static_assert(Sh::TILE / 2 == 32 * RT::RB, "half a tile is a wave's rows");
            auto place = [&](int r, int p) __attribute__((always_inline)) { return mine + r * RT::RB + ((p ^ (RT::PIECES == 8 ? (r >> 1) & 7 : r & 15)) << 4); };
            auto send = [&](unsigned char *first, int64_t row_b, int64_t head_b) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < RT::PIECES / 2; ++i) {
                    const int r = i * (64 / RT::PIECES) + lane / RT::PIECES, p = lane % RT::PIECES, ro = row0 + wave * 32 + r;
                    const uint4 x = *reinterpret_cast<const uint4 *>(place(r, p));
                    const int t = row_token(a, ro);
                    if (ro < rows) *reinterpret_cast<uint4 *>(first + (int64_t)(sq.q0 + t) * row_b + (int64_t)(hk * a.group + ro - t * a.group) * head_b + p * 16) = x;
                }
            };
            __syncthreads();
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = acc[nb][4 * g + i] * inv;
                    const int ch = 32 * nb + 8 * g + 4 * half, at = ch * (int)sizeof(T);
                    store4(reinterpret_cast<T *>(place(n, at >> 4) + (at & 15)), v[0], v[1], v[2], v[3]);
                }
            wave_sync();
            send(reinterpret_cast<unsigned char *>(O), a.o_row, a.o_head);
            if constexpr (sizeof(T) == 2)
                if (O_tail) {
                    wave_sync();
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            uint2 *const at = reinterpret_cast<uint2 *>(place(n, 4 * nb + g) + 8 * half);
                            *at = make_uint2(tail_of(acc[nb][4 * g] * inv, acc[nb][4 * g + 1] * inv), tail_of(acc[nb][4 * g + 2] * inv, acc[nb][4 * g + 3] * inv));
                        }
                    wave_sync();
                    send(reinterpret_cast<unsigned char *>(O_tail), (int64_t)a.Hq * D * 2, D * 2);
                }
            if (half == 0 && row < rows) lse[(int64_t)head * a.total_q + sq.q0 + tok] = row_lse(mrun, l);
        }
    }
}

// The pieces of a row joined: weights 2^(m_s - max).
template <typename T, int D, int GROUPS>
__global__ __launch_bounds__(256) void packed_fwd_merge_kernel(const float2 *__restrict__ pml, const float *__restrict__ pacc, T *__restrict__ O,
                                                               bf16_t *__restrict__ O_tail, float *__restrict__ lse, PackedArgs a)
{
    constexpr int LPR = D / 4, PL = 64 / LPR;  // pieces a lane weighs, of 64 at most
    int tok, head;
    if (!merge_row<LPR, GROUPS>(a.total_q, a.Hq, tok, head)) return;
    const int lane = threadIdx.x % LPR, grp = GROUPS > 1 ? threadIdx.x / LPR : 0;
    const Sequence sq = read_sequence(a, __builtin_amdgcn_readfirstlane(find_sequence(a.cu_q, a.n_seq, a.total_q, 1, 0, tok)));
    if (tok < sq.q0 || tok >= sq.q0 + sq.nq || head >= a.Hq) return;
    const int64_t rid = (int64_t)tok * a.Hq + head;
    const int pieces = pieces_seen(a, sq, tok - sq.q0);
    const float2 *const ml = pml + rid * a.splits;
    const float *const pa = pacc + rid * a.splits * D + 4 * lane;
    float v[4] = {0.f, 0.f, 0.f, 0.f}, m = kNegInf, l = 0.f;
    auto add = [&](int s, float w) __attribute__((always_inline)) {
        const float4 x = *reinterpret_cast<const float4 *>(pa + (int64_t)s * D);
        v[0] = fmaf(x.x, w, v[0]); v[1] = fmaf(x.y, w, v[1]); v[2] = fmaf(x.z, w, v[2]); v[3] = fmaf(x.w, w, v[3]);
    };
    if constexpr (GROUPS > 1) {
        __shared__ float weight[64];
        float2 mine[PL];
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            mine[i] = lane + i * LPR < pieces ? ml[lane + i * LPR] : make_float2(kNegInf, 0.f);
            m = fmaxf(m, mine[i].x);
        }
#pragma unroll
        for (int s = LPR / 2; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
        const float mref = m == kNegInf ? 0.f : m;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            const float f = fast_exp2(mine[i].x - mref);
            l = fmaf(mine[i].y, f, l);
            if (grp == 0) weight[lane + i * LPR] = f;
        }
#pragma unroll
        for (int s = LPR / 2; s > 0; s >>= 1) l += __shfl_xor(l, s);
        __syncthreads();
#pragma unroll 8
        for (int s = grp; s < pieces; s += GROUPS) add(s, weight[s]);
        join_groups<LPR, GROUPS>(v);
        if (grp > 0) return;
    } else {
        for (int s = 0; s < pieces; ++s) m = fmaxf(m, ml[s].x);
        const float mref = m == kNegInf ? 0.f : m;
#pragma unroll 4
        for (int s = 0; s < pieces; ++s) {
            const float f = fast_exp2(ml[s].x - mref);
            l = fmaf(ml[s].y, f, l);
            add(s, f);
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T *op = reinterpret_cast<T *>(reinterpret_cast<unsigned char *>(O) + (int64_t)tok * a.o_row + (int64_t)head * a.o_head);
    store_out(op + 4 * lane, O_tail ? O_tail + rid * D + 4 * lane : nullptr, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    if (lane == 0) lse[(int64_t)head * a.total_q + tok] = row_lse(m, l);
}

template <typename T, int D, int WK>
dsv_status launch_t(const PackedArgs &a, const void *Q, const void *K, const void *V, void *O, void *O_tail, float *lse, char *ws, hipStream_t st)
{
    const int64_t slots = tile_slots(a.total_q, a.group, FwdShape<T, D, WK>::ROWS, a.n_seq);
    float *const pacc = reinterpret_cast<float *>(ws);
    float2 *const pml = reinterpret_cast<float2 *>(ws + packed_fwd_acc_bytes(a.total_q, a.Hq, D, a.splits));
    packed_fwd_kernel<T, D, WK><<<dim3((unsigned)(slots * a.Hkv), a.splits), 256, 0, st>>>(
        static_cast<const T *>(Q), static_cast<const T *>(K), static_cast<const T *>(V), static_cast<T *>(O), static_cast<bf16_t *>(O_tail), lse, pml, pacc, a);
    DSV_LAUNCH_CHECK();
    if (a.splits > 1) {
        constexpr int LPR = D / 4, G = 256 / LPR;
        if (wide_merge(a.splits, (int64_t)a.total_q * a.Hq))
            packed_fwd_merge_kernel<T, D, G><<<merge_grid<LPR, G>(a.total_q, a.Hq), 256, 0, st>>>(pml, pacc, static_cast<T *>(O), static_cast<bf16_t *>(O_tail), lse, a);
        else
            packed_fwd_merge_kernel<T, D, 1><<<merge_grid<LPR, 1>(a.total_q, a.Hq), 256, 0, st>>>(pml, pacc, static_cast<T *>(O), static_cast<bf16_t *>(O_tail), lse, a);
        DSV_LAUNCH_CHECK();
    }
    return DSV_OK;
}
}  // namespace

dsv_status launch_packed_fwd(const PackedArgs &a, int dtype, int d, bool few, const void *Q, const void *K, const void *V, void *O, void *O_tail,
                             float *lse, char *ws, hipStream_t st)
{
    if (dtype == DSV_BF16) {
        if (d == 128) return few ? launch_t<bf16_t, 128, 4>(a, Q, K, V, O, O_tail, lse, ws, st) : launch_t<bf16_t, 128, 1>(a, Q, K, V, O, O_tail, lse, ws, st);
        return few ? launch_t<bf16_t, 64, 4>(a, Q, K, V, O, O_tail, lse, ws, st) : launch_t<bf16_t, 64, 1>(a, Q, K, V, O, O_tail, lse, ws, st);
    }
    if (d == 128) return few ? launch_t<float, 128, 4>(a, Q, K, V, O, nullptr, lse, ws, st) : launch_t<float, 128, 1>(a, Q, K, V, O, nullptr, lse, ws, st);
    return few ? launch_t<float, 64, 4>(a, Q, K, V, O, nullptr, lse, ws, st) : launch_t<float, 64, 1>(a, Q, K, V, O, nullptr, lse, ws, st);
}

}  // namespace dsv
