// Keys out of the pages of an 8-bit cache, for the forward of attention.  Values are widened with their page's scale by the conversion itself
// (v_cvt_scalef32; exact, the scales being powers of two).  Pages begin on multiples of 16 tokens, so 16 keys in a row have one page.
//
// Values of 8 bits are bf16 ones, whatever the queries' type; fp32 queries and weights go into the products as three bf16 words, 24 bits, whose
// products with them are exact in the 32-bit sums: three bf16 products where eight of fp32 would take five times as long.
//
// The weights of a bf16 call: two words, 16 bits, in blocks of 32 rows, which are bound by memory (caches as below, d = 128, captured, us, two words and one: 64 of
// 2047 .. 19948 86 and 86, twelve of 1 .. 16001 24.7 and 23.9, 24 of 6000 .. 8300 with four queries each 89.1 and 88.0; eight of 900 14.2 and 13.5); one in
// blocks of 128, which are bound by the products (2 x 1560 queries on 21840 and 7800 332 and 263; 4 x 4096 on 32768, 32 heads on eight 12514 and 9764).
#pragma once

#include "cache.h"

namespace dsv {

struct CachedArgs : PackedArgs {
    CacheArgs c;
    const uint8_t *K8, *V8;
    const float *kscale, *vscale;
};
__device__ __forceinline__ Sequence read_sequence(const CachedArgs &a, int i) { return read_cached(a.c, i); }

dsv_status launch_cache_fwd(const CachedArgs &a, int dtype, int d, bool few, const void *Q, void *O, float *lse, char *ws, hipStream_t st);

// Values of 8 bits as operands of the products: 8 of them in bf16, 4 in fp32.
__device__ __forceinline__ bf16x8_t widen8(uint32_t lo, uint32_t hi, float s)
{
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
    return __builtin_bit_cast(bf16x8_t, make_uint4(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
                                                   __builtin_bit_cast(uint32_t, d)));
}

// fp32 as bf16 words, the largest first; what is left behind the last is below 2^-24 of the whole.
constexpr int words_of(int bytes) { return bytes == 4 ? 3 : 1; }
template <typename T, int D> struct OwnRows;
template <int D> struct OwnRows<bf16_t, D> {  // as they are
    Frag<bf16_t> w[1][D / 16];
    __device__ __forceinline__ void set(const Frag<bf16_t> (&q)[D / 16])
    {
#pragma unroll
        for (int m = 0; m < D / 16; ++m) w[0][m] = q[m];
    }
};
template <int D> struct OwnRows<float, D> {
    Frag<bf16_t> w[3][D / 16];
    __device__ __forceinline__ void set(const Frag<float> (&q)[D / 8])
    {
#pragma unroll
        for (int m = 0; m < D / 16; ++m) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = q[2 * m + (i >> 2)].v[i & 3];
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                uint32_t p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
                    x[2 * i] -= __uint_as_float(p[i] << 16);
                    x[2 * i + 1] -= __uint_as_float(p[i] & 0xFFFF0000u);
                }
                w[k][m].v = __builtin_bit_cast(bf16x8_t, make_uint4(p[0], p[1], p[2], p[3]));
            }
        }
    }
};
// Weights as N bf16 words.
template <int N> struct WeightWords {
    Weights<bf16_t> w[N];
    __device__ __forceinline__ explicit WeightWords(const Weights<bf16_t> &x)
    {
        static_assert(N == 1, "rounded already");
        w[0] = x;
    }
    __device__ __forceinline__ explicit WeightWords(const Weights<float> &x)
    {
        floatx16_t r = x.v;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            w[k].set(r);
            if (k + 1 == N) break;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint4 h = __builtin_bit_cast(uint4, w[k].v[s]);
                const uint32_t p[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    r[8 * s + 2 * i] -= __uint_as_float(p[i] << 16);
                    r[8 * s + 2 * i + 1] -= __uint_as_float(p[i] & 0xFFFF0000u);
                }
            }
        }
    }
};
// Which 16 bytes of Q hold channels c .. of step m: bf16 eight of them, fp32 four, two such to a step of eight.
template <typename T> __device__ __forceinline__ int piece_of(int channel, int m) { return sizeof(T) == 2 ? channel / 8 : channel / 4 + (m & 1); }

// Transposing LDS read of bytes (ds_read_b64_tr_b8): inside every block of 16 lanes, lane i receives eight bytes, the e-th being byte i % 8 at the
// address passed by lane 2 e + i / 8 of the block.
typedef int32_t s32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s32x2_t lds_s32x2_t;

// For blocks of 32 rows whose four waves share the keys: every wave reads 32 keys of its own, K straight into the products' registers, V by way of
// LDS of its own, turned there; no wave waits for another.  The next 32 keys' bytes, and the pages of those after them, are on their way meanwhile.
// Bound by memory: 64 caches of 2047 .. 19948, two heads, group 7, d = 128: 81 us, 4.3 TB/s (tiles that the four waves laid into LDS together: 126).
template <typename T, int D> struct PageWaves {
    typedef FwdShape<bf16_t, D, 4> Sh;
    typedef Weights<float> W;
    static constexpr int NK = D / 32;                  // 16-byte pieces of a key to a lane: the pieces 2 j + half, two steps of the products each
    static constexpr int PPR = D / 16, RPL = 64 / PPR; // pieces of a key, keys of a load of V
    static constexpr int WORDS = words_of(sizeof(T));
    static constexpr int WEIGHT_WORDS = sizeof(T) == 2 ? 2 : 3;  // the second costs up to 0.8 us; a bf16 weight's rounding would be as large as O's
    struct Step {
        uint4 k[NK], v[NK];
        float ks, vs[2];
        int k0;
    };
    const CachedArgs &a;
    const int32_t *pages;
    unsigned char *vt;
    int hk, wave, last_page, nk, pg[2];
    OwnRows<T, D> own;

    __device__ __forceinline__ explicit PageWaves(const CachedArgs &args) : a(args) {}
    __device__ __forceinline__ static int piece(int m, int half)
    {
        const int step = sizeof(T) == 2 ? m : m / 2;
        return piece_of<T>(16 * (2 * (step / 2) + half) + 8 * (step & 1), m);
    }
    __device__ __forceinline__ void begin(const CachedArgs &, int si, const Sequence &sq, int hk_, int wave_, const Frag<T> (&q)[D * sizeof(T) / 32])
    {
        own.set(q);
        hk = hk_;
        wave = wave_;
        nk = sq.nk;
        last_page = max(0, (sq.nk - 1) >> a.c.page_log2);
        pages = a.c.table + (int64_t)si * a.c.max_pages;
    }
    __device__ __forceinline__ void find_pages(int k0)
    {
#pragma unroll
        for (int g = 0; g < 2; ++g) pg[g] = min(max(pages[min((k0 + 16 * g) >> a.c.page_log2, last_page)], 0), a.c.n_pages - 1);
    }
    // the bytes of keys k0 .. + 31, whose pages were found; and the pages of keys `then`
    __device__ __forceinline__ void request(int k0, int then, Step &st)
    {
        const int lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5, mask = a.c.page - 1;
        const int64_t of0 = (int64_t)pg[0] * a.Hkv + hk, of1 = (int64_t)pg[1] * a.Hkv + hk, page_b = (int64_t)a.c.page * D;
        const int64_t at0 = of0 * page_b + (int64_t)(k0 & mask) * D, at1 = of1 * page_b + (int64_t)((k0 + 16) & mask) * D;  // of keys 0 and 16
        st.k0 = k0;
        const uint8_t *const kp = a.K8 + (n < 16 ? at0 : at1) + (n & 15) * D + half * 16;
#pragma unroll
        for (int j = 0; j < NK; ++j) st.k[j] = *reinterpret_cast<const uint4 *>(kp + 32 * j);
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int r0 = i * RPL;  // 8 or 16 keys of one half
            st.v[i] = *reinterpret_cast<const uint4 *>(a.V8 + (r0 < 16 ? at0 : at1) + (r0 & 15) * D + lane * 16);
        }
        st.ks = n < 16 ? a.kscale[of0] : a.kscale[of1];
        st.vs[0] = a.vscale[of0];
        st.vs[1] = a.vscale[of1];
        find_pages(then);
    }
    // V's rows in LDS: piece p at place p ^ turn(r), so that the 16 rows of a transposing read lie over all banks
    __device__ __forceinline__ static int at(int r, int p) { return r * D + ((p ^ (D == 128 ? 2 * ((r >> 1) & 3) : 2 * ((r >> 2) & 1))) << 4); }
    __device__ __forceinline__ void scores(const Step &st, int, const Frag<T> (&)[D * sizeof(T) / 32], floatx16_t (&s)[1]) const
    {
        s[0] = zero16();
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            const uint32_t w[4] = {st.k[j].x, st.k[j].y, st.k[j].z, st.k[j].w};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const Frag<bf16_t> f{widen8(w[2 * i], w[2 * i + 1], st.ks)};
#pragma unroll
                for (int k = WORDS - 1; k >= 0; --k) s[0] = product(f, own.w[k][2 * j + i], s[0]);
            }
        }
    }
    __device__ __forceinline__ void add(const Step &st, int, const W &weights, floatx16_t (&acc)[D / 32]) const
    {
        const int lane = threadIdx.x & 63, e = (lane >> 1) & 7, half = lane >> 5;
        const int r = (e < 4 ? e : 4 + e) + 4 * half, p = (lane >> 4) & 1, sub = (lane & 1) * 8;
        const WeightWords<WEIGHT_WORDS> w(weights);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int nb = 0; nb < D / 32; ++nb) {
                const s32x2_t x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_s32x2_t *)(vt + at(16 * g + r, 2 * nb + p) + sub));
                const bf16x8_t v = widen8((uint32_t)x[0], (uint32_t)x[1], st.vs[g]);
#pragma unroll
                for (int k = WEIGHT_WORDS - 1; k >= 0; --k) acc[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w.w[k].v[g], acc[nb], 0, 0, 0);
            }
    }
    template <typename Scores, typename Rest>
    __device__ __forceinline__ void walk(const CachedArgs &, int kbeg, int kend, unsigned char *ka, unsigned char *va, unsigned char *kb, unsigned char *vb, Scores scores,
                                         Rest rest)
    {
        vt = (wave & 2 ? va : ka) + (wave & 1) * (Sh::TILE / 2);
        const int mine = 32 * wave;  // of the block's 128 keys
        auto run = [&](int k0, Step &st) __attribute__((always_inline)) {
            const int lane = threadIdx.x & 63;
            const bool edge = st.k0 + 32 > nk;
            wave_sync();  // reads of the keys before are done with
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                const int r = i * RPL + lane / PPR;
                // behind the sequence's end zeros, whatever the page holds there (a weight of zero times a NaN is one)
                if (edge && st.k0 + r >= nk) st.v[i] = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4 *>(vt + at(r, lane % PPR)) = st.v[i];
            }
            wave_sync();
            floatx16_t s[1];
            scores(st, s);
            rest(k0, s, st);
        };
        if (kbeg + mine >= kend) return;
        Step one, two;
        find_pages(kbeg + mine);
        request(kbeg + mine, kbeg + 128 + mine, one);
        for (int k0 = kbeg; k0 + mine < kend; k0 += 256) {
            if (k0 + 128 + mine < kend) request(k0 + 128 + mine, k0 + 256 + mine, two);
            run(k0, one);
            if (k0 + 128 + mine < kend) {
                if (k0 + 256 + mine < kend) request(k0 + 256 + mine, k0 + 384 + mine, one);
                run(k0 + 128, two);
            }
        }
    }
};

// For blocks of 128 rows: the waves bring the bytes of the tile after next into registers while one is worked on, and widen and lay those of the next
// into LDS, as rows loaded directly would be, between the products of this one's scores.  A load of a wave is one kilobyte of one page, so its page
// and scales are the wave's.  Two streams of 1560 queries on 21840 and 7800 keys, eight heads on two, d = 128, bf16: 263 us a call (nine pieces).  Of a kernel
// of 287 us (eight pieces, traced) the widening with its writes took 25, the loads 20, both together 67.  Bytes two tiles ahead: 265
// against 257; eight waves to 256 rows, each with half of the widening: 242 to 287 by how their rounds fall, against 256.
template <typename T, int D> struct PageTiles {
    typedef FwdShape<bf16_t, D, 1> Sh;
    typedef RowTile<bf16_t, D> RT;
    typedef Weights<T> W;
    static constexpr int WORDS = words_of(sizeof(T));
    static constexpr int RPL = 1024 / D, PPR = D / 16;     // tokens of a load, 16-byte pieces of a token
    static constexpr int N = Sh::KEYS / RPL / 4;           // loads of a wave for a tile of K, and of V
    const CachedArgs &a;
    const int32_t *pages;
    int hk, wave, last_page, nk, row, piece_no;
    uint4 raw[2 * N];                                       // K's, then V's
    float scale[2 * N];
    int at0, pg[N];
    uint32_t of_lane;
    unsigned char *next_k, *next_v;
    bool more;
    OwnRows<T, D> own;

    __device__ __forceinline__ explicit PageTiles(const CachedArgs &args) : a(args) {}
    __device__ __forceinline__ static int piece(int m, int half) { return piece_of<T>(8 * (2 * (sizeof(T) == 2 ? m : m / 2) + half), m); }
    __device__ __forceinline__ void begin(const CachedArgs &, int si, const Sequence &sq, int hk_, int wave_, const Frag<T> (&q)[D * sizeof(T) / 32])
    {
        own.set(q);
        hk = hk_;
        wave = wave_;
        nk = sq.nk;
        last_page = max(0, (sq.nk - 1) >> a.c.page_log2);
        pages = a.c.table + (int64_t)si * a.c.max_pages;
        // A lane takes eight channels of a row's first half and the eight across from them: the eight lanes that write 16 bytes at once then write
        // to all banks (with sixteen side by side half of them met, a quarter of all LDS cycles).  d = 64: of rows two apart.
        const int g = (threadIdx.x & 63) / PPR;
        row = D == 128 ? g : (g & 12) | ((g & 1) << 1) | ((g & 2) >> 1);
        piece_no = (threadIdx.x & 63) % PPR;
        of_lane = (uint32_t)(row * D + piece_no * 8);
    }
    __device__ __forceinline__ void find_pages(int k0)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) pg[i] = min(max(pages[min((k0 + (i * 4 + wave) * RPL) >> a.c.page_log2, last_page)], 0), a.c.n_pages - 1);
    }
    // the bytes of the tile that begins at key k0, whose pages were found, on their way into registers; and the pages of the one after it
    __device__ __forceinline__ void request(int k0)
    {
        at0 = k0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t of = (int64_t)pg[i] * a.Hkv + hk;
            const int64_t at = (of * a.c.page + ((k0 + (i * 4 + wave) * RPL) & (a.c.page - 1))) * D;
            raw[i] = halves(a.K8 + at + of_lane);
            raw[N + i] = halves(a.V8 + at + of_lane);
            scale[i] = a.kscale[of];
            scale[N + i] = a.vscale[of];
        }
        find_pages(k0 + Sh::KEYS);
    }
    __device__ __forceinline__ static uint4 halves(const uint8_t *p)
    {
        const uint2 lo = *reinterpret_cast<const uint2 *>(p), hi = *reinterpret_cast<const uint2 *>(p + D / 2);
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
    // one of the 2 N loads into the next tile; behind the sequence's end zeros, whatever the page holds there (a weight of zero times a NaN is one)
    __device__ __forceinline__ void put(int j)
    {
        const int r = (j % N * 4 + wave) * RPL + row;
        unsigned char *const tile = j < N ? next_k : next_v;
        uint4 w = raw[j];
        const float s = scale[j];
        if (at0 + Sh::KEYS > nk && at0 + r >= nk) w = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<bf16x8_t *>(tile + RT::at(r, piece_no)) = widen8(w.x, w.y, s);
        *reinterpret_cast<bf16x8_t *>(tile + RT::at(r, PPR + piece_no)) = widen8(w.z, w.w, s);
    }
    // as tile_scores(), the next tile's puts between the steps
    __device__ __forceinline__ void scores(const unsigned char *kt, int r, const Frag<T> (&)[D * sizeof(T) / 32], floatx16_t (&s)[Sh::KT])
    {
        constexpr int NM = D / 16;
        const int half = (threadIdx.x & 63) >> 5;
        Frag<bf16_t> f[kAhead][Sh::KT];
        auto fetch = [&](int m) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < Sh::KT; ++t) f[m % kAhead][t] = row_frag<bf16_t, D>(kt, r + 32 * t, m, half);
        };
#pragma unroll
        for (int t = 0; t < Sh::KT; ++t) s[t] = zero16();
#pragma unroll
        for (int m = 0; m < kAhead; ++m) fetch(m);
        pin_order();
#pragma unroll
        for (int m = 0; m < NM; ++m) {
#pragma unroll
            for (int k = WORDS - 1; k >= 0; --k)
#pragma unroll
                for (int t = 0; t < Sh::KT; ++t) s[t] = product(f[m % kAhead][t], own.w[k][m], s[t]);
            if (m + kAhead < NM) fetch(m + kAhead);
            if (m % 2 == 1 && m / 2 < 2 * N && more) put(m / 2);
            pin_order();
        }
    }
    // as weighted_rows(), every operand for all words of the weights
    __device__ __forceinline__ void add(const unsigned char *vt, int r0, const W &weights, floatx16_t (&acc)[D / 32]) const
    {
        typedef RowSum<bf16_t, D> RS;
        const WeightWords<WORDS> w(weights);
        typename RS::Operand f[RS::AHEAD];
#pragma unroll
        for (int i = 0; i < RS::AHEAD; ++i) f[i] = RS::fetch(vt, r0, i);
        pin_order();
#pragma unroll
        for (int i = 0; i < RS::STEPS; ++i) {
#pragma unroll
            for (int k = WORDS - 1; k >= 0; --k) RS::step(i, f[i % RS::AHEAD], w.w[k], acc);
            if (i + RS::AHEAD < RS::STEPS) f[i % RS::AHEAD] = RS::fetch(vt, r0, i + RS::AHEAD);
            pin_order();
        }
    }
    template <typename Scores, typename Rest>
    __device__ __forceinline__ void walk(const CachedArgs &, int kbeg, int kend, unsigned char *ka, unsigned char *va, unsigned char *kb, unsigned char *vb, Scores scores,
                                         Rest rest)
    {
        static_assert(Sh::NBUF == 2, "one barrier a tile: the next one is laid beside it");
        auto tile = [&](int k0, unsigned char *kt, unsigned char *vt, unsigned char *kn, unsigned char *vn) __attribute__((always_inline)) {
            next_k = kn;
            next_v = vn;
            more = k0 + Sh::KEYS < kend;
            floatx16_t s[Sh::KT];
            scores(kt, s);
            if (k0 + 2 * Sh::KEYS < kend) request(k0 + 2 * Sh::KEYS);
            rest(k0, s, vt);
            __syncthreads();
        };
        find_pages(kbeg);
        request(kbeg);
        next_k = ka;
        next_v = va;
#pragma unroll
        for (int j = 0; j < 2 * N; ++j) put(j);
        if (kbeg + Sh::KEYS < kend) request(kbeg + Sh::KEYS);
        __syncthreads();
        for (int k0 = kbeg; k0 < kend; k0 += 2 * Sh::KEYS) {
            tile(k0, ka, va, kb, vb);
            if (k0 + Sh::KEYS < kend) tile(k0 + Sh::KEYS, kb, vb, ka, va);
        }
    }
};

}  // namespace dsv
