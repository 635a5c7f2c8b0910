// Tiles of keys out of the pages of an 8-bit cache, for the forward of attention.
//
// A row is half as long as in bf16 and comes by way of registers: the next tile's bytes are on their way while one is worked on, then widened with
// the page's scale by the conversion itself (v_cvt_scalef32; exact, the scales being powers of two) and laid into LDS as rows loaded directly would be.
// A load of a wave is one kilobyte of one page (8 or 16 tokens, and pages begin on multiples of 16), so its page and scales are the wave's.
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

// Eight values, low ones first.
__device__ __forceinline__ void widen8(uint32_t lo, uint32_t hi, float s, bf16_t *to)
{
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
    *reinterpret_cast<uint4 *>(to) = make_uint4(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d));
}
__device__ __forceinline__ void widen4(uint32_t w, float s, float *to)
{
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, true);
    *reinterpret_cast<float4 *>(to) = make_float4(a[0], a[1], b[0], b[1]);
}

template <typename T, int D, int WK> struct PageTiles {
    typedef FwdShape<T, D, WK> Sh;
    typedef RowTile<T, D> RT;
    static constexpr int RPL = 1024 / D, PPR = D / 16;     // tokens of a load, 16-byte pieces of a token
    static constexpr int N = Sh::KEYS / RPL / 4;           // loads of a wave for a tile of K, and of V
    const CachedArgs &a;
    const int32_t *pages;
    int hk, wave, last_page, nk, row, piece;
    uint4 k8[N], v8[N];
    float ks[N], vs[N];
    int at0;

    __device__ __forceinline__ explicit PageTiles(const CachedArgs &args) : a(args) {}
    __device__ __forceinline__ void begin(const CachedArgs &, int si, const Sequence &sq, int hk_, int wave_)
    {
        hk = hk_;
        wave = wave_;
        nk = sq.nk;
        last_page = max(0, (sq.nk - 1) >> a.c.page_log2);
        pages = a.c.table + (int64_t)si * a.c.max_pages;
        row = (threadIdx.x & 63) / PPR;
        piece = (threadIdx.x & 63) % PPR;
    }
    // bytes of the tile that begins at key k0, on their way into registers
    __device__ __forceinline__ void request(int k0)
    {
        at0 = k0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int k = k0 + (i * 4 + wave) * RPL;
            const int pg = min(max(pages[min(k >> a.c.page_log2, last_page)], 0), a.c.n_pages - 1);
            const int64_t of = (int64_t)pg * a.Hkv + hk;
            const int64_t at = of * a.c.page * D + (k & (a.c.page - 1)) * D + row * D + piece * 16;
            k8[i] = *reinterpret_cast<const uint4 *>(a.K8 + at);
            v8[i] = *reinterpret_cast<const uint4 *>(a.V8 + at);
            ks[i] = a.kscale[of];
            vs[i] = a.vscale[of];
        }
    }
    __device__ __forceinline__ void put(uint4 w, float s, int r, unsigned char *tile) const
    {
        if constexpr (sizeof(T) == 2) {
            widen8(w.x, w.y, s, reinterpret_cast<bf16_t *>(tile + RT::at(r, 2 * piece)));
            widen8(w.z, w.w, s, reinterpret_cast<bf16_t *>(tile + RT::at(r, 2 * piece + 1)));
        } else {
            widen4(w.x, s, reinterpret_cast<float *>(tile + RT::at(r, 4 * piece)));
            widen4(w.y, s, reinterpret_cast<float *>(tile + RT::at(r, 4 * piece + 1)));
            widen4(w.z, s, reinterpret_cast<float *>(tile + RT::at(r, 4 * piece + 2)));
            widen4(w.w, s, reinterpret_cast<float *>(tile + RT::at(r, 4 * piece + 3)));
        }
    }
    // the tile asked for last, into LDS; behind the sequence's end zeros, whatever the page holds there (a weight of zero times a NaN is one)
    __device__ __forceinline__ void land(unsigned char *kt, unsigned char *vt)
    {
        const bool edge = at0 + Sh::KEYS > nk;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = (i * 4 + wave) * RPL + row;
            if (edge && at0 + r >= nk) k8[i] = v8[i] = make_uint4(0, 0, 0, 0);
            put(k8[i], ks[i], r, kt);
            put(v8[i], vs[i], r, vt);
        }
    }
    template <typename Scores, typename Rest>
    __device__ __forceinline__ void walk(const CachedArgs &, int kbeg, int kend, unsigned char *ka, unsigned char *va, unsigned char *kb, unsigned char *vb, Scores scores,
                                         Rest rest)
    {
        auto tile = [&](int k0, unsigned char *kt, unsigned char *vt) __attribute__((always_inline)) {
            land(kt, vt);
            __syncthreads();
            if (k0 + Sh::KEYS < kend) request(k0 + Sh::KEYS);
            floatx16_t s[Sh::KT];
            scores(kt, s);
            rest(k0, s, vt);
        };
        request(kbeg);
        if constexpr (Sh::NBUF == 2) {
            for (int k0 = kbeg; k0 < kend; k0 += 2 * Sh::KEYS) {
                tile(k0, ka, va);
                if (k0 + Sh::KEYS < kend) tile(k0 + Sh::KEYS, kb, vb);
            }
        } else {
            for (int k0 = kbeg; k0 < kend; k0 += Sh::KEYS) {
                if (k0 > kbeg) __syncthreads();  // the tile before is done with
                tile(k0, ka, va);
            }
        }
    }
};

}  // namespace dsv
