// New keys and values into an 8-bit cache, the keys turned by their positions on the way.
//
//   a page, head and tensor: s = max(scale of the values it holds, least power of two with max |new| <= 448 s);
//   values it holds times (their scale / s), new ones over s, each to the nearest e4m3
//
// Bound by memory for whole clips (two or four bytes in, one out), by latency for single tokens: a block takes one touched page of a sequence, of one or
// several heads, and holds the new values in registers between the maximum and the rounding.  32568 tokens of 16 heads, d = 128, bf16: 98 us, 4.1 TB/s
// (a copy of 1 GiB: 5.1), in fp32 136, 4.9; with each head's loads begun only when the one before was written, and the form of turning
// read at run time, 141.  Twelve single tokens: 5.5 us.
#include <algorithm>

#include "cache.h"

namespace dsv {
namespace {

constexpr int kLeastExp = -117;  // 2^-9 of it, the least e4m3 value, is a normal fp32 number still
constexpr int kMostExp = 119;    // 448 of it is finite
constexpr float kLargest = 0x1p119f;

// The least power of two s with most <= 448 s = 1.75 * 2^8 s, by its bits.
__device__ __forceinline__ float scale_of(float most)
{
    const uint32_t b = __float_as_uint(most);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)(min(max(e, kLeastExp), kMostExp) + 127) << 23);
}

// Places for the pages that sequences may touch: ceil(new tokens / page) of each, and one more where a page may be gone on with.
__host__ __device__ __forceinline__ int page_gap(const CacheArgs &a) { return a.max_new == 1 ? 1 : 2; }
__host__ __forceinline__ int64_t page_slots(const CacheArgs &a) { return a.total / a.page + (int64_t)a.n_seq * page_gap(a); }

// Four values to e4m3, rounded to nearest even; infinities become NaN, as NaN is.  CUT: beyond 448 (only past the largest scale) 448, where the conversion
// itself would make it NaN.
template <bool CUT = false> __device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d)
{
    auto fit = [](float x) { return CUT && fabsf(x) < __builtin_inff() ? fminf(fmaxf(x, -448.f), 448.f) : x; };
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(fit(a), fit(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fit(c), fit(d), w, true);
}
template <bool CUT> __device__ __forceinline__ uint2 pack8(const float (&f)[8], float by)
{
    return make_uint2(pack_e4m3<CUT>(f[0] * by, f[1] * by, f[2] * by, f[3] * by), pack_e4m3<CUT>(f[4] * by, f[5] * by, f[6] * by, f[7] * by));
}
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float by)
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return pack_e4m3(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
}

// Sixteens of a page's new rows, job = row * (D / 16) + sixteen: as loaded, and as numbers.
template <typename T> struct Raw;
template <> struct Raw<bf16_t> {
    uint4 a, b;
    __device__ __forceinline__ void load(const bf16_t *x, const Sixteen &s)
    {
        a = *reinterpret_cast<const uint4 *>(x + s.first);
        b = *reinterpret_cast<const uint4 *>(x + s.second);
    }
    __device__ __forceinline__ void numbers(float (&f)[8], float (&g)[8]) const
    {
        unpack(Piece<bf16_t, 8>{a}, f);
        unpack(Piece<bf16_t, 8>{b}, g);
    }
};
template <> struct Raw<float> {
    float4 a, b, c, d;
    __device__ __forceinline__ void load(const float *x, const Sixteen &s)
    {
        a = *reinterpret_cast<const float4 *>(x + s.first);
        b = *reinterpret_cast<const float4 *>(x + s.first + 4);
        c = *reinterpret_cast<const float4 *>(x + s.second);
        d = *reinterpret_cast<const float4 *>(x + s.second + 4);
    }
    __device__ __forceinline__ void numbers(float (&f)[8], float (&g)[8]) const
    {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        g[0] = c.x; g[1] = c.y; g[2] = c.z; g[3] = c.w; g[4] = d.x; g[5] = d.y; g[6] = d.z; g[7] = d.w;
    }
};

enum TurnForm { kStraight, kEights, kAnyPairs };

// Sixteen channels from c0 on whose pairs lie anywhere: pairs and other channels (bytes: D is at most 128), the same for all rows and heads.
struct AnySixteen {
    uint32_t pair[4], other[4], turned, second;  // the last two: a bit a channel
    __device__ __forceinline__ AnySixteen(const TurnArgs &t, int c0) : pair{}, other{}, turned(0), second(0)
    {
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            if (c0 + c >= 2 * t.total) continue;
            int p, o;
            bool sec;
            pair_of(t, c0 + c, p, sec, o);
            pair[c / 4] |= (uint32_t)p << 8 * (c % 4);
            other[c / 4] |= (uint32_t)o << 8 * (c % 4);
            turned |= 1u << c;
            second |= (sec ? 1u : 0u) << c;
        }
    }
    static __device__ __forceinline__ int byte(const uint32_t (&w)[4], int c) { return (int)(w[c / 4] >> 8 * (c % 4) & 0xFFu); }
};
// what each channel, and its other one, is multiplied by
__device__ __forceinline__ void any_turns(const TurnArgs &t, const AnySixteen &s, int64_t token, float2 (&by)[16])
{
    int pos[3];
    read_position(t, token, pos);
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        by[c] = make_float2(1.f, 0.f);
        if (!(s.turned >> c & 1)) continue;
        by[c] = turn_of(t, pos, AnySixteen::byte(s.pair, c));
        if (!(s.second >> c & 1)) by[c].y = -by[c].y;
    }
}
template <typename T> __device__ __forceinline__ void turn_any(const AnySixteen &s, const float2 (&by)[16], const T *x, float (&f)[8], float (&g)[8])
{
    T o[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) o[c] = x[AnySixteen::byte(s.other, c)];  // of a channel that is not turned: the row's first, unused
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        float &v = c < 8 ? f[c & 7] : g[c & 7];
        v = s.turned >> c & 1 ? v * by[c].x + to_f32(o[c]) * by[c].y : v;
    }
}

template <TurnForm FORM> __device__ __forceinline__ auto channels(const TurnArgs &t, int c0)
{
    if constexpr (FORM == kAnyPairs) return AnySixteen(t, c0);
    else return 0;
}

// One tensor's new rows of one page, for heads h0, h0 + step, ...: the next head's loads are under way while one is rounded.
template <typename T, int D, int N, TurnForm FORM>
__device__ __forceinline__ void append_page(const TurnArgs &turns, const T *__restrict__ src, int64_t row_s, int64_t head_s, uint8_t *pool, float *scales,
                                            const CacheArgs &a, int pg, int64_t token0, int begun, int count, int h0, int step, float (&red)[2][16])
{
    constexpr int PER = D / 16;
    const bool interleaved = turns.layout == DSV_TURN_INTERLEAVED;
    Sixteen six[N];
    int row[N];
    float2 t[FORM == kEights ? N : 1][8];
    float2 any[FORM == kAnyPairs ? N : 1][16];  // the turns of all heads
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int job = (int)threadIdx.x + j * (int)blockDim.x;
        row[j] = job / PER;
        six[j] = Sixteen{16 * (job % PER), 16 * (job % PER) + 8, -1};
        if constexpr (FORM == kEights) six[j] = sixteen_of(turns, job % PER);
    }
    const std::conditional_t<FORM == kAnyPairs, AnySixteen, int> chans = channels<FORM>(turns, 16 * ((int)threadIdx.x % PER));  // of all its jobs
    Raw<T> raw[N];
    auto load = [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (row[j] < count) raw[j].load(src + (token0 + row[j]) * row_s + h * head_s, six[j]);
    };
    load(h0);
    if constexpr (FORM == kEights) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (row[j] < count && six[j].pair >= 0) {
                int pos[3];
                read_position(turns, token0 + row[j], pos);
#pragma unroll
                for (int i = 0; i < 8; ++i) t[j][i] = turn_of(turns, pos, six[j].pair + i);
            }
    }
    if constexpr (FORM == kAnyPairs) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (row[j] < count) any_turns(turns, chans, token0 + row[j], any[j]);
    }
    int flip = 0;
    for (int h = h0; h < a.Hkv; h += step) {
        float f[N][8], g[N][8], most = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (row[j] >= count) continue;
            raw[j].numbers(f[j], g[j]);
            if constexpr (FORM == kEights)
                if (six[j].pair >= 0) turn_sixteen<false>(interleaved, turns.total - six[j].pair, t[j], f[j], g[j]);
            if constexpr (FORM == kAnyPairs) turn_any(chans, any[j], src + (token0 + row[j]) * row_s + h * head_s, f[j], g[j]);
#pragma unroll
            for (int c = 0; c < 8; ++c) most = fmaxf(most, fmaxf(fabsf(f[j][c]), fabsf(g[j][c])));  // of the numbers: fmaxf passes over NaN
        }
        if (h + step < a.Hkv) load(h + step);
        const int64_t at = (int64_t)pg * a.Hkv + h;
        const float held = begun > 0 ? scales[at] : 0.f;
        auto of_block = [&](float x) __attribute__((always_inline)) {
#pragma unroll
            for (int s = 32; s > 0; s >>= 1) x = fmaxf(x, __shfl_xor(x, s));
            if (blockDim.x > 64) {
                if ((threadIdx.x & 63) == 0) red[flip][threadIdx.x >> 6] = x;
                __syncthreads();
                for (int w = 0; w < (int)blockDim.x / 64; ++w) x = fmaxf(x, red[flip][w]);
                flip ^= 1;
            }
            return x;
        };
        most = of_block(most);
        if (most == __builtin_inff()) {  // one infinity would leave nothing of the page's others: the largest of those (all lanes come here, or none)
            float rest = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (row[j] >= count) continue;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    rest = fabsf(f[j][c]) < __builtin_inff() ? fmaxf(rest, fabsf(f[j][c])) : rest;
                    rest = fabsf(g[j][c]) < __builtin_inff() ? fmaxf(rest, fabsf(g[j][c])) : rest;
                }
            }
            most = of_block(rest);
        }
        const float s = fmaxf(held, scale_of(most)), inv = 1.f / s;  // exact: a power of two
        uint8_t *const to = pool + at * a.page * D;
        if (held > 0.f && s != held) {  // the values that the page holds, to the larger scale
            const float by = held * inv;
            for (int i = threadIdx.x; i < begun * PER; i += blockDim.x) {
                uint4 w = reinterpret_cast<const uint4 *>(to)[i];
                w = make_uint4(rescale4(w.x, by), rescale4(w.y, by), rescale4(w.z, by), rescale4(w.w, by));
                reinterpret_cast<uint4 *>(to)[i] = w;
            }
        }
        auto write = [&](auto cut) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (row[j] >= count) continue;
                uint8_t *const y = to + (begun + row[j]) * D;
                const uint2 lo = pack8<decltype(cut)::value>(f[j], inv), hi = pack8<decltype(cut)::value>(g[j], inv);
                if (!interleaved && FORM == kEights) {
                    *reinterpret_cast<uint2 *>(y + six[j].first) = lo;
                    *reinterpret_cast<uint2 *>(y + six[j].second) = hi;
                } else {  // side by side
                    *reinterpret_cast<uint4 *>(y + six[j].first) = make_uint4(lo.x, lo.y, hi.x, hi.y);
                }
            }
        };
        if (s < kLargest) write(std::false_type{});
        else write(std::true_type{});
        if (threadIdx.x == 0) scales[at] = s;
    }
}

// blockIdx: x a page that some sequence may touch, y the first head (others gridDim.y further), z K or V.  N: sixteens of a page a lane.  MOST: lanes, at most.
template <typename T, int D, int N, int MOST, TurnForm FORM>
__global__ __launch_bounds__(MOST) void cache_append_kernel(AppendIn in, uint8_t *K8, uint8_t *V8, float *kscale, float *vscale, CacheArgs a)
{
    __shared__ float red[2][16];
    const int si = __builtin_amdgcn_readfirstlane(find_sequence(a.cu, a.n_seq, a.total, 1, a.page, (int)blockIdx.x, page_gap(a)));
    const Sequence sq = read_cached(a, si);
    const int start = sq.nk - sq.nq, place = (int)blockIdx.x - first_slot(a.cu[si], a.total, 1, a.page, si * page_gap(a));
    if (start < 0 || place < 0 || sq.nq == 0) return;  // a cache shorter than what goes in
    const int page_no = (start >> a.page_log2) + place;
    const int64_t page0 = (int64_t)page_no << a.page_log2;
    if (page0 >= sq.nk) return;
    const int begun = max(start - (int)page0, 0), count = min((int)(sq.nk - page0), a.page) - begun;
    const int pg = a.table[(int64_t)si * a.max_pages + page_no];
    if (pg < 0 || pg >= a.n_pages) return;
    const int64_t token0 = (int64_t)sq.q0 + (page0 + begun - start);  // of the first new row of this page
    if (blockIdx.z == 0)
        append_page<T, D, N, FORM>(in.turn, static_cast<const T *>(in.K), in.k_row, in.k_head, K8, kscale, a, pg, token0, begun, count, blockIdx.y, gridDim.y, red);
    else
        append_page<T, D, N, kStraight>(in.turn, static_cast<const T *>(in.V), in.v_row, in.v_head, V8, vscale, a, pg, token0, begun, count, blockIdx.y, gridDim.y, red);
}

// Heads to a block, one after another with the sines that they share: as many as leave 2048 blocks of 256 lanes, or as many
// lanes.  32568 tokens of 16 heads, d = 128, bf16, us: in 1024 blocks (of both tensors together) 115, 3084 96, 4112 101, 7200 106, 15420 142.
constexpr int64_t kBlocks = 2048;
template <typename T, int D, int N, int MOST>
dsv_status launch_n(const CacheArgs &a, const AppendIn &in, int threads, uint8_t *K8, uint8_t *V8, float *kscale, float *vscale, hipStream_t st)
{
    const int64_t slots = page_slots(a);
    const int64_t heads = std::min<int64_t>(a.Hkv, std::max<int64_t>(1, kBlocks * 256 / MOST / slots));
    if (slots * threads >= (int64_t)1 << 32) return DSV_EUNSUPPORTED;  // lanes of a grid
    const dim3 grid((unsigned)slots, (unsigned)heads, 2);
    if (in.turn.total == 0) cache_append_kernel<T, D, N, MOST, kStraight><<<grid, threads, 0, st>>>(in, K8, V8, kscale, vscale, a);
    else if (in.eights) cache_append_kernel<T, D, N, MOST, kEights><<<grid, threads, 0, st>>>(in, K8, V8, kscale, vscale, a);
    else cache_append_kernel<T, D, N, MOST, kAnyPairs><<<grid, threads, 0, st>>>(in, K8, V8, kscale, vscale, a);
    DSV_LAUNCH_CHECK();
    return DSV_OK;
}
template <typename T, int D>
dsv_status launch_d(const CacheArgs &a, const AppendIn &in, uint8_t *K8, uint8_t *V8, float *kscale, float *vscale, hipStream_t st)
{
    int rows = 1;  // new ones of a page, at most
    while (rows < std::min(a.page, a.max_new)) rows *= 2;
    // A lane holds two sixteens at most.  Pages of 256, 20900 tokens of 16 heads, bf16, us a call: in 1024 lanes 74, in 256 of eight sixteens each 151; pairs that
    // lie anywhere 229, 592 (captured, in 1024 lanes: 60, 204).  1024 lanes leave 128 registers each: of pairs that lie anywhere 155 are spilled (fp32
    // 176; of pairs in eights 12 in fp32).
    const int jobs = rows * (D / 16);
    if (jobs <= 256) return launch_n<T, D, 1, 256>(a, in, std::max(64, jobs), K8, V8, kscale, vscale, st);
    if (jobs <= 512) return launch_n<T, D, 2, 256>(a, in, 256, K8, V8, kscale, vscale, st);
    if (jobs <= 1024) return launch_n<T, D, 2, 512>(a, in, 512, K8, V8, kscale, vscale, st);
    if constexpr (D == 128)
        if (jobs <= 2048) return launch_n<T, D, 2, 1024>(a, in, 1024, K8, V8, kscale, vscale, st);
    return DSV_EUNSUPPORTED;
}
}  // namespace

dsv_status launch_cache_append(const CacheArgs &a, const AppendIn &in, int dtype, int d, uint8_t *K8, uint8_t *V8, float *kscale, float *vscale, hipStream_t st)
{
    if (dtype == DSV_BF16)
        return d == 128 ? launch_d<bf16_t, 128>(a, in, K8, V8, kscale, vscale, st) : launch_d<bf16_t, 64>(a, in, K8, V8, kscale, vscale, st);
    return d == 128 ? launch_d<float, 128>(a, in, K8, V8, kscale, vscale, st) : launch_d<float, 64>(a, in, K8, V8, kscale, vscale, st);
}

}  // namespace dsv
