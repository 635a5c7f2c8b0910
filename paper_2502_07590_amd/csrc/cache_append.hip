// New keys and values into an 8-bit cache, the keys turned by their positions on the way.
//
//   a page, head and tensor: s = max(scale of the values it holds, least power of two with max |new| <= 448 s);
//   values it holds times (their scale / s), new ones over s, each to the nearest e4m3
//
// Bound by memory for whole clips (two or four bytes in, one out), by latency for single tokens: a block takes the touched pages of one sequence one by
// one, of one or several heads, and holds the new values in registers between the maximum and the rounding.
#include <algorithm>

#include "cache.h"

namespace dsv {
namespace {

constexpr int kLeastExp = -117;  // 2^-9 of it, the least e4m3 value, is a normal fp32 number still
constexpr int kMostExp = 119;    // 448 of it is finite

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

// Four values to e4m3, rounded to nearest even; beyond 448 (only past the largest scale) to 448, infinities to NaN as NaN is.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d)
{
    auto fit = [](float x) { return fabsf(x) < __builtin_inff() ? fminf(fmaxf(x, -448.f), 448.f) : __builtin_nanf(""); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(fit(a), fit(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fit(c), fit(d), w, true);
}
__device__ __forceinline__ uint2 pack8(const float (&f)[8], float by)
{
    return make_uint2(pack_e4m3(f[0] * by, f[1] * by, f[2] * by, f[3] * by), pack_e4m3(f[4] * by, f[5] * by, f[6] * by, f[7] * by));
}
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float by)
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return pack_e4m3(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
}

// blockIdx: x a page that some sequence may touch, y the first head (others gridDim.y further), z K or V.  N: sixteens of a page a lane.
template <typename T, int D, int N>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendIn in, uint8_t *__restrict__ K8, uint8_t *__restrict__ V8, float *__restrict__ kscale,
                                                           float *__restrict__ vscale, CacheArgs a)
{
    __shared__ float red[2][4];
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

    const bool is_k = blockIdx.z == 0;
    const T *const src = static_cast<const T *>(is_k ? in.K : in.V);
    const int64_t row_s = is_k ? in.k_row : in.v_row, head_s = is_k ? in.k_head : in.v_head;
    uint8_t *const pool = is_k ? K8 : V8;
    float *const scales = is_k ? kscale : vscale;
    const bool turned = is_k && in.turn.total > 0;
    const int64_t token0 = (int64_t)sq.q0 + (page0 + begun - start);  // of the first new row of this page
    constexpr int PER = D / 16;

    Sixteen six[N];
    int row[N];
    float2 t[N][8];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int job = (int)threadIdx.x + j * (int)blockDim.x;
        row[j] = job / PER;
        six[j] = Sixteen{16 * (job % PER), 16 * (job % PER) + 8, -1};
        if (turned && in.eights) {
            six[j] = sixteen_of(in.turn, job % PER);
            if (row[j] < count && six[j].pair >= 0) {
                int pos[3];
                read_position(in.turn, token0 + row[j], pos);
#pragma unroll
                for (int i = 0; i < 8; ++i) t[j][i] = turn_of(in.turn, pos, six[j].pair + i);
            }
        }
    }
    int turn_no = 0;
    for (int h = blockIdx.y; h < a.Hkv; h += gridDim.y) {
        float f[N][8], g[N][8], most = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (row[j] >= count) continue;
            const T *const x = src + (token0 + row[j]) * row_s + h * head_s;
            load8(x + six[j].first, f[j]);
            load8(x + six[j].second, g[j]);
            if (six[j].pair >= 0) turn_sixteen<false>(in.turn.layout == DSV_TURN_INTERLEAVED, t[j], f[j], g[j]);
            if (turned && !in.eights) {
                int pos[3];
                read_position(in.turn, token0 + row[j], pos);
                for (int i = 0; i < in.turn.total; ++i) {  // any number of pairs: those that have a channel here
                    int lo, hi;
                    pair_channels(in.turn, i, lo, hi);
                    const int c0 = six[j].first;
                    if ((lo < c0 || lo >= c0 + 16) && (hi < c0 || hi >= c0 + 16)) continue;
                    float u = to_f32(x[lo]), v = to_f32(x[hi]);
                    turn<false>(u, v, turn_of(in.turn, pos, i));
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        f[j][c] = lo == c0 + c ? u : hi == c0 + c ? v : f[j][c];
                        g[j][c] = lo == c0 + 8 + c ? u : hi == c0 + 8 + c ? v : g[j][c];
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) {  // numbers alone: one infinity would leave nothing of the page's others
                most = fabsf(f[j][c]) < __builtin_inff() ? fmaxf(most, fabsf(f[j][c])) : most;
                most = fabsf(g[j][c]) < __builtin_inff() ? fmaxf(most, fabsf(g[j][c])) : most;
            }
        }
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
        if ((threadIdx.x & 63) == 0) red[turn_no][threadIdx.x >> 6] = most;
        const int64_t at = (int64_t)pg * a.Hkv + h;
        const float held = begun > 0 ? scales[at] : 0.f;
        __syncthreads();
        for (int w = 0; w < (int)blockDim.x / 64; ++w) most = fmaxf(most, red[turn_no][w]);
        turn_no ^= 1;
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
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (row[j] >= count) continue;
            uint8_t *const y = to + (begun + row[j]) * D;
            *reinterpret_cast<uint2 *>(y + six[j].first) = pack8(f[j], inv);
            *reinterpret_cast<uint2 *>(y + six[j].second) = pack8(g[j], inv);
        }
        if (threadIdx.x == 0) scales[at] = s;
    }
}

template <typename T, int D, int N>
dsv_status launch_n(const CacheArgs &a, const AppendIn &in, int threads, uint8_t *K8, uint8_t *V8, float *kscale, float *vscale, hipStream_t st)
{
    const int64_t slots = page_slots(a);
    const int64_t heads = std::min<int64_t>(a.Hkv, std::max<int64_t>(1, 2048 / slots));
    cache_append_kernel<T, D, N><<<dim3((unsigned)slots, (unsigned)heads, 2), threads, 0, st>>>(in, K8, V8, kscale, vscale, a);
    DSV_LAUNCH_CHECK();
    return DSV_OK;
}
template <typename T, int D>
dsv_status launch_d(const CacheArgs &a, const AppendIn &in, uint8_t *K8, uint8_t *V8, float *kscale, float *vscale, hipStream_t st)
{
    int rows = 1;  // new ones of a page, at most
    while (rows < std::min(a.page, a.max_new)) rows *= 2;
    const int jobs = rows * (D / 16), threads = std::min(256, std::max(64, jobs));
    switch ((jobs + threads - 1) / threads) {
        case 1: return launch_n<T, D, 1>(a, in, threads, K8, V8, kscale, vscale, st);
        case 2: return launch_n<T, D, 2>(a, in, threads, K8, V8, kscale, vscale, st);
        case 4: return launch_n<T, D, 4>(a, in, threads, K8, V8, kscale, vscale, st);
        case 8: return launch_n<T, D, 8>(a, in, threads, K8, V8, kscale, vscale, st);
        default: return DSV_EUNSUPPORTED;
    }
}
}  // namespace

dsv_status launch_cache_append(const CacheArgs &a, const AppendIn &in, int dtype, int d, uint8_t *K8, uint8_t *V8, float *kscale, float *vscale, hipStream_t st)
{
    if (dtype == DSV_BF16)
        return d == 128 ? launch_d<bf16_t, 128>(a, in, K8, V8, kscale, vscale, st) : launch_d<bf16_t, 64>(a, in, K8, V8, kscale, vscale, st);
    return d == 128 ? launch_d<float, 128>(a, in, K8, V8, kscale, vscale, st) : launch_d<float, 64>(a, in, K8, V8, kscale, vscale, st);
}

}  // namespace dsv
