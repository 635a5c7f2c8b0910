// C ABI of what stands around the attention of a block: rotary positions, gated norms, the 8-bit cache and attention over it.  Argument checks,
// forms and workspace layout, as in api.hip.
#include <algorithm>
#include <cmath>

#include "cache_tiles.h"
#include "checks.h"
#include "gated_norm.h"
#include "norm.h"
#include "rotary.h"

namespace dsv {
namespace {

constexpr int64_t kMostStride = (int64_t)1 << 40;
bool ok_stride(int64_t s) { return s >= 0 && s < kMostStride; }
bool in_place_or_apart(const void *out, int64_t out_stride, const void *in, int64_t in_stride) { return out != in || out_stride == in_stride; }

// ---- rotary positions
dsv_status check_turn(const dsv_rotary *p)
{
    if (p->axes < 1 || p->axes > 3 || p->layout < DSV_TURN_INTERLEAVED || p->layout > DSV_TURN_AXIS_HALVES || !std::isfinite(p->gain)) return DSV_EINVAL;
    int64_t total = 0;
    for (int i = 0; i < p->axes; ++i) {
        if (p->pairs[i] < 0) return DSV_EINVAL;
        total += p->pairs[i];
    }
    return total < 1 || 2 * total > p->d ? DSV_EINVAL : DSV_OK;
}
dsv_status check_rotary(const dsv_rotary *p)
{
    if (!p || p->tokens < 0 || p->heads < 1 || p->d < 1 || p->flags) return DSV_EINVAL;
    if (!supported_dtype(p->dtype) || p->d > kMaxNormWidth) return DSV_EUNSUPPORTED;
    if (check_turn(p) != DSV_OK) return DSV_EINVAL;
    for (const dsv_rows *s : {&p->x, &p->y})
        if (!ok_stride(s->row) || !ok_stride(s->head)) return DSV_EINVAL;
    if (!rows_apart(p->y, p->tokens, p->heads, p->d)) return DSV_EINVAL;
    // places of a launch
    if ((wide_t)p->tokens * p->heads * (p->d / 16 + 1) >= 1ll << 31 || (int64_t)p->tokens * p->d >= 1ll << 31) return DSV_EUNSUPPORTED;
    return DSV_OK;
}
TurnArgs turn_args(const dsv_rotary &p, const int32_t *pos, const double *freq)
{
    TurnArgs t{};
    t.pos = pos;
    t.freq = freq;
    t.axes = p.axes;
    t.end0 = p.pairs[0];
    t.end1 = t.end0 + (p.axes > 1 ? p.pairs[1] : 0);
    t.total = t.end1 + (p.axes > 2 ? p.pairs[2] : 0);
    t.layout = p.layout;
    t.gain = p.gain;
    return t;
}
dsv_status run_rotary(const dsv_rotary *p, bool back, const void *X, const int32_t *pos, const double *freq, void *Y, void *hip_stream)
{
    const dsv_status st = check_rotary(p);
    if (st != DSV_OK) return st;
    const size_t es = esize(p->dtype);
    if (!freq || !on_elements({freq}, 8) || !on_elements({pos}, 4) || !on_elements({X, Y}, es)) return DSV_EINVAL;
    if (p->tokens > 0 && (!X || !Y || !pos)) return DSV_EINVAL;
    if (!in_place_or_apart(Y, p->y.row, X, p->x.row) || !in_place_or_apart(Y, p->y.head, X, p->x.head)) return DSV_EINVAL;
    if (p->tokens == 0) return DSV_OK;
    RotaryArgs a{turn_args(*p, pos, freq), p->tokens, p->heads, p->d, p->x.row, p->x.head, p->y.row, p->y.head};
    const bool wide = eights(p->layout, p->axes, p->pairs, p->d) && aligned16(X) && aligned16(Y) && ok_strides(p->x, es) && ok_strides(p->y, es);
    return launch_rotary(a, p->dtype, wide, back, X, Y, static_cast<hipStream_t>(hip_stream));
}

// ---- gated norm
dsv_status check_gated(const dsv_gated_norm *p)
{
    if (!p) return DSV_EINVAL;
    if (p->tokens < 0 || p->n < 1 || p->n_seg < 1 || p->flags) return DSV_EINVAL;
    if (p->kind != DSV_NORM_LAYER && p->kind != DSV_NORM_RMS) return DSV_EINVAL;
    if ((p->post != 0 && p->post != 1) || !std::isfinite(p->eps) || !(p->eps >= 0.f) || !std::isfinite(p->residual)) return DSV_EINVAL;
    if (!supported_dtype(p->dtype) || p->n > kMaxNormWidth) return DSV_EUNSUPPORTED;
    if ((int64_t)p->n_seg * ((p->n + 31) / 32) >= (1 << 24) - (1 << 16)) return DSV_EUNSUPPORTED;  // blocks of a launch: as many, or one a segment and 32768
    return DSV_OK;
}
struct Row {
    const void *p;
    int64_t stride;
};
// Strides of the tensors that are there.  Outputs: `rows` of n elements apart.
bool ok_inputs(std::initializer_list<Row> in)
{
    for (const Row &r : in)
        if (r.p && !ok_stride(r.stride)) return false;
    return true;
}
bool ok_outputs(int rows, int n, std::initializer_list<Row> out)
{
    for (const Row &r : out)
        if (r.p && (!ok_stride(r.stride) || (rows > 1 && r.stride < n))) return false;
    return true;
}
GatedNormArgs gated_args(const dsv_gated_norm &p, const int32_t *cu)
{
    GatedNormArgs a{};
    a.cu = cu;
    a.tokens = p.tokens, a.n = p.n, a.n_seg = p.n_seg;
    a.eps = p.eps, a.residual = p.residual;
    a.rms = p.kind == DSV_NORM_RMS, a.post = p.post;
    a.x = p.x, a.y = p.y, a.h = p.h, a.z = p.z, a.gate = p.gate, a.scale = p.scale, a.shift = p.shift;
    a.dz = p.dz, a.dh = p.dh, a.dx = p.dx, a.dy = p.dy, a.dgate = p.dgate, a.dscale = p.dscale, a.dshift = p.dshift;
    return a;
}
// whether every tensor's rows begin on 16 bytes and fill whole ones
bool wide_rows(int n, int dtype, std::initializer_list<Row> rows)
{
    const int64_t unit = 16 / (int64_t)esize(dtype);
    if (n % unit) return false;
    for (const Row &r : rows)
        if (r.p && (!aligned16(r.p) || r.stride % unit)) return false;
    return true;
}

// ---- cache
int32_t longest_cache(const dsv_cache &p) { return (int32_t)std::min<int64_t>(p.max_len, (int64_t)p.page * p.max_pages); }
dsv_status check_cache(const dsv_cache *p)
{
    if (!p || p->n_seq < 1 || p->total < 0 || p->max_new < 0 || p->max_len < 0 || p->flags) return DSV_EINVAL;
    if (p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv || p->n_pages < 1 || p->max_pages < 1 || p->page < 1) return DSV_EINVAL;
    if (p->causal != 0 && p->causal != 1) return DSV_EINVAL;
    if (!(p->scale >= 1e-30f && p->scale <= 1e30f)) return DSV_EINVAL;
    if (!supported_dtype(p->dtype) || !supported_d(p->d)) return DSV_EUNSUPPORTED;
    if (p->page < 16 || p->page > 256 || (p->page & (p->page - 1)) || (int64_t)p->page * p->max_pages >= 1ll << 31) return DSV_EUNSUPPORTED;
    if (longest_cache(*p) > 1 << 30) return DSV_EUNSUPPORTED;  // the kernels count keys in 32 bits, a piece or four tiles ahead
    if ((int64_t)p->total * p->Hq >= 1ll << 31 || (int64_t)p->total * p->Hq * (p->Hq / p->Hkv) >= 1ll << 32) return DSV_EUNSUPPORTED;
    if ((int64_t)p->total * p->Hq / 32 + (int64_t)p->n_seq * p->Hkv >= 1 << 24) return DSV_EUNSUPPORTED;
    return DSV_OK;
}
// what the kernels read of the cache, in whole elements and 16 bytes
bool ok_cache(const int32_t *cu, const int32_t *lens, const int32_t *table, const void *K8, const void *V8, const float *kscale, const float *vscale)
{
    return cu && lens && table && kscale && vscale && on_elements({cu, lens, table, kscale, vscale}, 4) && ok_ptrs({K8, V8});
}
CacheArgs cache_args(const dsv_cache &p, const int32_t *cu, const int32_t *lens, const int32_t *table)
{
    CacheArgs a{};
    a.cu = cu, a.lens = lens, a.table = table;
    a.n_seq = p.n_seq, a.total = p.total, a.max_new = std::min(p.max_new, p.total);
    a.Hkv = p.Hkv, a.n_pages = p.n_pages, a.page = p.page, a.max_pages = p.max_pages;
    while ((1 << a.page_log2) < p.page) ++a.page_log2;
    a.max_len = longest_cache(p);
    return a;
}
// The packed forward's tiles, in pieces of their own: lengths of caches, which the kernels alone know, are anything up to the longest (blocks of a piece that
// a cache does not reach end at once).
Walk walk_of(const dsv_cache &p)
{
    const int64_t g = p.Hq / p.Hkv, longest = longest_cache(p), own = p.total * g, max_own = (int64_t)std::min(p.max_new, p.total) * g;
    Walk w{};
    w.few = few_rows(own, p.Hkv, p.n_seq, longest);
    const int64_t rows = w.few ? 32 : 128, most = (max_own + rows - 1) / rows;
    const int64_t tiles = std::min<int64_t>((int64_t)p.n_seq * most, own / rows + p.n_seq) * p.Hkv;
    int64_t chunk = longest;
    if (w.few) {
        // Bound by memory.  Twelve caches of up to 16001, four heads, group 4, d = 128, us without the join: pieces of 256 keys 23.6, 384 21.1, 512 19.9, 768
        // 18.9; 64 caches of 2047 .. 19900, two heads, group 7: 640 keys 84, 1280 80, 2560 89; five of up to 1023 in fp32, two heads: 256 10, 512 15.
        // Short caches go in one piece: a join costs as much as six more steps of a wave, and its launch and workspace on the host besides.  Eight caches of up to 400,
        // 800 and 1000 keys, four heads, group 4, d = 128, us captured into a graph: 10.3, 10.9, 10.7 in pieces, 9.0, 11.9, 13.1 in one, and by
        // itself 22 and 17; fp32, four caches of 1000, two heads, d = 64: 9.6 and 12.2, d = 128: 12.7 and 19.8 (500: 12.5 and 13.0).
        if (longest > (p.dtype == DSV_F32 && p.d == 128 ? 512 : 1024))
            chunk = std::max(tiles * longest / 2048, std::min<int64_t>(512, std::max<int64_t>(256, tiles * longest / 512)));
    } else if (longest > 0) {
        // Time in keys that a block walks: those of a piece and 100 to begin and to end, times the rounds of all blocks, each counted by the keys it has; and
        // the join.  Rounds lie between the whole ones and as many as the blocks fill, with 0.6 for those that end late.  The sequence of most queries is taken
        // to have the longest cache; of the others nothing is known, so nine parts of the time with an eighth of it for each stand beside one with all of it.
        // us by the rule, in one piece and at best of 1 to 64, bf16, d = 128 unless said: 32 x 256 queries on 8000, 32 heads on eight: 1149 (one piece); 4 x 4096 on
        // 32768: 9310 (one), two pieces 9220; 8 x 1560 on 21840, 16 heads on 16: 2659 (five), 2777, 2591, on four: 2456 (four), 2701; 2 x 1560 on
        // 20280, 16 on four: 638 (four), 669, 602, eight on two: 331 (nine), 479, 309; in fp32 774 (nine), 845, 725; 2 x 1560 on 21840 and 7800, eight on
        // two: 251 (nine), 508, 244; 300 on each of 30000, 4000 and 200, 16 on four: 129 (ten), 713; eight on two, fp32: 225 (twenty), 1217; 3 to 221
        // on eight of 108 to 9368, 16 on four: 77 (eleven), 230, 65; 8 x 200 on 9000, twelve on three, d = 64: 85 (nine), 158; 1045 and 63 on 8208 and
        // 192, twelve on three: 85 (five), 200; 129 on 14912, 16 on four, fp32: 72 (twelve), 604.  78 calls, most of them drawn: 4.7 % from the best in the mean, 22 at most;
        // a rule that charged every block the longest, whatever its keys, 8.9 and 33.  70 others: 0.98 of that rule's time in the mean, 0.57 to 1.23.
        const bool bf16 = p.dtype == DSV_BF16;
        const int per_cu = !bf16 ? (p.d == 128 ? 1 : 2) : (p.d == 128 ? 2 : 3);
        const double key = 1e-9 * (bf16 ? (p.d == 128 ? 37 : 32) : (p.d == 128 ? 41 : 44));  // seconds, a block among others
        const double at_once = 256.0 * per_cu, of_longest = (double)(most * p.Hkv), others = std::max(0.0, (double)tiles - of_longest), ends = 100;
        const double join = (double)p.total * p.Hq * p.d * 8.0 / 5.7e12 / key;  // a piece, written and read
        double best = 0;
        int64_t before = 0;
        for (int64_t s = 1; s <= 64; ++s) {
            const int64_t c = std::max<int64_t>(256, ((longest + s - 1) / s + 127) / 128 * 128);
            if (c == before) continue;
            before = c;
            const int64_t pieces = (longest + c - 1) / c;
            const double walk = (double)std::min(c, longest) + ends;
            auto rounds = [&](double part) {  // the others' caches: so much of the longest
                const double keys = part * (double)longest, x = (of_longest * (double)pieces + others * (keys + ends * std::ceil(keys / (double)c)) / walk) / at_once;
                return std::max(1.0, 0.5 * (std::ceil(x) + x + 0.6));
            };
            const double t = (0.9 * rounds(0.125) + 0.1 * rounds(1.0)) * walk + (pieces > 1 ? join * (double)pieces + 128.0 : 0.0);
            if (s == 1 || t < 0.98 * best) {
                best = t;
                chunk = c;
            }
        }
    }
    chunk = (std::max(chunk, (longest + 63) / 64) + 127) / 128 * 128;
    w.chunk = chunk < longest ? (int)chunk : 0;
    w.splits = w.chunk ? (int)((longest + chunk - 1) / chunk) : 1;
    return w;
}
size_t cache_fwd_bytes(const dsv_cache &p, const Walk &w)
{
    return w.splits > 1 ? packed_fwd_acc_bytes(p.total, p.Hq, p.d, w.splits) + align_up((size_t)p.total * p.Hq * w.splits * 8, 256) : 0;
}
}  // namespace
}  // namespace dsv

using namespace dsv;

extern "C" {

dsv_status dsv_rotary_fwd(const dsv_rotary *p, const void *X, const int32_t *pos, const double *freq, void *Y, void *hip_stream)
{
    return run_rotary(p, false, X, pos, freq, Y, hip_stream);
}

dsv_status dsv_rotary_bwd(const dsv_rotary *p, const void *dY, const int32_t *pos, const double *freq, void *dX, void *hip_stream)
{
    return run_rotary(p, true, dY, pos, freq, dX, hip_stream);
}

dsv_status dsv_rotary_freqs(int32_t pairs, double base, int32_t scaling, double factor, double original, double low, double high, double *freq, float *gain)
{
    if (pairs < 1 || !freq || !(base > 1.0) || !(factor >= 1.0) || !std::isfinite(base) || !std::isfinite(factor)) return DSV_EINVAL;
    if (scaling < DSV_SCALE_NONE || scaling > DSV_SCALE_PARTS) return DSV_EINVAL;
    if (scaling == DSV_SCALE_PARTS && !(original > 0.0 && low >= 0.0 && high > low && std::isfinite(original) && std::isfinite(high))) return DSV_EINVAL;
    if (scaling == DSV_SCALE_BASE && pairs > 1) base *= std::pow(factor, (double)pairs / (pairs - 1));
    for (int32_t i = 0; i < pairs; ++i) {
        double f = std::pow(base, -(double)i / pairs);
        if (scaling == DSV_SCALE_LINEAR) f /= factor;
        if (scaling == DSV_SCALE_PARTS) {
            const double turns = original * f / (2.0 * 3.14159265358979323846), keep = std::min(1.0, std::max(0.0, (turns - low) / (high - low)));
            f *= keep + (1.0 - keep) / factor;
        }
        freq[i] = f;
    }
    if (gain) *gain = scaling == DSV_SCALE_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    return DSV_OK;
}

dsv_status dsv_gated_norm_fwd(const dsv_gated_norm *p, const void *X, const void *Y, const int32_t *cu, const void *gate, const void *scale, const void *shift,
                              void *Z, void *H, float *stats, void *hip_stream)
{
    const dsv_status st = check_gated(p);
    if (st != DSV_OK) return st;
    if (!ok_inputs({{X, p->x}, {Y, p->y}, {gate, p->gate}, {scale, p->scale}, {shift, p->shift}}) || !ok_outputs(p->tokens, p->n, {{Z, p->z}, {H, p->h}})) return DSV_EINVAL;
    if (!cu || !on_elements({cu}, 4) || !aligned16(stats) || !on_elements({X, Y, gate, scale, shift, Z, H}, esize(p->dtype))) return DSV_EINVAL;
    if (p->tokens > 0 && !Y && (H || gate || p->post)) return DSV_EINVAL;
    if (p->tokens > 0 && (!X || !Z || !stats || (Y && !H))) return DSV_EINVAL;
    if (H && !in_place_or_apart(H, p->h, X, p->x)) return DSV_EINVAL;
    if (p->tokens == 0) return DSV_OK;
    const bool wide = wide_rows(p->n, p->dtype, {{X, p->x}, {Y, p->y}, {gate, p->gate}, {scale, p->scale}, {shift, p->shift}, {Z, p->z}, {H, p->h}});
    return launch_gated_fwd(gated_args(*p, cu), p->dtype, wide, {X, Y, gate, scale, shift}, Z, H, reinterpret_cast<float4 *>(stats), static_cast<hipStream_t>(hip_stream));
}

size_t dsv_gated_norm_bwd_workspace(const dsv_gated_norm *p)
{
    if (check_gated(p) != DSV_OK) return 0;
    return gated_bwd_bytes(p->tokens, p->n, p->n_seg, p->dtype);
}

dsv_status dsv_gated_norm_bwd(const dsv_gated_norm *p, const void *X, const void *Y, const int32_t *cu, const void *gate, const void *scale, const float *stats,
                              const void *dZ, const void *dH, void *dX, void *dY, float *dgate, float *dscale, float *dshift, void *workspace, size_t ws_bytes,
                              void *hip_stream)
{
    dsv_status st = check_gated(p);
    if (st != DSV_OK) return st;
    if (!ok_inputs({{X, p->x}, {Y, p->y}, {gate, p->gate}, {scale, p->scale}, {dZ, p->dz}, {dH, p->dh}})) return DSV_EINVAL;
    if (!ok_outputs(p->tokens, p->n, {{dX, p->dx}, {dY, p->dy}}) || !ok_outputs(p->n_seg, p->n, {{dgate, p->dgate}, {dscale, p->dscale}, {dshift, p->dshift}})) return DSV_EINVAL;
    if (!cu || !on_elements({cu, dgate, dscale, dshift}, 4) || !aligned16(stats) || !on_elements({X, Y, gate, scale, dZ, dH, dX, dY}, esize(p->dtype))) return DSV_EINVAL;
    if (p->tokens > 0 && !Y && (gate || dY || dgate || p->post)) return DSV_EINVAL;
    if (p->tokens > 0 && (!X || !stats || !dZ || !dX || (Y && !dY))) return DSV_EINVAL;
    if (dH && !in_place_or_apart(dX, p->dx, dH, p->dh)) return DSV_EINVAL;
    st = check_workspace(workspace, ws_bytes, dgate || dscale || dshift ? gated_bwd_bytes(p->tokens, p->n, p->n_seg, p->dtype) : 0);
    if (st != DSV_OK) return st;
    const bool wide = wide_rows(p->n, p->dtype, {{X, p->x}, {Y, p->y}, {gate, p->gate}, {scale, p->scale}, {dZ, p->dz}, {dH, p->dh}, {dX, p->dx}, {dY, p->dy}});
    return launch_gated_bwd(gated_args(*p, cu), p->dtype, wide, {X, Y, gate, scale, nullptr}, reinterpret_cast<const float4 *>(stats), dZ, dH, dX, dY, dgate, dscale,
                            dshift, static_cast<float *>(workspace), static_cast<hipStream_t>(hip_stream));
}

dsv_status dsv_cache_append(const dsv_cache *p, const dsv_rotary *turn, const void *K, const void *V, const int32_t *cu, const int32_t *lens, const int32_t *table,
                            const int32_t *pos, const double *freq, void *K8, void *V8, float *kscale, float *vscale, void *hip_stream)
{
    const dsv_status st = check_cache(p);
    if (st != DSV_OK) return st;
    if (turn && (turn->d != p->d || check_turn(turn) != DSV_OK)) return DSV_EINVAL;
    if (!ok_cache(cu, lens, table, K8, V8, kscale, vscale)) return DSV_EINVAL;
    if (!ok_strides(p->k, esize(p->dtype)) || !ok_strides(p->v, esize(p->dtype))) return DSV_EINVAL;
    if (p->total > 0 && !ok_ptrs({K, V})) return DSV_EINVAL;
    if (turn && (!freq || !on_elements({freq}, 8) || (p->total > 0 && !pos) || !on_elements({pos}, 4))) return DSV_EINVAL;
    if (p->total == 0 || p->max_new == 0) return DSV_OK;
    AppendIn in{K, V, p->k.row, p->k.head, p->v.row, p->v.head, turn ? turn_args(*turn, pos, freq) : TurnArgs{},
                turn && eights(turn->layout, turn->axes, turn->pairs, p->d)};
    return launch_cache_append(cache_args(*p, cu, lens, table), in, p->dtype, p->d, static_cast<uint8_t *>(K8), static_cast<uint8_t *>(V8), kscale, vscale,
                               static_cast<hipStream_t>(hip_stream));
}

size_t dsv_cache_attn_fwd_workspace(const dsv_cache *p)
{
    if (check_cache(p) != DSV_OK) return 0;
    return cache_fwd_bytes(*p, walk_of(*p));
}

dsv_status dsv_cache_attn_fwd(const dsv_cache *p, const void *Q, const int32_t *cu, const int32_t *lens, const int32_t *table, const void *K8, const void *V8,
                              const float *kscale, const float *vscale, void *O, float *lse, void *workspace, size_t ws_bytes, void *hip_stream)
{
    dsv_status st = check_cache(p);
    if (st != DSV_OK) return st;
    if (!ok_cache(cu, lens, table, K8, V8, kscale, vscale) || !on_elements({lse}, 4)) return DSV_EINVAL;
    if (!ok_strides(p->q, esize(p->dtype)) || !ok_strides(p->o, esize(p->dtype)) || !rows_apart(p->o, p->total, p->Hq, p->d)) return DSV_EINVAL;
    if (p->total > 0 && (!ok_ptrs({Q, O}) || !lse)) return DSV_EINVAL;
    const Walk w = walk_of(*p);
    st = check_workspace(workspace, ws_bytes, cache_fwd_bytes(*p, w));
    if (st != DSV_OK) return st;
    if (p->total == 0) return DSV_OK;
    const int64_t es = (int64_t)esize(p->dtype);
    CachedArgs a{};
    a.cu_q = cu;
    a.n_seq = p->n_seq, a.total_q = p->total, a.max_q = p->max_new;
    a.Hq = p->Hq, a.Hkv = p->Hkv, a.group = p->Hq / p->Hkv;
    a.magic = reciprocal(a.group);
    a.causal = p->causal;
    a.scale = p->scale;
    a.q_row = p->q.row * es, a.q_head = p->q.head * es, a.o_row = p->o.row * es, a.o_head = p->o.head * es;
    a.splits = w.splits, a.chunk = w.chunk;
    a.c = cache_args(*p, cu, lens, table);
    a.K8 = static_cast<const uint8_t *>(K8), a.V8 = static_cast<const uint8_t *>(V8);
    a.kscale = kscale, a.vscale = vscale;
    return launch_cache_fwd(a, p->dtype, p->d, w.few, Q, O, lse, static_cast<char *>(workspace), static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
