// C ABI of attention over packed sequences and of layer norm: argument checks, forms and workspace layout, as in api.hip.
#include <algorithm>
#include <cmath>

#include "checks.h"
#include "norm.h"
#include "packed_attn.h"

namespace dsv {
namespace {

dsv_status check_packed(const dsv_packed *p, bool grad)
{
    if (!p) return DSV_EINVAL;
    if (p->n_seq < 1 || p->total_q < 0 || p->total_k < 0 || p->max_q < 0 || p->max_k < 0) return DSV_EINVAL;
    if (p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv) return DSV_EINVAL;
    if (p->causal != 0 && p->causal != 1) return DSV_EINVAL;
    if (p->flags || !(p->scale >= 1e-30f && p->scale <= 1e30f)) return DSV_EINVAL;  // lse / scale and scale * log2(e) are finite
    if (!supported_dtype(p->dtype) || !supported_d(p->d)) return DSV_EUNSUPPORTED;
    const size_t es = esize(p->dtype);
    for (const dsv_rows *s : {&p->q, &p->k, &p->v, &p->o})
        if (!ok_strides(*s, es)) return DSV_EINVAL;
    if (!grad && !rows_apart(p->o, p->total_q, p->Hq, p->d)) return DSV_EINVAL;
    if (grad) {
        for (const dsv_rows *s : {&p->dO, &p->dq, &p->dk, &p->dv})
            if (!ok_strides(*s, es)) return DSV_EINVAL;
        if (!rows_apart(p->dq, p->total_q, p->Hq, p->d) || !rows_apart(p->dk, p->total_k, p->Hkv, p->d) || !rows_apart(p->dv, p->total_k, p->Hkv, p->d))
            return DSV_EINVAL;
    }
    // the kernels place the rows of a tile by 32-bit offsets from its first
    const int64_t most = 1ll << 32, group = p->Hq / p->Hkv;
    for (const dsv_rows *s : {&p->q, &p->k, &p->v, grad ? &p->dO : &p->q})  // the forward reads no layout of the backward: those may hold anything
        if (128 * s->row * (int64_t)es >= most) return DSV_EUNSUPPORTED;
    for (const dsv_rows *s : {&p->q, &p->dO})
        if (grad && ((wide_t)128 * s->row + (wide_t)(group - 1) * s->head) * (int64_t)es >= most) return DSV_EUNSUPPORTED;
    // row / group by a 32-bit reciprocal, and the blocks of a launch
    if ((int64_t)p->total_q * p->Hq >= 1ll << 31 || (int64_t)p->total_q * p->Hq * (p->Hq / p->Hkv) >= 1ll << 32) return DSV_EUNSUPPORTED;
    if ((int64_t)p->total_q * p->Hq / 32 + (int64_t)p->n_seq * p->Hkv >= 1 << 24) return DSV_EUNSUPPORTED;
    if ((int64_t)p->total_k * p->Hkv / 32 + (int64_t)p->n_seq * p->Hkv >= 1 << 24) return DSV_EUNSUPPORTED;
    return DSV_OK;
}

PackedArgs packed_args(const dsv_packed &p, bool grad, const int32_t *cu_q, const int32_t *cu_k)
{
    const int64_t es = (int64_t)esize(p.dtype);
    PackedArgs a{};
    a.cu_q = cu_q;
    a.cu_k = cu_k;
    a.n_seq = p.n_seq;
    a.total_q = p.total_q;
    a.total_k = p.total_k;
    a.max_q = p.max_q;
    a.max_k = p.max_k;
    a.Hq = p.Hq;
    a.Hkv = p.Hkv;
    a.group = p.Hq / p.Hkv;
    a.magic = reciprocal(a.group);
    a.causal = p.causal;
    a.scale = p.scale;
    a.q_row = p.q.row * es, a.q_head = p.q.head * es;
    a.k_row = p.k.row * es, a.k_head = p.k.head * es;
    a.v_row = p.v.row * es, a.v_head = p.v.head * es;
    a.o_row = p.o.row * es, a.o_head = p.o.head * es;
    a.splits = 1;
    if (!grad) return a;
    a.do_row = p.dO.row * es, a.do_head = p.dO.head * es;
    a.dq_row = p.dq.row * es, a.dq_head = p.dq.head * es;
    a.dk_row = p.dk.row * es, a.dk_head = p.dk.head * es;
    a.dv_row = p.dv.row * es, a.dv_head = p.dv.head * es;
    return a;
}

// A step's cost: blocks of 128 rows a CU runs at once, operations a pair of rows (and channel), the rate it reaches with the chip full, and
// how many results a piece leaves per own row.
struct StepCost {
    bool bf16;
    int per_cu;
    double flops, rate;
    int results;
};
Walk plan_walk(const StepCost &cost, int d, bool causal, int64_t own, int64_t max_own, int64_t heads, int64_t n_seq, int64_t other, int64_t max_other)
{
    constexpr int64_t kUnit = 128, kMaxSplits = 64;
    Walk w{};
    w.splits = 1;
    const int64_t pieces = std::max<int64_t>(1, max_other / kMinChunk);
    w.few = few_rows(own, heads, n_seq, max_other);
    int64_t chunk = max_other;
    const double rest = (double)(n_seq - 1), longest = (double)std::max<int64_t>(max_other, 1);
    const double rest_own = (double)std::max<int64_t>(own - max_own, 0), rest_other = n_seq > 1 ? (double)std::max<int64_t>(other - max_other, 0) / rest : 0.0;
    if (w.few) {
        if (max_own <= 32) {
            // One tile a sequence and head, the other axis read once: bound by memory, and pieces of any number fill it; so long that all blocks
            // together walk about 512 of them.
            const double tiles = (double)(own / 32 + n_seq) / (double)n_seq;
            chunk = std::max({(int64_t)(tiles * (double)other * (double)heads) / (2 * kCus), kMinChunk, (max_other + kMaxSplits - 1) / kMaxSplits});
        } else {
            // Rounds of blocks, by what a block takes: the walk, and as long as two tiles of 128 to begin and to join.  Forward, us, by the rule
            // above and by this one: fp32, 1024 + 700 tokens, two heads, d = 64: 23.4 (four pieces), 19.3 (two); 2048 tokens, one head, d = 128:
            // fp32 45.4 (six), 31.0 (four), bf16 17.1 (six), 16.7 (eight).
            const double at_once = (double)kCus * (cost.bf16 ? 2 : 1);
            const double tiles = (double)((max_own + 31) / 32), more = rest_own / 32 + rest / 2;
            double best = 0;
            int64_t before = 0;
            for (int64_t s = 1; s <= std::min(kMaxSplits, (max_other + kMinChunk - 1) / kMinChunk); ++s) {
                const int64_t c = ((max_other + s - 1) / s + kUnit - 1) / kUnit * kUnit;
                if (c == before) continue;
                before = c;
                const double of_longest = (double)((max_other + c - 1) / c), seen = causal ? 0.75 + 0.25 / of_longest : 1.0;
                const double blocks = (double)heads * (tiles * of_longest + more * std::max(1.0, std::ceil(rest_other / (double)c))) * seen;
                const double t = std::ceil(blocks / at_once) * (2.0 + (double)c / 128) + (s > 1 ? 1.0 : 0.0);
                if (s == 1 || t < best) {
                    best = t;
                    chunk = c;
                }
            }
        }
    } else {
        // Without pieces the longest blocks set the time, or the CUs that run one block more than others; pieces cost writing and reading their
        // results.  Times are in those of a block of 128 own rows by the longest other axis; one sequence is taken to be the longest, the rest alike.
        // Measured, us with the joins, in one piece and as chosen: L = 20280, 4 heads, bf16, d = 128: forward 975, 889 (two); dq 1490, 1325 (two);
        // dkdv 1622, 1529 (two).  Causal, 16384 tokens, 4 heads: forward 377, 351 (two); dq 551, 505 (two); dkdv 565 (one).  Causal, 4096 tokens, 4
        // heads: 79, 48 (four); 118, 63 (four); 126, 67 (three).
        const double cus = (double)kCus;
        const double blocks = (double)((max_own + 127) / 128) * (double)heads;
        double work = blocks;
        if (n_seq > 1)
            work += (rest_own / 128 + rest / 2) * (double)heads * rest_other / longest;
        const double mean = work * (causal ? 0.5 : 1.0) / cus;
        const double block_s = cost.flops * d * 128.0 * longest / (cost.rate / cus);  // with a CU to itself, were it then as fast as with others
        const double alone = cost.per_cu > 1 ? 0.65 * cost.per_cu : 1.0;              // how much slower it is
        const double piece_s = (double)own * (double)heads * d * 8.0 * cost.results * (causal ? 0.5 : 1.0) / 4e12;  // written and read
        double best = 0;
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (s > pieces) break;
            // blocks all alike come in whole rounds; of many lengths they are taken to fill the CUs but for a little, as if the longest began first;
            // their pieces are alike again, and a CU that runs one at a time is idle for half of one at the end.  They begin in the order of packing
            // (causal rows in its reverse): 20280 + 8192 + 4096 tokens, four heads, d = 128, bf16, 1004 us forward and 3477 backward, packed the
            // other way round 1055 and 3794.
            const double left = cost.per_cu > 1 ? 0.1 * cost.per_cu / s : s > 1 ? 0.5 / s : 0.1;
            const double rounds = n_seq == 1 && !causal ? std::ceil(work * s / cus) / s : mean + left;
            const double t = std::max(rounds, alone / s) * block_s + (s > 1 ? s * piece_s + 5e-6 : 0.0);
            if (s == 1 || t < 0.965 * best) {
                best = t;
                chunk = (max_other + s - 1) / s;
            }
        }
    }
    chunk = (chunk + kUnit - 1) / kUnit * kUnit;
    if (chunk >= max_other) return w;
    w.chunk = (int)chunk;
    w.splits = (int)((max_other + chunk - 1) / chunk);
    return w;
}
enum Step { kFwd, kDq, kDkdv };
Walk walk_of(const dsv_packed &p, Step step)
{
    const bool bf16 = p.dtype == DSV_BF16;
    const int64_t g = p.Hq / p.Hkv;
    // operations a pair and channel, and rates: as measured at 32768 tokens.  (fp32 dK and dV: those of blocks of 128 keys, where launch_dkdv runs blocks
    // of 32, one a CU: four times as many as counted, and so more pieces than they need.)
    StepCost c{};
    c.bf16 = bf16;
    c.per_cu = step == kDkdv ? (p.d == 64 ? 2 : 1) : bf16 ? (p.d == 64 ? 3 : 2) : (p.d == 64 ? 2 : 1);
    c.flops = step == kFwd ? 4 : 8;
    c.rate = bf16 ? 1.1e15 : 1e14;
    c.results = step == kDkdv ? 2 : 1;
    if (step == kDkdv)
        return plan_walk(c, p.d, p.causal != 0, p.total_k, std::min(p.max_k, p.total_k), p.Hkv, p.n_seq, (int64_t)p.total_q * g, std::min(p.max_q, p.total_q) * g);
    return plan_walk(c, p.d, p.causal != 0, (int64_t)p.total_q * g, std::min(p.max_q, p.total_q) * g, p.Hkv, p.n_seq, p.total_k, std::min(p.max_k, p.total_k));
}

size_t fwd_bytes(const dsv_packed &p)
{
    const Walk w = walk_of(p, kFwd);
    return w.splits > 1 ? packed_fwd_acc_bytes(p.total_q, p.Hq, p.d, w.splits) + align_up((size_t)p.total_q * p.Hq * w.splits * 8, 256) : 0;
}
size_t bwd_bytes(const dsv_packed &p)
{
    return packed_stat_bytes(p.total_q, p.Hq) +
           std::max(packed_dq_bytes(p.total_q, p.Hq, p.d, walk_of(p, kDq).splits), packed_dkdv_bytes(p.total_k, p.Hkv, p.d, walk_of(p, kDkdv).splits));
}

dsv_status check_norm(const dsv_norm *p, bool grad)
{
    if (!p) return DSV_EINVAL;
    if (p->tokens < 0 || p->heads < 1 || p->n < 1 || p->flags || !std::isfinite(p->eps) || !(p->eps >= 0.f)) return DSV_EINVAL;
    if (!supported_dtype(p->dtype) || p->n > kMaxNormWidth || (int64_t)p->tokens * p->heads >= 1ll << 31) return DSV_EUNSUPPORTED;
    const int64_t most = (int64_t)1 << 40;
    for (const dsv_rows *s : {&p->x, grad ? &p->dy : &p->y, grad ? &p->dx : &p->y})
        if (s->row < 0 || s->head < 0 || s->row >= most || s->head >= most) return DSV_EINVAL;
    if (!rows_apart(grad ? p->dx : p->y, p->tokens, p->heads, p->n)) return DSV_EINVAL;
    return DSV_OK;
}
NormArgs norm_args(const dsv_norm &p)
{
    return NormArgs{p.tokens, p.heads, p.n, p.eps, p.x.row, p.x.head, p.y.row, p.y.head, p.dy.row, p.dy.head, p.dx.row, p.dx.head};
}
bool wide_rows(const dsv_norm &p, std::initializer_list<const void *> ps, std::initializer_list<dsv_rows> strides)
{
    const int64_t unit = 16 / (int64_t)esize(p.dtype);
    if (p.n % unit) return false;
    for (const void *q : ps)
        if (!aligned16(q)) return false;
    for (const dsv_rows &s : strides)
        if (s.row % unit || s.head % unit) return false;
    return true;
}
}  // namespace
}  // namespace dsv

using namespace dsv;

extern "C" {

size_t dsv_packed_attn_fwd_workspace(const dsv_packed *p)
{
    if (check_packed(p, false) != DSV_OK) return 0;
    return fwd_bytes(*p);
}

dsv_status dsv_packed_attn_fwd(const dsv_packed *p, const void *Q, const void *K, const void *V, const int32_t *cu_q, const int32_t *cu_k, void *O,
                               void *O_tail, float *lse, void *workspace, size_t ws_bytes, void *hip_stream)
{
    dsv_status st = check_packed(p, false);
    if (st != DSV_OK) return st;
    if (!cu_q || !cu_k || !on_elements({cu_q, cu_k, lse}, 4)) return DSV_EINVAL;
    if (p->total_q > 0 && (!ok_ptrs({Q, O}) || !lse)) return DSV_EINVAL;
    if (p->total_k > 0 && !ok_ptrs({K, V})) return DSV_EINVAL;
    if (O_tail && (p->dtype != DSV_BF16 || !aligned16(O_tail))) return DSV_EINVAL;
    st = check_workspace(workspace, ws_bytes, fwd_bytes(*p));
    if (st != DSV_OK) return st;
    if (p->total_q == 0) return DSV_OK;
    const Walk w = walk_of(*p, kFwd);
    PackedArgs a = packed_args(*p, false, cu_q, cu_k);
    a.splits = w.splits;
    a.chunk = w.chunk;
    return launch_packed_fwd(a, p->dtype, p->d, w.few, Q, K, V, O, O_tail, lse, static_cast<char *>(workspace), static_cast<hipStream_t>(hip_stream));
}

size_t dsv_packed_attn_bwd_workspace(const dsv_packed *p)
{
    if (check_packed(p, true) != DSV_OK) return 0;
    return bwd_bytes(*p);
}

dsv_status dsv_packed_attn_bwd(const dsv_packed *p, const void *Q, const void *K, const void *V, const int32_t *cu_q, const int32_t *cu_k, const void *O,
                               const void *O_tail, const float *lse, const void *dO, void *dQ, void *dK, void *dV, void *workspace, size_t ws_bytes,
                               void *hip_stream)
{
    dsv_status st = check_packed(p, true);
    if (st != DSV_OK) return st;
    if (!cu_q || !cu_k || !on_elements({cu_q, cu_k, lse}, 4)) return DSV_EINVAL;
    if (p->total_q > 0 && (!ok_ptrs({Q, O, dO, dQ}) || !lse)) return DSV_EINVAL;
    if (p->total_k > 0 && !ok_ptrs({K, V, dK, dV})) return DSV_EINVAL;
    if (O_tail && (p->dtype != DSV_BF16 || !aligned16(O_tail))) return DSV_EINVAL;
    st = check_workspace(workspace, ws_bytes, bwd_bytes(*p));
    if (st != DSV_OK) return st;
    const Walk q = walk_of(*p, kDq), k = walk_of(*p, kDkdv);
    const PackedBwdPlan plan{q.few, k.few, q.splits, q.chunk, k.splits, k.chunk};
    return launch_packed_bwd(packed_args(*p, true, cu_q, cu_k), plan, p->dtype, p->d, Q, K, V, O, O_tail, lse, dO, dQ, dK, dV, static_cast<char *>(workspace),
                             static_cast<hipStream_t>(hip_stream));
}

dsv_status dsv_layer_norm_fwd(const dsv_norm *p, const void *X, const void *gamma, const void *beta, void *Y, float *mean, float *rstd, void *hip_stream)
{
    dsv_status st = check_norm(p, false);
    if (st != DSV_OK) return st;
    if (p->tokens > 0 && (!X || !Y || !mean || !rstd)) return DSV_EINVAL;
    if (!on_elements({X, gamma, beta, Y}, esize(p->dtype)) || !on_elements({mean, rstd}, 4)) return DSV_EINVAL;
    if (p->tokens == 0) return DSV_OK;
    const bool wide = wide_rows(*p, {X, gamma, beta, Y}, {p->x, p->y});
    return launch_norm_fwd(norm_args(*p), p->dtype, wide, X, gamma, beta, Y, mean, rstd, static_cast<hipStream_t>(hip_stream));
}

// the pointers do not enter: as many blocks as rows of either alignment may take
static size_t norm_bwd_bytes(const dsv_norm &p)
{
    const NormArgs a = norm_args(p);
    return align_up((size_t)std::max(norm_bwd_blocks(a, p.dtype, false), norm_bwd_blocks(a, p.dtype, true)) * 2 * p.n * 4, 256);
}

size_t dsv_layer_norm_bwd_workspace(const dsv_norm *p)
{
    if (check_norm(p, true) != DSV_OK) return 0;
    return norm_bwd_bytes(*p);
}

dsv_status dsv_layer_norm_bwd(const dsv_norm *p, const void *X, const void *gamma, const float *mean, const float *rstd, const void *dY, void *dX,
                              float *dgamma, float *dbeta, void *workspace, size_t ws_bytes, void *hip_stream)
{
    dsv_status st = check_norm(p, true);
    if (st != DSV_OK) return st;
    if (p->tokens > 0 && (!X || !mean || !rstd || !dY || !dX)) return DSV_EINVAL;
    if (!dgamma != !dbeta) return DSV_EINVAL;
    if (!on_elements({X, gamma, dY, dX}, esize(p->dtype)) || !on_elements({mean, rstd, dgamma, dbeta}, 4)) return DSV_EINVAL;
    st = check_workspace(workspace, ws_bytes, dgamma ? norm_bwd_bytes(*p) : 0);
    if (st != DSV_OK) return st;
    const bool wide = wide_rows(*p, {X, gamma, dY, dX}, {p->x, p->dy, p->dx});
    return launch_norm_bwd(norm_args(*p), p->dtype, wide, X, gamma, mean, rstd, dY, dX, dgamma, dbeta, dgamma ? static_cast<float *>(workspace) : nullptr,
                           static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
