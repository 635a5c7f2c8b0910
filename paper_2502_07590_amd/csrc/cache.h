// A cache of K and V in 8 bits, page by page: what its kernels and their callers share.
//
// A page holds `page` tokens of every head, [Hkv][page][d] e4m3 values each of K and V, and one scale a head: a power of two, so that widening
// a value to bf16 is exact, and moving a page's values to a larger scale exact but for those that leave the normal range.
#pragma once

#include "packed_attn.h"
#include "rotary.h"

namespace dsv {

struct CacheArgs {
    const int32_t *cu, *lens, *table;
    int32_t n_seq, total, max_new;
    int32_t Hkv, n_pages, page, page_log2, max_pages;
    int32_t max_len;  // at most what a row of the table holds
};
// New tokens of a sequence: tokens q0 .. q0 + nq - 1 of the call's tensors, the last nq of the nk that its pages then hold.  Whatever cu and lens say,
// nothing leads out of the tensors or the row of the table.
__device__ __forceinline__ Sequence read_cached(const CacheArgs &a, int i)
{
    Sequence s;
    s.q0 = min(max(a.cu[i], 0), a.total);
    s.nq = min(min(max(a.cu[i + 1], s.q0), a.total) - s.q0, a.max_new);
    s.k0 = 0;
    s.nk = min(max(a.lens[i], 0), a.max_len);
    return s;
}

struct AppendIn {
    const void *K, *V;
    int64_t k_row, k_head, v_row, v_head;  // elements
    TurnArgs turn;                          // total = 0: K goes in as it is
    bool eights;
};
dsv_status launch_cache_append(const CacheArgs &a, const AppendIn &in, int dtype, int d, uint8_t *K8, uint8_t *V8, float *kscale, float *vscale, hipStream_t st);

}  // namespace dsv
