// Prints how calls of attention over the cache run: of each descriptor on the standard input, a line "few pieces keys-a-piece workspace".  The library's
// own plan, built into this program by including its source.
#include <cstdio>

#include "api_block.hip"

int main()
{
    int n_seq, total, max_new, max_len, Hq, Hkv, d, dtype, n_pages, page, max_pages, causal;
    while (std::scanf("%d %d %d %d %d %d %d %d %d %d %d %d", &n_seq, &total, &max_new, &max_len, &Hq, &Hkv, &d, &dtype, &n_pages, &page, &max_pages, &causal) == 12) {
        dsv_cache p{};
        p.n_seq = n_seq, p.total = total, p.max_new = max_new, p.max_len = max_len;
        p.Hq = Hq, p.Hkv = Hkv, p.d = d, p.dtype = dtype;
        p.n_pages = n_pages, p.page = page, p.max_pages = max_pages;
        p.causal = causal, p.scale = 1.f;
        if (dsv::check_cache(&p) != DSV_OK) {
            std::printf("refused\n");
            continue;
        }
        const dsv::Walk w = dsv::walk_of(p);
        std::printf("%d %d %d %zu\n", w.few ? 1 : 0, w.splits, w.chunk, dsv_cache_attn_fwd_workspace(&p));
    }
    return 0;
}
