// Driver for a sanitized build of the host side of packed attention and layer norm: descriptor checks, split plans and workspace sizes over
// the range of what a descriptor can hold; every call returns before any kernel launch (a query, or an argument error).
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "dsv.h"

#define CHECK(c) do { if (!(c)) { std::fprintf(stderr, "check failed: %s (line %d)\n", #c, __LINE__); std::exit(1); } } while (0)

static dsv_packed packed(int n_seq, int64_t tq, int64_t tk, int64_t mq, int64_t mk, int Hq, int Hkv, int d, int dtype, int causal)
{
    dsv_packed p{};
    p.n_seq = n_seq, p.total_q = (int32_t)tq, p.total_k = (int32_t)tk, p.max_q = (int32_t)mq, p.max_k = (int32_t)mk;
    p.Hq = Hq, p.Hkv = Hkv, p.d = d, p.dtype = dtype, p.causal = causal, p.scale = 0.1f;
    p.q = p.o = p.dO = p.dq = dsv_rows{(int64_t)Hq * d, d};
    p.k = p.v = p.dk = p.dv = dsv_rows{(int64_t)Hkv * d, d};
    return p;
}

int main()
{
    void *one = reinterpret_cast<void *>(256);
    int32_t *ints = static_cast<int32_t *>(one);
    float *floats = static_cast<float *>(one);
    const int64_t sizes[] = {0, 1, 2, 63, 64, 65, 127, 128, 129, 1000, 8192, 20280, 131072, 1 << 20, 1 << 24, (1 << 28) + 17, 0x7FFFFFFF};
    int accepted = 0, split = 0;
    for (int64_t tq : sizes)
        for (int64_t tk : sizes)
            for (int n_seq : {1, 2, 3, 65, 4096, 0x7FFFFFFF})
                for (int heads : {1, 4, 16, 1 << 20})
                    for (int group : {1, 3, 8, 64})
                        for (int form = 0; form < 8; ++form) {
                            if ((int64_t)heads * group > 0x7FFFFFFF) continue;
                            const dsv_packed p = packed(n_seq, tq, tk, form & 4 ? 0x7FFFFFFF : tq / n_seq, form & 4 ? 0x7FFFFFFF : tk, heads * group, heads,
                                                        form & 1 ? 64 : 128, form & 2 ? DSV_BF16 : DSV_F32, n_seq % 2);
                            const size_t f = dsv_packed_attn_fwd_workspace(&p), b = dsv_packed_attn_bwd_workspace(&p);
                            // what a forward keeps: at most 64 pieces of every row's sums and statistics
                            CHECK(f <= ((size_t)p.total_q * p.Hq * 64 * (p.d + 2) * 4 + 512));
                            CHECK(f == 0 || p.total_k > 0);
                            if (tq == 0) continue;  // nothing to keep: the call itself would launch
                            const dsv_status st = dsv_packed_attn_bwd(&p, one, one, one, ints, ints, one, nullptr, floats, one, one, one, one, nullptr, 0, nullptr);
                            if (b) {
                                CHECK(b >= (size_t)p.total_q * p.Hq * 8 && st == DSV_EWORKSPACE);
                                CHECK(dsv_packed_attn_bwd(&p, one, one, one, ints, ints, one, nullptr, floats, one, one, one, one, one, b - 1, nullptr) == DSV_EWORKSPACE);
                                ++accepted;
                                split += f > 0;
                            } else {
                                CHECK(st == DSV_EUNSUPPORTED);
                            }
                        }
    CHECK(accepted > 1000 && split > 100);
    for (int tokens : {0, 1, 77, 32768, 0x7FFFFFFF})
        for (int heads : {1, 16, 65536, 0x7FFFFFFF})
            for (int n = 1; n <= 8200; n += n < 300 ? 1 : 97)
                for (int dtype : {DSV_F32, DSV_BF16}) {
                    dsv_norm p{};
                    p.tokens = tokens, p.heads = heads, p.n = n, p.dtype = dtype, p.eps = 1e-5f;
                    p.x = p.y = p.dy = p.dx = dsv_rows{(int64_t)heads * n, n};
                    const size_t b = dsv_layer_norm_bwd_workspace(&p);
                    CHECK(b <= (size_t)1024 * 2 * n * 4 + 256);
                    if (b) CHECK(dsv_layer_norm_bwd(&p, one, one, floats, floats, one, one, floats, floats, one, b - 1, nullptr) == DSV_EWORKSPACE);
                    if (n > 8192) CHECK(dsv_layer_norm_fwd(&p, one, one, one, one, floats, floats, nullptr) == DSV_EUNSUPPORTED);
                }
    std::printf("packed checks sanitizer run ok\n");
    return 0;
}
