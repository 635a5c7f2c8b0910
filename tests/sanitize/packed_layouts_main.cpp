// Driver for a sanitized build of the host side of packed attention and layer norm: layouts whose strides times counts pass 64 bits, and
// layouts that a call does not read.  Every call returns before any kernel launch (a query, or an argument error).
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "dsv.h"

#define CHECK(c) do { if (!(c)) { std::fprintf(stderr, "check failed: %s (line %d)\n", #c, __LINE__); std::exit(1); } } while (0)

static void *const one = reinterpret_cast<void *>(256);
static int32_t *const ints = static_cast<int32_t *>(one);
static float *const floats = static_cast<float *>(one);

// Whether a backward is accepted (it then lacks its workspace) or refused for what the descriptor says.
static bool accepted(const dsv_packed &p)
{
    const dsv_status st = dsv_packed_attn_bwd(&p, one, one, one, ints, ints, one, nullptr, floats, one, one, one, one, nullptr, 0, nullptr);
    CHECK(st == DSV_EWORKSPACE || st == DSV_EINVAL || st == DSV_EUNSUPPORTED);
    CHECK((st == DSV_EWORKSPACE) == (dsv_packed_attn_bwd_workspace(&p) > 0));
    return st == DSV_EWORKSPACE;
}
static bool accepted(const dsv_norm &p)
{
    const dsv_status st = dsv_layer_norm_bwd(&p, one, one, floats, floats, one, one, floats, floats, nullptr, 0, nullptr);
    CHECK(st == DSV_EWORKSPACE || st == DSV_EINVAL || st == DSV_EUNSUPPORTED);
    return st == DSV_EWORKSPACE;
}
// rows of n elements, one [rows, heads] of them, apart from one another: in more bits than any product here needs
static bool apart(const dsv_rows &s, int64_t rows, int64_t heads, int64_t n)
{
    const __int128 row = s.row, head = s.head;
    if (rows <= 1 && heads <= 1) return true;
    if (rows <= 1) return head >= n;
    if (heads <= 1) return row >= n;
    return (head >= n && row >= (heads - 1) * head + n) || (row >= n && head >= (rows - 1) * row + n);
}

int main()
{
    const int64_t strides[] = {0, 8, 64, 128, 1 << 10, 1 << 20, 1ll << 33, 1ll << 34, (1ll << 39) + 8, (1ll << 40) - 8};
    int yes = 0, no = 0;
    for (int heads : {1, 2, 64, 1 << 20, 15728640})      // of outputs; few enough blocks for a launch
        for (int tokens : {0, 1, 2, 3, 1000})
            for (int64_t row : strides)
                for (int64_t head : strides)
                    for (int which = 0; which < 3; ++which) {
                        if ((int64_t)tokens * heads / 32 + heads >= 1 << 24) continue;
                        dsv_packed p{};
                        p.n_seq = 1, p.total_q = p.max_q = p.total_k = p.max_k = tokens;
                        p.Hq = p.Hkv = heads, p.d = 64, p.dtype = DSV_BF16, p.scale = 0.1f;
                        p.q = p.k = p.v = p.o = p.dO = p.dq = p.dk = p.dv = dsv_rows{64, (int64_t)64 * (tokens ? tokens : 1)};
                        if (tokens > 0) CHECK(accepted(p));
                        (which == 0 ? p.dq : which == 1 ? p.dk : p.dv) = dsv_rows{row, head};
                        if (tokens == 0) continue;       // nothing to keep: an accepted call would go on
                        const bool want = apart(dsv_rows{row, head}, tokens, heads, 64);
                        CHECK(accepted(p) == want);
                        ++(want ? yes : no);
                    }
    // shared heads far from one another, of queries that do not exist too
    for (int heads : {2, 1 << 20, 15728640, 0x7FFFFFFF})
        for (int tokens : {0, 1, 16})
            for (int64_t head : strides) {
                dsv_packed p{};
                p.n_seq = 1, p.total_q = p.max_q = tokens, p.total_k = p.max_k = 5, p.Hq = heads, p.Hkv = 1, p.d = 64, p.dtype = DSV_BF16, p.scale = 0.1f;
                p.q = p.o = p.dO = p.dq = dsv_rows{64, 64 * 16};
                p.k = p.v = p.dk = p.dv = dsv_rows{64, 64};
                p.q.head = p.dO.head = head;
                const bool fits = (__int128)128 * 64 * 2 + (__int128)(heads - 1) * head * 2 < (__int128)1 << 32 && (__int128)tokens * heads * heads < (__int128)1 << 32;
                CHECK(dsv_packed_attn_bwd_workspace(&p) == 0 || fits);
                if (tokens > 0) CHECK(accepted(p) == fits);
                ++(fits ? yes : no);
            }
    for (int heads : {1, 2, 1 << 20, 1073741823})
        for (int tokens : {1, 2, 1000, 1073741823})
            for (int64_t row : strides)
                for (int64_t head : strides) {
                    if ((int64_t)tokens * heads >= 1ll << 31) continue;
                    dsv_norm p{};
                    p.tokens = tokens, p.heads = heads, p.n = 64, p.dtype = DSV_F32, p.eps = 1e-5f;
                    p.x = p.y = p.dy = p.dx = dsv_rows{(int64_t)heads * 64 % (1ll << 40), 64};
                    p.dx = dsv_rows{row, head};
                    const bool want = apart(p.dx, tokens, heads, 64);
                    CHECK(accepted(p) == want);
                    ++(want ? yes : no);
                }
    CHECK(yes > 300 && no > 300);
    // what the forward does not read
    for (int64_t left : {(int64_t)1 << 26, (int64_t)1 << 62, (int64_t)0x5555555555555555, INT64_MIN, (int64_t)-8}) {
        dsv_packed p{};
        p.n_seq = 8, p.total_q = 8, p.total_k = 80000, p.max_q = 1, p.max_k = 10000, p.Hq = 8, p.Hkv = 2, p.d = 128, p.dtype = DSV_BF16, p.scale = 0.1f;
        p.q = p.o = dsv_rows{1024, 128};
        p.k = p.v = dsv_rows{256, 128};
        const size_t need = dsv_packed_attn_fwd_workspace(&p);
        p.dO = p.dq = p.dk = p.dv = dsv_rows{left, left};
        CHECK(need > 0 && dsv_packed_attn_fwd_workspace(&p) == need);
        CHECK(dsv_packed_attn_fwd(&p, one, one, one, ints, ints, one, nullptr, floats, one, need - 1, nullptr) == DSV_EWORKSPACE);
    }
    std::printf("packed layouts sanitizer run ok: %d accepted, %d refused\n", yes, no);
    return 0;
}
