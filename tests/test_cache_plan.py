"""How calls of attention over the cache are planned: rows to a block, pieces of the keys, and with them the workspace.  The library's own host code, built with
sanitizers for the CPU; no kernel."""
import os
import subprocess

import pytest

from cache_calls import BEHIND_4_GB, LARGE_TILES, NONSENSE, any_large

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all"]
INT_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """plan(descriptors) -> [(few, pieces, keys a piece, workspace)], None for a descriptor that is refused."""
    from paper_2502_07590_amd.build import CSRC, HIPCC_FLAGS, _hipcc
    tmp = tmp_path_factory.mktemp("plan")
    flags = [f for f in HIPCC_FLAGS if f != "-O3" and not f.startswith("--offload-arch")] + ["-O1", "-g", "--offload-host-only", *SAN]
    objs = []
    for src in (os.path.join(ROOT, "tests", "sanitize", "cache_plan_main.cpp"), os.path.join(CSRC, "api_packed.hip")):
        objs.append(str(tmp / (os.path.basename(src) + ".o")))
        res = subprocess.run([_hipcc(), "-x", "hip", *flags, "-c", src, "-o", objs[-1]], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-3000:]
    exe = str(tmp / "plan")
    # the kernels' launchers are not there; no line here calls them
    res = subprocess.run([_hipcc(), "--offload-host-only", *SAN, "-Wl,--unresolved-symbols=ignore-all", "-o", exe, *objs], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")

    def run(descriptors):
        res = subprocess.run([exe], input="\n".join(" ".join(str(int(x)) for x in c) for c in descriptors), capture_output=True, text=True, env=env)
        assert res.returncode == 0, res.stderr[-3000:]
        lines = res.stdout.splitlines()
        assert len(lines) == len(descriptors)
        return [None if x == "refused" else tuple(int(y) for y in x.split()) for x in lines]

    return run


def described(new, lens, Hq, Hkv, d, page, dtype, causal=True, behind=0, max_len=None):
    pages = [-(-n // page) for n in lens]
    return (len(new), sum(new) + behind, max(new), INT_MAX if max_len is None else max_len, Hq, Hkv, d, 1 if dtype == "bf16" else 0, sum(pages) + 1, page, max(max(pages), 1) + 1, causal)


def test_the_calls_for_blocks_of_128_rows_run_in_them(plan):
    calls = [described(*c, causal, 2, max(c[1])) for c in LARGE_TILES for causal in (False, True)]
    got = plan(calls)
    assert not any(few for few, *_ in got)
    assert sum(pieces > 1 for _, pieces, *_ in got) >= len(got) // 2 and sum(pieces == 1 for _, pieces, *_ in got) >= 4
    more = [described(*call, causal, behind) for call, causal, _, behind in map(any_large, range(8))] + [described(*BEHIND_4_GB)]
    n_seq, T, most, Hq, Hkv, d, page, max_pages = NONSENSE
    more += [(n_seq, T, most, INT_MAX, Hq, Hkv, d, dtype, 6, page, max_pages, True) for dtype in (0, 1)]
    assert not any(few for few, *_ in plan(more))


def test_workspaces_hold_every_piece(plan):
    """Pieces are whole tiles, cover the longest cache, are no more than a join takes, and the workspace holds what all of them leave."""
    calls = [(n, total, max(1, most), max_len, Hkv * g, Hkv, d, dtype, 1000, 64, max(1, -(-max_len // 64)), causal)
             for n, total, most in ((1, 1, 1), (1, 1560, 1560), (3, 77, 60), (64, 64, 1), (300, 90000, 300), (7, 20000, 9000))
             for max_len in (1, 255, 1024, 1025, 9000, 70001, 1 << 24, 1 << 30) for Hkv, g in ((1, 1), (2, 7), (16, 2), (128, 1)) for d in (64, 128) for dtype in (0, 1) for causal in (0, 1)]
    split = 0
    for c, got in zip(calls, plan(calls)):
        assert got is not None, c
        few, pieces, keys, ws = got
        rows, d, longest = c[1] * c[4], c[6], min(c[3], c[9] * c[10])
        assert 1 <= pieces <= 64, c
        if pieces == 1:
            assert keys == 0 and ws == 0, c
            continue
        split += 1
        assert keys % 128 == 0 and (pieces - 1) * keys < longest <= pieces * keys and longest + keys < 2 ** 31, c
        assert rows * pieces * (d + 2) * 4 <= ws <= rows * pieces * (d + 2) * 4 + 512, c
    assert split > 200


def equal(n, new, length, Hq, Hkv, d=128, dtype="bf16"):
    return described([new] * n, [length] * n, Hq, Hkv, d, 64, dtype, max_len=length)


def test_calls_that_fill_the_chip_are_not_cut_into_pieces(plan):
    """Batches of one size whose blocks of 128 rows fill the chip four times over: pieces would save nothing, and leave hundreds of MB to write and to join."""
    for c in (equal(32, 256, 8000, 32, 8), equal(4, 4096, 32768, 32, 8), equal(12, 3400, 5000, 32, 8), equal(4, 2000, 1500, 12, 12, dtype="f32"), equal(32, 1142, 1684, 12, 4, dtype="f32"),
              equal(16, 1560, 4000, 16, 16, d=64)):
        assert plan([c]) == [(0, 1, 0, 0)], c
    # three times over: the last round is worth a few
    assert all(pieces <= 5 for _, pieces, *_ in plan([equal(8, 1560, 21840, 16, 16), equal(8, 1560, 21840, 16, 4)]))


def test_long_caches_that_leave_the_chip_empty_are_cut(plan):
    """One long cache among short ones, and a few long ones: blocks for all CUs."""
    calls = [described([300] * 3, [30000, 4000, 200], 16, 4, 128, 64, "bf16", max_len=30000), described([1560] * 2, [21840, 7800], 8, 2, 128, 64, "bf16", max_len=21840),
             described([129], [14912], 16, 4, 128, 64, "f32", max_len=14912), described([1045, 63], [8208, 192], 12, 3, 128, 64, "bf16", max_len=8208)]
    for (few, pieces, *_), (at_least, at_most) in zip(plan(calls), ((8, 24), (4, 12), (10, 12), (4, 6))):
        assert not few and at_least <= pieces <= at_most
