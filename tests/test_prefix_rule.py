"""How shared-prefix attention calls are cut (csrc/rl_prefix_rule.h, compiled here with
g++): every run is covered within its partial results, and the ways of a call (CPU)."""
import ctypes

import pytest

import prefix_paths as paths

CALLS = [(max_pages, batch, groups, hq, hkv)
         for max_pages in (1, 16, 31, 32, 64, 65, 255, 256, 257, 900, 4096)
         for batch, groups in ((1, 1), (8, 1), (64, 8), (65, 64), (512, 64), (512, 512), (4097, 3))
         for hq, hkv in ((4, 1), (32, 8), (64, 4), (8, 8))]


@pytest.mark.parametrize("hq,hkv", [(4, 1), (32, 8), (64, 4), (8, 8)])
def test_runs_are_covered_within_their_partial_results(hq, hkv):
    lib = paths.library()
    part = (ctypes.c_int * 2)()
    for call in CALLS:
        if call[3:] != (hq, hkv):
            continue
        r = paths.rule(*call)
        most = {"wanted_shared": 0, "wanted_own": 0}
        for pages in sorted({0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 255, 256, 257, 511, 512,
                             513, call[0] - 1, call[0]}):
            if pages > call[0]:
                continue
            for which in most:
                count, each, more = paths.splits(pages, r[which], r["least_shift"])
                assert (count == 0) == (pages == 0)
                most[which] = max(most[which], count)
                at = 0
                for i in range(count):
                    lib.part(pages, r[which], r["least_shift"], i, part)
                    assert part[0] == at and 1 <= part[1] <= lib.most_pages()
                    at += part[1]
                assert at == pages
        # a row's shared results, then its own, fit its slots; all units fit the plan
        assert most["wanted_shared"] + most["wanted_own"] <= r["slots"]
        tiles = -(-(call[1] * hq // hkv) // lib.tile_rows()) + call[2]
        assert tiles * most["wanted_shared"] + call[1] * most["wanted_own"] <= r["max_units"]


def test_ways_of_calls():
    def ways(n, prefix, own, hq=8, hkv=2, width=100, behind=0):
        lens = [prefix * 16 + own] * n + [5] * behind
        return paths.ways(width, hq, hkv, lens, [0, n], [prefix])

    assert ways(8, 20, 9, width=64) == {"rows"}
    assert ways(8, 20, 9) >= {"small", "unshared", "spread"}
    assert ways(8, 60, 9) >= {"small", "shared32", "shared once", "alone", "shared splits"}
    assert ways(8, 60, 9, behind=60) >= {"planned", "shared32"}
    assert ways(40, 60, 9, behind=60) >= {"planned", "shared128", "shared32", "tiles"}
    assert ways(16, 60, 3000, hkv=2) >= {"shared64", "own splits"}
    assert ways(300, 20, 9) >= {"planned", "shared128", "tiles", "merge"}
    assert "memory" in ways(4097, 0, 9, hq=1, hkv=1)
    assert ways(700, 0, 200, hq=8, hkv=8, width=65) >= {"alone", "queued"}
    assert "stolen" in ways(900, 0, 200, hq=8, hkv=8, width=65)
