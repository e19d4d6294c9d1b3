"""How shared-prefix attention calls are cut (csrc/rl_prefix_rule.h, compiled here with
g++): every run is covered within its partial results, and the ways of a call (CPU)."""
import collections
import ctypes
import random

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


def calls():
    rng = random.Random(7)
    for hq, hkv, count, most in ((4, 1, 40, 40), (32, 8, 6, 9), (32, 8, 64, 8), (8, 8, 2, 32),
                                 (64, 4, 1, 128), (64, 4, 30, 4), (2, 1, 100, 5), (16, 1, 3, 40)):
        sizes = [rng.choice([0, 1, most, rng.randint(1, most)]) for _ in range(count)]
        prefix = [rng.choice([0, 1, 20, 47, 48, 49, 64, 257, 700, rng.randint(1, 100)]) for _ in sizes]
        start = [2]
        for n in sizes:
            start.append(start[-1] + n)
        lengths = [40, 0]
        for n, pages in zip(sizes, prefix):
            lengths += [rng.choice([0, max(0, pages * 16 - 1), pages * 16, pages * 16 + 1,
                                    pages * 16 + rng.randint(1, 600),
                                    pages * 16 + rng.randint(1, 6000)]) for _ in range(n)]
        lengths += [rng.randint(0, 3000) for _ in range(3)]
        yield hq, hkv, lengths, start, prefix


@pytest.mark.parametrize("call", list(calls()), ids=lambda c: "%d-%d-%d" % (c[0], c[1], len(c[2])))
def test_units_cover_every_key_once_and_know_who_else_reads_it(call):
    """Each row meets each of its sequence's keys in one unit; its partial results have
    places of their own; and a unit is marked where another reads pages of it, which is
    what decides on the loads' hint."""
    hq, hkv, lengths, start, prefix = call
    G, width = hq // hkv, max(800, max(-(-n // 16) for n in lengths))
    found, parts = paths.units(width, hq, hkv, lengths, start, prefix)
    r = paths.rule(width, len(lengths), len(prefix), hq, hkv)
    assert not r["by_rows"] and len(found) <= r["max_units"]
    member = {}
    for g, pages in enumerate(prefix):
        for b in range(start[g], start[g + 1]):
            if pages and lengths[b] >= pages * 16:
                member[b] = g
    keys, slots = collections.Counter(), collections.defaultdict(list)
    readers = collections.Counter()
    for u in found:
        pages = range(u["page0"], u["page0"] + u["pages"])
        for c in pages:   # a page that members share has one name
            g = member.get(u["table_row"])
            u.setdefault("names", []).append(
                ("g", g, c) if g is not None and c < prefix[g] else (u["table_row"], c))
        readers.update(u["names"])
        last = min(u["limit"], (u["page0"] + u["pages"]) * 16)
        for row in range(u["row0"], u["row0"] + abs(u["rows"])):
            b = row // G
            if lengths[b] < u["need"]:
                continue
            assert b == u["table_row"] or member[b] == member[u["table_row"]]
            keys[row] += last - u["page0"] * 16
            slots[row].append((u["slot"], u["page0"] * 16, last))
    for b, n in enumerate(lengths):
        for row in range(b * G, (b + 1) * G):
            assert keys[row] == n
            spans = sorted(s[1:] for s in slots[row])
            assert all(x[1] == y[0] for x, y in zip(spans, spans[1:]))
            places = sorted(s[0] for s in slots[row])
            if places == [-1]:
                assert parts[b] == (0, 1)
            else:
                assert places == list(range(sum(parts[b]))) and len(places) <= r["slots"]
    for u in found:
        others = any(readers[x] > 1 for x in u["names"])
        lone = u["table_row"] in member and u["page0"] < prefix[member[u["table_row"]]] and not any(
            b != u["table_row"] and member.get(b) == member[u["table_row"]]
            for b in range(len(lengths)))   # its group's others have ended
        assert (u["rows"] < 0) == others or lone, u
