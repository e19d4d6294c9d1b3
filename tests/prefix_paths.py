"""Which ways a shared-prefix attention call goes: the library's own rule
(csrc/rl_prefix_rule.h, compiled here with g++) over a problem's lengths and groups,
so that a test can say which path it means and fails when a call no longer takes it."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAGE = 16

SOURCE = r"""
#include "rl_prefix_rule.h"
using namespace rl_da;
extern "C" {
void rule(int max_pages, int batch, int groups, int hq, int hkv, long long* out)
{
    const PrefixRule r = prefix_rule(max_pages, batch, groups, hq, hkv);
    const long long v[] = {r.by_rows, r.small, r.unshared_pages, r.alone_pages, r.wanted_shared,
                           r.wanted_own, r.least_shift, r.slots, r.max_units};
    for (int i = 0; i < 9; ++i)
        out[i] = v[i];
}
void splits(int pages, int wanted, int least_shift, int* out)
{
    const Splits s = splits_of(pages, wanted, least_shift);
    out[0] = s.count, out[1] = s.pages, out[2] = s.more;
}
void part(int pages, int wanted, int least_shift, int i, int* out)
{
    const Splits s = splits_of(pages, wanted, least_shift);
    out[0] = s.first(i), out[1] = s.size(i);
}
struct Call : PrefixRule { int batch, max_pages, group_shift; };
// A sequence's units as the plans make them, eight numbers each; returns their number.
// group: the sequence's, as far as it is a member (-1: of none).
static int put(const Unit& u, int* out)
{
    const int v[] = {u.table_row, u.page0, u.pages, u.limit, u.row0, u.rows, u.slot, u.need};
    for (int i = 0; i < 8; ++i)
        out[i] = v[i];
    return 8;
}
int own_units(int max_pages, int batch, int groups, int hq, int hkv, int b, int len, int prefix,
              int company, int* parts, int* out)
{
    Call a;
    static_cast<PrefixRule&>(a) = prefix_rule(max_pages, batch, groups, hq, hkv);
    a.batch = batch, a.max_pages = max_pages, a.group_shift = __builtin_ctz(hq / hkv);
    const Own o = own_of(a, len, prefix, company);
    parts[0] = o.shared, parts[1] = o.s.count;
    for (int i = 0; i < o.s.count; ++i)
        out += put(own_unit(a, b, o, i), out);
    return o.s.count;
}
int shared_units(int max_pages, int batch, int groups, int hq, int hkv, int start, int end,
                 int prefix, int leader, int* out)
{
    Call a;
    static_cast<PrefixRule&>(a) = prefix_rule(max_pages, batch, groups, hq, hkv);
    a.batch = batch, a.max_pages = max_pages, a.group_shift = __builtin_ctz(hq / hkv);
    const Shared h = shared_of(a, start, end, prefix);
    for (int i = 0; i < h.units(); ++i)
        out += put(shared_unit(a, h, leader, i), out);
    return h.units();
}
int tile_rows() { return kTileRows; }
int resident() { return kResident; }
int most_pages() { return kMaxSplitPages; }
int spread_rows() { return kSpreadRows; }
}
"""

FIELDS = ("by_rows", "small", "unshared_pages", "alone_pages", "wanted_shared", "wanted_own",
          "least_shift", "slots", "max_units")


@functools.lru_cache(None)
def library():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "rule.cpp"), os.path.join(d, "rule.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC",
                        "-I", os.path.join(ROOT, "paper_2512_22492_amd", "csrc"), src, "-o", so],
                       check=True)
        return ctypes.CDLL(so)


def rule(max_pages, batch, groups, hq, hkv):
    out = (ctypes.c_longlong * 9)()
    library().rule(max_pages, batch, groups, hq, hkv, out)
    return dict(zip(FIELDS, out))


def splits(pages, wanted, least_shift):
    """(count, pages of each, one more of the first so many)."""
    out = (ctypes.c_int * 3)()
    library().splits(pages, wanted, least_shift, out)
    return tuple(out)


UNIT = ("table_row", "page0", "pages", "limit", "row0", "rows", "slot", "need")


def units(max_pages, hq, hkv, lengths, group_start, prefix_pages):
    """(the units of a call that is not attended by rows, each a dict; every sequence's
    numbers of shared and own partial results)."""
    lib, batch, groups = library(), len(lengths), len(prefix_pages)
    sizes = (max_pages, batch, groups, hq, hkv)
    buf, n = (ctypes.c_int * (8 * 4096))(), (ctypes.c_int * 2)()
    found, parts = [], []

    def take(count):
        for i in range(count):
            found.append(dict(zip(UNIT, buf[8 * i:8 * i + 8])))

    member = {}
    for g in range(groups):
        inside = [b for b in range(group_start[g], group_start[g + 1])
                  if prefix_pages[g] and lengths[b] >= prefix_pages[g] * PAGE]
        member.update({b: g for b in inside})
        if inside:
            take(lib.shared_units(*sizes, group_start[g], group_start[g + 1], prefix_pages[g],
                                  inside[0], buf))
    for b, length in enumerate(lengths):
        g = member.get(b)
        take(lib.own_units(*sizes, b, length, 0 if g is None else prefix_pages[g],
                           g is not None and group_start[g + 1] - group_start[g] > 1, n, buf))
        parts.append(tuple(n))
    return found, parts


def ways(max_pages, hq, hkv, lengths, group_start, prefix_pages):
    """The names of the ways the call takes:
      rows                     one kernel, a work-group per sequence and kv head; else
      small, planned, memory   planned in the attention kernel, by a launch of its own, and
                               that one with its tables in memory
      shared16 .. shared128    units on shared pages of up to so many query rows
      shared splits, tiles     a prefix in several splits, a group in several tiles
      shared once              a unit whose pages no other unit reads
      unshared                 members that read their prefix with their own pages
      own, own splits, alone   own runs of a work-group, in several splits, of a wavefront
      queued, stolen           places beyond the first round, beyond the third
      spread, merge            how partial results are joined"""
    lib = library()
    batch, groups, G = len(lengths), len(prefix_pages), hq // hkv
    r = rule(max_pages, batch, groups, hq, hkv)
    if r["by_rows"]:
        return {"rows"}
    found = {"small"} if r["small"] else {"planned"}
    if batch > 4096 or groups > 2048:
        found.add("memory")
    lengths = [max(0, min(int(n), max_pages * PAGE)) for n in lengths]
    first = [0] * batch
    units = alone = 0
    for g in range(groups):
        pages = max(0, min(int(prefix_pages[g]), max_pages))
        s0, s1 = (max(0, min(int(x), batch)) for x in group_start[g:g + 2])
        members = [b for b in range(s0, s1) if lengths[b] >= pages * PAGE]
        if not pages or not members:
            continue
        if pages <= r["unshared_pages"]:
            found.add("unshared")
            continue
        for b in members:
            first[b] = pages
        rows = (s1 - s0) * G
        tiles = -(-rows // lib.tile_rows())
        count = splits(pages, r["wanted_shared"], r["least_shift"])[0]
        for t in range(tiles):
            n = min(lib.tile_rows(), rows - t * lib.tile_rows())
            found.add("shared%d" % next(c for c in (16, 32, 64, 128) if n <= c))
        units += tiles * count
        found |= {"shared splits"} if count > 1 else set()
        found.add("tiles" if tiles > 1 else "shared once")
    for b, n in enumerate(lengths):
        pages = -(-n // PAGE) - first[b]
        if pages <= 0:
            continue
        count = splits(pages, r["wanted_own"], r["least_shift"])[0]
        if count == 1 and pages <= r["alone_pages"]:
            found.add("alone")
            alone += 1
        else:
            found.add("own splits" if count > 1 else "own")
            units += count
    places = units * hkv + -(-alone * hkv // 4)
    if not r["small"]:
        found |= {"queued"} if places > lib.resident() else set()
        found |= {"stolen"} if places > 3 * lib.resident() else set()
    found.add("spread" if batch * hq < lib.spread_rows() else "merge")
    return found


def ways_of(p):
    """ways() of a problem that carries its group_start and prefix_pages."""
    start = [] if p.group_start is None else p.group_start.cpu().tolist()
    return ways(p.max_pages, p.num_q_heads, p.num_kv_heads, p.seq_lens.cpu().tolist(), start,
                p.prefix_pages.cpu().tolist())
