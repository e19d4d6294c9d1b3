"""GPU decode attention over shared prefixes against the fp64 oracle's decode of
the same cache (the oracle reads every sequence's whole table row; shared pages are
just pages that several rows name)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2512_22492_amd import binding as B
from paper_2512_22492_amd import workloads

from gpu_util import (P_ROUND, PV_ROUND, bf16_to_f64, check_close, device, oracle_ref)

pytestmark = pytest.mark.gpu

PAGE = 16


def extra(p, ref):
    """Allowance on top of one bf16 ulp.  Own keys' weights enter the value product as
    two bf16 terms (PV_ROUND M1); a group of many rows may round its shared keys'
    weights to one bf16 each, normalised by the sum of the same rounded weights in
    bf16 pools and of the unrounded ones in e4m3 pools: at most P_ROUND (M1 + |o|)
    either way, as worked out for extend."""
    # A rounding by a relative e changes a sum of w_j c_j s_j by at most e sum w_j |c_j| |s_j|
    # = e M1.  oracle_ref clears the codes' signs only, so |s_j| is passed in; with the
    # positive scales of other tests that is the same number.
    signed, p.v_scale = p.v_scale, None if p.v_scale is None else p.v_scale.abs()
    m1 = oracle_ref(p, abs_values=True)
    p.v_scale = signed
    return P_ROUND * (m1 + np.abs(ref)) + PV_ROUND * m1


def problem(sizes, prefix, lengths, hq=8, hkv=2, kv="bf16", layout="hnd", seed=1, max_pages=None,
            before=0, behind=0, poison=True):
    """Groups of `sizes` sequences sharing `prefix` pages each; `before` and `behind`
    sequences outside any group at the batch's ends.  Lengths per sequence.  Slots
    past each sequence's end hold NaN where nobody else reads them, and so do the
    pages that no table names; entries past a sequence's pages are out of range."""
    lengths = [int(x) for x in lengths]
    assert len(lengths) == before + sum(sizes) + behind
    start = np.concatenate([[0], np.cumsum(sizes)]) + before
    width = max(1, max(-(-L // PAGE) for L in lengths), max(list(prefix) + [0]))
    p = workloads.make_problem("prefix", batch=len(lengths), num_q_heads=hq, num_kv_heads=hkv,
                               lengths=[width * PAGE] * len(lengths), kv_dtype=kv, seed=seed,
                               layout=layout, max_pages=max(max_pages or 0, width))
    table = p.block_table.clone()
    for g, n in enumerate(prefix):
        if sizes[g]:
            table[start[g]:start[g + 1], :n] = table[start[g], :n].clone()
    p.block_table = table
    p.seq_lens = torch.tensor(lengths, dtype=torch.int32)
    if poison:
        seen = {}
        for b, L in enumerate(lengths):
            for c in range(-(-L // PAGE)):
                page = int(table[b, c])
                seen[page] = max(seen.get(page, 0), min(L - c * PAGE, PAGE))
        nan = 0x7F if kv != "bf16" else float("nan")
        for page in range(p.num_pages):
            live = seen.get(page, 0)
            for pool in (p.k_pool, p.v_pool):
                if layout == "nhd":
                    pool[page, live:] = nan
                else:
                    pool[page, :, live:] = nan
            if live == 0 and kv != "bf16":
                p.k_scale[page] = float("nan")
                p.v_scale[page] = float("nan")
    g = p.to(device())
    # the oracle never looks at entries past a sequence's pages; nor may the kernel
    wild = g.block_table.clone()
    for b, L in enumerate(lengths):
        wild[b, -(-L // PAGE):] = p.num_pages + 12345
    g.block_table = wild
    g.group_start = torch.tensor(start.astype(np.int32), device=device())
    g.prefix_pages = torch.tensor(list(prefix), dtype=torch.int32, device=device())
    return g


def run(p, **kw):
    out = torch.full_like(p.q, float("nan"))
    B.prefix_attention(p, p.group_start, p.prefix_pages, out, **kw)
    torch.cuda.synchronize()
    return out


def check(p, what, **kw):
    print("case", what, flush=True)
    ref = oracle_ref(p)
    out = run(p, **kw)
    print(check_close(bf16_to_f64(out), ref, what, extra_abs=extra(p, ref)))
    return out


LAYOUTS = ["hnd", "nhd", "hnd_kv"]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2), (4, 1), (16, 2), (16, 1)])
def test_head_layouts(hq, hkv, kv, layout):
    """1, 2, 4, 8 and 16 query heads per kv head; lengths around page ends, a group
    of one, an empty sequence, one at its prefix's very end, one shorter than it."""
    p = problem([4, 1, 3], [5, 2, 1], [80, 81, 95, 200, 47, 16, 0, 9], hq=hq, hkv=hkv, kv=kv,
                layout=layout, seed=10)
    check(p, "heads %d/%d %s %s" % (hq, hkv, kv, layout))


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("size", [1, 2, 3, 4, 5, 8, 9, 16, 17, 31, 33, 65, 130])
def test_group_sizes(size, kv):
    """Rows per shared unit from one to several tiles, G = 4."""
    rng = np.random.default_rng(size)
    p = problem([size], [20], 20 * PAGE + rng.integers(0, 70, size), hq=8, hkv=2, kv=kv, seed=20)
    check(p, "group of %d %s" % (size, kv))


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_many_groups_of_all_kinds(kv):
    """Groups without members, without sequences, without a prefix, sequences outside
    any group on both sides, finished ones and ones shorter than their prefix."""
    rng = np.random.default_rng(3)
    sizes = [3, 0, 8, 1, 0, 5, 2, 7, 4]
    prefix = [0, 4, 9, 3, 0, 1, 12, 6, 30]
    lengths = []
    for n, pages in zip(sizes, prefix):
        lengths += list(pages * PAGE + rng.integers(0, 200, n))
    lengths = np.array([17, 300] + lengths + [1, 0, 64])
    lengths[rng.random(lengths.size) < 0.2] = 0
    at = 2 + int(np.cumsum(sizes)[4])
    lengths[at:at + 5] = [3, 0, 15, 7, 1]        # nobody fills group 5's page
    lengths[-5] = 30 * PAGE - 1                  # one token short of its prefix
    p = problem(sizes, prefix, lengths, hq=16, hkv=4, kv=kv, seed=30, before=2, behind=3)
    check(p, "kinds of groups " + kv)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_long_prefixes_and_long_responses_are_split(kv, layout):
    """Runs past one unit's 256 pages, shared and own, in a table wider than both."""
    p = problem([6, 2], [300, 33], [300 * PAGE + n for n in (1, 700, 0, 4500, 5000, 16)]
                + [33 * PAGE + 9000, 33 * PAGE + 2], hq=4, hkv=1, kv=kv, layout=layout, seed=40,
                max_pages=900)
    check(p, "splits %s %s" % (kv, layout))


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_one_prefix_under_a_large_batch(kv):
    rng = np.random.default_rng(5)
    n = 150
    lens = 64 * PAGE + rng.integers(0, 90, n)
    lens[7] = 0
    lens[100] = 63 * PAGE
    p = problem([n], [64], lens, hq=16, hkv=1, kv=kv, seed=50)
    check(p, "system prompt " + kv)


def test_no_groups_is_a_decode_step():
    p = problem([], [], [0, 1, 15, 16, 17, 300, 4200], before=7, seed=60)
    assert p.group_start.numel() == 1
    check(p, "no groups")
    p.group_start = None
    ref, out = oracle_ref(p), torch.full_like(p.q, float("nan"))
    rc, n = B.rl_prefix_attn_workspace_size(p.max_pages, p.batch, 0, 8, 2)
    ws = torch.empty(n, dtype=torch.uint8, device=device())
    assert B.rl_prefix_attn(p.q, p.k_pool, p.v_pool, None, None, p.num_pages, p.block_table,
                            p.max_pages, p.seq_lens, p.batch, None, None, 0, 8, 2,
                            scale=p.scale, out=out, workspace=ws,
                            workspace_bytes=n) == B.RL_DA_OK
    torch.cuda.synchronize()
    check_close(bf16_to_f64(out), ref, extra_abs=extra(p, ref))


@pytest.mark.parametrize("groups", [1500, 2500, 5000])
def test_more_sequences_and_groups_than_the_plan_has_threads(groups):
    rng = np.random.default_rng(6)
    sizes = [int(x) for x in rng.integers(0, 3, groups)]
    prefix = [int(x) for x in rng.integers(0, 3, groups)]
    lens = np.repeat(prefix, sizes) * PAGE + rng.integers(0, 20, sum(sizes))
    p = problem(sizes, prefix, lens, hq=1, hkv=1, seed=70, poison=False)
    check(p, "%d groups of %d sequences" % (groups, sum(sizes)))


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("batch", [1, 63, 64, 65])
def test_small_calls_and_the_next_larger(batch, kv):
    """Up to 64 sequences and groups a call is planned in another way than above: the
    same groups either way, down to groups of one and sequences in none."""
    rng = np.random.default_rng(batch)
    sizes, left = [], batch - min(batch - 1, 3)
    while left:
        sizes.append(int(rng.integers(0, min(left, 9) + 1)))
        left -= sizes[-1]
    prefix = [int(x) for x in rng.integers(0, 40, len(sizes))]
    lens = np.repeat(prefix, sizes) * PAGE + rng.integers(0, 700, sum(sizes))
    behind = batch - sum(sizes)
    lens = np.concatenate([lens, rng.integers(0, 300, behind)])
    lens[rng.random(batch) < 0.1] = 0
    p = problem(sizes, prefix, lens, hq=8, hkv=2, kv=kv, seed=71, behind=behind)
    check(p, "batch %d %s" % (batch, kv))


def test_many_groups_of_few_sequences():
    """64 and 65 groups, most without sequences, over a batch of 40."""
    for groups in (64, 65):
        sizes = [1 if g % 3 == 1 else (2 if g % 7 == 0 else 0) for g in range(groups)]
        sizes[-1] += 40 - sum(sizes)
        prefix = [(5 * g) % 11 for g in range(groups)]
        lens = np.repeat(prefix, sizes) * PAGE + np.arange(40) * 3
        check(problem(sizes, prefix, lens, hq=4, hkv=1, seed=72), "%d groups" % groups)


def test_scales_of_either_sign_and_zero():
    for scale in (0.0, -0.125, 2.0):
        p = problem([5, 3], [6, 2], [100, 96, 130, 0, 97, 32, 50, 33], seed=80, kv="bf16")
        p.scale = scale
        check(p, "scale %g" % scale)


def test_extreme_scores_and_infinities_in_masked_places():
    """Scores that leave fp16's range and one key that takes all the weight; slots past
    the lengths hold infinities."""
    p = problem([4], [3], [60, 48, 100, 49], hq=8, hkv=2, seed=81, poison=False)
    p.q.mul_(300.0)
    last = [int(p.block_table[b, 3]) for b in (0, 2, 3)]
    p.k_pool[last[0], :, 12:] = float("inf")
    p.v_pool[last[0], :, 12:] = float("-inf")
    p.v_pool[last[2], :, 1:] = float("inf")
    check(p, "extreme scores")


def test_a_row_of_one_token_is_its_value():
    p = problem([3], [1], [16, 17, 1], hq=4, hkv=4, seed=82)
    p.seq_lens[0] = 0
    out = check(p, "one token")
    assert torch.equal(out[2], p.v_pool[int(p.block_table[2, 0]), :, 0])
    assert not out[0].any()


def test_results_repeat_and_do_not_depend_on_other_sequences_values():
    p = problem([8, 5], [40, 7], [40 * PAGE + 37 * i for i in range(8)]
                + [7 * PAGE + 11 * i for i in range(5)], hq=8, hkv=2, seed=90)
    first = run(p)
    for _ in range(3):
        assert torch.equal(run(p).view(torch.int16), first.view(torch.int16))
    # another batch through the same table: sequence 3's own pages change
    own = p.block_table[3, 40:42].long()
    p.k_pool[own] = 1.0
    changed = run(p)
    keep = [i for i in range(13) if i != 3]
    assert torch.equal(changed[keep].view(torch.int16), first[keep].view(torch.int16))
    assert not torch.equal(changed[3], first[3])


def test_workspace_of_any_contents_on_another_stream():
    p = problem([9, 4], [12, 3], [200 + 31 * i for i in range(13)], seed=91, kv="fp8_e4m3")
    want = run(p)
    rc, n = B.rl_prefix_attn_workspace_size(p.max_pages, p.batch, 2, 8, 2)
    assert rc == B.RL_DA_OK
    s = torch.cuda.Stream()
    for fill in (0x00, 0xFF, 0x7F):
        guard = torch.full((n + 64,), fill, dtype=torch.uint8, device=device())
        out = torch.full_like(p.q, float("nan"))
        s.wait_stream(torch.cuda.current_stream())
        B.prefix_attention(p, p.group_start, p.prefix_pages, out, stream=s, workspace=guard[:n])
        s.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        assert (guard[n:] == fill).all()
    # the object's own workspace, on a stream of the caller's and after the object is gone
    out = torch.full_like(p.q, float("nan"))
    B.PrefixAttention(p, p.group_start, p.prefix_pages)(p.q, out, s)
    s.synchronize()
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))


def test_bad_pages_and_lengths_are_reported_and_stay_where_they_are():
    p = problem([3, 3], [2, 2], [50, 60, 40, 50, 60, 40], seed=92, poison=False)
    err = torch.zeros(1, dtype=torch.int32, device=device())
    want = run(p, device_error=err)
    assert int(err) == 0
    bad = p.block_table.clone()
    bad[4, 2] = -1                               # an own page of sequence 4
    good, p.block_table = p.block_table, bad
    out = run(p, device_error=err)
    assert int(err) == B.RL_DA_DEVERR_PAGE_OUT_OF_RANGE
    keep = [0, 1, 2, 3, 5]
    assert torch.equal(out[keep].view(torch.int16), want[keep].view(torch.int16))
    bad[4, 2] = good[4, 2]
    bad[0:3, 1] = p.num_pages                    # a shared page of group 0
    err.zero_()
    out = run(p, device_error=err)
    assert int(err) == B.RL_DA_DEVERR_PAGE_OUT_OF_RANGE
    assert torch.equal(out[3:].view(torch.int16), want[3:].view(torch.int16))
    # a length beyond the table is cut there
    p.block_table = good.clone()
    p.block_table[1, 3] = good[0, 3]
    p.seq_lens[1] = p.max_pages * PAGE
    err.zero_()
    full = run(p, device_error=err)
    assert int(err) == 0
    p.seq_lens[1] = p.max_pages * PAGE + 1
    out = run(p, device_error=err)
    assert int(err) == B.RL_DA_DEVERR_LENGTH_TOO_LONG
    assert torch.equal(out.view(torch.int16), full.view(torch.int16))


def test_groups_that_run_backwards_write_only_their_outputs():
    """group_start is a precondition; a call that breaks it stays inside its buffers."""
    p = problem([6, 6, 6], [4, 4, 4], [100] * 18, hq=16, hkv=1, seed=93)
    rc, n = B.rl_prefix_attn_workspace_size(p.max_pages, p.batch, 3, 16, 1)
    guard = torch.full((n + 256,), 0x5A, dtype=torch.uint8, device=device())
    out = torch.full((19, 16, 128), 7.0, dtype=torch.bfloat16, device=device())
    for starts in ([0, 18, 0, 18], [12, 18, -5, 1000], [18, 0, 18, 0]):
        p.group_start.copy_(torch.tensor(starts, dtype=torch.int32))
        B.prefix_attention(p, p.group_start, p.prefix_pages, out[:18], workspace=guard[:n])
        torch.cuda.synchronize()
        assert (guard[n:] == 0x5A).all() and (out[18] == 7.0).all()


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_replays_equal_the_eager_run(kv):
    """Captured once, replayed as the sequences grow, with eager work on another
    workspace between the replays."""
    lens = [20 * PAGE + 7 * i for i in range(10)] + [33, 0]
    p = problem([10, 2], [20, 2], lens, hq=8, hkv=2, kv=kv, seed=94, max_pages=40, poison=False)
    full = p.block_table.clone()
    full[:] = 0
    for b in range(p.batch):                      # room to grow into
        pages = torch.arange(40, dtype=torch.int32) + 40 * b
        full[b] = pages.to(device()) % p.num_pages
    full[:10, :20] = full[0, :20].clone()
    full[10:, :2] = full[10, :2].clone()
    p.block_table.copy_(full)
    attn = B.PrefixAttention(p, p.group_start, p.prefix_pages)
    out = torch.full_like(p.q, float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        attn(p.q, out, side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attn(p.q, out, torch.cuda.current_stream())
    for step in range(5):
        eager = run(p)
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16)), step
        ref = oracle_ref(p)
        check_close(bf16_to_f64(out), ref, "step %d" % step, extra_abs=extra(p, ref))
        p.seq_lens += 11
    del g


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_pages_beyond_4_gib(layout):
    """Page offsets past 32 bits: the same pages at the end of a 4.3 GiB pool and in a
    small one give the same bits, split and whole, shared and own."""
    small = problem([5, 2], [70, 3], [70 * PAGE + 9 * i for i in range(5)] + [50, 61], hq=32,
                    hkv=8, layout=layout, seed=95, poison=False)
    want = run(small)
    n = small.num_pages
    pages = (9 << 29) // (8 * PAGE * 128 * 2)            # 4.5 GiB
    shape = (pages,) + tuple(small.k_pool.shape[1:])
    k, v = (torch.empty(shape, dtype=torch.bfloat16, device=device()) for _ in range(2))
    k[-n:], v[-n:] = small.k_pool, small.v_pool
    big = workloads.DecodeProblem(**{**{f: x for f, x in small.__dict__.items()
                                        if f not in ("group_start", "prefix_pages")},
                                     "k_pool": k, "v_pool": v,
                                     "block_table": small.block_table + (pages - n)})
    big.group_start, big.prefix_pages = small.group_start, small.prefix_pages
    assert torch.equal(run(big).view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("size", [1, 6, 14, 40])
def test_page_scales_of_any_sign(size):
    """e4m3 slabs whose scales are negative or zero, under every way to share a unit (4, 24,
    56 and 128 query rows), with a call's scale of either sign."""
    n = size + 60                                  # past what is planned in the kernel
    p = problem([size], [70], [70 * PAGE + 5 * i for i in range(size)] + [20] * 60, hq=4, hkv=1,
                kv="fp8_e4m3", seed=96, behind=60)
    p.k_scale[::3] *= -1.0
    p.k_scale[1::7] = 0.0
    p.v_scale[::5] *= -2.0
    for scale in (p.scale, -2.0 * p.scale):
        p.scale = scale
        check(p, "%d of %d, scale %g" % (size, n, scale))


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("size", [6, 14, 40])
def test_steep_scores_under_shared_units(size, kv):
    """One key takes nearly all the weight, and another one further on."""
    p = problem([size] + [1] * 60, [70] + [0] * 60,
                [70 * PAGE + 5 * i for i in range(size)] + [3] * 60, hq=4, hkv=1, kv=kv, seed=97)
    p.q.mul_(40.0)
    check(p, "steep, %d %s" % (size, kv))
