"""GPU decode attention over shared prefixes, path by path: sizes that reach each of the
ways a call can go, against the fp64 oracle's decode of the same cache."""
import numpy as np
import pytest
import torch

from gpu_util import P_ROUND, PV_ROUND, bf16_to_f64, check_close, device, oracle_ref
from paper_2512_22492_amd import binding as B
from prefix_paths import rule, ways_of
from test_gpu_prefix import problem, run

pytestmark = pytest.mark.gpu

PAGE = 16


def magnitudes(p):
    """The weighted mean of |v| (weights as they are)."""
    signed, p.v_scale = p.v_scale, None if p.v_scale is None else p.v_scale.abs()
    m1 = oracle_ref(p, abs_values=True)
    p.v_scale = signed
    return m1


def allowance(p, ref):
    """PV_ROUND M1 for weights in two bf16 terms, and the rows of tiles of more than 64
    query rows (in e4m3 pools 32) may hold those of their shared keys in one: at most
    P_ROUND (M1 + |o|) more, as worked out for extend."""
    m1 = magnitudes(p)
    start, pages = p.group_start.cpu().tolist(), p.prefix_pages.cpu().tolist()
    r = rule(p.max_pages, p.batch, len(pages), p.num_q_heads, p.num_kv_heads)
    G, lens = p.num_q_heads // p.num_kv_heads, p.seq_lens.cpu().tolist()
    coarse = np.zeros((p.batch, 1, 1))
    for g, n in enumerate(pages):
        if n <= r["unshared_pages"] or r["by_rows"]:
            continue
        rows = (start[g + 1] - start[g]) * G
        for b in range(start[g], start[g + 1]):
            tile = (b - start[g]) * G // 128
            many = min(128, rows - 128 * tile) > (64 if p.kv_dtype == "bf16" else 32)
            coarse[b] = many and lens[b] >= n * PAGE
    return PV_ROUND * m1 + coarse * P_ROUND * (m1 + np.abs(ref))


def check(p, what, expect, without=(), **kw):
    """Against the oracle, on a call that takes the expected ways."""
    print("case", what, flush=True)
    found = ways_of(p)
    assert found >= set(expect) and not found & set(without), found
    ref = oracle_ref(p)
    out = run(p, **kw)
    print(check_close(bf16_to_f64(out), ref, what, extra_abs=allowance(p, ref)))
    return out


def bits(t):
    return t.view(torch.int16)


def way(rows):
    """The way of a unit of so many query rows."""
    return "shared%d" % next(c for c in (16, 32, 64, 128) if rows <= c)


def check_two_terms(p, what, **kw):
    """Against the oracle, with the allowance of weights held in two bf16 terms."""
    print("case", what, flush=True)
    ref, m1 = oracle_ref(p), oracle_ref(p, abs_values=True)
    out = run(p, **kw)
    print(check_close(bf16_to_f64(out), ref, what, extra_abs=PV_ROUND * m1))
    return out


@pytest.mark.parametrize("kv,layout", [("bf16", "hnd"), ("bf16", "nhd"), ("fp8_e4m3", "hnd"),
                                       ("fp8_e4m3", "hnd_kv")])
def test_work_groups_that_take_short_runs_again_and_again(kv, layout):
    """Own runs of 1 to 16 pages, four to a work-group and turn, on twice the places
    that 512 work-groups take at once, and longer and empty ones between."""
    rng = np.random.default_rng(11)
    n = 560
    lens = rng.integers(1, 16 * PAGE + 1, n)
    lens[rng.random(n) < 0.03] = 0
    lens[::40] = rng.integers(17 * PAGE, 19 * PAGE, lens[::40].size)
    p = problem([], [], lens, before=n, hq=16, hkv=8, kv=kv, layout=layout, seed=100)
    assert (np.count_nonzero((lens > 0) & (lens <= 16 * PAGE)) * 8) // 4 > 2 * 512
    first = check_two_terms(p, "short runs %s %s" % (kv, layout))
    for _ in range(5):
        assert torch.equal(run(p).view(torch.int16), first.view(torch.int16))


def grouped(size, pages, own, *, planned=False, before=0, wide=True, **kw):
    """One group of `size` sequences that share `pages` pages and have own[i % len(own)]
    tokens of their own; `planned`: among more sequences than a small call has, of one to
    four tokens."""
    behind = max(0, 66 - size - before) if planned else 0
    lens = [3] * before + [pages * PAGE + own[i % len(own)] for i in range(size)] \
        + [1 + i % 4 for i in range(behind)]
    return problem([size], [pages], lens, before=before, behind=behind,
                   max_pages=max(pages + 8, 66) if wide else None, **kw)


@pytest.mark.parametrize("planned", [False, True], ids=["small", "planned"])
@pytest.mark.parametrize("size,hq,way", [(3, 8, "shared16"), (4, 8, "shared16"), (5, 8, "shared32"),
                                         (8, 8, "shared32"), (9, 8, "shared64"),
                                         (13, 8, "shared64"), (16, 8, "shared64"),
                                         (5, 16, "shared64"), (21, 4, "shared64")])
@pytest.mark.parametrize("pages", [49, 52, 70])
def test_bf16_groups_of_up_to_64_rows_hold_weights_in_two_terms(pages, size, hq, way, planned):
    """A weight held in one bf16 term is off by up to 2^-9 of itself, and a sum of some
    hundred of them by more than what is allowed here."""
    p = grouped(size, pages, (0, 5, 40, 90), planned=planned, hq=hq, hkv=2, seed=101)
    assert ways_of(p) >= {way, "planned" if planned else "small"}
    check_two_terms(p, "%d x %d heads, %d pages" % (size, hq, pages))


PLAN = {False: "small", True: "planned"}
BOTH = pytest.mark.parametrize("planned", [False, True], ids=["small", "planned"])
KINDS = pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])


def several(sizes, prefix, own, planned, **kw):
    """Groups with own[i] tokens each behind their prefixes, among single sequences where
    the call is to be planned by a launch of its own."""
    lens = [n * PAGE for n, size in zip(prefix, sizes) for _ in range(size)]
    lens = [a + own[i % len(own)] for i, a in enumerate(lens)]
    behind = max(0, 66 - len(lens)) if planned else 0
    return problem(sizes, prefix, lens + [1 + 5 * i % 60 for i in range(behind)], behind=behind,
                   max_pages=max(prefix) + 20, **kw)


@BOTH
@KINDS
@pytest.mark.parametrize("layout", ["hnd", "nhd", "hnd_kv"])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2), (4, 1), (16, 2), (16, 1)])
def test_head_layouts_of_shared_units(hq, hkv, layout, kv, planned):
    """1, 2, 4, 8 and 16 query heads per kv head; page counts around a stage of four."""
    p = several([5, 1, 9, 4], [49, 51, 70, 52], (0, 1, 15, 16, 17, 300, 40), planned, hq=hq,
                hkv=hkv, kv=kv, layout=layout, seed=110)
    p.seq_lens[3] = 49 * PAGE - 1                  # one token short of its prefix
    p.seq_lens[8] = 0
    G = hq // hkv
    expect = {way(n * G) for n in (5, 1, 4)} | {way(9 * G) if 9 * G <= 128 else "tiles"}
    check(p, "heads %d/%d %s %s" % (hq, hkv, kv, layout),
          {PLAN[planned], "alone", "own"} | expect)


@BOTH
@KINDS
@pytest.mark.parametrize("layout", ["hnd", "nhd", "hnd_kv"])
@pytest.mark.parametrize("size,hq,hkv", [(10, 8, 2), (16, 8, 2), (17, 8, 2), (33, 8, 2),
                                         (20, 4, 2), (33, 2, 1), (65, 2, 1), (5, 16, 2),
                                         (9, 16, 2), (17, 16, 2), (3, 16, 1), (8, 16, 1)])
def test_units_that_a_work_group_walks_together(size, hq, hkv, layout, kv, planned):
    """40 to 136 query rows a group, as one unit and as two tiles, whose last stage holds
    one to four pages."""
    pages = 49 + (size + len(layout)) % 4
    p = grouped(size, pages, (0, 3, 16, 70, 33), planned=planned, hq=hq, hkv=hkv, kv=kv,
                layout=layout, seed=111)
    rows = size * hq // hkv
    check(p, "%d rows, %d pages" % (rows, pages),
          {PLAN[p.batch > 64], "shared64" if rows <= 64 else "shared128",
           "tiles" if rows > 128 else "shared once"})


@BOTH
@KINDS
def test_groups_of_all_kinds(kv, planned):
    """Groups without members, without sequences, without a prefix, sequences outside any
    group on both sides, finished ones and ones shorter than their prefix."""
    rng = np.random.default_rng(3)
    sizes = [3, 0, 8, 1, 0, 5, 2, 7, 4, 20]
    prefix = [0, 60, 49, 55, 0, 70, 12, 66, 130, 64]
    lengths = []
    for n, pages in zip(sizes, prefix):
        lengths += list(pages * PAGE + rng.integers(0, 200, n))
    behind = 20 if planned else 3
    lengths = np.array([17, 300] + lengths + [1 + 37 * i for i in range(behind)])
    lengths[rng.random(lengths.size) < 0.15] = 0
    at = 2 + sum(sizes[:5])
    lengths[at:at + 5] = [3, 0, 15, 70 * PAGE - 1, 1]        # nobody fills group 5's pages
    p = problem(sizes, prefix, lengths, hq=16, hkv=4, kv=kv, seed=112, before=2, behind=behind,
                max_pages=150)
    check(p, "kinds of groups " + kv, {PLAN[planned], "unshared", "shared32", "shared128", "own"})


@KINDS
@pytest.mark.parametrize("batch", [1, 2, 63, 64, 65])
def test_small_calls_with_shared_units_and_the_next_larger(batch, kv):
    rng = np.random.default_rng(batch)
    sizes, left = [], batch - min(batch - 1, 3)
    while left:
        sizes.append(int(rng.integers(0, min(left, 9) + 1)))
        left -= sizes[-1]
    prefix = [int(x) for x in rng.integers(30, 120, len(sizes))]
    prefix[int(np.argmax(sizes))] = 77
    lens = np.repeat(prefix, sizes) * PAGE + rng.integers(0, 700, sum(sizes))
    behind = batch - sum(sizes)
    lens = np.concatenate([lens, rng.integers(0, 300, behind)])
    lens[rng.random(batch) < 0.1] = 0
    lens[int(np.sum(sizes[:int(np.argmax(sizes))]))] = 77 * PAGE + 5
    p = problem(sizes, prefix, lens, hq=8, hkv=2, kv=kv, seed=113, behind=behind, max_pages=170)
    found = ways_of(p)
    assert any(w.startswith("shared") for w in found)
    check(p, "batch %d %s" % (batch, kv), {PLAN[batch > 64]})


def test_many_groups_most_without_sequences():
    """64 and 65 groups over a batch of 40: planned in the kernel and by a launch."""
    for groups in (64, 65):
        sizes = [1 if g % 3 == 1 else (2 if g % 7 == 0 else 0) for g in range(groups)]
        sizes[-1] += 40 - sum(sizes)
        prefix = [45 + (5 * g) % 11 for g in range(groups)]
        lens = np.repeat(prefix, sizes) * PAGE + np.arange(40) * 3
        p = problem(sizes, prefix, lens, hq=4, hkv=1, seed=114, max_pages=80)
        check(p, "%d groups" % groups, {PLAN[groups > 64], "shared16", "unshared"})


@BOTH
@KINDS
@pytest.mark.parametrize("size", [1, 6, 14, 32])
def test_call_scales_of_either_sign_and_zero(size, kv, planned):
    """Under units of 4, 24, 56 and 128 query rows, whose last stage is one page (its
    masked blocks meet a multiplier of zero)."""
    p = grouped(size, 53, (0, 20, 90), planned=planned, hq=4, hkv=1, kv=kv, seed=115)
    for scale in (0.0, -0.125, 2.0):
        p.scale = scale
        check(p, "%d sequences, scale %g" % (size, scale),
              {PLAN[planned], way(4 * size)})


@BOTH
@KINDS
@pytest.mark.parametrize("size", [3, 8, 14, 30])
def test_steep_scores_and_infinities_in_masked_places(size, kv, planned):
    """One key takes nearly all the weight; slots past the lengths and pages that no
    table names hold infinities."""
    p = grouped(size, 57, (0, 9, 25, 160), planned=planned, hq=8, hkv=2, kv=kv, seed=116)
    p.q.mul_(60.0)
    if kv == "bf16":
        for pool in (p.k_pool, p.v_pool):           # what was NaN
            pool[pool.isnan()] = float("inf")
    check(p, "steep, %d %s" % (size, kv), {PLAN[planned], "alone"})


def queued(kv="bf16", layout="hnd", seed=117, grow=0):
    """A call of more places than 512 work-groups take at once: shared units of every kind,
    own runs of a work-group and of a wavefront."""
    sizes, prefix = [3, 8, 14, 30, 1, 40], [60, 70, 49, 64, 66, 53]
    rng = np.random.default_rng(seed)
    lens = np.repeat(prefix, sizes) * PAGE + rng.integers(0, 300, sum(sizes))
    lens[4], lens[5], lens[20] = 71 * PAGE, 0, 49 * PAGE - 3
    p = problem(sizes, prefix, lens, hq=32, hkv=8, kv=kv, layout=layout, seed=seed,
                max_pages=70 + 20 + grow)
    assert ways_of(p) >= {"planned", "queued", "shared16", "shared32", "shared64", "shared128",
                          "tiles", "own", "alone", "merge"}
    return p


@KINDS
def test_results_repeat_and_other_sequences_do_not_matter(kv):
    p = queued(kv)
    ref = oracle_ref(p)
    first = run(p)
    check_close(bf16_to_f64(first), ref, "queued", extra_abs=allowance(p, ref))
    for _ in range(10):
        assert torch.equal(bits(run(p)), bits(first))
    own = p.block_table[4, 70:71].long()           # sequence 4's own page
    p.v_pool[own] = 0x38 if kv != "bf16" else 1.0
    changed = run(p)
    keep = [i for i in range(p.batch) if i != 4]
    assert torch.equal(bits(changed[keep]), bits(first[keep]))
    assert not torch.equal(changed[4], first[4])


@KINDS
@pytest.mark.parametrize("shape", ["small", "queued"])
def test_workspaces_of_any_contents_on_another_stream(shape, kv):
    if shape == "queued":
        p = queued(kv)
    else:
        p = several([9, 4, 20], [60, 49, 53], (31, 0, 90, 400), False, hq=8, hkv=2, kv=kv, seed=118)
        assert ways_of(p) >= {"small", "shared16", "shared64", "shared128"}
    want = run(p)
    rc, n = B.rl_prefix_attn_workspace_size(p.max_pages, p.batch, p.prefix_pages.numel(),
                                            p.num_q_heads, p.num_kv_heads)
    assert rc == B.RL_DA_OK
    s = torch.cuda.Stream()
    for fill in (0x00, 0xFF, 0x7F):
        guard = torch.full((n + 64,), fill, dtype=torch.uint8, device=device())
        out = torch.full_like(p.q, float("nan"))
        s.wait_stream(torch.cuda.current_stream())
        B.prefix_attention(p, p.group_start, p.prefix_pages, out, stream=s, workspace=guard[:n])
        s.synchronize()
        assert torch.equal(bits(out), bits(want))
        assert (guard[n:] == fill).all() and not (guard[:n] == fill).all()
    out = torch.full_like(p.q, float("nan"))
    B.PrefixAttention(p, p.group_start, p.prefix_pages)(p.q, out, s)
    s.synchronize()
    assert torch.equal(bits(out), bits(want))


@BOTH
@KINDS
@pytest.mark.parametrize("size", [3, 8, 14, 30])
def test_bad_shared_and_own_pages_and_lengths_are_reported(size, kv, planned):
    """An entry out of the pool among a group's shared pages, a sequence's own ones of
    either kind of run, and a length past the table; the others' outputs stay."""
    p = several([size, 2], [50, 60], (70, 200, 30), planned, hq=8, hkv=2, kv=kv, seed=119)
    assert ways_of(p) >= {PLAN[planned], way(4 * size), "alone", "own"}
    err = torch.zeros(1, dtype=torch.int32, device=device())
    want, good = run(p, device_error=err), p.block_table.clone()
    assert int(err) == 0
    every = set(range(p.batch))

    def broken(rows, column, page, lost):
        p.block_table = good.clone()
        p.block_table[rows, column] = page
        err.zero_()
        out = run(p, device_error=err)
        assert int(err) == B.RL_DA_DEVERR_PAGE_OUT_OF_RANGE
        keep = sorted(every - set(lost))
        assert torch.equal(bits(out[keep]), bits(want[keep]))

    broken(slice(0, size), 17, p.num_pages, range(size))      # shared
    broken(slice(0, size), 49, -1, range(size))
    broken(1, 51, -7, [1])                                    # own, four wavefronts'
    broken(2, 51, 1 << 30, [2])                               # own, one wavefront's
    p.block_table = good.clone()
    p.block_table[1] = good[1, 0]
    p.block_table[0:size, :50] = good[0, :50]
    p.seq_lens[1] = p.max_pages * PAGE
    err.zero_()
    full = run(p, device_error=err)
    assert int(err) == 0
    p.seq_lens[1] += 1
    out = run(p, device_error=err)
    assert int(err) == B.RL_DA_DEVERR_LENGTH_TOO_LONG
    assert torch.equal(bits(out), bits(full))


@BOTH
def test_group_tables_that_run_backwards_write_only_their_outputs(planned):
    """group_start is a precondition; a call that breaks it stays inside its buffers."""
    n = 90 if planned else 60
    p = problem([n // 3] * 3, [50, 50, 50], [50 * PAGE + 100] * n, hq=16, hkv=1, seed=120,
                max_pages=70)
    assert ways_of(p) >= {PLAN[planned], "shared128", "tiles"}
    rc, size = B.rl_prefix_attn_workspace_size(p.max_pages, p.batch, 3, 16, 1)
    guard = torch.full((size + 256,), 0x5A, dtype=torch.uint8, device=device())
    out = torch.full((n + 1, 16, 128), 7.0, dtype=torch.bfloat16, device=device())
    for starts in ([0, n, 0, n], [n // 2, n, -5, 1000], [n, 0, n, 0], [n, n, n, 0]):
        p.group_start.copy_(torch.tensor(starts, dtype=torch.int32))
        B.prefix_attention(p, p.group_start, p.prefix_pages, out[:n], workspace=guard[:size])
        torch.cuda.synchronize()
        assert (guard[size:] == 0x5A).all() and (out[n] == 7.0).all()


@KINDS
@pytest.mark.parametrize("shape", ["small", "queued"])
def test_replays_of_planned_calls_equal_the_eager_run(shape, kv):
    """Captured once and replayed as the sequences grow, with eager calls on another
    workspace between the replays: each replay plans anew and its counters start anew."""
    if shape == "queued":
        p = queued(kv, grow=10)
    else:
        p = several([9, 4, 20], [60, 49, 53], (31, 0, 90, 200), False, hq=8, hkv=2, kv=kv, seed=121)
        assert ways_of(p) >= {"small", "shared16", "shared64", "shared128"}
    table = p.block_table.clone()                  # room to grow into
    wild = (table < 0) | (table >= p.num_pages)
    table[wild] = (torch.arange(int(wild.sum()), device=device(), dtype=torch.int32) * 7
                   % p.num_pages)
    p.block_table = table
    if kv == "bf16":
        for pool in (p.k_pool, p.v_pool):
            pool[pool.isnan()] = 0.5
    else:
        for pool in (p.k_pool, p.v_pool):
            pool[pool == 0x7F] = 0x30
        for scale in (p.k_scale, p.v_scale):
            scale[scale.isnan()] = 0.01
    attn = B.PrefixAttention(p, p.group_start, p.prefix_pages)
    out = torch.full_like(p.q, float("nan"))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attn(p.q, out, torch.cuda.current_stream())
    for step in range(5):
        eager = run(p)
        for again in range(2):
            out.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(bits(out), bits(eager)), (step, again)
        ref = oracle_ref(p)
        check_close(bf16_to_f64(out), ref, "step %d" % step, extra_abs=allowance(p, ref))
        p.seq_lens += 13
    del g


def test_two_planned_calls_at_once_on_two_streams():
    """Two caches with their own objects and streams, enqueued without waiting."""
    runs = []
    for seed in (122, 123):
        p = queued(seed=seed)
        runs.append((p, B.PrefixAttention(p, p.group_start, p.prefix_pages), torch.cuda.Stream(),
                     torch.full_like(p.q, float("nan"))))
    alone = [run(p) for p, _, _, _ in runs]
    torch.cuda.synchronize()
    for _ in range(20):
        for p, attend, s, out in runs:
            attend(p.q, out, s)
    torch.cuda.synchronize()
    for (p, attend, s, out), want in zip(runs, alone):
        assert torch.equal(bits(out), bits(want))
