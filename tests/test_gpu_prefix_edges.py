"""Shared-prefix attention at the edges of what its header allows: numbers of kv heads that
are no power of two, prefixes outside the table, windows past 65536 tokens, finished
sequences whose queries hold anything, empty tables' worth of groups."""
import numpy as np
import pytest
import torch

from gpu_util import bf16_to_f64, check_close, device, oracle_ref
from prefix_paths import ways_of
from test_gpu_prefix import problem, run
from test_gpu_prefix_paths import BOTH, KINDS, PAGE, PLAN, allowance, bits, check, grouped, several

pytestmark = pytest.mark.gpu


@BOTH
@KINDS
@pytest.mark.parametrize("hq,hkv", [(12, 3), (40, 5), (7, 7), (48, 3), (22, 11)])
def test_any_number_of_kv_heads(hq, hkv, kv, planned):
    p = several([6, 2, 11], [49, 51, 53], (0, 9, 33, 120), planned, hq=hq, hkv=hkv, kv=kv, seed=130,
                layout="nhd" if hkv == 5 else "hnd")
    check(p, "%d/%d %s" % (hq, hkv, kv), {"small" if p.batch <= 64 else "planned"})


@BOTH
@KINDS
def test_prefixes_outside_the_table_are_clamped(kv, planned):
    """A negative prefix is none; one past the table's width has the members that fill it."""
    p = several([3, 4, 2], [60, 80, 60], (0, 40, 7), planned, kv=kv, seed=131)
    p.seq_lens[:3] = torch.tensor([20, 0, 300], dtype=torch.int32)
    table = p.block_table.clone()
    wild = table >= p.num_pages
    table[wild] = 0
    table[3:7] = table[3].clone()                  # group 1 shares its whole row
    p.block_table = table
    for pool in (p.k_pool, p.v_pool):              # page 0 and the row's end are read now
        if kv == "bf16":
            pool[pool.isnan()] = 0.25
        else:
            pool[pool == 0x7F] = 0x30
    if kv != "bf16":
        for s in (p.k_scale, p.v_scale):
            s[s.isnan()] = 0.01
    p.seq_lens[3:7] = torch.tensor([p.max_pages * PAGE] * 3 + [p.max_pages * PAGE - 1],
                                   dtype=torch.int32)
    # a limit as the rule sees it, for the allowance
    p.prefix_pages.copy_(torch.tensor([0, p.max_pages, 60], dtype=torch.int32))
    ref = oracle_ref(p)
    extra = allowance(p, ref)
    want = run(p)
    check_close(bf16_to_f64(want), ref, "clamped", extra_abs=extra)
    for low, high in ((-3, p.max_pages + 1), (-(1 << 31), (1 << 31) - 1)):
        p.prefix_pages.copy_(torch.tensor([low, high, 60], dtype=torch.int32))
        assert torch.equal(bits(run(p)), bits(want))


@KINDS
@pytest.mark.parametrize("size", [2, 12])
def test_windows_past_65536_tokens(kv, size):
    lens = (66000, 70001, 4400 * PAGE, 65537)
    p = problem([size], [4097], [lens[i % 4] for i in range(size)], hq=4, hkv=1, kv=kv, seed=132,
                poison=False)
    check(p, "long, %d" % size, {"small", "shared splits", "own"})
    p.prefix_pages[0] = 5
    check(p, "long own runs, %d" % size, {"small", "own splits"})


@BOTH
@KINDS
@pytest.mark.parametrize("size", [4, 8, 16, 30])
def test_queries_of_finished_sequences_hold_anything(size, kv, planned):
    """Their rows sit in units with those of members: NaN and infinities there stay there."""
    p = grouped(size, 57, (0, 30, 100), planned=planned, hq=8, hkv=2, kv=kv, seed=133)
    want = run(p)
    gone = [0, size - 1]
    p.seq_lens[gone] = 0
    p.q[0] = float("nan")
    p.q[size - 1] = float("inf")
    p.block_table[gone] = -5
    out = run(p)
    keep = [b for b in range(p.batch) if b not in gone]
    assert "shared%d" % next(c for c in (16, 32, 64, 128) if 4 * size <= c) in ways_of(p)
    assert torch.equal(bits(out[keep]), bits(want[keep]))
    assert not out[gone].any()


@KINDS
def test_tables_in_memory_with_shared_units(kv):
    """More sequences than the plan keeps in LDS, groups with and without members."""
    rng = np.random.default_rng(134)
    sizes = [int(x) for x in rng.integers(0, 5, 2100)]
    prefix = [int(x) for x in rng.integers(0, 4, 2100)]
    sizes[7], prefix[7], sizes[1500], prefix[1500] = 150, 3, 40, 2
    lens = np.repeat(prefix, sizes) * PAGE + rng.integers(0, 30, sum(sizes))
    lens[rng.random(lens.size) < 0.1] = 0
    p = problem(sizes, prefix, lens, hq=2, hkv=1, kv=kv, seed=134, poison=False)
    check(p, "%d sequences" % len(lens), {"planned", "memory", "shared16", "shared128", "tiles",
                                          "alone", "queued"})
    assert torch.equal(bits(run(p)), bits(run(p)))
