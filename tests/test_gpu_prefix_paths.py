"""GPU decode attention over shared prefixes, path by path: sizes that reach each of the
ways a call can go, against the fp64 oracle's decode of the same cache."""
import numpy as np
import pytest
import torch

from gpu_util import PV_ROUND, bf16_to_f64, check_close, oracle_ref
from prefix_paths import ways_of
from test_gpu_prefix import problem, run

pytestmark = pytest.mark.gpu

PAGE = 16


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
