"""GPU decode attention over shared prefixes, path by path: sizes that reach each of the
ways a call can go, against the fp64 oracle's decode of the same cache."""
import numpy as np
import pytest
import torch

from gpu_util import PV_ROUND, bf16_to_f64, check_close, oracle_ref
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
