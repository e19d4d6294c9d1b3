"""That the allowance for weights in two bf16 terms tells them from weights in one: the
softmax of a decode step in fp64 with its weights rounded either way (CPU)."""
import numpy as np
import pytest

from paper_2512_22492_amd import workloads

from gpu_util import PV_ROUND, check_close, oracle_ref, rne_bf16


@pytest.mark.parametrize("seed", [1, 2, 3])
@pytest.mark.parametrize("keys", [17, 100, 800])
def test_one_term_is_past_the_allowance_of_two(keys, seed):
    p = workloads.make_problem("terms", batch=2, num_q_heads=8, num_kv_heads=2,
                               lengths=[keys, keys], kv_dtype="bf16", seed=seed)
    ref, m1 = oracle_ref(p), oracle_ref(p, abs_values=True)
    out = {1: np.zeros_like(ref), 2: np.zeros_like(ref)}
    for b in range(2):
        pages = p.block_table[b].long()
        k, v = (x[pages].transpose(1, 2).reshape(-1, 2, 128)[:keys].double().numpy()
                for x in (p.k_pool, p.v_pool))
        for h in range(8):
            s = k[:, h // 4] @ p.q[b, h].double().numpy() * p.scale
            w = np.exp(s - s.max())
            hi = rne_bf16(w)
            lo = rne_bf16(w - hi)
            out[1][b, h] = rne_bf16(hi @ v[:, h // 4] / hi.sum())
            out[2][b, h] = rne_bf16((hi + lo) @ v[:, h // 4] / w.sum())
    check_close(out[2], ref, "two terms", extra_abs=PV_ROUND * m1)
    with pytest.raises(AssertionError, match="exceeds one bf16 ulp"):
        check_close(out[1], ref, "one term", extra_abs=PV_ROUND * m1)
