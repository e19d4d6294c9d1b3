"""Rotate-and-append of calls with more pages than one turn of their work-groups: bit for
bit what the same tokens give in smaller calls, and the queries against an fp64 rotation."""
import numpy as np
import pytest
import torch

from paper_2512_22492_amd import binding as B

from gpu_util import device
from test_gpu_rope import ARITH, D, f64, norms, problem, rotated, snapshot, table, tokens

pytestmark = pytest.mark.gpu

PAGE = 16


@pytest.mark.parametrize("interleaved,rotary", [(False, 128), (True, 64)])
@pytest.mark.parametrize("hq,hkv", [(32, 8), (64, 4), (7, 3)])
@pytest.mark.parametrize("kv,layout", [("bf16", "hnd"), ("bf16", "nhd"), ("fp8_e4m3", "hnd"),
                                       ("fp8_e4m3", "nhd"), ("fp8_e4m3", "hnd_kv")])
def test_prompts_have_the_bits_of_smaller_calls(kv, layout, hq, hkv, interleaved, rotary):
    """Sequences of 300 to 400 tokens: past 1024 pages a work-group walks a page's head
    rows in several turns (for 48 and 72 of them), and in smaller calls in one."""
    print("case", kv, layout, hq, hkv, interleaved, flush=True)
    n = 56
    rng = np.random.default_rng(40)
    new, prior = [int(x) for x in rng.integers(300, 400, n)], [int(x) for x in rng.integers(0, 40, n)]
    new[3], new[9] = 0, 1
    tiles = (max(new) + 14) // PAGE + 1
    heads = hq + 2 * hkv
    assert n * tiles >= 1024 and (heads < 24 or -(-heads // 6) > 4)
    p = problem(new, prior, hq=hq, hkv=hkv, kv=kv, layout=layout, seed=41)
    other = p.clone_pools()
    q, k, v = tokens(p, new, 42, fused=True)
    cs, w = table(512, rotary), norms(43)
    start = np.concatenate([[0], np.cumsum(new)])
    q_out, q_other = (torch.full((sum(new), hq, D), 3.0, dtype=torch.bfloat16, device=device())
                      for _ in range(2))
    kw = dict(q_norm=w[0], k_norm=w[1], interleaved=interleaved)
    B.rope_append(p, q, k, v, cs, q_out, torch.tensor(start, dtype=torch.int32, device=device()),
                  max(new), **kw)
    whole = other.block_table, other.seq_lens
    for b0 in range(0, n, 8):                      # 8 sequences of 25 pages a call
        rows = slice(int(start[b0]), int(start[b0 + 8]))
        other.block_table = whole[0][b0:b0 + 8].contiguous()
        other.seq_lens = p.seq_lens[b0:b0 + 8].contiguous()
        other.batch = 8
        part = torch.tensor(start[b0:b0 + 9] - start[b0], dtype=torch.int32, device=device())
        B.rope_append(other, q[rows], k[rows], v[rows], cs, q_other[rows], part,
                      max(new[b0:b0 + 8]), **kw)
    torch.cuda.synchronize()
    assert torch.equal(q_out.view(torch.int16), q_other.view(torch.int16))
    for a, b in zip(snapshot(p), snapshot(other)):
        assert a is None or torch.equal(a.contiguous().view(torch.uint8),
                                        b.contiguous().view(torch.uint8))
    pos = np.concatenate([np.arange(x) + y for x, y in zip(new, prior)])
    some = np.arange(0, len(pos), 13)
    want, size = rotated(q[some], pos[some], cs, rotary, interleaved, w[0])
    err = np.abs(f64(q_out[some]) - want)
    assert np.all(err <= 2.0 ** -8 * (np.abs(want) + ARITH * size) + ARITH * size + 1e-38)
