"""Rotate-and-append into e4m3 pages beside rl_kv_append, byte for byte: values, and key
dims that no rotation reaches, of every kind that bf16 holds."""
import numpy as np
import pytest
import torch

from paper_2512_22492_amd import binding as B

from gpu_util import device
from test_gpu_rope import problem, snapshot, tokens

pytestmark = pytest.mark.gpu

PRIOR = [0, 3, 15, 16, 40]
ROTARY = 16


def special(kind, x, gen):
    """x with a third of its elements replaced."""
    pick = {"zeros": [0.0, -0.0, 1e-40, -1e-40, 9e-41, -9.3e-39, 1e-30, -1e-30],
            "nan": [float("nan"), -0.0, 1.0, -1.0],
            "inf": [float("inf"), float("-inf"), -0.0, 1.0],
            "large": [3.3e38, -3.3e38, 1e20, -1e20, -0.0, 1e-20]}[kind]
    table = torch.tensor(pick, dtype=torch.float64).to(torch.bfloat16)
    if kind == "nan":   # of either sign
        table = torch.cat([table, torch.tensor([0x7FC0, 0xFFC0 - 0x10000], dtype=torch.int16)
                           .view(torch.bfloat16)])
    at = torch.randint(0, len(table), x.shape, generator=gen)
    use = torch.rand(x.shape, generator=gen) < 0.33
    return torch.where(use.to(x.device), table[at].to(x.device), x)


@pytest.mark.parametrize("form", ["token", "few", "pages"])
@pytest.mark.parametrize("kind", ["zeros", "nan", "inf", "large"])
def test_special_values_have_the_appends_bytes(kind, form):
    print("case", kind, form, flush=True)
    new = [1] * 5
    p = problem([6] * 5, PRIOR, kv="fp8_e4m3", seed=31)
    other = p.clone_pools()
    cs = torch.cat([torch.ones(80, ROTARY // 2), torch.zeros(80, ROTARY // 2)], 1).to(device())
    start = torch.arange(6, dtype=torch.int32, device=device())
    gen = torch.Generator().manual_seed(32)
    seen = False
    for step in range(6):
        q, k, v = tokens(p, new, 70 + step)
        k[..., ROTARY:] = special(kind, k[..., ROTARY:], gen)
        v = special(kind, v, gen)
        q_out = torch.empty_like(q)
        if form == "token":
            B.rope_append(p, q, k, v, cs, q_out)
        else:
            B.rope_append(p, q, k, v, cs, q_out, start, 8 if form == "few" else 20)
        B.kv_append(other, k, v)
        p.seq_lens += 1
        other.seq_lens = p.seq_lens
        torch.cuda.synchronize()
        for name, a, b in zip(("k", "v", "k scale", "v scale"), snapshot(p), snapshot(other)):
            a, b = (t.contiguous().view(torch.uint8).cpu().numpy() for t in (a, b))
            differ = np.argwhere(a != b)
            assert len(differ) == 0, (step, name, len(differ),
                                      [(int(a[tuple(i)]), int(b[tuple(i)])) for i in differ[:6]])
        seen |= bool((p.v_pool == 0x80).any())
    assert seen or kind == "nan"   # negative zeros among the codes
