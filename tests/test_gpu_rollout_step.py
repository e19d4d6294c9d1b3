"""The operators of a rollout together: prompts and replies of several tokens and
single tokens go into one paged cache through the rotating append, and every step
attends, extends or decodes with the prompt's pages shared.  Everything is checked
against the fp64 oracle's attention over the cache as the appends left it, and the
cache against a plain fp64 rotation (bf16) or rl_kv_append's own rule (e4m3 values)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2512_22492_amd import binding as B
from paper_2512_22492_amd import workloads

from gpu_util import (KV, P_ROUND, PV_ROUND, bf16_to_f64, check_close, device, extend_extra,
                      oracle_ref)

pytestmark = pytest.mark.gpu

PAGE, D = 16, 128


def rotation(rows):
    a = np.arange(rows)[:, None] * 1e4 ** (-np.arange(0, D, 2) / D)
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1)).float().to(device())


def rotate64(x, pos, cs):
    x, cs = x.double().cpu(), cs.double().cpu()[pos][:, None]
    c, s, a, b = cs[..., :64], cs[..., 64:], x[..., :64], x[..., 64:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


class Rollout:
    """`prompts` prompts with `size` responses each over one cache: the whole pages of a
    prompt are shared, its last tokens are in a page of each response's own."""

    def __init__(self, kv, layout, lengths, size, hq=8, hkv=2, room=60, seed=5):
        self.lengths, self.size = lengths, size
        n = len(lengths) * size
        width = max(-(-(L + room) // PAGE) for L in lengths)
        p = workloads.make_problem("rollout", batch=n, num_q_heads=hq, num_kv_heads=hkv,
                                   lengths=[width * PAGE] * n, kv_dtype=kv, layout=layout,
                                   seed=seed, max_pages=width + 3).to(device())
        table = p.block_table.clone()
        for i, L in enumerate(lengths):
            table[i * size:(i + 1) * size, :L // PAGE] = table[i * size, :L // PAGE].clone()
        p.block_table = table
        self.p, self.cs = p, rotation(width * PAGE + 1)
        self.start = torch.arange(0, n + 1, size, dtype=torch.int32, device=device())
        self.pages = torch.tensor([L // PAGE for L in lengths], dtype=torch.int32,
                                  device=device())
        self.gen = torch.Generator().manual_seed(seed)

    def tokens(self, n):
        hq, hkv = self.p.num_q_heads, self.p.num_kv_heads
        x = torch.randn((n, hq + 2 * hkv, D), generator=self.gen).to(torch.bfloat16).to(device())
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]

    def view(self, rows, lens):
        """The cache with the table rows `rows` as its sequences, of lengths lens."""
        p = self.p
        q = workloads.DecodeProblem(**{**p.__dict__, "batch": len(rows),
                                       "block_table": p.block_table[rows].contiguous(),
                                       "seq_lens": torch.tensor(lens, dtype=torch.int32,
                                                                device=device())})
        return q

    def append_many(self, rows, before, new):
        """new[i] tokens to table row rows[i]; returns (problem after, q, q_start)."""
        q, k, v = self.tokens(sum(new))
        start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32,
                             device=device())
        out = torch.empty_like(q).contiguous()
        B.rope_append(self.view(rows, before), q, k, v, self.cs, out, start, max(new))
        after = self.view(rows, [a + b for a, b in zip(before, new)])
        return after, out, start, (q, k, v)


def check_extend(p, q, start, new):
    out = torch.full_like(q, float("nan"))
    B.extend_attention(p, q, start, max(new), out)
    torch.cuda.synchronize()
    h = p.host_arrays()
    h["q_bits"] = q.cpu().view(torch.int16).numpy().view(np.uint16)
    args = dict(kv_dtype=KV[p.kv_dtype], q_start=start.cpu().numpy())
    ref = oracle.extend_attention(**h, **args)
    h["v_pool"] = h["v_pool"] & (np.uint16(0x7FFF) if p.kv_dtype == "bf16" else np.uint8(0x7F))
    m1 = oracle.extend_attention(**h, **args)
    check_close(bf16_to_f64(out), ref, "extend", extra_abs=extend_extra(p.kv_dtype, ref, m1))


@pytest.mark.parametrize("kv,layout", [("bf16", "hnd"), ("bf16", "nhd"), ("fp8_e4m3", "hnd"),
                                       ("fp8_e4m3", "hnd_kv")])
@pytest.mark.parametrize("lengths,size", [([100, 37, 16], 4), ([200 + 13 * i for i in range(10)], 8)],
                         ids=["small", "planned"])
def test_prompts_steps_and_a_reply(kv, layout, lengths, size):
    r = Rollout(kv, layout, lengths, size)
    p, n = r.p, len(lengths) * size
    # the prompts, once each, through the first response's table row
    leaders = list(range(0, n, size))
    after, q, start, (q0, k0, _) = r.append_many(leaders, [0] * len(leaders), lengths)
    pos = np.concatenate([np.arange(L) for L in lengths])
    want = rotate64(q0, pos, r.cs)
    # one rounding to bf16 (2^-8) of an fp32 rotation of unit-sized values
    assert (q.double().cpu() - want).abs().max() <= 2.0 ** -8 * want.abs().max() + 1e-5
    check_extend(after, q, start, lengths)
    # the other responses' copies of each prompt's last, partly filled page
    for i, L in enumerate(lengths):
        if L % PAGE:
            src = p.block_table[i * size, L // PAGE].long()
            for b in range(i * size + 1, (i + 1) * size):
                dst = p.block_table[b, L // PAGE].long()
                for t in (p.k_pool, p.v_pool, p.k_scale, p.v_scale):
                    if t is not None:
                        t[dst] = t[src]
    lens = np.repeat(lengths, size)
    p.seq_lens = torch.tensor(lens, dtype=torch.int32, device=device())
    # decode steps: append at the length, attend over one more
    append = B.RopeAppender(p, r.cs)
    now = workloads.DecodeProblem(**{**p.__dict__, "seq_lens": p.seq_lens + 1})
    attend = B.PrefixAttention(now, r.start, r.pages)
    out, rot = torch.empty_like(p.q), torch.empty_like(p.q)
    for step in range(4):
        q, k, v = r.tokens(n)
        append(q, k, v, rot)
        attend(rot, out)
        torch.cuda.synchronize()
        now.q = rot
        ref = oracle_ref(now)
        m1 = oracle_ref(now, abs_values=True)
        check_close(bf16_to_f64(out), ref, "step %d" % step,
                    extra_abs=P_ROUND * (m1 + np.abs(ref)) + PV_ROUND * m1)
        with B.DecodeAttention.for_problem(now) as plain:   # the unshared step agrees
            other = torch.empty_like(out)
            plain.run(rot, now.k_pool, now.v_pool, now.k_scale, now.v_scale, now.block_table,
                      now.seq_lens, now.scale, other)
            torch.cuda.synchronize()
        check_close(bf16_to_f64(other), ref, "unshared", extra_abs=PV_ROUND * m1)
        p.seq_lens += 1
        now.seq_lens += 1
    # a tool reply of several tokens to some of the responses
    rows = [0, size + 1, n - 1]
    before = [int(lens[b]) + 4 for b in rows]
    new = [17, 1, 30]
    after, q, start, _ = r.append_many(rows, before, new)
    check_extend(after, q, start, new)


def test_two_steps_at_once_on_two_streams():
    """Two caches, each with its own objects and stream, enqueued without waiting."""
    runs = []
    for seed in (1, 2):
        r = Rollout("bf16", "hnd", [300 + 40 * i for i in range(9)], 8, seed=seed)
        lens = np.repeat(r.lengths, 8) + 5
        r.p.seq_lens = torch.tensor(lens, dtype=torch.int32, device=device())
        runs.append((r, B.PrefixAttention(r.p, r.start, r.pages), torch.cuda.Stream(),
                     torch.empty_like(r.p.q)))
    alone = []
    for r, attend, s, out in runs:
        attend(r.p.q, out)
        torch.cuda.synchronize()
        alone.append(out.clone())
        out.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for r, attend, s, out in runs:
            attend(r.p.q, out, s)
    torch.cuda.synchronize()
    for (r, attend, s, out), want in zip(runs, alone):
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))


def test_a_step_captured_whole():
    """Append and attention of a planned call (72 sequences) in one graph, replayed with
    eager steps of another cache between, against eager steps on a copy."""
    lengths = [180 + 11 * i for i in range(9)]
    made = [Rollout("fp8_e4m3", "hnd", lengths, 8, seed=3) for _ in range(2)]
    other = Rollout("fp8_e4m3", "hnd", lengths, 8, seed=4)
    steps = []
    for r in made + [other]:
        lens = np.repeat(lengths, 8) + np.arange(72) % 7
        r.p.seq_lens = torch.tensor(lens, dtype=torch.int32, device=device())
        now = workloads.DecodeProblem(**{**r.p.__dict__, "seq_lens": r.p.seq_lens + 1})
        steps.append((r, now, B.RopeAppender(r.p, r.cs), B.PrefixAttention(now, r.start, r.pages),
                      torch.empty_like(r.p.q), torch.empty_like(r.p.q)))
    q, k, v = made[0].tokens(72)

    def run(step, stream):
        r, now, append, attend, rot, out = step
        append(q, k, v, rot, stream=stream)
        attend(rot, out, stream)
        r.p.seq_lens += 1
        now.seq_lens += 1

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(steps[0], torch.cuda.current_stream())
    for i in range(5):
        for t, x in zip((q, k, v), made[0].tokens(72)):
            t.copy_(x)
        g.replay()
        run(steps[1], None)
        run(steps[2], None)
        torch.cuda.synchronize()
        assert torch.equal(steps[0][5].view(torch.int16), steps[1][5].view(torch.int16)), i
        assert torch.equal(steps[0][0].p.k_pool, steps[1][0].p.k_pool), i
    del g
