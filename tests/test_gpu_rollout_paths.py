"""A rollout's steps whose attention takes shared units: prompts, appends, extend, shared
and unshared decode over one cache, two streams, and a step captured whole."""
import numpy as np
import pytest
import torch

from paper_2512_22492_amd import binding as B
from paper_2512_22492_amd import workloads

from gpu_util import PV_ROUND, bf16_to_f64, check_close, device, oracle_ref
from prefix_paths import ways_of
from test_gpu_prefix_paths import allowance, bits
from test_gpu_rollout_step import Rollout, check_extend

pytestmark = pytest.mark.gpu

PAGE = 16


def step_of(r):
    """The cache after an append of one token, with the groups."""
    now = workloads.DecodeProblem(**{**r.p.__dict__, "seq_lens": r.p.seq_lens + 1})
    now.group_start, now.prefix_pages = r.start, r.pages
    return now


@pytest.mark.parametrize("kv,layout", [("bf16", "hnd"), ("bf16", "nhd"), ("fp8_e4m3", "nhd"),
                                       ("fp8_e4m3", "hnd_kv")])
@pytest.mark.parametrize("lengths,size,ways", [
    ([1100, 837, 1003], 4, {"small", "shared16"}),
    ([1000 + 13 * i for i in range(5)], 14, {"planned", "shared64"}),
    ([1040, 990], 40, {"planned", "shared128", "tiles"})], ids=["small", "planned", "large"])
def test_prompts_steps_and_a_reply(kv, layout, lengths, size, ways):
    r = Rollout(kv, layout, lengths, size, room=150)
    p, n = r.p, len(lengths) * size
    leaders = list(range(0, n, size))
    after, q, start, _ = r.append_many(leaders, [0] * len(leaders), lengths)
    check_extend(after, q, start, lengths)
    for i, L in enumerate(lengths):    # each prompt's last, partly filled page
        if L % PAGE:
            src = p.block_table[i * size, L // PAGE].long()
            for b in range(i * size + 1, (i + 1) * size):
                dst = p.block_table[b, L // PAGE].long()
                for t in (p.k_pool, p.v_pool, p.k_scale, p.v_scale):
                    if t is not None:
                        t[dst] = t[src]
    lens = np.repeat(lengths, size)
    p.seq_lens = torch.tensor(lens, dtype=torch.int32, device=device())
    append = B.RopeAppender(p, r.cs)
    now = step_of(r)
    assert ways_of(now) >= ways
    attend = B.PrefixAttention(now, r.start, r.pages)
    out, rot = torch.empty_like(p.q), torch.empty_like(p.q)
    for step in range(3):
        q, k, v = r.tokens(n)
        append(q, k, v, rot)
        attend(rot, out)
        torch.cuda.synchronize()
        now.q = rot
        ref = oracle_ref(now)
        check_close(bf16_to_f64(out), ref, "step %d" % step, extra_abs=allowance(now, ref))
        with B.DecodeAttention.for_problem(now) as plain:   # the unshared step agrees
            other = torch.empty_like(out)
            plain.run(rot, now.k_pool, now.v_pool, now.k_scale, now.v_scale, now.block_table,
                      now.seq_lens, now.scale, other)
            torch.cuda.synchronize()
        check_close(bf16_to_f64(other), ref, "unshared",
                    extra_abs=PV_ROUND * oracle_ref(now, abs_values=True))
        p.seq_lens += 1
        now.seq_lens += 1
    rows = [0, size + 1, n - 1]        # a tool's reply to some of the responses
    before, new = [int(lens[b]) + 3 for b in rows], [17, 1, 30]
    after, q, start, _ = r.append_many(rows, before, new)
    check_extend(after, q, start, new)


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_two_steps_at_once_on_two_streams(kv):
    runs = []
    for seed in (1, 2):
        r = Rollout(kv, "hnd", [1000 + 40 * i for i in range(9)], 8, seed=seed)
        lens = np.repeat(r.lengths, 8) + 5 + np.arange(72) % 50
        r.p.seq_lens = torch.tensor(lens, dtype=torch.int32, device=device())
        assert ways_of(step_of(r)) >= {"planned", "shared32"}
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
        assert torch.equal(bits(out), bits(want))


@pytest.mark.parametrize("size,ways", [(8, {"planned", "shared32"}), (24, {"planned", "shared128"}),
                                       (5, {"small", "shared32"})])
def test_a_step_captured_whole(size, ways):
    """Append and attention in one graph, replayed with eager steps of another cache
    between, against eager steps on a copy."""
    lengths = [900 + 11 * i for i in range(9)]
    n = 9 * size
    made = [Rollout("fp8_e4m3", "hnd", lengths, size, seed=3) for _ in range(2)]
    other = Rollout("fp8_e4m3", "hnd", lengths, size, seed=4)
    steps = []
    for r in made + [other]:
        lens = np.repeat(lengths, size) + np.arange(n) % 7
        r.p.seq_lens = torch.tensor(lens, dtype=torch.int32, device=device())
        now = step_of(r)
        assert ways_of(now) >= ways
        steps.append((r, now, B.RopeAppender(r.p, r.cs), B.PrefixAttention(now, r.start, r.pages),
                      torch.empty_like(r.p.q), torch.empty_like(r.p.q)))
    q, k, v = made[0].tokens(n)

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
        for t, x in zip((q, k, v), made[0].tokens(n)):
            t.copy_(x)
        g.replay()
        run(steps[1], None)
        run(steps[2], None)
        torch.cuda.synchronize()
        assert torch.equal(bits(steps[0][5]), bits(steps[1][5])), i
        assert torch.equal(steps[0][0].p.k_pool, steps[1][0].p.k_pool), i
    del g
