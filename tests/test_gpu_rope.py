"""GPU rotate-and-append against a plain fp64 implementation: queries and bf16 keys
within a rounding, values and re-encoded e4m3 codes bit for bit, and the parts of
the cache that no new token reaches left as they were."""
import numpy as np
import pytest
import torch

from paper_2512_22492_amd import binding as B
from paper_2512_22492_amd import workloads

from gpu_util import device

pytestmark = pytest.mark.gpu

PAGE = 16
D = 128
LAYOUTS = ["hnd", "nhd", "hnd_kv"]
# fp32 arithmetic before the one rounding, relative to |a c| + |b s|: the mean of
# squares is 8 fused terms and 4 additions, a product and a sum with eps (14 roundings,
# halved by the square root), the root, its reciprocal, the two products of the norm
# and the two of the rotation: 7 + 6 = 13 roundings of 2^-24, under 2^-20.
ARITH = 2.0 ** -20


def problem(new, prior, hq=8, hkv=2, kv="bf16", layout="hnd", seed=1, max_pages=None):
    total = [max(0, a) + max(0, b) for a, b in zip(new, prior)]
    p = workloads.make_problem("rope", batch=len(new), num_q_heads=hq, num_kv_heads=hkv,
                               lengths=total, kv_dtype=kv, seed=seed, layout=layout,
                               pool_factor=1.5, max_pages=max_pages).to(device())
    p.seq_lens = torch.tensor(prior, dtype=torch.int32, device=device())
    return p


def tokens(p, new, seed, fused=False, magnitude=True):
    """q, k, v of the new tokens (bf16), whose magnitudes differ from token to token."""
    gen = torch.Generator().manual_seed(seed)
    T, hq, hkv = sum(new), p.num_q_heads, p.num_kv_heads
    x = torch.randn((T, hq + 2 * hkv, D), generator=gen)
    if magnitude:
        x *= torch.exp(2 * torch.randn((T, 1, 1), generator=gen))
    x = x.to(torch.bfloat16).to(device())
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    return (q, k, v) if fused else tuple(t.contiguous() for t in (q, k, v))


def table(rows, rotary, base=1e4):
    f = base ** (-np.arange(0, rotary, 2) / rotary)
    a = np.arange(rows)[:, None] * f
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1)).float().to(device())


def norms(seed):
    gen = torch.Generator().manual_seed(seed)
    return [(1 + 0.3 * torch.randn(D, generator=gen)).to(torch.bfloat16).to(device())
            for _ in range(2)]


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rotated(x, pos, cs, rotary, interleaved, weight=None, eps=1e-6):
    """(fp64 rotation, |a c| + |b s| per element) of head rows x [T, H, D]."""
    x = f64(x)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * f64(weight)
    cs = f64(cs)[pos][:, None]
    c, s = cs[..., :rotary // 2], cs[..., rotary // 2:]
    y, size = x.copy(), np.abs(x)
    lo = slice(0, rotary, 2) if interleaved else slice(0, rotary // 2)
    hi = slice(1, rotary, 2) if interleaved else slice(rotary // 2, rotary)
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    size[..., lo], size[..., hi] = abs(a * c) + abs(b * s), abs(b * c) + abs(a * s)
    return y, size


def slot_major(p, pool):
    """[P, page, Hkv, D] of a pool in any layout (codes stay codes)."""
    x = pool.detach().cpu()
    return x if p.layout == "nhd" else x.transpose(1, 2)


def e4m3(x):
    return x.view(torch.float8_e4m3fn)


def places(new, prior):
    """(sequence, position) of every new token, in row order."""
    return [(b, L + i) for b, (n, L) in enumerate(zip(new, prior)) for i in range(n)]


def snapshot(p):
    return [None if t is None else t.detach().clone()
            for t in (p.k_pool, p.v_pool, p.k_scale, p.v_scale)]


def check_call(p, new, prior, q, k, v, cs, *, rotary, interleaved=False, w=(None, None), eps=1e-6,
               before, q_out, q_was, skipped=()):
    """The cache and q_out after a call against the definition.  `skipped`: rows of
    tokens that the call had to leave out."""
    where = places(new, prior)
    live = [t for t in range(len(where)) if t not in set(skipped)]
    pos = np.array([where[t][1] if t not in set(skipped) else 0 for t in range(len(where))], int)
    qr, qe = rotated(q, pos, cs, rotary, interleaved, w[0], eps)
    kr, ke = rotated(k, pos, cs, rotary, interleaved, w[1], eps)
    got = f64(q_out)
    tol = 2.0 ** -8 * (np.abs(qr) + ARITH * qe) + ARITH * qe + 1e-38
    err = np.abs(got - qr)
    assert np.all(err[live] <= tol[live]), float((err - tol)[live].max())
    assert torch.equal(q_out[list(skipped)].view(torch.int16).cpu(),
                       q_was[list(skipped)].view(torch.int16).cpu())
    tab = p.block_table.cpu().numpy()
    home = [(int(tab[b, at // PAGE]), at % PAGE) if t in set(live) else None
            for t, (b, at) in enumerate(where)]
    pools = (p.k_pool, p.v_pool)
    if p.kv_dtype == "bf16":
        for pool, was, x, size in zip(pools, before[:2], (k, v), (ke, None)):
            now, old = slot_major(p, pool).clone(), slot_major(p, was)
            for t in live:
                page, slot = home[t]
                if size is None:
                    assert torch.equal(now[page, slot], x[t].cpu())
                else:
                    e = np.abs(f64(now[page, slot]) - kr[t])
                    assert np.all(e <= 2.0 ** -8 * (abs(kr[t]) + ARITH * size[t])
                                  + ARITH * size[t] + 1e-38)
                now[page, slot] = old[page, slot]
            assert torch.equal(now.view(torch.int16), old.view(torch.int16)), "elsewhere"
        return
    for name, pool, scale, was, s_was in (("k", p.k_pool, p.k_scale, before[0], before[2]),
                                          ("v", p.v_pool, p.v_scale, before[1], before[3])):
        now, old = slot_major(p, pool).clone(), slot_major(p, was)
        s_now, s_old = scale.cpu(), s_was.cpu()
        touched = {}
        for t in live:
            touched.setdefault(home[t][0], []).append(t)
        for page, rows in touched.items():
            x = kr[rows] if name == "k" else f64(v[rows])
            size = ke[rows] if name == "k" else 0 * x
            first = min(home[t][1] for t in rows)
            b, at = where[rows[0]]
            held = prior[b] - (at // PAGE) * PAGE if prior[b] > (at // PAGE) * PAGE else 0
            top = np.abs(x).max((0, 2))
            want = np.where(top > 0, top / 448, 1.0)
            if held:
                want = np.maximum(want, s_old[page].numpy().astype(np.float64))
            slack = ARITH * size.max((0, 2)) / 448 + 2.0 ** -23 * want
            assert np.all(np.abs(s_now[page].numpy() - want) <= slack), (name, page)
            if name == "v" and len(rows):   # no arithmetic before the encoding: exact
                top32 = torch.from_numpy(top).float()
                exact = torch.where(top32 > 0, top32 / 448.0, torch.ones_like(top32))
                if held:
                    exact = torch.maximum(exact, s_old[page])
                assert torch.equal(s_now[page], exact)
            s = s_now[page][:, None]
            # earlier tokens of the slab: their codes, or re-encoded at the grown scale
            ratio = (s_old[page] / s_now[page])[:, None]
            for slot in range(held):
                again = (e4m3(old[page, slot].contiguous()).float() * ratio).to(
                    torch.float8_e4m3fn).view(torch.uint8)
                grown = (s_now[page] != s_old[page])[:, None]
                assert torch.equal(now[page, slot], torch.where(grown, again, old[page, slot]))
                now[page, slot] = old[page, slot]
            for t, xt, et in zip(rows, x, size):
                slot = home[t][1]
                if name == "v":
                    y = (v[t].cpu().float() / s).clamp(-448, 448)
                    assert torch.equal(now[page, slot], y.to(torch.float8_e4m3fn).view(torch.uint8))
                else:
                    val = f64(e4m3(now[page, slot].contiguous())) * s.numpy().astype(np.float64)
                    # half a step of e4m3, 2^-4 of the value or half its smallest one,
                    # after the fp32 error and the division's rounding
                    tol = (2.0 ** -4 + 2.0 ** -22) * (abs(xt) + ARITH * et) + ARITH * et \
                        + 2.0 ** -10 * s.numpy()
                    assert np.all(np.abs(val - xt) <= tol), float((np.abs(val - xt) - tol).max())
                now[page, slot] = old[page, slot]
            s_now[page] = s_old[page]
            assert first >= held
        assert torch.equal(now, old) and torch.equal(s_now, s_old), "elsewhere"


def call(p, new, prior, *, rotary=D, interleaved=False, norm=False, fused=False, seed=5,
         q_start=None, rows=None, in_place=False, max_new=None, ragged=None, **kw):
    q, k, v = tokens(p, new, seed, fused)
    cs = table(rows or max(a + max(b, 0) for a, b in zip(new, prior)) + 1, rotary)
    w = norms(seed + 1) if norm else (None, None)
    before = snapshot(p)
    q_out = q if in_place else torch.full((sum(new), p.num_q_heads, D), 3.0,
                                          dtype=torch.bfloat16, device=device())
    q_in, q_was = q.clone(), q_out.clone()
    if ragged is None:
        ragged = any(n != 1 for n in new)
    if ragged:
        q_start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32,
                               device=device())
    B.rope_append(p, q, k, v, cs, q_out, q_start, max_new or max(new + [1]), q_norm=w[0],
                  k_norm=w[1], interleaved=interleaved, **kw)
    torch.cuda.synchronize()
    return dict(q=q_in, k=k, v=v, cs=cs, rotary=rotary, interleaved=interleaved, w=w,
                before=before, q_out=q_out, q_was=q_was)


ONE = dict(new=[1] * 9, prior=[0, 1, 14, 15, 16, 17, 100, 255, 256])
MANY = dict(new=[1, 2, 16, 0, 17, 33, 100, 15, 31], prior=[0, 15, 16, 9, 0, 14, 7, 1, 250])


# calls of a few tokens per sequence, within a page and over two
FEW = dict(new=[1, 2, 8, 0, 7, 8, 3, 5], prior=[0, 15, 8, 9, 9, 0, 30, 250])


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("interleaved,rotary", [(False, 128), (False, 96), (True, 128)])
def test_a_few_tokens_have_the_bits_of_many(interleaved, rotary, kv, layout):
    """Up to eight tokens per sequence against the definition, and bit for bit what a
    call gives whose bound allows more (which goes by pages)."""
    outs = []
    for most in (8, 20):
        p = problem(**FEW, kv=kv, layout=layout, seed=15)
        r = call(p, **FEW, norm=rotary == 128, rotary=rotary, interleaved=interleaved, fused=True,
                 max_new=most)
        check_call(p, **FEW, **r)
        outs.append([r["q_out"]] + [t for t in snapshot(p) if t is not None])
    for a, b in zip(*outs):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("shape", [ONE, MANY], ids=["one", "many"])
def test_layouts(shape, kv, layout):
    p = problem(**shape, kv=kv, layout=layout, hq=8, hkv=2)
    check_call(p, **shape, **call(p, **shape, norm=True))


@pytest.mark.parametrize("shape", [ONE, MANY], ids=["one", "many"])
@pytest.mark.parametrize("rotary", [16, 32, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations(rotary, interleaved, shape):
    for kv in ("bf16", "fp8_e4m3"):
        p = problem(**shape, kv=kv, seed=2)
        check_call(p, **shape, **call(p, **shape, rotary=rotary, interleaved=interleaved,
                                      norm=rotary == 64))


@pytest.mark.parametrize("shape", [ONE, MANY], ids=["one", "many"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 1), (5, 5), (64, 8), (64, 4)])
def test_heads_and_fused_projections(hq, hkv, shape):
    for kv in ("bf16", "fp8_e4m3"):
        p = problem(**shape, hq=hq, hkv=hkv, kv=kv, seed=3)
        check_call(p, **shape, **call(p, **shape, fused=True, norm=True))


@pytest.mark.parametrize("shape", [ONE, MANY], ids=["one", "many"])
def test_queries_in_place(shape):
    p = problem(**shape, seed=4)
    check_call(p, **shape, **call(p, **shape, in_place=True, rotary=64))


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_one_token_by_either_form_has_the_same_bits(kv):
    """Single tokens through the one-token form, through q_start, and as a batch whose
    bound allows several."""
    outs = []
    for kw in (dict(), dict(ragged=True), dict(ragged=True, max_new=20)):
        p = problem(**ONE, kv=kv, seed=6)
        r = call(p, **ONE, norm=True, **kw)
        check_call(p, **ONE, **r)
        outs.append([r["q_out"]] + [t for t in snapshot(p) if t is not None])
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_without_rotation_the_bytes_are_the_appends(kv, layout):
    """Cosine 1 and sine 0: step after step the cache equals rl_kv_append's."""
    new, prior = [1] * 5, [0, 3, 15, 16, 40]
    p = problem([6] * 5, prior, kv=kv, layout=layout, seed=7)
    other = p.clone_pools()
    cs = torch.cat([torch.ones(80, 64), torch.zeros(80, 64)], 1).to(device())
    for step in range(6):
        q, k, v = tokens(p, new, 70 + step)
        q_out = torch.empty_like(q)
        B.rope_append(p, q, k, v, cs, q_out)
        B.kv_append(other, k, v)
        p.seq_lens += 1
        other.seq_lens = p.seq_lens
        torch.cuda.synchronize()
        assert torch.equal(q_out.view(torch.int16), q.view(torch.int16))
        for a, b in zip(snapshot(p), snapshot(other)):
            if a is not None:
                assert torch.equal(a.contiguous().view(torch.uint8),
                                   b.contiguous().view(torch.uint8)), step


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("many", [False, True, "few"])
def test_tokens_that_have_no_place_are_left_out(many, kv):
    """Negative lengths, positions past the table and past the rotation table, pages
    out of range: reported, and nothing of them is written."""
    new = {False: [1] * 5, True: [4, 5, 20, 3, 2], "few": [4, 5, 8, 3, 2]}[many]
    prior = [-1, 30, 12, 40, 3]
    room = [a + max(b, 0) for a, b in zip(new, prior)]
    p = problem(room, [0] * 5, kv=kv, seed=8, max_pages=4)
    p.seq_lens = torch.tensor(prior, dtype=torch.int32, device=device())
    err = torch.zeros(1, dtype=torch.int32, device=device())
    where = places(new, prior)
    good = p.block_table.clone()
    # (what is broken, its bit, rows left out beside sequence 0's)
    p.block_table[2, 1] = p.num_pages
    p.block_table[4, 0] = -3
    gone = [t for t, (b, at) in enumerate(where)
            if b == 0 or (b == 2 and at // PAGE == 1) or b == 4]
    r = call(p, new, prior, rows=64, device_error=err)
    assert int(err) == (B.RL_DA_DEVERR_PAGE_OUT_OF_RANGE if many or True else 0)
    check_call(p, new, [max(x, 0) for x in prior], **r, skipped=gone)
    # the rotation table ends inside the new tokens
    p.block_table.copy_(good)
    err.zero_()
    end = 33 if many else 31
    gone = [t for t, (b, at) in enumerate(where) if b == 0 or at >= end]
    r = call(p, new, prior, rows=end, device_error=err)
    assert int(err) == B.RL_DA_DEVERR_LENGTH_TOO_LONG
    check_call(p, new, [max(x, 0) for x in prior], **r, skipped=gone)
    # the block table ends inside the new tokens
    narrow = good[:, :2].contiguous()
    p.block_table = narrow
    err.zero_()
    gone = [t for t, (b, at) in enumerate(where) if b == 0 or at >= 32]
    r = call(p, new, prior, rows=64, device_error=err)
    assert int(err) == B.RL_DA_DEVERR_LENGTH_TOO_LONG
    check_call(p, new, [max(x, 0) for x in prior], **r, skipped=gone)


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_zero_rows_and_rows_behind_the_last(kv):
    """All-zero tokens (scale 1 on a fresh slab, zero rows of the norm stay zero) and
    output rows past the last sequence's tokens."""
    new, prior = [3, 20], [16, 5]
    p = problem(new, prior, kv=kv, seed=9)
    q, k, v = (torch.zeros_like(t) for t in tokens(p, new, 1))
    cs, w, before = table(64, D), norms(3), snapshot(p)
    q_out = torch.full((30, p.num_q_heads, D), 3.0, dtype=torch.bfloat16, device=device())
    q_start = torch.tensor([0, 3, 23], dtype=torch.int32, device=device())
    big = [torch.zeros((30,) + t.shape[1:], dtype=t.dtype, device=device()) for t in (q, k, v)]
    B.rope_append(p, *big, cs, q_out, q_start, 20, q_norm=w[0], k_norm=w[1])
    torch.cuda.synchronize()
    assert (q_out[23:] == 3.0).all() and not q_out[:23].any()
    check_call(p, new, prior, q, k, v, cs, rotary=D, w=w, before=before, q_out=q_out[:23],
               q_was=q_out[:23])


def test_far_positions():
    """Positions near the end of a 65536-token window, one past 2^16 in the table."""
    new, prior = [1, 1], [65535, 65536 + 14]
    p = problem(new, [0, 0], seed=11, max_pages=4100)
    p.block_table[0, 4095] = 0
    p.block_table[1, 4096] = 1
    p.seq_lens = torch.tensor(prior, dtype=torch.int32, device=device())
    check_call(p, new, prior, **call(p, new, prior, norm=True))


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_replays_equal_the_eager_call(kv):
    """A captured append replayed while the sequences grow, with an eager append of
    other tokens to another cache between the replays."""
    new, prior = [1] * 6, [0, 7, 15, 31, 32, 90]
    room = [10] * 6
    p, e = (problem(room, prior, kv=kv, seed=12) for _ in range(2))
    other = problem(room, prior, kv=kv, seed=13)
    cs, w = table(128, D), norms(2)
    q, k, v = tokens(p, new, 14)
    q_out, q_eager = torch.empty_like(q), torch.empty_like(q)
    app = B.RopeAppender(p, cs, q_norm=w[0], k_norm=w[1])
    eager = B.RopeAppender(e, cs, q_norm=w[0], k_norm=w[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        app(q, k, v, q_out, stream=torch.cuda.current_stream())
    for step in range(5):
        for t, x in zip((q, k, v), tokens(p, new, 20 + step)):
            t.copy_(x)
        g.replay()
        eager(q, k, v, q_eager)
        B.rope_append(other, q, v, k, cs, torch.empty_like(q))
        torch.cuda.synchronize()
        assert torch.equal(q_out, q_eager), step
        for a, b in zip(snapshot(p), snapshot(e)):
            assert a is None or torch.equal(a, b), step
        p.seq_lens += 1
        e.seq_lens += 1
    del g


@pytest.mark.parametrize("shape", [ONE, MANY, FEW], ids=["one", "many", "few"])
def test_pages_beyond_4_gib(shape):
    """Page offsets past 32 bits: the pages at the end of a 4.3 GiB pool receive what those
    of a small pool receive."""
    for kv, gib in (("bf16", 9), ("fp8_e4m3", 9)):
        small = problem(**shape, hq=8, hkv=8, kv=kv, seed=16)
        n, page_bytes = small.num_pages, small.k_pool[0].numel() * small.k_pool.element_size()
        pages = (gib << 29) // page_bytes
        k, v = (torch.empty((pages,) + tuple(small.k_pool.shape[1:]), dtype=small.k_pool.dtype,
                            device=device()) for _ in range(2))
        k[-n:], v[-n:] = small.k_pool, small.v_pool
        more = {}
        if kv != "bf16":
            for name in ("k_scale", "v_scale"):
                s = torch.ones((pages, 8), device=device())
                s[-n:] = getattr(small, name)
                more[name] = s
        big = workloads.DecodeProblem(**{**small.__dict__, "k_pool": k, "v_pool": v,
                                         "block_table": small.block_table + (pages - n), **more})
        outs = []
        for p in (small, big):
            q, kn, vn = tokens(p, shape["new"], 17)
            q_out = torch.empty_like(q)
            start = torch.tensor(np.concatenate([[0], np.cumsum(shape["new"])]),
                                 dtype=torch.int32, device=device())
            B.rope_append(p, q, kn, vn, table(400, D), q_out, start, max(shape["new"]))
            torch.cuda.synchronize()
            outs.append([q_out] + [t[-n:] for t in (p.k_pool, p.v_pool, p.k_scale, p.v_scale)
                                   if t is not None])
        for a, b in zip(*outs):
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
        del big, k, v, more, outs, p
