"""Attention over a prefix that sequences share, and the append that rotates on
the way into the cache: what a rollout of several responses to each prompt runs,
as cases that can be timed and compared with their plain forms.

A rollout engine samples several responses to one prompt.  The prompt's pages
are in the cache once, and every response's block table starts with them; a
decode step projects each sequence's new token, normalises and rotates its query
and key, appends key and value, and attends.  Prompts and turns of several
tokens go through the same append before their prefill.

Shapes are those of paper_2512_22492_amd/workloads.py and perf/cases.py (head
layouts, page size, window); lengths belong to the case (drawn from its own
"shape_seed"), so its work does not depend on the seed its values are made from.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # False: run() computes the plain forms; True: it calls the framework

DEV = "cuda"
PAGE = 16
D = 128
WINDOW = 65536   # the rollout's context window in tokens
# query heads / kv heads: Qwen3-8B, its TP = 8 share, Qwen3-32B, Qwen3-235B, the
# "tiny" workload's, and a layout without grouping
HEADS = [(32, 8), (4, 1), (64, 8), (64, 4), (8, 2), (8, 8)]


# ------------------------------------------------------------------ cases ---

def _prefix(name, groups, size, heads, prompt, response, kv="bf16", layout="hnd", done=0.0,
            window=0, shape_seed=0):
    """`groups` prompts with `size` responses each; lengths in tokens.  A share
    `done` of the sequences has ended (length 0)."""
    c = dict(op="prefix", groups=groups, size=size, hq=heads[0], hkv=heads[1], prompt=prompt,
             response=response, kv=kv, layout=layout, done=done, window=window,
             shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def _rope(name, batch, heads, new, prior, kv="bf16", layout="hnd", norm=True, rotary=D,
          interleaved=False, shape_seed=0):
    """Each sequence gets `new` tokens after `prior` cached ones."""
    c = dict(op="rope", batch=batch, hq=heads[0], hkv=heads[1], new=new, prior=prior, kv=kv,
             layout=layout, norm=norm, rotary=rotary, interleaved=interleaved,
             shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest step: four responses to one short prompt
        _prefix("prefix_tiny", 1, "fixed:4", (8, 2), "fixed:200", "uniform:1:40", shape_seed=1),
        # the end of a rollout on one GPU of eight: a few long responses left
        _prefix("prefix_few_left", 3, "uniform:1:8", (4, 1), "uniform:500:2000",
                "uniform:2000:16000", window=WINDOW, shape_seed=2),
        # the middle of a rollout: 64 prompts x 8 responses
        _prefix("prefix_rollout", 64, "fixed:8", (32, 8), "uniform:200:2000",
                "lognormal:1500:0.8:16:8192", shape_seed=3),
        # one long system prompt under a whole batch that has just begun to answer
        _prefix("prefix_system", 1, "fixed:256", (64, 4), "fixed:8192", "uniform:1:300",
                shape_seed=4),
        # the start of a rollout over long prompts, e4m3 token-major pools
        _prefix("prefix_start_e4m3", 64, "fixed:8", (64, 8), "uniform:1000:4000",
                "uniform:1:200", kv="fp8_e4m3", layout="nhd", shape_seed=5),
        # continuous batching: groups of any size, some responses ended, odd lengths
        _prefix("prefix_ragged", 37, "uniform:1:33", (32, 8), "uniform:0:1500",
                "uniform:1:900", layout="hnd_kv", done=0.1, shape_seed=6),
        # the smallest append: one token of four sequences
        _rope("rope_tiny", 4, (8, 2), "fixed:1", "uniform:1:512", norm=False, shape_seed=7),
        # the append of the rollout's decode step
        _rope("rope_step", 512, (32, 8), "fixed:1", "uniform:200:1000", shape_seed=8),
        # the same into e4m3 pools, whose slab scales grow
        _rope("rope_step_e4m3", 256, (64, 8), "fixed:1", "uniform:64:1024", kv="fp8_e4m3",
              shape_seed=9),
        # prompts on their way into an empty cache
        _rope("rope_prompts", 48, (32, 8), "uniform:100:2000", "fixed:0", shape_seed=10),
        # a turn of a few hundred tokens for every sequence, e4m3 token-major pools,
        # half of each head rotated in interleaved pairs
        _rope("rope_turns_e4m3", 64, (64, 4), "uniform:64:512", "uniform:100:2000",
              kv="fp8_e4m3", layout="nhd", norm=False, rotary=64, interleaved=True,
              shape_seed=11),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kv = rng.choice(["bf16", "fp8_e4m3"])
    layout = rng.choice(["hnd", "hnd", "nhd", "hnd_kv"])
    seed = rng.randrange(1 << 30)
    if rng.random() < 0.55:
        while True:
            heads = rng.choice(HEADS)
            groups = _log_int(rng, 1, 96)
            n = _log_int(rng, 1, 256)
            prompt, resp = _log_int(rng, 16, 12000), _log_int(rng, 1, 16000)
            c = _prefix(None, groups,
                        rng.choice(["fixed:%d" % n, "uniform:%d:%d" % ((n + 3) // 4, n)]), heads,
                        rng.choice(["fixed:%d" % prompt,
                                    "uniform:%d:%d" % (prompt // 3, prompt)]),
                        rng.choice(["fixed:%d" % resp,
                                    "uniform:%d:%d" % (max(1, resp // 8), resp),
                                    "lognormal:%d:0.8:1:%d" % (resp, min(4 * resp, 40000))]),
                        kv=kv, layout=layout, done=rng.choice([0.0, 0.0, 0.1, 0.5]),
                        window=rng.choice([0, 0, WINDOW]), shape_seed=seed)
            if groups * n > 768 or (c["window"] and groups * n > 256):
                continue
            w = work(c)
            if w["bytes"] <= 4.0e9 and w["flops"] <= 7.0e10:
                return c
    while True:
        batch = _log_int(rng, 1, 768)
        one = rng.random() < 0.5
        new = 1 if one else _log_int(rng, 2, 4000)
        prior = 0 if rng.random() < 0.25 else _log_int(rng, 1, 8000)
        c = _rope(None, batch, rng.choice(HEADS),
                  rng.choice(["fixed:%d" % new, "uniform:%d:%d" % (new // 6, new)]),
                  rng.choice(["fixed:%d" % prior, "uniform:%d:%d" % (prior // 4, prior)]),
                  kv=kv, layout=layout, norm=rng.random() < 0.5,
                  rotary=rng.choice([128, 128, 64, 96, 32]),
                  interleaved=rng.random() < 0.3, shape_seed=seed)
        new_l, prior_l = _new_prior(c)
        pool = int((-(-(new_l + prior_l) // PAGE)).sum()) * PAGE * c["hkv"] * D * 4
        if int(new_l.sum()) and work(c)["bytes"] <= 1.5e9 and pool <= 1.2e9:
            return c


# ----------------------------------------------------------------- shapes ---

def _lengths(text, n, rng):
    kind, *rest = text.split(":")
    v = [float(x) for x in rest]
    if kind == "fixed":
        return np.full(n, int(v[0]), np.int64)
    if kind == "uniform":
        return rng.integers(int(v[0]), int(v[1]), size=n, endpoint=True, dtype=np.int64)
    return np.clip(np.rint(v[0] * np.exp(v[1] * rng.standard_normal(n))), v[2],
                   v[3]).astype(np.int64)


def _groups(case):
    """(start of each group, prompt tokens of each group, length of each sequence)."""
    rng = np.random.default_rng([int(case["shape_seed"]), 1])
    sizes = _lengths(case["size"], case["groups"], rng)
    prompts = _lengths(case["prompt"], case["groups"], rng)
    start = np.concatenate([[0], np.cumsum(sizes)])
    lens = np.repeat(prompts, sizes) + _lengths(case["response"], int(start[-1]), rng)
    lens = np.where(rng.random(lens.size) < case["done"], 0, np.minimum(lens, WINDOW))
    return start, prompts, lens


def _new_prior(case):
    rng = np.random.default_rng([int(case["shape_seed"]), 2])
    return _lengths(case["new"], case["batch"], rng), _lengths(case["prior"], case["batch"], rng)


# ---------------------------------------------------------------- prepare ---

def _randn(shape, gen, spread=1.0):
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    flat = x.view(-1)
    for s in range(0, flat.numel(), 1 << 27):
        part = flat[s:s + (1 << 27)]
        part.copy_(torch.randn(part.numel(), generator=gen, device=DEV) * spread)
    return x


def _pools(case, pages, gen):
    """{k, v, ks, vs}: pools in the case's layout, e4m3 codes as bytes with a scale per
    (page, kv head) slab that maps its largest value to about 448."""
    hkv, kv = case["hkv"], case["kv"]
    shape = (pages, PAGE, hkv, D) if case["layout"] == "nhd" else (pages, hkv, PAGE, D)
    if kv == "bf16":
        k, v, ks, vs = _randn(shape, gen), _randn(shape, gen), None, None
    else:
        def codes():
            return (_randn(shape, gen, 100.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
                    .view(torch.uint8))

        def scales():
            return (torch.rand((pages, hkv), generator=gen, device=DEV) + 0.5) / 100.0
        k, v, ks, vs = codes(), codes(), scales(), scales()
    if case["layout"] == "hnd_kv":
        both = torch.stack([k, v], dim=2)
        k, v = both[:, :, 0], both[:, :, 1]
    return dict(k=k, v=v, ks=ks, vs=vs)


def _prefix_inputs(case, seed):
    start, prompts, lens = _groups(case)
    shared = prompts // PAGE                 # whole pages of the prompt
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 1009 + 3)
    rng = np.random.default_rng([int(case["shape_seed"]), int(seed)])
    need = -(-lens // PAGE)
    width = max(1, int(need.max()), int(shared.max()))
    group = np.repeat(np.arange(case["groups"]), np.diff(start))
    first = shared[group]                    # pages of each sequence that it shares
    total = int(shared.sum() + np.maximum(need - first, 0).sum())
    pages = rng.permutation(total + 1)
    table = np.full((lens.size, case["window"] // PAGE or width), pages[total], np.int32)
    at = 0
    for g in range(case["groups"]):
        run_of = pages[at:at + shared[g]]
        at += int(shared[g])
        for b in range(start[g], start[g + 1]):
            table[b, :shared[g]] = run_of
            n = max(0, int(need[b] - shared[g]))
            table[b, shared[g]:shared[g] + n] = pages[at:at + n]
            at += n
    d = _pools(case, total + 1, gen)
    # queries of twice the keys' spread: scores with a standard deviation of 2
    d.update(q=_randn((lens.size, case["hq"], D), gen, 2.0), scale=1.0 / math.sqrt(D),
             table=torch.from_numpy(table).to(DEV),
             lens=torch.from_numpy(lens.astype(np.int32)).to(DEV),
             start=torch.from_numpy(start.astype(np.int32)).to(DEV),
             shared=torch.from_numpy(shared.astype(np.int32)).to(DEV),
             # what the engine's scheduler knows on the host as well
             host=(start.tolist(), shared.tolist(), lens.tolist()))
    return d


def _rope_inputs(case, seed):
    new, prior = _new_prior(case)
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 1009 + 4)
    rng = np.random.default_rng([int(case["shape_seed"]), int(seed)])
    need = -(-(new + prior) // PAGE)
    total = int(need.sum())
    pages = rng.permutation(total + 1)
    table = np.full((case["batch"], max(1, int(need.max()))), pages[total], np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = pages[at:at + n]
        at += n
    d = _pools(case, total + 1, gen)
    tokens, hq, hkv = int(new.sum()), case["hq"], case["hkv"]
    # the fused projection's output, and q, k, v as views of it; magnitudes that
    # differ from token to token, so that slab scales grow and stay
    qkv = _randn((tokens, hq + 2 * hkv, D), gen)
    qkv *= torch.exp(torch.randn((tokens, 1, 1), generator=gen, device=DEV)).to(qkv.dtype)
    r = case["rotary"]
    rows = int((new + prior).max()) + 1
    angle = (torch.arange(rows, device=DEV, dtype=torch.float64)[:, None] *
             1e6 ** (-torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / r))
    d.update(q=qkv[:, :hq], k_new=qkv[:, hq:hq + hkv], v_new=qkv[:, hq + hkv:],
             cos_sin=torch.cat([angle.cos(), angle.sin()], 1).float(),
             q_norm=None, k_norm=None, eps=1e-6, interleaved=case["interleaved"],
             q_out=torch.empty((tokens, hq, D), dtype=torch.bfloat16, device=DEV),
             table=torch.from_numpy(table).to(DEV),
             before=torch.from_numpy(prior.astype(np.int32)).to(DEV),
             q_start=None, max_new=int(new.max()), host=(new.tolist(), prior.tolist()))
    if not (new == 1).all():
        d["q_start"] = torch.from_numpy(
            np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
    if case["norm"]:
        d["q_norm"] = (1 + _randn((D,), gen, 0.2)).to(torch.bfloat16)
        d["k_norm"] = (1 + _randn((D,), gen, 0.2)).to(torch.bfloat16)
    return d


def _inputs(case, seed):
    return _prefix_inputs(case, seed) if case["op"] == "prefix" else _rope_inputs(case, seed)


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = dict(case)
    if own:
        from paper_2512_22492_amd import binding, workloads
        prefix = case["op"] == "prefix"
        p = workloads.DecodeProblem(
            name=case["op"], seed=int(seed), batch=int(st["table"].shape[0]),
            num_q_heads=case["hq"], num_kv_heads=case["hkv"], head_dim=D, page_size=PAGE,
            kv_dtype=case["kv"], layout=case["layout"], scale=1.0 / math.sqrt(D),
            q=st["q"], k_pool=st["k"], v_pool=st["v"], k_scale=st["ks"], v_scale=st["vs"],
            block_table=st["table"], seq_lens=st["lens"] if prefix else st["before"],
            pad_page=0)
        if prefix:
            st["out"] = torch.empty_like(st["q"])
            st["attend"] = binding.PrefixAttention(p, st["start"], st["shared"])
        else:
            st["append"] = binding.RopeAppender(
                p, st["cos_sin"], q_norm=st["q_norm"], k_norm=st["k_norm"], eps=st["eps"],
                interleaved=st["interleaved"])
    elif case["op"] == "rope":
        # where each new token goes, as an engine's scheduler lays it out
        new, prior = (np.asarray(x) for x in st["host"])
        seq = np.repeat(np.arange(new.size), new)
        i = np.arange(seq.size) - np.repeat(np.cumsum(new) - new, new)
        at = prior[seq] + i
        touched, place = np.unique(seq * (1 << 32) + at // PAGE, return_inverse=True)
        b, page = touched >> 32, touched & ((1 << 32) - 1)
        old = np.clip(prior[b] - page * PAGE, 0, PAGE)
        st["plain"] = {k: torch.from_numpy(np.ascontiguousarray(v)).to(DEV) for k, v in dict(
            seq=seq, at=at, place=place.reshape(-1), b=b, page=page, old=old).items()}
    return st


# -------------------------------------------------------------------- run ---

def _slabs(st, name, pages):
    """[..., Hkv, PAGE, D] fp32 of pages `pages` of pool "k" or "v"."""
    x = st[name][pages]
    if st["ks"] is not None:
        x = x.view(torch.float8_e4m3fn)
    x = x.float()
    if st["case"]["layout"] == "nhd":
        x = x.transpose(-3, -2)
    if st["ks"] is not None:
        x = x * st[name + "s"][pages][..., None, None]
    return x


def _plain_prefix(st):
    start, shared, lens = st["host"]
    hq, hkv = st["case"]["hq"], st["case"]["hkv"]
    G = hq // hkv
    out = torch.empty_like(st["q"])
    for g in range(len(shared)):
        P = shared[g] * PAGE
        if shared[g] and any(lens[start[g]:start[g + 1]]):
            pages = st["table"][start[g], :shared[g]]
            kp, vp = (_slabs(st, n, pages).transpose(0, 1).reshape(hkv, P, D) for n in "kv")
        else:
            kp = vp = torch.zeros((hkv, 0, D), device=DEV)
        for b0 in range(start[g], start[g + 1], 32):
            b1 = min(b0 + 32, start[g + 1])
            n = b1 - b0
            q = st["q"][b0:b1].float().view(n, hkv, G, D)
            cols = max(0, max(-(-L // PAGE) for L in lens[b0:b1]) - shared[g])
            S = cols * PAGE
            x = torch.empty((n, hkv, G, kp.shape[1] + S), device=DEV)
            Pk = kp.shape[1]
            x[..., :Pk] = ((q.transpose(0, 1).reshape(hkv, n * G, D) @ kp.transpose(1, 2))
                           .view(hkv, n, G, Pk).transpose(0, 1))
            if S:
                pages = st["table"][b0:b1, shared[g]:shared[g] + cols]
                ks, vs = (_slabs(st, m, pages).transpose(1, 2).reshape(n, hkv, S, D)
                          for m in "kv")
                x[..., Pk:] = q @ ks.transpose(2, 3)
            x *= st["scale"]
            dead = (torch.arange(Pk + S, device=DEV)[None] >= st["lens"][b0:b1, None])
            x.masked_fill_(dead[:, None, None], -math.inf)
            if Pk + S == 0:
                out[b0:b1] = 0
                continue
            top = x.amax(-1, keepdim=True)
            w = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
            o = (w[..., :Pk].transpose(0, 1).reshape(hkv, n * G, Pk) @ vp
                 ).view(hkv, n, G, D).transpose(0, 1)
            if S:
                o = o + w[..., Pk:] @ vs
            den = w.sum(-1, keepdim=True)
            o = torch.where(den > 0, o / den, torch.zeros_like(o))
            out[b0:b1] = o.reshape(n, hq, D).to(torch.bfloat16)
    return out


def _plain_rotate(st, x, weight):
    """RMS norm of each head (where there is a weight), then the rotation; fp32."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + st["eps"]) * weight.float()
    r = st["case"]["rotary"]
    cs = st["cos_sin"][st["plain"]["at"]][:, None]
    c, s = cs[..., :r // 2], cs[..., r // 2:]
    y = x.clone()
    if st["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * c - b * s, b * c + a * s
    return y


def _plain_rope(st):
    m = st["plain"]
    st["q_out"].copy_(_plain_rotate(st, st["q"], st["q_norm"]))
    k = _plain_rotate(st, st["k_new"], st["k_norm"])
    v = st["v_new"].float()
    nhd = st["case"]["layout"] == "nhd"
    if st["ks"] is None:
        page = st["table"][m["seq"], m["at"] // PAGE].long()
        slot = m["at"] % PAGE
        for pool, x in ((st["k"], k), (st["v"], v)):
            x = x.to(torch.bfloat16)
            if nhd:
                pool[page, slot] = x
            else:
                pool[page, :, slot] = x
        return
    page = st["table"][m["b"], m["page"]].long()
    slots = torch.arange(PAGE, device=DEV)
    earlier = slots[None] < m["old"][:, None]
    for pool, scale, x in ((st["k"], st["ks"], k), (st["v"], st["vs"], v)):
        hkv = x.shape[1]
        top = torch.zeros((page.numel(), hkv), device=DEV)
        top.scatter_reduce_(0, m["place"][:, None].expand(-1, hkv), x.abs().amax(-1), "amax")
        want = torch.where(top > 0, top / 448.0, torch.ones_like(top))
        was = scale[page]
        now = torch.where(m["old"][:, None] > 0, torch.maximum(was, want), want)
        scale[page] = now
        code = pool[page]
        if nhd:
            code = code.transpose(1, 2)
        grown = (code.view(torch.float8_e4m3fn).float() * (was / now)[..., None, None]
                 ).to(torch.float8_e4m3fn).view(torch.uint8)
        change = earlier[:, None, :, None] & (now != was)[..., None, None]
        code = torch.where(change, grown, code)
        y = (x / now[m["place"]][..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        code[m["place"], :, m["at"] % PAGE] = y.view(torch.uint8)
        pool[page] = code.transpose(1, 2) if nhd else code


def _cache_of(st):
    if st["ks"] is None:
        return [st["k"], st["v"]]
    return [st["k"].view(torch.float8_e4m3fn), st["v"].view(torch.float8_e4m3fn),
            st["ks"], st["vs"]]


def run(state):
    st = state
    if st["case"]["op"] == "prefix":
        if own:
            st["attend"](st["q"], st["out"], torch.cuda.current_stream())
            return st["out"]
        return _plain_prefix(st)
    if own:
        st["append"](st["q"], st["k_new"], st["v_new"], st["q_out"], st["q_start"],
                     st["max_new"], torch.cuda.current_stream())
    else:
        _plain_rope(st)
    return [st["q_out"]] + _cache_of(st)


# ------------------------------------------------------------------- work ---

def work(case):
    elt = 2 if case["kv"] == "bf16" else 1
    hq, hkv = case["hq"], case["hkv"]
    if case["op"] == "prefix":
        start, prompts, lens = _groups(case)
        shared = prompts // PAGE
        live = np.add.reduceat(np.append(lens, 0), start[:-1]) > 0
        mine = np.maximum(lens - np.repeat(shared * PAGE, np.diff(start)), 0)
        keys = int((shared * PAGE * live).sum() + mine.sum())
        pages = int((shared * live).sum() + (-(-mine // PAGE)).sum())
        n = keys * hkv * D * 2 * elt + 2 * lens.size * hq * D * 2 + 4 * (pages + lens.size)
        if elt == 1:
            n += pages * hkv * 2 * 4
        return {"bytes": n, "flops": 4 * D * hq * int(lens.sum())}
    new, prior = _new_prior(case)
    tokens = int(new.sum())
    far = np.zeros(int((new + prior).max()) + 2, np.int64)   # distinct positions
    np.add.at(far, prior, 1)
    np.add.at(far, prior + new, -1)
    n = tokens * (2 * hq * D * 2 + 2 * hkv * D * (2 + elt))
    n += 4 * case["rotary"] * int((np.cumsum(far) > 0).sum())
    pages = int((np.where(new > 0, (prior + new - 1) // PAGE - prior // PAGE + 1, 0)).sum())
    n += 4 * pages + 4 * case["batch"]
    if elt == 1:
        n += pages * hkv * 2 * 4
    return {"bytes": n, "flops": tokens * (hq + hkv) * (3 * case["rotary"]
                                                       + (4 * D if case["norm"] else 0))}


# ------------------------------------------------------------------ exact ---

def exact(case, seed):
    st = _inputs(case, seed)
    nhd = case["layout"] == "nhd"

    def wide(pool, scale, page, h):
        """Pages `page` of kv head h in 64 bits, as [tokens, D]."""
        x = pool[page, :, h] if nhd else pool[page, h]
        if scale is None:
            return x.double().reshape(-1, D)
        return (x.contiguous().view(torch.float8_e4m3fn).double()
                * scale[page, h].double()[:, None, None]).reshape(-1, D)

    if case["op"] == "prefix":
        lens = st["host"][2]
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
        G = case["hq"] // case["hkv"]
        if len(lens) * case["hkv"] > 8192:
            return None
        for b, L in enumerate(lens):
            page = st["table"][b, :-(-L // PAGE)].long()
            for h in range(case["hkv"] if L else 0):
                k = wide(st["k"], st["ks"], page, h)[:L]
                v = wide(st["v"], st["vs"], page, h)[:L]
                s = (k @ st["q"][b, h * G:(h + 1) * G].double().T.contiguous()) / D ** 0.5
                out[b, h * G:(h + 1) * G] = torch.softmax(s, 0).T.contiguous() @ v
        return out

    new, prior = st["host"]
    r, half = case["rotary"], case["rotary"] // 2
    where = torch.tensor([p + i for n, p in zip(new, prior) for i in range(n)], device=DEV)
    turn = torch.complex(st["cos_sin"][where, :half].double(),
                         st["cos_sin"][where, half:].double())[:, None]

    def rotated(x, w):
        x = x.double()
        if w is not None:
            x = x / (x.square().sum(-1, keepdim=True) / D + st["eps"]).sqrt() * w.double()
        pairs = (x[..., :r].unflatten(-1, (half, 2)) if case["interleaved"]
                 else x[..., :r].unflatten(-1, (2, half)).transpose(-1, -2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z if case["interleaved"] else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), x[..., r:]], -1)

    q, k, v = (rotated(st["q"], st["q_norm"]), rotated(st["k_new"], st["k_norm"]),
               st["v_new"].double())
    outs, scales = [q], []
    for name, x in (("k", k), ("v", v)):
        pool, scale = st[name], st[name + "s"]
        # in the order [page, slot, head, dim], whatever the layout
        value = pool if scale is None else pool.view(torch.float8_e4m3fn)
        value = value.double() if nhd else value.double().transpose(1, 2)
        value = value.clone()
        scale = None if scale is None else scale.double()
        t = 0
        for b, (n, p) in enumerate(zip(new, prior)):
            for j in range(p // PAGE, -(-(p + n) // PAGE) if n and scale is not None else 0):
                lo, hi = max(p, j * PAGE), min(p + n, (j + 1) * PAGE)
                page = int(st["table"][b, j])
                piece = x[t + lo - p:t + hi - p]
                top = piece.abs().amax((0, 2)) / 448
                top = torch.where(top > 0, top, torch.ones_like(top))
                grown = torch.maximum(scale[page], top) if lo > j * PAGE else top
                first = lo - j * PAGE
                if first:
                    value[page, :first] *= (scale[page] / grown)[None, :, None]
                value[page, first:hi - j * PAGE] = piece / grown[None, :, None]
                scale[page] = grown
            t += n
        if scale is None:
            row = torch.repeat_interleave(torch.arange(len(new), device=DEV),
                                          torch.tensor(new, device=DEV))
            value[st["table"][row, where // PAGE].long(), where % PAGE] = x
        outs.append(value if nhd else value.transpose(1, 2))
        scales.append(scale)
    return outs + ([] if scales[0] is None else scales)
