"""What rl_rope_append and rl_prefix_attn refuse, at the C entry and in the binding,
before anything reaches a device (CPU)."""
import types

import pytest
import torch

from paper_2512_22492_amd import binding as B

FAKE = 1 << 20
INVALID, UNSUPPORTED, OK = B.RL_DA_ERR_INVALID_ARG, B.RL_DA_ERR_UNSUPPORTED, B.RL_DA_OK


def rope(**kw):
    args = dict(q=FAKE, q_stride=4096, k_new=FAKE, k_stride=1024, v_new=FAKE, v_stride=1024,
                q_start=FAKE, max_q_per_seq=4, cos_sin=FAKE, num_positions=64, rotary_dim=128,
                interleaved=0, q_norm=None, k_norm=None, norm_eps=1e-6, q_out=2 * FAKE,
                k_pool=FAKE, v_pool=FAKE, k_scale=None, v_scale=None, num_pages=16,
                block_table=FAKE, max_pages=4, seq_lens=FAKE, batch=0, num_q_heads=32,
                num_kv_heads=8)
    args.update(kw)
    return B.rl_rope_append(**args)


@pytest.mark.parametrize("status,kw", [
    (OK, dict()), (OK, dict(batch=2, max_q_per_seq=0)), (OK, dict(q_start=None, max_q_per_seq=1)),
    (OK, dict(q_norm=FAKE, k_norm=FAKE)), (OK, dict(interleaved=1, rotary_dim=16)),
    (OK, dict(q_stride=6144, k_stride=6144, v_stride=6144)), (OK, dict(q_out=FAKE)),
    (INVALID, dict(q=None)), (INVALID, dict(k_new=None)), (INVALID, dict(v_new=None)),
    (INVALID, dict(cos_sin=None)), (INVALID, dict(q_out=None)), (INVALID, dict(k_pool=None)),
    (INVALID, dict(v_pool=None)), (INVALID, dict(block_table=None)),
    (INVALID, dict(seq_lens=None)), (INVALID, dict(batch=-1)), (INVALID, dict(max_q_per_seq=-1)),
    (INVALID, dict(num_q_heads=0)), (INVALID, dict(num_kv_heads=-8)),
    (INVALID, dict(max_pages=0)), (INVALID, dict(num_pages=0)),
    (INVALID, dict(num_positions=0)), (INVALID, dict(rotary_dim=0)),
    (INVALID, dict(q_start=None)),                      # several tokens need q_start
    (INVALID, dict(q_norm=FAKE)), (INVALID, dict(k_norm=FAKE)),
    (INVALID, dict(q_norm=FAKE, k_norm=FAKE, norm_eps=-1.0)),
    (INVALID, dict(q_norm=FAKE, k_norm=FAKE, norm_eps=float("nan"))),
    (INVALID, dict(kv_dtype=7)), (INVALID, dict(layout=3)),
    (INVALID, dict(layout=2)),                          # not one slab apart
    (INVALID, dict(k_scale=FAKE, v_scale=FAKE)), (INVALID, dict(kv_dtype=1)),
    (INVALID, dict(q=FAKE + 2)), (INVALID, dict(v_new=FAKE + 8)),
    (INVALID, dict(cos_sin=FAKE + 4)), (INVALID, dict(q_out=FAKE + 8)),
    (INVALID, dict(q_norm=FAKE + 2, k_norm=FAKE)), (INVALID, dict(k_pool=FAKE + 8)),
    (INVALID, dict(q_stride=4088)), (INVALID, dict(k_stride=1028)),
    (INVALID, dict(v_stride=512)), (INVALID, dict(q_stride=-4096)),
    (INVALID, dict(q_out=FAKE, q_stride=6144)),         # rows would overwrite each other
    (UNSUPPORTED, dict(head_dim=64)), (UNSUPPORTED, dict(page_size=32)),
    (UNSUPPORTED, dict(rotary_dim=8)), (UNSUPPORTED, dict(rotary_dim=72)),
    (UNSUPPORTED, dict(rotary_dim=144)), (UNSUPPORTED, dict(max_pages=1 << 27)),
    (UNSUPPORTED, dict(batch=1 << 20, max_q_per_seq=1 << 20)),
    # pages of 2 GiB: 2^19 kv heads in bf16
    (UNSUPPORTED, dict(num_kv_heads=1 << 19, k_stride=1 << 26, v_stride=1 << 26)),
])
def test_rope_append_host_checks(status, kw):
    assert rope(**kw) == status, kw


def prefix(**kw):
    args = dict(q=FAKE, k_pool=FAKE, v_pool=FAKE, k_scale=None, v_scale=None, num_pages=16,
                block_table=FAKE, max_pages=4, seq_lens=FAKE, batch=0, group_start=FAKE,
                prefix_pages=FAKE, num_groups=3, num_q_heads=32, num_kv_heads=8, out=2 * FAKE,
                workspace=FAKE, workspace_bytes=1 << 40)
    args.update(kw)
    return B.rl_prefix_attn(**args)


@pytest.mark.parametrize("status,kw", [
    (OK, dict()), (OK, dict(num_groups=0, group_start=None, prefix_pages=None)),
    (INVALID, dict(q=None)), (INVALID, dict(k_pool=None)), (INVALID, dict(v_pool=None)),
    (INVALID, dict(block_table=None)), (INVALID, dict(seq_lens=None)), (INVALID, dict(out=None)),
    (INVALID, dict(workspace=None)), (INVALID, dict(group_start=None)),
    (INVALID, dict(prefix_pages=None)), (INVALID, dict(num_groups=-1)),
    (INVALID, dict(batch=-1)), (INVALID, dict(max_pages=0)), (INVALID, dict(num_pages=0)),
    (INVALID, dict(num_q_heads=30)), (INVALID, dict(num_q_heads=0)),
    (INVALID, dict(num_kv_heads=0)), (INVALID, dict(scale=float("inf"))),
    (INVALID, dict(kv_dtype=2)), (INVALID, dict(kv_dtype=1)),
    (INVALID, dict(k_scale=FAKE, v_scale=FAKE)), (INVALID, dict(layout=-1)),
    (INVALID, dict(layout=2)), (INVALID, dict(q=FAKE + 8)), (INVALID, dict(out=2 * FAKE + 2)),
    (INVALID, dict(v_pool=FAKE + 4)), (INVALID, dict(workspace=FAKE + 8)),
    (INVALID, dict(batch=2, workspace_bytes=255)),
    (INVALID, dict(batch=2, out=FAKE)), (INVALID, dict(batch=2, out=FAKE + 2 * 32 * 256 - 16)),
    (INVALID, dict(batch=2, out=FAKE - 16)),
    (UNSUPPORTED, dict(head_dim=64)), (UNSUPPORTED, dict(page_size=8)),
    (UNSUPPORTED, dict(num_q_heads=24)), (UNSUPPORTED, dict(num_q_heads=256)),
    (UNSUPPORTED, dict(batch=1 << 30)), (UNSUPPORTED, dict(max_pages=1 << 27)),
    (UNSUPPORTED, dict(num_q_heads=1 << 19, num_kv_heads=1 << 19)),
])
def test_prefix_attn_host_checks(status, kw):
    assert prefix(**kw) == status, kw


def test_prefix_workspace_size():
    def size(*a):
        rc, n = B.rl_prefix_attn_workspace_size(*a)
        assert rc == OK
        return n

    # room for every row's partial results
    assert size(256, 64, 8, 32, 8) >= 64 * 32 * 2 * (128 + 2) * 4
    assert size(512, 64, 8, 32, 8) >= size(256, 64, 8, 32, 8)
    assert size(4096, 0, 0, 32, 8) >= 0
    for bad in ((0, 64, 8, 32, 8), (256, -1, 8, 32, 8), (256, 64, -1, 32, 8),
                (256, 64, 8, 0, 8), (256, 64, 8, 32, 0), (256, 64, 8, 30, 8)):
        assert B.rl_prefix_attn_workspace_size(*bad)[0] == INVALID
    assert B.rl_prefix_attn_workspace_size(1 << 27, 64, 8, 32, 8)[0] == UNSUPPORTED
    lib = B.load_library()
    assert lib.rl_prefix_attn_workspace_size(256, 64, 8, 32, 8, None) == INVALID


def cache(batch=3, hq=4, hkv=2, pages=4):
    pool = torch.zeros((8, hkv, 16, 128), dtype=torch.bfloat16)
    return types.SimpleNamespace(
        kv_dtype="bf16", layout="hnd", num_q_heads=hq, num_kv_heads=hkv, head_dim=128,
        page_size=16, batch=batch, num_pages=8, max_pages=pages, scale=1.0, k_pool=pool,
        v_pool=pool.clone(), k_scale=None, v_scale=None,
        q=torch.zeros((batch, hq, 128), dtype=torch.bfloat16),
        block_table=torch.zeros((batch, pages), dtype=torch.int32),
        seq_lens=torch.ones(batch, dtype=torch.int32))


def test_binding_checks_prefix_tensors(monkeypatch):
    p = cache()
    start = torch.tensor([0, 3], dtype=torch.int32)
    pages = torch.tensor([2], dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):         # the cache is not on one
        B.PrefixAttention(p, start, pages)
    for s, n in ((start.long(), pages), (start, pages.long()), (start[:1], pages),
                 (start, pages.view(1, 1)), (start, torch.tensor([1, 2], dtype=torch.int32)),
                 ([0, 3], pages)):
        with pytest.raises(ValueError, match="group_start|prefix_pages"):
            B.PrefixAttention(p, s, n)
    monkeypatch.setattr(B, "_device_index", lambda d: 0)
    monkeypatch.setattr(B, "_on_device", lambda i, fn, *args: fn(*args))
    need = B.rl_prefix_attn_workspace_size(4, 3, 1, 4, 2)[1]
    ws = torch.zeros(need, dtype=torch.uint8)
    for bad in (ws[:-1], ws[::2], ws.view(torch.int32), ws.view(2, -1), 7):
        with pytest.raises(ValueError, match="workspace"):
            B.PrefixAttention(p, start, pages, bad)
    with pytest.raises(ValueError, match="device_error"):
        B.PrefixAttention(p, start, pages, ws, torch.zeros(1))
    attn = B.PrefixAttention(p, start, pages, ws)
    seen = []
    attn._fn = lambda *a: seen.append(a) or OK
    out = torch.empty_like(p.q)
    attn(p.q, out)
    assert len(seen[0]) == len(B.load_library().rl_prefix_attn.argtypes)
    for q, o in ((p.q[:2], out), (p.q, out[:, :2]), (p.q.float(), out), (p.q, out.transpose(0, 1))):
        with pytest.raises(ValueError, match="q |out "):
            attn(q, o)
    attn._fn = lambda *a: B.RL_DA_ERR_HIP
    with pytest.raises(B.RLDecodeAttnError):
        attn(p.q, out)


def test_binding_checks_rope_tensors(monkeypatch):
    p = cache()
    cs = torch.zeros((32, 128))
    with pytest.raises(ValueError, match="GPU"):
        B.RopeAppender(p, cs)
    w = torch.ones(128, dtype=torch.bfloat16)
    for kw in (dict(cos_sin=cs.double()), dict(cos_sin=cs[0]), dict(cos_sin=cs[:, ::2]),
               dict(q_norm=w), dict(k_norm=w), dict(q_norm=w.float(), k_norm=w),
               dict(q_norm=w, k_norm=w[:64]), dict(device_error=torch.zeros(1))):
        with pytest.raises(ValueError, match="cos_sin|norm|device_error"):
            B.RopeAppender(p, **{**dict(cos_sin=cs), **kw})
    monkeypatch.setattr(B, "_device_index", lambda d: 0)
    monkeypatch.setattr(B, "_on_device", lambda i, fn, *args: fn(*args))
    app = B.RopeAppender(p, cs, q_norm=w, k_norm=w)
    seen = []
    app._fn = lambda *a: seen.append(a) or OK
    fused = torch.zeros((3, 8, 128), dtype=torch.bfloat16)
    q, k, v = fused[:, :4], fused[:, 4:6], fused[:, 6:]
    out = torch.empty((3, 4, 128), dtype=torch.bfloat16)
    app(q, k, v, out)
    assert len(seen[0]) == len(B.load_library().rl_rope_append.argtypes)
    assert seen[0][1] == seen[0][3] == seen[0][5] == 1024   # the fused rows' stride
    app(q.contiguous(), k.contiguous(), v.contiguous(), out)
    assert seen[1][1:6:2] == (512, 256, 256)
    start = torch.tensor([0, 1, 1, 3], dtype=torch.int32)
    app(q, k, v, out, start, 2)
    assert seen[2][6] == start.data_ptr() and seen[2][7] == 2
    app(q[:0], k[:0], v[:0], out[:0], torch.zeros(4, dtype=torch.int32), 1)
    assert len(seen) == 3                                    # nothing to do
    odd = torch.zeros((3, 4 * 128 + 4), dtype=torch.bfloat16)[:, :512].unflatten(1, (4, 128))
    wide = torch.zeros((3, 4, 256), dtype=torch.bfloat16)[..., :128]
    bad = [(q[:2], k, v, out), (q, k[:2], v, out), (q, k, v, out[:2]), (q.float(), k, v, out),
           (q[..., :64], k, v, out), (odd, k, v, out), (wide, k, v, out),
           (q[:, [0, 1, 2]], k, v, out), (q, k, v, fused[:, :4]),
           (q[:1].expand(3, 4, 128), k, v, out)]
    for args in bad:
        with pytest.raises(ValueError):
            app(*args)
    for s in (start.long(), start[:3], [0, 1, 1, 3]):
        with pytest.raises(ValueError, match="q_start"):
            app(q, k, v, out, s, 2)
    with pytest.raises(ValueError):
        app(q, k, v[:2], out, start, 2)
