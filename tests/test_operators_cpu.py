"""Refusals of the operators outside the module step, and the rotary frequencies: host arithmetic only, nothing is enqueued."""
import ctypes
import math

import pytest

from test_abi_cpu import B  # noqa: F401  (the module fixture that builds the library if need be)

FAKE = ctypes.c_void_p(0x1000)  # aligned, never dereferenced on the host


def test_frequencies(B):
    f = B.mrem_rotary_frequencies(64).tolist()
    assert all(math.isclose(v, 10000.0 ** (-2 * i / 64), rel_tol=1e-14) for i, v in enumerate(f))
    g = B.mrem_rotary_frequencies(64, scaling=B.MREM_ROTARY_LINEAR, factor=8.0).tolist()
    assert all(math.isclose(8 * v, w, rel_tol=1e-14) for v, w in zip(g, f))
    # in a larger base the slowest pair turns `factor` times slower, the fastest as before
    g = B.mrem_rotary_frequencies(64, scaling=B.MREM_ROTARY_BASE, factor=8.0).tolist()
    assert g[0] == 1.0 and math.isclose(8 * g[-1], f[-1], rel_tol=1e-12)
    # bands: 32 rotations or more over the trained positions stay, one or less is divided, monotone between
    g = B.mrem_rotary_frequencies(64, scaling=B.MREM_ROTARY_BANDS, factor=8.0, trained=4096.0, fast=32.0, slow=1.0).tolist()
    for v, w in zip(g, f):
        turns = 4096 * w / (2 * math.pi)
        if turns >= 32:
            assert v == w
        elif turns <= 1:
            assert math.isclose(8 * v, w, rel_tol=1e-14)
        else:
            assert w / 8 < v < w
    assert any(v == w for v, w in zip(g, f)) and any(math.isclose(8 * v, w) for v, w in zip(g, f))
    assert B.mrem_rotary_frequencies(2, scaling=B.MREM_ROTARY_BASE, factor=8.0).tolist() == [1.0]
    for bad, status in [(dict(rotary_dim=0), B.MREM_EINVAL), (dict(rotary_dim=7), B.MREM_ESHAPE), (dict(scaling=4), B.MREM_EINVAL), (dict(base=0.0), B.MREM_EINVAL),
                        (dict(base=math.inf), B.MREM_EINVAL), (dict(scaling=1, factor=-1.0), B.MREM_EINVAL), (dict(scaling=3, fast=1.0), B.MREM_EINVAL),
                        (dict(scaling=3, trained=math.nan), B.MREM_EINVAL)]:
        with pytest.raises(B.MremError) as e:
            B.mrem_rotary_frequencies(**{"rotary_dim": 64, **bad})
        assert e.value.status == status, bad


def test_rotary_refusals(B):
    good = dict(x=FAKE, y=FAKE, dtype=0, rows=4, heads=2, dim=64, ld_x=128, ld_y=128, r=64, inter=0, amp=1.0, freq=FAKE, pos=None, seq=4)
    bad = [(dict(x=None), "x"), (dict(y=ctypes.c_void_p(0x1008)), "y"), (dict(dtype=2), "dtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"),
           (dict(heads=0), "heads"), (dict(dim=0, r=2), "head_dim"), (dict(dim=513), "head_dim"), (dict(r=66), "rotary_dim"), (dict(r=63), "rotary_dim"),
           (dict(r=0), "rotary_dim"), (dict(ld_x=127), "stride"), (dict(ld_y=127), "stride"), (dict(ld_y=136), "in place"), (dict(inter=2), "interleaved"),
           (dict(freq=None), "freq"), (dict(freq=ctypes.c_void_p(0x1004)), "freq"), (dict(pos=ctypes.c_void_p(0x1002)), "positions"), (dict(seq=0), "seq")]
    for fn in (B._lib.mrem_rotary_forward, B._lib.mrem_rotary_backward):
        for change, word in bad:
            assert fn(*{**good, **change}.values(), None) in (B.MREM_EINVAL, B.MREM_ESHAPE) and word in B.mrem_last_error(), change
        assert fn(*{**good, "rows": 0, "x": None, "y": None}.values(), None) == B.MREM_OK


def attention_cfg(B, **change):
    return B.mrem_attention_config(**{**dict(dtype=0, batch=2, q_heads=4, kv_heads=2, head_dim=64, causal=1, window=0, scale=0.125, q_rows=8, k_rows=8,
                                             ld_q=256, ld_k=128, ld_v=128, ld_out=256), **change})


def test_attention_refusals(B):
    def forward(cfg, q=FAKE, k=FAKE, v=FAKE, qs=FAKE, ks=FAKE, ql=None, kl=None, out=FAKE, lse=FAKE, ws=FAKE, n=1 << 40):
        return B._lib.mrem_attention_forward(ctypes.byref(cfg), q, k, v, qs, ks, ql, kl, out, lse, ws, n, None)

    def backward(cfg, q=FAKE, k=FAKE, v=FAKE, qs=FAKE, ks=FAKE, ql=None, kl=None, out=FAKE, lse=FAKE, ws=FAKE, n=1 << 40, do=FAKE, dq=FAKE, dk=FAKE, dv=FAKE):
        return B._lib.mrem_attention_backward(ctypes.byref(cfg), q, k, v, out, lse, do, qs, ks, ql, kl, dq, dk, dv, ws, n, None)

    shapes = [dict(dtype=2), dict(head_dim=96), dict(head_dim=0), dict(kv_heads=0), dict(kv_heads=3), dict(q_heads=0), dict(batch=0), dict(causal=2), dict(window=-1),
              dict(causal=0, window=5), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(q_rows=-1), dict(q_rows=1 << 31), dict(k_rows=1 << 31),
              dict(q_rows=1 << 30), dict(ld_q=255), dict(ld_q=248), dict(ld_k=120), dict(ld_v=136 + 4), dict(ld_out=-256), dict(ld_v=(1 << 21) + 8), dict(batch=1 << 20, kv_heads=64, q_heads=64, ld_q=4096, ld_k=4096, ld_v=4096, ld_out=4096)]
    odd = ctypes.c_void_p(0x1008)
    for fn in (forward, backward):
        for change in shapes:
            assert fn(attention_cfg(B, **change)) in (B.MREM_EINVAL, B.MREM_ESHAPE) and B.mrem_last_error(), change
            assert B.mrem_attention_workspace_bytes(attention_cfg(B, **change), 1) == 0
        for name in ("q", "k", "v", "out", "lse"):
            for p in (None, odd):
                assert fn(attention_cfg(B), **{name: p}) == B.MREM_EINVAL and name in B.mrem_last_error(), name
        for name in ("qs", "ks", "ql", "kl"):
            assert fn(attention_cfg(B), **{name: ctypes.c_void_p(0x1002)}) == B.MREM_EINVAL
        assert fn(attention_cfg(B, q_rows=9), qs=None) == B.MREM_ESHAPE and "multiple of batch" in B.mrem_last_error()
        assert fn(attention_cfg(B, k_rows=9), ks=None) == B.MREM_ESHAPE
        assert fn(attention_cfg(B, q_rows=0, k_rows=0), q=None, k=None, v=None, out=None, lse=None) == B.MREM_OK
    for name in ("do", "dq", "dk", "dv"):
        for p in (None, odd):
            assert backward(attention_cfg(B), **{name: p}) == B.MREM_EINVAL
    need = B.mrem_attention_workspace_bytes(attention_cfg(B), 1)
    assert need >= 4 * 8 * 4
    assert backward(attention_cfg(B), n=4 * 8 * 4 - 1) == B.MREM_EWORKSPACE and "workspace" in B.mrem_last_error()
    assert backward(attention_cfg(B), ws=None) == B.MREM_EINVAL and backward(attention_cfg(B), ws=odd) == B.MREM_EINVAL
    # single tokens with many keys: parts of the keys meet in the workspace
    long = attention_cfg(B, batch=1, q_rows=1, k_rows=65536)
    need = B.mrem_attention_workspace_bytes(long, 0)
    assert need > 0 and forward(long, n=need - 1) == B.MREM_EWORKSPACE
    assert B._lib.mrem_attention_forward(None, *[FAKE] * 10, 0, None) == B.MREM_EINVAL


def test_attention_refuses_outputs_that_are_inputs(B):
    cfg, tensors = attention_cfg(B), [ctypes.c_void_p(0x10000 * (i + 1)) for i in range(9)]
    q, k, v, out, lse, do, dq, dk, dv = tensors
    for o, l in ((q, lse), (k, lse), (v, lse), (out, q), (out, out)):
        assert B._lib.mrem_attention_forward(ctypes.byref(cfg), q, k, v, FAKE, FAKE, None, None, o, l, FAKE, 1 << 40, None) == B.MREM_EINVAL
        assert "output" in B.mrem_last_error()
    for a, b, c in [(x, dk, dv) for x in tensors[:6]] + [(dq, x, dv) for x in tensors[:7]] + [(dq, dk, x) for x in tensors[:8]]:
        assert B._lib.mrem_attention_backward(ctypes.byref(cfg), q, k, v, out, lse, do, FAKE, FAKE, None, None, a, b, c, FAKE, 1 << 40, None) == B.MREM_EINVAL
        assert "output" in B.mrem_last_error()


def test_distill_refusals(B):
    good = dict(x=FAKE, dtype=0, rows=4, vocab=100, ld=100, top=FAKE, index=FAKE, k=8, tlse=None, temp=1.0, w=None, scale=1.0, lr=FAKE, lo=FAKE, g=None, ldg=100)
    odd = ctypes.c_void_p(0x1001)
    bad = [(dict(x=None), "logits"), (dict(x=odd), "logits"), (dict(dtype=5), "dtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 22), "rows"), (dict(vocab=0), "vocab"),
           (dict(vocab=(1 << 19) + 1, ld=1 << 20), "vocab"), (dict(ld=99), "stride"), (dict(g=FAKE, ldg=99), "stride"), (dict(k=0), "k must"), (dict(k=1025), "k must"),
           (dict(temp=0.0), "temperature"), (dict(temp=-1.0), "temperature"), (dict(temp=math.nan), "temperature"), (dict(scale=math.inf), "scale"), (dict(top=None), "top_logits"),
           (dict(index=None), "top_index"), (dict(lr=None), "loss_rows"), (dict(lr=odd), "misaligned"), (dict(tlse=odd), "misaligned"), (dict(g=odd), "misaligned"),
           (dict(g=FAKE, ldg=104), "in place")]
    for change, word in bad:
        assert B._lib.mrem_distill_loss(*{**good, **change}.values(), None) in (B.MREM_EINVAL, B.MREM_ESHAPE) and word in B.mrem_last_error(), change
    assert B._lib.mrem_distill_loss(*{**good, "rows": 0, "x": None, "top": None, "index": None, "lr": None, "lo": None}.values(), None) == B.MREM_OK


def test_binding_refuses_tensors_that_do_not_fit(B):
    import torch
    zeros = lambda *n, dtype=torch.float32: torch.zeros(*n, dtype=dtype)  # noqa: E731
    q, k = zeros(8, 4, 64), zeros(8, 2, 64)
    for bad in (dict(q=q[:, :, ::2]), dict(q=q.transpose(0, 1)), dict(q=q.double()), dict(k=k.bfloat16()), dict(k=k[:7]), dict(q=q.reshape(8, 256)), dict(q=q[:7])):
        t = {"q": q, "k": k, "v": k, "out": q, **bad}
        with pytest.raises(ValueError):
            B.attention_config(t["q"], t["k"], t["v"], t["out"], 2)
    cfg = B.attention_config(q, k, k, q, 2, causal=1)
    assert (cfg.q_rows, cfg.q_heads, cfg.kv_heads, cfg.head_dim, cfg.ld_q, cfg.ld_k) == (8, 4, 2, 64, 256, 128)
    lse, starts = zeros(4, 8), zeros(3, dtype=torch.int32)
    for bad in (dict(q=q[:7]), dict(lse=lse.t().contiguous()), dict(q_start=starts[:2]), dict(q_start=starts.long()), dict(q=zeros(8, 8, 64)[:, :4]), {}):  # the last: not on a GPU
        t = {"q": q, "q_start": starts, "lse": lse, **bad}
        with pytest.raises(ValueError):
            B.mrem_attention_forward(cfg, t["q"], k, k, t["q_start"], starts, None, None, q, t["lse"], None)
    x, z, i = zeros(4, 100), zeros(4, 8), zeros(4, 8, dtype=torch.int32)
    for bad in (dict(x=x.t()), dict(x=x.half()), dict(z=z[:3]), dict(i=i.long()), dict(g=x.bfloat16()), dict(g=x[:, :99]), {}):
        t = {"x": x, "z": z, "i": i, "g": None, **bad}
        with pytest.raises(ValueError):
            B.mrem_distill_loss(t["x"], t["z"], t["i"], None, 1.0, None, 1.0, zeros(4), None, t["g"])
    with pytest.raises(ValueError):
        B.mrem_rotary_forward(q, q[:7], 64, 0, 1.0, zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        B.mrem_rotary_forward(q, q, 64, 0, 1.0, zeros(32))
