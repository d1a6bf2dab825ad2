"""mrem_attention_forward and mrem_attention_backward against the formulas in 64 bits, element by element.  Tolerances count roundings:
with u = half a step of the type (2^-8 for bf16, 2^-24 for fp32) a stored value is off by u of itself, and so is a probability or a score
gradient where it becomes an operand; a score of D products is off by less than D + 4 roundings of 32 bits of sum |q| |k|, and a
probability by that factor."""
import math

import pytest

pytestmark = pytest.mark.gpu
F32 = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2109_15082_amd import binding as B
    default = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)  # what other modules of a run have set is no matter here
    yield torch, B
    torch.set_default_dtype(default)


def case_tensors(torch, B, q_lens, k_lens, hq, hk, d, dtype, causal, window, layout, seed=0, scale=None, spare=3):
    """layout: packed (starts), padded (starts and lengths, as many rows a sequence), plain (neither: all lengths alike)"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = len(q_lens)
    dt = getattr(torch, dtype)
    dev = lambda v: torch.tensor(v, device="cuda", dtype=torch.int32)  # noqa: E731

    def place(lens):
        each = max(max(lens), 1) + (2 if layout == "padded" else 0)
        starts = [0]
        for m in lens:
            starts.append(starts[-1] + (m if layout == "packed" else each))
        return starts, starts[-1] + (spare if layout == "packed" else 0)

    (qs, q_rows), (ks, k_rows) = place(q_lens), place(k_lens)
    t = {"qs": qs, "ks": ks, "q_lens": q_lens, "k_lens": k_lens, "causal": causal, "window": window, "hq": hq, "hk": hk}
    # heads of other tensors between the rows, so that strides count; rows of no sequence hold NaN
    for name, rows, heads in (("q", q_rows, hq), ("k", k_rows, hk), ("v", k_rows, hk), ("dout", q_rows, hq)):
        whole = torch.full((rows, heads + (1 if name != "dout" else 0), d), math.nan, device="cuda", dtype=dt)
        t[name] = whole[:, :heads]
    for s0, m, s1, l in zip(qs, q_lens, ks, k_lens):
        for name, at, rows in (("q", s0, m), ("dout", s0, m), ("k", s1, l), ("v", s1, l)):
            part = t[name][at:at + rows]
            part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    t["out"], t["lse"] = torch.full((q_rows, hq, d), 3.0, device="cuda", dtype=dt), torch.full((hq, q_rows), 3.0, device="cuda")
    t["cfg"] = B.attention_config(t["q"], t["k"], t["v"], t["out"], n, causal, window, scale)
    t["where"] = {"packed": (dev(qs), dev(ks), None, None), "padded": (dev(qs), dev(ks), dev(q_lens), dev(k_lens)), "plain": (None,) * 4}[layout]
    t["ws"] = torch.full((B.mrem_attention_workspace_bytes(t["cfg"], 1) + 16,), 0xA5, device="cuda", dtype=torch.uint8)
    for name, like in (("dq", "q"), ("dk", "k"), ("dv", "v")):
        whole = torch.full((t[like].shape[0], t[like].shape[1] + 1, d), 3.0, device="cuda", dtype=dt)
        t[name] = whole[:, :-1]
    return t


def run(B, t, backward=True):
    B.mrem_attention_forward(t["cfg"], t["q"], t["k"], t["v"], *t["where"], t["out"], t["lse"], t["ws"])
    if backward:
        t["ws"].fill_(0x5A)
        B.mrem_attention_backward(t["cfg"], t["q"], t["k"], t["v"], t["out"], t["lse"], t["dout"], *t["where"], t["dq"], t["dk"], t["dv"], t["ws"])


def check(torch, t, backward=True):
    u = torch.finfo(t["q"].dtype).eps / 2
    scale, d, group = t["cfg"].scale, t["cfg"].head_dim, t["hq"] // t["hk"]
    used_q = torch.zeros(t["q"].shape[0], dtype=torch.bool, device="cuda")
    used_k = torch.zeros(t["k"].shape[0], dtype=torch.bool, device="cuda")

    def near(got, want, tol, what):
        # probabilities under 2^-126 are zero in 32 bits: at most some 1000 terms of them, times values under 1000
        off, tol = (got.double() - want).abs(), tol + 1e6 * 2.0 ** -126
        assert (off <= tol).all(), (what, (off - tol).max().item(), off.max().item(), want.abs().max().item())

    for s0, m, s1, l in zip(t["qs"], t["q_lens"], t["ks"], t["k_lens"]):
        used_q[s0:s0 + m] = True
        used_k[s1:s1 + l] = True
        p0 = torch.arange(m, device="cuda")[:, None] + l - m
        j = torch.arange(l, device="cuda")
        seen = torch.ones(m, l, dtype=torch.bool, device="cuda")
        if t["causal"]:
            seen &= j <= p0
        if t["window"]:
            seen &= j > p0 - t["window"]
        for c in range(t["hk"]):
            k, v = t["k"][s1:s1 + l, c].double(), t["v"][s1:s1 + l, c].double()
            sums = [torch.zeros(l, d, device="cuda", dtype=torch.float64) for _ in range(4)]  # dk, dv and their tolerances
            for h in range(c * group, (c + 1) * group):
                q, do = t["q"][s0:s0 + m, h].double(), t["dout"][s0:s0 + m, h].double()
                x = (scale * torch.mm(q, k.t())).masked_fill(~seen, -math.inf)
                # a score's error, as a factor of its exponential; twice: the row's sum is off by as much
                es = 2 * ((d + 4) * F32 * scale * torch.mm(q.abs(), k.abs().t()) * seen).amax(1, keepdim=True) + 64 * F32 if l else torch.zeros(m, 1, device="cuda", dtype=torch.float64)
                lse = torch.logsumexp(x, 1) if l else torch.full((m,), -math.inf, device="cuda", dtype=torch.float64)
                none = lse == -math.inf
                p = torch.exp(x - lse.masked_fill(none, 0)[:, None])
                o = torch.mm(p, v)
                err = (u + es + (l + 8) * F32)  # of a probability as an operand, and of sums over the keys
                eo = err * torch.mm(p, v.abs()) + u * o.abs()
                near(t["out"][s0:s0 + m, h], o, eo, "out")
                got = t["lse"][h, s0:s0 + m].double()
                assert torch.equal(got == -math.inf, none)
                near(got[~none], lse[~none], (es[:, 0] + (l + 8) * F32 + 4 * F32 * lse.abs())[~none], "lse")
                if not backward:
                    continue
                dp = torch.mm(do, v.t())
                delta = (p * dp).sum(1, keepdim=True)
                ds = p * (dp - delta) * scale
                el = es + 8 * F32 + 8 * F32 * lse.masked_fill(none, 0).abs()[:, None]  # of p = exp(s - lse)
                # dp and delta are sums of d products; delta comes from the stored out, in bf16 only where a row sees more than 128 keys
                ed = torch.mm(do.abs(), v.abs().t()) * (d + 4) * F32
                stored = ((eo + (d + 4) * F32 * o.abs()) * do.abs()).sum(1, keepdim=True)
                if t["q"].dtype == torch.bfloat16 and (l <= 128 or 0 < t["window"] <= 128):
                    stored = (el + (l + 8) * F32) * (stored + (p * (dp - delta)).abs().sum(1, keepdim=True)) + (d + 4) * F32 * (o.abs() * do.abs()).sum(1, keepdim=True)
                ed = ed + stored
                eds = (u + el) * ds.abs() + scale * p * ed * (1 + u)
                near(t["dq"][s0:s0 + m, h], torch.mm(ds, k), torch.mm(eds + l * F32 * ds.abs(), k.abs()) + u * torch.mm(ds, k).abs(), "dq")
                sums[0] += torch.mm(ds.t(), q)
                sums[1] += torch.mm(p.t(), do)
                sums[2] += torch.mm((eds + group * m * F32 * ds.abs()).t(), q.abs())
                sums[3] += torch.mm((p * (u + el + group * m * F32)).t(), do.abs())
            if backward:
                near(t["dk"][s1:s1 + l, c], sums[0], sums[2] + u * sums[0].abs(), "dk")
                near(t["dv"][s1:s1 + l, c], sums[1], sums[3] + u * sums[1].abs(), "dv")
    # rows of no sequence are as they were
    assert (t["out"][~used_q] == 3).all() and (t["lse"][:, ~used_q] == 3).all()
    if backward:
        assert (t["dq"][~used_q] == 3).all() and (t["dk"][~used_k] == 3).all() and (t["dv"][~used_k] == 3).all()
        for name in ("dq", "dk", "dv"):  # the heads between
            x = t[name]
            assert (x.as_strided((x.shape[0], x.shape[2]), (x.stride(0), 1), x.storage_offset() + x.shape[1] * x.shape[2]) == 3).all()


SHAPES = [  # q_lens, k_lens, query heads, key heads, head_dim
    ([1], [1], 1, 1, 32),
    ([1, 1, 1], [1, 65, 300], 8, 2, 64),
    ([1] * 5, [0, 33, 511, 129, 128], 8, 1, 128),
    ([3, 0, 70, 1], [3, 5, 70, 0], 2, 2, 64),
    ([31, 32, 33], [31, 32, 33], 3, 1, 32),
    ([127, 129, 5], [127, 129, 5], 4, 4, 128),
    ([40, 200], [7, 130], 6, 2, 64),        # more queries than keys: with a causal mask the first ones see nothing
    ([17, 4], [400, 260], 12, 3, 128),      # a piece of a prompt behind earlier keys
    ([257], [257], 5, 5, 64),
    ([2, 3, 1, 5], [2, 3, 1, 5], 2, 2, 128),  # gradients that are differences of few products
    ([40] * 150, [40] * 150, 2, 2, 64),      # short ones in blocks of 128 rows
]
MASKS = [(0, 0), (1, 0), (1, 1), (1, 50)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("causal,window", MASKS)
@pytest.mark.parametrize("q_lens,k_lens,hq,hk,d", SHAPES)
def test_lengths_heads_and_masks(env, q_lens, k_lens, hq, hk, d, causal, window, dtype):
    torch, B = env
    for layout in ("packed", "padded"):
        t = case_tensors(torch, B, q_lens, k_lens, hq, hk, d, dtype, causal, window, layout, seed=len(q_lens) + d)
        run(B, t)
        check(torch, t)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,length,hq,hk,d,causal", [(3, 48, 4, 2, 64, 1), (5, 1, 4, 4, 32, 0), (2, 130, 2, 1, 128, 1)])
def test_without_starts(env, n, length, hq, hk, d, causal, dtype):
    torch, B = env
    t = case_tensors(torch, B, [length] * n, [length] * n, hq, hk, d, dtype, causal, 0, "plain")
    run(B, t)
    check(torch, t)


@pytest.mark.parametrize("hq,hk,d,dtype", [(8, 2, 128, "bfloat16"), (2, 2, 64, "float32"), (16, 1, 32, "bfloat16")])
@pytest.mark.parametrize("window", [0, 700])
def test_single_tokens_with_keys_shared_out(env, hq, hk, d, dtype, window):
    torch, B = env
    t = case_tensors(torch, B, [1, 1, 1], [3001, 1, 2048], hq, hk, d, dtype, 1, window, "packed", spare=0)
    assert B.mrem_attention_workspace_bytes(t["cfg"], 0) > 0
    run(B, t, backward=False)
    check(torch, t, backward=False)


def test_many_sequences(env):
    """more than the 64 that a wavefront looks at together, empty ones among them"""
    torch, B = env
    lens = [(7 * i) % 23 if i % 5 else 0 for i in range(200)]
    t = case_tensors(torch, B, lens, lens, 2, 1, 64, "bfloat16", 1, 0, "packed")
    run(B, t)
    check(torch, t)


def test_long_and_large_scores(env):
    """scores far apart: maxima that rise from tile to tile, probabilities that underflow"""
    torch, B = env
    t = case_tensors(torch, B, [600], [600], 2, 1, 64, "bfloat16", 0, 0, "packed", scale=4.0)
    ramp = torch.linspace(0.01, 2.0, 600, device="cuda")[:, None, None]
    t["k"][:600].mul_(ramp)
    run(B, t)
    check(torch, t)


def test_one_visible_key_has_no_gradient_and_runs_repeat(env):
    torch, B = env
    t = case_tensors(torch, B, [70, 1], [70, 1], 4, 2, 64, "bfloat16", 1, 1, "packed")
    run(B, t)
    assert (t["dq"][:71] == 0).all() and (t["dk"][:71] == 0).all()
    for h in range(4):
        assert torch.equal(t["out"][:71, h], t["v"][:71, h // 2])
    for q_lens, window, d in (([70, 1], 1, 32), ([1, 1, 1], 0, 128)):
        t = case_tensors(torch, B, q_lens, q_lens, 16, 2, d, "float32", 1, window, "packed")
        run(B, t)
        assert (t["dq"][:sum(q_lens)] == 0).all() and (t["dk"][:sum(q_lens)] == 0).all()
    t = case_tensors(torch, B, [500, 33], [500, 33], 4, 2, 128, "bfloat16", 1, 0, "packed")
    run(B, t)
    first = [t[n].clone() for n in ("out", "lse", "dq", "dk", "dv")]
    run(B, t)
    assert all(torch.equal(a, t[n]) for a, n in zip(first, ("out", "lse", "dq", "dk", "dv")))


def test_gradients_against_differences(env):
    """in fp32, along random directions: (L(x + e d) - L(x - e d)) / 2 e of L = out . dout, whose error is that of 32-bit sums / e plus e^2"""
    torch, B = env
    t = case_tensors(torch, B, [9, 40], [21, 40], 4, 2, 32, "float32", 1, 30, "packed")
    run(B, t)
    used = 49
    base = {n: t[n].clone() for n in "qkv"}
    g = torch.Generator(device="cuda").manual_seed(7)
    for name in "qkv":
        rows = 49 if name == "q" else 61
        direction = torch.randn(t[name][:rows].shape, generator=g, device="cuda")
        direction /= direction.norm()
        want = (t["d" + name][:rows].double() * direction.double()).sum().item()
        e, sides = 0.05, []
        for sign in (1, -1):
            t[name][:rows] = base[name][:rows] + sign * e * direction
            run(B, t, backward=False)
            sides.append((t["out"][:used].double() * t["dout"][:used].double()).sum().item())
        t[name][:rows] = base[name][:rows]
        # the third derivative along a unit direction is of order one here
        assert abs((sides[0] - sides[1]) / (2 * e) - want) < 2e-3 * max(1.0, abs(want)), name


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("q_lens,k_lens,hq,hk,d,window", [([150], [150], 4, 2, 64, 0), ([150], [150], 2, 2, 128, 40), ([1, 3], [700, 300], 8, 2, 128, 90), ([9000], [9000], 8, 8, 32, 33)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_not_finite_reaches_what_sees_it_only(env, q_lens, k_lens, hq, hk, d, window, bad, dtype):
    """one key, value, query and output gradient each: what does not see it gives what it gives without"""
    torch, B = env
    names = ("out", "lse", "dq", "dk", "dv")
    t = case_tensors(torch, B, q_lens, k_lens, hq, hk, d, dtype, 1, window, "packed")
    run(B, t)
    want = {n: t[n].clone() for n in names}
    off, q_at, k_at = k_lens[0] - q_lens[0], q_lens[0] // 2, (k_lens[0] - q_lens[0]) + q_lens[0] // 2
    token, key = torch.arange(t["q"].shape[0], device="cuda"), torch.arange(t["k"].shape[0], device="cuda")
    sees = (token < q_lens[0]) & (token + off >= k_at) & ((window == 0) | (token + off - (window or 0) < k_at))    # queries that see the key
    seen = (key < k_lens[0]) & (key <= q_at + off) & ((window == 0) | (key > q_at + off - (window or 0)))          # keys that the query sees
    # rows formed again do without one rounding of their operands: as far off as the module's tests allow, element by element
    tol = 2e-2 if dtype == "bfloat16" else 1e-4
    close = lambda a, b: ((a.float() - b.float()).abs() <= tol * (b.float().abs() + b.float().abs().max())).all()  # noqa: E731
    for name, at in (("v", k_at), ("k", k_at), ("q", q_at), ("dout", q_at)):
        kept = t[name][at, 0].clone()
        t[name][at, 0, 3] = bad
        run(B, t)
        t[name][at, 0] = kept
        heads = hq // hk if name in ("k", "v") else 1
        hit = sees if name in ("k", "v") else token == q_at                                       # rows of these heads
        # the queries' side: what the poisoned heads' other rows, and all other heads, give
        for n in ("out", "dq"):
            clean = torch.ones(t[n].shape[:2], dtype=torch.bool, device="cuda")
            clean[:, :heads] = ~hit[:, None]
            assert torch.isfinite(t[n].float()[clean]).all() and close(t[n][clean], want[n][clean]), (name, n)
        # the keys' side: those that no hit query sees
        reached = seen if name in ("q", "dout") else torch.zeros_like(key, dtype=torch.bool)
        if name in ("k", "v"):
            first, last = int(token[sees].min()) if sees.any() else 0, int(token[sees].max()) if sees.any() else -1
            reached = (key < k_lens[0]) & (key <= last + off) & ((window == 0) | (key > first + off - (window or 0))) & bool(sees.any())
        for n in ("dk", "dv"):
            clean = torch.ones(t[n].shape[:2], dtype=torch.bool, device="cuda")
            clean[:, 0] = ~reached
            assert torch.isfinite(t[n].float()[clean]).all() and close(t[n][clean], want[n][clean]), (name, n)
        # and it does arrive
        if name == "v":
            assert not torch.isfinite(t["out"][hit][:, :heads, 3].float()).any()
        if name == "dout":
            assert not torch.isfinite(t["dv"][seen][:, 0, 3].float()).any()
    run(B, t)
    assert all(torch.equal(t[n], want[n]) for n in names)


def test_no_sequence_has_rows(env):
    torch, B = env
    t = case_tensors(torch, B, [0, 0], [0, 0], 2, 1, 64, "bfloat16", 1, 0, "packed")
    run(B, t)
    check(torch, t)
    t = case_tensors(torch, B, [0], [5], 2, 1, 64, "bfloat16", 1, 0, "packed", spare=0)
    assert t["q"].shape[0] == 0
    run(B, t)
    assert (t["dk"][:5] == 0).all() and (t["dv"][:5] == 0).all()
    t = case_tensors(torch, B, [5], [0], 2, 1, 64, "bfloat16", 0, 0, "packed", spare=0)
    assert t["k"].shape[0] == 0
    run(B, t)
    assert (t["out"] == 0).all() and (t["lse"] == -math.inf).all() and (t["dq"] == 0).all()


def test_starts_and_lengths_beyond_the_rows_are_cut(env):
    torch, B = env
    t = case_tensors(torch, B, [20, 30], [20, 30], 2, 1, 64, "bfloat16", 1, 0, "packed", spare=0)
    run(B, t)
    want = [t[n].clone() for n in ("out", "lse", "dq", "dk", "dv")]
    starts = torch.tensor([-5, 20, 1 << 30], device="cuda", dtype=torch.int32)
    lens = torch.tensor([1 << 30, 1 << 30], device="cuda", dtype=torch.int32)
    t["where"] = (starts, starts, lens, lens)
    run(B, t)
    assert all(torch.equal(a, t[n]) for a, n in zip(want, ("out", "lse", "dq", "dk", "dv")))


def test_captured_and_replayed_on_another_stream(env):
    torch, B = env
    t = case_tensors(torch, B, [1, 90, 200], [2500, 90, 200], 4, 2, 64, "bfloat16", 1, 0, "packed")
    run(B, t)
    torch.cuda.synchronize()
    names = ("out", "lse", "dq", "dk", "dv")
    want = [t[n].clone() for n in names]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run(B, t)
    for i in range(3):
        for n in names:
            t[n].fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, t[n]) for a, n in zip(want, names)), i
        t["q"].mul_(0.5)                      # other inputs, eagerly, between the replays
        run(B, t)
        want = [t[n].clone() for n in names]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_rows_as_far_apart_as_allowed(env, dtype):
    """queries, keys and values side by side in rows of 2^21 elements, and their gradients: offsets pass 2^31 elements and 2^32 bytes"""
    torch, B = env
    hq, hk, d, ld = 4, 2, 64, 1 << 21
    for q_lens, k_lens in (([700, 400], [600, 500]), ([1, 1], [900, 300])):
        t = case_tensors(torch, B, q_lens, k_lens, hq, hk, d, dtype, 1, 0, "packed", spare=0)
        rows, at = max(sum(q_lens), sum(k_lens)), {"q": 0, "k": hq + 1, "v": hq + hk + 2}
        heads = {"q": hq, "k": hk, "v": hk}
        for names, fill in ((("q", "k", "v"), math.nan), (("dq", "dk", "dv"), 3.0), (("out",), 3.0), (("dout",), math.nan)):
            whole = torch.full((rows, ld), fill, device="cuda", dtype=t["q"].dtype)
            for name in names:
                n = {"out": "q", "dout": "q"}.get(name, name[-1])
                new = whole.as_strided((t[name].shape[0], heads[n], d), (ld, d, 1), at[n] * d)
                new.copy_(t[name])
                t[name] = new
        t["cfg"] = B.attention_config(t["q"], t["k"], t["v"], t["out"], len(q_lens), 1, 0)
        assert t["cfg"].ld_q == t["cfg"].ld_v == t["cfg"].ld_out == ld
        run(B, t)
        check(torch, t)
