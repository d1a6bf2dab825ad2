"""mrem_distill_loss against the loss's formula and its gradient in 64 bits.  In 32 bits are only an exponential (its argument is off by
two roundings of itself) and the up to 160 additions that lead to a row's sums; what is listed is formed in 64."""
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


def inputs(torch, rows, vocab, k, dtype, tail, seed=0, apart=0, near=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = 3 * torch.randn(rows, vocab + apart, generator=g, device="cuda")
    at = torch.rand(rows, vocab, generator=g, device="cuda").argsort(1)[:, :k] if vocab <= 5000 else torch.randint(0, vocab // k, (rows, k), generator=g, device="cuda") + torch.arange(k, device="cuda") * (vocab // k)
    n = at.shape[1]
    z = 4 + 2 * torch.randn(rows, n, generator=g, device="cuda")
    if near:  # a student that agrees with its teacher
        x.scatter_(1, at, z + 4)
    if n < k:  # entries that are not there
        at = torch.cat((at, torch.full((rows, k - n), -1, device="cuda")), 1)
        z = torch.cat((z, torch.full((rows, k - n), math.nan, device="cuda")), 1)
    s = {"x": x.to(getattr(torch, dtype))[:, :vocab], "at": at.int().contiguous(), "z": z.contiguous(), "lse": None, "w": None}
    if tail:
        s["lse"] = None if n == 0 else torch.logsumexp(torch.where(at < 0, -math.inf, z).double(), 1).add(torch.rand(rows, generator=g, device="cuda") + 0.01).float()
    return s


def expected(torch, s, temperature, scale):
    """loss rows and gradient in 64 bits, and their tolerances"""
    x = s["x"].double() / temperature
    rows, vocab = x.shape
    there = (s["at"] >= 0) & (s["at"] < vocab)
    at = torch.where(there, s["at"], 0).long()
    z = torch.where(there, s["z"].double() / temperature, -math.inf)
    log_total = torch.logsumexp(z, 1, keepdim=True) if s["lse"] is None else s["lse"].double()[:, None]
    log_p = torch.where(z == -math.inf, -math.inf, z - log_total)
    p = log_p.exp()
    listed = torch.zeros(rows, vocab, device="cuda", dtype=torch.int32).scatter_add_(1, at, there.int()) > 0
    target = torch.zeros(rows, vocab, device="cuda", dtype=torch.float64).scatter_add_(1, at, p)
    top = x.amax(1, keepdim=True)
    log_q = x - top - (x - top).exp().sum(1, keepdim=True).log()
    q = log_q.exp()
    mass = p.sum(1, keepdim=True)
    loss = torch.where(p > 0, p * (log_p - log_q.gather(1, at)), 0.0).sum(1)
    grad = mass * q - target
    rest = (1 - mass).clamp(min=0) if s["lse"] is not None else torch.zeros_like(mass)
    share = torch.where(listed, 0.0, q).sum(1, keepdim=True)
    loss = loss + torch.where(rest > 0, rest * (rest.log() - share.log()), 0.0)[:, 0]
    grad = grad + torch.where(rest > 0, rest * q - torch.where(listed, 0.0, rest * q / share), 0.0)
    w = torch.ones(rows, device="cuda", dtype=torch.float64) if s["w"] is None else s["w"].double()
    f = (w * scale / temperature)[:, None]
    # of a sum of exponentials: additions, and each term's argument
    e_all = (160 + 4 * (q * (x - top).abs().nan_to_num(posinf=0)).sum(1, keepdim=True)) * F32
    others = torch.where(listed, 0.0, q) / share.clamp(min=1e-300)
    e_rest = (160 + 4 * (others * (x - top).abs().nan_to_num(posinf=0)).sum(1, keepdim=True)) * F32
    tol_loss = ((mass + rest) * e_all + rest * e_rest)[:, 0] + F32 * loss.abs() + 1e-14
    u = torch.finfo(s["x"].dtype).eps / 2
    e_q = e_all + (8 + 4 * (x - top).abs().nan_to_num(posinf=0)) * F32
    tol_grad = f.abs() * (q * ((mass + rest) * e_q) + torch.where(listed, 0.0, rest * others * (e_q + e_rest))) + u * (grad * f).abs() + 1e-38
    dead = (w == 0)
    return torch.where(dead, 0.0, loss), torch.where(dead[:, None], 0.0, grad * f), tol_loss, tol_grad, w


def run(torch, B, s, temperature=1.0, scale=1.0, apart=0, with_grad=True):
    rows, vocab = s["x"].shape
    loss_rows, loss = torch.full((rows,), math.nan, device="cuda"), torch.full((1,), math.nan, device="cuda")
    grad = torch.full((rows, vocab + apart), 7.0, device="cuda", dtype=s["x"].dtype)[:, :vocab] if with_grad else None
    B.mrem_distill_loss(s["x"], s["z"], s["at"], s["lse"], temperature, s["w"], scale, loss_rows, loss, grad)
    return loss, loss_rows, grad


def check(torch, s, got, temperature=1.0, scale=1.0):
    loss, rows, grad = got
    want, want_grad, tol_loss, tol_grad, w = expected(torch, s, temperature, scale)
    off = torch.where(rows == want, 0.0, (rows.double() - want).abs())  # (infinite where all tokens are listed and the teacher expects others)
    assert (off <= tol_loss).all(), (off - tol_loss).max().item()
    total = (w * want).sum() * scale
    assert loss == total or abs(loss.double() - total) <= (w.abs() * tol_loss).sum() * abs(scale) + 2 * F32 * total.abs()
    if grad is not None:
        off = (grad.double() - want_grad).abs()
        assert (off <= tol_grad).all(), (off - tol_grad).max().item()


SIZES = [(1, 1, 1), (3, 2, 1), (5, 7, 9), (4, 33, 5), (7, 1003, 17), (3, 8192, 64), (3, 8200, 64), (2, 16391, 300), (2, 30522, 1024), (2, 65537, 3), (2, 131072, 33), (2, 131079, 100)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("rows,vocab,k", SIZES)
def test_loss_and_gradient(env, rows, vocab, k, tail, dtype):
    torch, B = env
    for seed, (temperature, scale, apart) in enumerate([(1.0, 1.0, 0), (2.5, -0.75, 3)]):
        s = inputs(torch, rows, vocab, k, dtype, tail, seed, apart, near=bool(seed))
        check(torch, s, run(torch, B, s, temperature, scale, 2 * apart), temperature, scale)


def test_the_largest_vocabulary(env):
    torch, B = env
    s = inputs(torch, 1, 1 << 19, 1024, "float32", 1)
    check(torch, s, run(torch, B, s))


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("tail", [0, 1])
def test_entries_that_are_missing_or_listed_twice(env, tail, dtype):
    torch, B = env
    s = inputs(torch, 6, 500, 40, dtype, tail)
    s["at"][0, 3], s["at"][0, 9], s["at"][0, 11] = s["at"][0, 2], s["at"][0, 2], s["at"][0, 30]
    s["at"][1, :] = s["at"][1, 0]
    s["at"][2, ::2] = -1
    s["at"][3, 5], s["at"][3, 6] = 500, 2147483647
    s["at"][4, :] = -7                       # none is there
    s["z"][5, 4] = -math.inf                 # probability zero
    if tail:
        s["lse"] += 4                        # the masses of repeated entries stay below one
    check(torch, s, run(torch, B, s))


def test_masked_logits_and_rows_without_weight(env):
    torch, B = env
    s = inputs(torch, 8, 777, 12, "bfloat16", 1)
    hidden = torch.rand(8, 777, device="cuda") < 0.5
    hidden.scatter_(1, s["at"].long(), False)
    s["x"][hidden] = -math.inf               # tokens that the student cannot give
    s["x"][2], s["z"][2] = math.nan, math.nan
    s["w"] = torch.rand(8, device="cuda") + 0.5
    s["w"][2] = 0
    got = run(torch, B, s, 2.0, 3.0)
    assert got[1][2] == 0 and (got[2][2] == 0).all()
    s["x"][2], s["z"][2] = 0.0, 0.0          # what the oracle computes there is put to zero by the weight
    check(torch, s, got, 2.0, 3.0)
    # the student excludes what the teacher expects: an infinite loss, and no NaN in other rows
    s["x"][1, s["at"][1, 0].long()] = -math.inf
    s["x"][3, 5] = math.nan
    got = run(torch, B, s, 2.0, 3.0)
    assert got[1][1] == math.inf and torch.isnan(got[1][3]) and torch.isfinite(got[1][[0, 2, 4, 5, 6, 7]]).all()


@pytest.mark.parametrize("vocab", [1003, 40000, 140001])
def test_in_place_and_without_gradient_and_repeated(env, vocab):
    torch, B = env
    s = inputs(torch, 5, vocab, 50, "bfloat16", 1, apart=5)
    loss, rows, grad = run(torch, B, s)
    again = run(torch, B, s)
    assert torch.equal(loss, again[0]) and torch.equal(rows, again[1]) and torch.equal(grad, again[2])
    plain = run(torch, B, s, with_grad=False)
    assert torch.equal(loss, plain[0]) and torch.equal(rows, plain[1])
    B.mrem_distill_loss(s["x"], s["z"], s["at"], s["lse"], 1.0, None, 1.0, rows, None, s["x"])
    assert torch.equal(s["x"], grad)


def test_no_rows_and_replays(env):
    torch, B = env
    loss = torch.full((1,), 5.0, device="cuda")
    e = torch.empty(0, 8, device="cuda")
    B.mrem_distill_loss(torch.empty(0, 100, device="cuda"), e, e.int(), None, 1.0, None, 1.0, torch.empty(0, device="cuda"), loss, None)
    assert loss.item() == 0
    s = inputs(torch, 9, 5000, 20, "bfloat16", 1)
    rows, grad = torch.empty(9, device="cuda"), torch.empty_like(s["x"])
    call = lambda: B.mrem_distill_loss(s["x"], s["z"], s["at"], s["lse"], 1.0, None, 1.0, rows, loss, grad)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        s["x"].mul_(0.7)
        call()
        want = loss.clone(), rows.clone(), grad.clone()
        for t in (loss, rows, grad):
            t.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(rows, want[1]) and torch.equal(grad, want[2])


@pytest.mark.parametrize("vocab", [1003, 140001])
def test_rows_far_apart(env, vocab):
    """offsets that pass 2^31 elements, of rows that a block holds and of rows that it reads twice"""
    torch, B = env
    rows, ld = 600, 1 << 22
    s = inputs(torch, rows, vocab, 9, "bfloat16", 1)
    want = run(torch, B, s)
    near, far = s["x"], torch.full((rows, ld), math.nan, device="cuda", dtype=torch.bfloat16)
    s["x"] = far[:, 5:5 + vocab]
    s["x"].copy_(near)
    loss_rows, loss = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda")
    B.mrem_distill_loss(s["x"], s["z"], s["at"], s["lse"], 1.0, s["w"], 1.0, loss_rows, loss, s["x"])
    assert torch.equal(loss, want[0]) and torch.equal(loss_rows, want[1]) and torch.equal(s["x"], want[2])
    assert far[:, :5].isnan().all() and far[:, 5 + vocab:].isnan().all()
