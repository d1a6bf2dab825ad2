"""The operators outside the module step as a training pass of a decoder student calls them, one after the other: projection, rotary
positions in place, attention with shared key heads over packed texts, output projection, logits, the loss on the teacher's top logits, and
back.  Against automatic differentiation of the same model in 64 bits; the projections are torch's."""
import pytest

pytestmark = pytest.mark.gpu

LENS, WIDTH, HQ, HK, D, ROTARY, VOCAB, K = [37, 1, 80, 12], 96, 4, 2, 32, 24, 611, 9
WINDOW, TEMPERATURE, SCALING = 30, 2.0, dict(scaling=3, factor=8.0, trained=64.0, fast=8.0, slow=1.0)


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2109_15082_amd import binding as B
    default = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)  # what other modules of a run have set is no matter here
    yield torch, B
    torch.set_default_dtype(default)


class Student:
    """The buffers of one pass, and its calls."""

    def __init__(self, torch, B, dtype):
        g = torch.Generator(device="cuda").manual_seed(11)
        self.torch, self.B, rows = torch, B, sum(LENS)
        rand = lambda *s, f=1.0: (f * torch.randn(s, generator=g, device="cuda")).to(dtype)  # noqa: E731
        self.x = rand(rows, WIDTH)
        self.w = {"qkv": rand((HQ + 2 * HK) * D, WIDTH, f=WIDTH ** -0.5), "o": rand(WIDTH, HQ * D, f=(HQ * D) ** -0.5), "head": rand(VOCAB, WIDTH, f=2 * WIDTH ** -0.5)}
        starts = [sum(LENS[:i]) for i in range(len(LENS) + 1)]
        self.starts = torch.tensor(starts, device="cuda", dtype=torch.int32)
        self.pos = torch.cat([torch.arange(n) for n in LENS]).to("cuda", torch.int32)
        self.freq = B.mrem_rotary_frequencies(ROTARY, **SCALING).cuda()
        self.index = torch.rand(rows, VOCAB, generator=g, device="cuda").argsort(1)[:, :K].int().contiguous()
        self.top = (3 + torch.randn(rows, K, generator=g, device="cuda")).contiguous()
        self.rest = (torch.logsumexp(self.top / TEMPERATURE, 1) + 0.2).contiguous()
        self.weight = (torch.rand(rows, generator=g, device="cuda") > 0.3).float()
        self.scale = TEMPERATURE ** 2 / rows
        empty = lambda *s: torch.empty(s, device="cuda", dtype=dtype)  # noqa: E731
        self.qkv, self.dqkv = empty(rows, HQ + 2 * HK, D), empty(rows, HQ + 2 * HK, D)
        self.out, self.lse = empty(rows, HQ, D), torch.empty(HQ, rows, device="cuda")
        self.logits = empty(rows, VOCAB)
        self.loss, self.loss_rows = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda")
        q, k, v = self.parts(self.qkv)
        self.cfg = B.attention_config(q, k, v, self.out, len(LENS), causal=1, window=WINDOW)
        self.ws = torch.empty(B.mrem_attention_workspace_bytes(self.cfg, 1), device="cuda", dtype=torch.uint8)
        self.grads = {n: torch.empty_like(w) for n, w in self.w.items()}

    @staticmethod
    def parts(t):
        return t[:, :HQ], t[:, HQ:HQ + HK], t[:, HQ + HK:]

    def run(self):
        torch, B, rows = self.torch, self.B, self.x.shape[0]
        turned, where = self.qkv[:, :HQ + HK], (self.starts, self.starts, None, None)
        torch.mm(self.x, self.w["qkv"].t(), out=self.qkv.view(rows, -1))
        B.mrem_rotary_forward(turned, turned, ROTARY, 0, 1.1, self.freq, self.pos)
        B.mrem_attention_forward(self.cfg, *self.parts(self.qkv), *where, self.out, self.lse, self.ws)
        hidden = torch.mm(self.out.view(rows, -1), self.w["o"].t())
        torch.mm(hidden, self.w["head"].t(), out=self.logits)
        # the gradient takes the logits' place
        B.mrem_distill_loss(self.logits, self.top, self.index, self.rest, TEMPERATURE, self.weight, self.scale, self.loss_rows, self.loss, self.logits)
        torch.mm(self.logits.t(), hidden, out=self.grads["head"])
        dhidden = torch.mm(self.logits, self.w["head"])
        torch.mm(dhidden.t(), self.out.view(rows, -1), out=self.grads["o"])
        dout = torch.mm(dhidden, self.w["o"]).view(rows, HQ, D)
        B.mrem_attention_backward(self.cfg, *self.parts(self.qkv), self.out, self.lse, dout, *where, *self.parts(self.dqkv), self.ws)
        turned = self.dqkv[:, :HQ + HK]
        B.mrem_rotary_backward(turned, turned, ROTARY, 0, 1.1, self.freq, self.pos)
        torch.mm(self.dqkv.view(rows, -1).t(), self.x, out=self.grads["qkv"])

    def oracle(self):
        """loss and gradients by automatic differentiation in 64 bits"""
        torch, rows = self.torch, self.x.shape[0]
        w = {n: t.double().requires_grad_() for n, t in self.w.items()}
        qkv = torch.mm(self.x.double(), w["qkv"].t()).view(rows, -1, D)
        turn = torch.polar(torch.tensor(1.1, dtype=torch.float64, device="cuda"), self.pos.double()[:, None, None] * self.freq)
        h = qkv[:, :HQ + HK]
        pair = torch.complex(h[..., :ROTARY // 2], h[..., ROTARY // 2:ROTARY]) * turn
        h = torch.cat((pair.real, pair.imag, h[..., ROTARY:]), -1)
        at, outs = 0, []
        for n in LENS:
            back = torch.arange(n, device="cuda")[:, None] - torch.arange(n, device="cuda")
            hidden = (back < 0) | (back >= WINDOW)
            heads = []
            for i in range(HQ):
                c = HQ + i // (HQ // HK)
                s = torch.mm(h[at:at + n, i], h[at:at + n, c].t()) * D ** -0.5
                heads.append(torch.mm(torch.softmax(s.masked_fill(hidden, float("-inf")), 1), qkv[at:at + n, c + HK]))
            outs.append(torch.stack(heads, 1))
            at += n
        logits = torch.mm(torch.mm(torch.cat(outs).reshape(rows, -1), w["o"].t()), w["head"].t())
        log_q = torch.log_softmax(logits / TEMPERATURE, 1)
        index = self.index.long()
        log_p = self.top.double() / TEMPERATURE - self.rest.double()[:, None]
        p = log_p.exp()
        rest = 1 - p.sum(1)
        others = torch.logsumexp(log_q.scatter(1, index, float("-inf")), 1)
        loss = ((p * (log_p - log_q.gather(1, index))).sum(1) + rest * (rest.log() - others)) * self.weight
        loss = loss.sum() * self.scale
        loss.backward()
        return loss.detach(), {n: t.grad for n, t in w.items()}


@pytest.mark.parametrize("dtype,tol", [("float32", 1e-4), ("bfloat16", 2e-2)])  # as the module step's gradients are held
def test_gradients_of_a_student(env, dtype, tol):
    torch, B = env
    s = Student(torch, B, getattr(torch, dtype))
    s.run()
    loss, grads = s.oracle()
    assert abs(s.loss.item() / loss.item() - 1) < tol
    for n, want in grads.items():
        off = (s.grads[n].double() - want).abs()
        assert off.norm() <= tol * want.norm() and (off <= tol * (want.abs() + want.abs().max())).all(), (n, (off.norm() / want.norm()).item())


def test_two_passes_at_once_and_a_captured_one(env):
    """two students on two streams, each with its own buffers, and the pass of a third one replayed between: the same bits as alone"""
    torch, B = env
    students = [Student(torch, B, torch.bfloat16) for _ in range(3)]
    for i, s in enumerate(students):
        s.x.mul_(1 + i)
        s.run()
    torch.cuda.synchronize()
    want = [{**{n: g.clone() for n, g in s.grads.items()}, "loss": s.loss.clone()} for s in students]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        students[2].run()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s in students:
            for g in (*s.grads.values(), s.loss):
                g.fill_(9)
        torch.cuda.synchronize()
        for s, st in zip(students, streams):
            with torch.cuda.stream(st):
                s.run()
        graph.replay()
        torch.cuda.synchronize()
        for s, w in zip(students, want):
            assert all(torch.equal(s.grads[n], w[n]) for n in s.grads) and torch.equal(s.loss, w["loss"])
