"""Operators that a training pass of a language-model student calls one after the other, as cases that can be timed and compared:
rotary positions between projection and attention, attention with its gradients, and the distillation loss on a teacher's top
logits with its gradient.

    kind       one pass                                                   returns
    rotary     mrem_rotary_forward, or with backward = 1 its gradient     the rotated heads
    attention  mrem_attention_forward                                     outputs, log-sum-exps
    train      mrem_attention_forward and mrem_attention_backward         the same, and the gradients of queries, keys and values
    distill    mrem_distill_loss                                          the loss, the rows' losses, the gradient of the logits

With `own` false, `run` computes the same from elementary operations in 32 bits (angles and the teacher's probabilities in 64).
Widths and heads are those of the repository's workloads (12 and 16 heads of 64) or generic ones (32 query heads on 8 key heads of 128).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
#: most (query, key, head) triples of a drawn attention case, and most logits of a drawn loss: those of the largest listed ones
MAX_SCORES = 2 * 32 * 4096 * 4096
MAX_LOGITS = 4096 * 128000
MAX_ROTATED = 8192 * 48 * 128


def _rotary(name, rows, seq, heads, dim, rotary_dim, layout, scaling, dtype, backward=0, far=0, ld_heads=0):
    return {"name": name, "kind": "rotary", "rows": rows, "seq": seq, "heads": heads, "dim": dim, "rotary_dim": rotary_dim, "layout": layout,
            "scaling": scaling, "dtype": dtype, "backward": backward, "far": far, "ld_heads": ld_heads or heads}


def _attention(name, kind, batch, q_len, k_len, q_heads, kv_heads, dim, dtype, causal=0, window=0, min_len=0, packed=0):
    """`q_len`, `k_len`: the longest sequence's; lengths are spread evenly over [min_len, k_len] (0: all are k_len).  packed: sequences
    follow each other without padding, five rows of no sequence behind the last one; otherwise each has k_len rows of its own."""
    return {"name": name, "kind": kind, "batch": batch, "q_len": q_len, "k_len": k_len, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "causal": causal, "window": window, "min_len": min_len, "packed": packed}


def _distill(name, rows, vocab, k, dtype, tail, temperature, weighted=0):
    return {"name": name, "kind": "distill", "rows": rows, "vocab": vocab, "k": k, "dtype": dtype, "tail": tail, "temperature": temperature,
            "weighted": weighted}


def listed():
    return [
        # sixteen tokens of as many requests, far into long contexts: the smallest call, where latency counts
        _rotary("rotary_16_tokens", 16, 1, 40, 128, 128, "half", "bands", "bf16", far=120000, ld_heads=48),
        # queries and keys of two sequences of 4096 tokens, where the projection left them beside the values
        _rotary("rotary_8192_packed", 8192, 4096, 40, 128, 128, "half", "base", "bf16", ld_heads=48),
        # the gradient at the repository's width, neighbouring pairs, a part of each head, in the check type
        _rotary("rotary_backward_part_f32", 5003, 5003, 12, 64, 20, "interleaved", "linear", "f32", backward=1),
        # one new token for each of sixteen sequences of up to 8192
        _attention("attention_single_tokens", "attention", 16, 1, 8192, 32, 8, 128, "bf16", causal=1, min_len=700),
        # the repository's reading-comprehension batches: 384 tokens, key padding, every token sees every valid one
        _attention("attention_1024_s384", "attention", 16, 384, 384, 16, 16, 64, "bf16", min_len=128),
        # a prompt of odd length
        _attention("attention_prompt_6001", "attention", 1, 6001, 6001, 32, 8, 128, "bf16", causal=1),
        # four short sentences in the check type
        _attention("train_sentences_f32", "train", 4, 77, 77, 12, 12, 64, "f32", min_len=9, packed=1),
        # texts of all lengths one behind the other, at the repository's width 768
        _attention("train_768_packed", "train", 24, 777, 777, 12, 12, 64, "bf16", causal=1, min_len=30, packed=1),
        # long texts, four query heads on a key head
        _attention("train_4096", "train", 2, 4096, 4096, 32, 8, 128, "bf16", causal=1),
        # a longer one that looks back 1024 tokens
        _attention("train_8192_window", "train", 1, 8192, 8192, 16, 4, 64, "bf16", causal=1, window=1024),
        # the vocabulary of the repository's kind of encoder, 4096 tokens as in its workloads
        _distill("distill_30522", 4096, 30522, 32, "bf16", 0, 2.0, weighted=1),
        # the largest vocabularies, with the teacher's remaining probability
        _distill("distill_128000", 4096, 128000, 64, "bf16", 1, 1.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: 1 .. 8192 tokens, heads of 32, 64 and 128 with 1 .. 8 query heads a key head, vocabularies of 1000 .. 128000."""
    kind = rng.choice(["rotary"] * 3 + ["attention"] * 4 + ["train"] * 5 + ["distill"] * 4)
    dim = rng.choice([32, 64, 64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "rotary":
        heads = rng.choice([4, 8, 12, 16, 20, 40])
        rows = _log_int(rng, 1, min(8192, MAX_ROTATED // (2 * heads * dim)))
        c = _rotary("", rows, max(1, rows // rng.choice([1, 2, 4])), heads, dim, rng.choice([dim, dim, dim // 2, dim // 4, 20]), rng.choice(["half", "interleaved"]),
                    rng.choice(["none", "linear", "base", "bands"]), dtype, rng.choice([0, 1]), rng.choice([0, 0, 30000]), heads + rng.choice([0, 0, 4]))
    elif kind == "distill":
        vocab = _log_int(rng, 1000, 128000)
        c = _distill("", _log_int(rng, 1, min(8192, MAX_LOGITS // vocab // 2)), vocab, _log_int(rng, 1, 256), dtype, rng.choice([0, 1]),
                     rng.choice([1.0, 1.0, 2.0, 4.0]), rng.choice([0, 1]))
    else:
        kv_heads, group = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 1, 2, 4, 8])
        k_len = _log_int(rng, 1, 4096 if dtype == "bf16" else 512)
        q_len = k_len if kind == "train" else rng.choice([1, 1, min(k_len, 7), k_len, k_len])
        batch = _log_int(rng, 1, max(1, min(64, MAX_SCORES // (4 * kv_heads * group * q_len * k_len), (1 << 28) // (kv_heads * group * dim * k_len))))
        causal = rng.choice([0, 1, 1])
        c = _attention("", kind, batch, q_len, k_len, kv_heads * group, kv_heads, dim, dtype, causal, rng.choice([0, 0, max(1, k_len // 3)]) if causal else 0,
                       rng.choice([0, max(1, k_len // 8)]), rng.choice([0, 1]) if q_len == k_len else 0)
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(DTYPES[dtype])


#: what scales the frequencies: (kind, factor, positions the model was trained on, rotations over them above which a pair stays, below which it is divided)
SCALINGS = {"none": (0, 1.0, 4096.0, 32.0, 1.0), "linear": (1, 4.0, 4096.0, 32.0, 1.0), "base": (2, 4.0, 4096.0, 32.0, 1.0), "bands": (3, 32.0, 4096.0, 32.0, 1.0)}


def _frequencies(rotary_dim, scaling, base=10000.0):
    """Radians a position of every pair."""
    kind, factor, trained, fast, slow = SCALINGS[scaling]
    if kind == 2 and rotary_dim > 2:
        base *= factor ** (rotary_dim / (rotary_dim - 2))
    f = base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / rotary_dim)
    if kind == 1:
        f = f / factor
    if kind == 3:
        keep = ((trained * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    return f


def _amplitude(scaling):
    return 0.1 * math.log(SCALINGS[scaling][1]) + 1 if scaling == "bands" else 1.0


def _lengths(case, seed):
    """k lengths and q lengths of the sequences, the same ones for every seed, in an order of the seed."""
    b, lo, hi = case["batch"], case["min_len"] or case["k_len"], case["k_len"]
    k = [hi - (hi - lo) * i // max(1, b - 1) for i in range(b)]
    order = torch.randperm(b, generator=torch.Generator().manual_seed(seed)).tolist()
    k = [k[i] for i in order]
    return k, k if case["q_len"] == case["k_len"] else [min(case["q_len"], n) for n in k]


def _starts(lens, rows_each):
    at = [0]
    for n in lens:
        at.append(at[-1] + (rows_each or n))
    return at


def _rows(case):
    """Rows of q and of k: the padded batch, or the packed sequences and five more."""
    if case["packed"]:
        n = sum(_lengths(case, 0)[0]) + 5
        return n, n
    return case["batch"] * case["q_len"], case["batch"] * case["k_len"]


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["kind"] == "rotary":
        rows, heads, dim = case["rows"], case["heads"], case["dim"]
        s["x"] = _randn(g, (rows, case["ld_heads"], dim), case["dtype"])[:, :heads]
        s["y"] = torch.zeros((rows, heads, dim), device="cuda", dtype=DTYPES[case["dtype"]])
        s["positions"] = torch.randint(0, case["far"], (rows,), generator=g, device="cuda", dtype=torch.int32) if case["far"] else None
        s["amplitude"] = _amplitude(case["scaling"])
        s["freq"] = _frequencies(case["rotary_dim"], case["scaling"]).cuda()
        return s
    if case["kind"] == "distill":
        rows, vocab, k = case["rows"], case["vocab"], case["k"]
        x = torch.randn((rows, vocab), generator=g, device="cuda", dtype=torch.float32) * 2
        # one listed token in each of k parts of the vocabulary, in another order for every row
        edges = torch.arange(k + 1, device="cuda") * vocab // k
        at = edges[:-1] + (torch.rand((rows, k), generator=g, device="cuda") * (edges[1:] - edges[:-1])).long().clamp(max=vocab - 1)
        at = at.gather(1, torch.rand((rows, k), generator=g, device="cuda").argsort(1))
        z = 6 + 3 * torch.randn((rows, k), generator=g, device="cuda").sort(1, descending=True).values
        # the student half agrees with the teacher
        x.scatter_(1, at, (0.5 * z + 0.5 * x.gather(1, at) + 2))
        s["x"] = x.to(DTYPES[case["dtype"]])
        s["index"], s["top"] = at.int(), z.contiguous()
        rest = torch.empty((rows, 1), device="cuda").uniform_(0.02, 0.3, generator=g)  # probability of all other tokens
        s["lse"] = (torch.logsumexp(z / case["temperature"], 1) - torch.log1p(-rest[:, 0])).contiguous() if case["tail"] else None
        s["weight"] = (torch.rand(rows, generator=g, device="cuda") > 0.2).float() if case["weighted"] else None
        s["scale"] = case["temperature"] ** 2 / rows
        s["loss_rows"], s["loss"] = torch.zeros(rows, device="cuda"), torch.zeros(1, device="cuda")
        s["grad"] = torch.zeros_like(s["x"])
        return s
    (qr, kr), (hq, hk, d) = _rows(case), (case["q_heads"], case["kv_heads"], case["dim"])
    k_len, q_len = _lengths(case, seed)
    dev = lambda v: torch.tensor(v, device="cuda", dtype=torch.int32)  # noqa: E731
    s["q_start"], s["k_start"] = dev(_starts(q_len, 0 if case["packed"] else case["q_len"])), dev(_starts(k_len, 0 if case["packed"] else case["k_len"]))
    s["q_lens"], s["k_lens"] = dev(q_len), dev(k_len)
    if case["q_len"] == case["k_len"]:  # training or a prompt: the three of them side by side, as a projection leaves them
        qkv = _randn(g, (qr, hq + 2 * hk, d), case["dtype"])
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    else:
        s["q"], s["k"], s["v"] = _randn(g, (qr, hq, d), case["dtype"]), _randn(g, (kr, hk, d), case["dtype"]), _randn(g, (kr, hk, d), case["dtype"])
    s["out"] = torch.zeros((qr, hq, d), device="cuda", dtype=DTYPES[case["dtype"]])
    s["lse"] = torch.zeros((hq, qr), device="cuda")
    if case["kind"] == "train":
        s["dout"] = _randn(g, (qr, hq, d), case["dtype"])
        dqkv = torch.zeros((qr, hq + 2 * hk, d), device="cuda", dtype=DTYPES[case["dtype"]])
        s["dq"], s["dk"], s["dv"] = dqkv[:, :hq], dqkv[:, hq:hq + hk], dqkv[:, hq + hk:]
    if own:
        from paper_2109_15082_amd import binding as B
        s["cfg"] = B.attention_config(s["q"], s["k"], s["v"], s["out"], case["batch"], causal=case["causal"], window=case["window"])
        s["workspace"] = torch.empty(B.mrem_attention_workspace_bytes(s["cfg"], case["kind"] == "train"), device="cuda", dtype=torch.uint8)
    return s


# ---- one pass ----------------------------------------------------------------


def run(s):
    if own:
        return _run_own(s)
    return {"rotary": _plain_rotary, "distill": _plain_distill}.get(s["kind"], _plain_attention)(s)


def _run_own(s):
    from paper_2109_15082_amd import binding as B
    if s["kind"] == "rotary":
        f = B.mrem_rotary_backward if s["backward"] else B.mrem_rotary_forward
        f(s["x"], s["y"], s["rotary_dim"], int(s["layout"] == "interleaved"), s["amplitude"], s["freq"], s["positions"], s["seq"])
        return s["y"]
    if s["kind"] == "distill":
        B.mrem_distill_loss(s["x"], s["top"], s["index"], s["lse"], s["temperature"], s["weight"], s["scale"], s["loss_rows"], s["loss"], s["grad"])
        return s["loss"], s["loss_rows"], s["grad"]
    where = (s["q_start"], s["k_start"], None if s["packed"] else s["q_lens"], None if s["packed"] else s["k_lens"])
    B.mrem_attention_forward(s["cfg"], s["q"], s["k"], s["v"], *where, s["out"], s["lse"], s["workspace"])
    if s["kind"] == "attention":
        return s["out"], s["lse"]
    B.mrem_attention_backward(s["cfg"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], *where, s["dq"], s["dk"], s["dv"], s["workspace"])
    return s["out"], s["lse"], s["dq"], s["dk"], s["dv"]


def _plain_rotary(s):
    x, r = s["x"], s["rotary_dim"]
    pos = s["positions"] if s["positions"] is not None else torch.arange(x.shape[0], device=x.device) % s["seq"]
    ang = pos.double()[:, None, None] * s["freq"]
    cos, sin = (torch.cos(ang) * s["amplitude"]).float(), (torch.sin(ang) * s["amplitude"]).float()
    if s["backward"]:
        sin = -sin
    part = x[..., :r].float()
    a, b = (part[..., 0::2], part[..., 1::2]) if s["layout"] == "interleaved" else (part[..., :r // 2], part[..., r // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    part = torch.stack((a, b), -1).flatten(-2) if s["layout"] == "interleaved" else torch.cat((a, b), -1)
    return torch.cat((part.to(x.dtype), x[..., r:]), -1)


def _pad(x, start, lens, most):
    """[rows, heads, dim] -> [batch, heads, most, dim] in 32 bits, zero beyond the lengths; and which rows those are."""
    at = torch.arange(most, device=x.device)
    valid = at < lens[:, None]
    rows = (start[:-1, None] + at).long().clamp(max=x.shape[0] - 1)
    return (x[rows].float() * valid[..., None, None]).transpose(1, 2).contiguous(), rows[valid], valid


def _unpad(v, rows, valid, like):
    """The inverse of _pad, zeros in rows of no sequence."""
    out = torch.zeros(like.shape, device=like.device, dtype=like.dtype)
    out[rows] = v.transpose(1, 2)[valid].to(like.dtype)
    return out


def _seen(s, q_most, k_most):
    i, j = torch.arange(q_most, device="cuda")[:, None], torch.arange(k_most, device="cuda")
    q_len, k_len = s["q_lens"][:, None, None].long(), s["k_lens"][:, None, None].long()
    seen = (j < k_len) & (i < q_len)
    if s["causal"]:
        seen = seen & (j <= i + k_len - q_len)
    if s["window"]:
        seen = seen & (j > i + k_len - q_len - s["window"])
    return seen[:, None]


def _plain_attention(s):
    group, scale = s["q_heads"] // s["kv_heads"], s["dim"] ** -0.5
    q, rows, valid = _pad(s["q"], s["q_start"], s["q_lens"], s["q_len"])
    k, k_rows, k_valid = _pad(s["k"], s["k_start"], s["k_lens"], s["k_len"])
    v, _, _ = _pad(s["v"], s["k_start"], s["k_lens"], s["k_len"])
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    x = (q @ k.transpose(2, 3).contiguous()) * scale
    x = x.masked_fill_(~_seen(s, s["q_len"], s["k_len"]), -math.inf)
    top = x.amax(3, keepdim=True)
    p = x.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(3, keepdim=True)
    lse = torch.zeros(s["lse"].shape, device="cuda")
    lse[:, rows] = (top + total.log())[..., 0].transpose(1, 2)[valid].t()
    p = p.div_(torch.where(total == 0, torch.ones_like(total), total))
    o = p @ v
    out = _unpad(o, rows, valid, s["out"])
    if s["kind"] == "attention":
        return out, lse
    do, _, _ = _pad(s["dout"], s["q_start"], s["q_lens"], s["q_len"])
    shared = lambda t: t.unflatten(1, (s["kv_heads"], group)).sum(2)  # noqa: E731
    dv = shared(p.transpose(2, 3).contiguous() @ do)
    dp = do @ v.transpose(2, 3).contiguous()
    ds = dp.sub_((p * dp).sum(3, keepdim=True)).mul_(p).mul_(scale)  # a row that sees one key: exactly zero
    dq = ds @ k
    dk = shared(ds.transpose(2, 3).contiguous() @ q)
    return out, lse, _unpad(dq, rows, valid, s["q"]), _unpad(dk, k_rows, k_valid, s["k"]), _unpad(dv, k_rows, k_valid, s["v"])


def _plain_distill(s):
    x, at, t = s["x"].float() / s["temperature"], s["index"].long(), s["temperature"]
    z = s["top"].double() / t
    top = x.amax(1, keepdim=True)
    e = (x - top).exp()
    total = e.sum(1, keepdim=True)
    log_q = (x.gather(1, at) - top).double() - total.double().log()
    if s["lse"] is None:
        log_p = z - z.amax(1, keepdim=True)
        log_p = log_p - log_p.exp().sum(1, keepdim=True).log()
    else:
        log_p = z - s["lse"].double()[:, None]
    p = log_p.exp()
    rows = (p * (log_p - log_q)).sum(1)
    q = e / total
    w = (s["weight"].double() if s["weight"] is not None else torch.ones_like(rows))
    if s["lse"] is None:
        grad = q * p.sum(1, keepdim=True).float()
    else:
        r = (1 - p.sum(1, keepdim=True)).clamp(min=0)
        others = q.scatter(1, at, 0.0).sum(1, keepdim=True).double()
        rows = rows + (r * (r.log() - others.log()))[:, 0]
        grad = (q * (1 - r / others).float())
    listed = log_q.exp() * (p.sum(1, keepdim=True) if s["lse"] is None else 1) - p
    grad = grad.scatter(1, at, listed.float()).mul_((w * s["scale"] / t).float()[:, None])
    rows = rows * (w != 0)
    return (s["scale"] * (w * rows).sum()).float().reshape(1), rows.float(), grad.to(s["x"].dtype)


# ---- what a pass cannot do without -------------------------------------------


def _pairs(case):
    """(query, key) pairs that are seen, over the sequences."""
    total = 0
    for k, q in zip(*_lengths(case, 0)):
        if not case["causal"]:
            total += q * k
            continue
        last = torch.arange(q, dtype=torch.int64) + k - q + 1  # keys up to the query's own
        total += int((last.clamp(max=case["window"]) if case["window"] else last).clamp(min=0).sum())
    return total


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rotary":
        n = case["rows"] * case["heads"]
        return {"bytes": 2 * n * case["dim"] * size + 4 * case["rows"] * (case["far"] > 0) + 4 * case["rotary_dim"], "flops": 3 * n * case["rotary_dim"]}
    if case["kind"] == "distill":
        n = case["rows"] * case["vocab"]
        return {"bytes": 2 * n * size + case["rows"] * (8 * case["k"] + 12), "flops": 6 * n}
    k_lens, q_lens = _lengths(case, 0)
    q, k, lse = sum(q_lens) * case["q_heads"] * case["dim"] * size, sum(k_lens) * case["kv_heads"] * case["dim"] * size, 4 * sum(q_lens) * case["q_heads"]
    flops = 4 * case["dim"] * case["q_heads"] * _pairs(case)
    if case["kind"] == "attention":
        return {"bytes": 2 * q + 2 * k + lse, "flops": flops}
    return {"bytes": 4 * q + 4 * k + lse, "flops": 3.5 * flops}  # two products forward, five backward


# ---- the definitions in 64 bits ----------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        x, r = s["x"].double(), case["rotary_dim"]
        pos = torch.arange(case["rows"], device="cuda") % case["seq"] if s["positions"] is None else s["positions"]
        turn = torch.polar(torch.full((case["rows"], 1, r // 2), s["amplitude"], device="cuda", dtype=torch.float64), torch.outer(pos.double(), s["freq"])[:, None])
        if case["backward"]:
            turn = turn.conj()
        shape = (r // 2, 2) if case["layout"] == "interleaved" else (2, r // 2)
        pair = x[..., :r].unflatten(-1, shape)
        pair = pair if case["layout"] == "interleaved" else pair.transpose(-1, -2)
        pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        x[..., :r] = (pair if case["layout"] == "interleaved" else pair.transpose(-1, -2)).flatten(-2)
        return x
    if case["kind"] == "distill":
        rows, grad = torch.empty(case["rows"], device="cuda", dtype=torch.float64), torch.empty(s["x"].shape, device="cuda", dtype=torch.float64)
        w = torch.ones_like(rows) if s["weight"] is None else s["weight"].double()
        for a in range(0, case["rows"], 512):  # the loss's own derivative, by its terms' formulas
            b = slice(a, a + 512)
            x, at = s["x"][b].double() / case["temperature"], s["index"][b].long()
            log_q = torch.log_softmax(x, 1)
            z = s["top"][b].double() / case["temperature"]
            log_p = torch.log_softmax(z, 1) if s["lse"] is None else z - s["lse"][b].double()[:, None]
            p = log_p.exp()
            rows[b] = (p * log_p).sum(1) - (p * log_q.gather(1, at)).sum(1)
            g = p.sum(1, keepdim=True) * log_q.exp()
            g.scatter_add_(1, at, -p)
            if s["lse"] is not None:
                left = -torch.expm1(torch.logsumexp(log_p, 1))
                log_others = torch.logsumexp(log_q.scatter(1, at, -math.inf), 1)
                rows[b] += left * (left.log() - log_others)
                g += left[:, None] * log_q.exp()
                g -= left[:, None] * (log_q.scatter(1, at, -math.inf) - log_others[:, None]).exp()
            grad[b] = g * (w[b] * s["scale"] / case["temperature"])[:, None]
        rows = torch.where(w == 0, torch.zeros_like(rows), rows)
        return (torch.dot(w, rows) * s["scale"]).reshape(1), rows, grad
    q, k, v = (s[n].double() for n in "qkv")
    out, lse = torch.zeros(s["out"].shape, device="cuda", dtype=torch.float64), torch.zeros(s["lse"].shape, device="cuda", dtype=torch.float64)
    train = case["kind"] == "train"
    dq, dk, dv = (torch.zeros(t.shape, device="cuda", dtype=torch.float64) for t in (q, k, v))
    group = case["q_heads"] // case["kv_heads"]
    for b, (n, m) in enumerate(zip(s["q_lens"].tolist(), s["k_lens"].tolist())):
        i, j = int(s["q_start"][b]), int(s["k_start"][b])
        far = (torch.arange(n, device="cuda")[:, None] + (m - n)) - torch.arange(m, device="cuda")  # how far back a key lies
        hidden = (far < 0 if case["causal"] else torch.zeros_like(far, dtype=torch.bool)) | ((far >= case["window"]) if case["window"] else False)
        for h in range(case["q_heads"]):
            c = h // group
            a = torch.mm(q[i:i + n, h], k[j:j + m, c].t()) / math.sqrt(case["dim"])
            a = a.masked_fill(hidden, -math.inf)
            lse[h, i:i + n] = torch.logsumexp(a, 1)
            p = torch.exp(a - torch.where(lse[h, i:i + n] == -math.inf, torch.zeros_like(lse[h, i:i + n]), lse[h, i:i + n])[:, None])
            out[i:i + n, h] = torch.mm(p, v[j:j + m, c])
            if train:
                do = s["dout"][i:i + n, h].double()
                dv[j:j + m, c] += torch.mm(p.t(), do)
                dp = torch.mm(do, v[j:j + m, c].t())
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(case["dim"])
                dq[i:i + n, h] = torch.mm(ds, k[j:j + m, c])
                dk[j:j + m, c] += torch.mm(ds.t(), q[i:i + n, h])
    return (out, lse, dq, dk, dv) if train else (out, lse)
