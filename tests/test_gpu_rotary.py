"""mrem_rotary_forward and mrem_rotary_backward against the formula in 64 bits: layouts, parts of a head, odd sizes, scalings, strides,
far positions, in place, and the gradient as the transposed rotation."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2109_15082_amd import binding as B
    default = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)  # what other modules of a run have set is no matter here
    yield torch, B
    torch.set_default_dtype(default)


def turned(torch, x, pos, freq, r, interleaved, amplitude, sign):
    """(result, |x1| + |x2| of each value's pair) in 64 bits"""
    x = x.double()
    angle = pos.double()[:, None, None] * freq.to(x.device)
    c, s = amplitude * angle.cos(), sign * amplitude * angle.sin()
    y, size = x.clone(), torch.zeros_like(x)
    i, j = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., i], x[..., j]
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    size[..., i] = size[..., j] = a.abs() + b.abs()
    return y, size


def check(torch, got, want, size, amplitude):
    # one rounding to the type; sine, cosine and two products and a sum in 32 bits, each within a few of 2^-24 of |x1| + |x2|
    tol = torch.finfo(got.dtype).eps / 2 * want.abs() + 8 * 2.0 ** -24 * amplitude * size
    assert ((got.double() - want).abs() <= tol).all(), (got.double() - want).abs().sub(tol).max().item()


CASES = [  # rows, heads, head_dim, rotary_dim, heads between rows
    (1, 1, 2, 2, 1), (3, 5, 64, 64, 5), (17, 3, 128, 32, 7), (5, 2, 80, 20, 2), (2, 7, 33, 18, 8), (1500, 4, 64, 48, 12), (3, 1, 512, 512, 1), (1, 40, 128, 128, 48)]


@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows,heads,dim,r,apart", CASES)
def test_rotation_and_its_gradient(env, rows, heads, dim, r, apart, dtype, interleaved):
    torch, B = env
    dt = getattr(torch, dtype)
    g = torch.Generator().manual_seed(rows * 1000 + dim)
    x = torch.randn(rows, apart, dim, generator=g, dtype=torch.float64).to(dt).cuda()[:, :heads]
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (rows,), generator=g, dtype=torch.int64).to(torch.int32).cuda()
    pos[0] = 0
    freq = B.mrem_rotary_frequencies(r)
    for fn, sign in ((B.mrem_rotary_forward, 1), (B.mrem_rotary_backward, -1)):
        y = torch.full((rows, heads, dim), math.nan, dtype=dt, device="cuda")
        fn(x, y, r, interleaved, 1.25, freq.cuda(), pos)
        want, size = turned(torch, x, pos, freq, r, interleaved, 1.25, sign)
        check(torch, y, want, size, 1.25)
        assert torch.equal(y[..., r:], x[..., r:])
        # in place, between the neighbouring heads, which keep what they hold
        whole = torch.full((rows, apart, dim), 7.0, dtype=dt, device="cuda")
        part = whole[:, :heads]
        part.copy_(x)
        fn(part, part, r, interleaved, 1.25, freq.cuda(), pos)
        assert torch.equal(part, y) and (whole[:, heads:] == 7).all()


def test_positions_of_rows_of_sequences_and_no_rows(env):
    torch, B = env
    x = torch.randn(21, 2, 64, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    freq = B.mrem_rotary_frequencies(64).cuda()
    B.mrem_rotary_forward(x, y, 64, 0, 1.0, freq, None, 7)
    B.mrem_rotary_forward(x, z, 64, 0, 1.0, freq, torch.arange(21, device="cuda", dtype=torch.int32) % 7)
    assert torch.equal(y, z) and torch.equal(y[::7], x[::7])  # position 0 turns nothing
    B.mrem_rotary_forward(x[:0], y[:0], 64, 0, 1.0, freq)
    # what is not finite stays in its pair
    x[3, 1, 5] = math.inf
    B.mrem_rotary_forward(x, z, 64, 0, 1.0, freq, None, 7)
    bad = ~torch.isfinite(z)
    assert bad[3, 1, 5] and bad[3, 1, 37] and bad.sum() == 2


def test_more_rows_than_a_launch_has_blocks(env):
    torch, B = env
    n = (4 << 20) + 5
    x = torch.randn(n, 1, 2, device="cuda")
    y, freq = torch.empty_like(x), B.mrem_rotary_frequencies(2)
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    B.mrem_rotary_forward(x, y, 2, 1, 1.0, freq.cuda(), pos)
    check(torch, y, *turned(torch, x, pos, freq, 2, 1, 1.0, 1), 1.0)


def test_rows_far_apart(env):
    """offsets that pass 2^31 elements, in pieces and value by value"""
    torch, B = env
    rows, ld = 1100, 1 << 21
    whole, freq = torch.full((rows, ld), 7.0, device="cuda", dtype=torch.bfloat16), B.mrem_rotary_frequencies(64).cuda()
    x = torch.randn(rows, 2, 64, device="cuda").bfloat16()
    for odd in (0, 3):
        near = torch.empty(rows, 128 + odd, device="cuda", dtype=torch.bfloat16).as_strided((rows, 2, 64), (128 + odd, 64, 1))
        far = whole.as_strided((rows, 2, 64), (ld - odd, 64, 1))
        near.copy_(x)
        far.copy_(x)
        for y in (near, far):
            B.mrem_rotary_forward(y, y, 64, 0, 1.0, freq)
        assert torch.equal(far, near)
        far.fill_(7.0)
    assert (whole == 7).all()
