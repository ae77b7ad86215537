"""spense_block_norm through the binding, against the formulas in 64 bits.

With u = 2^-24 a sum of squares passes at most 56 fp32 roundings on its way through a thread
(up to 40 terms), a wave (6) and the workgroup (16), half of which its root keeps; rsqrt,
weight, gate and scale add fewer than eight.  So t is within 40 u of its value, r within 40 u
(|alpha x| + |g t|), and n within what these errors make of it plus 40 u |n|; each rounded
output adds half a step of its type.
"""
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
TINY = 1e-38  # results in the denormal range are not looked at more closely


@pytest.fixture(scope="module")
def S():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_10445_amd as S
    return S


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def rand(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def formula(x, y, post, gate, alpha, w, eps):
    """(r, bound of r, n, bound of n) in float64."""
    d = lambda t: None if t is None else t.detach().cpu().double()  # noqa: E731
    x, y, post, gate, w = d(x), d(y), d(post), d(gate), d(w)
    if y is None:
        r, dr = x, torch.zeros_like(x)
    else:
        t = y if post is None else y / torch.sqrt(y.pow(2).mean(1, keepdim=True) + eps) * post
        t = t if gate is None else t * gate
        r, dr = alpha * x + t, 40 * U * ((alpha * x).abs() + t.abs())
    ms = r.pow(2).mean(1, keepdim=True)
    n = r / torch.sqrt(ms + eps) * (1 if w is None else w)
    norm = lambda v: v.pow(2).sum(1, keepdim=True).sqrt()  # noqa: E731
    inv = 1 / torch.sqrt(ms + eps)
    dn = (dr + r.abs() * norm(dr) / norm(r).clamp_min(1e-300)) * inv * (1 if w is None else w.abs()) + 40 * U * n.abs()
    return r, dr, n, dn


def decoded(q):
    return q.cpu().view(torch.float8_e4m3fn).double()


def check(o, r, dr, n, dn, xdt, ydt):
    if o.residual is not None:
        err = (o.residual.cpu().double() - r).abs()
        assert torch.all(err <= dr + HALF[xdt] * (r.abs() + dr) + TINY), float((err - dr).max())
    if o.normed is not None:
        err = (o.normed.cpu().double() - n).abs()
        assert torch.all(err <= dn + HALF[ydt] * (n.abs() + dn) + TINY), float((err - dn).max())
    if o.codes is not None:
        s = o.scales.cpu().double()
        want = n.abs().amax(1) / 448
        assert torch.all(((s - torch.where(want == 0, torch.ones_like(want), want)).abs())
                         <= dn.amax(1) / 448 + 2 * U * want + TINY)
        v, c = n / s[:, None], decoded(o.codes)
        step = torch.exp2(torch.floor(torch.log2(torch.maximum(v.abs(), c.abs()).clamp_min(2.0 ** -6))) - 3)
        assert torch.all((c - v).abs() <= step / 2 + dn / s[:, None] + 2 * U * v.abs() + TINY)


T = {"bf16": torch.bfloat16, "f32": torch.float32}
# vectors of 8 in one, two and four pieces a thread, single elements, rows of four passes
SIZES = [(1, 1), (3, 7), (2, 64), (5, 520), (64, 5120), (7, 4099), (3, 8200), (2, 16392), (2, 9001), (2, 33001), (1, 40000)]


@pytest.mark.parametrize("M,K", SIZES)
@pytest.mark.parametrize("xt,yt", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_sandwich(S, M, K, xt, yt):
    say(f"[norm] {xt} {yt} {M}x{K}")
    x, y = rand(1, M, K, dtype=T[xt], scale=3), rand(2, M, K, dtype=T[yt], scale=0.3)
    post, w = 1 + rand(3, K, scale=0.1), 1 + rand(4, K, scale=0.1)
    gate = rand(5, M, K, dtype=T[yt])
    if (M + K) % 2:
        post, w = post.bfloat16(), w.bfloat16()
        gate = gate[0].contiguous()
    o = S.block_norm(x.cuda(), y.cuda(), post_weight=post.cuda(), gate=gate.cuda(), residual_scale=0.75,
                     weight=w.cuda(), eps=1e-5, normed=True)
    torch.cuda.synchronize()
    check(o, *formula(x, y, post, gate, 0.75, w, 1e-5), T[xt], T[yt])
    if yt == "f32":  # the codes are those of the fp32 norm
        q, s = S.quantize_fp8(o.normed)
        assert torch.equal(q, o.codes) and torch.equal(s, o.scales)


@pytest.mark.parametrize("K", [48, 333, 5120])
@pytest.mark.parametrize("parts", ["x", "x w", "y", "y post", "y gate", "y w"])
def test_parts(S, K, parts):
    """Every optional operand alone, each output alone."""
    p, M = parts.split(), 6
    x = rand(11, M, K, dtype=torch.bfloat16)
    y = rand(12, M, K, dtype=torch.bfloat16) if "y" in p else None
    post = 1 + rand(13, K, scale=0.2) if "post" in p else None
    gate = rand(14, K, dtype=torch.bfloat16) if "gate" in p else None
    w = 1 + rand(15, K, scale=0.2) if "w" in p else None
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    ref = formula(x, y, post, gate, -1.5, w, 1e-6)
    kw = dict(post_weight=up(post), gate=up(gate), residual_scale=-1.5, weight=up(w))
    both = S.block_norm(up(x), up(y), normed=True, **kw)
    check(both, *ref, torch.bfloat16, torch.bfloat16)
    assert (both.residual is None) == (y is None)
    only_q = S.block_norm(up(x), up(y), **kw)
    only_n = S.block_norm(up(x), up(y), normed=True, quantize=False, **kw)
    assert torch.equal(only_q.codes, both.codes) and torch.equal(only_q.scales, both.scales) and only_q.normed is None
    assert torch.equal(only_n.normed, both.normed) and only_n.codes is None
    if y is not None:
        only_r = S.block_norm(up(x), up(y), quantize=False, **kw)
        assert torch.equal(only_r.residual, both.residual) and only_r.normed is None


@pytest.mark.parametrize("K,pitch", [(256, 264), (256, 272), (255, 301), (20000, 20001), (5120, 5128)])
def test_strides_and_in_place(S, K, pitch):
    """Rows inside wider buffers: the columns behind them stay as they were; r over x, n over y."""
    M = 5
    xw, yw = (rand(s, M, pitch, dtype=torch.bfloat16).cuda() for s in (21, 22))
    x0, y0 = xw.clone(), yw.clone()
    ref = S.block_norm(xw[:, :K].contiguous(), yw[:, :K].contiguous(), normed=True)
    qw = torch.full((M, pitch), 7, dtype=torch.uint8, device="cuda")
    o = S.block_norm(xw[:, :K], yw[:, :K], residual_out=xw[:, :K], normed_out=yw[:, :K], codes_out=qw[:, :K])
    torch.cuda.synchronize()
    # a row's sums are taken in another order on another path: fp32 roundings, seen as at most one step
    for a, b in ((o.residual, ref.residual), (o.normed, ref.normed)):
        assert torch.all((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 1e-30)
    assert torch.equal(xw[:, K:], x0[:, K:]) and torch.equal(yw[:, K:], y0[:, K:]) and torch.all(qw[:, K:] == 7)


@pytest.mark.parametrize("K", [40, 1000, 1003, 4096, 8192, 8200])
@pytest.mark.parametrize("wscale", [1.0, 1e-25, 1e22])
def test_many_rows_codes(S, K, wscale):
    """Codes of many rows are those that quantize_fp8 gives for the fp32 norm: ties, signed zeros, small
    values and scales far from 1 among them."""
    M = 600
    x = rand(51, M, K) * torch.exp(rand(52, M, K) * 3)  # many values far below the row's largest
    x[3, :7], x[4, 5] = -0.0, float("nan")
    x[7] = torch.round(x[7].clamp(-8, 8))
    w = (rand(53, K).abs() + 0.5) * wscale
    o = S.block_norm(x.cuda(), weight=w.cuda(), normed=True)
    q, s = S.quantize_fp8(o.normed)
    assert torch.equal(q, o.codes) and torch.equal(s, o.scales)


def test_many_rows_in_place(S):
    """r over x and n over y with ragged last pieces and two pieces a thread."""
    M, K = 700, 2051
    x, y, w = rand(61, M, K).cuda(), rand(62, M, K).cuda(), (1 + rand(63, K, scale=0.1)).cuda()
    ref = S.block_norm(x, y, post_weight=w, weight=w, normed=True)
    o = S.block_norm(x, y, post_weight=w, weight=w, residual_out=x, normed_out=y)
    assert o.residual.data_ptr() == x.data_ptr() and all(torch.equal(a, b) for a, b in zip(o, ref))


@pytest.mark.parametrize("K", [300, 2056])
def test_rows_far_apart(S, K):
    """Offsets past 32 bits: rows 3 x 2^29 elements apart in every operand."""
    M, pitch = 4, 3 << 29
    x, y, g = rand(71, M, K), rand(72, M, K, dtype=torch.bfloat16), rand(73, M, K, dtype=torch.bfloat16)

    def far(t):
        v = torch.empty((M - 1) * pitch + K, dtype=t.dtype, device="cuda").as_strided((M, K), (pitch, 1))
        v.copy_(t)
        return v

    ref = S.block_norm(x.cuda(), y.cuda(), gate=g.cuda(), normed=True)
    q = torch.empty((M - 1) * pitch + K, dtype=torch.uint8, device="cuda").as_strided((M, K), (pitch, 1))
    fx, fy = far(x), far(y)
    o = S.block_norm(fx, fy, gate=far(g), residual_out=fx, normed_out=fy, codes_out=q)
    for a, b in zip(o, ref):
        assert torch.equal(a, b)


def test_rows_do_not_touch_each_other(S):
    """A zero row, an infinity and a NaN stay in their rows."""
    M, K = 6, 512
    x = rand(31, M, K)
    x[1], x[2, 5], x[4, 7] = 0, float("inf"), float("nan")
    o = S.block_norm(x.cuda(), normed=True)
    q, n, s = o.codes.cpu(), o.normed.cpu(), o.scales.cpu()
    assert torch.all(q[1] == 0) and s[1] == 1 and torch.all(n[1] == 0)
    assert torch.all(torch.isnan(n[4])) and torch.all((q[4] & 0x7F) == 0x7F)
    assert torch.isnan(n[2, 5]) and torch.all(n[2, :5] == 0)
    keep = [0, 3, 5]
    clean = S.block_norm(x[keep].cuda(), normed=True)
    assert torch.equal(clean.codes.cpu(), q[keep]) and torch.equal(clean.normed.cpu(), n[keep])


def test_repeats_stream_and_graph(S):
    x, y = rand(41, 33, 2048, dtype=torch.bfloat16).cuda(), rand(42, 33, 2048, dtype=torch.bfloat16).cuda()
    ref = S.block_norm(x, y, normed=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o = S.block_norm(x, y, normed=True)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(o, ref))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = S.block_norm(x, y, normed=True)
    for seed in (43, 44, 45):
        x.copy_(rand(seed, 33, 2048, dtype=torch.bfloat16))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o, S.block_norm(x, y, normed=True)))


def test_binding_refuses(S):
    x, y = torch.zeros(4, 32, device="cuda"), torch.zeros(4, 32, device="cuda")
    w = torch.ones(32, device="cuda")
    for kw in (dict(y=y[:, :16]), dict(gate=w), dict(post_weight=w), dict(y=y, gate=w.bfloat16()),
               dict(y=y, post_weight=w, weight=w.bfloat16()), dict(weight=w[:16]), dict(quantize=False),
               dict(y=y, residual_out=x.bfloat16()), dict(y=y.cpu()), dict(residual_out=x),
               dict(y=y, codes_out=torch.zeros(4, 16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            S.block_norm(x, **kw)
    for bad in (x.cpu(), x[0].expand(4, 32), x.t(), x[0]):
        with pytest.raises(ValueError):
            S.block_norm(bad)
    for kw in (dict(eps=-1.0), dict(y=y, residual_out=y.clone(), normed_out=x), dict(y=y, residual_out=y)):
        with pytest.raises((S.SpenseError, ValueError)):
            S.block_norm(x, **kw)
    empty = S.block_norm(torch.zeros(0, 32, device="cuda"), normed=True)
    assert empty.normed.shape == (0, 32) and empty.codes.shape == (0, 32)
