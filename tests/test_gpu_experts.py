"""spense_gemm_experts and mlp_experts through the binding, against the formula in 64 bits.

Integer cases (entries up to 3, power-of-two scales) are exact in every order of summation and
compared bit for bit.  Random cases: the fp8 matrix instructions add the products of a lane's
chunk with 13 fractional bits of the largest, so a sum is within (2^-12 + 2 K u) of the sum of
magnitudes (u = 2^-24), then two scales and half a step of the output type.
"""
import re
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def S():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_10445_amd as S
    return S


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def weights(S, g, E, N, K, split, db, ints):
    """(PackedExperts, E x N x K float64 values, E x N scales)."""
    draw = torch.randint(-3, 4, (E, N, K), generator=g).float() if ints else torch.randn(E, N, K, generator=g)
    reg = draw[:, :db] if split == 0 else draw[:, :, :db]
    if reg.numel():  # keep two random entries of each four
        r = torch.rand(reg.reshape(E, reg.shape[1], -1, 4).shape, generator=g)
        keep = torch.zeros_like(r).scatter_(-1, r.argsort(-1)[..., :2], 1.0)
        reg.copy_((reg.reshape(r.shape) * keep).reshape(reg.shape))
    q = draw.to(torch.float8_e4m3fn)
    sc = 2.0 ** torch.randint(-2, 3, (E, N), generator=g) if ints else 0.5 + torch.rand(E, N, generator=g)
    mask = (q.float() != 0).to(torch.uint8)
    pws = [S.tile(S.compress(q[e].view(torch.uint8).cuda(), mask[e].cuda(), split, db)) for e in range(E)]
    return S.stack_experts(pws), q.double(), sc.float()


def tokens(g, T, K, ints):
    x = (torch.randint(-3, 4, (T, K), generator=g).float() if ints else torch.randn(T, K, generator=g)).to(torch.float8_e4m3fn)
    xs = 2.0 ** torch.randint(-2, 3, (T,), generator=g) if ints else 0.5 + torch.rand(T, generator=g)
    return x, xs.float()


def choices(g, kind, T, top, E):
    if kind == "even":
        return torch.randint(-1, E, (T, top), generator=g, dtype=torch.int32)
    if kind == "skewed":
        return (torch.rand(T, top, generator=g) ** 4 * (E + 1)).int()
    return torch.full((T, top), E - 1, dtype=torch.int32)  # one expert has them all


def check(y, order, offsets, x, xs, W, sc, top, exact, f32):
    n = int(offsets[-1])
    for e in range(W.shape[0]):
        a, b = int(offsets[e]), int(offsets[e + 1])
        if a == b:
            continue
        src = order[a:b].long() // top
        acc, mag = x[src].double() @ W[e].t(), x[src].double().abs() @ W[e].abs().t()
        f = sc[e].double()[None, :] * xs[src].double()[:, None]
        want, got = acc * f, y[a:b]
        if exact:
            want = want.float() if f32 else want.float().bfloat16()
            assert torch.equal(got, want), f"expert {e}"
        else:
            err = (2.0 ** -12 + 2 * W.shape[2] * U) * mag * f.abs() + 4 * U * want.abs()
            half = U if f32 else 2.0 ** -8
            assert torch.all((got.double() - want).abs() <= err + half * (want.abs() + err)), f"expert {e}"
    return n


CASES = [  # T, top, E, N, K, split, dense_begin
    (1, 1, 1, 16, 32, 0, 0), (1, 8, 16, 208, 512, 0, 160), (3, 2, 5, 257, 96, 0, 128), (9, 4, 8, 300, 1056, 1, 512),
    (40, 2, 4, 130, 2080, 1, 1568), (64, 1, 64, 96, 544, 0, 96), (33, 3, 6, 144, 1024, 1, 0), (50, 6, 7, 400, 640, 0, 400),
    (150, 2, 5, 256, 512, 0, 192), (400, 2, 9, 272, 992, 1, 736), (513, 1, 3, 389, 1536, 0, 256), (260, 4, 2, 128, 320, 1, 320),
    (700, 3, 1, 130, 416, 0, 64),
]


@pytest.mark.parametrize("T,top,E,N,K,split,db", CASES)
@pytest.mark.parametrize("kind", ["even", "skewed", "one"])
def test_experts_exact(S, T, top, E, N, K, split, db, kind):
    say(f"[experts] T={T} top={top} E={E} {N}x{K} split={split} db={db} {kind}")
    g = torch.Generator().manual_seed(T + N + K)
    (pe, W, sc), (x, xs) = weights(S, g, E, N, K, split, db, True), tokens(g, T, K, True)
    groups = S.group_rows(choices(g, kind, T, top, E).reshape(-1).cuda(), E)
    order, offsets = groups.order.cpu(), groups.offsets.cpu()
    for f32 in (False, True):
        out = torch.full((T * top, N), 9.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        y, = S.gemm_experts(x.view(torch.uint8).cuda(), [pe], groups, [sc.cuda()], xs.cuda(), top=top, outs=[out], out_f32=f32)
        n = check(y.cpu(), order, offsets, x, xs, W, sc, top, True, f32)
        assert torch.all(y[n:] == 9)  # rows of no expert


LONG = [  # K beyond what the short-K kernel keeps in LDS: two and four waves a workgroup, tiles of 16 and 32
    (1, 2, 3, 208, 3616, 0, 160), (3, 2, 5, 130, 3744, 1, 1600), (8, 1, 8, 1601, 3616, 0, 1200), (20, 2, 2, 257, 4096, 0, 128),
    (37, 2, 4, 96, 4128, 1, 4096), (9, 3, 3, 48, 5120, 1, 0),
]


@pytest.mark.parametrize("T,top,E,N,K,split,db", LONG)
@pytest.mark.parametrize("kind", ["even", "one"])
def test_long_rows_exact(S, T, top, E, N, K, split, db, kind):
    test_experts_exact(S, T, top, E, N, K, split, db, kind)


@pytest.mark.parametrize("T,top,E,N,K,split,db", LONG)
def test_long_rows_random(S, T, top, E, N, K, split, db):
    test_experts_random(S, T, top, E, N, K, split, db)


LARGE = [  # many rows an expert: tiles of up to 128 positions, and (from 256 of those on) of 256
    (450, 1, 2, 300, 352, 0, 112), (520, 2, 2, 136, 256, 0, 136), (640, 1, 1, 400, 1056, 1, 1056), (999, 3, 5, 264, 480, 1, 0),
    (1040, 1, 8, 2200, 288, 0, 1648), (700, 2, 9, 2065, 352, 1, 160), (530, 2, 11, 2190, 256, 0, 0), (1300, 1, 6, 3200, 320, 1, 320),
    (2600, 1, 10, 1700, 288, 0, 848),
]


@pytest.mark.parametrize("T,top,E,N,K,split,db", LARGE)
@pytest.mark.parametrize("kind", ["even", "skewed", "one"])
def test_large_groups_exact(S, T, top, E, N, K, split, db, kind):
    test_experts_exact(S, T, top, E, N, K, split, db, kind)


@pytest.mark.parametrize("T,top,E,N,K,split,db", LARGE)
def test_large_groups_random(S, T, top, E, N, K, split, db):
    test_experts_random(S, T, top, E, N, K, split, db)


@pytest.mark.parametrize("T,top,E,N,K,db", [(1, 4, 8, 96, 256, 64), (40, 2, 5, 130, 512, 96), (90, 2, 4, 160, 320, 160),
                                            (150, 3, 6, 257, 544, 128), (600, 1, 2, 300, 352, 112), (1040, 1, 8, 1101, 288, 624),
                                            (700, 2, 9, 1100, 352, 0), (2600, 1, 10, 700, 256, 700)])
@pytest.mark.parametrize("kind", ["even", "skewed"])
def test_glu_pair(S, T, top, E, N, K, db, kind):
    """The producer half of the MLP gives the codes and scales of its steps, bit for bit."""
    say(f"[glu] T={T} top={top} E={E} {N}x{K} db={db} {kind}")
    g = torch.Generator().manual_seed(T + N)
    gate, up = weights(S, g, E, N, K, 0, db, False), weights(S, g, E, N, K, 0, db, False)
    x, xs = tokens(g, T, K, False)
    X, XS, sc = x.view(torch.uint8).cuda(), xs.cuda() / K ** 0.5, [gate[2].cuda(), up[2].cuda()]
    groups = S.group_rows(choices(g, kind, T, top, E).reshape(-1).cuda(), E)
    n = int(groups.offsets[-1])
    for scales in ((sc, XS), ([None, None], None)):
        G, U_ = S.gemm_experts(X, [gate[0], up[0]], groups, *scales, top=top, out_f32=True)
        want = S.glu_quantize_fp8(G[:n].contiguous(), U_[:n].contiguous())
        q, s = S.gemm_experts_glu_fp8(X, gate[0], up[0], groups, *scales[0], scales[1], top=top)
        assert torch.equal(s[:n], want[1]) and torch.equal(q[:n], want[0])


LENGTHS = [0, 1, 63, 64, 65, 128, 129, 191, 192, 193, 255, 256, 257, 319, 320, 321, 384, 385, 448, 449, 512, 513, 576, 577, 0]


@pytest.mark.parametrize("E,N,K,split,db", [(25, 700, 96, 0, 304), (100, 200, 64, 1, 32)])
def test_group_lengths(S, E, N, K, split, db):
    """Tiles of every length, beginning anywhere; with 100 experts two a lane of the search for a tile."""
    g = torch.Generator().manual_seed(E)
    lens = torch.tensor(LENGTHS * 4)[:E][torch.randperm(E, generator=g)]
    idx = torch.repeat_interleave(torch.arange(E, dtype=torch.int32), lens)
    idx = torch.cat([idx, torch.full((13,), -1, dtype=torch.int32)])[torch.randperm(int(lens.sum()) + 13, generator=g)]
    T = idx.numel()
    (pe, W, sc), (x, xs) = weights(S, g, E, N, K, split, db, True), tokens(g, T, K, True)
    groups, X = S.group_rows(idx.cuda(), E), x.view(torch.uint8).cuda()
    order, offsets = groups.order.cpu(), groups.offsets.cpu()
    assert torch.equal(offsets.diff().long(), lens)
    for f32 in (False, True):
        out = torch.full((T, N), 9.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        S.gemm_experts(X, [pe], groups, [sc.cuda()], xs.cuda(), outs=[out], out_f32=f32)
        n = check(out.cpu(), order, offsets, x, xs, W, sc, 1, True, f32)
        assert torch.all(out[n:] == 9)
    if split == 0:
        up = weights(S, g, E, N, K, split, db, True)
        s2 = [sc.cuda() / 64, up[2].cuda()]
        G, U_ = S.gemm_experts(X, [pe, up[0]], groups, s2, xs.cuda(), out_f32=True)
        want = S.glu_quantize_fp8(G[:n].contiguous(), U_[:n].contiguous())
        q, s = S.gemm_experts_glu_fp8(X, pe, up[0], groups, *s2, xs.cuda())
        assert torch.equal(s[:n], want[1]) and torch.equal(q[:n], want[0])


@pytest.mark.parametrize("T,top,E,N,K,split,db", CASES)
def test_experts_random(S, T, top, E, N, K, split, db):
    g = torch.Generator().manual_seed(T + N + K + 1)
    (pe, W, sc), (x, xs) = weights(S, g, E, N, K, split, db, False), tokens(g, T, K, False)
    groups = S.group_rows(choices(g, "even", T, top, E).reshape(-1).cuda(), E)
    order, offsets = groups.order.cpu(), groups.offsets.cpu()
    for f32 in (False, True):
        call = lambda: S.gemm_experts(x.cuda().view(torch.uint8), [pe], groups, [sc.cuda()], xs.cuda(), top=top, out_f32=f32)[0]  # noqa: E731,B023
        y = call()
        n = check(y.cpu(), order, offsets, x, xs, W, sc, top, False, f32)
        for _ in range(3):
            assert torch.equal(call()[:n], y[:n])


@pytest.mark.parametrize("T,E,N,K,split,db", [(5, 4, 160, 544, 0, 112), (30, 3, 200, 512, 1, 256), (300, 3, 264, 1024, 0, 128)])
def test_pair_gathered_and_strided(S, T, E, N, K, split, db):
    """Two weights in one launch equal two launches; gathered rows; X and Y inside wider buffers; no scales."""
    g = torch.Generator().manual_seed(T)
    ws = [weights(S, g, E, N, K, split, db, True) for _ in range(2)]
    x, xs = tokens(g, T, K, True)
    groups = S.group_rows(choices(g, "even", T, 1, E).reshape(-1).cuda(), E)
    n = int(groups.offsets[-1])
    X, XS = x.view(torch.uint8).cuda(), xs.cuda()
    both = S.gemm_experts(X, [w[0] for w in ws], groups, [w[2].cuda() for w in ws], XS)
    for y, (pe, W, sc) in zip(both, ws):
        one, = S.gemm_experts(X, [pe], groups, [sc.cuda()], XS)
        assert torch.equal(y[:n], one[:n])
        wide_x = torch.zeros(T, K + 32, dtype=torch.uint8, device="cuda")
        wide_x[:n, :K] = X[groups.order[:n].long()]
        wide_x[n:] = 0x7F
        xs_p = XS[groups.order.long()]
        out = torch.full((T, N + 5), 3.0, dtype=torch.bfloat16, device="cuda")
        S.gemm_experts(wide_x[:, :K], [pe], groups, [sc.cuda()], xs_p, gathered=True, outs=[out[:, :N]])
        assert torch.equal(out[:n, :N], one[:n]) and torch.all(out[:, N:] == 3) and torch.all(out[n:] == 3)
        plain, = S.gemm_experts(X, [pe], groups, out_f32=True)
        ones = torch.ones(E, N), torch.ones(T)
        check(plain.cpu(), groups.order.cpu(), groups.offsets.cpu(), x, ones[1], W, ones[0], 1, True, True)


def test_no_rows(S):
    g = torch.Generator().manual_seed(1)
    pe, _, _ = weights(S, g, 3, 64, 128, 0, 32, True)
    X = torch.zeros(6, 128, dtype=torch.uint8, device="cuda")
    groups = S.group_rows(torch.full((6,), -1, dtype=torch.int32, device="cuda"), 3)
    out = torch.full((6, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    S.gemm_experts(X, [pe], groups, outs=[out])
    assert torch.all(out == 2)
    y, = S.gemm_experts(X[:0], [pe], S.group_rows(torch.zeros(0, dtype=torch.int32, device="cuda"), 3))
    assert y.shape == (0, 64)


@pytest.mark.parametrize("T", [20, 400])
def test_rows_outside_give_zeros(S, T):
    """order and offsets of another making: rows outside X are zeros, offsets past n are n."""
    g = torch.Generator().manual_seed(2)
    pe, W, sc = weights(S, g, 2, 64, 128, 0, 32, True)
    x, xs = tokens(g, T, 128, True)
    order = torch.arange(T, dtype=torch.int32)
    order[3], order[8] = -9, 2 ** 31 - 1
    groups = S.RowGroups(T, 2, torch.cat([order, order, torch.tensor([-7, T // 2, 2 ** 31 - 1], dtype=torch.int32)]).cuda())
    y, = S.gemm_experts(x.view(torch.uint8).cuda(), [pe], groups, [sc.cuda()], xs.cuda(), out_f32=True)
    y = y.cpu()
    assert torch.all(y[3] == 0) and torch.all(y[8] == 0)
    order = torch.arange(T)
    y[3], y[8] = (x[3].double() @ W[0].t() * sc[0] * xs[3]).float(), (x[8].double() @ W[0].t() * sc[0] * xs[8]).float()
    check(y, order, torch.tensor([0, T // 2, T]), x, xs, W, sc, 1, True, True)


def test_non_finite_rows_stay_alone(S):
    g = torch.Generator().manual_seed(3)
    for T in (24, 300):
        pe, W, sc = weights(S, g, 2, 96, 512, 0, 64, True)
        x, xs = tokens(g, T, 512, True)
        groups = S.group_rows(choices(g, "even", T, 1, 2).reshape(-1).abs().cuda(), 2)
        X = x.view(torch.uint8).cuda()
        clean, = S.gemm_experts(X, [pe], groups, [sc.cuda()], xs.cuda())
        X[5, 7] = 0x7F
        y, = S.gemm_experts(X, [pe], groups, [sc.cuda()], xs.cuda())
        at = int(groups.inverse[5])
        keep = torch.arange(T, device="cuda") != at
        assert torch.equal(y[keep], clean[keep]) and torch.any(torch.isnan(y[at]))


@pytest.mark.parametrize("T,E,N,K", [(5, 2, 40, 128), (5, 2, 40, 3584), (40, 2, 70, 3584), (300, 2, 130, 128), (700, 1, 5602, 128)])
@pytest.mark.parametrize("f32", [False, True])
def test_outputs_far_apart(S, T, E, N, K, f32):
    """Offsets of the output past 32 bits, in every kernel."""
    g = torch.Generator().manual_seed(T + N)
    pe, W, sc = weights(S, g, E, N, K, 0, 32, True)
    x, xs = tokens(g, T, K, True)
    groups = S.group_rows(choices(g, "even", T, 1, E).reshape(-1).cuda(), E)
    pitch = -(-(9 << 29) // T) + 3
    dt = torch.float32 if f32 else torch.bfloat16
    y = torch.empty((T - 1) * pitch + N, dtype=dt, device="cuda").as_strided((T, N), (pitch, 1))
    S.gemm_experts(x.view(torch.uint8).cuda(), [pe], groups, [sc.cuda()], xs.cuda(), outs=[y], out_f32=f32)
    check(y.cpu(), groups.order.cpu(), groups.offsets.cpu(), x, xs, W, sc, 1, True, f32)


@pytest.mark.parametrize("T,top,E,H,I", [(6, 2, 3, 256, 96), (300, 2, 4, 256, 96), (1300, 2, 2, 256, 1408)])
def test_mlp_of_a_non_finite_token(S, T, top, E, H, I):
    """A token whose scale is NaN and one with an infinite weight leave the others as they are."""
    g = torch.Generator().manual_seed(T)
    gate, up, down = weights(S, g, E, I, H, 0, 64, False), weights(S, g, E, I, H, 0, 64, False), weights(S, g, E, H, I, 1, 64, False)
    x, xs = tokens(g, T, H, False)
    idx, w = torch.randint(0, E, (T, top), generator=g, dtype=torch.int32), torch.rand(T, top, generator=g)
    run = lambda xs, w: S.mlp_experts(x.view(torch.uint8).cuda(), xs.cuda(), idx.cuda(), w.cuda(), gate[0], up[0], down[0],  # noqa: E731
                                      *(v[2].cuda() / 64 for v in (gate, up, down))).cpu()
    clean = run(xs, w)
    assert torch.all(torch.isfinite(clean))
    xs[2], w[4, 1] = float("nan"), float("inf")
    y = run(xs, w)
    keep = [t for t in range(T) if t not in (2, 4)]
    assert torch.equal(y[keep], clean[keep]) and torch.all(torch.isnan(y[2])) and not torch.any(torch.isfinite(y[4]))


def decoded_glu(S, G, U):
    q, s = S.glu_quantize_fp8(G, U)
    return q.cpu().view(torch.float8_e4m3fn), s.cpu()


@pytest.mark.parametrize("T,top,E,H,I,db", [(1, 2, 4, 256, 96, 64), (7, 3, 5, 512, 160, 128), (130, 2, 4, 320, 256, 192),
                                            (300, 2, 2, 256, 128, 0)])
def test_mlp_experts(S, T, top, E, H, I, db):
    """The whole path against its steps in 64 bits; H's codes may sit a step off where h / s is near a
    midpoint, so the oracle takes the codes that the same G and U give."""
    g = torch.Generator().manual_seed(T + I)
    gate, up = weights(S, g, E, I, H, 0, db, False), weights(S, g, E, I, H, 0, db, False)
    down = weights(S, g, E, H, I, 1, db, False)
    x, xs = tokens(g, T, H, False)
    xs = xs / H ** 0.5
    idx, w = choices(g, "even", T, top, E), torch.rand(T, top, generator=g)
    idx[0] = -1  # a token without experts
    X, XS = x.view(torch.uint8).cuda(), xs.cuda()
    sc = [v[2].cuda() for v in (gate, up, down)]
    y = S.mlp_experts(X, XS, idx.cuda(), w.cuda(), gate[0], up[0], down[0], *sc)
    groups = S.group_rows(idx.reshape(-1).cuda(), E)
    n = int(groups.offsets[-1])
    G, U_ = S.gemm_experts(X, [gate[0], up[0]], groups, sc[:2], XS, top=top, out_f32=True)
    hq, hs = decoded_glu(S, G[:n].contiguous(), U_[:n].contiguous())
    order, off = groups.order.cpu().long(), groups.offsets.cpu()
    want, mag = torch.zeros(T, H, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    for e in range(E):
        for p in range(int(off[e]), int(off[e + 1])):
            h = hq[p].double() * hs[p].double()
            row = (h @ down[1][e].t()) * down[2][e].double() * w.reshape(-1)[order[p]].double()
            want[order[p] // top] += row
            mag[order[p] // top] += (h.abs() @ down[1][e].abs().t()) * down[2][e].double() * w.reshape(-1)[order[p]].double()
    err = (2.0 ** -12 + 2 * I * U) * mag + 8 * U * mag
    assert torch.all((y.cpu().double() - want).abs() <= err + 2.0 ** -8 * (want.abs() + err))
    assert torch.all(y[0] == 0)


def test_captured_and_on_streams(S):
    g = torch.Generator().manual_seed(11)
    T, top, E, H, I = 20, 2, 6, 256, 96
    gate, up, down = weights(S, g, E, I, H, 0, 64, False), weights(S, g, E, I, H, 0, 64, False), weights(S, g, E, H, I, 1, 64, False)
    sc = [v[2].cuda() for v in (gate, up, down)]
    x, xs = tokens(g, T, H, False)
    X, XS, idx, w = x.view(torch.uint8).cuda(), xs.cuda(), choices(g, "even", T, top, E).cuda(), torch.rand(T, top, generator=g).cuda()
    call = lambda: S.mlp_experts(X, XS, idx, w, gate[0], up[0], down[0], *sc)  # noqa: E731
    ref = call()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        outs = []
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(call())
        torch.cuda.synchronize()
        assert all(torch.equal(o, ref) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = call()
    for seed in (1, 2, 3):
        g = torch.Generator().manual_seed(seed)
        x, xs = tokens(g, T, H, False)
        X.copy_(x.view(torch.uint8)), XS.copy_(xs), idx.copy_(choices(g, "skewed", T, top, E))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, call())


def test_norm_adapters_experts_together(S):
    """A block as a program runs it: norm, a projection with adapters, norm around it, experts."""
    g = torch.Generator().manual_seed(21)
    T, top, E, H, I, R = 33, 2, 4, 256, 96, 8
    x = torch.randn(T, H, generator=g).bfloat16().cuda()
    w1, w2 = 1 + 0.1 * torch.randn(H, generator=g).cuda(), 1 + 0.1 * torch.randn(H, generator=g).cuda()
    proj = weights(S, g, 1, H, H, 0, 192, False)
    pe = proj[0]
    pw = S.PackedWeight(H, H, S.SPENSE_FP8_E4M3FN, 0, 192, pe.values[0], pe.meta[0], pe.dense[0], S.SPENSE_LAYOUT_TILED)
    psc = (proj[2][0] / H ** 0.5).cuda()
    A, B = torch.randn(3, R, H, generator=g).bfloat16(), torch.randn(3, H, R, generator=g).bfloat16()
    pool = S.AdapterPool(A.cuda(), B.cuda(), torch.full((3,), 0.01, device="cuda"))
    users = torch.randint(-1, 3, (T,), generator=g, dtype=torch.int32)
    n1 = S.block_norm(x, weight=w1, normed=True)
    a = S.gemm_adapters(n1.codes, pw, pool, S.group_rows(users.cuda(), 3), psc, n1.scales, A_x=n1.normed)
    n2 = S.block_norm(x, a, weight=w2, residual_scale=0.5)
    gate, up, down = weights(S, g, E, I, H, 0, 64, False), weights(S, g, E, I, H, 0, 64, False), weights(S, g, E, H, I, 1, 64, False)
    idx, w = choices(g, "even", T, top, E).cuda(), torch.rand(T, top, generator=g).cuda()
    sc = [v[2].cuda() for v in (gate, up, down)]
    y = S.mlp_experts(n2.codes, n2.scales, idx, w, gate[0], up[0], down[0], *sc)
    # the projection and adapters in 64 bits from the norm's outputs (tolerances of the single tests)
    q = n1.codes.cpu().view(torch.float8_e4m3fn).double() * n1.scales.cpu().double()[:, None]
    base = q @ (proj[1][0] * psc.cpu().double()[:, None]).t()
    mag = q.abs() @ (proj[1][0] * psc.cpu().double()[:, None]).abs().t()
    nx = n1.normed.cpu().double()
    for t in range(T):
        if users[t] >= 0:
            v = nx[t] @ A[users[t]].double().t() * 0.01
            base[t] += v @ B[users[t]].double().t()
            mag[t] += (nx[t].abs() @ A[users[t]].double().abs().t() * 0.01) @ B[users[t]].double().abs().t()
    err = (2.0 ** -12 + 2 * H * U + 2.0 ** -16) * mag
    assert torch.all((a.cpu().double() - base).abs() <= err + 2.0 ** -8 * (base.abs() + err))
    r = 0.5 * x.cpu().double() + a.cpu().double()
    assert torch.all((n2.residual.cpu().double() - r).abs() <= 2.0 ** -8 * r.abs() + 1e-6)
    assert torch.all(torch.isfinite(y)) and y.shape == (T, H)


def test_binding_refuses(S):
    g = torch.Generator().manual_seed(1)
    pe, _, sc = weights(S, g, 3, 64, 128, 0, 32, True)
    other, _, _ = weights(S, g, 3, 64, 128, 0, 48, True)
    X = torch.zeros(6, 128, dtype=torch.uint8, device="cuda")
    groups = S.group_rows(torch.zeros(6, dtype=torch.int32, device="cuda"), 3)
    for kw in (dict(experts=[]), dict(experts=[pe] * 3), dict(X=X[:5]), dict(X=X[:, :96]), dict(X=X.bfloat16()), dict(top=0),
               dict(top=2), dict(groups=S.group_rows(torch.zeros(6, dtype=torch.int32, device="cuda"), 4)),
               dict(w_scales=[sc]), dict(w_scales=[sc.cuda()[:2]]), dict(w_scales=[None, None]),
               dict(x_scale=torch.ones(5, device="cuda")), dict(outs=[torch.zeros(6, 63, dtype=torch.bfloat16, device="cuda")])):
        with pytest.raises((ValueError, TypeError)):
            S.gemm_experts(**{"X": X, "experts": [pe], "groups": groups, **kw})
    with pytest.raises(S.SpenseError):
        S.gemm_experts(X, [pe, other], groups)
    with pytest.raises(ValueError):
        S.stack_experts([])
    row_major = S.PackedWeight.empty(64, 128, S.SPENSE_FP8_E4M3FN, 0, 32)
    with pytest.raises(ValueError):
        S.stack_experts([row_major])
    with pytest.raises(ValueError):
        S.mlp_experts(X, torch.ones(6, device="cuda"), torch.zeros(5, 2, dtype=torch.int32, device="cuda"),
                      torch.zeros(5, 2, device="cuda"), pe, pe, pe)


# Sizes at which the short-K kernel gives a wave several row tiles (the rule goes by the sizes only; what it chooses is
# in the dispatch log and checked): rows of activations, experts, N, K, split, dense_begin, weights -> positions
# of a tile, row tiles of a wave.  Their last workgroups give waves fewer tiles than that, or none.
STREAMS = [
    (135, 27, 1746, 160, 0, 1296, 1, 16, 2), (264, 44, 1046, 1056, 0, 720, 1, 16, 2), (165, 55, 1677, 160, 1, 96, 1, 16, 3),
    (53, 53, 1803, 1056, 1, 736, 1, 16, 3), (330, 55, 2404, 160, 0, 2400, 1, 16, 4), (385, 55, 2526, 1056, 1, 768, 1, 16, 4),
    (60, 60, 3077, 160, 1, 64, 1, 16, 5), (260, 52, 4185, 160, 0, 4176, 1, 16, 6), (224, 56, 4837, 160, 0, 4832, 1, 16, 7),
    (480, 60, 4963, 704, 0, 4960, 1, 16, 8), (39, 39, 1066, 160, 0, 528, 2, 16, 3), (110, 55, 2424, 160, 0, 1808, 2, 16, 8),
    (896, 56, 445, 160, 0, 304, 1, 32, 2), (742, 53, 445, 1056, 0, 304, 1, 32, 2), (520, 52, 1050, 160, 1, 0, 1, 32, 3),
    (986, 58, 1028, 1056, 1, 768, 1, 32, 3), (731, 43, 1976, 160, 1, 96, 1, 32, 4), (792, 44, 1558, 1056, 0, 1168, 1, 32, 4),
    (520, 52, 1662, 160, 0, 1648, 1, 32, 5), (688, 43, 3242, 160, 1, 64, 1, 32, 6), (880, 55, 2385, 160, 0, 2384, 1, 32, 7),
    (583, 53, 2888, 160, 0, 2880, 1, 32, 8), (731, 43, 368, 160, 0, 272, 2, 32, 3), (688, 43, 1220, 160, 0, 912, 2, 32, 8),
    (2585, 55, 485, 160, 0, 352, 1, 64, 2), (1456, 52, 422, 1120, 0, 288, 1, 64, 2), (1040, 52, 1029, 160, 1, 64, 1, 64, 3),
    (1357, 59, 1036, 1056, 1, 736, 1, 64, 3), (1720, 43, 1303, 1056, 0, 912, 1, 64, 3), (1664, 52, 1320, 160, 0, 912, 1, 64, 4),
    (2120, 53, 2081, 160, 1, 96, 1, 64, 5), (1196, 52, 1995, 160, 0, 1984, 1, 64, 6), (1908, 53, 3100, 160, 1, 0, 1, 64, 7),
    (900, 40, 5120, 1408, 1, 1056, 1, 64, 7), (1484, 53, 2841, 160, 0, 2832, 1, 64, 8), (1204, 43, 405, 160, 0, 288, 2, 64, 3),
    (1333, 43, 1225, 160, 0, 912, 2, 64, 8),
]


def launches(capfd):
    """(kernel, positions of a tile, row tiles of a wave) of the grouped products in the dispatch log."""
    line = re.compile(r"spense: experts .* -> (.*) positions=(\d+) waves=\d+ tiles_wave=(\d+) ")
    return [(m[1], int(m[2]), int(m[3])) for m in map(line.match, capfd.readouterr().err.splitlines()) if m]


def weights_on_gpu(S, g, E, N, K, split, db):
    """As ``weights`` with integers, drawn on the GPU: (PackedExperts, E x N x K values (float8), E x N scales)."""
    q = torch.empty(E, N, K, dtype=torch.float8_e4m3fn, device="cuda")
    pws = []
    for e in range(E):
        w = torch.randint(-3, 4, (N, K), generator=g, device="cuda").float()
        reg = w[:db] if split == 0 else w[:, :db]
        if reg.numel():
            r = torch.rand(reg.shape[0], reg.shape[1] // 4, 4, generator=g, device="cuda")
            keep = torch.zeros_like(r).scatter_(-1, r.argsort(-1)[..., :2], 1.0)
            reg.copy_((reg.reshape(r.shape) * keep).reshape(reg.shape))
        q[e] = w.to(torch.float8_e4m3fn)
        pws.append(S.tile(S.compress(q[e].view(torch.uint8), (w != 0).to(torch.uint8), split, db)))
    return S.stack_experts(pws), q, 2.0 ** torch.randint(-2, 3, (E, N), generator=g, device="cuda").float()


@pytest.mark.parametrize("n,E,N,K,split,db,k,positions,tiles", STREAMS)
def test_several_row_tiles_a_wave(S, capfd, n, E, N, K, split, db, k, positions, tiles):
    """A wave's second row tile and those after it: addresses, scales, sums begun anew, the ragged last workgroup."""
    say(f"[experts] n={n} E={E} {N}x{K} split={split} db={db} weights={k}")
    g = torch.Generator(device="cuda")
    g.manual_seed(n + N + K)
    ws = [weights_on_gpu(S, g, E, N, K, split, db) for _ in range(k)]
    x = torch.randint(-3, 4, (n, K), generator=g, device="cuda").to(torch.float8_e4m3fn)
    xs = 2.0 ** torch.randint(-2, 3, (n,), generator=g, device="cuda").float()
    idx = (torch.rand(n, generator=g, device="cuda") ** 1.5 * (E + 1)).int() - 1  # uneven; some in no group
    idx[idx == E // 2] = 0  # an expert without rows
    groups = S.group_rows(idx, E)
    order, offsets = groups.order.long(), groups.offsets.tolist()
    for f32 in (False, True):
        dt = torch.float32 if f32 else torch.bfloat16
        outs = [torch.full((n, N), 9.0, dtype=dt, device="cuda") for _ in range(k)]
        prev = S.spense_set_log(2)
        try:
            capfd.readouterr()
            S.gemm_experts(x.view(torch.uint8), [w[0] for w in ws], groups, [w[2] for w in ws], xs, outs=outs, out_f32=f32)
            assert launches(capfd) == [("stream", positions, tiles)]
        finally:
            S.spense_set_log(prev)
        for y, (_, q, sc) in zip(outs, ws):
            for e in range(E):
                a, b = offsets[e], offsets[e + 1]
                acc = x[order[a:b]].double() @ q[e].double().t().contiguous()
                want = acc * sc[e].double() * xs[order[a:b], None].double()
                assert torch.equal(y[a:b], want.float().to(dt)), f"expert {e}"
            assert torch.all(y[offsets[E]:] == 9)


def glu_bounds(x, xs, W, sc, src):
    """(value, bound) in 64 bits of rows src times one expert's weight: the error of ``check`` before rounding."""
    f = sc.double()[None, :] * xs[src].double()[:, None]
    acc, mag = x[src].double() @ W.t() * f, x[src].double().abs() @ W.abs().t() * f.abs()
    return acc, (2.0 ** -12 + 2 * W.shape[1] * U) * mag + 4 * U * acc.abs()


def check_codes(q, s, h, dh):
    """Codes and scales of rows whose values are within dh of h."""
    q, s = q.view(torch.float8_e4m3fn).double(), s.double()
    want = h.abs().amax(1) / 448
    assert torch.all((s - want).abs() <= dh.amax(1) / 448 + 2 * U * want)
    v = h / s[:, None]
    step = torch.exp2(torch.floor(torch.log2(torch.maximum(v.abs(), q.abs()).clamp_min(2.0 ** -6))) - 3)
    assert torch.all((q - v).abs() <= step / 2 + dh / s[:, None] + 2 * U * v.abs())


def check_h(q, s, x, xs, gate, up, order, offsets, top):
    """The quantised middle of the MLP against 64 bits.  |silu'| < 1.1 and |silu(g)| <= |g|; exp(-g) is off by
    2 |g| u for its argument, and exp, division and products add fewer than 16 roundings."""
    for e in range(gate[1].shape[0]):
        a, b = int(offsets[e]), int(offsets[e + 1])
        if a == b:
            continue
        src = order[a:b].long() // top
        g, dg = glu_bounds(x, xs, gate[1][e], gate[2][e], src)
        u, du = glu_bounds(x, xs, up[1][e], up[2][e], src)
        silu = g / (1 + torch.exp(-g))
        h = u * silu
        check_codes(q[a:b], s[a:b], h, du * silu.abs() + 1.1 * dg * (u.abs() + du) + (2 * g.abs() + 16) * U * h.abs())


def kernels(capfd):
    return [name for name, _, _ in launches(capfd)]


@pytest.mark.parametrize("T,top,E,N,K,db,kernel", [
    (3, 2, 5, 130, 5120, 96, "rows"), (20, 2, 2, 96, 4128, 32, "rows"), (40, 2, 5, 130, 512, 96, "stream"),
    (90, 2, 4, 160, 320, 160, "stream"), (150, 3, 6, 257, 544, 128, "128x128"), (1040, 1, 8, 1101, 288, 624, "256x256"),
    (700, 2, 9, 1100, 352, 0, "256x256"), (2600, 1, 10, 700, 256, 700, "256x256"), (300, 2, 3, 3201, 608, 2400, "256x256")])
def test_pair_against_the_formula(S, capfd, T, top, E, N, K, db, kernel):
    """G, U and H's codes of a gate / up pair, each against 64 bits, in every kernel that computes two weights."""
    say(f"[pair] T={T} top={top} E={E} {N}x{K} db={db} {kernel}")
    g = torch.Generator().manual_seed(T + N + 5)
    gate, up = weights(S, g, E, N, K, 0, db, False), weights(S, g, E, N, K, 0, db, False)
    x, xs = tokens(g, T, K, False)
    xs = xs / K ** 0.5
    X, XS, sc = x.view(torch.uint8).cuda(), xs.cuda(), [gate[2].cuda(), up[2].cuda()]
    groups = S.group_rows(choices(g, "even", T, top, E).reshape(-1).cuda(), E)
    order, offsets = groups.order.cpu(), groups.offsets.cpu()
    prev = S.spense_set_log(2)
    try:
        capfd.readouterr()
        both = S.gemm_experts(X, [gate[0], up[0]], groups, sc, XS, top=top, out_f32=True)
        q, s = S.gemm_experts_glu_fp8(X, gate[0], up[0], groups, *sc, XS, top=top)
        assert kernels(capfd) == [kernel, kernel + (", gate/up paired" if kernel == "256x256" else "")]
    finally:
        S.spense_set_log(prev)
    for y, w in zip(both, (gate, up)):
        check(y.cpu(), order, offsets, x, xs, w[1], w[2], top, False, True)
    check_h(q.cpu(), s.cpu(), x, xs, gate, up, order, offsets, top)


@pytest.mark.parametrize("T,top,E,H,I,db,which", [
    (1, 2, 4, 256, 96, 64, ["stream"] * 2), (7, 3, 5, 512, 160, 128, ["stream"] * 2), (2, 2, 3, 3616, 96, 32, ["rows", "stream"]),
    (300, 2, 2, 256, 128, 0, ["128x128"] * 2), (1300, 2, 2, 1440, 672, 320, ["256x256, gate/up paired", "256x256"])])
def test_mlp_steps_against_the_formula(S, capfd, T, top, E, H, I, db, which):
    """The whole MLP: H's codes against 64 bits, then the output against 64 bits from these codes."""
    say(f"[mlp] T={T} top={top} E={E} hidden={H} inter={I} db={db}")
    g = torch.Generator().manual_seed(T + I + 7)
    gate, up = weights(S, g, E, I, H, 0, db, False), weights(S, g, E, I, H, 0, db, False)
    down = weights(S, g, E, H, I, 1, db, False)
    x, xs = tokens(g, T, H, False)
    xs = xs / H ** 0.5
    idx, w = choices(g, "even", T, top, E), torch.rand(T, top, generator=g)
    X, XS, sc = x.view(torch.uint8).cuda(), xs.cuda(), [v[2].cuda() for v in (gate, up, down)]
    prev = S.spense_set_log(2)
    try:
        capfd.readouterr()
        y = S.mlp_experts(X, XS, idx.cuda(), w.cuda(), gate[0], up[0], down[0], *sc).cpu().double()
        assert kernels(capfd) == which
    finally:
        S.spense_set_log(prev)
    groups = S.group_rows(idx.reshape(-1).cuda(), E)
    order, offsets = groups.order.cpu().long(), groups.offsets.cpu()
    q, s = (v.cpu() for v in S.gemm_experts_glu_fp8(X, gate[0], up[0], groups, *sc[:2], XS, top=top))
    check_h(q, s, x, xs, gate, up, order, offsets, top)
    want, mag = torch.zeros(T, H, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    for e in range(E):
        p = slice(int(offsets[e]), int(offsets[e + 1]))
        h = q[p].view(torch.float8_e4m3fn).double() * s[p].double()[:, None]
        f = down[2][e].double()[None, :] * w.reshape(-1)[order[p], None].double()
        want.index_add_(0, order[p] // top, h @ down[1][e].t() * f)
        mag.index_add_(0, order[p] // top, h.abs() @ down[1][e].abs().t() * f)
    err = (2.0 ** -12 + 2 * I * U + 8 * U) * mag
    assert torch.all((y - want).abs() <= err + 2.0 ** -8 * (want.abs() + err))


@pytest.mark.parametrize("T,top,E,N,K,split,db", [(1500, 2, 1000, 40, 64, 0, 16), (9, 8, 1024, 16, 96, 1, 32), (9000, 2, 1000, 16, 32, 0, 16),
                                                  (18000, 2, 600, 18, 32, 0, 0), (35000, 2, 600, 16, 32, 1, 0)])
def test_many_experts(S, T, top, E, N, K, split, db):
    """Up to sixteen experts a lane in the search for a tile, from tiles of 16 positions to tiles of 256."""
    test_experts_exact(S, T, top, E, N, K, split, db, "even")
    test_experts_exact(S, T, top, E, N, K, split, db, "skewed")
