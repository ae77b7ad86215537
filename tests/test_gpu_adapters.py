"""spense_add_adapters through the binding, against the formula in 64 bits.

A x is a sum of K fp32 products (at most K + 40 roundings of u = 2^-24 with the partials and
the two scales), V = s A x enters B V within 2^-17, B V is a sum of 2 R products, base and the
rounding of Y follow.  On small integers every one of these is exact.
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


def inputs(seed, M, K, N, R, count, x, base, ints=False, idx=None):
    g = torch.Generator().manual_seed(seed)
    if ints:
        draw = lambda *s: torch.randint(-2, 3, s, generator=g).float()  # noqa: E731
    else:
        draw = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    X = draw(M, K)
    xs = None
    if x == "fp8":
        X = X.to(torch.float8_e4m3fn)
        xs = 2.0 ** torch.randint(-2, 3, (M,), generator=g) if ints else 0.5 + torch.rand(M, generator=g)
    else:
        X = X.bfloat16()
    A, B = draw(count, R, K).bfloat16(), draw(count, N, R).bfloat16()
    if ints:  # few non-zeros: |V| below 2^16 scaled, sums exact
        A = A * (torch.rand(count, R, K, generator=g) < 0.25)
    sc = 2.0 ** torch.randint(-2, 3, (count,), generator=g) if ints else torch.randn(count, generator=g)
    bd = draw(M, N).to(torch.bfloat16 if base == "bf16" else torch.float32)
    idx = torch.randint(-1, count, (M,), generator=g, dtype=torch.int32) if idx is None else idx.to(torch.int32)
    return X, xs, A, B, sc, bd, idx


def formula(X, xs, A, B, sc, bd, idx):
    """(Y, bound before the last rounding) in float64."""
    x = X.double() if xs is None else X.double() * xs.double()[:, None]
    y, e = bd.double().clone(), torch.zeros(bd.shape, dtype=torch.float64)
    R, K = A.shape[1:]
    for a in range(A.shape[0]):
        m = (idx == a).nonzero().flatten()
        if not len(m):
            continue
        s = 1.0 if sc is None else sc[a].double()
        Ad, Bd = A[a].double(), B[a].double()
        v = s * (x[m] @ Ad.t())
        mag = abs(s) * (x[m].abs() @ Ad.abs().t())
        dv = (K + 40) * U * mag + 2.0 ** -17 * v.abs()
        add = v @ Bd.t()
        y[m] += add
        e[m] = dv @ Bd.abs().t() + (2 * R + 8) * U * ((v.abs() + dv) @ Bd.abs().t()) + 2 * U * (bd[m].double().abs() + add.abs())
    return y, e


def call(S, t, count, **kw):
    X, xs, A, B, sc, bd, idx = [None if v is None else v.cuda() for v in t]
    pool = S.AdapterPool(A, B, sc)
    return S.add_adapters(bd, X, pool, S.group_rows(idx, count), x_scale=xs, **kw)


SIZES = [  # M, K, N, R, count
    (1, 32, 1, 8, 1), (1, 5120, 1024, 16, 4), (3, 96, 40, 24, 2), (17, 512, 333, 8, 5), (40, 1024, 2048, 64, 7),
    (64, 2080, 777, 16, 64), (70, 256, 520, 128, 3), (130, 544, 264, 40, 1), (200, 512, 96, 16, 4), (517, 1056, 1000, 32, 3),
    (300, 640, 512, 64, 9), (5, 25600, 64, 8, 1000),
]


@pytest.mark.parametrize("M,K,N,R,count", SIZES)
@pytest.mark.parametrize("x", ["fp8", "bf16"])
def test_random(S, M, K, N, R, count, x):
    for base, f32 in (("f32", False), ("bf16", False), ("bf16", True), ("f32", True)):
        say(f"[adapters] M={M} K={K} N={N} R={R} count={count} {x} {base} f32={f32}")
        t = inputs(M + K, M, K, N, R, count, x, base)
        y = call(S, t, count, out_f32=f32).cpu().double()
        want, e = formula(*t)
        half = U if f32 else 2.0 ** -8
        assert torch.all((y - want).abs() <= e + half * (want.abs() + e) + 1e-38)


@pytest.mark.parametrize("M,K,N,R,count", SIZES)
@pytest.mark.parametrize("x", ["fp8", "bf16"])
def test_integers_exact(S, M, K, N, R, count, x):
    K = min(K, 2080)
    t = inputs(M, M, K, N, R, count, x, "f32", ints=True)
    say(f"[adapters exact] M={M} K={K} N={N} R={R} count={count} {x}")
    y = call(S, t, count, out_f32=True).cpu().double()
    assert torch.equal(y, formula(*t)[0])


# Sizes at which a workgroup of the second launch takes more than two steps of 128 columns (by a rule on the sizes;
# what it chooses is in the dispatch log and checked): M, K, N, R, count -> tokens of a tile, steps.  N ends in
# different steps, inside a piece of eight and of 32 columns and between them.
WIDE = [
    (64, 64, 8201, 16, 64, 16, 8), (64, 32, 25601, 8, 64, 16, 8), (96, 64, 6657, 64, 90, 16, 8), (160, 64, 7004, 128, 150, 16, 8),
    (64, 64, 5003, 24, 64, 16, 4), (100, 96, 3360, 40, 90, 16, 4), (64, 544, 4097, 16, 64, 16, 4), (2048, 64, 8190, 64, 16, 32, 4),
    (2048, 64, 4001, 16, 16, 32, 4), (1024, 96, 8328, 32, 8, 32, 4), (520, 64, 16385, 8, 5, 32, 4),
]


def chosen(capfd):
    """(tokens of a tile, steps) of the adapter calls in the dispatch log."""
    line = re.compile(r"spense: adapters .* -> tile_tokens=(\d+) k_slices=\d+ steps=(\d+) ")
    return [(int(m[1]), int(m[2])) for m in map(line.match, capfd.readouterr().err.splitlines()) if m]


@pytest.mark.parametrize("M,K,N,R,count,tokens,steps", WIDE)
@pytest.mark.parametrize("base", ["f32", "bf16"])
def test_many_columns_a_workgroup(S, capfd, M, K, N, R, count, tokens, steps, base):
    """Exact integers with fp32 outputs, random values with the base's type, and the latter over base itself."""
    say(f"[adapters wide] M={M} K={K} N={N} R={R} count={count} {base}")
    prev = S.spense_set_log(2)
    try:
        t = inputs(M + N, M, K, N, R, count, "fp8", base, ints=True)
        capfd.readouterr()
        assert torch.equal(call(S, t, count, out_f32=True).cpu().double(), formula(*t)[0])
        assert chosen(capfd) == [(tokens, steps)]
    finally:
        S.spense_set_log(prev)
    t = inputs(M + N, M, K, N, R, count, "bf16", base)
    y = call(S, t, count, out_f32=base == "f32")
    want, e = formula(*t)
    assert torch.all((y.cpu().double() - want).abs() <= e + (U if base == "f32" else 2.0 ** -8) * (want.abs() + e) + 1e-38)
    pool, g = S.AdapterPool(*(v.cuda() for v in t[2:5])), S.group_rows(t[6].cuda(), count)
    over = torch.full((M, N + 3), 5.0, dtype=t[5].dtype, device="cuda")
    over[:, :N] = t[5].cuda()
    S.add_adapters(over[:, :N], t[0].cuda(), pool, g, out=over[:, :N], out_f32=base == "f32")
    assert torch.equal(over[:, :N], y) and torch.all(over[:, N:] == 5)


@pytest.mark.parametrize("kind", ["none", "one", "runs", "last"])
@pytest.mark.parametrize("M", [2, 150, 700])
def test_groupings(S, kind, M):
    """Nobody has an adapter, everybody the same, requests in runs of tokens, one token only."""
    count = 6
    idx = {"none": torch.full((M,), -1), "one": torch.full((M,), 4), "runs": torch.arange(M) // 37 % (count + 1),
           "last": torch.where(torch.arange(M) == M - 1, 5, -7)}[kind]
    t = inputs(M, M, 320, 296, 16, count, "bf16", "f32", idx=idx)
    y = call(S, t, count, out_f32=True).cpu()
    want, e = formula(*t)
    assert torch.all((y.double() - want).abs() <= e + U * want.abs())
    free = (t[6] < 0) | (t[6] >= count)
    assert torch.equal(y[free], t[5][free])


@pytest.mark.parametrize("N", [256, 300, 301])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_in_place_and_strides(S, N, dt):
    """out is base (rows without an adapter keep every bit, -0 and NaN among them), columns behind
    the rows stay; X and base inside wider buffers."""
    M, K, R, count = 90, 128, 16, 3
    t = list(inputs(9, M, K, N, R, count, "bf16", dt))
    t[5][0] = float("nan")
    t[5][1] = -0.0
    t[6][:2] = -1
    ref = call(S, t, count, out_f32=dt == "f32")
    wide = torch.full((M, N + 13), 5.0, dtype=t[5].dtype)
    wide[:, :N] = t[5]
    wide = wide.cuda()
    wx = torch.zeros(M, K + 24, dtype=torch.bfloat16)
    wx[:, :K] = t[0]
    pool = S.AdapterPool(*(v.cuda() for v in t[2:5]))
    g = S.group_rows(t[6].cuda(), count)
    y = S.add_adapters(wide[:, :N], wx.cuda()[:, :K], pool, g, out=wide[:, :N], out_f32=dt == "f32")
    assert y.data_ptr() == wide.data_ptr() and torch.all(wide[:, N:] == 5)
    bits = torch.int16 if dt == "bf16" else torch.int32
    assert torch.equal(y.contiguous().view(bits)[1:], ref.view(bits)[1:]) and torch.all(torch.isnan(y[0]))
    assert torch.equal(y[1].cpu().contiguous().view(bits), t[5][1].view(bits))


@pytest.mark.parametrize("M,N", [(6, 130), (200, 520)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rows_far_apart(S, M, N, dt):
    """Offsets past 32 bits in base and out."""
    K, R, count = 64, 16, 2
    t = inputs(13, M, K, N, R, count, "bf16", dt)
    f32 = dt == "f32"
    ref = call(S, t, count, out_f32=f32)
    pool = S.AdapterPool(*(v.cuda() for v in t[2:5]))
    pitch = -(-(9 << 29) // M) + 3
    far = torch.empty((M - 1) * pitch + N, dtype=t[5].dtype, device="cuda").as_strided((M, N), (pitch, 1))
    far.copy_(t[5])
    S.add_adapters(far, t[0].cuda(), pool, S.group_rows(t[6].cuda(), count), out=far, out_f32=f32)
    assert torch.equal(far.contiguous(), ref)


def test_non_finite_tokens_stay_alone(S):
    M, K, N, R = 20, 256, 64, 16
    t = inputs(3, M, K, N, R, 1, "bf16", "f32", idx=torch.zeros(M))
    clean = call(S, t, 1, out_f32=True)
    t[0][4, 9], t[0][7, 3] = float("nan"), float("inf")
    y = call(S, t, 1, out_f32=True)
    assert torch.all(torch.isnan(y[4])) and not torch.any(torch.isfinite(y[7]))
    keep = [m for m in range(M) if m not in (4, 7)]
    assert torch.equal(y[keep], clean[keep])
    q = inputs(3, M, K, N, R, 1, "fp8", "f32", idx=torch.zeros(M))
    q[0].view(torch.uint8)[5, 1] = 0x7F
    y = call(S, q, 1, out_f32=True)
    assert torch.all(torch.isnan(y[5])) and torch.all(torch.isfinite(y[6]))


def test_non_finite_entries_of_a_pool_stay_where_they_belong(S):
    """An infinity or NaN in A reaches its adapter's tokens, one in B one column of these; nothing else changes."""
    M, K, N, R, count = 40, 256, 72, 16, 3
    t = inputs(4, M, K, N, R, count, "bf16", "f32", idx=torch.arange(M) % (count + 1))
    clean = call(S, t, count, out_f32=True)
    t[2][0, 5, 7], t[3][1, 33, 2], t[3][2, 70, 11] = float("inf"), float("inf"), float("nan")
    y = call(S, t, count, out_f32=True)
    hit = torch.zeros(M, N, dtype=torch.bool)
    hit[t[6] == 0], hit[t[6] == 1, 33], hit[t[6] == 2, 70] = True, True, True
    hit = hit.cuda()
    assert torch.equal(y[~hit], clean[~hit]) and not torch.any(torch.isfinite(y[hit]))


def test_rows_outside_are_skipped(S):
    """order and offsets of another making: entries outside [0, M) and offsets past M name nothing."""
    M, K, N, R = 40, 64, 128, 8
    t = inputs(5, M, K, N, R, 2, "bf16", "f32", idx=torch.zeros(M))
    pool = S.AdapterPool(*(v.cuda() for v in t[2:5]))
    order = torch.arange(M, dtype=torch.int32)
    order[3], order[8] = -5, 2 ** 30
    offsets = torch.tensor([-4, 20, 10 ** 9], dtype=torch.int32)
    g = S.RowGroups(M, 2, torch.cat([order, order, offsets]).cuda())
    out = torch.full((M, N), 7.0, device="cuda")
    S.add_adapters(t[5].cuda(), t[0].cuda(), pool, g, out=out, out_f32=True)
    t[6][:], t[6][20:] = 0, 1
    want, e = formula(*t)
    keep = [m for m in range(M) if m not in (3, 8)]
    assert torch.all((out.cpu().double() - want).abs()[keep] <= (e + U * want.abs())[keep]) and torch.all(out[[3, 8]] == 7)


def test_two_streams_and_graph(S):
    """Calls in flight together hold workspaces of their own; a captured call replays on new inputs."""
    ts = [inputs(s, 48, 2048, 1024, 16, 8, "bf16", "f32") for s in (1, 2)]
    refs = [call(S, t, 8) for t in ts]
    dev = [[None if v is None else v.cuda() for v in t] for t in ts]
    pools = [S.AdapterPool(*d[2:5]) for d in dev]
    groups = [S.group_rows(d[6], 8) for d in dev]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        outs = []
        for d, p, g, s in zip(dev, pools, groups, streams):
            with torch.cuda.stream(s):
                outs.append(S.add_adapters(d[5], d[0], p, g))
        torch.cuda.synchronize()
        assert all(torch.equal(o, r) for o, r in zip(outs, refs))
    graph = torch.cuda.CUDAGraph()
    X, idx, base = dev[0][0], dev[0][6], dev[0][5]
    with torch.cuda.graph(graph):
        o = S.add_adapters(base, X, pools[0], S.group_rows(idx, 8))
    for seed in (7, 8, 9):
        t = inputs(seed, 48, 2048, 1024, 16, 8, "bf16", "f32")
        for dst, src in ((X, t[0]), (idx, t[6]), (base, t[5])):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, S.add_adapters(base, X, pools[0], S.group_rows(idx, 8)))


@pytest.mark.parametrize("M", [5, 130])
def test_gemm_adapters(S, M):
    """A Spense projection with adapters on its own codes, and on other activations."""
    import gen

    N, K, R, count = 512, 1024, 16, 5
    mx = gen.make_matrix(3, 0, "w", N, K, gen.OUTPUT, 0.25, gen.FP8)
    pw = S.tile(S.compress(torch.from_numpy(mx.W).cuda(), torch.from_numpy(mx.mask).cuda(), 0, mx.dense_begin))
    sw = torch.from_numpy(mx.sw).cuda()
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(M)).bfloat16().cuda()
    q, xs = S.quantize_fp8(x)
    t = inputs(M, M, K, N, R, count, "bf16", "f32")
    pool, g = S.AdapterPool(*(v.cuda() for v in t[2:5])), S.group_rows(t[6].cuda(), count)
    base = S.gemm(q, pw, sw, xs, out_f32=True)
    for f32 in (False, True):
        y = S.gemm_adapters(q, pw, pool, g, sw, xs, out_f32=f32)
        assert torch.equal(y, S.add_adapters(base, q, pool, g, xs, out_f32=f32))
        y = S.gemm_adapters(q, pw, pool, g, sw, xs, A_x=x, out_f32=f32)
        assert torch.equal(y, S.add_adapters(base, x, pool, g, out_f32=f32))


@pytest.mark.parametrize("x", ["fp8", "bf16"])
def test_one_row_of_an_odd_pitch(S, x):
    """A single token that is a row of a wider buffer, whatever the pitch (one row has none), in
    add_adapters and in gemm_adapters."""
    import gen

    N, K, R, count = 512, 1024, 16, 5
    t = inputs(17, 1, K, N, R, count, x, "f32", idx=torch.tensor([3]))
    pool, g, bd = S.AdapterPool(*(v.cuda() for v in t[2:5])), S.group_rows(t[6].cuda(), count), t[5].cuda()
    X, xs = t[0].cuda(), None if t[1] is None else t[1].cuda()
    X = X.view(torch.uint8) if x == "fp8" else X
    ref = S.add_adapters(bd, X, pool, g, x_scale=xs)
    wide = torch.zeros(3, K + 5, dtype=X.dtype, device="cuda")
    wide[0, :K] = X[0]
    for row in (wide[:1, :K], wide[0, :K].expand(1, K)):
        assert torch.equal(S.add_adapters(bd, row, pool, g, x_scale=xs), ref)
    if x == "fp8":
        mx = gen.make_matrix(3, 0, "w", N, K, gen.OUTPUT, 0.25, gen.FP8)
        pw = S.tile(S.compress(torch.from_numpy(mx.W).cuda(), torch.from_numpy(mx.mask).cuda(), 0, mx.dense_begin))
        sw = torch.from_numpy(mx.sw).cuda()
        assert torch.equal(S.gemm_adapters(wide[:1, :K], pw, pool, g, sw, xs), S.gemm_adapters(X, pw, pool, g, sw, xs))


def test_binding_refuses(S):
    t = inputs(1, 8, 64, 32, 8, 2, "bf16", "f32")
    X, _, A, B, sc, bd, idx = [None if v is None else v.cuda() for v in t]
    pool, g = S.AdapterPool(A, B, sc), S.group_rows(idx, 2)
    for bad in ((A.float(), B), (A, B[:, :, :4]), (A[:1], B), (A.transpose(1, 2), B), (A, B, sc[:1]), (A, B.cpu())):
        with pytest.raises((ValueError, TypeError)):
            S.AdapterPool(*bad)
    for kw in (dict(X=X[:4]), dict(X=X.float()), dict(X=X[:, :32]), dict(X=X[0].expand(8, 64)),
               dict(base=bd[0].expand(8, 32)), dict(base=bd[:, :8]), dict(base=bd.half()),
               dict(groups=S.group_rows(idx, 3)), dict(groups=S.group_rows(idx[:4], 2)), dict(x_scale=sc),
               dict(out=torch.zeros(8, 31, dtype=torch.bfloat16, device="cuda")), dict(X=X.view(torch.int16))):
        with pytest.raises((ValueError, TypeError)):
            S.add_adapters(**{"base": bd, "X": X, "pool": pool, "groups": g, **kw})
    with pytest.raises(S.SpenseError):  # rank 4
        S.add_adapters(bd, X, S.AdapterPool(A[:, :4].contiguous(), B[:, :, :4].contiguous()), g)
    assert S.add_adapters(bd[:0], X[:0], pool, S.group_rows(idx[:0], 2)).shape == (0, 32)
