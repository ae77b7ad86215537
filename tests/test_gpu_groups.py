"""spense_group_rows and spense_combine_rows through the binding: the first against a stable
sort, the second against 64-bit sums (a sum of `top` fused products in fp32 is within top u of
the sum of their magnitudes, u = 2^-24, plus half a step of the output type)."""
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def S():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_10445_amd as S
    return S


def sorted_rows(idx, groups):
    key = np.where((idx >= 0) & (idx < groups), idx, groups)
    order = np.argsort(key, kind="stable")
    offsets = np.searchsorted(key[order], np.arange(groups + 1), side="left")
    inverse = np.empty(len(idx), np.int64)
    inverse[order] = np.arange(len(idx))
    return order, np.where(key < groups, inverse, -1), offsets


@pytest.mark.parametrize("groups", [1, 2, 7, 64, 511, 512, 1000, 1024])
@pytest.mark.parametrize("n", [0, 1, 63, 64, 65, 1000, 1025, 20011])
def test_group_rows(S, n, groups):
    print(f"[group] n={n} groups={groups}", file=sys.stderr, flush=True)
    r = np.random.default_rng(n + 7 * groups)
    for kind in ("even", "skewed", "one", "none"):
        if kind == "even":
            idx = r.integers(-2, groups + 2, n)
        elif kind == "skewed":
            idx = np.minimum(r.geometric(0.3, n) - 1, groups)
        elif kind == "one":
            idx = np.full(n, groups - 1)
        else:
            idx = np.where(r.random(n) < 0.5, -2 ** 31, 2 ** 31 - 1)
        idx = idx.astype(np.int32)
        g = S.group_rows(torch.from_numpy(idx).cuda(), groups)
        order, inverse, offsets = sorted_rows(idx, groups)
        assert np.array_equal(g.order.cpu().numpy(), order)
        assert np.array_equal(g.inverse.cpu().numpy(), inverse)
        assert np.array_equal(g.offsets.cpu().numpy(), offsets)


def test_group_rows_replayed(S):
    idx = torch.zeros(700, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = S.group_rows(idx, 33)
    for seed in range(4):
        new = np.random.default_rng(seed).integers(-1, 34, 700).astype(np.int32)
        idx.copy_(torch.from_numpy(new))
        g.replay()
        torch.cuda.synchronize()
        order, inverse, offsets = sorted_rows(new, 33)
        assert np.array_equal(o.order.cpu().numpy(), order) and np.array_equal(o.offsets.cpu().numpy(), offsets)
        assert np.array_equal(o.inverse.cpu().numpy(), inverse)


@pytest.mark.parametrize("T,top,N", [(1, 1, 1), (3, 2, 255), (17, 8, 1024), (64, 6, 5120), (5, 3, 1030), (2, 4, 2052)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("out_f32", [False, True])
def test_combine_rows(S, T, top, N, dt, out_f32):
    gen = torch.Generator().manual_seed(T + N)
    idx = torch.randint(-1, 9, (T * top,), generator=gen, dtype=torch.int32)
    idx[:top] = -1  # a token without any row
    D, w = torch.randn(T * top, N, generator=gen).to(dt), torch.randn(T, top, generator=gen)
    g = S.group_rows(idx.cuda(), 8)
    inv = g.inverse.cpu().long()
    Dg = D.cuda()
    Dg[int(g.offsets[-1]):] = float("nan")  # rows in no group are not read
    y = S.combine_rows(Dg, g, w.cuda(), top, out_f32=out_f32)
    terms = torch.where((inv >= 0)[:, None], w.reshape(-1, 1).double() * D.double()[inv.clamp_min(0)], 0.0).reshape(T, top, N)
    want, mag = terms.sum(1), terms.abs().sum(1)
    half = U if out_f32 else 2.0 ** -8
    assert torch.all((y.cpu().double() - want).abs() <= top * U * mag + half * (want.abs() + top * U * mag) + 1e-38)
    assert torch.all(y[0] == 0)
    plain = S.combine_rows(Dg, g, None, top, out_f32=True)  # ones
    terms = torch.where((inv >= 0)[:, None], D.double()[inv.clamp_min(0)], 0.0).reshape(T, top, N)
    assert torch.all((plain.cpu().double() - terms.sum(1)).abs() <= (top + 1) * U * terms.abs().sum(1))


def test_combine_rows_far_apart(S):
    """Offsets past 32 bits: rows of D and Y 2^30 elements apart."""
    T, top, N, pitch = 3, 2, 260, 1 << 30
    idx = torch.tensor([2, 0, 1, 1, 3, 0], dtype=torch.int32).cuda()
    g = S.group_rows(idx, 3)
    D = torch.empty(5 * pitch + N, device="cuda").as_strided((6, N), (pitch, 1))
    D.copy_(torch.randn(6, N, generator=torch.Generator().manual_seed(3)))
    w = torch.rand(T, top, generator=torch.Generator().manual_seed(4)).cuda()
    out = torch.empty(2 * pitch + N, device="cuda").as_strided((T, N), (pitch, 1))
    S.combine_rows(D, g, w, top=top, out=out, out_f32=True)
    assert torch.equal(out, S.combine_rows(D.contiguous(), g, w, top=top, out_f32=True))


def test_combine_rows_strided(S):
    T, top, N = 9, 2, 100
    gen = torch.Generator().manual_seed(5)
    g = S.group_rows(torch.randint(0, 4, (T * top,), generator=gen, dtype=torch.int32).cuda(), 4)
    D = torch.randn(T * top, 131, generator=gen).cuda()
    out = torch.full((T, 117), 3.0, dtype=torch.bfloat16, device="cuda")
    w = torch.randn(T, top, generator=gen).cuda()
    S.combine_rows(D[:, 3:103], g, w, top, out=out[:, :N])
    assert torch.equal(out[:, :N], S.combine_rows(D[:, 3:103].contiguous(), g, w, top)) and torch.all(out[:, N:] == 3)


def test_binding_refuses(S):
    idx = torch.zeros(8, dtype=torch.int32, device="cuda")
    for bad in (idx.long(), idx.cpu(), idx.reshape(2, 4), idx[::2]):
        with pytest.raises(ValueError):
            S.group_rows(bad, 4)
    for groups in (0, -3, 1025):
        with pytest.raises(S.SpenseError):
            S.group_rows(idx, groups)
    g = S.group_rows(idx, 4)
    D = torch.zeros(8, 16, device="cuda")
    for kw in (dict(D=D[:7]), dict(top=3), dict(top=0), dict(weights=torch.zeros(4, device="cuda")),
               dict(weights=torch.zeros(8, device="cuda").half()), dict(D=D[0].expand(8, 16)),
               dict(out=torch.zeros(3, 16, device="cuda"))):
        with pytest.raises(ValueError):
            S.combine_rows(**{"D": D, "groups": g, "top": 2, **kw})
