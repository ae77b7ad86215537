"""Refusals of the norm, grouping, adapter and expert calls before anything touches a device
(CPU): pointers are made-up addresses."""
import pytest

A = 1 << 20  # a 16-byte aligned address that nothing reads


@pytest.fixture(scope="module")
def S():
    import paper_2606_10445_amd as S
    return S


def norm_args(S, **kw):
    a = dict(M=4, K=64, x=A, ldx=64, x_type=2, y_type=2, y=A, ldy=64, gate=A, ldg=0, post_weight=A, weight=A, w_type=3,
             residual_scale=1.0, eps=1e-6, residual=A, ldr=64, normed=A, ldn=64, q=A, ldq=64, scales=A)
    a.update(kw)
    return S.spense_block_norm_t(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(M=-1), -1), (dict(K=-1), -1), (dict(M=1 << 31), -1), (dict(K=1 << 31), -1),
    (dict(x_type=1), -1), (dict(y_type=0), -1), (dict(w_type=9), -1), (dict(eps=-1e-6), -1), (dict(eps=float("nan")), -1),
    (dict(eps=float("inf")), -1), (dict(y=None), -1), (dict(y=None, gate=None), -1), (dict(q=None), -1),
    (dict(scales=None), -1), (dict(residual=None, normed=None, q=None, scales=None), -1), (dict(ldx=63), -1),
    (dict(ldy=1), -1), (dict(ldg=8), -1), (dict(ldr=0), -1), (dict(ldn=63), -1), (dict(ldq=63), -1),
    (dict(x=A + 1), -2), (dict(y=A + 1), -2), (dict(weight=A + 2), -2), (dict(normed=A + 1), -2), (dict(scales=A + 2), -2),
])
def test_block_norm_refuses(S, kw, code):
    assert S.spense_block_norm(norm_args(S, **kw), None) == code
    assert S.spense_last_error()


def test_block_norm_of_nothing(S):
    assert S._lib.spense_block_norm(None, None) == -1
    assert S.spense_block_norm(norm_args(S, M=0, x=None), None) == 0
    assert S.spense_block_norm(norm_args(S, K=0, x=None), None) == 0
    assert S.spense_last_error() == ""


@pytest.mark.parametrize("args", [(A, -1, 4, A, A, A), (A, 1 << 31, 4, A, A, A), (A, 8, 0, A, A, A), (A, 8, 1025, A, A, A),
                                  (None, 8, 4, A, A, A), (A, 8, 4, None, A, A), (A, 8, 4, A, A, None)])
def test_group_rows_refuses(S, args):
    assert S.spense_group_rows(*args, None) == -1


def test_combine_rows_refuses(S):
    good = dict(D=A, d_type=2, n=8, ldd=16, inverse=A, weights=A, T=4, top=2, N=16, Y=A, ldy=16, out_flags=0, stream=None)
    for kw, code in ((dict(D=None), -1), (dict(inverse=None), -1), (dict(Y=None), -1), (dict(d_type=1), -1),
                     (dict(n=-1), -1), (dict(T=-1), -1), (dict(N=-1), -1), (dict(top=0), -1), (dict(ldd=15), -1),
                     (dict(ldy=15), -1), (dict(out_flags=2), -1), (dict(T=1 << 30, top=4), -1), (dict(D=A + 1), -2),
                     (dict(Y=A + 1), -2), (dict(T=1 << 24, N=1 << 20, ldd=1 << 20, ldy=1 << 20), -1)):
        assert S.spense_combine_rows(**{**good, **kw}) == code, kw
    assert S.spense_combine_rows(**{**good, "T": 0}) == 0 and S.spense_combine_rows(**{**good, "N": 0, "Y": None}) == 0
