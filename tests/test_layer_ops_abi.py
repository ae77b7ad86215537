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
             residual_scale=1.0, eps=1e-6, residual=2 * A, ldr=64, normed=3 * A, ldn=64, q=A, ldq=64, scales=A)
    a.update(kw)
    return S.spense_block_norm_t(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(M=-1), -1), (dict(K=-1), -1), (dict(M=1 << 31), -1), (dict(K=1 << 31), -1),
    (dict(x_type=1), -1), (dict(y_type=0), -1), (dict(w_type=9), -1), (dict(eps=-1e-6), -1), (dict(eps=float("nan")), -1),
    (dict(eps=float("inf")), -1), (dict(y=None), -1), (dict(y=None, gate=None), -1), (dict(q=None), -1),
    (dict(scales=None), -1), (dict(residual=None, normed=None, q=None, scales=None), -1), (dict(ldx=63), -1),
    (dict(ldy=1), -1), (dict(ldg=8), -1), (dict(ldr=0), -1), (dict(ldn=63), -1), (dict(ldq=63), -1),
    (dict(x=A + 1), -2), (dict(y=A + 1), -2), (dict(weight=A + 2), -2), (dict(normed=A + 1), -2), (dict(scales=A + 2), -2),
    (dict(y=2 * A), -1), (dict(normed=2 * A), -1), (dict(x=3 * A), -1), (dict(M=1 << 28), -1),
    (dict(M=1 << 22, K=520, ldx=520, ldy=520, ldr=520, ldn=520, ldq=520), -1), (dict(M=1 << 22, K=4), -1),
])
def test_block_norm_refuses(S, kw, code):
    assert S.spense_block_norm(norm_args(S, **kw), None) == code
    assert S.spense_last_error()


@pytest.mark.parametrize("kw", [dict(residual=A, ldr=72), dict(normed=A, ldn=72), dict(residual=A, ldx=72),
                                dict(normed=A, ldy=128, K=32)])
def test_block_norm_refuses_an_input_overwritten_at_another_pitch(S, kw):
    """In place, a row's outputs would go over other rows' inputs before these are read."""
    x, y = (A, 5 * A) if "residual" in kw else (5 * A, A)
    base = dict(x=x, y=y, residual=6 * A, normed=7 * A, q=8 * A, gate=9 * A, weight=10 * A, post_weight=11 * A)
    assert S.spense_block_norm(norm_args(S, **{**base, **kw}), None) == -1
    assert "leading dimension" in S.spense_last_error()


def test_block_norm_of_nothing(S):
    assert S._lib.spense_block_norm(None, None) == -1
    assert S.spense_block_norm(norm_args(S, K=0), None) == -1
    assert S.spense_block_norm(norm_args(S, M=0, x=None), None) == 0
    assert S.spense_last_error() == ""


@pytest.mark.parametrize("args", [(A, -1, 4, A, A, A), (A, (1 << 20) + 1, 4, A, A, A), (A, 8, 0, A, A, A),
                                  (A, 8, 1025, A, A, A), (None, 8, 4, A, A, A), (A, 8, 4, None, A, A), (A, 8, 4, A, A, None)])
def test_group_rows_refuses(S, args):
    assert S.spense_group_rows(*args, None) == -1


def test_combine_rows_refuses(S):
    good = dict(D=A, d_type=2, n=8, ldd=16, inverse=A, weights=A, T=4, top=2, N=16, Y=2 * A, ldy=16, out_flags=0, stream=None)
    for kw, code in ((dict(D=None), -1), (dict(inverse=None), -1), (dict(Y=None), -1), (dict(d_type=1), -1),
                     (dict(n=-1), -1), (dict(T=-1), -1), (dict(N=-1), -1), (dict(top=0), -1), (dict(ldd=15), -1),
                     (dict(ldy=15), -1), (dict(out_flags=2), -1), (dict(T=1 << 18, top=5), -1), (dict(n=(1 << 20) + 1), -1), (dict(Y=A), -1), (dict(D=A + 1), -2),
                     (dict(Y=A + 1), -2), (dict(T=1 << 19, N=1 << 20, ldd=1 << 20, ldy=1 << 20), -1)):
        assert S.spense_combine_rows(**{**good, **kw}) == code, kw
    assert S.spense_combine_rows(**{**good, "T": 0}) == 0 and S.spense_combine_rows(**{**good, "N": 0, "Y": None}) == 0


def pool(S, **kw):
    return S.spense_adapters_t(**{**dict(count=4, R=16, K=64, N=48, A=A, B=A, scale=None), **kw})


def test_add_adapters_refuses(S):
    good = dict(X=A, x_type=2, M=8, ldx=64, x_scale=None, order=A, offsets=A, base=A, base_type=3, ldb=48, Y=2 * A, ldy=48,
                out_flags=0, ws=A, ws_bytes=1 << 20, stream=None)

    def call(pool_kw={}, **kw):
        return S.spense_add_adapters(pool=pool(S, **pool_kw), **{**good, **kw})

    for kw, code in ((dict(X=None), -1), (dict(order=None), -1), (dict(offsets=None), -1), (dict(base=None), -1),
                     (dict(Y=None), -1), (dict(x_type=3), -1), (dict(base_type=1), -1), (dict(out_flags=4), -1),
                     (dict(M=-1), -1), (dict(M=(1 << 20) + 1), -1), (dict(ldx=63), -1), (dict(ldb=47), -1), (dict(ldy=47), -1),
                     (dict(X=A + 2), -2), (dict(ldx=68), -2), (dict(base=A + 2), -2), (dict(Y=A + 1), -2),
                     (dict(Y=A), -1),  # base in the place of Y, of another type
                     (dict(Y=A, out_flags=1, ldy=64), -1), (dict(ws=None), -4), (dict(ws_bytes=0), -4),
                     (dict(ws=A + 8), -2)):
        assert call(**kw) == code, kw
    for kw, code in ((dict(count=0), -1), (dict(count=1025), -1), (dict(R=0), -1), (dict(R=12), -1), (dict(R=136), -1),
                     (dict(K=0), -1), (dict(N=0), -1), (dict(K=48), -2), (dict(A=None), -1), (dict(B=None), -1),
                     (dict(A=A + 8), -2), (dict(K=1 << 27), -1)):
        assert call(kw, ldx=max(64, kw.get("K", 64))) == code, kw
        if "A" not in kw and "B" not in kw and kw.get("K") != 1 << 27:
            assert S.spense_adapters_workspace_size(8, pool(S, **kw)) == 0
    big = dict(M=1 << 20, ldb=1 << 21, ldy=1 << 21, ws_bytes=1 << 40)
    assert call(dict(N=1 << 21), **big) == -1 and "grid" in S.spense_last_error()
    assert S._lib.spense_add_adapters(A, 2, 8, 64, None, A, A, None, A, 3, 48, A, 48, 0, A, 1 << 20, None) == -1
    assert call(M=0) == 0 and S.spense_adapters_workspace_size(0, pool(S)) == 0
    need = S.spense_adapters_workspace_size(8, pool(S))
    assert need >= 8 * 16 * 4 and call(ws_bytes=need - 1) == -4


def test_adapter_workspace_grows_with_the_batch(S):
    """The workspace of a batch covers 1 to 8 slices of M x R fp32 sums, whatever the sizes."""
    for M in (1, 2, 15, 16, 17, 63, 64, 127, 128, 2048, 100000):
        for count in (1, 3, 64, 1024):
            for K in (32, 512, 5120, 25600):
                for R in (8, 16, 40, 64, 72, 128):
                    n = S.spense_adapters_workspace_size(M, pool(S, count=count, K=K, R=R))
                    assert n % (M * R * 4) == 0 and 1 <= n // (M * R * 4) <= min(8, max(1, -(-K // 512)))


def test_gemm_experts_refuses(S):
    import ctypes

    P = ctypes.POINTER(S.spense_packed_t)

    def desc(**kw):
        d = dict(dtype=1, split=0, N=64, K=128, dense_begin=32, values=A, values_ld=64, meta=A, meta_ld=4, dense=A,
                 dense_ld=128, layout=1)
        return S.spense_packed_t(**{**d, **kw})

    def call(descs=None, Y=(2 * A,), ldy=(64,), **kw):
        descs = [desc()] if descs is None else descs
        k = max(1, len(descs))
        parr = (P * k)(*[None if d is None else ctypes.pointer(d) for d in descs])
        a = dict(X=A, rows_x=8, ldx=128, x_scale=None, order=A, top=1, offsets=A, n=8, count=4, weights=len(descs),
                 packed_array=parr, w_scales_array=None, Y_array=(ctypes.c_void_p * len(Y))(*Y),
                 ldy_array=(ctypes.c_int64 * len(ldy))(*ldy), out_flags=0, stream=None)
        return S.spense_gemm_experts(**{**a, **kw})

    for kw, code in ((dict(X=None), -1), (dict(offsets=None), -1), (dict(rows_x=-1), -1), (dict(n=-1), -1),
                     (dict(n=(1 << 20) + 1), -1),
                     (dict(top=0), -1), (dict(count=0), -1), (dict(count=1025), -1), (dict(weights=0), -1), (dict(weights=3), -1),
                     (dict(packed_array=None), -1), (dict(Y_array=None), -1), (dict(ldy_array=None), -1), (dict(out_flags=2), -1),
                     (dict(ldx=127), -1), (dict(ldx=136), -2), (dict(X=A + 8), -2), (dict(Y=(None,)), -1), (dict(Y=(A + 1,)), -2),
                     (dict(ldy=(63,)), -1), (dict(rows_x=1 << 30), -1)):
        assert call(**kw) == code, kw
        assert S.spense_last_error()
    for bad, code in ((dict(layout=0), -1), (dict(dtype=2), -1), (dict(K=96 + 8), -2), (dict(values=None), -1), (dict(dense=A + 8), -2),
                      (dict(K=0), -1), (dict(dense_begin=65), -1)):
        assert call([desc(**bad)]) == code, bad
    assert call([None]) == -1
    two = dict(Y=(2 * A, 4 * A), ldy=(64, 64))
    for bad in (dict(N=80), dict(K=160), dict(dense_begin=48), dict(split=1)):
        assert call([desc(), desc(**bad)], **two) == -1, bad
    assert call([desc(), desc()], Y=(2 * A, 2 * A), ldy=(64, 64)) == -1
    wide = dict(N=1 << 20, dense_begin=0, values=None, meta=None, K=512, dense_ld=512)
    assert call([desc(**wide)], n=1 << 20, ldy=(1 << 20,), ldx=512) == -1 and "grid" in S.spense_last_error()
    assert call(n=0, X=None) == 0


def test_gemm_experts_glu_refuses(S):
    import ctypes

    def desc(**kw):
        d = dict(dtype=1, split=0, N=64, K=128, dense_begin=32, values=A, values_ld=64, meta=A, meta_ld=4, dense=A,
                 dense_ld=128, layout=1)
        return S.spense_packed_t(**{**d, **kw})

    size = S.spense_gemm_experts_glu_fp8_workspace_size

    def call(gate={}, up={}, **kw):
        a = dict(X=A, rows_x=8, ldx=128, x_scale=None, order=A, top=1, offsets=A, n=8, count=4,
                 gate=None if gate is None else ctypes.byref(desc(**gate)),
                 up=None if up is None else ctypes.byref(desc(**up)), w_scale_gate=None, w_scale_up=None, q=A, ldq=64,
                 scales=A, ws=A, ws_bytes=size(8, 4, 64), stream=None)
        return S._lib.spense_gemm_experts_glu_fp8(*{**a, **kw}.values())

    for kw, code in ((dict(X=None), -1), (dict(offsets=None), -1), (dict(rows_x=-1), -1), (dict(n=-1), -1),
                     (dict(n=(1 << 20) + 1), -1), (dict(top=0), -1), (dict(count=0), -1), (dict(count=1025), -1),
                     (dict(gate=None), -1), (dict(up=None), -1), (dict(ldx=127), -1), (dict(ldx=136), -2), (dict(X=A + 8), -2),
                     (dict(q=None), -1), (dict(scales=None), -1), (dict(ldq=63), -1), (dict(ws=None), -4),
                     (dict(ws_bytes=size(8, 4, 64) - 1), -4), (dict(ws=A + 128), -2)):
        assert call(**kw) == code, kw
        assert S.spense_last_error()
    for bad in (dict(N=80), dict(K=160), dict(dense_begin=48), dict(split=1), dict(dtype=2), dict(layout=0)):
        assert call(up=bad) == -1, bad
    assert call(gate=dict(split=1), up=dict(split=1)) == -1
    assert call(n=0, X=None, q=None, ws=None) == 0 and S.spense_last_error() == ""


def test_glu_workspace_size(S):
    """fp32 G and U, or H and its maxima, of every row; 0 for sizes that the call refuses."""
    size = S.spense_gemm_experts_glu_fp8_workspace_size
    for bad in ((0, 4, 64), (-1, 4, 64), ((1 << 20) + 1, 4, 64), (8, 0, 64), (8, 1025, 64), (8, 4, 0), (8, 4, 1 << 31)):
        assert size(*bad) == 0, bad
    for n in (1, 2, 17, 300, 4096, 100000, 1 << 20):
        for count in (1, 5, 64, 1024):
            for N in (1, 16, 100, 1536, 25600):
                assert n * N * 4 < size(n, count, N) <= 2 * (n * (N + 63) * 4 + 256)


def test_the_pitch_of_a_single_row_does_not_matter(S):
    """One activation row may come from a buffer of any pitch; seen by the next refusal of such a call."""
    import ctypes

    args = dict(X=A, x_type=2, M=1, ldx=65, x_scale=None, order=A, offsets=A, pool=pool(S), base=A, base_type=3, ldb=48,
                Y=2 * A, ldy=48, out_flags=0, ws=None, ws_bytes=0, stream=None)
    assert S.spense_add_adapters(**args) == -4
    assert S.spense_add_adapters(**{**args, "x_type": 1}) == -4
    assert S.spense_add_adapters(**{**args, "M": 2}) == -2
    assert S.spense_add_adapters(**{**args, "ldx": 63}) == -1
    d = S.spense_packed_t(1, 0, 64, 128, 32, A, 64, A, 4, A, 128, 1)

    def glu(rows_x, ldx):
        return S.spense_gemm_experts_glu_fp8(A, rows_x, ldx, None, A, 8, A, 8, 4, ctypes.byref(d), ctypes.byref(d), None,
                                             None, A, 64, A, None, 0, None)

    assert glu(1, 129) == -4 and glu(2, 129) == -2 and glu(1, 127) == -1


def test_gemm_adapters_makes_its_device_current(S, monkeypatch):
    """The projection of gemm_adapters runs with the tensors' device current, as the adapters do."""
    import contextlib
    from types import SimpleNamespace

    import torch

    entered, calls = [], []

    @contextlib.contextmanager
    def device(dev):
        entered.append(dev)
        yield
        entered.pop()

    monkeypatch.setattr(S, "_device", device)
    monkeypatch.setattr(S, "_on_gpu", lambda dev, *tensors: None)
    monkeypatch.setattr(S, "gemm", lambda X, *a, **kw: calls.append(list(entered)) or X)
    monkeypatch.setattr(S, "add_adapters", lambda base, *a, **kw: base)
    X = torch.zeros(2, 32)
    S.gemm_adapters(X, SimpleNamespace(N=8, dense=X), SimpleNamespace(N=8, A=X), None)
    assert calls == [[X.device]]


def test_gemm_adapters_refuses_tensors_on_the_cpu(S):
    from types import SimpleNamespace

    import torch

    X = torch.zeros(2, 32)
    with pytest.raises(ValueError, match="GPU"):
        S.gemm_adapters(X, SimpleNamespace(N=8, dense=X), SimpleNamespace(N=8, A=X), None)


def test_row_tiles_a_wave_rule(S, capfd):
    """The short-K kernel and its row tiles a wave at the sizes that the GPU tests of them take, by the dispatch log."""
    import ctypes

    import torch
    from test_gpu_experts import STREAMS, launches

    if torch.cuda.is_available():
        pytest.skip("made-up addresses: the calls must end at the device check")
    prev = S.spense_set_log(2)
    try:
        for n, E, N, K, split, db, k, positions, tiles in STREAMS:
            d = S.spense_packed_t(1, split, N, K, db, A, K, A, K, A, K, 1)
            parr = (ctypes.POINTER(S.spense_packed_t) * k)(*[ctypes.pointer(d)] * k)
            yarr, larr = (ctypes.c_void_p * k)(*[A * (2 + i) for i in range(k)]), (ctypes.c_int64 * k)(*[N] * k)
            capfd.readouterr()
            assert S.spense_gemm_experts(A, n, K, None, A, 1, A, n, E, k, parr, None, yarr, larr, 0, None) < 0
            assert launches(capfd) == [("stream", positions, tiles)]
    finally:
        S.spense_set_log(prev)
    assert {(t[7], t[8]) for t in STREAMS} == {(p, t) for p in (16, 32, 64) for t in range(2, 9)}


def test_adapter_columns_rule(S, capfd):
    """Tokens of a tile and steps of a workgroup at the sizes that the GPU tests of them take, by the dispatch log;
    the calls end at the missing workspace."""
    from test_gpu_adapters import WIDE, chosen

    prev = S.spense_set_log(2)
    try:
        for M, K, N, R, count, tokens, steps in WIDE:
            capfd.readouterr()
            assert S.spense_add_adapters(A, 2, M, K, None, A, A, pool(S, count=count, R=R, K=K, N=N), A, 3, N, 2 * A, N, 0,
                                         None, 0, None) == -4
            assert chosen(capfd) == [(tokens, steps)]
    finally:
        S.spense_set_log(prev)
    assert {t[5:] for t in WIDE} == {(16, 4), (16, 8), (32, 4)}
