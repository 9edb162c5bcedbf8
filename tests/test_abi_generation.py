"""Refusals of the generation-step operators, without a GPU: every C call here fails
validation (its addresses are made up and never read), every binding call fails
before the library is reached."""
import ctypes
import os

import pytest
import torch

from paper_2502_19405_amd import repops as rp

A, B, C, D, E, F, G, W = (0x1000000 * (i + 1) for i in range(8))
no_gpu_only = pytest.mark.skipif(os.path.exists("/dev/kfd"),
                                 reason="fake-pointer validation tests run only without a GPU")
FAR = (1 << 31) - 1


def order(**kw):
    return ctypes.byref(rp.Order(**kw).c())


def launch(kind, p=()):
    return ctypes.byref(rp.Launch(kind, p).c())


def refuse(base, call, cases):
    """call(**base with a case's changes) gives the case's status."""
    for change, want in cases:
        assert set(change) <= set(base), change
        assert call(**{**base, **change}) == want, change


@no_gpu_only
def test_add_rmsnorm_rows_refusals():
    f = rp.load().repops_add_rmsnorm_rows

    def call(o, rows, cols, X, ldx, R, ldr, gamma, S, lds, Y, ldy, Q, ldq, scale, rstd, launch):
        return f(o, rows, cols, X, ldx, R, ldr, gamma, 1e-5, S, lds, Y, ldy, Q, ldq, scale, rstd,
                 launch, None)
    base = dict(o=order(), rows=4, cols=8, X=A, ldx=8, R=B, ldr=8, gamma=C, S=D, lds=8, Y=E, ldy=8,
                Q=F, ldq=8, scale=G, rstd=W, launch=None)
    wave = rp.LAUNCH_ROWS_WAVE
    refuse(base, call, [
        (dict(o=None), rp.ERR_ORDER), (dict(o=order(version=2)), rp.ERR_ORDER),
        (dict(o=order(row_width=3)), rp.ERR_ORDER),
        (dict(rows=-1), rp.ERR_SHAPE), (dict(cols=-1), rp.ERR_SHAPE), (dict(cols=0), rp.ERR_SHAPE),
        (dict(rows=FAR + 1), rp.ERR_SHAPE), (dict(cols=(1 << 24) + 1, ldx=1 << 25), rp.ERR_SHAPE),
        (dict(ldx=1 << 62), rp.ERR_SHAPE), (dict(ldq=(1 << 63) - 1), rp.ERR_SHAPE),
        (dict(X=None), rp.ERR_NULL), (dict(S=None, Y=None, Q=None, scale=None), rp.ERR_NULL),
        (dict(Q=None), rp.ERR_NULL), (dict(scale=None), rp.ERR_NULL),
        (dict(ldx=7), rp.ERR_STRIDE), (dict(ldr=7), rp.ERR_STRIDE), (dict(lds=0), rp.ERR_STRIDE),
        (dict(ldy=7), rp.ERR_STRIDE), (dict(ldq=7), rp.ERR_STRIDE),
        (dict(S=A + 4), rp.ERR_ALIAS), (dict(S=A, lds=9), rp.ERR_ALIAS), (dict(Y=B + 32), rp.ERR_ALIAS),
        (dict(S=E), rp.ERR_ALIAS), (dict(S=A, Y=A), rp.ERR_ALIAS),
        (dict(Q=A), rp.ERR_ALIAS), (dict(Q=B + 127), rp.ERR_ALIAS), (dict(Q=D), rp.ERR_ALIAS),
        (dict(scale=A), rp.ERR_ALIAS), (dict(scale=F + 28), rp.ERR_ALIAS), (dict(scale=C), rp.ERR_ALIAS),
        (dict(rstd=G), rp.ERR_ALIAS), (dict(rstd=C + 28), rp.ERR_ALIAS), (dict(Y=C), rp.ERR_ALIAS),
        (dict(launch=launch(rp.LAUNCH_GEMM_TILED)), rp.ERR_LAUNCH),
        (dict(launch=launch(wave, (3,))), rp.ERR_LAUNCH),
        (dict(launch=launch(wave, (1, 3))), rp.ERR_LAUNCH),
        (dict(launch=launch(wave, (4, 2))), rp.ERR_LAUNCH),
        (dict(launch=launch(wave, (4,)), o=order(row_width=32)), rp.ERR_LAUNCH),
        (dict(rows=0), rp.OK),
        (dict(rows=0, X=None, S=None, Y=None, Q=None, scale=None), rp.OK)])
    wide = dict(base, cols=4097, ldx=4097, ldr=4097, lds=4097, ldy=4097, ldq=4097)
    refuse(wide, call, [(dict(launch=launch(wave, (4,))), rp.ERR_LAUNCH),
                        (dict(launch=launch(wave, (1, 2))), rp.ERR_LAUNCH)])


@no_gpu_only
def test_add_rmsnorm_backward_rows_refusals():
    f = rp.load().repops_add_rmsnorm_backward_rows

    def call(o, rows, cols, S, lds, dY, lddy, dS, ldds, rstd, gamma, dX, lddx, dgamma, ws, wsb, launch):
        return f(o, rows, cols, S, lds, dY, lddy, dS, ldds, rstd, gamma, dX, lddx, dgamma, ws, wsb,
                 launch, None)
    base = dict(o=order(), rows=200, cols=8, S=A, lds=8, dY=B, lddy=8, dS=C, ldds=8, rstd=D, gamma=E,
                dX=F, lddx=8, dgamma=G, ws=W, wsb=1 << 20, launch=None)
    refuse(base, call, [
        (dict(o=order(row_combine=7)), rp.ERR_ORDER), (dict(rows=-1), rp.ERR_SHAPE),
        (dict(cols=0), rp.ERR_SHAPE), (dict(S=None), rp.ERR_NULL), (dict(dY=None), rp.ERR_NULL),
        (dict(rstd=None), rp.ERR_NULL), (dict(dX=None, dgamma=None), rp.OK),
        (dict(lds=7), rp.ERR_STRIDE), (dict(lddy=7), rp.ERR_STRIDE), (dict(ldds=7), rp.ERR_STRIDE),
        (dict(lddx=7), rp.ERR_STRIDE), (dict(dX=A + 4), rp.ERR_ALIAS), (dict(dX=C + 4), rp.ERR_ALIAS),
        (dict(dX=C, lddx=9), rp.ERR_ALIAS), (dict(dX=D), rp.ERR_ALIAS), (dict(dgamma=C), rp.ERR_ALIAS),
        (dict(dgamma=E), rp.ERR_ALIAS), (dict(dgamma=F), rp.ERR_ALIAS),
        (dict(ws=None), rp.ERR_WORKSPACE), (dict(wsb=4), rp.ERR_WORKSPACE),
        (dict(ws=C), rp.ERR_ALIAS), (dict(launch=launch(rp.LAUNCH_ROWS_WAVE, (3,))), rp.ERR_LAUNCH)])


@no_gpu_only
def test_quantize_rows_refusals():
    f = rp.load().repops_quantize_rows

    def call(rows, cols, X, ldx, Q, ldq, scale, launch):
        return f(rows, cols, X, ldx, Q, ldq, scale, launch, None)
    base = dict(rows=4, cols=8, X=A, ldx=8, Q=B, ldq=8, scale=C, launch=None)
    refuse(base, call, [
        (dict(rows=-1), rp.ERR_SHAPE), (dict(cols=-1), rp.ERR_SHAPE), (dict(rows=FAR + 1), rp.ERR_SHAPE),
        (dict(cols=FAR + 1), rp.ERR_SHAPE), (dict(ldx=1 << 62), rp.ERR_SHAPE),
        (dict(X=None), rp.ERR_NULL), (dict(Q=None), rp.ERR_NULL), (dict(scale=None), rp.ERR_NULL),
        (dict(ldx=7), rp.ERR_STRIDE), (dict(ldq=7), rp.ERR_STRIDE),
        (dict(Q=A), rp.ERR_ALIAS), (dict(Q=A + 127), rp.ERR_ALIAS), (dict(scale=A + 64), rp.ERR_ALIAS),
        (dict(scale=B + 28), rp.ERR_ALIAS),
        (dict(launch=launch(rp.LAUNCH_ROWS_WAVE, (4,))), rp.ERR_LAUNCH),
        (dict(rows=0, X=None, Q=None, scale=None), rp.OK)])


@no_gpu_only
def test_matmul_q8_refusals():
    f = rp.load().repops_matmul_q8

    def call(m, n, k, a, lda, sa, b, ldb, sb, bias, c, ldc, launch):
        return f(m, n, k, a, lda, sa, b, ldb, sb, bias, c, ldc, launch, None)
    base = dict(m=4, n=8, k=16, a=A, lda=16, sa=B, b=C, ldb=16, sb=D, bias=E, c=F, ldc=8, launch=None)
    refuse(base, call, [
        (dict(m=-1), rp.ERR_SHAPE), (dict(n=-1), rp.ERR_SHAPE), (dict(k=-1), rp.ERR_SHAPE),
        (dict(k=rp.Q8_MAX_K + 1, lda=1 << 20, ldb=1 << 20), rp.ERR_SHAPE),
        (dict(m=FAR + 1), rp.ERR_SHAPE), (dict(n=FAR + 1, ldc=1 << 40), rp.ERR_SHAPE),
        (dict(ldc=1 << 62), rp.ERR_SHAPE), (dict(lda=1 << 62), rp.ERR_SHAPE),
        (dict(a=None), rp.ERR_NULL), (dict(b=None), rp.ERR_NULL), (dict(sa=None), rp.ERR_NULL),
        (dict(sb=None), rp.ERR_NULL), (dict(c=None), rp.ERR_NULL),
        (dict(lda=15), rp.ERR_STRIDE), (dict(ldb=15), rp.ERR_STRIDE), (dict(ldc=7), rp.ERR_STRIDE),
        (dict(c=A), rp.ERR_ALIAS), (dict(c=C + 127), rp.ERR_ALIAS), (dict(c=B - 124), rp.ERR_ALIAS),
        (dict(c=D), rp.ERR_ALIAS), (dict(c=E), rp.ERR_ALIAS),
        (dict(launch=launch(rp.LAUNCH_GEMM_MFMA, (0,))), rp.ERR_LAUNCH),
        (dict(m=0, a=None, c=None), rp.OK), (dict(n=0, b=None, c=None), rp.OK)])


@no_gpu_only
def test_sample_rows_refusals():
    lib = rp.load()

    def call(rows, vocab, L, ldl, u, T, k, p, m, token, prob, ws, wsb, launch):
        return lib.repops_sample_rows(rows, vocab, L, ldl, u, T, k, p, m, token, prob, ws, wsb, launch,
                                      None)
    base = dict(rows=4, vocab=64, L=A, ldl=64, u=B, T=B + 64, k=B + 128, p=B + 192, m=B + 256, token=C,
                prob=D, ws=None, wsb=0, launch=None)
    refuse(base, call, [
        (dict(rows=-1), rp.ERR_SHAPE), (dict(vocab=-1), rp.ERR_SHAPE), (dict(rows=FAR + 1), rp.ERR_SHAPE),
        (dict(vocab=(1 << 20) + 1, ldl=1 << 21), rp.ERR_SHAPE), (dict(ldl=1 << 62), rp.ERR_SHAPE),
        (dict(L=None), rp.ERR_NULL), (dict(u=None), rp.ERR_NULL), (dict(token=None), rp.ERR_NULL),
        (dict(ldl=63), rp.ERR_STRIDE), (dict(token=A), rp.ERR_ALIAS), (dict(prob=A + 1020), rp.ERR_ALIAS),
        (dict(token=B), rp.ERR_ALIAS), (dict(prob=B + 128), rp.ERR_ALIAS), (dict(token=B + 260), rp.ERR_ALIAS),
        (dict(prob=C + 12), rp.ERR_ALIAS),
        (dict(launch=launch(rp.LAUNCH_ROWS_WAVE, (1,))), rp.ERR_LAUNCH),
        (dict(rows=0, L=None, u=None, token=None), rp.OK)])
    need = rp.sample_workspace(4, 100000)
    assert need > 0 and need % 8 == 0 and rp.sample_workspace(4, 64) == 0 == rp.sample_workspace(0, 100000)
    long = dict(base, vocab=100000, ldl=100000, ws=W, wsb=need)
    refuse(long, call, [
        (dict(ws=None), rp.ERR_WORKSPACE), (dict(wsb=need - 1), rp.ERR_WORKSPACE),
        (dict(ws=W + 4), rp.ERR_STRIDE), (dict(ws=A + 8), rp.ERR_ALIAS), (dict(token=W + 8), rp.ERR_ALIAS),
        (dict(ws=B), rp.ERR_ALIAS)])
    assert lib.repops_sample_workspace(4, 64, None) == rp.ERR_NULL
    with pytest.raises(rp.RepopsError):
        rp.sample_workspace(1, (1 << 20) + 1)
    # only few long rows need one: a workspace for many rows is not one for few
    assert rp.sample_workspace(300, 100000) == 0 == rp.sample_workspace(1, 40000)
    # bounded for any number of rows
    assert max(rp.sample_workspace(r, v) for r in (1, 1000, FAR) for v in (20000, 1 << 20)) <= 64 << 20


def test_binding_refusals():
    X, v = torch.zeros(4, 8), torch.zeros(4)
    q, sq, row = torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4), torch.zeros(8)
    # device tensors are asked for, shapes and types before that
    for call in (lambda: rp.add_rmsnorm_rows(X, X, row), lambda: rp.add_rmsnorm_quantize_rows(X),
                 lambda: rp.add_rmsnorm_backward_rows(X, X, v), lambda: rp.quantize_rows(X),
                 lambda: rp.matmul_q8(q, sq, q, sq), lambda: rp.sample_rows(X, v)):
        with pytest.raises(TypeError, match="must be a device tensor"):
            call()
    for call in (lambda: rp.add_rmsnorm_rows(X.double()), lambda: rp.quantize_rows(X.half()),
                 lambda: rp.add_rmsnorm_backward_rows(X.double(), X, v),
                 lambda: rp.matmul_q8(X, sq, q, sq), lambda: rp.sample_rows(X.bfloat16(), v)):
        with pytest.raises(TypeError, match="must be (float32|int8)"):
            call()
    for call in (lambda: rp.add_rmsnorm_rows(X.t()[:, ::2]), lambda: rp.quantize_rows(X.t()),
                 lambda: rp.add_rmsnorm_rows(row), lambda: rp.sample_rows(X.t(), torch.zeros(8)),
                 lambda: rp.matmul_q8(q.t(), row, q.t(), row)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError, match="inner dimensions differ"):
        rp.matmul_q8(q, sq, q[:, :7], sq)


class Meta:
    """Stands for a device tensor whose checks run and whose memory is never reached."""

    def __init__(self, t, device=0):
        self.t, self.device_index = t, device

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.device_index

    @property
    def is_cuda(self):
        return True

    def new_empty(self, *a, **k):
        return Meta(self.t.new_empty(*a, **k), self.device_index)

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        return Meta(func(args[0].t, *args[1:], **(kwargs or {})), args[0].device_index)


def test_binding_checks_shapes_types_and_devices():
    f, i8 = torch.float32, torch.int8
    m = lambda *shape, dtype=f, device=0: Meta(torch.zeros(*shape, dtype=dtype), device)  # noqa: E731
    X = m(4, 8)
    bad = [
        lambda: rp.add_rmsnorm_rows(X, m(3, 8)), lambda: rp.add_rmsnorm_rows(X, X, m(4)),
        lambda: rp.add_rmsnorm_rows(X, X, out=m(4, 9)), lambda: rp.add_rmsnorm_rows(X, X, rstd_out=m(8)),
        lambda: rp.add_rmsnorm_rows(X, m(4, 8, device=1)),
        lambda: rp.add_rmsnorm_quantize_rows(X, q_out=m(4, 7, dtype=i8)),
        lambda: rp.add_rmsnorm_quantize_rows(X, scale_out=m(5)),
        lambda: rp.add_rmsnorm_backward_rows(X, m(4, 7), m(4)),
        lambda: rp.add_rmsnorm_backward_rows(X, X, m(3)),
        lambda: rp.add_rmsnorm_backward_rows(X, X, m(4), dS=m(8, 4)),
        lambda: rp.add_rmsnorm_backward_rows(X, X, m(4), dgamma_out=m(4)),
        lambda: rp.quantize_rows(X, q_out=m(8, 4, dtype=i8)), lambda: rp.quantize_rows(X, scale_out=m(2, 2)),
        lambda: rp.matmul_q8(m(4, 8, dtype=i8), m(5), m(3, 8, dtype=i8), m(3)),
        lambda: rp.matmul_q8(m(4, 8, dtype=i8), m(4), m(3, 8, dtype=i8), m(4)),
        lambda: rp.matmul_q8(m(4, 8, dtype=i8), m(4), m(3, 8, dtype=i8), m(3), m(4)),
        lambda: rp.matmul_q8(m(4, 8, dtype=i8), m(4), m(3, 8, dtype=i8, device=1), m(3)),
        lambda: rp.matmul_q8(m(4, 8, dtype=i8), m(4), m(3, 8, dtype=i8), m(3), out=m(3, 4)),
        lambda: rp.sample_rows(X, m(5)), lambda: rp.sample_rows(X, m(4), m(3)),
        lambda: rp.sample_rows(X, m(4), token_out=m(8, dtype=torch.int32)),
        lambda: rp.sample_rows(X, m(4, device=1)),
        lambda: rp.sample_rows(X, m(4), workspace=m(64, device=1))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    wrong = [
        lambda: rp.add_rmsnorm_rows(X, m(4, 8, dtype=torch.float64)),
        lambda: rp.add_rmsnorm_rows(X, out=m(4, 8, dtype=torch.float16)),
        lambda: rp.add_rmsnorm_quantize_rows(X, q_out=m(4, 8, dtype=torch.uint8)),
        lambda: rp.quantize_rows(X, q_out=m(4, 8)),
        lambda: rp.matmul_q8(m(4, 8), m(4), m(3, 8, dtype=i8), m(3)),
        lambda: rp.matmul_q8(m(4, 8, dtype=i8), m(4, dtype=torch.float64), m(3, 8, dtype=i8), m(3)),
        lambda: rp.sample_rows(X, m(4), top_k=m(4, dtype=torch.int64)),
        lambda: rp.sample_rows(X, m(4), top_p=m(4, dtype=torch.float64)),
        lambda: rp.sample_rows(X, m(4), token_out=m(4, dtype=torch.int64))]
    for call in wrong:
        with pytest.raises(TypeError, match="must be"):
            call()
