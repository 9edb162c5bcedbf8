"""GPU parity of the generation-step operators against their CPU oracle (0 ULP)
and against plain formulas in 64 bits: residual addition with RMSNorm (fp32 and
8-bit outputs, forward and backward), the row quantiser, the product of 8-bit
operands and the drawing of a token."""
import numpy as np
import pytest

import oracle
from bitcmp import assert_bits_equal
from gpu_util import announce, dev, host
from oracle import generation
from paper_2502_19405_amd import inputs

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def rp():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2502_19405_amd import repops
    repops.load()
    return repops


def launches(rp, cols):
    out = [("auto", None), ("generic", rp.Launch(rp.LAUNCH_ROWS_GENERIC))]
    if cols <= 4096:
        out += [(f"wave{w}", rp.Launch(rp.LAUNCH_ROWS_WAVE, (w,))) for w in (1, 4, 8)]
    out += [(f"split{S}", rp.Launch(rp.LAUNCH_ROWS_WAVE, (1, S))) for S in (2, 4, 8)
            if cols <= S * 2048]
    return out


# --------------------------------------------------------------------------
# addition with norm
# --------------------------------------------------------------------------

NORM_SHAPES = [(1, 1), (3, 2), (5, 63), (1, 64), (7, 65), (130, 100), (9, 768), (33, 1001),
               (4, 2048), (3, 4096), (2, 4097), (2, 14336), (1, 20000)]


@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
def test_add_rmsnorm_bits_every_launch(rp, rows, cols):
    g = inputs.rng(900 + rows + cols)
    X, R = inputs.normal(g, (rows, cols)), inputs.normal(g, (rows, cols), var=4.0)
    gamma = (1 + inputs.uniform(g, (cols,), -0.5, 0.5)).astype(np.float32)
    S, Y, rstd = generation.add_rmsnorm_rows(X, R, gamma)
    Q, scale = generation.quantize_rows(Y)
    import torch
    for name, launch in launches(rp, cols):
        announce("add_rmsnorm", rows, cols, name)
        stat = torch.empty(rows, device="cuda:0")
        s, y = rp.add_rmsnorm_rows(dev(X), dev(R), dev(gamma), launch=launch, rstd_out=stat)
        assert_bits_equal(host(s), S, f"S {name}")
        assert_bits_equal(host(y), Y, f"Y {name}")
        assert_bits_equal(host(stat), rstd, f"rstd {name}")
        y2 = torch.empty(rows, cols, device="cuda:0")
        s, q, sc = rp.add_rmsnorm_quantize_rows(dev(X), dev(R), dev(gamma), launch=launch, out=y2)
        assert_bits_equal(host(s), S, f"S with codes {name}")
        assert_bits_equal(host(y2), Y, f"Y with codes {name}")
        assert_bits_equal(host(sc), scale, f"scale {name}")
        assert np.array_equal(host(q), Q), name


@pytest.mark.parametrize("W,combine,kb", [(64, 0, 64), (16, 0, 3), (64, 1, 0), (1, 0, 64)])
def test_add_rmsnorm_orders_and_optional_operands(rp, W, combine, kb):
    g = inputs.rng(930)
    X, R = inputs.normal(g, (70, 333)), inputs.normal(g, (70, 333))
    dY, dS = inputs.normal(g, (70, 333)), inputs.normal(g, (70, 333))
    order = rp.Order(row_width=W, row_combine=combine, k_block=kb)
    kw = dict(row_width=W, row_combine=combine)
    import torch
    for r, gamma in ((R, None), (None, inputs.normal(g, (333,))), (None, None)):
        S, Y, rstd = generation.add_rmsnorm_rows(X, r, gamma, **kw)
        opt = lambda a: None if a is None else dev(a)  # noqa: E731
        stat = torch.empty(70, device="cuda:0")
        announce("add_rmsnorm order", W, combine, kb, r is None, gamma is None)
        s, y = rp.add_rmsnorm_rows(dev(X), opt(r), opt(gamma), order=order, rstd_out=stat)
        assert_bits_equal(host(s), S)
        assert_bits_equal(host(y), Y)
        for ds in (None, dS):
            dX, dg = generation.add_rmsnorm_backward_rows(S, dY, rstd, gamma, ds, k_block=kb, **kw)
            dx, dgam = rp.add_rmsnorm_backward_rows(s, dev(dY), stat, opt(gamma), dS=opt(ds),
                                                    order=order)
            assert_bits_equal(host(dx), dX)
            assert_bits_equal(host(dgam), dg)


BWD_SHAPES = [(1, 1), (5, 63), (130, 64), (200, 100), (70, 768), (33, 1001), (64, 2048), (65, 2049),
              (80, 4096), (3, 5000), (2, 14336), (16640, 96), (16500, 1025)]


@pytest.mark.parametrize("rows,cols", BWD_SHAPES)
def test_add_rmsnorm_backward_bits_every_launch(rp, rows, cols):
    g = inputs.rng(950 + rows + cols)
    S = inputs.normal(g, (rows, cols), var=2.0)
    dY, dS = inputs.normal(g, (rows, cols)), inputs.normal(g, (rows, cols))
    gamma = (1 + inputs.uniform(g, (cols,), -0.5, 0.5)).astype(np.float32)
    _, _, rstd = generation.add_rmsnorm_rows(S, None, gamma)
    dX, dg = generation.add_rmsnorm_backward_rows(S, dY, rstd, gamma, dS)
    s, dy, ds, rs, gm = dev(S), dev(dY), dev(dS), dev(rstd), dev(gamma)
    for name, launch in launches(rp, cols):
        announce("add_rmsnorm backward", rows, cols, name)
        dx, dgam = rp.add_rmsnorm_backward_rows(s, dy, rs, gm, dS=ds, launch=launch)
        assert_bits_equal(host(dx), dX, f"dX {name}")
        assert_bits_equal(host(dgam), dg, f"dgamma {name}")
        dx, none = rp.add_rmsnorm_backward_rows(s, dy, rs, gm, dS=ds, launch=launch,
                                                need_dgamma=False)
        assert none is None
        assert_bits_equal(host(dx), dX, f"dX alone {name}")
        inplace = ds.clone()  # the residual stream's gradient updated in place
        rp.add_rmsnorm_backward_rows(s, dy, rs, gm, dS=inplace, launch=launch, dx_out=inplace)
        assert_bits_equal(host(inplace), dX, f"dX in place of dS {name}")


def test_add_rmsnorm_backward_without_ds_is_rmsnorm_backward(rp):
    g = inputs.rng(960)
    S, dY = inputs.normal(g, (100, 512)), inputs.normal(g, (100, 512))
    rstd = inputs.uniform(g, (100,), 0.5, 2.0)
    announce("backward without dS")
    a = rp.add_rmsnorm_backward_rows(dev(S), dev(dY), dev(rstd))
    b = rp.rmsnorm_backward_rows(dev(S), dev(dY), dev(rstd))
    assert_bits_equal(host(a[0]), host(b[0]))
    assert_bits_equal(host(a[1]), host(b[1]))


@pytest.mark.parametrize("rows,cols", [(37, 200), (6, 4096), (3, 9001)])
def test_add_rmsnorm_against_formulas_in_64_bits(rp, rows, cols):
    """Bounds in units of U = 2^-24 (half a step): S is one rounding.  From the
    rounded S, a lane's chain of ceil(n / 64) fused steps, six tree additions and a
    division give ms within (n/64 + 8) U, halved by the square root, which with the
    quotient and two products gives y within (n/128 + 9) U.  dX carries b's
    error, (n/64 + 12) U of mean |g t|, and at most six roundings of its terms."""
    g = inputs.rng(970 + cols)
    X, R, dY, dS = (inputs.normal(g, (rows, cols)) for _ in range(4))
    gamma = (1 + inputs.uniform(g, (cols,), -0.5, 0.5)).astype(np.float32)
    import torch
    announce("add_rmsnorm in 64 bits", rows, cols)
    stat = torch.empty(rows, device="cuda:0")
    s, y = rp.add_rmsnorm_rows(dev(X), dev(R), dev(gamma), rstd_out=stat)
    dx, dg = rp.add_rmsnorm_backward_rows(s, dev(dY), stat, dev(gamma), dS=dev(dS))
    s, y, dx, dg = (host(t).astype(np.float64) for t in (s, y, dx, dg))
    exact = X.astype(np.float64) + R
    assert (np.abs(s - exact) <= U * np.abs(exact)).all()
    root = np.sqrt((s * s).mean(1, keepdims=True) + np.float64(np.float32(1e-5)))
    t = s / root
    want = t * gamma
    c = np.ceil(cols / 64)
    assert (np.abs(y - want) <= (c / 2 + 9) * U * np.abs(want) + 1e-40).all()
    gy = dY.astype(np.float64) * gamma
    b = (gy * t).mean(1, keepdims=True)
    want = (gy - t * b) / root + dS
    size = (np.abs(gy) + np.abs(t) * np.abs(gy * t).mean(1, keepdims=True)) / root
    assert (np.abs(dx - want) <= (2 * c + 24) * U * size + 2 * U * np.abs(want)).all()
    want = (dY * t).sum(0)
    assert (np.abs(dg - want) <= (64 + rows / 64 + c / 2 + 12) * U * np.abs(dY * t).sum(0)).all()


def test_add_rmsnorm_gradient_against_differences(rp):
    """The loss sum(y dy) + sum(s ds) in 64 bits from the GPU's Y and S.  A central
    difference of step h errs by h^2 / 6 of the third derivative, below 40 at these
    sizes (a root mean square of about 1.4 over 40 columns), and by the rounding of
    the two losses: ten U of their terms' size each, over 2 h."""
    g = inputs.rng(975)
    X, R, dY, dS = (inputs.normal(g, (2, 40)) for _ in range(4))
    gamma = (1 + inputs.uniform(g, (40,), -0.5, 0.5)).astype(np.float32)
    import torch
    stat = torch.empty(2, device="cuda:0")

    def terms(x, gm):
        s, y = rp.add_rmsnorm_rows(dev(x), dev(R), dev(gm), rstd_out=stat)
        return host(y).astype(np.float64) * dY, host(s).astype(np.float64) * dS
    announce("add_rmsnorm differences")
    ty, ts = terms(X, gamma)
    size = np.abs(ty).sum() + np.abs(ts).sum()
    s, _ = rp.add_rmsnorm_rows(dev(X), dev(R), dev(gamma))
    dx, dg = (host(v) for v in rp.add_rmsnorm_backward_rows(s, dev(dY), stat, dev(gamma), dS=dev(dS)))
    h = 2.0 ** -6
    bound = 7 * h * h + 20 * U * size / (2 * h)

    def slope(a, i, f):
        lo, hi = a.copy(), a.copy()
        lo[i] -= np.float32(h)
        hi[i] += np.float32(h)
        up, down = sum(t.sum() for t in f(hi)), sum(t.sum() for t in f(lo))
        return (up - down) / (float(hi[i]) - float(lo[i]))
    for i in ((0, 0), (1, 17), (1, 39)):
        assert abs(slope(X, i, lambda x: terms(x, gamma)) - dx[i]) <= bound
    assert abs(slope(gamma, (5,), lambda gm: terms(X, gm)) - dg[5]) <= bound


def test_add_rmsnorm_in_place_padded_and_rows_behind(rp):
    import torch
    g = inputs.rng(980)
    X, R = inputs.normal(g, (40, 300)), inputs.normal(g, (40, 300))
    S, Y, _ = generation.add_rmsnorm_rows(X, R)
    Q, scale = generation.quantize_rows(Y)
    for cols_ld in (300, 301, 320):
        announce("add_rmsnorm padded", cols_ld)
        x, r = (torch.full((44, cols_ld), 7.0, device="cuda:0") for _ in range(2))
        x[:40, :300], r[:40, :300] = dev(X), dev(R)
        q = torch.full((44, cols_ld), 99, dtype=torch.int8, device="cuda:0")
        sc = torch.full((44,), -1.0, device="cuda:0")
        # the sum in place of the residual, the norm in place of x
        rp.add_rmsnorm_quantize_rows(x[:40, :300], r[:40, :300], sum_out=r[:40, :300],
                                     out=x[:40, :300], q_out=q[:40, :300], scale_out=sc[:40])
        assert_bits_equal(host(r)[:40, :300], S)
        assert_bits_equal(host(x)[:40, :300], Y)
        assert_bits_equal(host(sc)[:40], scale)
        assert np.array_equal(host(q)[:40, :300], Q)
        for t, fill in ((x, 7.0), (r, 7.0), (q, 99)):
            t = host(t)
            assert (t[40:] == fill).all() and (t[:, 300:] == fill).all()
        assert (host(sc)[40:] == -1.0).all()


def special_rows(cols):
    """Rows at the ends of the quantiser's range."""
    f = np.float32
    rows = [np.zeros(cols), -np.zeros(cols), np.full(cols, 1e-45), np.full(cols, 3e-43),
            np.linspace(-1e-38, 1e-38, cols), np.full(cols, 3.4e38), np.linspace(-127, 127, cols),
            np.linspace(-63.5, 63.5, cols)]
    for bad in (np.inf, -np.inf, np.nan):
        r = np.ones(cols)
        r[cols // 2] = bad
        rows.append(r)
    return np.stack(rows).astype(f)


@pytest.mark.parametrize("cols", [1, 7, 64, 255, 1024, 4096, 14336, 40001])
def test_quantize_rows(rp, cols):
    import torch
    g = inputs.rng(990 + cols)
    X = np.concatenate([special_rows(cols), inputs.normal(g, (9, cols), var=1e-3)])
    Q, scale = generation.quantize_rows(X)
    announce("quantize_rows", cols)
    q, sc = rp.quantize_rows(dev(X))
    assert_bits_equal(host(sc), scale)
    assert np.array_equal(host(q), Q)
    for off, pad in ((0, 1), (1, 4), (4, 0)):  # rows of every alignment
        x = torch.full((len(X) + 1, off + cols + pad), 3.0, device="cuda:0")
        x[:-1, off:off + cols] = dev(X)
        b = torch.full(x.shape, 99, dtype=torch.int8, device="cuda:0")
        announce("quantize_rows", cols, off, pad)
        rp.quantize_rows(x[:-1, off:off + cols], q_out=b[:-1, off:off + cols])
        b = host(b)
        assert np.array_equal(b[:-1, off:off + cols], Q)
        b[:-1, off:off + cols] = 99
        assert (b == 99).all()


def test_quantize_rows_errs_by_half_a_step(rp):
    """RN(y RN(1 / scale)) is within 127 * 2 U < 2^-16 of y / scale, so a code is
    within half a step and 2^-16."""
    g = inputs.rng(995)
    X = inputs.normal(g, (50, 777))
    announce("quantize_rows half a step")
    q, sc = (host(t).astype(np.float64) for t in rp.quantize_rows(dev(X)))
    top = np.abs(X).max(1).astype(np.float64)
    assert (np.abs(sc - top / 127) <= U * top / 127).all()
    assert (np.abs(q - X / sc[:, None]) <= 0.5 + 2.0 ** -16).all()
    assert (np.abs(q).max(1) == 127).all()


# --------------------------------------------------------------------------
# 8-bit product
# --------------------------------------------------------------------------

Q8_SHAPES = [(1, 1, 1), (1, 5, 0), (3, 2, 7), (1, 64, 64), (4, 1000, 4096), (16, 33, 100),
             (17, 129, 129), (31, 64, 1024), (33, 65, 63), (64, 64, 64), (65, 127, 999),
             (100, 300, 500), (128, 128, 128), (129, 257, 192), (333, 1001, 999), (256, 512, 4096),
             (300, 1024, 48), (5, 4096, 14336), (40, 200, 30000), (513, 770, 640),
             (100, 90, 15), (70, 70, 1), (200, 33, 16), (129, 70, 17), (40, 200, 5000),
             (300, 64, 8192), (64, 1024, 4096), (1000, 100, 4096), (513, 300, 1500),
             (1100, 1300, 333), (260, 5000, 270)]


def codes(g, *shape):
    return np.clip(np.rint(inputs.normal(g, shape, var=1600.0)), -128, 127).astype(np.int8)


@pytest.mark.parametrize("m,n,k", Q8_SHAPES)
def test_matmul_q8(rp, m, n, k):
    g = inputs.rng(1000 + m + n + k)
    A, B = codes(g, m, k), codes(g, n, k)
    sa, sb = inputs.uniform(g, (m,), 0.01, 0.1), inputs.uniform(g, (n,), 1e-4, 1e-3)
    bias = inputs.uniform(g, (n,), -1, 1)
    for b in (None, bias):
        announce("matmul_q8", m, n, k, b is not None)
        got = host(rp.matmul_q8(dev(A), dev(sa), dev(B), dev(sb), None if b is None else dev(b)))
        assert_bits_equal(got, generation.matmul_q8(A, sa, B, sb, b))
        prod = (A.astype(np.float64) @ B.astype(np.float64).T) * sa[:, None] * sb
        exact = prod if b is None else prod + b
        # RN(acc) and two products, then the bias: three roundings and one
        assert (np.abs(got - exact) <= 3.01 * U * np.abs(prod) + 1.01 * U * np.abs(exact)).all()


@pytest.mark.parametrize("m,n,k", [(5, 70, 200), (130, 140, 256), (70, 300, 999)])
def test_matmul_q8_strides_alignments_and_surroundings(rp, m, n, k):
    import torch
    g = inputs.rng(1050 + k)
    A, B = codes(g, m, k), codes(g, n, k)
    sa, sb = inputs.uniform(g, (m,), 0.01, 0.1), inputs.uniform(g, (n,), 1e-4, 1e-3)
    want = generation.matmul_q8(A, sa, B, sb)
    for off_a, off_b, pad in ((0, 0, 0), (0, 0, 16), (1, 0, 3), (0, 5, 11), (4, 8, 28), (16, 16, 64)):
        announce("matmul_q8 strides", m, n, k, off_a, off_b, pad)
        a = torch.full((m + 1, k + off_a + pad), 77, dtype=torch.int8, device="cuda:0")
        b = torch.full((n + 1, k + off_b + pad), -99, dtype=torch.int8, device="cuda:0")
        c = torch.full((m + 2, n + 7), -5.0, device="cuda:0")
        a[:m, off_a:off_a + k], b[:n, off_b:off_b + k] = dev(A), dev(B)
        rp.matmul_q8(a[:m, off_a:off_a + k], dev(sa), b[:n, off_b:off_b + k], dev(sb),
                     out=c[1:m + 1, 3:n + 3])
        got = host(c)
        assert_bits_equal(got[1:m + 1, 3:n + 3], want)
        got[1:m + 1, 3:n + 3] = -5.0
        assert (got == -5.0).all()


def test_matmul_q8_largest_sums(rp):
    k = rp.Q8_MAX_K
    one = dev(np.ones(3, np.float32))
    for a, b, want in ((-128, -128, k * 16384.0), (-128, 127, -k * 16256.0), (127, 127, k * 16129.0)):
        announce("matmul_q8 largest", a, b)
        A, B = np.full((3, k), a, np.int8), np.full((3, k), b, np.int8)
        got = host(rp.matmul_q8(dev(A), one, dev(B), one))
        assert (got == np.float32(want)).all()


# --------------------------------------------------------------------------
# drawing a token
# --------------------------------------------------------------------------

def draw_inputs(seed, rows, vocab, std=2.5, peaks=4):
    g = inputs.rng(seed)
    L = inputs.normal(g, (rows, vocab), var=std * std)
    for r in range(rows):
        L[r, g.integers(0, vocab, peaks)] = g.uniform(6, 12, peaks).astype(np.float32)
    return L, g.random(rows, dtype=np.float32)


def check_draw(rp, L, u, what, **p):
    announce("sample_rows", what, L.shape)
    params = {k: v for k, v in p.items() if v is not None}
    token, prob = rp.sample_rows(dev(L), dev(u), **{k: dev(v) for k, v in params.items()})
    wt, wp = generation.sample_rows(L, u, **params)
    token = host(token)
    assert np.array_equal(token, wt), (what, np.flatnonzero(token != wt)[:5], token, wt)
    assert_bits_equal(host(prob), wp, what)
    return token


def full(rows, v, t=np.float32):
    return np.full(rows, v, t)


VOCABS = [1, 2, 3, 64, 255, 1000, 4097, 32000, 50257, 128000]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("what", ["none", "top_k", "top_p", "min_p", "all", "mixed"])
def test_sample_rows(rp, vocab, what):
    rows = 9
    L, u = draw_inputs(2000 + vocab, rows, vocab)
    p = {}
    if what in ("top_k", "all"):
        p["top_k"] = full(rows, min(50, vocab), np.int32)
    if what in ("top_p", "all"):
        p["top_p"] = full(rows, 0.9)
    if what in ("min_p", "all"):
        p["min_p"] = full(rows, 0.02)
    if what == "all":
        p["temperature"] = full(rows, 0.7)
    if what == "mixed":
        p = {"temperature": np.array([0, 1, 0.3, 5, 1e-3, 1e30, np.inf, np.nan, -1], np.float32),
             "top_k": np.array([0, 1, 2, vocab, vocab + 5, -3, 7, 40, 1 << 30], np.int32),
             "top_p": np.array([1, 0.5, 0, -1, 0.99, 2, np.nan, 1e-30, 0.9999999], np.float32),
             "min_p": np.array([0, 1, 0.5, 2, 1e-45, -1, np.nan, 1e-6, 0.1], np.float32)}
    check_draw(rp, L, u, what, **p)


def test_sample_rows_every_parameter_pair(rp):
    k, pp, mp, T = np.meshgrid([0, 1, 5, 300], [1.0, 0.0, 0.3, 0.95], [0.0, 0.01, 0.3, 1.0],
                               [0.5, 1.0, 3.0], indexing="ij")
    rows = k.size
    L, u = draw_inputs(2100, rows, 777)
    check_draw(rp, L, u, "pairs", top_k=k.ravel().astype(np.int32), top_p=pp.ravel().astype(np.float32),
               min_p=mp.ravel().astype(np.float32), temperature=T.ravel().astype(np.float32))


@pytest.mark.parametrize("vocab", [5, 1000, 40000, 131072])
def test_sample_rows_equal_and_special_logits(rp, vocab):
    g = inputs.rng(2200 + vocab)
    low, inf, nan = np.float32(-3.4028235e38), np.float32(np.inf), np.float32(np.nan)
    at = g.integers(0, vocab, 3)
    rows = [np.zeros(vocab), np.where(np.arange(vocab) % 2, -0.0, 0.0),    # all equal
            np.full(vocab, low), np.full(vocab, -inf), np.full(vocab, inf),
            np.where(np.arange(vocab) < vocab - 1, -inf, 1.5),             # one left
            g.integers(0, 3, vocab), g.integers(0, 2, vocab) * 1e-30,
            inputs.normal(g, (vocab,), var=1e-8), np.arange(vocab) * 1e-4,
            np.where(np.arange(vocab) % 3 == 0, -inf, 0.25), -np.arange(vocab) * 1e-3]
    L = np.stack(rows).astype(np.float32)
    some = inputs.normal(g, (4, vocab))
    some[0, at[0]], some[1, at[1]], some[2, at[2]] = nan, inf, -inf
    some[3, :] = low
    some[3, at[0]] = 2.0
    L = np.concatenate([L, some])
    n = len(L)
    for j, u in enumerate((0.0, 0.3, 0.99999994)):
        u = full(n, u)
        check_draw(rp, L, u, f"special {j}")
        check_draw(rp, L, u, f"special filters {j}", top_k=full(n, 3 + 2000 * j, np.int32),
                   top_p=full(n, 0.7), min_p=full(n, 0.01))
        check_draw(rp, L, u, f"special hot {j}", temperature=full(n, np.inf), top_p=full(n, 0.5))
        check_draw(rp, L, u, f"special greedy {j}", temperature=full(n, 0.0))
    check_draw(rp, L, np.resize(np.array([nan, -1, 1, 2, inf, -inf], np.float32), n), "odd u")


@pytest.mark.parametrize("vocab,std", [(1, 1), (130, 2.5), (777, 2.5), (20011, 2.5), (20011, 0.01),
                                       (60013, 0.3)])
def test_sample_rows_of_many_rows(rp, vocab, std):
    """More rows than compute units, wide and narrow (one bucket may hold them all),
    every filter in turn."""
    rows = 260
    L, u = draw_inputs(2250 + vocab, rows, vocab, std=std, peaks=0 if std < 1 else 4)
    L[::7] = np.rint(L[::7] * np.float32(8 / std)) * np.float32(std / 8)  # equal logits
    L[3::11, ::3] = -np.inf
    g = inputs.rng(2260 + vocab)
    pick = lambda *v: g.choice(np.array(v), rows)  # noqa: E731
    check_draw(rp, L, u, "many rows")
    check_draw(rp, L, u, "many rows filters", temperature=pick(0, 1, 0.3, 5, 1e30).astype(np.float32),
               top_k=pick(0, 1, 40, 3000, vocab).astype(np.int32),
               top_p=pick(1, 0.5, 0, 0.99).astype(np.float32),
               min_p=pick(0, 0.1, 1, 0.001).astype(np.float32))


@pytest.mark.parametrize("ranked", [False, True])
def test_sample_rows_against_64_bits(rp, ranked):
    """A draw's place in the plain 64-bit distribution: each weight is off by at
    most 2^-44 and the target by two roundings, so u lies within n 2^-43 + 2^-50 of
    the token's stretch."""
    rows, vocab = 64, 9973
    L, u = draw_inputs(2300, rows, vocab)
    T = 0.8
    p = {"temperature": full(rows, T)}
    if ranked:
        p["top_k"] = full(rows, 100, np.int32)
    token = check_draw(rp, L, u, "64 bits", **p)
    z = L.astype(np.float64) / np.float64(np.float32(T))
    for r in range(rows):
        rank = np.argsort(-z[r], kind="stable")
        e = np.exp(z[r][rank] - z[r].max())
        if ranked:
            rank, e = rank[:100], e[:100]
        i = int(np.flatnonzero(rank == token[r])[0])
        c = np.cumsum(e)
        slack = (len(e) * 2.0 ** -43 + c[-1] * 2.0 ** -50)
        assert c[i] - e[i] - slack <= u[r] * c[-1] <= c[i] + slack


def test_sample_rows_frequencies(rp):
    """65536 draws of one row of six tokens at evenly spread u: a token's count is
    its probability's share of the grid, off by less than two points."""
    rows = 65536
    row = np.array([0.0, 1.0, -1.0, 2.0, 0.5, -np.inf], np.float32)
    L = np.tile(row, (rows, 1))
    u = ((np.arange(rows) + 0.5) / rows).astype(np.float32)
    announce("sample_rows frequencies")
    token = host(rp.sample_rows(dev(L), dev(u))[0])
    p = np.exp(row.astype(np.float64))
    p /= p.sum()
    assert (np.abs(np.bincount(token, minlength=6) - p * rows) < 2).all()


def test_sample_rows_strided_and_surroundings(rp):
    import torch
    L, u = draw_inputs(2400, 6, 5000)
    want, wp = generation.sample_rows(L, u)
    for off, pad in ((0, 0), (1, 2), (4, 12)):
        announce("sample_rows strided", off, pad)
        big = torch.full((8, 5000 + off + pad), 1e9, device="cuda:0")
        big[:6, off:off + 5000] = dev(L)
        tok = torch.full((9,), -7, dtype=torch.int32, device="cuda:0")
        prob = torch.full((9,), -7.0, device="cuda:0")
        rp.sample_rows(big[:6, off:off + 5000], dev(u), token_out=tok[1:7], prob_out=prob[1:7])
        assert host(tok).tolist() == [-7, *want.tolist(), -7, -7]
        assert_bits_equal(host(prob)[1:7], wp)
    announce("sample_rows empty")
    t, q = rp.sample_rows(torch.empty(3, 0, device="cuda:0"), dev(u[:3]))
    assert host(t).tolist() == [-1, -1, -1] and host(q).tolist() == [0, 0, 0]
