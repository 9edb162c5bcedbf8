"""The generation-step operators as a program uses them: chained, captured into
graphs, on other streams, from several threads of work at once, in place, and on
tensors whose offsets pass 32 bits."""
import numpy as np
import pytest

from bitcmp import assert_bits_equal
from gpu_util import announce, dev, host, same_bits
from oracle import generation
from paper_2502_19405_amd import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rp():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2502_19405_amd import repops
    repops.load()
    return repops


def program(seed, t, h, f, vocab):
    g = inputs.rng(seed)
    weight = lambda n, k: generation.quantize_rows(inputs.normal(g, (n, k), var=1.0 / k))  # noqa: E731
    return {"X": inputs.normal(g, (t, h)), "R": inputs.normal(g, (t, h)),
            "gamma": (1 + inputs.uniform(g, (h,), -0.1, 0.1)).astype(np.float32),
            "gate": weight(f, h), "up": weight(f, h), "down": weight(h, f), "head": weight(vocab, h),
            "u": g.random(t, dtype=np.float32), "temperature": np.full(t, 0.8, np.float32),
            "top_k": np.full(t, 40, np.int32), "top_p": np.full(t, 0.95, np.float32)}


def on_device(p):
    return {k: [dev(a) for a in v] if isinstance(v, tuple) else dev(v) for k, v in p.items()}


def generate(pipelines, d):
    """One block's feed-forward and the next token."""
    ff = pipelines.llama_feed_forward_q8(d["X"], d["R"], d["gamma"], d["gate"], d["up"], d["down"],
                                         keep=True)
    nt = pipelines.llama_next_token(ff["S"], ff["D"], d["gamma"], d["head"], d["u"], d["temperature"],
                                    d["top_k"], d["top_p"], keep=True)
    return ff, nt


def generate_oracle(p):
    ff = generation.feed_forward_q8(p["X"], p["R"], p["gamma"], p["gate"], p["up"], p["down"])
    nt = generation.next_token(ff["S"], ff["D"], p["gamma"], p["head"], p["u"],
                               temperature=p["temperature"], top_k=p["top_k"], top_p=p["top_p"])
    return ff, nt


def assert_same(got, want, what=""):
    for part, ref in zip(got, want):
        for name, w in ref.items():
            if w.dtype == np.float32:
                assert_bits_equal(host(part[name]), w, f"{what} {name}")
            else:
                assert np.array_equal(host(part[name]), w), f"{what} {name}"


@pytest.mark.parametrize("t,h,f,vocab", [(1, 256, 512, 1000), (4, 512, 1024, 32000), (37, 200, 333, 999),
                                         (130, 256, 704, 20000)])
def test_generation_step(rp, t, h, f, vocab):
    from paper_2502_19405_amd import pipelines
    p = program(3000 + t, t, h, f, vocab)
    announce("generation step", t, h, f, vocab)
    assert_same(generate(pipelines, on_device(p)), generate_oracle(p))


@pytest.mark.parametrize("t,h,n", [(33, 200, 130), (256, 512, 256)])
def test_training_step(rp, t, h, n):
    from paper_2502_19405_amd import pipelines
    g = inputs.rng(3100 + t)
    X, R, dS = (inputs.normal(g, (t, h)) for _ in range(3))
    W, dY = inputs.normal(g, (h, n), var=1.0 / h), inputs.normal(g, (t, n))
    gamma = (1 + inputs.uniform(g, (h,), -0.1, 0.1)).astype(np.float32)
    want = generation.norm_linear(X, R, gamma, W, dY, dS)
    announce("training step", t, h, n)
    S, Y, saved = pipelines.norm_linear_forward(dev(X), dev(R), dev(gamma), dev(W))
    dX, dgamma, dW = pipelines.norm_linear_backward(saved, dev(gamma), dev(W), dev(dY), dev(dS))
    for name, a, b in zip(("S", "Y", "dX", "dgamma", "dW"), (S, Y, dX, dgamma, dW), want):
        assert_bits_equal(host(a), b, name)


def capture(fn):
    import torch
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fn()
    return graph, out


def test_graphs_replay_a_generation_step(rp):
    """Two captured programs, each with buffers and workspaces of its own, replayed in
    turn and on two streams at once, with new inputs between the replays and eager
    calls of the same operators beside them."""
    import torch

    from paper_2502_19405_amd import pipelines
    sizes = ((3, 256, 512, 60000), (40, 128, 384, 70000))
    ds = [on_device(program(3200 + i, *s)) for i, s in enumerate(sizes)]
    announce("graph", "capture")
    graphs = [capture(lambda d=d: generate(pipelines, d)) for d in ds]
    streams = [torch.cuda.Stream() for _ in ds]
    for rep in range(4):
        ps = [program(3210 + 10 * rep + i, *s) for i, s in enumerate(sizes)]
        for d, p in zip(ds, ps):
            for name, v in on_device(p).items():
                for dst, src in zip(d[name], v) if isinstance(v, list) else ((d[name], v),):
                    dst.copy_(src)
        for _, out in graphs:
            for part in out:
                for t in part.values():
                    t.zero_()
        torch.cuda.synchronize()
        announce("graph", "replay", rep)
        if rep % 2:
            for (graph, _), s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    graph.replay()
        else:
            for graph, _ in graphs:
                graph.replay()
            eager = [generate(pipelines, d) for d in ds]
        torch.cuda.synchronize()
        for i, ((_, out), p) in enumerate(zip(graphs, ps)):
            want = generate_oracle(p)
            assert_same(out, want, f"graph {i} replay {rep}")
            if rep % 2 == 0:
                assert_same(eager[i], want, f"eager {i} {rep}")


def test_graph_replays_the_backward(rp):
    import torch
    rows, cols = 300, 768
    g = inputs.rng(3300)
    S, dY, dS = (torch.empty(rows, cols, device="cuda:0") for _ in range(3))
    rstd, gamma = torch.empty(rows, device="cuda:0"), torch.empty(cols, device="cuda:0")
    dX, dg = torch.empty_like(S), torch.empty_like(gamma)
    ws = torch.empty(rp.rmsnorm_backward_workspace(rows, cols) // 4, device="cuda:0")

    def step():
        rp.add_rmsnorm_backward_rows(S, dY, rstd, gamma, dS, dx_out=dX, dgamma_out=dg, workspace=ws)
    for t in (S, dY, dS, rstd, gamma):
        t.fill_(1.0)
    graph, _ = capture(step)
    for rep in range(3):
        s, dy, ds = (inputs.normal(g, (rows, cols)) for _ in range(3))
        gm = (1 + inputs.uniform(g, (cols,), -0.5, 0.5)).astype(np.float32)
        _, _, r = generation.add_rmsnorm_rows(s, None, gm)
        for t, a in zip((S, dY, dS, rstd, gamma), (s, dy, ds, r, gm)):
            t.copy_(dev(a))
        dX.zero_(), dg.zero_()
        torch.cuda.synchronize()
        announce("backward graph", rep)
        graph.replay()
        want = generation.add_rmsnorm_backward_rows(s, dy, r, gm, ds)
        assert_bits_equal(host(dX), want[0])
        assert_bits_equal(host(dg), want[1])
        eager = rp.add_rmsnorm_backward_rows(S, dY, rstd, gamma, dS)
        assert same_bits(eager[0], dX) and same_bits(eager[1], dg)


def test_other_streams_and_calls_at_once(rp):
    """Inputs made on a side stream, the operators on it without waiting for the
    default stream; two draws with workspaces of their own in flight together."""
    import torch
    g = inputs.rng(3400)
    jobs = []
    for rows, vocab in ((20, 90000), (3, 128000)):
        L, u = inputs.normal(g, (rows, vocab), var=6.0), g.random(rows, dtype=np.float32)
        p = np.full(rows, 0.9, np.float32)
        jobs.append((L, u, p, generation.sample_rows(L, u, top_p=p)))
    held = [[torch.from_numpy(a).to("cuda:0") for a in j[:3]] for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for rep in range(5):
        announce("streams", rep)
        out = []
        for (L, u, p), s in zip(held, streams):
            with torch.cuda.stream(s):
                out.append(rp.sample_rows(L + 0.0, u, top_p=p))
        torch.cuda.synchronize()
        for (token, prob), (_, _, _, want) in zip(out, jobs):
            assert np.array_equal(host(token), want[0])
            assert_bits_equal(host(prob), want[1])


IN_PLACE = [("S on X, Y on R", True, "X", "R"), ("S on R, Y on X", True, "R", "X"),
            ("Y on X", True, None, "X"), ("S on X", True, "X", None),
            ("no R, Y on X", False, None, "X"), ("no R, S on X", False, "X", None)]


@pytest.mark.parametrize("what,has_r,s_on,y_on", IN_PLACE)
def test_norm_in_place_every_launch(rp, what, has_r, s_on, y_on):
    for rows, cols in ((9, 130), (3, 5000), (2, 17000)):
        g = inputs.rng(3500 + cols)
        X, R = inputs.normal(g, (rows, cols)), inputs.normal(g, (rows, cols))
        S, Y, _ = generation.add_rmsnorm_rows(X, R if has_r else None)
        Q, scale = generation.quantize_rows(Y)
        kinds = [("auto", None), ("generic", rp.Launch(rp.LAUNCH_ROWS_GENERIC))]
        if cols <= 4096:
            kinds.append(("wave", rp.Launch(rp.LAUNCH_ROWS_WAVE, (4,))))
        if cols <= 8 * 2048:
            kinds.append(("split", rp.Launch(rp.LAUNCH_ROWS_WAVE, (1, 8))))
        for name, launch in kinds:
            announce("in place", what, rows, cols, name)
            t = {"X": dev(X), "R": dev(R)}
            s, q, sc = rp.add_rmsnorm_quantize_rows(
                t["X"], t["R"] if has_r else None, launch=launch,
                sum_out=t[s_on] if s_on else None, out=t[y_on] if y_on else None)
            if has_r or s_on:
                assert_bits_equal(host(s), S, f"S {name}")
            if y_on:
                assert_bits_equal(host(t[y_on]), Y, f"Y {name}")
            assert_bits_equal(host(sc), scale, f"scale {name}")
            assert np.array_equal(host(q), Q), name


def test_backward_in_place(rp):
    """dX on S, dY or dS (the kernels that read rows twice stand aside there)."""
    for rows, cols in ((130, 200), (70, 4096), (20, 14336)):
        g = inputs.rng(3600 + cols)
        S, dY, dS = (inputs.normal(g, (rows, cols)) for _ in range(3))
        gamma = (1 + inputs.uniform(g, (cols,), -0.5, 0.5)).astype(np.float32)
        _, _, rstd = generation.add_rmsnorm_rows(S, None, gamma)
        want = generation.add_rmsnorm_backward_rows(S, dY, rstd, gamma, dS)
        for on in ("S", "dY", "dS"):
            announce("backward in place", rows, cols, on)
            t = {"S": dev(S), "dY": dev(dY), "dS": dev(dS)}
            dx, dg = rp.add_rmsnorm_backward_rows(t["S"], t["dY"], dev(rstd), dev(gamma), t["dS"],
                                                  dx_out=t[on])
            assert dx is t[on]
            assert_bits_equal(host(dx), want[0], on)
            assert_bits_equal(host(dg), want[1], on)


def test_same_tensor_twice(rp):
    """X as its own residual, one matrix of codes as both operands."""
    g = inputs.rng(3700)
    X = inputs.normal(g, (50, 384))
    announce("same tensor twice")
    x = dev(X)
    s, y = rp.add_rmsnorm_rows(x, x)
    S, Y, _ = generation.add_rmsnorm_rows(X, X)
    assert_bits_equal(host(s), S)
    assert_bits_equal(host(y), Y)
    q, sc = rp.quantize_rows(x)
    Q, SC = generation.quantize_rows(X)
    assert_bits_equal(host(rp.matmul_q8(q, sc, q, sc, sc)), generation.matmul_q8(Q, SC, Q, SC, SC))


# --------------------------------------------------------------------------
# offsets past 32 bits
# --------------------------------------------------------------------------

def ends(rows):
    return [0, 1, rows // 2, rows - 2, rows - 1]


def test_norm_and_quantiser_past_2_31_elements(rp):
    import torch
    rows, cols = 530_000, 4096  # 2.17e9 elements
    announce("long norm", rows, cols)
    X = torch.empty(rows, cols, device="cuda:0").normal_()
    R = torch.empty(rows, cols, device="cuda:0").normal_()
    at = ends(rows)
    x, r = host(X[at]), host(R[at])
    stat, Q = torch.empty(rows, device="cuda:0"), torch.empty(rows, cols, dtype=torch.int8, device="cuda:0")
    announce("long norm", "forward")
    _, q, sc = rp.add_rmsnorm_quantize_rows(X, R, sum_out=X, out=R, q_out=Q, rstd_out=stat)
    S, Y, rstd = generation.add_rmsnorm_rows(x, r)
    codes, scale = generation.quantize_rows(Y)
    assert_bits_equal(host(X[at]), S)
    assert_bits_equal(host(R[at]), Y)
    assert_bits_equal(host(stat[at]), rstd)
    assert_bits_equal(host(sc[at]), scale)
    assert np.array_equal(host(q[at]), codes)
    announce("long norm", "quantiser")
    Q.zero_()
    q, sc = rp.quantize_rows(R, q_out=Q)
    assert_bits_equal(host(sc[at]), scale)
    assert np.array_equal(host(q[at]), codes)
    announce("long norm", "backward")
    dx, dg = rp.add_rmsnorm_backward_rows(X, R, stat, None, R, dx_out=R)  # dY = dS = Y
    want, _ = generation.add_rmsnorm_backward_rows(S, Y, rstd, None, Y)
    assert_bits_equal(host(dx[at]), want)
    # dgamma sums y t = y^2, of mean 1: its sums over 530000 rows of about unit squares
    # (variance 2) stay within ten standard deviations, 10 sqrt(2 / 530000) < 0.02
    assert (np.abs(host(dg).astype(np.float64) / rows - 1) < 0.02).all()


def test_product_past_2_31_codes(rp):
    import torch
    n, k = 150_001, 14_336  # 2.15e9 codes
    for m in (3, 70):
        g = inputs.rng(3800 + m)
        B = torch.empty(n, k, dtype=torch.int8, device="cuda:0").random_(-128, 128)
        A = g.integers(-128, 128, (m, k)).astype(np.int8)
        sa, sb = inputs.uniform(g, (m,), 0.01, 0.1), inputs.uniform(g, (n,), 0.01, 0.1)
        announce("long product", m, n, k)
        got = rp.matmul_q8(dev(A), dev(sa), B, dev(sb))
        at = [0, 1, n // 2, n - 130, n - 2, n - 1]
        assert_bits_equal(host(got[:, at].contiguous()), generation.matmul_q8(A, sa, host(B[at]), sb[at]))
        # the long operand on the left
        announce("long product", n, m, k)
        got = rp.matmul_q8(B, dev(sb), dev(A), dev(sa))
        assert_bits_equal(host(got[at]), generation.matmul_q8(host(B[at]), sb[at], A, sa))


def test_draw_past_2_31_logits(rp):
    import torch
    for rows, vocab in ((2100, 1 << 20), (140_000, 16_000)):
        announce("long draw", rows, vocab)
        L = torch.empty(rows, vocab, device="cuda:0").normal_(0, 2.5)
        g = inputs.rng(3900)
        u = g.random(rows, dtype=np.float32)
        p, k = np.full(rows, 0.9, np.float32), g.choice(np.array([0, 50, 1000], np.int32), rows)
        token, prob = rp.sample_rows(L, dev(u), top_k=dev(k), top_p=dev(p))
        at = ends(rows)
        want = generation.sample_rows(host(L[at]), u[at], top_k=k[at], top_p=p[at])
        assert np.array_equal(host(token[at]), want[0])
        assert_bits_equal(host(prob[at]), want[1])
        assert int(token.min()) >= 0
        del L


def test_overlaps_are_refused_before_any_launch(rp):
    import torch
    x, r = torch.ones(8, 64, device="cuda:0"), torch.ones(8, 64, device="cuda:0")
    q = torch.zeros(8, 64, dtype=torch.int8, device="cuda:0")
    v = torch.ones(8, device="cuda:0")
    announce("overlaps refused")
    for call in (lambda: rp.add_rmsnorm_rows(x, r, sum_out=x, out=x),
                 lambda: rp.add_rmsnorm_rows(x[:4], r[:4], sum_out=x[2:6]),
                 lambda: rp.add_rmsnorm_quantize_rows(x, r, q_out=x.view(torch.int8)[:, :64]),
                 lambda: rp.quantize_rows(x, q_out=x.view(torch.int8)[:, 64:128]),
                 lambda: rp.add_rmsnorm_backward_rows(x, r, v, dgamma_out=r[0]),
                 lambda: rp.matmul_q8(q, v, q, v, out=x[:, :8], bias=x[0, :8]),
                 lambda: rp.sample_rows(x, v, prob_out=v)):
        with pytest.raises(rp.RepopsError):
            call()
    assert (host(x) == 1).all() and (host(r) == 1).all() and (host(q) == 0).all() and (host(v) == 1).all()
