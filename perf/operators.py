"""The operators around the products of a Llama generation step, and their plain forms.

Residual addition with RMSNorm (fp32 output, or 8 bits with a scale per row; and
its gradients), the row quantiser, the product of 8-bit operands and the drawing
of a token from given random numbers.  ``listed()`` fixes points of each range of
sizes, ``draw()`` picks others; the widths are those of the package's own Llama
layers (4096 / 14336), the DistilBERT block (768) and generic ones, the
vocabularies generic.

``run`` computes the plain forms with elementary torch operations, or, where
``own`` is true, makes the calls of ``paper_2502_19405_amd.repops``.  ``exact``
restates each in 64 bits.  Values held in 8 bits are returned as what they stand
for, q * scale, in bfloat16: an 8-bit code has at most 7 significant bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # Eight sequences' next tokens entering a layer: a call where latency counts.
        {"name": "norm_decode", "op": "norm", "rows": 8, "cols": 4096, "q8": False},
        # Prefill of two long prompts, the normalised rows handed to an 8-bit product.
        {"name": "norm_q8_prefill", "op": "norm", "rows": 8192, "cols": 4096, "q8": True},
        # Training: forward and backward of a Llama layer's norm over 4 x 1024 tokens.
        {"name": "norm_train", "op": "norm_train", "rows": 4096, "cols": 4096},
        # The same where neither size fits anything: a short last batch, an odd width.
        {"name": "norm_train_odd", "op": "norm_train", "rows": 1531, "cols": 1001},
        # Decoding: the gated activations of 64 tokens before the down projection.
        {"name": "quant_activations", "op": "quant", "rows": 64, "cols": 14336},
        # Laying out a Llama weight: one scale per output feature.
        {"name": "quant_weight", "op": "quant", "rows": 14336, "cols": 4096},
        # Decoding: four tokens through a linear layer, bound by reading the weight.
        {"name": "q8_decode", "op": "q8", "m": 4, "n": 14336, "k": 4096, "bias": False},
        # Sizes that fit no tile and rows that are not aligned, with a bias.
        {"name": "q8_ragged", "op": "q8", "m": 333, "n": 1001, "k": 999, "bias": True},
        # Prefill of 8192 tokens: the largest product of the layer.
        {"name": "q8_prefill", "op": "q8", "m": 8192, "n": 14336, "k": 4096, "bias": False},
        # One sequence's next token, all filters on.
        {"name": "sample_one", "op": "sample", "rows": 1, "vocab": 32000, "temperature": 0.8,
         "top_k": 50, "top_p": 0.95, "min_p": 0.02, "mixed": False},
        # A serving batch whose requests ask for different filters, greedy ones among them.
        {"name": "sample_batch", "op": "sample", "rows": 64, "vocab": 128000, "temperature": 0.9,
         "top_k": 200, "top_p": 0.9, "min_p": 0.01, "mixed": True},
        # Many samples from the whole distribution of a large vocabulary.
        {"name": "sample_all", "op": "sample", "rows": 512, "vocab": 131072, "temperature": 1.0,
         "top_k": 0, "top_p": 1.0, "min_p": 0.0, "mixed": False},
    ]


def _log_int(rng, lo, hi):
    """An integer whose logarithm is uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_train", "quant", "q8", "q8", "sample", "sample"])
    if op in ("norm", "norm_train"):
        cols = rng.choice([768, 4096, _log_int(rng, 64, 16384)])
        top = 8192 * 4096 if op == "norm" else 4096 * 4096
        case = {"op": op, "rows": _log_int(rng, 1, top // cols), "cols": cols}
        if op == "norm":
            case["q8"] = rng.random() < 0.6
        return case
    if op == "quant":
        cols = rng.choice([4096, 14336, _log_int(rng, 64, 16384)])
        return {"op": op, "rows": _log_int(rng, 1, 14336 * 4096 // cols), "cols": cols}
    if op == "q8":
        m = rng.choice([rng.randint(1, 32), _log_int(rng, 1, 8192)])
        n, k = rng.choice([(4096, 4096), (14336, 4096), (4096, 14336), (1024, 4096), (32000, 4096),
                           (_log_int(rng, 64, 8192), _log_int(rng, 64, 8192)),
                           (_log_int(rng, 64, 8192), _log_int(rng, 64, 8192))])
        m = min(m, 8192 * 14336 * 4096 // (n * k))
        return {"op": op, "m": m, "n": n, "k": k, "bias": rng.random() < 0.5}
    vocab = rng.choice([32000, 128000, _log_int(rng, 256, 131072)])
    return {"op": op, "rows": _log_int(rng, 1, 512), "vocab": vocab,
            "temperature": round(rng.uniform(0.3, 1.6), 3),
            "top_k": rng.choice([0, 0, 1, 40, _log_int(rng, 1, 2000)]),
            "top_p": rng.choice([1.0, 0.9, round(rng.uniform(0.1, 0.999), 3)]),
            "min_p": rng.choice([0.0, 0.0, 0.05, round(rng.uniform(0.001, 0.3), 3)]),
            "mixed": rng.random() < 0.5}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(std)

    def uniform(*shape, lo=0.0, hi=1.0):
        return torch.rand(shape, generator=g, device=DEV, dtype=torch.float32).mul_(hi - lo).add_(lo)

    def codes(*shape):  # 8-bit values as a quantiser leaves them: normal, clipped at the ends
        return normal(*shape, std=32.0).round_().clamp_(-127, 127).to(torch.int8)

    op = case["op"]
    s = {"case": dict(case)}
    if op in ("norm", "norm_train"):
        r, c = case["rows"], case["cols"]
        s.update(X=normal(r, c), R=normal(r, c, std=2.0), gamma=uniform(c, lo=0.5, hi=1.5))
        if op == "norm_train":
            s.update(dY=normal(r, c, std=0.01), dS=normal(r, c, std=0.01))
        return s
    if op == "quant":
        s["X"] = normal(case["rows"], case["cols"], std=0.02)
        return s
    if op == "q8":
        m, n, k = case["m"], case["n"], case["k"]
        s.update(A=codes(m, k), a_scale=uniform(m, lo=0.01, hi=0.05), B=codes(n, k),
                 b_scale=uniform(n, lo=0.0002, hi=0.001), bias=None)
        if case["bias"]:
            s["bias"] = uniform(n, lo=-0.5, hi=0.5)
        return s
    rows, vocab = case["rows"], case["vocab"]
    s["logits"] = normal(rows, vocab, std=2.5)
    # a few likely tokens in each row, as a model that has settled on them gives
    peaks = (torch.rand((rows, 8), generator=g, device=DEV) * vocab).long().clamp_(max=vocab - 1)
    s["logits"].scatter_(1, peaks, uniform(rows, 8, lo=6.0, hi=14.0))
    s["u"] = uniform(rows)
    t = torch.full((rows,), case["temperature"], device=DEV, dtype=torch.float32)
    k = torch.full((rows,), case["top_k"], device=DEV, dtype=torch.int32)
    p = torch.full((rows,), case["top_p"], device=DEV, dtype=torch.float32)
    m = torch.full((rows,), case["min_p"], device=DEV, dtype=torch.float32)
    if case["mixed"]:  # every request its own: some without a filter, some greedy
        at = torch.arange(rows, device=DEV)
        k[at % 2 == 1] = 0
        p[at % 3 == 1] = 1.0
        m[at % 5 != 2] = 0.0
        t[at % 7 == 3] = 0.0
    s.update(temperature=t, top_k=k, top_p=p, min_p=m)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    return (_own if own else _plain)[op](state)


def _stands_for(q, scale):
    """q * scale in bfloat16, from codes (int8, or whole numbers in float32)."""
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    return torch.mul(q, scale[:, None], out=out)


def _codes_plain(y):
    scale = y.abs().amax(1) / torch.full((1,), 127.0, device=y.device)
    return (y / scale[:, None]).round_().clamp_(-127, 127), scale


def _norm_plain(s):
    S = s["X"] + s["R"]
    rstd = 1.0 / torch.sqrt((S * S).mean(1, keepdim=True) + 1e-5)
    Y = S * rstd * s["gamma"]
    if not s["case"].get("q8"):
        return {"S": S, "Y": Y}
    q, scale = _codes_plain(Y)
    return {"S": S, "Q": _stands_for(q, scale), "scale": scale}


def _norm_train_plain(s):
    S = s["X"] + s["R"]
    rstd = 1.0 / torch.sqrt((S * S).mean(1, keepdim=True) + 1e-5)
    t = S * rstd
    Y = t * s["gamma"]
    g = s["dY"] * s["gamma"]
    dX = rstd * (g - t * (g * t).mean(1, keepdim=True)) + s["dS"]
    return {"S": S, "Y": Y, "dX": dX, "dgamma": (s["dY"] * t).sum(0)}


def _quant_plain(s):
    q, scale = _codes_plain(s["X"])
    return {"Q": _stands_for(q, scale), "scale": scale}


def _q8_plain(s):
    C = s["A"].float() @ s["B"].float().t()
    C = C * s["a_scale"][:, None] * s["b_scale"]
    return C if s["bias"] is None else C + s["bias"]


def _sample_plain(s):
    # 64 bits: a random number next to a border decides between two tokens
    v, index = torch.sort(s["logits"], dim=1, descending=True, stable=True)
    greedy = s["temperature"] <= 0
    temperature = torch.where(greedy, 1.0, s["temperature"].double())[:, None]
    v = v.double()
    d = (v - v[:, :1]) / temperature
    w = torch.exp(d)
    before = torch.cumsum(w, 1) - w
    at = torch.arange(w.shape[1], device=w.device)
    k = torch.where(s["top_k"] > 0, s["top_k"], w.shape[1])[:, None]
    keep = at < k
    p = s["top_p"].double()[:, None]
    keep &= (before < p * (w * keep).sum(1, keepdim=True)) | (p >= 1)
    m = s["min_p"].double()[:, None]
    keep &= (d >= torch.log(m)) | (m <= 0)
    keep &= (at == 0) | ~greedy[:, None]
    keep[:, 0] = True
    w = w * keep
    c = torch.cumsum(w, 1)
    i = (c <= s["u"].double()[:, None] * c[:, -1:]).sum(1)
    i = torch.minimum(i, keep.sum(1) - 1)[:, None]
    prob = w.gather(1, i) / c[:, -1:]
    return {"token": index.gather(1, i)[:, 0].int(), "prob": prob[:, 0].float()}


_plain = {"norm": _norm_plain, "norm_train": _norm_train_plain, "quant": _quant_plain,
          "q8": _q8_plain, "sample": _sample_plain}


def _repops():
    from paper_2502_19405_amd import repops
    return repops


def _norm_own(s):
    if not s["case"]["q8"]:
        S, Y = _repops().add_rmsnorm_rows(s["X"], s["R"], s["gamma"])
        return {"S": S, "Y": Y}
    S, Q, scale = _repops().add_rmsnorm_quantize_rows(s["X"], s["R"], s["gamma"])
    return {"S": S, "Q": _stands_for(Q, scale), "scale": scale}


def _norm_train_own(s):
    rstd = torch.empty(s["X"].shape[0], dtype=torch.float32, device=DEV)
    S, Y = _repops().add_rmsnorm_rows(s["X"], s["R"], s["gamma"], rstd_out=rstd)
    dX, dgamma = _repops().add_rmsnorm_backward_rows(S, s["dY"], rstd, s["gamma"], dS=s["dS"])
    return {"S": S, "Y": Y, "dX": dX, "dgamma": dgamma}


def _quant_own(s):
    Q, scale = _repops().quantize_rows(s["X"])
    return {"Q": _stands_for(Q, scale), "scale": scale}


def _q8_own(s):
    return _repops().matmul_q8(s["A"], s["a_scale"], s["B"], s["b_scale"], s["bias"])


def _sample_own(s):
    token, prob = _repops().sample_rows(s["logits"], s["u"], temperature=s["temperature"],
                                        top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return {"token": token, "prob": prob}


_own = {"norm": _norm_own, "norm_train": _norm_train_own, "quant": _quant_own, "q8": _q8_own,
        "sample": _sample_own}


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "norm":
        e = case["rows"] * case["cols"]
        return {"bytes": e * (13 if case["q8"] else 16) + 4 * case["cols"], "flops": 5 * e}
    if op == "norm_train":
        e = case["rows"] * case["cols"]
        return {"bytes": 28 * e + 8 * case["cols"], "flops": 16 * e}
    if op == "quant":
        e = case["rows"] * case["cols"]
        return {"bytes": 5 * e + 4 * case["rows"], "flops": 2 * e}
    if op == "q8":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k + n * k + 4 * (m * n + m + n), "flops": 2 * m * n * k}
    e = case["rows"] * case["vocab"]
    return {"bytes": 4 * e + 28 * case["rows"], "flops": 3 * e}


def _exact_codes(y):
    step = y.abs().max(dim=1).values.div(127)
    return {"Q": torch.mul(torch.round(torch.div(y.t(), step)), step).t(), "scale": step}


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if op in ("norm", "norm_train"):
        n = case["cols"]
        S = torch.add(d["X"], d["R"])
        root = torch.linalg.vector_norm(S, dim=1).square().div(n).add(1e-5).sqrt()
        unit = torch.div(S.t(), root).t()
        Y = torch.mul(unit, d["gamma"])
        if op == "norm":
            return {"S": S, **_exact_codes(Y)} if case["q8"] else {"S": S, "Y": Y}
        # y = gamma s / root: dy/ds has the diagonal gamma / root and -gamma s s^T / (n root^3)
        back = torch.mul(d["dY"], d["gamma"])
        along = torch.mul(back, S).sum(1) / (n * root.pow(3))
        dX = d["dS"] + torch.div(back.t(), root).t() - torch.mul(S.t(), along).t()
        return {"S": S, "Y": Y, "dX": dX, "dgamma": torch.mul(unit, d["dY"]).sum(0)}
    if op == "quant":
        return _exact_codes(d["X"])
    if op == "q8":
        left, right = torch.mul(d["A"].t(), d["a_scale"]).t(), torch.mul(d["B"].t(), d["b_scale"])
        C = torch.mm(left, right.contiguous())
        return C if s["bias"] is None else torch.add(C, d["bias"])
    # the draw, row by row on the host: walk the tokens from the likeliest down
    h = {k: v.cpu().numpy() for k, v in d.items()}
    prob = np.empty(case["rows"])
    for r in range(case["rows"]):
        z = h["logits"][r]
        walk = np.lexsort((np.arange(z.size), -z))
        if h["temperature"][r] <= 0:
            prob[r] = 1.0
            continue
        e = np.exp((z[walk] - z[walk[0]]) / h["temperature"][r])
        count = z.size
        if h["top_k"][r] > 0:
            count = min(count, int(h["top_k"][r]))
        total = np.add.accumulate(e[:count])
        if h["top_p"][r] < 1:
            count = min(count, 1 + int(np.searchsorted(total, h["top_p"][r] * total[-1])))
        if h["min_p"][r] > 0:
            count = min(count, max(1, int((e >= h["min_p"][r]).sum())))
        total = total[:count]
        i = int(np.searchsorted(total, h["u"][r] * total[-1], side="right"))
        prob[r] = e[min(i, count - 1)] / total[-1]
    return {"token": None, "prob": torch.from_numpy(prob)}
