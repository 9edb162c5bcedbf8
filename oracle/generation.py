"""CPU oracle of the generation-step operators (TEST INFRASTRUCTURE ONLY).

The residual addition with its norm is one binary32 addition and the norm's
oracle; the 8-bit codes are numpy's binary32 divisions, products and rounding to even
(all IEEE operations); the 8-bit product is an exact integer product and three rounded
multiplications; the drawing of a token is ``sample_ref.c``.  No code is shared
with the GPU path.
"""
from __future__ import annotations

import ctypes
import os
import subprocess

import numpy as np

import oracle

_HERE = os.path.dirname(os.path.abspath(__file__))
_SRC = os.path.join(_HERE, "sample_ref.c")
LIB_PATH = os.path.join(_HERE, "libsample_ref.so")
CFLAGS = ["-std=c11", "-O2", "-ffp-contract=off", "-fno-fast-math", "-mfma", "-fPIC", "-shared",
          "-Wall"]
_lib = None


def build(out: str | None = None, src: str | None = None) -> str:
    out = out or LIB_PATH
    tmp = out + ".tmp"
    subprocess.run(["gcc", *CFLAGS, "-o", tmp, src or _SRC, "-lm"], check=True)
    os.replace(tmp, out)
    return out


def load(path: str | None = None):
    global _lib
    if _lib is not None and path is None:
        return _lib
    if path is None and not os.path.exists(LIB_PATH):
        build()
    lib = ctypes.CDLL(path or LIB_PATH)
    f, i32, i64 = ctypes.c_float, ctypes.c_int32, ctypes.c_int64
    lib.sample_ref_weight.restype, lib.sample_ref_weight.argtypes = ctypes.c_uint64, [ctypes.c_double]
    lib.sample_ref_log.restype, lib.sample_ref_log.argtypes = ctypes.c_double, [f]
    lib.sample_ref_row.restype = i32
    lib.sample_ref_row.argtypes = [i64, ctypes.c_void_p, f, f, i32, f, f, ctypes.POINTER(f)]
    if path is None:
        _lib = lib
    return lib


def _f32(a):
    return np.ascontiguousarray(a, np.float32)


def quantize_rows(Y):
    """(codes, scales) of the rows of Y."""
    Y = _f32(Y)
    with np.errstate(all="ignore"):
        top = np.abs(Y).max(axis=1, initial=0.0) if Y.size else np.zeros(len(Y), np.float32)
        top = np.where(np.isfinite(Y).all(axis=1), top, np.float32(np.nan)).astype(np.float32)
        scale = (top / np.float32(127.0)).astype(np.float32)
        lift = np.where(scale < np.float32(2.0 ** -100), np.float32(2.0 ** 120), np.float32(1.0))
        r = (np.float32(1.0) / (scale * lift).astype(np.float32)).astype(np.float32)
        q = np.rint(((Y * lift[:, None]).astype(np.float32) * r[:, None]).astype(np.float32))
        q = np.where(scale[:, None] > 0, np.clip(q, -127, 127), 0)
    return q.astype(np.int8), scale


def add_rmsnorm_rows(X, R=None, gamma=None, eps=1e-5, **order):
    """(S, Y, rstd)."""
    S = _f32(X) if R is None else (_f32(X) + _f32(R)).astype(np.float32)
    Y, rstd = oracle.rmsnorm_rows(S, gamma, eps, with_stats=True, **order)
    return S, Y, rstd


def add_rmsnorm_backward_rows(S, dY, rstd, gamma=None, dS=None, **order):
    """(dX, dgamma)."""
    dX, dgamma = oracle.rmsnorm_backward_rows(S, dY, rstd, gamma, **order)
    return dX if dS is None else (dX + _f32(dS)).astype(np.float32), dgamma


def matmul_q8(A, a_scale, B, b_scale, bias=None):
    """Integer sums as float64 products, exact below 2^53."""
    acc = A.astype(np.float64) @ B.astype(np.float64).T
    C = acc.astype(np.float32)
    C = (C * _f32(a_scale)[:, None]).astype(np.float32)
    C = (C * _f32(b_scale)).astype(np.float32)
    return C if bias is None else (C + _f32(bias)).astype(np.float32)


def sample_rows(L, u, temperature=None, top_k=None, top_p=None, min_p=None, lib=None):
    """(tokens, probabilities)."""
    lib = lib or load()
    L = _f32(L)
    rows, n = L.shape

    def at(p, r, default):
        return default if p is None else p[r].item()
    tokens, probs = np.empty(rows, np.int32), np.empty(rows, np.float32)
    for r in range(rows):
        row, p = np.ascontiguousarray(L[r]), ctypes.c_float(0)
        tokens[r] = lib.sample_ref_row(n, row.ctypes.data, float(u[r]), at(temperature, r, 1.0),
                                       at(top_k, r, 0), at(top_p, r, 1.0), at(min_p, r, 0.0),
                                       ctypes.byref(p))
        probs[r] = p.value
    return tokens, probs


def feed_forward_q8(X, R, gamma, gate, up, down, eps=1e-5):
    """llama_feed_forward_q8's values by name."""
    S, N, _ = add_rmsnorm_rows(X, R, gamma, eps)
    Q, scale = quantize_rows(N)
    G, U = matmul_q8(Q, scale, *gate), matmul_q8(Q, scale, *up)
    H = oracle.swiglu(G, U)
    HQ, h_scale = quantize_rows(H)
    return {"S": S, "Q": Q, "scale": scale, "G": G, "U": U, "H": H, "HQ": HQ, "h_scale": h_scale,
            "D": matmul_q8(HQ, h_scale, *down)}


def next_token(X, R, gamma, head, u, eps=1e-5, **filters):
    """llama_next_token's values by name."""
    Q, scale = quantize_rows(add_rmsnorm_rows(X, R, gamma, eps)[1])
    logits = matmul_q8(Q, scale, *head)
    token, prob = sample_rows(logits, u, **filters)
    return {"Q": Q, "scale": scale, "logits": logits, "token": token, "prob": prob}


def norm_linear(X, R, gamma, W, dY, dS=None, eps=1e-5):
    """(S, Y, dX, dgamma, dW) of norm_linear_forward and its backward."""
    S, N, rstd = add_rmsnorm_rows(X, R, gamma, eps)
    dX, dgamma = add_rmsnorm_backward_rows(S, oracle.matmul(dY, W, trans_b=True), rstd, gamma, dS)
    return S, oracle.matmul(N, W), dX, dgamma, oracle.matmul(N, dY, trans_a=True)
