"""A dense product with its epilogue (oracle; test infrastructure), in binary64:

    out = residual + act(x W^T + bias)      or      residual + act(x W^T + bias) * (x U^T + bias_up)
"""
import math

import numpy as np

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activate(v, activation):
    v = np.asarray(v, dtype=np.float64)
    with np.errstate(over="ignore"):
        if activation == "relu":
            return np.where(v < 0, 0.0, v)
        if activation == "gelu":
            return 0.5 * v * _erfc(-v / math.sqrt(2.0))
        if activation == "gelu_tanh":
            return 0.5 * v * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
        if activation == "silu":
            return v / (1.0 + np.exp(-v))
    assert activation == "none"
    return v


def apply(x, w, bias=None, w_up=None, bias_up=None, activation="none", residual=None):
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    out = activate(x @ w.T + (0.0 if bias is None else np.asarray(bias, dtype=np.float64)), activation)
    if w_up is not None:
        out = out * (x @ np.asarray(w_up, dtype=np.float64).T + (0.0 if bias_up is None else np.asarray(bias_up, dtype=np.float64)))
    return out if residual is None else np.asarray(residual, dtype=np.float64) + out


def magnitude(x, w, bias=None):
    """|x| |W|^T + |bias|: what the roundings of a sum of these products are relative to."""
    m = np.abs(np.asarray(x, dtype=np.float64)) @ np.abs(np.asarray(w, dtype=np.float64)).T
    return m if bias is None else m + np.abs(np.asarray(bias, dtype=np.float64))
