"""Gate of a sparse block (oracle; test infrastructure): scores, balance bias, groups, top-k, weights, one token at a time.

    scores   s = softmax(z) over all experts, or 1 / (1 + exp(-z))
    choice   c = s + balance; an expert with z = -inf has s = 0 and comes after all others
    groups   equal runs of experts; a group's value is its largest c or the sum of its two largest; the best `top_groups` stay
    experts  the k largest c of the groups that stay; without a balance bias by z itself, which orders them as s does
    weights  s of the chosen, over their sum if renormalised, times scale

Equal values: the lower group, the lower expert.  A NaN comes last.  Binary64 throughout.
"""
import math

import numpy as np


def scores(z, score):
    z = np.asarray(z, dtype=np.float64)
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-z))
    top = max((v for v in z if not math.isnan(v)), default=0.0)
    if top == -np.inf:
        return np.zeros_like(z)
    with np.errstate(invalid="ignore"):
        e = np.exp(z - top)
        return e / np.sum(e)


def _place(v):
    """Sorts descending, -inf behind numbers, NaN behind -inf."""
    return (1, 0.0) if math.isnan(v) else (0, -v)


def choose_token(z, gate, top_k, balance=None):
    z = np.asarray(z, dtype=np.float64)
    E = len(z)
    s = scores(z, gate.score)
    c = [-np.inf if z[e] == -np.inf else s[e] + (0.0 if balance is None else float(balance[e])) for e in range(E)]
    by = list(z) if balance is None else c
    size = E // gate.num_groups
    groups = list(range(gate.num_groups))
    if gate.top_groups < gate.num_groups:
        value = {}
        for g in groups:
            best = sorted((v for v in (c if gate.group_score == "top2" else by)[g * size:(g + 1) * size] if not math.isnan(v)), reverse=True)
            live = [v for v in best if v > -np.inf]
            value[g] = sum(live[:2]) if live and gate.group_score == "top2" else live[0] if live else -np.inf
        groups = sorted(groups, key=lambda g: (-value[g], g))[:gate.top_groups]
    experts = [e for e in range(E) if e // size in groups]
    ids = sorted(experts, key=lambda e: (_place(by[e]), e))[:top_k]
    w = s[ids]
    if gate.renormalise:
        total = np.sum(w)
        w = np.zeros_like(w) if total == 0 else w / total
    return np.asarray(ids, dtype=np.int32), w * gate.scale


def choose(z, gate, top_k, balance=None):
    """ids int32 [T, k], weights float64 [T, k] of logits [T, E]."""
    rows = [choose_token(row, gate, top_k, balance) for row in np.asarray(z, dtype=np.float64)]
    return np.array([i for i, _ in rows], dtype=np.int32).reshape(len(rows), top_k), np.array([w for _, w in rows]).reshape(len(rows), top_k)


def logits(hidden, w_router, bias=None, addend=None):
    z = np.asarray(hidden, dtype=np.float64) @ np.asarray(w_router, dtype=np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, dtype=np.float64)
    return z if addend is None else z + np.asarray(addend, dtype=np.float64)
