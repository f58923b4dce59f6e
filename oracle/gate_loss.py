"""What a gate is trained with (oracle; test infrastructure), in binary64, a token at a time: how its choice uses the experts, the balance loss
and the z loss, and the gradient of the mixture weights and of both losses on the logits.

    q_te   softmax(z_t), or sigmoid(z_te) / sum_i sigmoid(z_ti)
    balance = mean over sequences s with tokens of  E / (k T_s^2) sum_e c_se P_se,   P_se = sum_t q_te        z = mean over tokens of (log sum exp z_t)^2
"""
import numpy as np


def _exp_from_largest(z, among=None):
    """exp(z - largest) and the largest (0 where nothing is left)."""
    top = np.max(z if among is None else among, initial=-np.inf)
    top = 0.0 if np.isneginf(top) else top
    with np.errstate(over="ignore", invalid="ignore"):
        return np.exp(z - top), top


def log_sum(z):
    if np.isneginf(z).all():
        return 0.0
    e, top = _exp_from_largest(z)
    return top + np.log(e.sum())


def softmax(z):
    e, _ = _exp_from_largest(z)
    total = e.sum()
    return e if total == 0 else e / total


def sigmoid(z):
    """sigmoid(z) and 1 - sigmoid(z)."""
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z)), 1.0 / (1.0 + np.exp(z))


def scaled_sigmoids(z):
    """Sigmoids times one positive factor that keeps the largest of them in range."""
    c = min(np.max(z, initial=-np.inf), 0.0)
    if np.isneginf(c):
        return np.zeros_like(z)
    return np.exp(z - c) / (1.0 + np.exp(z)) if c < 0 else sigmoid(z)[0]


def shares(z, sigmoid_scores):
    """The scores divided by their sum."""
    if not sigmoid_scores:
        return softmax(z)
    s = scaled_sigmoids(z)
    total = s.sum()
    return s if total == 0 else s / total


def sequences(T, offsets):
    return [(0, T)] if offsets is None else list(zip(offsets[:-1], offsets[1:]))


def balance(z, ids, gate, mask=None, offsets=None):
    """(losses [2], counts [S, E], score sums [S, E], kept [S])."""
    z, ids = np.asarray(z, dtype=np.float64), np.asarray(ids)
    T, E = z.shape
    k = ids.shape[1]
    seqs = sequences(T, offsets)
    counts, sums, kept = np.zeros((len(seqs), E), np.int32), np.zeros((len(seqs), E)), np.zeros(len(seqs), np.int32)
    squares = []
    for s, (a, b) in enumerate(seqs):
        for t in range(a, b):
            if mask is not None and not mask[t]:
                continue
            kept[s] += 1
            for i in ids[t]:
                if 0 <= i < E:
                    counts[s, i] += 1
            sums[s] += shares(z[t], gate.score == "sigmoid")
            squares.append(log_sum(z[t]) ** 2)
    per = [E / (k * float(n) ** 2) * (c * p).sum() for n, c, p in zip(kept, counts, sums) if n]
    return np.array([np.mean(per) if per else 0.0, np.mean(squares) if squares else 0.0]), counts, sums, kept


def weights(z_t, ids_t, gate):
    """Mixture weights of one token's choice."""
    E = len(z_t)
    ok = (ids_t >= 0) & (ids_t < E)
    at = np.where(ok, ids_t, 0)
    if gate.renormalise:
        w = shares(np.where(ok, z_t[at], -np.inf), gate.score == "sigmoid")
    else:
        w = (sigmoid(z_t)[0] if gate.score == "sigmoid" else softmax(z_t))[at]
    return np.where(ok, w, 0.0) * gate.scale


def backward(z, ids, gate, top_k, d_weights=None, d_losses=None, counts=None, kept=None, mask=None, offsets=None):
    """(gradient [T, E], magnitude [T, E] of the terms it is a sum of)."""
    z = np.asarray(z, dtype=np.float64)
    T, E = z.shape
    out, size = np.zeros((T, E)), np.zeros((T, E))
    of = np.full(T, -1)
    for s, (a, b) in enumerate(sequences(T, offsets)):
        of[a:b] = s
    sig = gate.score == "sigmoid"
    if d_losses is not None:
        d_losses, kept, counts = np.asarray(d_losses, np.float64), np.asarray(kept, np.float64), np.asarray(counts, np.float64)
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        p, rest = softmax(z[t]), sigmoid(z[t])[1]
        if d_losses is not None and of[t] >= 0 and kept[of[t]] > 0:
            q = shares(z[t], sig)
            G = d_losses[0] * E * counts[of[t]] / (top_k * (kept > 0).sum() * kept[of[t]] ** 2)
            back = q * rest if sig else q
            zl = d_losses[1] * 2 / kept.sum() * log_sum(z[t]) * p
            out[t] += back * (G - (q * G).sum()) + zl
            size[t] += back * (np.abs(G) + (q * np.abs(G)).sum()) + np.abs(zl)
        if d_weights is not None:
            at = np.asarray(ids[t])
            ok = (at >= 0) & (at < E)
            at, d = np.where(ok, at, 0), np.where(ok, np.asarray(d_weights[t], np.float64) * gate.scale, 0.0)
            if gate.renormalise:
                r = shares(np.where(ok, z[t][at], -np.inf), sig)
                one, big = r * (d - (r * d).sum()), r * (np.abs(d) + (r * np.abs(d)).sum())
                if sig:
                    one, big = one * rest[at], big * rest[at]
            elif sig:
                one = sigmoid(z[t])[0][at] * rest[at] * d
                big = np.abs(one)
            else:
                one = p[at] * d
                big = np.abs(one)
                out[t] -= p * one.sum()
                size[t] += p * big.sum()
            np.add.at(out[t], at[ok], one[ok])
            np.add.at(size[t], at[ok], big[ok])
    return out, size
