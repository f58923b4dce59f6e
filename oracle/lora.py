"""Low-rank adapters beside a shared projection (oracle; test infrastructure), one token at a time, in binary64:

    out_t = base_t + scale_a * B_a (A_a x_t),  a = ids_t;  out_t = base_t where ids_t is no adapter.
"""
import numpy as np


def apply(x, a, b, scale, ids, base=None):
    x, a, b, scale = (np.asarray(v, dtype=np.float64) for v in (x, a, b, scale))
    out = np.zeros((x.shape[0], b.shape[1])) if base is None else np.array(base, dtype=np.float64)
    for t, i in enumerate(np.asarray(ids)):
        if 0 <= i < a.shape[0]:
            out[t] += scale[i] * (b[i] @ (a[i] @ x[t]))
    return out


def magnitude(x, a, b, scale, ids):
    """|scale| |B| (|A| |x|): what the roundings of a sum of these products are relative to."""
    return apply(np.abs(x), np.abs(a), np.abs(b), np.abs(scale), ids)


def groups(ids, num_adapters):
    """Tokens by adapter, ascending; those without one (or with an id out of range) last, as adapter -1."""
    ids = np.asarray(ids)
    out = [(i, np.flatnonzero(ids == i).tolist()) for i in range(num_adapters)]
    out.append((-1, np.flatnonzero((ids < 0) | (ids >= num_adapters)).tolist()))
    return [(i, rows) for i, rows in out if rows]
