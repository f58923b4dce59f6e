"""What stands around a sparse block's routed experts: products with an epilogue, and the gate's losses and gradients; and the same in elementary torch.

Four kinds of cases:

  linear    `exmoe_linear`: residual + act(x W^T + bias), BF16 or (a router's logits) FP32 results.
  shared    a shared expert by two of them: silu(x W^T) * (x U^T), then the down matrix with the routed experts' output as residual.
  loss      `exmoe_balance_loss`: per sequence how often each expert was chosen and the sum of its scores, the balance loss and the z loss.
  backward  `exmoe_gate_backward`: the gradient on the logits of the mixture weights and of both losses.

Hidden states N(0, 1), weights N(0, 0.02), as the layer's synthetic inputs; logits N(0, 1) with experts that are liked and disliked; sequences
of uneven lengths, the tokens behind a sequence's end masked.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _linear(tokens, k, n, activation="none", gated=False, bias=False, residual=False, dtype="bfloat16", stride=0):
    return dict(kind="linear", tokens=tokens, k=k, n=n, activation=activation, gated=gated, bias=bias, residual=residual, dtype=dtype, stride=stride)


def _shared(tokens, d_model, d_ff):
    return dict(kind="shared", tokens=tokens, d_model=d_model, d_ff=d_ff)


def _gate(kind, tokens, experts, top_k, score="softmax", dtype="float32", sequences=0, masked=0.0, off=0.0, **more):
    return dict(kind=kind, tokens=tokens, experts=experts, top_k=top_k, score=score, dtype=dtype, sequences=sequences, masked=masked, off=off, **more)


def _backward(tokens, experts, top_k, renormalise=False, scale=1.0, weights=True, losses=True, **more):
    return _gate("backward", tokens, experts, top_k, renormalise=renormalise, scale=scale, weights=weights, losses=losses, **more)


def listed():
    return [
        # one user's token through a 2048 x 2048 projection, added to the residual stream
        dict(_linear(1, 2048, 2048, residual=True), name="linear_1"),
        # logits of a short prompt for a router of 60 experts, FP32 with a bias
        dict(_linear(250, 2048, 60, bias=True, dtype="float32"), name="linear_logits_250"),
        # a batch of odd size, an odd number of outputs, GELU with a bias; x is a column range of wider rows
        dict(_linear(777, 1408, 2049, activation="gelu", bias=True, residual=True, stride=2816), name="linear_777"),
        # prefill through a projection, added to the residual stream
        dict(_linear(8192, 2048, 2048, residual=True), name="linear_8192"),
        # the shared expert of a block with 1408-wide routed ones, one token
        dict(_shared(1, 2048, 5632), name="shared_1"),
        # ... a decode batch of odd size
        dict(_shared(45, 2048, 5632), name="shared_45"),
        # ... a batch of prompts
        dict(_shared(4096, 2048, 5632), name="shared_4096"),
        # the load of a decode batch: counts for the balance bias
        dict(_gate("loss", 16, 64, 8), name="loss_16"),
        # prompts of 12 sequences, the ends of some masked, BF16 logits, normalised sigmoids: one loss per sequence
        dict(_gate("loss", 8191, 256, 8, score="sigmoid", dtype="bfloat16", sequences=12, masked=0.1), name="loss_8191"),
        # a training batch of the 64-expert top-8 model as one sequence
        dict(_gate("loss", 131072, 64, 8), name="loss_131072"),
        # a fine-tuning step of odd size on 60 experts in use four at a time, renormalised softmax, some experts switched off
        dict(_backward(333, 60, 4, renormalise=True, off=0.05), name="backward_333"),
        # a training batch of a wide sigmoid gate, renormalised and scaled, 16 sequences
        dict(_backward(32768, 256, 8, renormalise=True, scale=2.5, score="sigmoid", sequences=16, masked=0.05), name="backward_32768"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "linear", "shared", "loss", "loss", "backward", "backward"))
    if kind == "linear":
        gated = rng.random() < 0.3
        k, n = 8 * _log_int(rng, 16, 704), rng.choice((8 * _log_int(rng, 8, 704), _log_int(rng, 8, 5632)))
        tokens = _log_int(rng, 1, 8192)
        while tokens * k * n * (2 if gated else 1) > 8192 * 2048 * 5632:
            tokens = (tokens + 1) // 2
        return _linear(tokens, k, n, activation=rng.choice(ACTIVATIONS), gated=gated, bias=rng.random() < 0.5, residual=rng.random() < 0.5,
                       dtype=rng.choice(("bfloat16", "bfloat16", "float32")), stride=rng.choice((0, 0, 2 * k)))
    if kind == "shared":
        return _shared(_log_int(rng, 1, 4096), 64 * rng.randint(4, 32), 64 * rng.randint(2, 88))
    experts = _log_int(rng, 8, 512)
    top_k = rng.randint(1, min(16, experts))
    tokens = _log_int(rng, 1, 131072)
    while tokens * experts > 131072 * 64:
        tokens = (tokens + 1) // 2
    sequences = rng.choice((0, 0, 1, _log_int(rng, 1, max(1, tokens // 16))))
    more = dict(score=rng.choice(("softmax", "sigmoid")), dtype=rng.choice(("float32", "bfloat16")), sequences=sequences, masked=rng.choice((0.0, 0.1)),
                off=rng.choice((0.0, 0.02)))
    if kind == "loss":
        return _gate("loss", tokens, experts, top_k, **more)
    weights = rng.random() < 0.75
    return _backward(tokens, experts, top_k, renormalise=rng.random() < 0.6, scale=rng.choice((1.0, 2.5)), weights=weights,
                     losses=not weights or rng.random() < 0.75, **more)


def _normal(g, std, *size, dtype=torch.bfloat16):
    return (torch.randn(*size, generator=g, device="cuda") * std).to(dtype)


def _sequences(g, case):
    """Offsets int32 [S + 1] of sequences of uneven lengths that cover the tokens, and the mask bool [T] of those that count."""
    T, S = case["tokens"], min(case["sequences"], case["tokens"])
    ends = None
    if S:
        lengths = torch.rand(S, generator=g, device="cuda", dtype=torch.float64) + 0.1
        ends = torch.floor(torch.cumsum(lengths, 0) / lengths.sum() * (T - S) + 0.5).long() + torch.arange(1, S + 1, device="cuda")
        ends[-1] = T
    mask = None
    if case["masked"]:
        stop = torch.full((1,), T, device="cuda") if ends is None else ends
        start = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), stop[:-1]])
        kept = stop - ((stop - start) * 2 * case["masked"] * torch.rand(len(stop), generator=g, device="cuda")).long()
        of = torch.searchsorted(stop[:-1].contiguous(), torch.arange(T, device="cuda"), right=True)
        mask = torch.arange(T, device="cuda") < kept[of]
    offsets = None if ends is None else torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), ends]).int()
    return offsets, mask


def _counts(ids, offsets, mask, E):
    """Per sequence how often each expert was chosen, int32 [S, E], and the tokens that count, int32 [S]."""
    T, k = ids.shape
    of = torch.zeros(T, dtype=torch.long, device=ids.device)
    S = 1
    if offsets is not None:
        S = len(offsets) - 1
        of = torch.searchsorted(offsets[1:-1].long().contiguous(), torch.arange(T, device=ids.device), right=True)
    kept = torch.ones(T, dtype=torch.int64, device=ids.device) if mask is None else mask.long()
    counts = torch.zeros(S * E, dtype=torch.int64, device=ids.device)
    counts.index_add_(0, (of[:, None] * E + ids.long()).flatten(), kept[:, None].expand(T, k).flatten())
    tokens = torch.zeros(S, dtype=torch.int64, device=ids.device).index_add_(0, of, kept)
    return counts.view(S, E).int(), tokens.int(), of, kept


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    T, kind, state = case["tokens"], case["kind"], {"case": case}
    if kind == "linear":
        K, N = case["k"], case["n"]
        state["x"] = _normal(g, 1.0, T, case["stride"] or K)[:, :K]
        state["w"] = _normal(g, 0.02, N, K)
        state["w_up"] = _normal(g, 0.02, N, K) if case["gated"] else None
        state["bias"] = _normal(g, 0.1, N, dtype=torch.float32) if case["bias"] else None
        state["bias_up"] = _normal(g, 0.1, N, dtype=torch.float32) if case["bias"] and case["gated"] else None
        state["residual"] = _normal(g, 1.0, T, N, dtype=getattr(torch, case["dtype"])) if case["residual"] else None
        return state
    if kind == "shared":
        H, F = case["d_model"], case["d_ff"]
        state["x"], state["routed"] = _normal(g, 1.0, T, H), _normal(g, 0.2, T, H)
        state["w"], state["w_up"], state["w_down"] = _normal(g, 0.02, F, H), _normal(g, 0.02, F, H), _normal(g, 0.02, H, F)
        return state
    E, k = case["experts"], case["top_k"]
    # what a program keeps of its model's configuration
    state["shape"] = SimpleNamespace(d_model=128, d_ff=128, num_experts=E, top_k=k)
    state["gate"] = SimpleNamespace(score=case["score"], num_groups=1, top_groups=1, group_score="max", renormalise=case.get("renormalise", False),
                                    scale=case.get("scale", 1.0))
    z = _normal(g, 1.0, T, E, dtype=torch.float32) + _normal(g, 0.5, E, dtype=torch.float32)
    if case["off"]:
        z[torch.rand(T, E, generator=g, device="cuda") < case["off"]] = -math.inf
    state["logits"] = z.to(getattr(torch, case["dtype"]))
    state["ids"] = torch.sort(state["logits"].float(), dim=1, descending=True, stable=True).indices[:, :k].int().contiguous()
    state["offsets"], state["mask"] = _sequences(g, case)
    if kind == "backward":
        state["counts"], state["kept"], _, _ = _counts(state["ids"], state["offsets"], state["mask"], E)
        state["d_weights"] = _normal(g, 1.0, T, k, dtype=torch.float32) if case["weights"] else None
        state["d_losses"] = torch.tensor([0.01, 0.001], device="cuda") * (0.5 + torch.rand(2, generator=g, device="cuda")) if case["losses"] else None
    return state


def _run_own(state):
    from paper_2608_15383_b200 import binding
    case = state["case"]
    kind = case["kind"]
    if kind == "linear":
        return binding.exmoe_linear(state["x"], state["w"], state["bias"], w_up=state["w_up"], bias_up=state["bias_up"], activation=case["activation"],
                                    residual=state["residual"], out_dtype=getattr(torch, case["dtype"]))
    if kind == "shared":
        act = binding.exmoe_linear(state["x"], state["w"], w_up=state["w_up"], activation="silu")
        return [act, binding.exmoe_linear(act, state["w_down"], residual=state["routed"])]
    if kind == "loss":
        return binding.exmoe_balance_loss(state["shape"], state["gate"], state["logits"], state["ids"], mask=state["mask"], offsets=state["offsets"])
    return binding.exmoe_gate_backward(state["shape"], state["gate"], state["logits"], state["ids"], d_weights=state["d_weights"], d_losses=state["d_losses"],
                                       counts=state["counts"] if case["losses"] else None, kept=state["kept"] if case["losses"] else None,
                                       mask=state["mask"], offsets=state["offsets"] if case["losses"] else None)


def _activate(v, activation):
    if activation == "relu":
        return v.clamp(min=0)
    if activation == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if activation == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if activation == "silu":
        return v / (1 + torch.exp(-v))
    return v


def _product(x, w, bias, w_up, bias_up, activation, residual, dtype):
    v = x.float() @ w.float().t()
    if bias is not None:
        v = v + bias
    v = _activate(v, activation)
    if w_up is not None:
        u = x.float() @ w_up.float().t()
        v = v * (u if bias_up is None else u + bias_up)
    return (v if residual is None else residual.float() + v).to(dtype)


def _softmax(z):
    """Probabilities and the logarithm of the sum: zeros and 0 where no expert is left."""
    top = z.amax(1, keepdim=True)
    none = top == -math.inf
    top = torch.where(none, 0, top)
    e = torch.exp(z - top)
    s = e.sum(1, keepdim=True)
    return e / torch.where(none, 1, s), torch.where(none, 0, top + torch.log(torch.where(none, 1, s)))


def _normalised(s):
    t = s.sum(1, keepdim=True)
    return s / torch.where(t > 0, t, 1), torch.where(t > 0, t, 1)


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    kind = case["kind"]
    if kind == "linear":
        return _product(state["x"], state["w"], state["bias"], state["w_up"], state["bias_up"], case["activation"], state["residual"], getattr(torch, case["dtype"]))
    if kind == "shared":
        act = _product(state["x"], state["w"], None, state["w_up"], None, "silu", None, torch.bfloat16)
        return [act, _product(act, state["w_down"], None, None, None, "none", state["routed"], torch.bfloat16)]
    E, k = case["experts"], case["top_k"]
    z, ids, offsets, mask = state["logits"].float(), state["ids"].long(), state["offsets"], state["mask"]
    p, lse = _softmax(z)
    sigmoid = case["score"] == "sigmoid"
    s = 1 / (1 + torch.exp(-z)) if sigmoid else p
    q, total = _normalised(s) if sigmoid else (p, None)
    if kind == "loss":
        counts, kept, of, keep = _counts(ids, offsets, mask, E)
        S = len(kept)
        if S == 1:
            sums = (q * keep[:, None]).sum(0, keepdim=True)
        else:
            sums = torch.zeros(S, E, device=z.device).index_add_(0, of, q * keep[:, None])
        n = kept.double()
        per = E / (k * n.clamp(min=1) ** 2) * (counts.double() * sums.double()).sum(1)
        balance = per.sum() / (kept > 0).sum().clamp(min=1)
        z_loss = (lse.double().squeeze(1) ** 2 * keep).sum() / n.sum().clamp(min=1)
        return torch.stack([balance, z_loss]).float(), counts, sums.float(), kept
    dz = torch.zeros_like(z)
    _, _, of, keep = _counts(ids, offsets, mask, E)
    if case["losses"]:
        counts, kept = state["counts"].double(), state["kept"].double()
        factor = state["d_losses"][0] * E / (k * (kept > 0).sum().clamp(min=1) * kept.clamp(min=1) ** 2)
        G = (factor[:, None] * counts).float()[of] * keep[:, None]
        G = G - (q * G).sum(1, keepdim=True)
        dz = s * (1 - s) * G / total if sigmoid else q * G
        dz = dz + (2 * state["d_losses"][1] / kept.sum().clamp(min=1)).float() * lse * p * keep[:, None]
    if case["weights"]:
        chosen = s.gather(1, ids)
        d = state["d_weights"] * case["scale"] * keep[:, None]
        if case["renormalise"]:
            w, t = _normalised(chosen)
            d = (d - (w * d).sum(1, keepdim=True)) / t
        ds = torch.zeros_like(z).scatter_add_(1, ids, d)
        dz = dz + (s * (1 - s) * ds if sigmoid else s * (ds - (s * ds).sum(1, keepdim=True)))
    return dz.to(state["logits"].dtype)


def work(case):
    T = case["tokens"]
    if case["kind"] == "linear":
        K, N, es, two = case["k"], case["n"], 4 if case["dtype"] == "float32" else 2, 2 if case["gated"] else 1
        return {"bytes": T * K * 2 + two * N * (K * 2 + (4 if case["bias"] else 0)) + T * N * es * (2 if case["residual"] else 1), "flops": 2 * two * T * K * N}
    if case["kind"] == "shared":
        H, F = case["d_model"], case["d_ff"]
        return {"bytes": 2 * (3 * H * F + 3 * T * H + T * F), "flops": 6 * T * H * F}
    E, k, S, es = case["experts"], case["top_k"], max(1, min(case["sequences"], T)), 4 if case["dtype"] == "float32" else 2
    read = T * (E * es + 4 * k + (1 if case["masked"] else 0))
    if case["kind"] == "loss":
        return {"bytes": read + S * (8 * E + 4), "flops": 8 * T * E}
    return {"bytes": read + T * E * es + (4 * T * k if case["weights"] else 0) + (S * (4 * E + 4) if case["losses"] else 0), "flops": 12 * T * E}


def _numpy(t):
    return t.double().cpu().numpy()


def _exact_product(x, w, activation, w_up=None, bias=None, bias_up=None, residual=None):
    def product(m, b):
        v = torch.matmul(m.double(), x.double().t())                       # outputs x tokens
        return (v if b is None else v + b.double()[:, None]).t()
    v = product(w, bias)
    v = {"none": lambda a: a, "relu": torch.relu, "silu": lambda a: a * torch.sigmoid(a), "gelu": lambda a: a * torch.special.ndtr(a),
         "gelu_tanh": lambda a: a * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3))}[activation](v)
    if w_up is not None:
        v = v * product(w_up, bias_up)
    return v if residual is None else v + residual.double()


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "linear":
        return _exact_product(state["x"], state["w"], case["activation"], state["w_up"], state["bias"], state["bias_up"], state["residual"]).cpu().numpy()
    if case["kind"] == "shared":
        act = _exact_product(state["x"], state["w"], "silu", state["w_up"])
        down = _exact_product(act.to(torch.bfloat16), state["w_down"], "none", residual=state["routed"])    # from what the first product stores
        return [act.cpu().numpy(), down.cpu().numpy()]
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    z, ids = _numpy(state["logits"]), state["ids"].cpu().numpy()
    keep = np.ones(T, bool) if state["mask"] is None else state["mask"].cpu().numpy()
    offsets = [0, T] if state["offsets"] is None else state["offsets"].cpu().tolist()
    bounds = list(zip(offsets[:-1], offsets[1:]))
    left = ~np.isneginf(z).all(1)
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        lse = np.where(left, np.logaddexp.reduce(z, axis=1), 0.0)
        p = np.where(left[:, None], np.exp(z - lse[:, None]), 0.0)
        s = 1 / (1 + np.exp(-z)) if case["score"] == "sigmoid" else p
        total = np.where(left, s.sum(1), 1.0)[:, None]
    q = s / total
    if case["kind"] == "loss":
        counts, sums, kept = np.zeros((len(bounds), E), np.int32), np.zeros((len(bounds), E)), np.zeros(len(bounds), np.int32)
        for i, (a, b) in enumerate(bounds):
            rows = np.arange(a, b)[keep[a:b]]
            counts[i], sums[i], kept[i] = np.bincount(ids[rows].ravel(), minlength=E), q[rows].sum(0), len(rows)
        some = kept > 0
        n = kept[some].astype(float)
        balance = np.mean(E / k * (counts[some] / n[:, None] * (sums[some] / n[:, None])).sum(1)) if some.any() else 0.0
        return [np.array([balance, np.mean(lse[keep] ** 2) if keep.any() else 0.0]), counts, sums, kept]
    ds = np.zeros((T, E))                                                  # gradient on the scores
    direct = np.zeros((T, E))
    if case["losses"]:
        counts, kept, d = _numpy(state["counts"]), _numpy(state["kept"]), _numpy(state["d_losses"])
        for i, (a, b) in enumerate(bounds):
            if kept[i]:
                f = counts[i] / kept[i] * (E / k) / kept[i] * d[0] / (kept > 0).sum()
                rows = np.arange(a, b)[keep[a:b]]
                ds[rows] = (f - q[rows] @ f[:, None]) / total[rows]
        direct[keep] = d[1] * 2 * lse[keep, None] * p[keep] / max(kept.sum(), 1)
    if case["weights"]:
        d = np.where(keep[:, None], _numpy(state["d_weights"]) * case["scale"], 0.0)
        if case["renormalise"]:
            c = np.take_along_axis(s, ids, 1)
            t = c.sum(1, keepdims=True)
            t = np.where(t > 0, t, 1.0)
            d = (d - (d * c / t).sum(1, keepdims=True)) / t
        np.add.at(ds, (np.arange(T)[:, None], ids), d)
    return (s * (1 - s) * ds if case["score"] == "sigmoid" else s * (ds - (s * ds).sum(1, keepdims=True))) + direct
