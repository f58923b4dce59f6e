"""The gate and the low-rank adapters of a sparse block: the calls a serving program makes, and the same in elementary torch.

Four kinds of cases:

  gate     `exmoe_route_gated`: hidden states to expert ids and mixture weights, by softmax or sigmoid scores, with a balance
           bias that enters the choice only, groups of experts, renormalised weights.
  logits   `exmoe_gate_logits`: the same choice from logits that another program's router has computed, FP32 or BF16.
  lora     `exmoe_lora_plan` and, per layer, `exmoe_lora`: the adapters of a batch's requests beside a projection that all
           requests share; the plan is made once per step and serves all its layers.
  adapted  both together: adapters beside the router's projection (FP32), then the choice.

Hidden states N(0, 1), router, adapter weights N(0, 0.02), as the layer's synthetic inputs; balance biases N(0, 0.05).
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False


def _gate(tokens, d_model, experts, top_k, score="softmax", groups=1, top_groups=1, group_score="max", renormalise=True, scale=1.0,
          balance=False, kind="gate", **more):
    return dict(kind=kind, tokens=tokens, d_model=d_model, experts=experts, top_k=top_k, score=score, groups=groups, top_groups=top_groups,
                group_score=group_score, renormalise=renormalise, scale=scale, balance=balance, **more)


def _logits(tokens, experts, top_k, dtype="float32", masked=0.0, **more):
    return _gate(tokens, 0, experts, top_k, kind="logits", dtype=dtype, masked=masked, **more)


def _lora(tokens, requests, adapters, rank, k, n, layers=1, dtype="bfloat16", base=True, stride=0):
    return dict(kind="lora", tokens=tokens, requests=requests, adapters=adapters, rank=rank, k=k, n=n, layers=layers, dtype=dtype, base=base,
                stride=stride)


def listed():
    return [
        # one user's token through the router of the 64-expert top-8 model, weights renormalised
        dict(_gate(1, 2048, 64, 8), name="gate_1"),
        # a decode batch of odd size: sigmoid gate, balance bias, 4 of 8 groups by their two best experts
        dict(_gate(37, 2048, 128, 8, score="sigmoid", groups=8, top_groups=4, group_score="top2", scale=2.5, balance=True), name="gate_37"),
        # a short prompt of odd length through a router of 60 experts in 4 groups
        dict(_gate(333, 2048, 60, 4, groups=4, top_groups=2), name="gate_333"),
        # a batch of prompts through a wide sigmoid gate with a balance bias and groups
        dict(_gate(8192, 4096, 256, 8, score="sigmoid", groups=8, top_groups=4, group_score="top2", scale=2.5, balance=True), name="gate_8192"),
        # logits of a decode batch from a router that runs elsewhere
        dict(_logits(16, 64, 8), name="logits_16"),
        # BF16 logits of a prompt of odd length: many exact ties, some experts switched off
        dict(_logits(8191, 256, 8, dtype="bfloat16", masked=0.02, groups=8, top_groups=3), name="logits_8191"),
        # one request's adapter beside a 2048 x 2048 projection of each of 16 layers
        dict(_lora(1, 1, 8, 16, 2048, 2048, layers=16), name="lora_1"),
        # 64 requests with 32 adapters (and some with none), one token each, 8 layers
        dict(_lora(64, 64, 32, 16, 2048, 2048, layers=8), name="lora_64"),
        # prompts of three requests of odd lengths, d_ff 1408 to d_model 2048, a larger rank; x is a column range of wider rows
        dict(_lora(777, 3, 4, 64, 1408, 2048, stride=2816), name="lora_777"),
        # a full prefill batch of a dozen requests
        dict(_lora(8192, 12, 16, 16, 2048, 2048), name="lora_8192"),
        # FP32 corrections of 60 router logits by adapters, nothing to add them to yet
        dict(_lora(250, 40, 20, 8, 2048, 60, dtype="float32", base=False), name="lora_logits_250"),
        # a decode batch whose adapters reach the router too: corrections of its logits, then the choice
        dict(_gate(48, 2048, 64, 8, kind="adapted", requests=48, adapters=16, rank=16), name="adapted_48"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_gate(rng, most_experts):
    groups = rng.choice((1, 1, 2, 4, 8))
    experts = groups * _log_int(rng, max(2, 8 // groups), most_experts // groups)
    top_groups = rng.randint(1, groups)
    top_k = rng.randint(1, min(16, top_groups * (experts // groups)))
    score = rng.choice(("softmax", "sigmoid"))
    return experts, top_k, dict(score=score, groups=groups, top_groups=top_groups, group_score=rng.choice(("max", "top2")),
                                renormalise=rng.random() < 0.6, scale=rng.choice((1.0, 2.5)), balance=rng.random() < 0.5)


def draw(rng):
    kind = rng.choice(("gate", "gate", "logits", "lora", "lora", "lora", "adapted"))
    if kind == "gate":
        experts, top_k, more = _draw_gate(rng, 256)
        return _gate(_log_int(rng, 1, 8192), rng.choice((64 * rng.randint(4, 64), 8 * rng.randint(32, 512))), experts, top_k, **more)
    if kind == "logits":
        experts, top_k, more = _draw_gate(rng, 512)
        return _logits(_log_int(rng, 1, 16384), experts, top_k, dtype=rng.choice(("float32", "bfloat16")), masked=rng.choice((0.0, 0.02, 0.3)), **more)
    if kind == "adapted":
        experts, top_k, more = _draw_gate(rng, 128)
        tokens = _log_int(rng, 1, 64)
        return _gate(tokens, 64 * rng.randint(4, 32), experts, top_k, kind="adapted", requests=rng.randint(1, tokens), adapters=_log_int(rng, 1, 32),
                     rank=8 * rng.randint(1, 4), **more)
    tokens, rank = _log_int(rng, 1, 8192), rng.choice((8, 16, 16, 32, 64))
    k, n = 8 * _log_int(rng, 32, 512), rng.choice((8 * _log_int(rng, 32, 512), _log_int(rng, 8, 4096)))
    while tokens * (3 * (k + n) + 2 * rank * (k + n) / 50) > 8192 * 3 * 4096:
        tokens //= 2
    k_and_stride = rng.choice((0, 2 * k))
    return _lora(tokens, _log_int(rng, 1, tokens), _log_int(rng, 1, 64), rank, k, n, layers=rng.randint(1, 4) if tokens < 200 else 1,
                 dtype=rng.choice(("bfloat16", "bfloat16", "float32")), base=rng.random() < 0.75, stride=k_and_stride)


def _normal(g, std, *size, dtype=torch.bfloat16):
    return (torch.randn(*size, generator=g, device="cuda") * std).to(dtype)


def _adapter_ids(g, case):
    """Requests of uneven lengths side by side, an adapter (or, for one request in ten, none) for each: int32 [tokens]."""
    T, R = case["tokens"], min(case["requests"], case["tokens"])
    lengths = torch.rand(R, generator=g, device="cuda") + 0.1
    ends = torch.floor(torch.cumsum(lengths, 0) / lengths.sum() * (T - R) + 0.5).long() + torch.arange(1, R + 1, device="cuda")
    request = torch.searchsorted(ends[:-1].contiguous(), torch.arange(T, device="cuda"), right=True)
    of_request = torch.randint(0, case["adapters"], (R,), generator=g, device="cuda")
    if R > 1:
        of_request[torch.rand(R, generator=g, device="cuda") < 0.1] = -1
    return of_request[request].int()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    T, kind, state = case["tokens"], case["kind"], {"case": case}
    if kind == "lora":
        K, N, r, n = case["k"], case["n"], case["rank"], case["adapters"]
        dtype = getattr(torch, case["dtype"])
        state["ids"] = _adapter_ids(g, case)
        state["scale"] = torch.rand(n, generator=g, device="cuda") + 1.0
        state["layers"] = []
        for _ in range(case["layers"]):
            x = _normal(g, 1.0, T, case["stride"] or K)[:, :K]
            state["layers"].append((x, _normal(g, 0.02, n, r, K), _normal(g, 0.02, n, N, r), _normal(g, 1.0, T, N, dtype=dtype) if case["base"] else None))
        return state
    E = case["experts"]
    # what a program keeps of its model's configuration
    state["shape"] = SimpleNamespace(d_model=case["d_model"] or 128, d_ff=128, num_experts=E, top_k=case["top_k"])
    state["gate"] = SimpleNamespace(score=case["score"], num_groups=case["groups"], top_groups=case["top_groups"], group_score=case["group_score"],
                                    renormalise=case["renormalise"], scale=case["scale"])
    state["balance"] = _normal(g, 0.05, E, dtype=torch.float32) if case["balance"] else None
    if kind == "logits":
        z = _normal(g, 1.0, T, E, dtype=torch.float32)
        if case["masked"]:
            z[:, torch.rand(E, generator=g, device="cuda") < case["masked"]] = -math.inf
        state["logits"] = z.to(getattr(torch, case["dtype"]))
        return state
    H = case["d_model"]
    state["hidden"], state["router"] = _normal(g, 1.0, T, H), _normal(g, 0.02, E, H)
    if kind == "adapted":
        n, r = case["adapters"], case["rank"]
        state["ids"] = _adapter_ids(g, case)
        state["scale"] = torch.rand(n, generator=g, device="cuda") + 1.0
        state["a"], state["b"] = _normal(g, 0.02, n, r, H), _normal(g, 0.02, n, E, r)
    return state


def _run_own(state):
    from paper_2608_15383_b200 import binding
    case = state["case"]
    kind, addend = case["kind"], None
    if kind == "lora":
        plan = binding.exmoe_lora_plan(state["ids"], case["adapters"])
        return [binding.exmoe_lora(plan, x, a, b, state["scale"], base=base, out_dtype=getattr(torch, case["dtype"])) for x, a, b, base in state["layers"]]
    if kind == "logits":
        return binding.exmoe_gate_logits(state["shape"], state["gate"], state["logits"], balance=state["balance"])
    if kind == "adapted":
        plan = binding.exmoe_lora_plan(state["ids"], case["adapters"])
        addend = binding.exmoe_lora(plan, state["hidden"], state["a"], state["b"], state["scale"], out_dtype=torch.float32)
    return binding.exmoe_route_gated(state["shape"], state["gate"], state["hidden"], state["router"], addend=addend, balance=state["balance"])


def _choose(z, case, balance):
    """Ids and weights from logits in 64 bits.  Without a balance bias scores are ordered as their logits are."""
    T, E = z.shape
    G, k = case["groups"], case["top_k"]
    low = torch.full_like(z[:, :1], -math.inf)
    off = z == low
    if case["score"] == "sigmoid":
        s = 1 / (1 + torch.exp(-z))
    else:
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - torch.where(top == low, 0, top))
        s = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    scored = torch.where(off, low, s if balance is None else s + balance.double())
    by = z if balance is None else scored
    order = torch.argsort(by, dim=1, descending=True, stable=True)
    if case["top_groups"] < G:
        if case["group_score"] == "max":
            of_group = by.view(T, G, -1).amax(2)
        else:
            best = scored.view(T, G, -1).topk(min(2, E // G), 2).values
            of_group = best[..., 0] + (torch.where(best[..., 1:] == -math.inf, 0, best[..., 1:])).sum(2)
        kept = torch.zeros_like(of_group, dtype=torch.int32)
        kept.scatter_(1, torch.argsort(of_group, dim=1, descending=True, stable=True)[:, :case["top_groups"]], 1)
        kept = kept.repeat_interleave(E // G, 1).gather(1, order)
        order = order.gather(1, torch.argsort(kept, dim=1, descending=True, stable=True))
    ids = order[:, :k]
    w = s.gather(1, ids)
    if case["renormalise"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return ids.int(), (w * case["scale"]).float()


def _adapter_product(x, a, b, scale, ids, dtype):
    """scale_a * B_a (A_a x) of every token, zero where it has no adapter: float or double [tokens, n]."""
    at = ids.long().clamp(min=0)
    v = torch.bmm(a[at].to(dtype), x.to(dtype).unsqueeze(2))
    return torch.bmm(b[at].to(dtype), v).squeeze(2) * torch.where(ids < 0, 0.0, scale[at]).to(dtype).unsqueeze(1)


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    kind = case["kind"]
    if kind == "lora":
        dtype = getattr(torch, case["dtype"])
        outs = []
        for x, a, b, base in state["layers"]:
            d = _adapter_product(x, a, b, state["scale"], state["ids"], torch.float32)
            outs.append((d if base is None else base.float() + d).to(dtype))
        return outs
    if kind == "logits":
        return _choose(state["logits"].double(), case, state["balance"])
    z = state["hidden"].double() @ state["router"].double().t()
    if kind == "adapted":
        z = z + _adapter_product(state["hidden"], state["a"], state["b"], state["scale"], state["ids"], torch.float64)
    return _choose(z, case, state["balance"])


def work(case):
    T = case["tokens"]
    if case["kind"] == "lora":
        used = min(case["adapters"], case["requests"], T)
        K, N, r, es = case["k"], case["n"], case["rank"], 4 if case["dtype"] == "float32" else 2
        per = T * K * 2 + T * N * es * (2 if case["base"] else 1) + used * r * (K + N) * 2
        return {"bytes": 4 * T + case["layers"] * per, "flops": case["layers"] * 2 * T * r * (K + N)}
    E, k, H = case["experts"], case["top_k"], case["d_model"]
    out = T * k * 8 + (4 * E if case["balance"] else 0)
    if case["kind"] == "logits":
        return {"bytes": T * E * (4 if case["dtype"] == "float32" else 2) + out, "flops": 4 * T * E}
    w = {"bytes": T * H * 2 + E * H * 2 + out, "flops": 2 * T * H * E}
    if case["kind"] == "adapted":
        used = min(case["adapters"], case["requests"], T)
        w["bytes"] += used * case["rank"] * (H + E) * 2 + 4 * T
        w["flops"] += 2 * T * case["rank"] * (H + E)
    return w


def _exact_choice(z, case, balance):
    """The definition, in numpy: scores, kept groups, then experts ordered by (kept, score, -id)."""
    T, E = z.shape
    G, k = case["groups"], case["top_k"]
    size = E // G
    off = np.isneginf(z)
    with np.errstate(over="ignore"):
        if case["score"] == "sigmoid":
            s = 1.0 / (1.0 + np.exp(-z))
        else:
            e = np.exp(z - np.where(off.all(1), 0.0, z.max(1))[:, None])
            s = e / np.maximum(e.sum(1), 1e-300)[:, None]
    c = np.where(off, -np.inf, s + (0.0 if balance is None else balance))
    key = z if balance is None else c
    lowest_first = np.broadcast_to(np.arange(E), z.shape)
    kept = np.ones_like(z)
    if case["top_groups"] < G:
        in_order = np.sort(c.reshape(T, G, size), axis=2)[:, :, ::-1]
        value = key.reshape(T, G, size).max(2)
        if case["group_score"] == "top2":
            value = in_order[:, :, 0] + (np.where(np.isneginf(in_order[:, :, 1]), 0.0, in_order[:, :, 1]) if size > 1 else 0.0)
        by_value = np.lexsort((np.broadcast_to(np.arange(G), value.shape), -value), axis=1)
        rank = np.argsort(by_value, axis=1)
        kept = np.repeat((rank < case["top_groups"]).astype(float), size, axis=1)
    ids = np.lexsort((lowest_first, -key, -kept), axis=1)[:, :k]
    w = np.take_along_axis(s, ids, 1)
    if case["renormalise"]:
        w = w / np.maximum(w.sum(1), 1e-300)[:, None]
    return ids.astype(np.int32), w * case["scale"]


def _numpy(t):
    return t.double().cpu().numpy()


def _exact_adapters(x, a, b, scale, ids):
    d = np.zeros((x.shape[0], b.shape[1]))
    for i in sorted(set(ids.tolist()) - {-1}):
        rows = ids == i
        d[rows] = (_numpy(x)[rows] @ _numpy(a[i]).T) @ _numpy(b[i]).T * float(scale[i])
    return d


def exact(case, seed):
    state = prepare(case, seed)
    balance = _numpy(state["balance"]) if state.get("balance") is not None else None
    ids = state["ids"].cpu().numpy() if "ids" in state else None
    if case["kind"] == "lora":
        return [_exact_adapters(x, a, b, state["scale"], ids) + (0.0 if base is None else _numpy(base)) for x, a, b, base in state["layers"]]
    if case["kind"] == "logits":
        return _exact_choice(_numpy(state["logits"]), case, balance)
    z = _numpy(state["hidden"]) @ _numpy(state["router"]).T
    if case["kind"] == "adapted":
        z = z + _exact_adapters(state["hidden"], state["a"], state["b"], state["scale"], ids)
    return _exact_choice(z, case, balance)
