"""Operators of a decode layer's feed-forward half, and the calls they are measured by.

  route   tokens to experts: scores, bias for balance, groups, top-k, weights   nm_moe_route
  moe     the chosen experts' gated products and their weighted sum             nm_moe_ffn
  act     product with bias, activation, gate and residual in its epilogue      nm_matmul_act

route  s = softmax(x) or sigmoid(x) over the E logits of a token, key = s + bias.  With groups of E / G experts: a group counts as its
       best key (or its two best added), the `keep` best groups stay.  The k largest keys, ties to the lowest index, in falling order;
       weight = s, divided by the chosen ones' sum where renormalised, times a scale.
moe    y[t] = residual[t] + sum_j w[t, j] * (act(x[t] Wg) o (x[t] Wu)) Wd, the weights those of expert experts[t, j]; an index outside
       the experts held here adds nothing.  Weights: up [E][d][2 inter] (gate | up) and down [E][inter][d] (layout 0), or transposed per
       expert (layout 1).  Without a gate: act(x Wu) Wd, up [E][d][inter].
act    C = act(A B + bias) + residual, or with a gate: B = (gate | up), C = act(A Bg + bg) o (A Bu + bu) + residual.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one token of a small model, its logits in fp32 as a narrow product leaves them: latency alone
        {"name": "route 1 token, 64 experts", "op": "route", "T": 1, "E": 64, "k": 6, "dtype": "f32", "score": "softmax", "bias": False, "groups": 1, "keep": 1, "best": 1,
         "renorm": True},
        # a full narrow batch, scores balanced by a bias, groups
        {"name": "route 16 tokens, 160 experts in groups", "op": "route", "T": 16, "E": 160, "k": 6, "dtype": "f32", "score": "sigmoid", "bias": True, "groups": 8, "keep": 3,
         "best": 2, "renorm": True},
        # a prompt's tokens, an odd number of experts, logits in 16 bits
        {"name": "route 1003 tokens, 97 experts", "op": "route", "T": 1003, "E": 97, "k": 4, "dtype": "bf16", "score": "softmax", "bias": False, "groups": 1, "keep": 1, "best": 1,
         "renorm": False},
        # a long prompt and many experts
        {"name": "route 8192 tokens, 320 experts in groups", "op": "route", "T": 8192, "E": 320, "k": 8, "dtype": "f32", "score": "sigmoid", "bias": True, "groups": 10,
         "keep": 4, "best": 2, "renorm": True},
        # one token of a decode step: every chosen expert's weights for a single row
        {"name": "moe 1 token, 6 of 64, 7168x1536", "op": "moe", "T": 1, "E": 64, "k": 6, "d": 7168, "inter": 1536, "act": "silu", "gated": True, "dtype": "bf16", "layout": 1,
         "residual": True},
        # a full narrow batch: nearly every expert, two rows each
        {"name": "moe 16 tokens, 6 of 64, 7168x1536", "op": "moe", "T": 16, "E": 64, "k": 6, "d": 7168, "inter": 1536, "act": "silu", "gated": True, "dtype": "bf16", "layout": 0,
         "residual": True},
        # small experts with ragged sizes, fp16
        {"name": "moe 67 tokens, 3 of 24, 2048x1000", "op": "moe", "T": 67, "E": 24, "k": 3, "d": 2048, "inter": 1000, "act": "gelu", "gated": True, "dtype": "f16", "layout": 1,
         "residual": False},
        # a chunk of a prompt: about a hundred rows an expert
        {"name": "moe 1024 tokens, 6 of 64, 7168x1536", "op": "moe", "T": 1024, "E": 64, "k": 6, "d": 7168, "inter": 1536, "act": "silu", "gated": True, "dtype": "bf16",
         "layout": 1, "residual": True},
        # the smallest projection of the decode step with a bias, one token
        {"name": "act 1 token 7168x576, bias", "op": "act", "M": 1, "N": 576, "K": 7168, "act": "none", "gated": False, "bias": True, "residual": False, "dtype": "bf16", "layout": 0},
        # a dense layer's or shared expert's gate and up projection, one token
        {"name": "act 1 token 7168x18432, gated", "op": "act", "M": 1, "N": 18432, "K": 7168, "act": "silu", "gated": True, "bias": False, "residual": False, "dtype": "bf16",
         "layout": 1},
        # its way back onto the residual stream, a full narrow batch
        {"name": "act 16 tokens 18432x7168, residual", "op": "act", "M": 16, "N": 7168, "K": 18432, "act": "none", "gated": False, "bias": False, "residual": True, "dtype": "bf16",
         "layout": 0},
        # many tokens, a ragged edge, everything in the epilogue
        {"name": "act 100 tokens 1536x24569, bias, gelu, residual", "op": "act", "M": 100, "N": 24569, "K": 1536, "act": "gelu_tanh", "gated": False, "bias": True, "residual": True,
         "dtype": "f16", "layout": 1},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["route", "route", "moe", "moe", "moe", "act", "act", "act"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8, 10])
        E = max(2, groups) * _log(rng, 2, 512 // max(2, groups)) - (1 if groups == 1 else 0)
        keep = rng.randint(1, groups)
        k = rng.randint(1, min(12, keep * (E // groups)))
        return {"op": op, "T": _log(rng, 1, 8192), "E": E, "k": k, "dtype": rng.choice(["f32", "f32", "bf16", "f16"]), "score": rng.choice(["softmax", "sigmoid"]),
                "bias": rng.random() < 0.5, "groups": groups, "keep": keep, "best": rng.choice([1, 2]) if E // groups > 1 else 1, "renorm": rng.random() < 0.7}
    acts = ["silu", "silu", "gelu", "gelu_tanh", "relu"]
    if op == "moe":
        d, inter = 8 * _log(rng, 32, 896), 8 * _log(rng, 8, 256)
        E = min(_log(rng, 2, 200), 64 * 7168 * 1536 // (d * inter))
        k = rng.randint(1, min(8, E))
        T = min(_log(rng, 1, 1024), 1024 * 6 * 7168 * 1536 // (d * inter * k))
        return {"op": op, "T": T, "E": E, "k": k, "d": d, "inter": inter, "act": rng.choice(acts), "gated": rng.random() < 0.85, "dtype": rng.choice(["bf16", "bf16", "f16"]),
                "layout": rng.randint(0, 1), "residual": rng.random() < 0.5}
    gated, layout = rng.random() < 0.5, rng.randint(0, 1)
    K = 8 * _log(rng, 8, 2304)
    N = _log(rng, 16, min(24576, 18432 * 7168 // K))
    return {"op": op, "M": _log(rng, 1, 128), "N": N if layout else -(-N // 8) * 8, "K": K, "act": rng.choice(acts if gated else acts + ["none", "none"]), "gated": gated,
            "bias": rng.random() < 0.5, "residual": rng.random() < 0.5, "dtype": rng.choice(["bf16", "bf16", "f16"]), "layout": layout}


def work(case):
    if case["op"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": T * E * (4 if case["dtype"] == "f32" else 2) + 4 * E * case["bias"] + 8 * T * k, "flops": T * E * (5 + k)}
    parts = 3 if case["gated"] else 2
    if case["op"] == "moe":
        T, E, k, d, inter = (case[n] for n in ("T", "E", "k", "d", "inter"))
        used = E * (1 - (1 - k / E) ** T)  # experts that some token has chosen, as each is as likely as the others
        return {"bytes": used * parts * d * inter * 2 + 2 * T * d * (3 if case["residual"] else 2) + 8 * T * k, "flops": 2 * T * k * parts * d * inter}
    M, N, K, two = case["M"], case["N"], case["K"], 1 + case["gated"]
    return {"bytes": 2 * (two * N * K + M * K + M * N * (1 + case["residual"]) + two * N * case["bias"]), "flops": 2 * M * N * K * two}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s, t=torch.float32: torch.randn(*s, generator=g, device="cuda", dtype=t)  # noqa: E731
    s, t = dict(case), TYPES[case["dtype"]]
    if case["op"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        s["logits"] = randn(T, E).to(t)
        s["balance"] = 0.1 * randn(E) if case["bias"] else None
        s["experts"] = torch.empty(T, k, dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty(T, k, device="cuda")
        s["scale"] = 2.5 if case["renorm"] else 1.0
        return s
    if case["op"] == "moe":
        T, E, k, d, inter = (case[n] for n in ("T", "E", "k", "d", "inter"))
        wide = inter * (1 + case["gated"])
        s["x"] = randn(T, d).to(t)
        s["experts"] = torch.rand(T, E, generator=g, device="cuda").topk(k, 1).indices.to(torch.int32)
        s["weights"] = torch.softmax(randn(T, k), 1)
        s["up"] = randn(*((E, wide, d) if case["layout"] else (E, d, wide)), t=t).mul_(0.02)
        s["down"] = randn(*((E, d, inter) if case["layout"] else (E, inter, d)), t=t).mul_(0.02)
        s["skip"] = randn(T, d).to(t) if case["residual"] else None
        s["y"] = torch.empty(T, d, dtype=t, device="cuda")
        s["workspace"] = torch.zeros((96 << 20) + T * k * (4 * d + 8 * inter + 64), dtype=torch.uint8, device="cuda")  # kept by the program, cleared once
        return s
    M, N, K, two = case["M"], case["N"], case["K"], 1 + case["gated"]
    s["A"] = randn(M, K).to(t)
    s["B"] = randn(*((two * N, K) if case["layout"] else (K, two * N)), t=t).mul_(0.02)
    s["b"] = randn(two * N).to(t) if case["bias"] else None
    s["skip"] = randn(M, N).to(t) if case["residual"] else None
    s["C"] = torch.empty(M, N, dtype=t, device="cuda")
    s["workspace"] = torch.zeros(96 << 20, dtype=torch.uint8, device="cuda")
    return s


def _act(name, x):
    if name == "none":
        return x
    if name == "relu":
        return x.clamp(min=0)
    if name == "silu":
        return x / (1 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))


def _plain_route(s):
    # In 64 bits: two keys next to each other decide which expert is chosen.
    x = s["logits"].double()
    if s["score"] == "softmax":
        x = torch.exp(x - x.amax(1, keepdim=True))
        score = x / x.sum(1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-x))
    key = score if s["balance"] is None else score + s["balance"].double()
    if s["groups"] > 1:
        by_group = key.view(key.shape[0], s["groups"], -1)
        of_group = by_group.sort(dim=2, descending=True).values[:, :, :s["best"]].sum(2)
        order = of_group.sort(dim=1, descending=True, stable=True).indices[:, :s["keep"]]
        kept = torch.zeros_like(of_group, dtype=torch.bool).scatter_(1, order, True)
        key = by_group.masked_fill(~kept[:, :, None], -math.inf).view_as(key)
    chosen = key.sort(dim=1, descending=True, stable=True).indices[:, :s["k"]]
    w = score.gather(1, chosen)
    if s["renorm"]:
        w = w / w.sum(1, keepdim=True)
    s["experts"].copy_(chosen)
    s["weights"].copy_(w * s["scale"])
    return s["experts"], s["weights"]


def _plain_moe(s):
    # The rows of each expert that is used, padded to the longest, against its weights.
    T, k, inter = s["T"], s["k"], s["inter"]
    e = s["experts"].reshape(-1).long()
    used, which, count = torch.unique(e, return_inverse=True, return_counts=True)
    order = which.argsort(stable=True)
    place = torch.arange(T * k, device="cuda") - (count.cumsum(0) - count)[which[order]]
    rows = torch.zeros(len(used), int(count.max()), s["d"], device="cuda")
    rows[which[order], place] = s["x"].float()[order // k]
    up, down = s["up"][used].float(), s["down"][used].float()
    if s["layout"]:
        up, down = up.transpose(1, 2), down.transpose(1, 2)
    h = torch.bmm(rows, up)
    h = _act(s["act"], h[..., :inter]) * h[..., inter:] if s["gated"] else _act(s["act"], h)
    y = torch.empty(T * k, s["d"], device="cuda")
    y[order] = torch.bmm(h, down)[which[order], place]
    y = (y.view(T, k, -1) * s["weights"][:, :, None]).sum(1)
    s["y"].copy_(y if s["skip"] is None else y + s["skip"].float())
    return s["y"]


def _plain_act(s):
    N = s["N"]
    z = s["A"].float() @ (s["B"].float().T if s["layout"] else s["B"].float())
    if s["b"] is not None:
        z = z + s["b"].float()
    z = _act(s["act"], z[:, :N]) * z[:, N:] if s["gated"] else _act(s["act"], z)
    s["C"].copy_(z if s["skip"] is None else z + s["skip"].float())
    return s["C"]


def _dtype(nm, s):
    return {"bf16": nm.BF16, "f16": nm.F16, "f32": nm.F32}[s["dtype"]]


def run(s):
    if own:
        import paper_2609_16009_b200 as nm

        if s["op"] == "route":
            nm.nm_moe_route(s["logits"], s["balance"], s["experts"], s["weights"], s["T"], s["E"], s["k"], _dtype(nm, s),
                            nm.SCORE_SIGMOID if s["score"] == "sigmoid" else nm.SCORE_SOFTMAX, groups=s["groups"], keep_groups=s["keep"], group_best=s["best"],
                            renormalise=s["renorm"], scale=s["scale"])
            return s["experts"], s["weights"]
        act = {"none": nm.ACT_NONE, "relu": nm.ACT_RELU, "silu": nm.ACT_SILU, "gelu": nm.ACT_GELU, "gelu_tanh": nm.ACT_GELU_TANH}[s["act"]]
        if s["op"] == "moe":
            nm.nm_moe_ffn(s["x"], s["experts"], s["weights"], s["up"], s["down"], s["y"], s["T"], s["d"], s["inter"], s["E"], s["k"], act, _dtype(nm, s), s["layout"],
                          s["workspace"], gated=s["gated"], residual=s["skip"])
            return s["y"]
        nm.nm_matmul_act(s["A"], s["B"], s["C"], s["M"], s["N"], s["K"], act, _dtype(nm, s), s["layout"], s["workspace"], gated=s["gated"], bias=s["b"], residual=s["skip"])
        return s["C"]
    return {"route": _plain_route, "moe": _plain_moe, "act": _plain_act}[s["op"]](s)


# ---- the definitions in 64 bits, written apart from the plain forms -------------------------------------------------------

def _act64(name, x):
    if name == "none":
        return x
    if name == "relu":
        return torch.where(x > 0, x, 0.0)
    if name == "silu":
        return x * torch.special.expit(x)
    if name == "gelu":
        return x * torch.special.ndtr(x)
    return x * torch.special.expit(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "route":
        x = s["logits"].double()
        T, E, G = case["T"], case["E"], case["groups"]
        score = torch.softmax(x, 1) if case["score"] == "softmax" else torch.special.expit(x)
        key = score + (0 if s["balance"] is None else s["balance"].double())
        # one choice at a time: the largest that is left, the first of equals
        left = key.clone()
        if G > 1:
            of = torch.arange(E, device="cuda") // (E // G)
            total = torch.stack([key[:, of == i].topk(case["best"], 1).values.sum(1) for i in range(G)], 1)
            kept = torch.zeros(T, G, dtype=torch.bool, device="cuda")
            for _ in range(case["keep"]):
                top = total.masked_fill(kept, -math.inf)
                kept[torch.arange(T, device="cuda"), (top == top.amax(1, keepdim=True)).int().argmax(1)] = True
            left[~kept[:, of]] = -math.inf
        out = []
        for _ in range(case["k"]):
            at = (left == left.amax(1, keepdim=True)).int().argmax(1)
            out.append(at)
            left[torch.arange(T, device="cuda"), at] = -math.inf
        chosen = torch.stack(out, 1)
        w = torch.take_along_dim(score, chosen, 1)
        return chosen.int(), w * s["scale"] / (w.sum(1, keepdim=True) if case["renorm"] else 1)
    if case["op"] == "moe":
        y = torch.zeros(case["T"], case["d"], dtype=torch.float64, device="cuda") if s["skip"] is None else s["skip"].double()
        for e in torch.unique(s["experts"]).tolist():
            t, j = (s["experts"] == e).nonzero(as_tuple=True)
            up, down = s["up"][e].double(), s["down"][e].double()
            z = torch.einsum("td,nd->tn" if case["layout"] else "td,dn->tn", s["x"][t].double(), up)
            parts = z.split(case["inter"], 1)
            h = _act64(case["act"], parts[0]) * (parts[1] if case["gated"] else 1)
            y.index_add_(0, t, s["weights"][t, j].double()[:, None] * torch.einsum("ti,di->td" if case["layout"] else "ti,id->td", h, down))
        return y
    B = s["B"].double()
    z = torch.einsum("mk,nk->mn" if case["layout"] else "mk,kn->mn", s["A"].double(), B)
    if s["b"] is not None:
        z += s["b"].double()
    parts = z.split(case["N"], 1)
    z = _act64(case["act"], parts[0])
    if case["gated"]:
        z = z * parts[1]
    return z if s["skip"] is None else z + s["skip"].double()
