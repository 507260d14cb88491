"""Operators that run on the layouts the loader writes, for measuring: the matrix product with its
epilogue over a weight as loaded (`linear`), the choice of experts (`route`) and the experts' products
over the stacked w13 and w2 (`experts`).

A case names the operator and its sizes:

    linear    y = act(x W^T + b) + r;  gated: y = act(x G^T + b_g) * (x U^T + b_u) + r with G and U
              the first and the second half of W's rows (a fused gate_up weight)
              t tokens, n rows of W (gated: two halves), k columns; act none, relu, gelu, gelu_tanh or
              silu; out "same" (x's type) or "f32"
    route     the top_k of e experts per token with their weights, from the logits: softmax or sigmoid
              scores, optionally a bias that counts for the choice alone, groups of which some are kept
              (by their best logit with softmax, by the sum of their two best scores with sigmoid),
              renormalised weights, a scale
    experts   y = sum over a token's chosen experts of weight * (silu(x G^T) * (x U^T)) D^T for e
              stacked experts [G; U] = w13 [e, 2 i, h] and D = w2 [e, h, i]; all_e experts in the
              model, of which this GPU holds e from `first` on (a choice held elsewhere adds nothing)

Sizes are those of the benchmark's decoders (hidden 4096 and 14336 wide or 8192 and 28672 wide; 8 experts
of 14336, two per token) and generic ones (128 experts of 768 at hidden 2048, eight per token).
"""
import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def linear(t, n, k, dtype="bf16", act="none", gated=False, bias=False, residual=False, out="same"):
    return {"op": "linear", "t": t, "n": n, "k": k, "dtype": dtype, "act": act, "gated": gated,
            "bias": bias, "residual": residual, "out": out}


def route(t, e, top_k, dtype="bf16", scoring="softmax", bias=False, groups=1, top_groups=1,
          renormalize=True, scale=1.0):
    return {"op": "route", "t": t, "e": e, "top_k": top_k, "dtype": dtype, "scoring": scoring,
            "bias": bias, "groups": groups, "top_groups": top_groups, "renormalize": renormalize,
            "scale": scale}


def experts(t, h, i, e, top_k, all_e=None, first=0, dtype="bf16", residual=False):
    return {"op": "experts", "t": t, "h": h, "i": i, "e": e, "top_k": top_k, "all_e": all_e or e,
            "first": first, "dtype": dtype, "residual": residual}


def listed():
    return [
        # one decoded token's choice of two among eight experts: latency alone
        dict(route(1, 8, 2), name="route_token"),
        # a prompt's choice of eight among 256 experts in groups, with a balance bias
        dict(route(4099, 256, 8, "f32", "sigmoid", True, 8, 4, True, 2.5), name="route_prompt"),
        # the router's logits for a batch of 64 sequences, one token each
        dict(linear(64, 8, 4096, out="f32"), name="linear_router"),
        # one decoded token through the fused q/k/v projection
        dict(linear(1, 6144, 4096), name="linear_qkv_token"),
        # 17 sequences, one token each, through the down projection, added to the residual stream
        dict(linear(17, 4096, 14336, residual=True), name="linear_down_17"),
        # an odd-sized fp16 layer with bias and GELU, its rows off the 16-byte grid
        dict(linear(777, 1003, 1100, "f16", "gelu", bias=True), name="linear_f16_odd"),
        # a prompt of 4096 tokens through the fused gate/up projection
        dict(linear(4096, 28672, 4096, act="silu", gated=True), name="linear_gate_up_4096"),
        # the widest projection: the larger decoder's gate/up on a prompt of 3000 tokens
        dict(linear(3000, 57344, 8192, act="silu", gated=True), name="linear_gate_up_wide"),
        # one decoded token through two of eight experts
        dict(experts(1, 4096, 14336, 8, 2), name="experts_token"),
        # a decoding batch of 64 sequences: every expert is read, few tokens each
        dict(experts(64, 4096, 14336, 8, 2, residual=True), name="experts_batch"),
        # a prompt of 4096 tokens
        dict(experts(4096, 4096, 14336, 8, 2), name="experts_prompt"),
        # a rank of four with 32 of 128 small experts, 512 tokens, eight choices each
        dict(experts(512, 2048, 768, 32, 8, 128, 32, "f16"), name="experts_rank"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("linear", "linear", "route", "experts", "experts"))
    if op == "route":
        groups = rng.choice((1, 1, 4, 8))
        e = rng.choice((8, 16, 60, 64, 128, 160, 256)) if groups == 1 else rng.choice((64, 128, 256))
        sigmoid = rng.random() < 0.5
        return route(_log(rng, 1, 16384), e, rng.randint(1, 8), rng.choice(("bf16", "f16", "f32")),
                     "sigmoid" if sigmoid else "softmax", sigmoid and rng.random() < 0.7, groups,
                     max(1, groups // 2), rng.random() < 0.7, rng.choice((1.0, 2.5)))
    if op == "linear":
        t = _log(rng, 1, 4096)
        gated = rng.random() < 0.35
        n = _log(rng, 64, 12288)
        k = _log(rng, 256, 14336)
        if rng.random() < 0.8:  # rows on the 16-byte grid, as nearly every model's are
            k = (k + 7) // 8 * 8
        if rng.random() < 0.5:
            n = (n + 127) // 128 * 128
        act = rng.choice(("silu", "gelu_tanh")) if gated else rng.choice(
            ("none", "none", "relu", "gelu", "gelu_tanh", "silu"))
        return linear(t, 2 * n if gated else n, k, rng.choice(("bf16", "bf16", "f16")), act, gated,
                      rng.random() < 0.4, rng.random() < 0.4, "f32" if rng.random() < 0.2 else "same")
    h = rng.choice((1024, 2048, 2560, 4096))
    all_e = rng.choice((8, 16, 60, 64, 128))
    e = all_e // 4 if rng.random() < 0.3 else all_e
    i = 8 * _log(rng, 32, min(512, 8 * 14336 * 4096 // (e * h * 8)))
    return experts(_log(rng, 1, 2048), h, i, e, rng.randint(1, min(8, all_e)), all_e,
                   rng.randint(0, all_e - e), rng.choice(("bf16", "bf16", "f16")),
                   rng.random() < 0.5)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)

    def normal(shape, dtype, scale=1.0):
        x = torch.randn(shape, generator=g, device="cuda", dtype=dtype)
        return x.mul_(scale) if scale != 1.0 else x

    dt, t = DTYPE[c["dtype"]], c["t"]
    if c["op"] == "route":
        c["logits"] = normal((t, c["e"]), torch.float32, 1.5).to(dt)
        c["b"] = normal((c["e"],), torch.float32, 0.1) if c["bias"] else None
        return c
    if c["op"] == "linear":
        n, k = c["n"], c["k"]
        odt = torch.float32 if c["out"] == "f32" else dt
        c["x"] = normal((t, k), dt)
        c["w"] = normal((n, k), dt, k ** -0.5)
        c["b"] = normal((n,), torch.float32, 0.5).to(dt) if c["bias"] else None
        c["r"] = normal((t, n // 2 if c["gated"] else n), odt) if c["residual"] else None
        return c
    h, i, e = c["h"], c["i"], c["e"]
    c["x"] = normal((t, h), dt)
    c["w13"] = normal((e, 2 * i, h), dt, h ** -0.5)
    c["w2"] = normal((e, h, i), dt, i ** -0.5)
    c["r"] = normal((t, h), dt) if c["residual"] else None
    top, ids = normal((t, c["all_e"]), torch.float32, 1.0).topk(c["top_k"], dim=1)
    c["ids"] = ids.to(torch.int32)
    c["weights"] = torch.softmax(top, dim=1)
    return c


# ---- plain forms --------------------------------------------------------------------------------

def _act(v, name):
    if name == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * 0.5 ** 0.5))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh((2 / math.pi) ** 0.5 * (v + 0.044715 * v * v * v)))
    return v


def _plain_linear(s):
    v = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        v = v + s["b"].float()
    if s["gated"]:
        half = s["n"] // 2
        v = _act(v[:, :half], s["act"]) * v[:, half:]
    else:
        v = _act(v, s["act"])
    if s["r"] is not None:
        v = v + s["r"].float()
    return v if s["out"] == "f32" else v.to(s["x"].dtype)


def _plain_route(s):
    logits = s["logits"].float()
    t, e = logits.shape
    if s["scoring"] == "sigmoid":
        score = 1 / (1 + torch.exp(-logits))
        key = score if s["b"] is None else score + s["b"]
    else:
        top = torch.exp(logits - logits.max(dim=1, keepdim=True).values)
        score = top / top.sum(dim=1, keepdim=True)
        key = logits
    if s["groups"] > 1:
        part = key.view(t, s["groups"], -1)
        two = 2 if s["scoring"] == "sigmoid" else 1
        best = torch.sort(part, dim=2, descending=True).values[:, :, :two].sum(dim=2)
        kept = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :s["top_groups"]]
        keep = torch.zeros(t, s["groups"], dtype=torch.bool, device=key.device)
        keep.scatter_(1, kept, True)
        key = torch.where(keep.unsqueeze(2), part, torch.full_like(part, -math.inf)).view(t, e)
    ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :s["top_k"]]
    weights = score.gather(1, ids)
    if s["renormalize"]:
        if s["scoring"] == "softmax":  # the softmax of the chosen logits
            chosen = logits.gather(1, ids)
            weights = torch.exp(chosen - chosen.max(dim=1, keepdim=True).values)
        weights = weights / weights.sum(dim=1, keepdim=True)
    return weights * s["scale"], ids.to(torch.int32)


def _plain_experts(s):
    t, h, i, e, top_k = s["t"], s["h"], s["i"], s["e"], s["top_k"]
    local = s["ids"].long() - s["first"]
    here = (local >= 0) & (local < e)
    pair = here.view(-1).nonzero().view(-1)
    expert = local.view(-1)[pair]
    x = s["x"].float()[pair // top_k]
    n = pair.numel()
    if n <= e:  # few pairs: each with its expert's matrices
        v = torch.bmm(s["w13"][expert].float(), x.unsqueeze(2)).squeeze(2)
        v = v[:, :i] / (1 + torch.exp(-v[:, :i])) * v[:, i:]
        v = torch.bmm(s["w2"][expert].float(), v.unsqueeze(2)).squeeze(2)
    else:  # the pairs of each expert side by side
        order = torch.sort(expert, stable=True).indices
        count = torch.bincount(expert, minlength=e)
        slot = torch.arange(n, device=x.device) - (count.cumsum(0) - count)[expert[order]]
        side = torch.zeros(e, int(count.max()), h, device=x.device)
        side[expert[order], slot] = x[order]
        u = torch.bmm(side, s["w13"].float().transpose(1, 2))
        u = u[..., :i] / (1 + torch.exp(-u[..., :i])) * u[..., i:]
        u = torch.bmm(u, s["w2"].float().transpose(1, 2))
        v = torch.empty(n, h, device=x.device)
        v[order] = u[expert[order], slot]
    every = torch.zeros(t * top_k, h, device=x.device)
    every[pair] = v * s["weights"].view(-1)[pair].unsqueeze(1)
    y = every.view(t, top_k, h).sum(dim=1)
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(s["x"].dtype)


def run(s):
    if not own:
        return {"linear": _plain_linear, "route": _plain_route, "experts": _plain_experts}[s["op"]](s)
    import paper_2607_18957_gb300 as cfa
    if s["op"] == "linear":
        return cfa.linear(s["x"], s["w"], s["b"], activation=s["act"], gated=s["gated"],
                          residual=s["r"], out_dtype="f32" if s["out"] == "f32" else None)
    if s["op"] == "route":
        return cfa.route(s["logits"], s["top_k"], scoring=s["scoring"], bias=s["b"],
                         groups=s["groups"], top_groups=s["top_groups"],
                         renormalize=s["renormalize"], scale=s["scale"])
    return cfa.experts(s["x"], s["ids"], s["weights"], s["w13"], s["w2"], first_expert=s["first"],
                       residual=s["r"])


# ---- work and exact values ----------------------------------------------------------------------

def work(case):
    c, t = case, case["t"]
    es = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "route":
        return {"bytes": t * (c["e"] * es + c["top_k"] * 8) + (4 * c["e"] if c["bias"] else 0),
                "flops": t * c["e"] * 4}
    if c["op"] == "linear":
        n, k = c["n"], c["k"]
        no = n // 2 if c["gated"] else n
        oes = 4 if c["out"] == "f32" else es
        return {"bytes": es * (t * k + n * k + (n if c["bias"] else 0))
                + oes * t * no * (2 if c["residual"] else 1), "flops": 2 * t * n * k}
    h, i, e = c["h"], c["i"], c["e"]
    read = e * (1 - (1 - c["top_k"] / c["all_e"]) ** t)  # experts that are chosen at all
    pairs = t * c["top_k"] * e / c["all_e"]
    return {"bytes": es * (read * 3 * h * i + t * h * (3 if c["residual"] else 2))
            + t * c["top_k"] * 8, "flops": 6 * pairs * h * i}


def exact(case, seed):
    if work(case)["flops"] > 8e12:
        return None
    s = prepare(case, seed)
    if s["op"] == "linear":
        y = torch.mm(s["x"].double(), s["w"].double().transpose(0, 1))
        if s["b"] is not None:
            y += s["b"].double()[None, :]
        a = y[:, :s["n"] // 2] if s["gated"] else y
        a = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0),
             "silu": lambda v: v * torch.sigmoid(v),
             "gelu": lambda v: v * torch.special.ndtr(v),
             "gelu_tanh": lambda v: v * torch.sigmoid(
                 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))}[s["act"]](a)
        y = a * y[:, s["n"] // 2:] if s["gated"] else a
        return y if s["r"] is None else y + s["r"].double()
    if s["op"] == "experts":
        y = torch.zeros(s["t"], s["h"], dtype=torch.float64, device="cuda")
        if s["r"] is not None:
            y += s["r"].double()
        for k in range(s["e"]):
            tok, j = torch.where(s["ids"] == s["first"] + k)
            if tok.numel():
                gate, up = torch.mm(s["x"][tok].double(), s["w13"][k].double().t()).chunk(2, dim=1)
                out = torch.mm(gate * torch.sigmoid(gate) * up, s["w2"][k].double().t())
                y.index_add_(0, tok, out * s["weights"][tok, j].double()[:, None])
        return y
    z = s["logits"].double()
    p = torch.sigmoid(z) if s["scoring"] == "sigmoid" else torch.softmax(z, dim=1)
    # the choice itself is made on 32-bit scores, as the operator's definition has it
    key = z if s["scoring"] == "softmax" else p.float()
    if s["b"] is not None:
        key = key + s["b"]
    if s["groups"] > 1:
        part = key.unflatten(1, (s["groups"], -1))
        best = part.amax(dim=2)
        if s["scoring"] == "sigmoid":
            best = part.topk(2, dim=2).values.sum(dim=2)
        rank = best.argsort(dim=1, descending=True, stable=True).argsort(dim=1)
        key = part.masked_fill((rank >= s["top_groups"])[:, :, None], -math.inf).flatten(1)
    ids = key.argsort(dim=1, descending=True, stable=True)[:, :s["top_k"]]
    w = torch.take_along_dim(p, ids, dim=1)
    if s["renormalize"]:
        w = w / w.sum(dim=1, keepdim=True)
    return w * s["scale"], None
