"""Operators of a decoding step around the products with the loaded parameters, for measuring: the norms
between blocks (`norm`), the rotation of queries and keys with the appending of keys and values to a
paged cache (`append`), the attention of new tokens over that cache (`attend`), and the log
probabilities of chosen tokens (`logprobs`).

A case names the operator and its sizes:

    norm      a = x, or x / rms(x) * (offset + post_weight); a *= act(gate); h = residual + scale * a;
              y = h / rms(h) * (offset + weight), rms(v) = sqrt(mean(v^2) + eps): t tokens of c columns
    append    t tokens of a fused q/k/v row (heads, kv_heads, kv_heads of dim): q and k rotated by
              position * frequency in the first `rot` of dim, pairs (i, i + rot / 2) or, interleaved,
              (2 i, 2 i + 1); k and v go to their slots of the cache [pages, page, kv_heads, dim],
              in 8 bits divided by their scales
    attend    `new` tokens of each of b sequences over its pages: token i sees the keys up to
              length - new + i, the last `window` of them with a window; the page table's rows are as
              wide as the longest sequence
    logprobs  log softmax(scale * logits) at each row's token, the entropy, and the `top` largest

Sizes are those of the benchmark's decoders (hidden 4096 or 8192, 32 or 64 query heads and 8 key/value
heads of 128, vocabularies of 32,000 and 128,256) and generic ones.
"""
import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32,
         "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}


def norm(t, c, dtype="bf16", residual=True, post=False, gate=False, scale=1.0, offset=0.0):
    return {"op": "norm", "t": t, "c": c, "dtype": dtype, "residual": residual, "post": post,
            "gate": gate, "scale": scale, "offset": offset}


def append(t, heads, kv_heads, dim, dtype="bf16", cache="same", rot=None, interleaved=False,
           stretch=1.0, first=0, page=16, layout="tokens"):
    return {"op": "append", "t": t, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "cache": dtype if cache == "same" else cache, "rot": rot or dim,
            "interleaved": interleaved, "stretch": stretch, "first": first, "page": page,
            "layout": layout}


def attend(b, least, most, heads, kv_heads, dim, dtype="bf16", cache="same", new=1, window=0, page=16,
           layout="tokens", lse=False):
    return {"op": "attend", "b": b, "least": least, "most": most, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "cache": dtype if cache == "same" else cache, "new": new, "window": window, "page": page,
            "layout": layout, "lse": lse}


def logprobs(t, v, dtype="f32", top=0, scale=1.0):
    return {"op": "logprobs", "t": t, "v": v, "dtype": dtype, "top": top, "scale": scale}


def listed():
    return [
        # one decoded token between two blocks: latency alone
        dict(norm(1, 4096), name="norm_token"),
        # a prompt's tokens between two blocks of the larger decoder
        dict(norm(4096, 8192), name="norm_prompt"),
        # a block with a norm behind it, a gate and a residual scale, rows off the 16-byte grid
        dict(norm(1777, 2307, "f16", post=True, gate=True, scale=0.25, offset=1.0), name="norm_gated_odd"),
        # one decoded token's q/k/v, at a far position
        dict(append(1, 32, 8, 128, first=100003), name="append_token"),
        # a prompt of 8192 tokens of the larger decoder, frequencies stretched for long contexts
        dict(append(8192, 64, 8, 128, stretch=8.0), name="append_prompt"),
        # 777 tokens, half of each head rotated in pairs of neighbours, into a cache in 8 bits whose
        # pages hold one head's tokens side by side
        dict(append(777, 32, 4, 96, "f16", "e4m3", rot=48, interleaved=True, first=4095, page=48,
                    layout="heads"), name="append_e4m3_partial"),
        # one sequence of a thousand tokens: latency
        dict(attend(1, 1000, 1000, 32, 8, 128), name="attend_one"),
        # a decoding batch of 64 sequences from one token to 8192
        dict(attend(64, 1, 8192, 32, 8, 128), name="attend_batch"),
        # two long sequences, the larger decoder's heads
        dict(attend(2, 100001, 131072, 64, 8, 128, page=64, lse=True), name="attend_long"),
        # four drafted tokens of 24 sequences, a cache in 8 bits, a window
        dict(attend(24, 500, 6000, 32, 8, 128, "f16", "e4m3", new=4, window=4096, page=24,
                    layout="heads"), name="attend_draft_e4m3"),
        # one decoded token with its 20 best alternatives
        dict(logprobs(1, 128256, top=20), name="logprobs_token"),
        # a scored prompt of 2048 tokens
        dict(logprobs(2048, 128256, "bf16", top=5, scale=1.25), name="logprobs_prompt"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "append", "attend", "attend", "logprobs"))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if op == "norm":
        c = _log(rng, 64, 16384)
        if rng.random() < 0.8:  # rows on the 16-byte grid, as nearly every model's are
            c = (c + 7) // 8 * 8
        residual = rng.random() < 0.7
        return norm(_log(rng, 1, min(16384, 4096 * 8192 // c)), c, rng.choice(("bf16", "f16", "f32")),
                    residual, rng.random() < 0.3, rng.random() < 0.3,
                    rng.choice((1.0, 0.22)) if residual else 1.0, rng.choice((0.0, 1.0)))
    if op == "logprobs":
        v = _log(rng, 1000, 262144)
        return logprobs(_log(rng, 1, min(4096, 2048 * 128256 // (2 * v))), v,
                        rng.choice(("f32", "f32", "bf16", "f16")), rng.randint(0, 20),
                        rng.choice((1.0, 1.0, 0.7, 2.0)))
    dim = rng.choice((64, 96, 128, 128, 128, 256))
    kv_heads = rng.choice((1, 2, 4, 8))
    heads = kv_heads * rng.choice((1, 3, 4, 6, 8, 16))
    cache = rng.choice(("same", "same", "e4m3"))
    page = rng.choice((16, 16, 32, 64, 24, 17, 128))
    layout = rng.choice(("tokens", "heads"))
    if op == "append":
        most = 8192 * 80 * 128 // ((heads + 2 * kv_heads) * dim)
        return append(_log(rng, 1, min(16384, most)), heads, kv_heads, dim, dtype, cache,
                      dim // rng.choice((1, 1, 2)), rng.random() < 0.4, rng.choice((1.0, 8.0)),
                      _log(rng, 1, 200000), page, layout)
    b = _log(rng, 1, 128)
    most = _log(rng, 64, max(64, min(131072, 2 ** 28 // (b * kv_heads * dim))))
    new = min(rng.choice((1, 1, 1, 2, 5)), most)
    return attend(b, rng.randint(new, most), most, heads, kv_heads, dim, dtype, cache, new,
                  rng.choice((0, 0, 100, 1024)), page, layout, rng.random() < 0.3)


def lengths_of(case):
    """The sequences' lengths, from `least` to `most` with equal ratios."""
    b, lo, hi = case["b"], case["least"], case["most"]
    return [hi if b == 1 else max(1, int(round(lo * (hi / lo) ** (i / (b - 1))))) for i in range(b)]


def frequencies_of(case):
    """Radians per position of each pair; beyond a wavelength the stretched ones turn that much slower,
    with a smooth passage, as contexts longer than those of the training want them."""
    half, stretch = case["rot"] // 2, case["stretch"]
    f = 500000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    if stretch != 1.0:
        turns = 8192 * f / (2 * math.pi)
        smooth = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
        f = f * (smooth + (1.0 - smooth) / stretch)
    return f


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)
    dt = DTYPE[c["dtype"]]

    def normal(shape, dtype=dt, scale=1.0):
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
        return x.mul_(scale).to(dtype) if dtype is not torch.float32 or scale != 1.0 else x

    def order(n):
        return torch.randperm(n, generator=g, device="cuda")

    if c["op"] == "norm":
        t, n = c["t"], c["c"]
        mid = 1.0 - c["offset"]
        c["x"] = normal((t, n))
        c["w"] = (normal((n,), torch.float32, 0.2) + mid).to(dt)
        c["p"] = (normal((n,), torch.float32, 0.2) + mid).to(dt) if c["post"] else None
        c["g"] = normal((t, n)) if c["gate"] else None
        c["r"] = normal((t, n), dt, 3.0) if c["residual"] else None
        return c
    if c["op"] == "logprobs":
        c["logits"] = normal((c["t"], c["v"]), dt, 2.5)
        c["tokens"] = torch.randint(0, c["v"], (c["t"],), generator=g, device="cuda",
                                    dtype=torch.int32)
        return c
    kv, dim, page = c["kv_heads"], c["dim"], c["page"]
    cdt, cscale = DTYPE[c["cache"]], 0.02 if c["cache"] == "e4m3" else 1.0
    c["k_scale"], c["v_scale"] = cscale, cscale * 0.75 if cscale != 1.0 else 1.0

    def cache(pages, scale):
        shape = (pages, page, kv, dim) if c["layout"] == "tokens" else (pages, kv, page, dim)
        x = torch.empty(shape, device="cuda", dtype=cdt)
        for i in range(0, pages, 4096):
            part = x[i:i + 4096]
            part.copy_(normal(part.shape, torch.float32).div_(scale).to(cdt))
        return x if c["layout"] == "tokens" else x.transpose(1, 2)

    if c["op"] == "append":
        t = c["t"]
        pages = (t + page - 1) // page + 3
        c["qkv"] = normal((t, (c["heads"] + 2 * kv) * dim))
        c["positions"] = torch.arange(c["first"], c["first"] + t, device="cuda", dtype=torch.int32)
        at = torch.arange(t, device="cuda")
        c["slots"] = (order(pages)[at // page] * page + at % page).to(torch.int32)
        c["k_cache"], c["v_cache"] = cache(pages, c["k_scale"]), cache(pages, c["v_scale"])
        c["frequencies"] = frequencies_of(c).cuda()
        return c
    lens = torch.tensor(lengths_of(c), device="cuda", dtype=torch.int32)
    c["lengths"] = lens[order(c["b"])].contiguous()
    per = (c["most"] + page - 1) // page
    held = ((c["lengths"] + page - 1) // page).long()
    pages = sum((n + page - 1) // page for n in lengths_of(c))
    table = torch.arange(per, device="cuda")[None, :] + (held.cumsum(0) - held)[:, None]
    c["pages"] = order(pages)[table.clamp(max=pages - 1)].to(torch.int32)
    c["k_cache"], c["v_cache"] = cache(pages, c["k_scale"]), cache(pages, c["v_scale"])
    shape = (c["b"], c["new"], c["heads"], dim)
    c["q"] = normal(shape if c["new"] > 1 else (c["b"], c["heads"], dim))
    return c


# ---- plain forms --------------------------------------------------------------------------------

def _rms(v, weight, offset):
    return v / torch.sqrt((v * v).mean(dim=1, keepdim=True) + 1e-6) * (weight.float() + offset)


def _plain_norm(s):
    dt, a = s["x"].dtype, s["x"].float()
    if s["p"] is not None:
        a = _rms(a, s["p"], s["offset"])
    if s["g"] is not None:
        gate = s["g"].float()
        a = a * (gate / (1 + torch.exp(-gate)))
    if s["r"] is None:
        return _rms(a, s["w"], s["offset"]).to(dt)
    h = s["r"].float() + s["scale"] * a
    return _rms(h, s["w"], s["offset"]).to(dt), h.to(dt)


def _plain_append(s):
    t, heads, kv, dim, rot = s["t"], s["heads"], s["kv_heads"], s["dim"], s["rot"]
    x = s["qkv"].float().view(t, heads + 2 * kv, dim)
    angle = s["positions"].double()[:, None] * s["frequencies"][None, :]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    part = x[:, :heads + kv, :rot]
    if s["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=3).flatten(2)
    else:
        a, b = part[..., :rot // 2], part[..., rot // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=2)
    turned = torch.cat((turned, x[:, :heads + kv, rot:]), dim=2)
    slots = s["slots"].long()
    at = (slots // s["page"], slots % s["page"])
    kc, vc = s["k_cache"], s["v_cache"]
    kc[at] = (turned[:, heads:] / s["k_scale"]).clamp(-448, 448).to(kc.dtype) \
        if s["cache"] == "e4m3" else turned[:, heads:].to(kc.dtype)
    vc[at] = (x[:, heads + kv:] / s["v_scale"]).clamp(-448, 448).to(vc.dtype) \
        if s["cache"] == "e4m3" else x[:, heads + kv:].to(vc.dtype)
    return turned[:, :heads].to(s["qkv"].dtype), kc, vc


def _plain_attend(s):
    b, new, heads, kv, dim = s["b"], s["new"], s["heads"], s["kv_heads"], s["dim"]
    group = heads // kv
    pages = s["pages"].long()

    def side_by_side(cache, scale):  # [b, kv, keys, dim]
        x = cache[pages].flatten(1, 2).transpose(1, 2).float()
        return x * scale if scale != 1.0 else x

    k = side_by_side(s["k_cache"], s["k_scale"])
    q = s["q"].float().view(b, new, kv, group, dim).permute(0, 2, 1, 3, 4).reshape(b, kv, -1, dim)
    z = (q @ k.transpose(2, 3) * dim ** -0.5).view(b, kv, new, group, -1)
    at = torch.arange(k.shape[2], device=k.device)[None, None, :]
    last = s["lengths"][:, None, None] - new + torch.arange(new, device=k.device)[None, :, None]
    seen = at <= last
    if s["window"]:
        seen = seen & (at > last - s["window"])
    z = torch.where(seen[:, None, :, None, :], z, torch.full_like(z, -math.inf))
    top = z.max(dim=4, keepdim=True).values
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    p = torch.exp(z - top)
    total = p.sum(dim=4, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = p.view(b, kv, new * group, -1) @ side_by_side(s["v_cache"], s["v_scale"])
    o = o.view(b, kv, new, group, dim).permute(0, 2, 1, 3, 4).reshape(s["q"].shape).to(s["q"].dtype)
    if not s["lse"]:
        return o
    lse = (top + torch.log(total)).view(b, kv, new, group).permute(0, 2, 1, 3)
    return o, lse.reshape(s["q"].shape[:-1])


def _plain_logprobs(s):
    z = s["logits"].float()
    z = z - z.max(dim=1, keepdim=True).values
    if s["scale"] != 1.0:
        z = z * s["scale"]
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True)
    log_total = torch.log(total)
    given = z.gather(1, s["tokens"].long()[:, None]) - log_total
    entropy = log_total - (e * z).sum(dim=1, keepdim=True) / total
    if not s["top"]:
        return given[:, 0], entropy[:, 0]
    best, ids = torch.sort(s["logits"], dim=1, descending=True, stable=True)
    ids = ids[:, :s["top"]]
    return given[:, 0], entropy[:, 0], z.gather(1, ids) - log_total, ids.to(torch.int32)


def run(s):
    if not own:
        return {"norm": _plain_norm, "append": _plain_append, "attend": _plain_attend,
                "logprobs": _plain_logprobs}[s["op"]](s)
    import paper_2607_18957_gb300 as cfa
    if s["op"] == "norm":
        return cfa.norm(s["x"], s["w"], residual=s["r"], gate=s["g"], post_weight=s["p"],
                        scale=s["scale"], offset=s["offset"])
    if s["op"] == "append":
        q = cfa.append(s["qkv"], s["k_cache"], s["v_cache"], s["slots"], heads=s["heads"],
                       positions=s["positions"], frequencies=s["frequencies"],
                       interleaved=s["interleaved"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return q, s["k_cache"], s["v_cache"]
    if s["op"] == "attend":
        return cfa.attend(s["q"], s["k_cache"], s["v_cache"], s["pages"], s["lengths"],
                          window=s["window"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                          lse=s["lse"])
    return cfa.logprobs(s["logits"], s["tokens"], top=s["top"], scale=s["scale"])


# ---- work and exact values ----------------------------------------------------------------------

def work(case):
    c, es = case, SIZE[case["dtype"]]
    if c["op"] == "norm":
        n = 2 + (2 if c["residual"] else 0) + (1 if c["gate"] else 0)
        return {"bytes": es * c["c"] * (n * c["t"] + (2 if c["post"] else 1)),
                "flops": c["t"] * c["c"] * 4 * (2 if c["post"] else 1)}
    if c["op"] == "logprobs":
        return {"bytes": c["t"] * (c["v"] * es + 12 + 8 * c["top"]), "flops": c["t"] * c["v"] * 5}
    h, kv, d, ces = c["heads"], c["kv_heads"], c["dim"], SIZE[c["cache"]]
    if c["op"] == "append":
        return {"bytes": c["t"] * (es * d * (2 * h + 2 * kv) + 2 * ces * d * kv + 8) + 4 * c["rot"],
                "flops": c["t"] * 3 * (h + kv) * c["rot"]}
    span = c["window"] + c["new"] - 1 if c["window"] else c["most"]
    keys = sum(min(n, span) for n in lengths_of(c))
    rows = c["b"] * c["new"] * h
    table = 4 * sum((n + c["page"] - 1) // c["page"] for n in lengths_of(c))
    return {"bytes": 2 * keys * kv * d * ces + 2 * rows * d * es + table + (4 * rows if c["lse"] else 0),
            "flops": 4 * keys * c["new"] * h * d}


def exact(case, seed):
    if case["op"] == "logprobs" and case["t"] * case["v"] > 3e8:
        return None
    s = prepare(case, seed)
    if s["op"] == "norm":
        def unit(v):
            return v * (v.pow(2).sum(1, keepdim=True) / s["c"] + 1e-6).rsqrt()
        a = s["x"].double()
        if s["post"]:
            a = unit(a) * (s["offset"] + s["p"].double())
        if s["gate"]:
            a = a * s["g"].double() * torch.sigmoid(s["g"].double())
        if not s["residual"]:
            return unit(a) * (s["offset"] + s["w"].double())
        h = torch.add(s["r"].double(), a, alpha=s["scale"])
        return unit(h) * (s["offset"] + s["w"].double()), h
    if s["op"] == "append":
        h, kv, d, rot = s["heads"], s["kv_heads"], s["dim"], s["rot"]
        x = s["qkv"].double().unflatten(1, (h + 2 * kv, d))
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           torch.outer(s["positions"].double(), s["frequencies"]))[:, None, :]
        first = torch.arange(rot // 2, device="cuda")
        i, j = (2 * first, 2 * first + 1) if s["interleaved"] else (first, first + rot // 2)
        both = torch.complex(x[..., i], x[..., j])[:, :h + kv] * turn
        x[:, :h + kv, i], x[:, :h + kv, j] = both.real, both.imag
        k, v = s["k_cache"].double().contiguous(), s["v_cache"].double().contiguous()
        most = 448.0 if s["cache"] == "e4m3" else math.inf
        k.view(-1, kv, d)[s["slots"].long()] = (x[:, h:h + kv] / s["k_scale"]).clamp(-most, most)
        v.view(-1, kv, d)[s["slots"].long()] = (x[:, h + kv:] / s["v_scale"]).clamp(-most, most)
        return x[:, :h], k, v
    if s["op"] == "attend":
        group = s["heads"] // s["kv_heads"]
        o = torch.zeros(s["b"], s["new"], s["heads"], s["dim"], dtype=torch.float64, device="cuda")
        lse = torch.full(o.shape[:-1], -math.inf, dtype=torch.float64, device="cuda")
        q = s["q"].double().view(o.shape)
        for b, n in enumerate(s["lengths"].tolist()):
            held = s["pages"][b, :(n + s["page"] - 1) // s["page"]].long()
            k = s["k_cache"][held].double().flatten(0, 1)[:n] * s["k_scale"]
            v = s["v_cache"][held].double().flatten(0, 1)[:n] * s["v_scale"]
            for i in range(s["new"]):
                end = n - s["new"] + i + 1
                begin = max(0, end - s["window"]) if s["window"] else 0
                if end <= begin:
                    continue
                heads = q[b, i].view(s["kv_heads"], group, -1)
                z = torch.einsum("hgd,nhd->hgn", heads, k[begin:end]) / math.sqrt(s["dim"])
                lse[b, i] = torch.logsumexp(z, dim=2).flatten()
                o[b, i] = torch.einsum("hgn,nhd->hgd", torch.softmax(z, dim=2),
                                       v[begin:end]).flatten(0, 1)
        o = o.view(s["q"].shape)
        return (o, lse.view(s["q"].shape[:-1])) if s["lse"] else o
    given, entropy, best = [], [], []
    ids = []
    for rows, tokens in zip(s["logits"].split(256), s["tokens"].split(256)):
        z = torch.log_softmax(rows.double() * s["scale"], dim=1)
        given.append(torch.take_along_dim(z, tokens.long()[:, None], dim=1)[:, 0])
        entropy.append(-(z.exp() * z).sum(dim=1))
        if s["top"]:
            best.append(rows.double().topk(s["top"], dim=1).values)
            ids.append(torch.logsumexp(rows.double() * s["scale"], dim=1, keepdim=True))
    if not s["top"]:
        return torch.cat(given), torch.cat(entropy)
    return (torch.cat(given), torch.cat(entropy),
            torch.cat(best) * s["scale"] - torch.cat(ids), None)
