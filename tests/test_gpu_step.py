"""norm, append and logprobs against plain forms in 64 bits.

Bounds are worst cases, element by element, with u = 2^-24 the rounding of fp32.  A sum of n terms in
fp32 is off by (n + 8) u of the sum of the terms' magnitudes; exp, erf, tanh, sine and cosine by up to
2^-21; the result by half a step of its type, and near zero by half that type's smallest step."""
import math

import pytest
import torch

import paper_2607_18957_gb300 as cfa

pytestmark = pytest.mark.gpu

BF16, F16, F32, F8 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
HALF_ULP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24, F8: 2.0 ** -4}
NEAR_ZERO = {BF16: 0.0, F16: 2.0 ** -25, F32: 0.0, F8: 2.0 ** -10}
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def cuda_device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def inside(t, extra=0, lead=0, fill=7.0):
    """A copy of a matrix as a view of a larger buffer: `lead` elements before it, rows `extra` apart."""
    rows, cols = t.shape
    buf = torch.full((lead + (rows + 2) * (cols + extra),), fill, dtype=t.dtype, device="cuda")
    view = buf[lead:].as_strided((rows, cols), (cols + extra, 1))
    view.copy_(t)
    return buf, view


def close(got, ref, bound):
    got = got.double()
    assert got.shape == ref.shape
    assert bool((torch.isfinite(got) == torch.isfinite(ref)).all())
    worst = torch.where(torch.isfinite(ref), (got - ref).abs() - bound, -1.0).max().item() if got.numel() else 0.0
    assert worst <= 0, f"off by {worst:g} more than the bound"


def rounded(v, ev, dtype):
    return ev + HALF_ULP[dtype] * (v.abs() + ev) + NEAR_ZERO[dtype]


# ---- norm ---------------------------------------------------------------------------------------

def act64(v, name):
    return {"none": lambda x: x, "relu": lambda x: x.clamp(min=0),
            "silu": lambda x: x * torch.sigmoid(x),
            "gelu": lambda x: 0.5 * x * (1 + torch.erf(x / math.sqrt(2))),
            "gelu_tanh": lambda x: 0.5 * x * (1 + torch.tanh(
                math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))}[name](v)


def rms64(v, ev, w, offset, eps):
    c = v.shape[-1]
    rms = torch.sqrt((v * v).mean(-1, keepdim=True) + eps)
    rel = (c + 8) * U + 8 * U + torch.sqrt((ev * ev).mean(-1, keepdim=True)) / rms
    m = (offset + w.double()) / rms
    y = v * m
    return y, y.abs() * rel * (1 + rel) + ev * m.abs() * (1 + rel) + v.abs() / rms * 2 * U * (
        abs(offset) + w.double().abs())


def norm64(x, w, r=None, g=None, act="silu", p=None, scale=1.0, eps=1e-6, offset=0.0):
    a, ea = x.double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    if p is not None:
        a, ea = rms64(a, ea, p, offset, eps)
    if g is not None:
        v = act64(g.double(), act)
        ea = ea * v.abs() + (a.abs() + ea) * 2.0 ** -20 * g.double().abs() + 2 * U * (a * v).abs()
        a = a * v
    h, eh = a * scale, ea * abs(scale) + 2 * U * (a * scale).abs()
    if r is not None:
        h = h + r.double()
        eh = eh + 2 * U * (h.abs() + eh)
    y, ey = rms64(h, eh, w, offset, eps)
    return y, rounded(y, ey, x.dtype), h, rounded(h, eh, x.dtype)


ROWS = [(1, 1), (3, 7), (1, 64), (300, 128), (5, 96), (2, 1000), (7, 1024), (33, 2307), (4, 4096),
        (130, 5120), (2, 8192), (3, 8200), (2, 12289), (3, 16384), (1, 16383)]


@pytest.mark.parametrize("t,c", ROWS)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_norm(t, c, dtype):
    g = gen(t * 131 + c)
    x, w, r = normal(g, (t, c), dtype), normal(g, (c,), dtype), normal(g, (t, c), dtype, 3.0)
    y64, ey, _, _ = norm64(x, w)
    close(cfa.norm(x, w), y64, ey)
    y64, ey, h64, eh = norm64(x, w, r, scale=0.37, offset=1.0, eps=1e-5)
    y, h = cfa.norm(x, w, residual=r, scale=0.37, offset=1.0, eps=1e-5)
    assert y.dtype == h.dtype == dtype
    close(y, y64, ey)
    close(h, h64, eh)


@pytest.mark.parametrize("t,c", [(1, 64), (5, 1003), (64, 2048), (3, 16384)])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (F16, F32), (F32, F32)])
def test_norm_of_every_part(t, c, act, dtype, wdtype):
    g = gen(t + c)
    x, w, p = normal(g, (t, c), dtype, 5.0), normal(g, (c,), wdtype), normal(g, (c,), wdtype)
    r, z = normal(g, (t, c), dtype), normal(g, (t, c), dtype, 2.0)
    for gate in (z, z[0]):
        y64, ey, h64, eh = norm64(x, w, r, gate.expand(t, c), act, p, -1.5)
        y, h = cfa.norm(x, w, residual=r, gate=gate, activation=act, post_weight=p, scale=-1.5)
        close(y, y64, ey)
        close(h, h64, eh)
        y64, ey, _, _ = norm64(x, w, None, gate.expand(t, c), act)
        close(cfa.norm(x, w, gate=gate, activation=act), y64, ey)


@pytest.mark.parametrize("lead,extra", [(0, 8), (1, 8), (8, 3), (3, 0)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_of_rows_apart(lead, extra, dtype):
    g = gen(lead * 10 + extra)
    t, c = 9, 520
    x, r, w = normal(g, (t, c), dtype), normal(g, (t, c), dtype), normal(g, (c,), dtype)
    ref = cfa.norm(x, w, residual=r)
    _, xv = inside(x, extra, lead)
    rbuf, rv = inside(r, extra, lead)
    ybuf, yv = inside(torch.zeros_like(x), extra, lead)
    y, h = cfa.norm(xv, w, residual=rv, out=(yv, rv))  # h in the residual's place
    assert y is yv and h is rv
    y64, ey, h64, eh = norm64(x, w, r)
    close(y, y64, ey)
    close(h, h64, eh)
    for buf in (rbuf, ybuf):
        mask = torch.ones_like(buf, dtype=torch.bool)
        mask[lead:].as_strided((t, c), (c + extra, 1)).fill_(False)
        assert bool((buf[mask] == 7.0).all())
    # in place on x, three dimensions
    x3 = x.clone().view(3, 3, c)
    y3 = cfa.norm(x3, w, out=x3)
    close(y3.view(t, c), *norm64(x, w)[:2])
    assert ref[0].shape == (t, c)


def test_norm_of_heads_inside_a_fused_row():
    g = gen(3)
    qkv = normal(g, (50, 6, 128), BF16)
    w = normal(g, (128,), BF16)
    y = cfa.norm(qkv.view(300, 128), w)
    close(y, *norm64(qkv.view(300, 128), w)[:2])


def test_norm_of_zeros_infinities_and_silu_far_below_zero():
    c = 256
    w = torch.ones(c, dtype=F32, device="cuda")
    x = torch.zeros(3, c, dtype=F32, device="cuda")
    x[1, 5], x[2, 6] = math.nan, math.inf
    y = cfa.norm(x, w)
    assert bool((y[0] == 0).all()) and bool(y[1].isnan().all())
    assert bool(y[2, 6].isnan()) and bool((y[2, :6] == 0).all())  # inf / inf, 0 / inf
    gate = torch.full((1, c), -100.0, device="cuda")
    big = torch.full((1, c), 2.0 ** 100, device="cuda")
    _, h = cfa.norm(big, w, gate=gate, residual=torch.zeros_like(big))
    want = 2.0 ** 100 * -100.0 / (1 + math.exp(100.0))
    assert bool(((h.double() / want - 1).abs() < 2.0 ** -18).all())


def test_norm_of_no_tokens():
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    w = torch.ones(64, dtype=BF16, device="cuda")
    assert cfa.norm(x, w).shape == (0, 64)


# ---- append -------------------------------------------------------------------------------------

def turned64(x, positions, f, interleaved, magnitude):
    """The first 2 len(f) values of each head turned, and the bound on the error in fp32."""
    half = f.shape[0]
    out, err = x.clone(), torch.zeros_like(x)
    angle = positions.double()[:, None] * f[None, :]
    off = (2.0 ** -20 + angle.abs() * 2.0 ** -50)[:, None, :]
    cos, sin = torch.cos(angle)[:, None, :] * magnitude, torch.sin(angle)[:, None, :] * magnitude
    at = torch.arange(half, device="cuda")
    i, j = (2 * at, 2 * at + 1) if interleaved else (at, at + half)
    a, b = x[..., i], x[..., j]
    out[..., i], out[..., j] = a * cos - b * sin, b * cos + a * sin
    err[..., i] = err[..., j] = (a.abs() + b.abs()) * off * abs(magnitude)
    return out, err


def make_cache(pages, page, kv, dim, dtype, layout, g):
    """[pages, page, kv, dim] in the memory order of `layout`."""
    if layout == "tokens":
        return normal(g, (pages, page, kv, dim), F32).to(dtype)
    if layout == "heads":
        return normal(g, (pages, kv, page, dim), F32).to(dtype).transpose(1, 2)
    if layout == "odd":  # off the 16-byte grid
        buf = normal(g, (pages, page, kv, dim + 1), F32).to(dtype)
        return buf[..., 1:]
    raise ValueError(layout)


CASES = [  # t, heads, kv, dim, rot, interleaved, page, layout
    (1, 32, 8, 128, 128, False, 16, "tokens"), (1, 4, 1, 8, 2, True, 1, "tokens"),
    (3, 3, 3, 64, 32, True, 5, "heads"), (7, 8, 2, 96, 48, False, 16, "heads"),
    (33, 6, 2, 80, 80, True, 17, "tokens"), (100, 5, 1, 256, 64, False, 64, "tokens"),
    (257, 2, 2, 72, 36, False, 24, "tokens"), (1023, 4, 2, 64, 64, False, 16, "heads"),
    (1024, 4, 2, 64, 64, True, 16, "tokens"), (2049, 7, 1, 128, 128, False, 32, "odd"),
    (1500, 2, 1, 512, 512, False, 16, "tokens"), (5, 2, 1, 512, 6, True, 3, "odd"),
    (1300, 8, 8, 16, 16, False, 7, "tokens"), (40, 2, 1, 128, 0, False, 16, "tokens")]


@pytest.mark.parametrize("t,heads,kv,dim,rot,interleaved,page,layout", CASES)
@pytest.mark.parametrize("dtype,cdtype", [(BF16, BF16), (F16, F16), (BF16, F8), (F16, F8)])
def test_append(t, heads, kv, dim, rot, interleaved, page, layout, dtype, cdtype):
    g = gen(t * 7 + dim + rot)
    pages = (t + page - 1) // page + 2
    qkv = normal(g, (t, (heads + 2 * kv) * dim), dtype, 2.0)
    kc, vc = (make_cache(pages, page, kv, dim, cdtype, layout, g) for _ in range(2))
    k0, v0 = kc.clone(), vc.clone()
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:t].to(torch.int32)
    positions = torch.randint(0, 1 << 20, (t,), generator=g, device="cuda", dtype=torch.int32)
    f, m = (cfa.rotary_frequencies(rot, 10000.0, scaling="ramp", factor=4.0, length=4096)
            if rot else ([], 1.0))
    f = torch.tensor(f, dtype=torch.float64, device="cuda")
    ks, vs = (0.03, 0.02) if cdtype is F8 else (1.0, 1.0)
    before = qkv.clone()
    q = cfa.append(qkv, kc, vc, slots, heads=heads, positions=positions if rot else None,
                   frequencies=f if rot else None, interleaved=interleaved, magnitude=m, k_scale=ks,
                   v_scale=vs)
    assert torch.equal(qkv, before) and q.shape == (t, heads, dim) and q.dtype == dtype
    x = qkv.double().view(t, heads + 2 * kv, dim)
    y, e = turned64(x[:, :heads + kv], positions, f, interleaved, m)
    close(q, y[:, :heads], rounded(y[:, :heads], e[:, :heads], dtype))
    at = (slots.long() // page, slots.long() % page)
    for c, c0, v, ev, scale in ((kc, k0, y[:, heads:], e[:, heads:], ks),
                                (vc, v0, x[:, heads + kv:], torch.zeros_like(x[:, heads + kv:]), vs)):
        v, ev = v / scale, ev / scale + (2 * U * (v / scale).abs() if cdtype is F8 else 0)
        if cdtype is F8:
            v = v.clamp(-448, 448)
        close(c[at], v, rounded(v, ev, cdtype))
        rest = torch.ones(pages, page, dtype=torch.bool, device="cuda")
        rest[at] = False
        assert torch.equal(c[rest].view(torch.uint8), c0[rest].view(torch.uint8))


def test_append_far_and_negative_positions():
    t, dim = 6, 64
    g = gen(5)
    qkv = normal(g, (t, 3 * dim), F16)
    kc, vc = (torch.zeros(1, 8, 1, dim, dtype=F16, device="cuda") for _ in range(2))
    positions = torch.tensor([0, -1, -(1 << 31), (1 << 31) - 1, 1 << 30, 123456789], dtype=torch.int32,
                             device="cuda")
    f = torch.tensor([10.0] + cfa.rotary_frequencies(dim)[0][1:], dtype=torch.float64, device="cuda")
    q = cfa.append(qkv, kc, vc, torch.arange(t, dtype=torch.int32, device="cuda"), heads=1,
                   positions=positions, frequencies=f)
    y, e = turned64(qkv.double().view(t, 3, dim)[:, :1], positions, f, False, 1.0)
    close(q, y, rounded(y, e, F16))


@pytest.mark.parametrize("t", [6, 1030])
def test_append_leaves_out_slots_that_are_not_there(t):
    g = gen(t)
    kv, dim, page, pages = 2, 64, 4, 400
    qkv = normal(g, (t, 6 * dim), BF16)
    kc, vc = (torch.zeros(pages + 2, page, kv, dim, dtype=BF16, device="cuda") for _ in range(2))
    slots = torch.arange(t, dtype=torch.int32, device="cuda")
    slots[0], slots[1], slots[2], slots[3] = -1, pages * page, (1 << 31) - 1, -(1 << 31)
    cfa.append(qkv, kc[1:-1], vc[1:-1], slots, heads=2)
    x = qkv.view(t, 6, dim)
    for c, v in ((kc, x[:, 2:4]), (vc, x[:, 4:])):
        flat = c[1:-1].reshape(-1, kv, dim)
        assert torch.equal(flat[4:t], v[4:]) and not bool(flat[:4].any()) and not bool(flat[t:].any())
        assert not bool(c[0].any()) and not bool(c[-1].any())


def test_append_in_place_and_beyond_448():
    t, heads, kv, dim = 9, 4, 2, 64
    g = gen(8)
    qkv = normal(g, (t, (heads + 2 * kv) * dim), BF16, 300.0)
    qkv[0, -1], qkv[1, -1] = math.inf, math.nan
    kc, vc = (torch.zeros(2, 8, kv, dim, dtype=F8, device="cuda") for _ in range(2))
    positions = torch.arange(t, dtype=torch.int32, device="cuda")
    f = torch.tensor(cfa.rotary_frequencies(dim)[0], dtype=torch.float64, device="cuda")
    want = cfa.append(qkv, kc, vc, positions, heads=heads, positions=positions, frequencies=f)
    k1, v1 = kc.clone(), vc.clone()
    own = qkv[:, :heads * dim].unflatten(1, (heads, dim))
    got = cfa.append(qkv, kc, vc, positions, heads=heads, positions=positions, frequencies=f, out=own)
    assert got is own and torch.equal(got, want)
    assert torch.equal(kc.view(torch.uint8), k1.view(torch.uint8))
    assert torch.equal(vc.view(torch.uint8), v1.view(torch.uint8))
    v = qkv.view(t, -1, dim)[:, heads + kv:].double().clamp(-448, 448)
    stored = vc.view(-1, kv, dim)[:t]
    assert stored[0, -1, -1].item() == 448.0 and bool(stored[1, -1, -1].isnan())
    fine = ~v.isnan()
    close(stored.double()[fine], v[fine], rounded(v, torch.zeros_like(v), F8)[fine])


def test_append_behind_32_bits():
    """A cache of 6 GiB: the last pages begin behind 2^32 bytes."""
    kv, dim, page = 8, 128, 16
    pages = (6 << 30) // (page * kv * dim * 2)
    kc = torch.empty(pages, page, kv, dim, dtype=BF16, device="cuda")
    vc = torch.empty(pages, page, kv, dim, dtype=BF16, device="cuda")
    kc[-2:].zero_(), vc[-2:].zero_()
    qkv = normal(gen(2), (page, 3 * kv * dim), BF16)
    slots = torch.arange((pages - 1) * page, pages * page, dtype=torch.int32, device="cuda")
    cfa.append(qkv, kc, vc, slots, heads=kv)
    x = qkv.view(page, 3, kv, dim)
    assert torch.equal(kc[-1], x[:, 1]) and torch.equal(vc[-1], x[:, 2])
    assert not bool(kc[-2].any()) and not bool(vc[-2].any())


def test_append_of_no_tokens():
    kc = torch.zeros(2, 4, 1, 64, dtype=BF16, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    q = cfa.append(torch.empty(0, 3 * 64, dtype=BF16, device="cuda"), kc, kc.clone(), none, heads=1)
    assert q.shape == (0, 1, 64)


# ---- logprobs -----------------------------------------------------------------------------------

def logprobs64(logits, tokens, top, scale):
    z = logits.double()
    z = (z - z.max(1, keepdim=True).values) * scale  # behind this 64 bits hold log sum exp beside 1e30 too
    n = logits.shape[1]
    lse = torch.logsumexp(z, 1, keepdim=True)
    p = torch.softmax(z, 1)
    given = torch.take_along_dim(z, tokens.long()[:, None], 1)[:, 0] - lse[:, 0]
    logp = z - lse
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    es = (n / 256 + 100) * 2 * U + 2.0 ** -19
    spread = z.max(1).values[:, None] - z
    spread = torch.where(torch.isfinite(spread), spread, torch.zeros_like(spread))
    e_given = es + 4 * U * (torch.take_along_dim(spread, tokens.long()[:, None], 1)[:, 0] + math.log(n))
    e_entropy = 2 * es * (1 + math.log(n)) + torch.zeros_like(entropy)
    ids = torch.sort(logits.float(), dim=1, descending=True, stable=True).indices
    ids = ids[:, :top].to(torch.int32)
    best = torch.take_along_dim(logp, ids.long(), 1)
    e_best = es + 4 * U * (torch.take_along_dim(spread, ids.long(), 1) + math.log(n))
    return (given, e_given), (entropy, e_entropy), (best, e_best), ids


def check_logprobs(logits, tokens, top, scale=1.0):
    got = cfa.logprobs(logits, tokens, top=top, scale=scale)
    given, entropy, best, ids = logprobs64(logits, tokens, top, scale)
    close(got[0], *given)
    close(got[1], *entropy)
    if top:
        assert torch.equal(got[3], ids)
        close(got[2], *best)
    else:
        assert len(got) == 2


VOCABS = [(1, 1), (2, 5), (3, 33), (1, 1000), (4, 4095), (5, 8193), (1, 32000), (7, 50257), (1, 128256),
          (80, 32000), (200, 5001), (700, 2048), (1, 262144), (3, 1000003)]


@pytest.mark.parametrize("t,v", VOCABS)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_logprobs(t, v, dtype):
    g = gen(t + v)
    logits = normal(g, (t, v), dtype, 2.5)
    tokens = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    check_logprobs(logits, tokens, min(20, v))
    check_logprobs(logits, tokens, 0, 0.7)
    check_logprobs(logits, tokens, min(32, v), 3.0)
    check_logprobs(logits, tokens, 1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lead,extra", [(1, 0), (3, 5), (8, 24)])
def test_logprobs_of_rows_apart(dtype, lead, extra):
    g = gen(lead)
    x = normal(g, (6, 5003), dtype, 2.0)
    _, view = inside(x, extra, lead, math.inf)
    tokens = torch.randint(0, 5003, (6,), generator=g, device="cuda", dtype=torch.int32)
    check_logprobs(view, tokens, 7)


@pytest.mark.parametrize("v", [40, 3001, 40000, 128256])
@pytest.mark.parametrize("t", [1, 300])
def test_logprobs_of_equal_and_ordered_logits(v, t):
    g = gen(v)
    tokens = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    up = torch.arange(v, device="cuda", dtype=F32)[None, :].expand(t, v) * (20.0 / v)
    for logits in (torch.full((t, v), 1.5, device="cuda"), up.contiguous(), up.flip(1).contiguous(),
                   (up * 3).floor(), torch.randint(0, 3, (t, v), generator=g, device="cuda").float(),
                   torch.where(torch.arange(v, device="cuda") % 2 == 0, -0.0, 0.0).expand(t, v).contiguous()):
        check_logprobs(logits, tokens, 32)
    check_logprobs((up * 3).floor().to(BF16), tokens, 20)


def test_logprobs_of_masked_logits():
    v = 5000
    logits = normal(gen(1), (6, v), F32)
    logits[0, 10:] = -math.inf        # ten left, twenty asked for
    logits[1] = -math.inf             # none
    logits[2, 77] = math.inf
    logits[3, 4999] = math.nan
    logits[4, ::2] = -math.inf
    logits[5] = 1e30
    tokens = torch.tensor([3, 3, 77, 5, 0, 4999], dtype=torch.int32, device="cuda")
    lp, ent, best, ids = cfa.logprobs(logits, tokens, top=20)
    given, entropy, ref, order = logprobs64(logits[[0, 4, 5]], tokens[[0, 4, 5]], 20, 1.0)
    close(lp[[0, 4, 5]], *given)
    close(ent[[0, 4, 5]], *entropy)
    close(best[[0, 4, 5]], *ref)
    assert torch.equal(ids[[0, 4, 5]], order)
    assert ids[0, 10:].tolist() == list(range(10, 20)) and bool((best[0, 10:] == -math.inf).all())
    assert lp[1].item() == -math.inf and ent[1].item() == 0.0
    assert bool((best[1] == -math.inf).all()) and ids[1].tolist() == list(range(20))
    assert bool(lp[2:4].isnan().all()) and bool(ent[2:4].isnan().all())
    assert bool(best[2:4].isnan().all()) and ids[2, 0].item() == 77
    assert lp[4].item() == -math.inf


def test_logprobs_of_nan_alone_and_tokens_that_are_none():
    v = 300
    logits = normal(gen(1), (5, v), F32)
    logits[4] = math.nan
    tokens = torch.tensor([-1, -(1 << 31), v, (1 << 31) - 1, 0], dtype=torch.int32, device="cuda")
    lp, ent, best, ids = cfa.logprobs(logits, tokens, top=3)
    assert lp[:2].tolist() == [0.0, 0.0] and bool(lp[2:].isnan().all())
    assert bool(ent[:4].isfinite().all()) and bool(ent[4].isnan())
    assert ids[4].tolist() == [0, 1, 2] and bool(best[4].isnan().all())


def test_logprobs_behind_32_bits():
    """Rows 2^24 apart, the last ones behind 2^32 elements."""
    rows, v = 260, 1000
    buf = torch.empty(rows << 24, dtype=BF16, device="cuda")
    view = buf.as_strided((rows, v), (1 << 24, 1))
    view.copy_(normal(gen(4), (rows, v), BF16))
    tokens = torch.arange(rows, dtype=torch.int32, device="cuda")
    check_logprobs(view, tokens, 5)


def test_logprobs_shapes():
    logits = normal(gen(2), (2, 3, 100), F32)
    tokens = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    out = cfa.logprobs(logits, tokens, top=4)
    assert [o.shape for o in out] == [(2, 3), (2, 3), (2, 3, 4), (2, 3, 4)]
    again = cfa.logprobs(logits, tokens, top=4, out=tuple(torch.empty_like(o) for o in out))
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    assert cfa.logprobs(logits[:0], tokens[:0])[0].shape == (0, 3)
    one = cfa.logprobs(logits[0, 0], tokens[0, 0])
    assert one[0].shape == () and one[0].item() == out[0][0, 0].item()


# ---- norm of many rows ----------------------------------------------------------------------------

@pytest.mark.parametrize("t,c", [(153, 1), (200, 7), (1000, 64), (1201, 130), (400, 1003), (333, 2307),
                                 (305, 8192), (700, 5121), (160, 16384), (155, 16383)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_norm_of_many_rows(t, c, dtype):
    g = gen(t + c)
    x, w, r = normal(g, (t, c), dtype), normal(g, (c,), dtype), normal(g, (t, c), dtype, 3.0)
    z, p = normal(g, (t, c), dtype), normal(g, (c,), F32)
    y64, ey, _, _ = norm64(x, w)
    close(cfa.norm(x, w), y64, ey)
    y64, ey, h64, eh = norm64(x, w.float(), r, z, "silu", p, 0.37, 1e-5, 1.0)
    y, h = cfa.norm(x, w.float(), residual=r, gate=z, post_weight=p, scale=0.37, offset=1.0, eps=1e-5)
    close(y, y64, ey)
    close(h, h64, eh)
    # with the results in the operands' places
    r2, z2 = r.clone(), z.clone()
    y2, h2 = cfa.norm(x, w.float(), residual=r2, gate=z2, post_weight=p, scale=0.37, offset=1.0, eps=1e-5,
                      out=(z2, r2))
    assert torch.equal(y2, y) and torch.equal(h2, h)
    # one gate for all
    y64, ey, _, _ = norm64(x, w, None, z[0].expand(t, c), "relu")
    close(cfa.norm(x, w, gate=z[0], activation="relu"), y64, ey)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("extras", [(0, 0, 0), (8, 8, 8), (3, 3, 3), (5, 13, 21), (1, 2, 3)])
@pytest.mark.parametrize("lead", [0, 1])
def test_norm_of_many_rows_apart(extras, lead, dtype):
    g = gen(sum(extras))
    t, c = 211, 517
    x, r, w = normal(g, (t, c), dtype), normal(g, (t, c), dtype), normal(g, (c,), dtype)
    (_, xv), (rb, rv), (yb, yv) = (inside(v, e, lead) for v, e in zip((x, r, torch.zeros_like(x)), extras))
    y, h = cfa.norm(xv, w, residual=rv, out=(yv, rv))
    y64, ey, h64, eh = norm64(x, w, r)
    close(y, y64, ey)
    close(h, h64, eh)
    for buf, e in ((rb, extras[1]), (yb, extras[2])):
        mask = torch.ones_like(buf, dtype=torch.bool)
        mask[lead:].as_strided((t, c), (c + e, 1)).fill_(False)
        assert bool((buf[mask] == 7.0).all())


@pytest.mark.parametrize("c", [16384, 16383])
def test_norm_behind_32_bits(c):
    """140,000 rows: the last ones begin behind 2^32 bytes and 2^31 elements."""
    t, g = 140000, gen(c)
    x = torch.zeros(t, c, dtype=BF16, device="cuda")
    r = torch.zeros(t, c, dtype=BF16, device="cuda")
    at = [0, 1, 65535, 131071, 131072, t - 2, t - 1]
    x[at], r[at] = normal(g, (len(at), c), BF16), normal(g, (len(at), c), BF16)
    w, r0 = normal(g, (c,), BF16), r[at].clone()
    y, h = cfa.norm(x, w, residual=r, out=(torch.empty_like(x), r))
    y64, ey, h64, eh = norm64(x[at], w, r0)
    close(y[at], y64, ey)
    close(h[at], h64, eh)
    assert not bool(y[2:65535].any()) and not bool(h[131073:t - 2].any())


def test_append_of_many_tokens():
    """Rows of q/k/v behind 2^32 bytes."""
    t, heads, kv, dim, page = 360000, 32, 8, 128, 64
    g = gen(1)
    qkv = torch.zeros(t, (heads + 2 * kv) * dim, dtype=BF16, device="cuda")
    at = torch.tensor([0, 1, 174762, 174763, 349525, t - 1], device="cuda")
    qkv[at] = normal(g, (len(at), qkv.shape[1]), BF16)
    pages = t // page
    kc, vc = (torch.empty(pages, page, kv, dim, dtype=BF16, device="cuda") for _ in range(2))
    slots = torch.arange(t, dtype=torch.int32, device="cuda").flip(0).contiguous()
    f = torch.tensor(cfa.rotary_frequencies(dim)[0], dtype=torch.float64, device="cuda")
    positions = torch.arange(t, dtype=torch.int32, device="cuda")
    q = cfa.append(qkv, kc, vc, slots, heads=heads, positions=positions, frequencies=f)
    x = qkv[at].double().view(len(at), -1, dim)
    y, e = turned64(x[:, :heads + kv], positions[at], f, False, 1.0)
    close(q[at], y[:, :heads], rounded(y[:, :heads], e[:, :heads], BF16))
    close(kc.view(-1, kv, dim)[t - 1 - at], y[:, heads:], rounded(y[:, heads:], e[:, heads:], BF16))
    assert torch.equal(vc.view(-1, kv, dim)[t - 1 - at].double(), x[:, heads + kv:])
    assert not bool(q[2:174762].any()) and not bool(kc.view(-1, kv, dim)[1:t - 1 - 349525].any())
