"""The operators on the loaded layout against plain forms in 64 bits.

Bounds are worst cases, element by element: a product's sum of K terms in fp32 is off by at most
(K + 8) 2^-23 of the sum of the terms' magnitudes (one unit in the last place of the largest partial
sum per addition, truncating or not); an activation's value by 2^-16 of its argument (exp to 100 units
in the last place) plus what the argument's error makes of it (slopes up to 1.2); the result by half
a unit in the last place of its type, and binary16's spacing near zero."""
import math

import pytest
import torch

import paper_2607_18957_gb300 as cfa

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_ULP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
NEAR_ZERO = {BF16: 0.0, F16: 2.0 ** -25, F32: 0.0}
SENTINEL = 333.0


@pytest.fixture(scope="module", autouse=True)
def cuda_device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.fixture(autouse=True)
def no_wait_ran_out(cuda_device):
    yield
    torch.cuda.synchronize()
    cfa.op_status()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def act64(v, name):
    return {"none": lambda x: x, "relu": lambda x: x.clamp(min=0),
            "silu": lambda x: x / (1 + torch.exp(-x)),
            "gelu": lambda x: 0.5 * x * (1 + torch.erf(x / math.sqrt(2))),
            "gelu_tanh": lambda x: 0.5 * x * (1 + torch.tanh(
                math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))}[name](v)


def product64(x, w):
    """x w^T in 64 bits and the bound on its error in fp32."""
    x, w = x.double(), w.double()
    return x @ w.t(), (x.abs() @ w.abs().t()) * ((x.shape[1] + 8) * 2.0 ** -23)


def activated64(v, ev, act, gated):
    """act (gated: times the other half) of values v known to ev, and the bound on it."""
    if not gated:
        if act == "none":
            return v, ev
        return act64(v, act), 1.2 * ev + 2.0 ** -16 * v.abs()
    h = v.shape[1] // 2
    a, u, eu = v[:, :h], v[:, h:], ev[:, h:]
    a, ea = activated64(a, ev[:, :h], act, False)
    return a * u, ea * u.abs() + a.abs() * eu + ea * eu + 2.0 ** -23 * (a * u).abs()


def linear64(x, w, b, act, gated, r, dtype):
    v, ev = product64(x, w)
    if b is not None:
        v = v + b.double()
        ev = ev + 2.0 ** -23 * v.abs()
    y, ey = activated64(v, ev, act, gated)
    if r is not None:
        y = y + r.double()
        ey = ey + 2.0 ** -23 * y.abs()
    return y, ey + HALF_ULP[dtype] * (y.abs() + ey) + NEAR_ZERO[dtype]


def close(got, ref, bound):
    got = got.double()
    assert got.shape == ref.shape
    assert bool(torch.isfinite(got).all())
    worst = ((got - ref).abs() - bound).max().item() if got.numel() else 0.0
    assert worst <= 0, f"off by {worst:g} more than the bound"


def inside(rows, cols, dtype, lead=0, extra=0, fill=float("nan")):
    """A [rows, cols] view of a larger buffer whose other values are `fill`: `lead` elements before
    it, row stride cols + extra, three rows after it."""
    buf = torch.full((lead + (rows + 3) * (cols + extra),), fill, dtype=dtype, device="cuda")
    return buf, buf[lead:].as_strided((rows, cols), (cols + extra, 1))


SIZES = [(1, 1, 8), (1, 128, 64), (2, 8, 4096), (3, 130, 72), (16, 96, 8), (17, 258, 1096),
         (33, 640, 264), (64, 128, 136), (100, 200, 328), (129, 384, 320), (256, 512, 512),
         (257, 1000, 520), (300, 514, 2048), (1000, 776, 1032)]


@pytest.mark.parametrize("t,n,k", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_linear(t, n, k, dtype):
    g = gen(t * 7919 + n * 31 + k)
    x, w = normal(g, (t, k), dtype), normal(g, (n, k), dtype, k ** -0.5)
    y = cfa.linear(x, w)
    assert y.dtype == dtype
    close(y, *linear64(x, w, None, "none", False, None, dtype))


@pytest.mark.parametrize("t,n,k", [(1, 34, 72), (5, 256, 136), (40, 66, 4104), (130, 300, 256),
                                   (515, 1040, 392)])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("gated", [False, True])
def test_linear_epilogue(t, n, k, act, gated):
    for dtype, bias_dtype, out in ((BF16, BF16, None), (F16, F32, None), (BF16, F32, "f32")):
        g = gen(n + k)
        x, w = normal(g, (t, k), dtype), normal(g, (n, k), dtype, 2 * k ** -0.5)
        no = n // 2 if gated else n
        b = normal(g, (n,), bias_dtype)
        r = normal(g, (t, no), F32 if out else dtype)
        y = cfa.linear(x, w, b, activation=act, gated=gated, residual=r, out_dtype=out)
        close(y, *linear64(x, w, b, act, gated, r, y.dtype))


@pytest.mark.parametrize("t,n,k,gated,act,out", [
    (171, 11200, 648, False, "none", None), (161, 10104, 784, False, "gelu", None),
    (161, 5440, 648, True, "silu", None), (197, 5064, 792, True, "gelu_tanh", None),
    (162, 11033, 720, False, "relu", None), (172, 5433, 680, True, "silu", None),
    (900, 6359, 392, False, "gelu_tanh", None), (900, 6362, 392, False, "silu", None),
    (2372, 904, 2560, False, "none", "f32"), (4808, 448, 2832, False, "gelu_tanh", "f32"),
    (4747, 196, 2248, True, "silu", "f32"), (4767, 386, 2544, False, "relu", "f32"),
    (4787, 462, 3104, False, "gelu", "f32"), (4821, 230, 2264, True, "silu", "f32"),
    (2438, 8, 32, False, "none", "f32"), (5, 5000, 32, False, "gelu", "f32"),
    (17, 16, 144, True, "gelu", None), (7, 18, 144, True, "silu", None)])
def test_linear_of_every_kind_of_tile(t, n, k, gated, act, out):
    """Tiles of one SM and of two, results of 2 and of 4 bytes on the 16-byte grid, off it and between
    words; n columns of results."""
    dtype = F16 if n % 3 else BF16
    g = gen(t + n + k)
    x = normal(g, (t, k), dtype)
    w = normal(g, (2 * n if gated else n, k), dtype, k ** -0.5)
    b = normal(g, (w.shape[0],), dtype)
    odt = F32 if out else dtype
    r = normal(g, (t, n), odt)
    for residual in (None, r):
        buf, y = inside(t, n, odt)
        assert cfa.linear(x, w, b, activation=act, gated=gated, residual=residual, out=y) is y
        close(y, *linear64(x, w, b, act, gated, residual, odt))
        assert bool(torch.isnan(buf[t * n:]).all())


@pytest.mark.parametrize("t,n,k", [(3, 16, 128), (70, 144, 128), (300, 2000, 320), (5, 24, 64),
                                   (9, 14, 192), (200, 310, 256), (600, 1030, 128), (2, 2, 64),
                                   (40, 6, 72)])
def test_linear_gated_rows_that_do_not_fill_their_tiles(t, n, k):
    """Halves of whole groups of 8 rows and others, whole blocks of 64 columns and others."""
    g = gen(n * 3 + k)
    x, w = normal(g, (t, k), F16), normal(g, (n, k), F16, k ** -0.5)
    close(cfa.linear(x, w, activation="silu", gated=True),
          *linear64(x, w, None, "silu", True, None, F16))


@pytest.mark.parametrize("t,n,k", [(1, 5, 3), (5, 33, 7), (19, 130, 1001), (150, 64, 250)])
def test_linear_columns_off_the_grid(t, n, k):
    g = gen(k)
    x, w = normal(g, (t, k), BF16), normal(g, (n, k), BF16, k ** -0.5)
    close(cfa.linear(x, w), *linear64(x, w, None, "none", False, None, BF16))


@pytest.mark.parametrize("gated", [False, True])
def test_linear_moves_a_large_weight_in_slices(gated):
    """Rows of 8003 elements start at every 2-byte phase; 6000 of them are more than one slice."""
    g = gen(21)
    t, n, k = 3, 6000, 8003
    x, w = normal(g, (t, k), BF16), normal(g, (n, k), BF16, k ** -0.5)
    b = normal(g, (n,), BF16)
    r = normal(g, (t, n // 2 if gated else n), BF16)
    y = cfa.linear(x, w, b, activation="silu", gated=gated, residual=r)
    close(y, *linear64(x, w, b, "silu", gated, r, BF16))


@pytest.mark.parametrize("t,n,k", [(3, 200, 4096), (64, 8, 14336), (200, 260, 4096), (33, 64, 1000)])
def test_fp32_results_are_rounded_as_fp32(t, n, k):
    """Parts of 256 columns, 16 truncated additions of at most 2^-23 of the partial sum each, then one
    rounding per part: far inside the bound of K of them."""
    g = gen(k)
    x, w = normal(g, (t, k), BF16), normal(g, (n, k), BF16, k ** -0.5)
    y = cfa.linear(x, w, out_dtype="f32")
    ref = x.double() @ w.double().t()
    size = x.double().abs() @ w.double().abs().t()
    adds = 16 + 2 + k // 256
    assert bool(((y.double() - ref).abs() <= adds * 2.0 ** -23 * size).all())
    assert ((y.double() - ref).norm() / ref.norm()).item() < 1e-6


@pytest.mark.parametrize("lead,extra", [(0, 0), (8, 8), (8, 24), (1, 0), (0, 1), (3, 13), (4, 4)])
@pytest.mark.parametrize("gated", [False, True])
def test_linear_inside_larger_buffers(lead, extra, gated):
    """NaN all around the operands must not be read into the result, and nothing around the result
    may be written."""
    g = gen(lead * 100 + extra)
    t, n, k = 37, 268, 200
    no = n // 2 if gated else n
    _, x = inside(t, k, BF16, lead, extra)
    _, w = inside(n, k, BF16, lead, extra)
    _, r = inside(t, no, BF16, lead, extra)
    ybuf, y = inside(t, no, BF16, lead, extra, SENTINEL)
    x.copy_(normal(g, (t, k), BF16))
    w.copy_(normal(g, (n, k), BF16, k ** -0.5))
    r.copy_(normal(g, (t, no), BF16))
    out = cfa.linear(x, w, activation="silu", gated=gated, residual=r, out=y)
    assert out is y
    close(y, *linear64(x, w, None, "silu", gated, r, BF16))
    y.fill_(SENTINEL)
    assert bool((ybuf == SENTINEL).all())


def test_linear_adds_in_place_and_keeps_leading_dimensions():
    g = gen(3)
    x, w = normal(g, (2, 3, 264), BF16), normal(g, (136, 264), BF16, 0.1)
    r = normal(g, (2, 3, 136), BF16)
    want = linear64(x.view(6, 264), w, None, "relu", False, r.clone().view(6, 136), BF16)
    y = cfa.linear(x, w, activation="relu", residual=r, out=r)
    assert y is r and y.shape == (2, 3, 136)
    close(y.view(6, 136), *want)


def test_linear_of_no_tokens():
    w = normal(gen(1), (16, 8), BF16)
    assert cfa.linear(torch.empty(0, 8, dtype=BF16, device="cuda"), w).shape == (0, 16)


def test_linear_repeats_bit_for_bit_and_on_other_streams():
    g = gen(9)
    x, w = normal(g, (19, 4096), BF16), normal(g, (520, 4096), BF16, 0.02)
    y = cfa.linear(x, w, out_dtype="f32")
    for _ in range(3):
        assert torch.equal(cfa.linear(x, w, out_dtype="f32"), y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = cfa.linear(x, w, out_dtype="f32", stream=side)
    b = cfa.linear(x, w, out_dtype="f32", stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(a, y) and torch.equal(b, y)


def test_linear_carries_infinities_and_nan_to_their_rows_alone():
    g = gen(4)
    x, w = normal(g, (20, 256), BF16), normal(g, (160, 256), BF16, 0.1)
    clean = cfa.linear(x, w)
    x[3, 5] = math.inf
    x[7, 250] = math.nan
    y = cfa.linear(x, w)
    rows = torch.ones(20, dtype=torch.bool, device="cuda")
    rows[[3, 7]] = False
    assert torch.equal(y[rows], clean[rows])
    assert bool(torch.isnan(y[7]).all())
    assert torch.equal(y[3].double(), torch.where(w[:, 5] > 0, math.inf, -math.inf).double())


def test_linear_in_a_graph():
    g = gen(11)
    x, w = normal(g, (5, 512), BF16), normal(g, (256, 512), BF16, 0.05)
    y = cfa.linear(x, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = cfa.linear(x, w)
    x.copy_(normal(g, (5, 512), BF16))
    graph.replay()
    assert torch.equal(z, cfa.linear(x, w)) and not torch.equal(z, y)


# ---- route --------------------------------------------------------------------------------------

def route64(logits, top_k, scoring, bias, groups, top_groups, renormalize, scale):
    """Token by token from the definition, in 64 bits."""
    out_w, out_i = [], []
    for row in logits.double().cpu().tolist():
        if scoring == "softmax":
            top = max(row)
            ex = [math.exp(v - top) if v > -math.inf else 0.0 for v in row]
            norm = sum(ex)
            score = [v / norm if norm else 0.0 for v in ex]
            key = list(row) if bias is None else [s + b for s, b in zip(score, bias)]
        else:
            score = [1 / (1 + math.exp(-v)) if v > -700 else 0.0 for v in row]
            key = score if bias is None else [s + b for s, b in zip(score, bias)]
        key = [k if v > -math.inf else -math.inf for k, v in zip(key, row)]
        size = len(row) // groups
        best = []
        for q in range(groups):
            part = sorted(key[q * size:(q + 1) * size], reverse=True)
            best.append(part[0] if scoring == "softmax" or size == 1 else part[0] + part[1])
        kept = sorted(range(groups), key=lambda q: (-best[q], q))[:top_groups]
        order = sorted((e for e in range(len(row)) if e // size in kept and key[e] > -math.inf),
                       key=lambda e: (-key[e], e))[:top_k]
        w = [score[e] for e in order]
        if renormalize and order:
            if scoring == "softmax":
                m = max(row[e] for e in order)
                w = [math.exp(row[e] - m) for e in order]
            total = sum(w)
            w = [v / total if total else 0.0 for v in w]
        pad = top_k - len(order)
        out_i.append(order + [-1] * pad)
        out_w.append([v * scale for v in w] + [0.0] * pad)
    return torch.tensor(out_w, dtype=torch.float64), torch.tensor(out_i, dtype=torch.int32)


def spread_logits(t, e, dtype, seed):
    """Logits on a grid of eighths: equal ones tie exactly and different ones stay apart."""
    g = gen(seed)
    return (torch.randint(-32, 33, (t, e), generator=g, device="cuda") / 8).to(dtype)


def check_route(logits, top_k, **kw):
    full = dict(scoring="softmax", bias=None, groups=1, top_groups=1, renormalize=True, scale=1.0)
    full.update(kw)
    w, i = cfa.route(logits, top_k, **full)
    b = full["bias"]
    full["bias"] = None if b is None else b.double().cpu().tolist()
    rw, ri = route64(logits, top_k, **full)
    assert i.dtype == torch.int32 and w.dtype == F32
    assert torch.equal(i.cpu(), ri)
    # exp and its sum to a few units in the last place each
    assert torch.allclose(w.cpu().double(), rw, rtol=2.0 ** -19, atol=1e-30)


@pytest.mark.parametrize("e,top_k", [(1, 1), (2, 1), (8, 2), (31, 31), (33, 7), (60, 4), (64, 6),
                                     (128, 8), (160, 6), (257, 8), (512, 32), (1024, 8)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route(e, top_k, dtype, scoring):
    for t, renormalize in ((1, True), (77, False)):
        check_route(spread_logits(t, e, dtype, e + t), top_k, scoring=scoring,
                    renormalize=renormalize, scale=1.0 if renormalize else 2.5)


@pytest.mark.parametrize("e,groups,top_groups,top_k", [(8, 8, 3, 2), (16, 4, 2, 3), (64, 8, 4, 8),
                                                       (256, 8, 4, 8), (96, 32, 5, 8),
                                                       (1024, 2, 1, 32)])
@pytest.mark.parametrize("scoring,bias", [("softmax", False), ("sigmoid", False), ("sigmoid", True),
                                          ("softmax", True)])
def test_route_groups_and_bias(e, groups, top_groups, top_k, scoring, bias):
    g = gen(e)
    # a bias on a grid of its own keeps the sums apart
    b = torch.randint(-64, 65, (e,), generator=g, device="cuda").float() / 16 if bias else None
    check_route(spread_logits(50, e, F32, e + 1), top_k, scoring=scoring, bias=b, groups=groups,
                top_groups=top_groups)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_masked_logits(scoring):
    z = spread_logits(6, 16, F32, 2)
    z[0] = -math.inf                       # nothing left
    z[1, 3:] = -math.inf                   # fewer than top_k
    z[2, ::2] = torch.finfo(F32).min       # the lowest value is a value
    z[3] = torch.finfo(F32).min
    z[4] = 2.0                             # all tie
    check_route(z, 4, scoring=scoring)
    check_route(z[:, :15], 4, scoring=scoring, renormalize=False)
    check_route(z, 4, scoring=scoring, groups=4, top_groups=2)


def test_route_nan_and_infinite_logits():
    z = spread_logits(3, 8, F32, 5)
    z[0, 2] = math.nan
    z[1, 4] = math.inf
    w, i = cfa.route(z, 2)
    assert 2 not in i[0].tolist() and bool(torch.isnan(w[0]).all())
    assert i[1, 0].item() == 4 and bool(torch.isnan(w[1]).all())
    check_route(z[2:], 2)
    w, i = cfa.route(z, 2, scoring="sigmoid", renormalize=False)
    assert 2 not in i[0].tolist() and bool(torch.isfinite(w).all())
    assert i[1, 0].item() == 4 and w[1, 0].item() == 1.0
    w, i = cfa.route(z, 2, bias=torch.zeros(8, device="cuda"))
    assert i[0].tolist() == [-1, -1] and w[0].tolist() == [0.0, 0.0]


def test_route_rows_apart_and_given_outputs():
    buf, z = inside(9, 12, BF16, 3, 5)
    z.copy_(spread_logits(9, 12, BF16, 8))
    w = torch.empty(9, 3, device="cuda")
    i = torch.empty(9, 3, dtype=torch.int32, device="cuda")
    a, b = cfa.route(z, 3, out=(w, i))
    assert a is w and b is i
    rw, ri = route64(z, 3, "softmax", None, 1, 1, True, 1.0)
    assert torch.equal(i.cpu(), ri) and torch.allclose(w.cpu().double(), rw, rtol=2.0 ** -19)
    assert cfa.route(z[:0], 3)[1].shape == (0, 3)


# ---- experts ------------------------------------------------------------------------------------

def experts64(x, ids, weights, w13, w2, act, first, residual):
    dtype = x.dtype
    e, h, i = w2.shape
    gated = w13.shape[1] == 2 * i
    y = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    ey = torch.zeros_like(y)
    size = torch.zeros_like(y)
    for k in range(e):
        tok, j = torch.where(ids == first + k)
        if not tok.numel():
            continue
        v, ev = product64(x[tok], w13[k])
        a, ea = activated64(v, ev, act, gated)
        ea = ea + HALF_ULP[dtype] * (a.abs() + ea) + NEAR_ZERO[dtype]
        o = a @ w2[k].double().t()
        eo = ea @ w2[k].double().abs().t()
        eo += (a.abs() + ea) @ w2[k].double().abs().t() * ((i + 8) * 2.0 ** -23)
        g = weights[tok, j].double()[:, None]
        y.index_add_(0, tok, o * g)
        ey.index_add_(0, tok, eo * g.abs())
        size.index_add_(0, tok, (o * g).abs())
    if residual is not None:
        y = y + residual.double()
        size = size + residual.double().abs()
    ey = ey + size * ((ids.shape[1] + 2) * 2.0 ** -23)
    return y, ey + HALF_ULP[dtype] * (y.abs() + ey) + NEAR_ZERO[dtype]


def expert_operands(t, h, i, e, top_k, all_e, dtype, seed, gated=True):
    g = gen(seed)
    x = normal(g, (t, h), dtype)
    w13 = normal(g, (e, 2 * i if gated else i, h), dtype, h ** -0.5)
    w2 = normal(g, (e, h, i), dtype, i ** -0.5)
    top, ids = torch.randn(t, all_e, generator=g, device="cuda").topk(top_k, dim=1)
    return x, ids.to(torch.int32), torch.softmax(top, dim=1), w13, w2


@pytest.mark.parametrize("t", [1, 2, 5, 33, 200, 700])
@pytest.mark.parametrize("h,i,e,top_k", [(256, 128, 8, 2), (72, 40, 4, 1), (520, 264, 60, 6),
                                         (1024, 768, 3, 3), (128, 8, 1, 1)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_experts(t, h, i, e, top_k, dtype):
    x, ids, w, w13, w2 = expert_operands(t, h, i, e, top_k, e, dtype, t + h + e)
    y = cfa.experts(x, ids, w, w13, w2)
    close(y, *experts64(x, ids, w, w13, w2, "silu", 0, None))


@pytest.mark.parametrize("t,h,i,e,top_k", [(1300, 624, 480, 48, 2), (900, 1000, 416, 6, 3)])
def test_experts_of_many_tokens_each(t, h, i, e, top_k):
    x, ids, w, w13, w2 = expert_operands(t, h, i, e, top_k, e, BF16, t + h)
    r = normal(gen(t), (t, h), BF16)
    y = cfa.experts(x, ids, w, w13, w2, residual=r)
    close(y, *experts64(x, ids, w, w13, w2, "silu", 0, r))


@pytest.mark.parametrize("t", [1, 70, 3000])
@pytest.mark.parametrize("gated,act", [(True, "gelu_tanh"), (False, "relu")])
def test_experts_of_one_rank(t, gated, act):
    """Experts 8 .. 15 of 32: the other choices add nothing, whatever their weights and ids."""
    x, ids, w, w13, w2 = expert_operands(t, 264, 96, 8, 4, 32, BF16, t, gated)
    r = normal(gen(t + 1), (t, 264), BF16)
    here = (ids >= 8) & (ids < 16)
    want = experts64(x, ids, w, w13, w2, act, 8, r)
    w = torch.where(here, w, math.nan)
    ids = torch.where(ids == 3, -1, torch.where(ids == 4, 2 ** 31 - 1,
                                                torch.where(ids == 5, -2 ** 31, ids)))
    y = cfa.experts(x, ids.int(), w, w13, w2, activation=act, first_expert=8, residual=r)
    close(y, *want)
    assert torch.equal(y[~here.any(dim=1)], r[~here.any(dim=1)])


def test_experts_all_on_one_none_and_twice():
    x, ids, w, w13, w2 = expert_operands(300, 128, 72, 5, 2, 5, BF16, 7)
    ids.fill_(3)
    w13[[0, 1, 2, 4]] = math.nan  # experts without tokens are not read into anything
    w2[[0, 1, 2, 4]] = math.nan
    close(cfa.experts(x, ids, w, w13, w2),
          *experts64(x, ids, w, w13, w2, "silu", 0, None))
    ids.fill_(-1)
    assert bool((cfa.experts(x, ids, w, w13, w2) == 0).all())
    assert cfa.experts(x[:0], ids[:0], w[:0], w13, w2).shape == (0, 128)


def test_experts_keep_bad_tokens_to_themselves():
    x, ids, w, w13, w2 = expert_operands(64, 256, 128, 4, 2, 4, BF16, 8)
    clean = cfa.experts(x, ids, w, w13, w2)
    x[10] = math.nan
    x[20, 0] = math.inf
    y = cfa.experts(x, ids, w, w13, w2)
    rows = torch.ones(64, dtype=torch.bool, device="cuda")
    rows[[10, 20]] = False
    assert torch.equal(y[rows], clean[rows])
    assert bool(torch.isnan(y[10]).all()) and not bool(torch.isfinite(y[20]).any())


@pytest.mark.parametrize("lead,extra", [(0, 8), (1, 0), (8, 3)])
def test_experts_inside_larger_buffers(lead, extra):
    x, ids, w, w13, w2 = expert_operands(21, 136, 56, 6, 2, 6, F16, 12)
    _, xv = inside(21, 136, F16, lead, extra)
    _, rv = inside(21, 136, F16, lead, extra)
    ybuf, yv = inside(21, 136, F16, lead, extra, SENTINEL)
    xv.copy_(x)
    rv.copy_(normal(gen(1), (21, 136), F16))
    need = 1 << 20
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN everywhere
    cfa.experts(xv, ids, w, w13, w2, residual=rv, out=yv, workspace=ws)
    close(yv, *experts64(x, ids, w, w13, w2, "silu", 0, rv))
    yv.fill_(SENTINEL)
    assert bool((ybuf == SENTINEL).all())


def test_experts_repeat_bit_for_bit_in_place_and_in_a_graph():
    x, ids, w, w13, w2 = expert_operands(130, 512, 256, 16, 4, 16, BF16, 13)
    y = cfa.experts(x, ids, w, w13, w2)
    for _ in range(3):
        assert torch.equal(cfa.experts(x, ids, w, w13, w2), y)
    r = normal(gen(2), (130, 512), BF16)
    want = cfa.experts(x, ids, w, w13, w2, residual=r)
    acc = r.clone()
    assert torch.equal(cfa.experts(x, ids, w, w13, w2, residual=acc, out=acc), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = cfa.experts(x, ids, w, w13, w2)
    ids.copy_(ids.flip(0))
    graph.replay()
    assert torch.equal(z, cfa.experts(x, ids, w, w13, w2))


@pytest.mark.parametrize("t,e,top_k", [(5000, 4, 4), (4100, 16, 8), (300, 1024, 8)])
def test_experts_of_many_pairs_and_of_many_experts(t, e, top_k):
    """More pairs than one block of the sort counts for itself, and the most experts there can be."""
    x, ids, w, w13, w2 = expert_operands(t, 64, 32, e, top_k, e, BF16, t + e)
    close(cfa.experts(x, ids, w, w13, w2), *experts64(x, ids, w, w13, w2, "silu", 0, None))


def test_offsets_past_32_bits():
    """A result and stacked weights of more than 2^31 elements."""
    g = gen(31)
    x, w = normal(g, (65600, 64), BF16), normal(g, (32800, 64), BF16, 0.125)
    y = cfa.linear(x, w)
    for rows in (slice(0, 40), slice(65472, 65600)):
        close(y[rows], *linear64(x[rows], w, None, "none", False, None, BF16))
    del y
    w13 = torch.empty(20, 28672, 4096, dtype=BF16, device="cuda")  # the others are never read
    w2 = torch.empty(20, 4096, 14336, dtype=BF16, device="cuda")
    w13[19] = normal(g, (28672, 4096), BF16, 4096 ** -0.5)
    w2[19] = normal(g, (4096, 14336), BF16, 14336 ** -0.5)
    x = normal(g, (9, 4096), BF16)
    ids = torch.full((9, 1), 19, dtype=torch.int32, device="cuda")
    weights = torch.rand(9, 1, generator=g, device="cuda")
    close(cfa.experts(x, ids, weights, w13, w2),
          *experts64(x, ids - 19, weights, w13[19:], w2[19:], "silu", 0, None))


def test_a_wait_that_runs_out_ends_and_is_reported():
    import ctypes
    from paper_2607_18957_gb300 import _lib
    word = ctypes.c_int(-1)
    assert _lib.load().cfa_selftest_op_timeout(-1, ctypes.byref(word)) == 0
    assert word.value == 1
    cfa.op_status()  # cleared
    x = normal(gen(1), (3, 64), BF16)  # and the context is as usable as before
    close(cfa.linear(x, x), *linear64(x, x, None, "none", False, None, BF16))


# ---- refusals -----------------------------------------------------------------------------------

def test_python_refusals():
    x = torch.zeros(4, 64, dtype=BF16, device="cuda")
    w = torch.zeros(32, 64, dtype=BF16, device="cuda")
    for bad in (lambda: cfa.linear(x, w[:, :32]),
                lambda: cfa.linear(x, w.half()),
                lambda: cfa.linear(x, w.cpu()),
                lambda: cfa.linear(x.cpu(), w.cpu()),
                lambda: cfa.linear(x, w.t()[:32, :32].t()),
                lambda: cfa.linear(x, w, torch.zeros(31, device="cuda")),
                lambda: cfa.linear(x, w, activation="swish"),
                lambda: cfa.linear(x, w[:31], gated=True),
                lambda: cfa.linear(x, w, residual=torch.zeros(4, 31, dtype=BF16, device="cuda")),
                lambda: cfa.linear(x, w, residual=torch.zeros(4, 32, device="cuda")),
                lambda: cfa.linear(x, w, out=torch.zeros(3, 32, dtype=BF16, device="cuda")),
                lambda: cfa.linear(x.clone().requires_grad_(), w),
                lambda: cfa.route(x, 2, scoring="relu"),
                lambda: cfa.route(x, 2, bias=torch.zeros(63, device="cuda")),
                lambda: cfa.route(x, 0),
                lambda: cfa.route(x.double(), 2)):
        with pytest.raises(ValueError):
            bad()
    for bad, name in ((lambda: cfa.linear(x, w, out=x[:, :32]), "CFA_ERR_OVERLAP"),
                      (lambda: cfa.linear(x.float(), w.float()), "CFA_ERR_DTYPE"),
                      (lambda: cfa.linear(x[:1].expand(4, 64), w), "CFA_ERR_INVAL"),
                      (lambda: cfa.linear(x, w, out=torch.zeros(4, 32, dtype=F16,
                                                                device="cuda")), "CFA_ERR_DTYPE"),
                      (lambda: cfa.route(x, 65), "CFA_ERR_INVAL"),
                      (lambda: cfa.route(x, 2, groups=3), "CFA_ERR_INVAL"),
                      (lambda: cfa.route(x, 2, groups=4, top_groups=5), "CFA_ERR_INVAL")):
        with pytest.raises(cfa.CfaError) as err:
            bad()
        assert err.value.name == name


def test_python_refusals_of_experts():
    x, ids, w, w13, w2 = expert_operands(4, 64, 32, 4, 2, 4, BF16, 1)
    for bad in (lambda: cfa.experts(x, ids.long(), w, w13, w2),
                lambda: cfa.experts(x, ids, w.half(), w13, w2),
                lambda: cfa.experts(x, ids, w[:3], w13, w2),
                lambda: cfa.experts(x, ids, w, w13[:, :40], w2),
                lambda: cfa.experts(x, ids, w, w13.half(), w2),
                lambda: cfa.experts(x, ids, w, w13, w2.transpose(1, 2)),
                lambda: cfa.experts(x[:, :32], ids, w, w13, w2),
                lambda: cfa.experts(x, ids, w, w13, w2, activation="gate"),
                lambda: cfa.experts(x, ids, w, w13, w2, residual=x[:3])):
        with pytest.raises(ValueError):
            bad()
    for bad, name in ((lambda: cfa.experts(x, ids, w, w13, w2, out=x), "CFA_ERR_OVERLAP"),
                      (lambda: cfa.experts(x, ids, w, w13, w2, workspace=torch.empty(
                          100, dtype=torch.uint8, device="cuda")), "CFA_ERR_INVAL"),
                      (lambda: cfa.experts(x, ids, w, w13, w2, first_expert=-1), "CFA_ERR_INVAL")):
        with pytest.raises(cfa.CfaError) as err:
            bad()
        assert err.value.name == name


# ---- the example --------------------------------------------------------------------------------

def test_example_loads_a_layer_and_runs_it():
    from examples import moe_layer
    for tokens in (1, 96):
        got, want = moe_layer.run(tokens=tokens, hidden=512, inter=704, experts=8)
        for name in want:
            err = (got[name].double() - want[name]).norm() / want[name].norm()
            assert err < 2.0 ** -7, (name, err.item())
