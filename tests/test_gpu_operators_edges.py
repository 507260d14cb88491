"""Edges of the operators on the loaded layout: many tokens with fp32 results, SiLU where exp(-v) leaves
fp32, groups of experts of which some cannot be chosen, threads that ask for waits that ran out."""
import ctypes
import math
import threading

import pytest
import torch

import paper_2607_18957_gb300 as cfa

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


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


def normal(seed, shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("t", [16256, 16257, 20000, 65536])
@pytest.mark.parametrize("n,k", [(8, 320), (200, 72)])
@pytest.mark.parametrize("gated", [False, True])
def test_fp32_results_of_many_tokens(t, n, k, gated):
    """A product's sum of K terms in fp32 is off by at most (K + 8) 2^-23 of the sum of the terms'
    magnitudes, relu by no more, a gated product by what the errors of its factors make of it, and
    the rounding to fp32 by 2^-24."""
    x, w = normal(t, (t, k), BF16), normal(n, (2 * n if gated else n, k), BF16, k ** -0.5)
    y = cfa.linear(x, w, activation="relu", gated=gated, out_dtype="f32")
    v = x.double() @ w.double().t()
    ev = (x.double().abs() @ w.double().abs().t()) * ((k + 8) * 2.0 ** -23)
    ref, bound = v.clamp(min=0), ev
    if gated:
        a, u, ea, eu = ref[:, :n], v[:, n:], ev[:, :n], ev[:, n:]
        ref, bound = a * u, ea * u.abs() + a * eu + ea * eu
    bound = bound + 2.0 ** -23 * (ref.abs() + bound)
    assert y.dtype == F32 and y.shape == (t, n)
    worst = ((y.double() - ref).abs() - bound).max().item()
    assert worst <= 0, f"off by {worst:g} more than the bound"


@pytest.mark.parametrize("t", [1, 40, 300])
@pytest.mark.parametrize("dtype,out", [(BF16, "f32"), (F16, "f32"), (BF16, None)])
@pytest.mark.parametrize("gated", [False, True])
def test_silu_of_arguments_far_below_zero(t, dtype, out, gated):
    """-77, -77.5, .. -88.5, where exp(-v) is just inside fp32 and the value a normal number of fp32
    and bf16.  The exponential is off by two units in the last place for fp32 results and by 2 + 1.173
    |v| for others, the sum by half a unit, the quotient by two; bf16's rounding by 2^-8."""
    v = -77.0 - 0.5 * torch.arange(24, device="cuda")
    x = torch.zeros(t, 16, dtype=dtype, device="cuda")
    x[:, 3] = 1.0
    w = torch.zeros(48 if gated else 24, 16, dtype=dtype, device="cuda")
    w[:24, 3] = v.to(dtype)
    if gated:
        w[24:, 3] = 1.0
    assert torch.equal(w[:24, 3].float(), v)
    y = cfa.linear(x, w, activation="silu", gated=gated, out_dtype=out).double()
    ref = (v.double() / (1 + torch.exp(-v.double()))).expand(t, 24)
    units = 5 if out else 5 + 1.173 * 88.5
    assert bool(((y - ref).abs() <= (units * 2.0 ** -23 + (0 if out else 2.0 ** -8)) * ref.abs()).all())


# ---- groups of experts --------------------------------------------------------------------------

def route_row(row, bias, top_k, scoring, groups, top_groups):
    """(ids, weights, margin) of one token from the definition, in 64 bits; margin: how far apart the
    closest two groups and the closest two keys lie that are told apart."""
    n, size = len(row), len(row) // groups
    top = max(row)
    if scoring == "softmax":
        norm = sum(math.exp(v - top) for v in row) if top > -math.inf else 1.0
        score = [math.exp(v - top) / norm if v > -math.inf else 0.0 for v in row]
    else:
        score = [1 / (1 + math.exp(-v)) if v > -math.inf else 0.0 for v in row]
    key = row if bias is None and scoring == "softmax" else [
        s + (0.0 if bias is None else b) for s, b in zip(score, bias or score)]
    free = [v > -math.inf and k == k and k > -math.inf for v, k in zip(row, key)]
    rank = []
    for q in range(groups):
        left = sorted((key[e] for e in range(q * size, (q + 1) * size) if free[e]), reverse=True)
        count = 2 if scoring == "sigmoid" else 1
        rank.append(sum(left[:count]) if left else -math.inf)
    order = sorted(range(groups), key=lambda q: (-rank[q], q))
    kept, margin = order[:top_groups], math.inf
    if top_groups < groups and rank[order[top_groups]] > -math.inf:
        margin = rank[order[top_groups - 1]] - rank[order[top_groups]]
    left = sorted((e for e in range(n) if free[e] and e // size in kept), key=lambda e: (-key[e], e))
    for a, b in zip(left[:top_k], left[1:]):
        margin = min(margin, key[a] - key[b])
    ids = left[:top_k]
    w = [score[e] for e in ids]
    if scoring == "softmax":
        w = [math.exp(row[e] - max(row[i] for i in ids)) for e in ids]
    total = sum(w)
    w = [v / total if total else 0.0 for v in w]
    pad = top_k - len(ids)
    return ids + [-1] * pad, w + [0.0] * pad, margin


def check_groups(z, top_k, scoring, bias, groups, top_groups):
    """Keys without a bias are fp32 values below 1, at most three units of 2^-24 off, their sums seven:
    choices that are 2^-20 apart have to be the definition's, and with a bias (below 4) those 2^-18 apart."""
    near = 2.0 ** -20 if bias is None else 2.0 ** -18
    w, i = cfa.route(z, top_k, scoring=scoring, bias=bias, groups=groups, top_groups=top_groups)
    b = None if bias is None else bias.double().cpu().tolist()
    clear = 0
    for row, gi, gw in zip(z.double().cpu().tolist(), i.cpu().tolist(), w.cpu().tolist()):
        ids, weights, margin = route_row(row, b, top_k, scoring, groups, top_groups)
        if margin < near:
            continue
        clear += 1
        assert gi == ids
        assert all(abs(x - y) <= 2.0 ** -19 * y for x, y in zip(gw, weights))
    assert clear >= 0.75 * z.shape[0]


def masked(z, groups, how, seed):
    t, e = z.shape
    part = z.view(t, groups, e // groups)
    r = torch.rand(part.shape, generator=torch.Generator(device="cuda").manual_seed(seed),
                   device="cuda")
    rank = r.argsort(dim=2).argsort(dim=2)
    if how == "one of each":
        part[rank == 0] = -math.inf
    elif how == "all but one":
        part[rank != 0] = -math.inf
    elif how == "a group":
        part[torch.arange(t), torch.arange(t) % groups] = -math.inf
    elif how == "half":
        part[r < 0.5] = -math.inf
    elif how == "nearly all":
        part[r < 0.95] = -math.inf
    return z


GROUPS = [(8, 4, 2, 2), (16, 4, 2, 3), (64, 8, 4, 8), (60, 4, 2, 6), (96, 32, 5, 8), (256, 8, 4, 8),
          (1024, 2, 1, 32)]
HOW = ["none", "one of each", "all but one", "a group", "half", "nearly all"]


@pytest.mark.parametrize("e,groups,top_groups,top_k", GROUPS)
@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("scoring,biased", [("softmax", False), ("sigmoid", False),
                                            ("sigmoid", True), ("softmax", True)])
def test_groups_with_masked_experts(e, groups, top_groups, top_k, how, scoring, biased):
    z = masked(normal(e, (40, e), F32, 1.5), groups, how, e + 1)
    bias = normal(e + 2, (e,), F32, 0.3) if biased else None
    check_groups(z, top_k, scoring, bias, groups, top_groups)


def test_a_masked_expert_leaves_its_group_its_rank():
    z = torch.tensor([[5.0, -math.inf, -3.0, -3.0]], device="cuda")
    w, i = cfa.route(z, 1, scoring="sigmoid", groups=2, top_groups=1)
    assert i.tolist() == [[0]] and w.tolist() == [[1.0]]
    z = torch.tensor([[-math.inf, -math.inf, -3.0, -math.inf]], device="cuda")
    bias = torch.tensor([4.0, 4.0, -2.0, 4.0], device="cuda")  # of experts that cannot be chosen
    w, i = cfa.route(z, 1, scoring="sigmoid", bias=bias, groups=2, top_groups=1)
    assert i.tolist() == [[2]] and w.tolist() == [[1.0]]


@pytest.mark.parametrize("e,groups,top_groups,top_k", GROUPS)
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("what", [math.nan, -math.inf])
def test_groups_with_a_bias_that_takes_experts_out(e, groups, top_groups, top_k, scoring, what):
    bias = normal(e + 3, (e,), F32, 0.3)
    bias[::5] = what
    check_groups(normal(e, (40, e), F32, 1.5), top_k, scoring, bias, groups, top_groups)


@pytest.mark.parametrize("size", [2, 3, 4, 8, 16])
def test_a_nan_in_the_bias_does_not_count_its_group_twice(size):
    """Two groups; the first has one key of 0.6 and NaN, the second two keys of 0.4: 0.6 < 0.8, whatever
    place the NaN has."""
    for at in range(1, size):
        z = torch.full((1, 2 * size), -30.0, device="cuda")
        z[0, 0] = math.log(0.6 / 0.4)
        z[0, size:size + 2] = -math.log(0.6 / 0.4)
        bias = torch.zeros(2 * size, device="cuda")
        bias[at] = math.nan
        for pad in (1, 8, 16):  # groups without a chance, so that a lane holds several keys
            zz = torch.cat([z, torch.full((1, 2 * size * (pad - 1)), -30.0, device="cuda")], dim=1)
            bb = torch.cat([bias, torch.zeros(2 * size * (pad - 1), device="cuda")])
            w, i = cfa.route(zz, 1, scoring="sigmoid", bias=bb, groups=2 * pad, top_groups=1)
            assert i.tolist() == [[size]] and w.tolist() == [[1.0]]


# ---- waits that ran out -------------------------------------------------------------------------

def test_a_thread_that_asks_takes_nothing_from_another():
    """The self-test's waits run out (and end) in one thread while another asks all the time: the first
    is told of them every time and the other never."""
    from paper_2607_18957_gb300 import _lib
    lib = _lib.load()
    over, told = threading.Event(), []

    def ask():
        torch.cuda.set_device(0)
        while not over.is_set():
            told.append(lib.cfa_op_status())

    other = threading.Thread(target=ask)
    other.start()
    words = []
    try:
        for _ in range(40):
            word = ctypes.c_int(-1)
            assert lib.cfa_selftest_op_timeout(-1, ctypes.byref(word)) == 0
            words.append(word.value)
    finally:
        over.set()
        other.join()
    assert words == [1] * 40
    assert told and set(told) == {0}


def test_products_run_on_after_the_waits_of_clusters_and_pairs_ran_out():
    """The self-test goes through single CTAs, clusters and pairs, without loads and with loads that are in
    flight when the others give up; none hangs or leaves anything behind for the products of each kind
    that follow."""
    from paper_2607_18957_gb300 import _lib
    word = ctypes.c_int(-1)
    assert _lib.load().cfa_selftest_op_timeout(0, ctypes.byref(word)) == 0 and word.value == 1
    for t, n, k in ((1, 128, 4096), (16, 256, 8192), (1024, 4096, 512)):
        x, w = normal(t, (t, k), BF16), normal(n, (n, k), BF16, k ** -0.5)
        ref = x.double() @ w.double().t()
        bound = (x.double().abs() @ w.double().abs().t()) * ((k + 8) * 2.0 ** -23)
        bound = bound + 2.0 ** -8 * (ref.abs() + bound)
        assert bool(((cfa.linear(x, w).double() - ref).abs() <= bound).all())


# ---- uneven experts -----------------------------------------------------------------------------

@pytest.mark.parametrize("t,e,top_k,first,held", [(512, 16, 4, 0, 16), (300, 32, 6, 8, 8),
                                                  (1100, 8, 2, 0, 8)])
def test_experts_of_which_one_has_many_times_its_share(t, e, top_k, first, held):
    """Most tokens name the first expert that is held, the rest is spread: its rows go through several
    tiles that were cut for the average.  A product's sum is off by at most (K + 8) 2^-23 of its terms'
    magnitudes, SiLU by 2^-16 of its argument and 1.2 times the argument's error, the activated values
    and the result by half a unit in the last place (2^-8)."""
    h, i = 136, 72
    g = torch.Generator(device="cuda").manual_seed(t)
    ids = torch.rand(t, e, generator=g, device="cuda").topk(top_k, dim=1).indices
    hot = (torch.rand(t, generator=g, device="cuda") < 0.9) & ~(ids == first).any(dim=1)
    ids[:, 0] = torch.where(hot, first, ids[:, 0])
    weights = torch.rand(t, top_k, generator=g, device="cuda")
    x = normal(t + 1, (t, h), BF16)
    w13, w2 = normal(2, (held, 2 * i, h), BF16, h ** -0.5), normal(3, (held, h, i), BF16, i ** -0.5)
    y = cfa.experts(x, ids.int(), weights, w13, w2, first_expert=first).double()
    ref, bound = torch.zeros_like(y), torch.zeros_like(y)
    u = 2.0 ** -23
    for k in range(held):
        tok, j = torch.where(ids == first + k)
        xk, w, d = x[tok].double(), w13[k].double(), w2[k].double()
        v, ev = xk @ w.t(), (xk.abs() @ w.abs().t()) * ((h + 8) * u)
        a, ea = v[:, :i] / (1 + torch.exp(-v[:, :i])), 1.2 * ev[:, :i] + 2.0 ** -16 * v[:, :i].abs()
        m, em = a * v[:, i:], ea * v[:, i:].abs() + (a.abs() + ea) * ev[:, i:]
        em = em + (2.0 ** -8 + u) * (m.abs() + em)
        o, eo = m @ d.t(), em @ d.abs().t() + ((m.abs() + em) @ d.abs().t()) * ((i + 8) * u)
        s = weights[tok, j].double()[:, None]
        ref.index_add_(0, tok, o * s)
        bound.index_add_(0, tok, (eo + (top_k + 2) * u * o.abs()) * s)
    bound = bound + 2.0 ** -8 * (ref.abs() + bound)
    assert bool(((y - ref).abs() <= bound).all())
