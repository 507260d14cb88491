"""A decoding step's operators at the edges of what their documentation allows."""
import ctypes
import math
import threading

import pytest
import torch

import paper_2607_18957_gb300 as cfa
from paper_2607_18957_gb300 import ops, step

pytestmark = pytest.mark.gpu

BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def cuda_device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


def attention(seed, lens=(700, 1, 200), heads=8, kv=2, dim=128, page=16):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(BF16)
    b, per = len(lens), (max(lens) + page - 1) // page
    table = torch.randperm(b * per, generator=g, device="cuda").to(torch.int32).view(b, per)
    return dict(q=normal(b, heads, dim), k_cache=normal(b * per, page, kv, dim),
                v_cache=normal(b * per, page, kv, dim), pages=table,
                lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"))


# ---- handles ------------------------------------------------------------------------------------

@pytest.mark.parametrize("handle", [0, 1])
def test_handles_of_the_default_stream(handle):
    """The default stream's own order holds for calls that are given its handle."""
    norm = cfa.norm(torch.ones(2, 64, device="cuda"), torch.ones(64, device="cuda"))
    assert norm.shape == (2, 64)
    with ops._elsewhere(handle, 0):
        assert ops._raw_stream(0) == torch.cuda.default_stream().cuda_stream
    big = torch.randn(4096, 4096, device="cuda").to(BF16)
    x, w = torch.zeros(300, 4096, device="cuda", dtype=BF16), torch.ones(4096, device="cuda", dtype=BF16)
    for i in range(5):
        x.zero_()
        y = big
        for _ in range(20):
            y = (big @ y).sign()
        x.copy_(y[:300] * (i + 1))
        got = cfa.norm(x, w, stream=handle)
        then = got.clone()  # on the default stream too, behind the call
        torch.cuda.synchronize()
        assert torch.equal(got, cfa.norm(x, w)) and torch.equal(then, got)


def test_a_call_is_in_the_order_of_the_threads_own_stream():
    own = torch.cuda.ExternalStream(2)
    big = torch.randn(4096, 4096, device="cuda").to(BF16)
    x, w = torch.zeros(300, 4096, device="cuda", dtype=BF16), torch.ones(4096, device="cuda", dtype=BF16)
    torch.cuda.synchronize()
    for i in range(5):
        with torch.cuda.stream(own):
            x.zero_()
            y = big
            for _ in range(20):
                y = (big @ y).sign()
            x.copy_(y[:300] * (i + 1))
            got = cfa.norm(x, w, stream=2)
            then = got.clone()
        own.synchronize()
        assert torch.equal(got, cfa.norm(x, w)) and torch.equal(then, got)


@pytest.mark.parametrize("current", [False, True])
def test_threads_with_streams_of_their_own(current):
    """Two threads' calls on cudaStreamPerThread, given or torch's current one, which overlap: the bits of
    calls in turn."""
    inputs = [attention(i, (60000, 30000)) for i in range(2)]
    want = [[t.clone() for t in cfa.attend(**a, lse=True)] for a in inputs]
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(2)

    def work(i):
        own = torch.cuda.ExternalStream(2)
        start.wait()
        for _ in range(40):
            if current:
                with torch.cuda.stream(own):
                    got = [cfa.attend(**inputs[i], lse=True) for _ in range(5)]
            else:
                got = [cfa.attend(**inputs[i], lse=True, stream=2) for _ in range(5)]
            own.synchronize()
            wrong.extend(i for g in got if not same(g, want[i]))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == []


def test_streams_that_are_made_and_destroyed_elsewhere():
    """Streams that are destroyed while their call is under way: the next gets the same handle, or not."""
    inputs = [attention(i, (60000, 30000)) for i in range(2)]
    want = [[t.clone() for t in cfa.attend(**a, lse=True)] for a in inputs]
    torch.cuda.synchronize()
    kept = dict(step._KEPT)
    cudart = torch.cuda.cudart()
    got = []
    for i in range(100):
        handle = ctypes.c_void_p()
        assert int(cudart.cudaStreamCreate(ctypes.addressof(handle))) == 0
        got.append(cfa.attend(**inputs[i % 2], lse=True, stream=handle.value))
        assert (0, handle.value) not in step._KEPT
        assert int(cudart.cudaStreamDestroy(handle.value)) == 0
    torch.cuda.synchronize()
    assert all(same(g, want[i % 2]) for i, g in enumerate(got))
    assert step._KEPT.keys() == kept.keys() and len(step._FOREIGN) <= 64


# ---- angles -------------------------------------------------------------------------------------

def test_angles_of_small_and_negative_frequencies():
    """Pairs (1, 0), whose second value is the sine alone: bf16 holds it however small it is.  The angle is off
    by 2^-52 of itself and 2^-65 turns a position, sine and rounding in fp32 by 2^-20 of the sine, the
    result by half a step, 2^-8."""
    f = [s * v for v in (1.0, 0.3, 1e-3, 1e-7, 1e-10, 1e-13, 1e-14, 1e-15) for s in (1, -1)]
    p = [1, 3, 1000, 123456789, (1 << 31) - 1, -1, -77, 1 - (1 << 31)]
    t, half = len(p), len(f)
    qkv = torch.zeros(t, 3 * 2 * half, device="cuda", dtype=BF16)
    qkv[:, :half] = 1.0
    cache = [torch.zeros(1, t, 1, 2 * half, device="cuda", dtype=BF16) for _ in range(2)]
    at = torch.arange(t, device="cuda", dtype=torch.int32)

    def turned(sign):
        return cfa.append(qkv, *cache, at, heads=1,
                          positions=torch.tensor([sign * x for x in p], dtype=torch.int32, device="cuda"),
                          frequencies=torch.tensor([sign * x for x in f], dtype=torch.float64, device="cuda"))
    q = turned(1)
    for i, x in enumerate(p):
        for j, v in enumerate(f):
            want, got = math.sin(x * v), q[i, 0, half + j].item()
            off = abs(x * v) * 2.0 ** -51 + abs(x) * 2.0 ** -65 * 2 * math.pi + abs(want) * 2.0 ** -20
            assert abs(got - want) <= off + (abs(want) + off) * 2.0 ** -8, (x, v)
    # the other way round by a position of the other sign
    assert torch.equal(turned(-1), q)


def test_frequencies_that_want_a_gradient_are_refused():
    qkv = torch.zeros(2, 3 * 64, device="cuda", dtype=BF16)
    cache = [torch.zeros(1, 2, 1, 64, device="cuda", dtype=BF16) for _ in range(2)]
    at = torch.arange(2, device="cuda", dtype=torch.int32)
    f = torch.zeros(32, device="cuda", dtype=torch.float64, requires_grad=True)
    with pytest.raises(ValueError, match="frequencies requires a gradient"):
        cfa.append(qkv, *cache, at, heads=1, positions=at, frequencies=f)
    with torch.no_grad():
        cfa.append(qkv, *cache, at, heads=1, positions=at, frequencies=f)


# ---- scales -------------------------------------------------------------------------------------

@pytest.mark.parametrize("cdtype", [BF16, F8])
def test_scales_below_fp32s_normal_range_of_large_scores(cdtype):
    """Scores of 2^122 to 2^127 times 2^-127 (over 8-bit keys 2^-57 times 2^-70): probabilities between 0.1
    and 10 times their mean.  Sums of powers of two are exact; the scale has at least 20 bits there, the
    values 8: 2^-8 for the result's rounding and 2^-10 for all else."""
    g = torch.Generator(device="cuda").manual_seed(5)
    heads, kv, dim, keys = 8, 2, 64, 200

    def signs(*shape):
        return (torch.randint(0, 2, shape, generator=g, device="cuda") * 2 - 1).float()
    q, k = signs(1, heads, dim), signs(13, 16, kv, dim)
    v = torch.randn(13, 16, kv, dim, generator=g, device="cuda").to(cdtype)
    z = torch.einsum("hgd,nhd->hgn", q.view(kv, -1, dim).double(), k.view(-1, kv, dim)[:keys].double()) / 32
    if cdtype is BF16:
        q, k, scale, k_scale = q * 2.0 ** 61, k * 2.0 ** 61, 2.0 ** -127, 1.0
    else:
        q, k, scale, k_scale = q * 2.0 ** 114, k * 2.0 ** 8, 2.0 ** -57, 2.0 ** -70
    pages = torch.arange(13, dtype=torch.int32, device="cuda")[None]
    lengths = torch.tensor([keys], dtype=torch.int32, device="cuda")
    o, lse = cfa.attend(q.to(BF16), k.to(cdtype), v, pages, lengths, scale=scale, k_scale=k_scale, lse=True)
    p, v = torch.softmax(z, 2), v.view(-1, kv, dim)[:keys].double()
    want = torch.einsum("hgn,nhd->hgd", p, v)
    bound = 2.0 ** -8 * want.abs() + 2.0 ** -10 * torch.einsum("hgn,nhd->hgd", p, v.abs())
    assert bool(((o.double().view_as(want) - want).abs() <= bound).all())
    assert (lse.double().view(kv, -1) - torch.logsumexp(z, 2)).abs().max() < 2.0 ** -16


@pytest.mark.parametrize("dtype,cdtype,score,value", [(torch.float16, torch.float16, -22.875, 60000.0),
                                                      (BF16, F8, -22.0, 448.0), (BF16, BF16, -60.0, 2.0 ** 60)])
def test_probabilities_far_below_the_largest(dtype, cdtype, score, value):
    """One key that takes nearly all with values of 0, a thousand of e^-22.9 or e^-22 of it (2^-33, 2^-32),
    which in fp16 are multiples of 2^-38 of the largest: off by 2^-39 of it each.  bf16 over bf16
    has no such floor.  The rest is fp32's, 2^-10 for it, and the result's rounding."""
    keys, dim = 1001, 64
    k, v = (torch.zeros(63, 16, 1, dim, device="cuda", dtype=cdtype) for _ in range(2))
    k.view(-1, dim)[1:, 0], v.view(-1, dim)[1:] = score, value
    q = torch.zeros(1, 1, dim, device="cuda", dtype=dtype)
    q[..., 0] = 1.0
    pages = torch.arange(63, dtype=torch.int32, device="cuda")[None]
    lengths = torch.tensor([keys], dtype=torch.int32, device="cuda")
    o = cfa.attend(q, k, v, pages, lengths, scale=1.0).double()
    n = keys - 1
    want = n * math.exp(score) * value / (1 + n * math.exp(score))
    floor = 0.0 if cdtype is BF16 else n * value * 2.0 ** -39
    bound = floor + want * 2.0 ** -10 + want * (2.0 ** -8 if dtype is BF16 else 2.0 ** -11)
    assert bool(((o - want).abs() <= bound).all()) and floor < want / 8


# ---- the example --------------------------------------------------------------------------------

@pytest.mark.parametrize("graph", [False, True])
def test_example_gives_the_log_probabilities_of_the_tokens_chosen(graph):
    """Of those that the next step takes in: the likeliest."""
    from examples import decode_step
    found, _, chosen = decode_step.run(sequences=4, hidden=256, steps=4, graph=graph)
    for (logits, lp, _, best, ids), tokens in zip(found, chosen):
        assert tokens == ids[:, 0].tolist() and torch.equal(lp, best[:, 0])
        z = torch.log_softmax(logits.double(), 1).gather(1, torch.tensor(tokens)[:, None])[:, 0]
        assert (lp - z).abs().max() < 2.0 ** -15  # fp32, as the sums of test_gpu_decode.py
