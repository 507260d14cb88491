"""A decoding step of all operators together: the example, captured and not; streams; graphs that share
operands; calls from several threads."""
import threading

import pytest
import torch

import paper_2607_18957_gb300 as cfa

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def cuda_device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("sequences,hidden", [(1, 256), (5, 512), (40, 512)])
def test_example_decodes(sequences, hidden, graph):
    """Seven products and three norms whose values are rounded to bf16 (2^-8 each): 2^-4 of the logits'
    norm covers sixteen such errors in a row.  The log probabilities are those of the logits given, to
    fp32: 2^-15."""
    from examples import decode_step
    found, wanted, given = decode_step.run(sequences=sequences, hidden=hidden, steps=3, graph=graph)
    assert len(found) == 3
    for (logits, lp, entropy, best, ids), rows, tokens in zip(found, wanted, given):
        z = torch.log_softmax(logits.double(), 1)
        assert bool(torch.isfinite(logits).all())
        top = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :best.shape[1]]
        assert torch.equal(ids.long(), top)
        assert (best - z.gather(1, top)).abs().max() < 2.0 ** -15
        assert (entropy + (z.exp() * z).sum(1)).abs().max() < 2.0 ** -15
        assert (lp - z.gather(1, torch.tensor(tokens)[:, None])[:, 0]).abs().max() < 2.0 ** -15
        for s, ref in enumerate(rows):
            if ref is not None:
                assert (logits[s].double() - ref).norm() < 2.0 ** -4 * ref.norm(), s


def operands(seed, b=3, heads=8, kv=2, dim=128, keys=700):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(BF16)
    pages = (keys + 15) // 16
    k, v = normal(b * pages, 16, kv, dim), normal(b * pages, 16, kv, dim)
    table = torch.randperm(b * pages, generator=g, device="cuda").to(torch.int32).view(b, pages)
    lengths = torch.tensor([keys, 1, keys // 3], dtype=torch.int32, device="cuda")[:b]
    return dict(q=normal(b, heads, dim), k_cache=k, v_cache=v, pages=table, lengths=lengths)


def all_calls(seed):
    """Each operator on operands of its own: functions without arguments."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, r = (torch.randn(300, 1024, generator=g, device="cuda").to(BF16) for _ in range(2))
    w = torch.ones(1024, device="cuda", dtype=BF16)
    logits = torch.randn(30, 40000, generator=g, device="cuda")
    tokens = torch.randint(0, 40000, (30,), generator=g, device="cuda", dtype=torch.int32)
    a = operands(seed)
    qkv = torch.randn(48, 12 * 128, generator=g, device="cuda").to(BF16)
    kc, vc = (torch.zeros(4, 16, 2, 128, device="cuda", dtype=BF16) for _ in range(2))
    at = torch.arange(48, device="cuda", dtype=torch.int32)
    f = torch.tensor(cfa.rotary_frequencies(128)[0], dtype=torch.float64, device="cuda")

    def append(**kw):
        q = cfa.append(qkv, kc, vc, at, heads=8, positions=at, frequencies=f, **kw)
        return q, kc, vc
    return {"norm": lambda **kw: cfa.norm(x, w, residual=r, **kw),
            "attend": lambda **kw: cfa.attend(**a, lse=True, **kw),
            "logprobs": lambda **kw: cfa.logprobs(logits, tokens, top=9, **kw), "append": append}


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("name", ["norm", "append", "attend", "logprobs"])
def test_streams_and_handles(name):
    want = [t.clone() for t in all_calls(1)[name]()]
    for as_handle in (False, True):
        call = all_calls(1)[name]
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        got = call(stream=s.cuda_stream if as_handle else s)
        s.synchronize()
        assert same(got, want)


@pytest.mark.parametrize("name", ["norm", "append", "attend", "logprobs"])
def test_graphs(name):
    """A captured call replayed after its operands have changed, and two graphs in turn."""
    calls = [all_calls(seed)[name] for seed in (1, 2)]
    want = [[t.clone() for t in c()] for c in calls]
    graphs, results = [], []
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            results.append(c())
    for _ in range(3):
        for g, r, w in zip(graphs, results, want):
            for t in r:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert same(r, w)


def test_a_graph_follows_lengths_and_shares_its_workspace():
    """Lengths grow between replays; another graph and calls outside use the same workspace in between."""
    a, b = operands(3), operands(4, b=2, heads=16, kv=2, dim=64, keys=5000)
    ws = torch.full((4 << 20,), 255, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs, results = [], []
    for o in (a, b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            results.append(cfa.attend(**o, lse=True, workspace=ws))
    for n in (0, 1, 15, 16, 17, 333, 700):
        a["lengths"].fill_(n)
        for g, r, o in zip(graphs, results, (a, b)):
            g.replay()
            torch.cuda.synchronize()
            assert same(r, cfa.attend(**o, lse=True))
            assert same(r, cfa.attend(**o, lse=True, workspace=ws))
            torch.cuda.synchronize()


def test_workspaces_are_the_streams():
    """Eager calls keep one per stream, grown where a call needs more; captured ones have their own."""
    from paper_2607_18957_gb300 import step
    small, large = operands(6, heads=2, kv=2, dim=64), operands(7, heads=32, kv=2, dim=128)
    want = [cfa.attend(**o, lse=True) for o in (small, large)]
    torch.cuda.synchronize()
    step._KEPT.clear()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a = cfa.attend(**small, lse=True)
        kept = step._KEPT[0, s.cuda_stream]
        b = cfa.attend(**large, lse=True)
        assert step._KEPT[0, s.cuda_stream].numel() > kept.numel() and len(step._KEPT) == 1
        kept = step._KEPT[0, s.cuda_stream]
        c = cfa.attend(**small, lse=True)
        assert step._KEPT[0, s.cuda_stream] is kept
    s.synchronize()
    assert same(a, want[0]) and same(b, want[1]) and same(c, want[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        r = cfa.attend(**large, lse=True)
    assert len(step._KEPT) == 1 and step._KEPT[0, s.cuda_stream] is kept
    # replays on another stream beside eager calls on the stream of the capture
    other = torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(other):
            g.replay()
        with torch.cuda.stream(s):
            b = cfa.attend(**large, lse=True)
    torch.cuda.synchronize()
    assert same(r, want[1]) and same(b, want[1])


def test_two_streams_at_once():
    """Calls that overlap, each with a workspace of its own."""
    a = [operands(i, keys=20000) for i in range(2)]
    want = [cfa.attend(**o, lse=True) for o in a]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in a]
    got = [[], []]
    for _ in range(20):
        for i, (o, s) in enumerate(zip(a, streams)):
            with torch.cuda.stream(s):
                got[i].append(cfa.attend(**o, lse=True))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(same(r, want[i]) for r in got[i])


def test_threads():
    want = {n: [t.clone() for t in c()] for n, c in all_calls(5).items()}
    wrong = []

    def work():
        with torch.cuda.stream(torch.cuda.Stream()):
            calls = all_calls(5)
            for _ in range(10):
                for n, c in calls.items():
                    r = c()
                    torch.cuda.current_stream().synchronize()
                    if not same(r, want[n]):
                        wrong.append(n)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == []


@pytest.mark.parametrize("name", ["norm", "append", "attend", "logprobs"])
def test_calls_behind_one_another(name):
    """A call's operands are written by the launch before it, which it may overlap."""
    g = torch.Generator(device="cuda").manual_seed(9)
    if name == "norm":
        w = torch.ones(2048, device="cuda", dtype=BF16)
        x = torch.randn(700, 2048, generator=g, device="cuda").to(BF16)
        for _ in range(50):
            y = cfa.norm(x, w)
            z = cfa.norm(y, w)
            torch.cuda.synchronize()
            assert torch.equal(z, cfa.norm(y, w))
    elif name == "logprobs":
        h, w = (torch.randn(8, 512, generator=g, device="cuda").to(BF16),
                torch.randn(30000, 512, generator=g, device="cuda").to(BF16))
        tokens = torch.arange(8, device="cuda", dtype=torch.int32)
        for _ in range(50):
            logits = cfa.linear(h, w, out_dtype="f32")
            r = cfa.logprobs(logits, tokens, top=3)
            torch.cuda.synchronize()
            assert same(r, cfa.logprobs(logits, tokens, top=3))
    else:
        heads, kv, dim = 8, 2, 128
        w = torch.randn((heads + 2 * kv) * dim, 512, generator=g, device="cuda").to(BF16)
        kc, vc = (torch.zeros(8, 16, kv, dim, device="cuda", dtype=BF16) for _ in range(2))
        at = torch.arange(64, device="cuda", dtype=torch.int32)
        f = torch.tensor(cfa.rotary_frequencies(dim)[0], dtype=torch.float64, device="cuda")
        pages = torch.arange(8, device="cuda", dtype=torch.int32).repeat(64, 1)
        for i in range(50):
            x = torch.randn(64, 512, generator=g, device="cuda").to(BF16)
            qkv = cfa.linear(x, w)
            q = cfa.append(qkv, kc, vc, at, heads=heads, positions=at, frequencies=f)
            o = cfa.attend(q, kc, vc, pages, at + 1)
            torch.cuda.synchronize()
            k1, v1 = kc.clone(), vc.clone()
            q2 = cfa.append(qkv, kc, vc, at, heads=heads, positions=at, frequencies=f)
            torch.cuda.synchronize()
            assert torch.equal(q, q2) and torch.equal(k1, kc) and torch.equal(v1, vc)
            assert torch.equal(o, cfa.attend(q, kc, vc, pages, at + 1))


def test_python_refusals():
    a = operands(1)
    x, w = torch.zeros(4, 64, dtype=BF16, device="cuda"), torch.ones(64, dtype=BF16, device="cuda")
    qkv = torch.zeros(2, 12 * 128, dtype=BF16, device="cuda")
    i2 = torch.zeros(2, dtype=torch.int32, device="cuda")
    f = torch.zeros(64, dtype=torch.float64, device="cuda")
    k, v = a["k_cache"], a["v_cache"]
    logits = torch.zeros(2, 50, device="cuda")
    for bad in (lambda: cfa.norm(x, w[:32]), lambda: cfa.norm(x, w.cpu()), lambda: cfa.norm(x.double(), w),
                lambda: cfa.norm(x, w, residual=x[:2]), lambda: cfa.norm(x, w, residual=x.float()),
                lambda: cfa.norm(x, w, gate=x[:, :32]), lambda: cfa.norm(x, w, gate=x, activation="swish"),
                lambda: cfa.norm(x, w, post_weight=w.float()), lambda: cfa.norm(x.t(), x[:, 0]),
                lambda: cfa.norm(x, w, out=x[:2]), lambda: cfa.norm(x, w.clone().requires_grad_()),
                lambda: cfa.norm(x, w, residual=x.clone().requires_grad_()),
                lambda: cfa.append(qkv, k, v, i2, heads=7), lambda: cfa.append(qkv, k, v, i2.long(), heads=8),
                lambda: cfa.append(qkv, k, v, i2[:1], heads=8), lambda: cfa.append(qkv, k, v[:1], i2, heads=8),
                lambda: cfa.append(qkv, k, v, i2, heads=8, positions=i2),
                lambda: cfa.append(qkv, k, v, i2, heads=8, positions=i2, frequencies=f.float()),
                lambda: cfa.append(qkv, k.float(), v.float(), i2, heads=8),
                lambda: cfa.append(qkv, k, v, i2, heads=8, out=torch.zeros(2, 8, 64, dtype=BF16, device="cuda")),
                lambda: cfa.append(qkv.cpu(), k, v, i2, heads=8),
                lambda: cfa.attend(**dict(a, q=a["q"][..., :64])), lambda: cfa.attend(**dict(a, q=a["q"].half())),
                lambda: cfa.attend(**dict(a, lengths=a["lengths"].long())),
                lambda: cfa.attend(**dict(a, pages=a["pages"][:2])),
                lambda: cfa.attend(**dict(a, q=a["q"].transpose(0, 1).contiguous().transpose(0, 1)[:, :, :])),
                lambda: cfa.attend(**a, out=torch.zeros_like(a["q"])[:2]),
                lambda: cfa.attend(**a, lse=True, out=(torch.zeros_like(a["q"]), torch.zeros(3, 7, device="cuda"))),
                lambda: cfa.attend(**a, workspace=torch.zeros(100, 2, dtype=torch.uint8, device="cuda")[:, 0]),
                lambda: cfa.logprobs(logits, i2.long()), lambda: cfa.logprobs(logits, i2[:1]),
                lambda: cfa.logprobs(logits.double(), i2), lambda: cfa.logprobs(logits, i2, top=-1),
                lambda: cfa.logprobs(logits, i2, out=(logits[:, 0],))):
        with pytest.raises(ValueError):
            bad()
    for bad, name in ((lambda: cfa.norm(x, w, out=x[:, :].as_strided((4, 64), (64, 1), 0)[0:4]), None),
                      (lambda: cfa.norm(x, w, eps=-1.0), "CFA_ERR_INVAL"),
                      (lambda: cfa.norm(x[:1].expand(4, 64), w), "CFA_ERR_INVAL"),
                      (lambda: cfa.append(qkv, k, v, i2, heads=8, k_scale=2.0), "CFA_ERR_INVAL"),
                      (lambda: cfa.append(qkv, k, k, i2, heads=8), "CFA_ERR_OVERLAP"),
                      (lambda: cfa.attend(**a, window=-1), "CFA_ERR_INVAL"),
                      (lambda: cfa.attend(**a, workspace=torch.zeros(100, dtype=torch.uint8, device="cuda")),
                       "CFA_ERR_INVAL"),
                      (lambda: cfa.attend(**a, out=a["q"]), "CFA_ERR_OVERLAP"),
                      (lambda: cfa.logprobs(logits, i2, top=51), "CFA_ERR_INVAL"),
                      (lambda: cfa.logprobs(logits, i2, scale=0.0), "CFA_ERR_INVAL")):
        if name is None:
            bad()  # in place is allowed
            continue
        with pytest.raises(cfa.CfaError) as err:
            bad()
        assert err.value.name == name
