"""The entry points of a decoding step's operators on the host (no GPU): sizes of workspaces, frequencies, and
every refusal that comes before any CUDA call, through the C ABI with pointers that are never read."""
import ctypes
import math

import pytest
import torch

import paper_2607_18957_gb300 as cfa
from paper_2607_18957_gb300 import _lib, ops, step
from paper_2607_18957_gb300 import build as cfa_build

P = 0x7F0000000000
BF16, F16, F32, I32 = (_lib.DTYPE[k] for k in ("bf16", "f16", "f32", "i32"))
F8 = 9
INVAL, OVERLAP, DTYPE, ALIGN = -1, -2, -10, -11
MIB = 1 << 20
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module", autouse=True)
def lib():
    cfa_build.build()
    return _lib.load()


def norm(**kw):
    a = dict(x=P, residual=0, gate=0, weight=P + 8 * MIB, post=0, y=P + 16 * MIB, h=0, tokens=4, cols=64,
             xs=64, rs=64, gs=64, ys=64, hs=64, dtype=BF16, wdtype=BF16, act=4, flags=0, scale=1.0,
             eps=1e-6, offset=0.0, reserved=0)
    a.update(kw)
    return step._NORM.pack(*a.values())


def append(**kw):
    a = dict(qkv=P, positions=P + MIB, slots=P + 2 * MIB, frequencies=P + 3 * MIB, q=P + 4 * MIB,
             k=P + 8 * MIB, v=P + 16 * MIB, tokens=4, xs=512, qs=256, kp=2048, kt=128, kh=64, vp=2048,
             vt=128, vh=64, pages=8, page=16, heads=4, kv=2, dim=64, rot=64, dtype=BF16, cdtype=BF16,
             flags=0, magnitude=1.0, ks=1.0, vs=1.0)
    a.update(kw)
    return step._APPEND.pack(*a.values())


def attend(**kw):
    a = dict(q=P, k=P + 8 * MIB, v=P + 16 * MIB, pages=P + MIB, lengths=P + 2 * MIB, out=P + 3 * MIB, lse=0,
             ws=P + 64 * MIB, ws_bytes=64 * MIB, sequences=3, qs=256, os=256, ps=4, kp=2048, kt=128, kh=64,
             vp=2048, vt=128, vh=64, new=1, max_pages=4, cache_pages=8, page=16, heads=4, kv=2, dim=64,
             window=0, dtype=BF16, cdtype=BF16, flags=0, scale=0.125, ks=1.0, vs=1.0)
    a.update(kw)
    return step._ATTEND.pack(*a.values())


def logprobs(**kw):
    a = dict(logits=P, tokens=P + 8 * MIB, logprobs=P + 9 * MIB, entropy=P + 10 * MIB, best=P + 11 * MIB,
             ids=P + 12 * MIB, rows=4, cols=100, stride=100, dtype=F32, top=5, scale=1.0, flags=0)
    a.update(kw)
    return step._LOGPROBS.pack(*a.values())


def test_struct_sizes(lib):
    for name, size in step.SIZES.items():
        assert lib.cfa_abi_sizeof(name.encode()) == size


@pytest.mark.parametrize("change,status", [
    *(({k: 0}, INVAL) for k in ("x", "weight", "y", "cols")), ({"tokens": -1}, INVAL),
    ({"tokens": 1 << 31}, INVAL), ({"cols": 16385, "xs": 20000, "ys": 20000}, INVAL),
    ({"xs": 63}, INVAL), ({"ys": 63}, INVAL), ({"xs": 1 << 31}, INVAL),
    ({"residual": P + 32 * MIB, "rs": 63}, INVAL), ({"gate": P + 32 * MIB, "gs": 63}, INVAL),
    ({"h": P + 32 * MIB, "hs": 0}, INVAL), ({"act": 5}, INVAL), ({"act": -1}, INVAL), ({"flags": 1}, INVAL),
    ({"reserved": 1}, INVAL), ({"scale": NAN}, INVAL), ({"offset": INF}, INVAL), ({"eps": -1.0}, INVAL),
    ({"eps": NAN}, INVAL), ({"dtype": I32}, DTYPE), ({"wdtype": F16}, DTYPE), ({"dtype": F8}, DTYPE),
    ({"x": P + 1}, ALIGN), ({"weight": P + 8 * MIB + 1}, ALIGN), ({"wdtype": F32, "weight": P + 2}, ALIGN),
    ({"gate": P + 32 * MIB + 1}, ALIGN), ({"h": P + 32 * MIB + 1}, ALIGN),
    ({"y": P + 64}, OVERLAP), ({"y": P, "ys": 72}, OVERLAP), ({"y": P + 8 * MIB - 32}, OVERLAP),
    ({"h": P + 16 * MIB}, OVERLAP), ({"h": P + 16 * MIB + 64}, OVERLAP),
    ({"residual": P + 16 * MIB + 16}, OVERLAP), ({"post": P + 16 * MIB}, OVERLAP),
    ({"gate": P + 16 * MIB, "gs": 0}, OVERLAP),
])
def test_norm_refuses(lib, change, status):
    assert lib.cfa_norm_async(norm(**change), None) == status
    assert lib.cfa_last_error(None).startswith(b"cfa_norm")


@pytest.mark.parametrize("change,status", [
    *(({k: 0}, INVAL) for k in ("qkv", "slots", "k", "v", "positions", "frequencies", "kv", "page")),
    ({"tokens": -1}, INVAL), ({"heads": -1}, INVAL), ({"heads": 8193}, INVAL), ({"kv": 8193}, INVAL),
    ({"pages": -1}, INVAL), ({"dim": 60}, INVAL), ({"dim": 520}, INVAL), ({"dim": 0}, INVAL),
    ({"rot": 63}, INVAL), ({"rot": 66}, INVAL), ({"rot": 0}, INVAL), ({"flags": 2}, INVAL),
    ({"magnitude": NAN}, INVAL), ({"xs": 511}, INVAL), ({"qs": 255}, INVAL), ({"kp": 63}, INVAL),
    ({"vt": 0}, INVAL), ({"kh": -64}, INVAL), ({"kp": 1 << 41}, INVAL),
    ({"ks": 0.5}, INVAL), ({"cdtype": F8, "ks": 0.0}, INVAL), ({"cdtype": F8, "vs": NAN}, INVAL),
    ({"cdtype": F8, "vs": -1.0}, INVAL), ({"pages": (1 << 31) - 1, "kp": 1 << 39}, INVAL),
    ({"dtype": F32}, DTYPE), ({"cdtype": F16}, DTYPE), ({"cdtype": 77}, DTYPE),
    ({"qkv": P + 1}, ALIGN), ({"q": P + 4 * MIB + 1}, ALIGN), ({"k": P + 8 * MIB + 1}, ALIGN),
    ({"slots": P + 2 * MIB + 2}, ALIGN), ({"frequencies": P + 3 * MIB + 4}, ALIGN),
    ({"q": P, "qs": 256}, OVERLAP), ({"q": P + 64, "qs": 512}, OVERLAP), ({"q": P + 8 * MIB}, OVERLAP),
    ({"k": P + 16 * MIB}, OVERLAP), ({"v": P}, OVERLAP), ({"q": P + 2 * MIB}, OVERLAP),
])
def test_append_refuses(lib, change, status):
    assert lib.cfa_append_async(append(**change), None) == status
    assert lib.cfa_last_error(None).startswith(b"cfa_append")


@pytest.mark.parametrize("change,status", [
    *(({k: 0}, INVAL) for k in ("q", "k", "v", "pages", "lengths", "out", "ws", "new", "kv", "heads", "page",
                                "cache_pages")),
    ({"sequences": -1}, INVAL), ({"dim": 80}, INVAL), ({"dim": 512}, INVAL), ({"heads": 3}, INVAL),
    ({"heads": 8194}, INVAL), ({"new": 1 << 18}, INVAL), ({"max_pages": -1}, INVAL),
    ({"max_pages": 1 << 27}, INVAL), ({"window": -1}, INVAL), ({"window": (1 << 30) + 1}, INVAL),
    ({"flags": 1}, INVAL), ({"scale": NAN}, INVAL), ({"qs": 255}, INVAL), ({"os": 255}, INVAL),
    ({"ps": 3}, INVAL), ({"kt": 63}, INVAL), ({"ws_bytes": 1000}, INVAL), ({"ks": 2.0}, INVAL),
    ({"cdtype": F8, "ks": 0.0}, INVAL), ({"sequences": 1 << 30, "max_pages": 64, "ps": 64}, INVAL),
    ({"dtype": F32}, DTYPE), ({"cdtype": F16}, DTYPE),
    ({"q": P + 8}, ALIGN), ({"qs": 260}, ALIGN), ({"os": 260}, ALIGN), ({"out": P + 3 * MIB + 8}, ALIGN),
    ({"k": P + 8 * MIB + 8}, ALIGN), ({"kt": 132}, ALIGN), ({"vp": 2052}, ALIGN), ({"vh": 68}, ALIGN),
    ({"cdtype": F8, "kt": 136}, ALIGN), ({"pages": P + MIB + 2}, ALIGN), ({"lse": P + 5 * MIB + 2}, ALIGN),
    ({"ws": P + 64 * MIB + 128}, ALIGN),
    ({"out": P}, OVERLAP), ({"out": P + 16 * MIB}, OVERLAP), ({"lse": P + 3 * MIB}, OVERLAP),
    ({"ws": P}, OVERLAP), ({"ws": P + 2 * MIB}, OVERLAP), ({"lse": P + MIB}, OVERLAP),
])
def test_attend_refuses(lib, change, status):
    assert lib.cfa_attend_async(attend(**change), None) == status
    assert lib.cfa_last_error(None).startswith(b"cfa_attend")


def test_attend_workspace(lib):
    need, other = ctypes.c_uint64(), ctypes.c_uint64()
    assert lib.cfa_attend_workspace(attend(), ctypes.byref(need)) == 0
    assert lib.cfa_attend_workspace(attend(sequences=4000, max_pages=5000, ws=0), ctypes.byref(other)) == 0
    assert need.value == other.value and need.value % 256 == 0
    assert lib.cfa_attend_workspace(attend(heads=64), ctypes.byref(other)) == 0
    assert need.value < other.value
    assert lib.cfa_attend_workspace(attend(), None) == INVAL
    assert lib.cfa_attend_workspace(attend(dim=80), ctypes.byref(need)) == INVAL and need.value == 0


@pytest.mark.parametrize("change,status", [
    *(({k: 0}, INVAL) for k in ("logits", "tokens", "logprobs", "entropy", "best", "ids", "cols")),
    ({"rows": -1}, INVAL), ({"cols": 1 << 31, "stride": 1 << 31}, INVAL), ({"top": -1}, INVAL),
    ({"top": 33}, INVAL), ({"cols": 4, "top": 5}, INVAL), ({"scale": 0.0}, INVAL), ({"scale": -1.0}, INVAL),
    ({"scale": NAN}, INVAL), ({"scale": INF}, INVAL), ({"flags": 1}, INVAL), ({"stride": 99}, INVAL),
    ({"dtype": I32}, DTYPE), ({"logits": P + 2}, ALIGN), ({"tokens": P + 8 * MIB + 2}, ALIGN),
    ({"ids": P + 12 * MIB + 1}, ALIGN), ({"logprobs": P + 16}, OVERLAP), ({"ids": P + 11 * MIB}, OVERLAP),
    ({"entropy": P + 9 * MIB + 4}, OVERLAP), ({"best": P + 8 * MIB}, OVERLAP),
])
def test_logprobs_refuses(lib, change, status):
    assert lib.cfa_logprobs_async(logprobs(**change), None) == status
    assert lib.cfa_last_error(None).startswith(b"cfa_logprobs")


def test_null_arguments(lib):
    for f in (lib.cfa_norm_async, lib.cfa_append_async, lib.cfa_attend_async, lib.cfa_logprobs_async):
        assert f(None, None) == INVAL


def test_nothing_to_do_needs_no_pointers(lib):
    assert lib.cfa_norm_async(norm(tokens=0, x=0, y=0), None) == 0
    assert lib.cfa_append_async(append(tokens=0, qkv=0, positions=0, slots=0, k=0, v=0), None) == 0
    assert lib.cfa_attend_async(attend(sequences=0, q=0, out=0, ws=0), None) == 0
    assert lib.cfa_logprobs_async(logprobs(rows=0, logits=0, tokens=0), None) == 0


def test_cpu_tensors_are_refused():
    x, w = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.bfloat16)
    i, c = torch.zeros(2, dtype=torch.int32), torch.zeros(1, 16, 1, 64, dtype=torch.bfloat16)
    for call in (lambda: cfa.norm(x, w), lambda: cfa.logprobs(x, i),
                 lambda: cfa.append(torch.zeros(2, 192, dtype=torch.bfloat16), c, c, i, heads=1),
                 lambda: cfa.attend(x[:, None], c, c, i[:, None], i)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_rotary_frequencies():
    f, m = cfa.rotary_frequencies(8, 10000.0)
    assert m == 1.0 and f == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-12)
    assert cfa.rotary_frequencies(8, 10000.0, scaling="linear", factor=4.0)[0] == pytest.approx(
        [0.25, 0.025, 0.0025, 0.00025], rel=1e-12)
    f, _ = cfa.rotary_frequencies(8, 10000.0, scaling="base", factor=4.0)
    assert f[0] == 1.0 and f[3] == pytest.approx(0.00025, rel=1e-12) and 0.025 < f[1] < 0.1
    # 16,384 positions: the first four pairs make more than four turns, the last 1.6
    f, m = cfa.rotary_frequencies(10, 10000.0, scaling="bands", factor=8.0, length=16384)
    g = [10000.0 ** (-i / 5) for i in range(5)]
    kept = (16384 * g[4] / (2 * math.pi) - 1) / 3
    assert 0 < kept < 1 and m == 1.0
    assert f == pytest.approx(g[:4] + [g[4] * (kept + (1 - kept) / 8)], rel=1e-12)
    f, m = cfa.rotary_frequencies(128, 10000.0, scaling="ramp", factor=16.0, length=4096)
    g = [10000.0 ** (-i / 64) for i in range(64)]
    assert m == pytest.approx(0.1 * math.log(16.0) + 1.0)
    assert f[0] == 1.0 and f[63] == pytest.approx(g[63] / 16, rel=1e-12)
    turns = [4096 * v / (2 * math.pi) for v in g]
    for i in range(64):  # kept above 32 turns, divided below one, between them in between
        if turns[i] > 36:
            assert f[i] == pytest.approx(g[i], rel=1e-12)
        elif turns[i] < 0.8:
            assert f[i] == pytest.approx(g[i] / 16, rel=1e-12)
        else:
            assert g[i] / 16 <= f[i] <= g[i]
    assert cfa.rotary_frequencies(64, scaling="ramp", factor=4.0, length=4096, magnitude=1.0)[1] == 1.0
    for bad in (dict(dim=7), dict(dim=0), dict(dim=8, base=1.0), dict(dim=8, factor=0.5),
                dict(dim=8, scaling="spiral"), dict(dim=8, scaling="bands", factor=2.0)):
        with pytest.raises(ValueError):
            cfa.rotary_frequencies(**bad)


class OnDevice1:
    """What the calls ask of an operand before they enter a stream's guard."""
    requires_grad = False
    device = torch.device("cuda", 1)

    def get_device(self):
        return 1

    def is_contiguous(self):
        return True


class Stream:
    def __init__(self, index):
        self.device = torch.device("cuda", index)


CALLS = {"norm": lambda x, s: cfa.norm(x, x, stream=s),
         "append": lambda x, s: cfa.append(x, x, x, x, heads=1, stream=s),
         "attend": lambda x, s: cfa.attend(x, x, x, x, x, stream=s),
         "logprobs": lambda x, s: cfa.logprobs(x, x, stream=s)}


@pytest.mark.parametrize("name", CALLS)
def test_streams_of_other_devices_are_refused_and_the_operands_entered(name, monkeypatch):
    if ops.torch is None:
        ops._start()
    entered = []

    class Guard:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            entered.append(self.stream)
            raise KeyError

        def __exit__(self, *exc):
            pass

    monkeypatch.setattr(torch.cuda, "stream", Guard)
    monkeypatch.setattr(ops, "_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:0.*cuda:1"):
        CALLS[name](OnDevice1(), Stream(0))
    assert entered == []
    s = Stream(1)
    with pytest.raises(KeyError):
        CALLS[name](OnDevice1(), s)
    assert entered == [s]
