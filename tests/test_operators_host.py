"""The operators' entry points on the host (no GPU): sizes of their workspaces, and every refusal that
comes before any CUDA call, through the C ABI with pointers that are never read."""
import ctypes

import pytest
import torch

import paper_2607_18957_gb300 as cfa
from paper_2607_18957_gb300 import _lib, ops
from paper_2607_18957_gb300 import build as cfa_build

P = 0x7F0000000000
BF16, F16, F32, I32 = (_lib.DTYPE[k] for k in ("bf16", "f16", "f32", "i32"))
INVAL, OVERLAP, DTYPE, ALIGN = -1, -2, -10, -11
MIB = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    cfa_build.build()
    return _lib.load()


def linear(**kw):
    a = dict(x=P, w=P + 64 * MIB, bias=0, residual=0, y=P + 128 * MIB, ws=0, ws_bytes=0, tokens=4,
             rows=64, cols=32, xs=32, wst=32, rs=64, ys=64, dtype=BF16, bias_dtype=BF16,
             y_dtype=BF16, act=0, flags=0, reserved=0)
    a.update(kw)
    return ops._LINEAR.pack(*a.values())


def route(**kw):
    a = dict(logits=P, bias=0, weights=P + MIB, ids=P + 2 * MIB, tokens=4, stride=16, experts=16,
             top_k=2, groups=1, top_groups=1, dtype=F32, scoring=0, flags=0, scale=1.0)
    a.update(kw)
    return ops._ROUTE.pack(*a.values())


def experts(**kw):
    a = dict(x=P, w13=P + MIB, w2=P + 2 * MIB, residual=0, ids=P + 3 * MIB,
             weights=P + 4 * MIB, y=P + 5 * MIB, ws=P + 64 * MIB, ws_bytes=64 * MIB, tokens=4,
             hidden=64, inter=32, xs=64, rs=64, ys=64, experts=4, first=0, top_k=2, dtype=BF16,
             act=4, flags=1)
    a.update(kw)
    return ops._EXPERTS.pack(*a.values())


def test_struct_sizes(lib):
    for name, size in ops.SIZES.items():
        assert lib.cfa_abi_sizeof(name.encode()) == size


@pytest.mark.parametrize("change,status", [
    ({"x": 0}, INVAL), ({"w": 0}, INVAL), ({"y": 0}, INVAL), ({"tokens": -1}, INVAL),
    ({"rows": 0}, INVAL), ({"cols": 0}, INVAL), ({"tokens": 1 << 31}, INVAL),
    ({"xs": 31}, INVAL), ({"wst": 31}, INVAL), ({"ys": 63}, INVAL), ({"xs": -32}, INVAL),
    ({"residual": P + 256 * MIB, "rs": 63}, INVAL), ({"wst": 1 << 31}, INVAL),
    ({"dtype": F32}, DTYPE), ({"dtype": 77}, DTYPE), ({"y_dtype": F16}, DTYPE),
    ({"bias": P + 200 * MIB, "bias_dtype": F16}, DTYPE), ({"act": 5}, INVAL), ({"act": -1}, INVAL),
    ({"flags": 2}, INVAL), ({"reserved": 1}, INVAL), ({"flags": 1, "rows": 63}, INVAL),
    ({"x": P + 1}, ALIGN), ({"w": P + 64 * MIB + 1}, ALIGN), ({"y": P + 128 * MIB + 1}, ALIGN),
    ({"y_dtype": F32, "y": P + 128 * MIB + 2}, ALIGN),
    ({"bias": P + 200 * MIB + 2, "bias_dtype": F32}, ALIGN),
    ({"y": P + 64}, OVERLAP), ({"y": P + 64 * MIB + 64}, OVERLAP),
    ({"residual": P + 128 * MIB + 16}, OVERLAP),
    ({"residual": P + 128 * MIB, "rs": 72}, OVERLAP),
    ({"bias": P + 128 * MIB + 16}, OVERLAP),
    # off the 16-byte grid: a workspace, large enough, aligned and apart
    ({"x": P + 2}, INVAL), ({"wst": 33, "ws": P + 300 * MIB, "ws_bytes": 64}, INVAL),
    ({"x": P + 2, "ws": P + 300 * MIB + 16, "ws_bytes": MIB}, ALIGN),
    ({"x": P + 2, "ws": P + 128 * MIB, "ws_bytes": MIB}, OVERLAP),
    # sizes whose product leaves 64 bits
    ({"tokens": (1 << 31) - 1, "ys": (1 << 31) - 1, "xs": (1 << 31) - 1, "rows": (1 << 31) - 1,
      "cols": (1 << 31) - 1, "wst": (1 << 31) - 1}, INVAL),
])
def test_linear_refuses(lib, change, status):
    assert lib.cfa_linear_async(linear(**change), None) == status
    assert lib.cfa_last_error(None).startswith(b"cfa_linear")


def test_linear_workspace(lib):
    need = ctypes.c_uint64()

    def bytes_of(**kw):
        assert lib.cfa_linear_workspace(linear(**kw), ctypes.byref(need)) == 0
        return need.value
    assert bytes_of() == 0
    assert bytes_of(x=P + 2) == 256                       # 4 rows of 32
    assert bytes_of(cols=31, xs=32, wst=32) == 0          # strides on the grid
    assert bytes_of(cols=31, xs=31, wst=32) == 256
    assert bytes_of(cols=31, xs=31, wst=31) == 256 + 64 * 32 * 2
    assert bytes_of(tokens=1, cols=31, xs=31, wst=32) == 0  # one row has no stride
    assert lib.cfa_linear_workspace(linear(), None) == INVAL
    assert lib.cfa_linear_workspace(linear(dtype=F32), ctypes.byref(need)) == DTYPE
    assert need.value == 0


@pytest.mark.parametrize("change,status", [
    ({"logits": 0}, INVAL), ({"weights": 0}, INVAL), ({"ids": 0}, INVAL), ({"tokens": -1}, INVAL),
    ({"experts": 0}, INVAL), ({"experts": 1025, "stride": 2000}, INVAL), ({"top_k": 0}, INVAL),
    ({"top_k": 17}, INVAL), ({"experts": 64, "stride": 64, "top_k": 33}, INVAL),
    ({"groups": 0}, INVAL), ({"groups": 3}, INVAL), ({"groups": 4, "top_groups": 5}, INVAL),
    ({"groups": 64, "experts": 128, "stride": 128}, INVAL), ({"top_groups": 0}, INVAL),
    ({"scoring": 2}, INVAL), ({"flags": 2}, INVAL), ({"stride": 15}, INVAL),
    ({"dtype": I32}, DTYPE), ({"logits": P + 2}, ALIGN), ({"ids": P + 2 * MIB + 1}, ALIGN),
    ({"bias": P + 3 * MIB + 2}, ALIGN), ({"ids": P + MIB}, OVERLAP), ({"weights": P}, OVERLAP),
    ({"bias": P + MIB}, OVERLAP),
])
def test_route_refuses(lib, change, status):
    assert lib.cfa_route_async(route(**change), None) == status
    assert lib.cfa_last_error(None).startswith(b"cfa_route")


@pytest.mark.parametrize("change,status", [
    *(({k: 0}, INVAL) for k in ("x", "w13", "w2", "ids", "weights", "y", "ws", "hidden", "inter",
                                "experts", "top_k")),
    ({"tokens": -1}, INVAL), ({"experts": 1025}, INVAL), ({"top_k": 33}, INVAL),
    ({"first": -1}, INVAL), ({"xs": 63}, INVAL), ({"ys": 63}, INVAL),
    ({"residual": P + 6 * MIB, "rs": 63}, INVAL), ({"ws_bytes": 1000}, INVAL), ({"act": 9}, INVAL),
    ({"flags": 4}, INVAL), ({"tokens": 1 << 30, "top_k": 4}, INVAL),
    ({"experts": 1024, "inter": 1 << 24}, INVAL), ({"dtype": F32}, DTYPE),
    ({"hidden": 60}, ALIGN), ({"inter": 36}, ALIGN), ({"w13": P + MIB + 8}, ALIGN),
    ({"w2": P + 2 * MIB + 8}, ALIGN), ({"ws": P + 64 * MIB + 16}, ALIGN),
    ({"ids": P + 3 * MIB + 2}, ALIGN), ({"x": P + 1}, ALIGN),
    ({"y": P}, OVERLAP), ({"y": P + 3 * MIB}, OVERLAP), ({"ws": P}, OVERLAP),
    ({"y": P + 64 * MIB}, OVERLAP), ({"residual": P + 5 * MIB + 16}, OVERLAP),
    ({"residual": P + 64 * MIB}, OVERLAP),
])
def test_experts_refuse(lib, change, status):
    assert lib.cfa_experts_async(experts(**change), None) == status
    assert lib.cfa_last_error(None).startswith(b"cfa_experts")


def test_null_arguments(lib):
    for f in (lib.cfa_linear_async, lib.cfa_route_async, lib.cfa_experts_async):
        assert f(None, None) == INVAL


def test_selftest_refuses_a_null_output(lib):
    assert lib.cfa_selftest_op_timeout(-1, None) == INVAL


def test_no_tokens_need_no_pointers(lib):
    assert lib.cfa_linear_async(linear(tokens=0, x=0, w=0, y=0), None) == 0
    assert lib.cfa_route_async(route(tokens=0, logits=0, weights=0, ids=0), None) == 0
    assert lib.cfa_experts_async(experts(tokens=0, x=0, y=0, ws=0, ws_bytes=0), None) == 0


def test_experts_workspace(lib):
    need, more = ctypes.c_uint64(), ctypes.c_uint64()
    assert lib.cfa_experts_workspace(experts(), ctypes.byref(need)) == 0
    assert lib.cfa_experts_workspace(experts(tokens=4000), ctypes.byref(more)) == 0
    assert 0 < need.value < more.value and need.value % 256 == 0
    assert lib.cfa_experts_workspace(experts(), None) == INVAL


def test_cpu_tensors_are_refused():
    x, w = torch.zeros(2, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.bfloat16)
    for call in (lambda: cfa.linear(x, w), lambda: cfa.route(x, 2)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
