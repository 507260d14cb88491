"""Operators on the loaded layout (cfa_linear_async, cfa_route_async, cfa_experts_async of cfa.h):
the matrix product with a weight in its fused layout, the choice of experts, and the products with
stacked experts.  Forward passes for serving; argument marshalling only.

Every call enqueues on `stream` (default: torch's current stream) and returns at once.  Outputs and
workspaces that a call makes come from torch's allocator, on that stream.  Operands are CUDA tensors
of one device whose last dimension is contiguous; rows may lie any distance apart.
"""
import struct

from . import _lib

__all__ = ["linear", "route", "experts", "op_status"]

ACTIVATION = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
SCORING = {"softmax": 0, "sigmoid": 1}
GATED, RENORMALIZE = 0x1, 0x1

_LINEAR = struct.Struct("<7Q7q4iIi")
_ROUTE = struct.Struct("<4Q2q6iIf")
_EXPERTS = struct.Struct("<9Q6q5iI")
SIZES = {"cfa_linear_args": _LINEAR.size, "cfa_route_args": _ROUTE.size,
         "cfa_experts_args": _EXPERTS.size}

torch = None
_CODE = None   # torch dtype -> CFA_DTYPE_*
_DTYPE = None  # dtype name -> torch dtype


def _start():
    global torch, _CODE, _DTYPE
    import torch as t
    _DTYPE = {"bf16": t.bfloat16, "f16": t.float16, "f32": t.float32}
    _CODE = {v: _lib.DTYPE[k] for k, v in _DTYPE.items()}
    torch = t


def _check(lib, st):
    if st != _lib.CFA_OK:
        from . import _check as check
        check(st)


def _operands(device, **tensors):
    grad = torch.is_grad_enabled()
    for name, t in tensors.items():
        if t is None:
            continue
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, not on {device}")
        if t.shape and t.stride(-1) != 1 and t.shape[-1] > 1:
            raise ValueError(f"{name}: the last dimension must be contiguous")
        if grad and t.requires_grad:
            raise ValueError(f"{name} requires a gradient, and the operators have no backward "
                             "pass: call them under torch.no_grad()")


def _code(t, name):
    c = _CODE.get(t.dtype)
    if c is None:
        raise ValueError(f"{name}: {t.dtype} is not supported")
    return c


def _one_of(table, name, what):
    v = table.get(name)
    if v is None:
        raise ValueError(f"unknown {what} {name!r}: one of {', '.join(table)}")
    return v


def _rows(t, name, cols):
    """A tensor [..., cols] as rows: (tensor, row count, row stride)."""
    if t.dim() == 2:
        n, c = t.shape
    elif t.dim() and t.shape[-1]:
        c = t.shape[-1]
        n = t.numel() // c
        t = t.view(n, c)  # raises where the rows do not lie evenly
    else:
        raise ValueError(f"{name}: shape {tuple(t.shape)}")
    if c != cols:
        raise ValueError(f"{name}: rows of {c}, not {cols}")
    return t, n, t.stride(0)


class _On:
    """The stream that a call enqueues on, current while it allocates."""

    def __init__(self, stream, device):
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=device)
        self.handle = stream.cuda_stream
        self.guard = torch.cuda.stream(stream)

    def __enter__(self):
        self.guard.__enter__()
        return self.handle

    def __exit__(self, *exc):
        self.guard.__exit__(*exc)


class _Current:
    def __init__(self, device):
        self.guard = None
        if device.index != torch.cuda.current_device():
            self.guard = torch.cuda.device(device)
        self.device = device

    def __enter__(self):
        if self.guard:
            self.guard.__enter__()
        return torch._C._cuda_getCurrentRawStream(self.device.index)

    def __exit__(self, *exc):
        if self.guard:
            self.guard.__exit__(*exc)


def _enter(stream, device):
    if device.type != "cuda":
        raise ValueError(f"the operators run on CUDA tensors, not on {device}")
    return _Current(device) if stream is None else _On(stream, device)


def _workspace(given, need, device):
    if given is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if given.device != device or not given.is_contiguous():
        raise ValueError("the workspace must be contiguous and on the operands' device")
    return given


def linear(x, weight, bias=None, *, activation="none", gated=False, residual=None, out=None,
           out_dtype=None, workspace=None, stream=None):
    """act(x weight^T + bias) + residual.

    x         [..., K] bf16 or fp16;  weight [N, K] of the same dtype, as loaded
    bias      [N] of x's dtype or fp32
    gated     weight holds N / 2 gate rows, then N / 2 up rows (a fused gate_up weight), and the
              result is act(gate) * up, N / 2 wide
    activation  "none", "relu", "gelu", "gelu_tanh" or "silu"
    residual  added after the activation, shaped and typed like the result; `out` may be the same
              tensor
    out, out_dtype  where the result goes, or its dtype ("f32", or x's: the default)
    workspace  uint8 tensor for operands off the 16-byte grid (default: allocated if needed)
    """
    if torch is None:
        _start()
    device = x.device
    _operands(device, x=x, weight=weight, bias=bias, residual=residual, out=out)
    if weight.dim() != 2:
        raise ValueError(f"weight: shape {tuple(weight.shape)}")
    n, k = weight.shape
    x2, t, xs = _rows(x, "x", k)
    code = _code(x, "x")
    if weight.dtype != x.dtype:
        raise ValueError(f"weight is {weight.dtype}, x {x.dtype}")
    if bias is not None and bias.shape != (n,):
        raise ValueError(f"bias: shape {tuple(bias.shape)}, not ({n},)")
    if gated and n % 2:
        raise ValueError(f"a gated weight has an even number of rows, not {n}")
    act = _one_of(ACTIVATION, activation, "activation")
    no = n // 2 if gated else n
    shape = x.shape[:-1] + (no,)
    lib = _lib.load()
    with _enter(stream, device) as handle:
        if out is None:
            dt = x.dtype if out_dtype is None else _one_of(_DTYPE, out_dtype, "out_dtype")
            out = torch.empty(shape, dtype=dt, device=device)
        elif out.shape != shape or (out_dtype is not None and
                                    out.dtype != _one_of(_DTYPE, out_dtype, "out_dtype")):
            raise ValueError(f"out: {out.dtype} {tuple(out.shape)}, not {tuple(shape)}")
        o2, _, os_ = _rows(out, "out", no)
        rp = rs = 0
        if residual is not None:
            if residual.shape != shape or residual.dtype != out.dtype:
                raise ValueError(f"residual: {residual.dtype} {tuple(residual.shape)}, not "
                                 f"{out.dtype} {tuple(shape)}")
            r2, _, rs = _rows(residual, "residual", no)
            rp = r2.data_ptr()
        xp, wp, ws = x2.data_ptr(), weight.data_ptr(), weight.stride(0)
        bp, bc = (0, 0) if bias is None else (bias.data_ptr(), _code(bias, "bias"))

        def pack(buf, size):
            return _LINEAR.pack(xp, wp, bp, rp, o2.data_ptr(), buf, size, t, n, k, xs, ws, rs,
                                os_, code, bc, _code(out, "out"), act, GATED if gated else 0, 0)
        buf = size = 0
        if (xp | wp | (xs | ws) * 2) & 15:
            need = _lib.ctypes.c_uint64()
            _check(lib, lib.cfa_linear_workspace(pack(0, 0), _lib.ctypes.byref(need)))
            if need.value:
                workspace = _workspace(workspace, need.value, device)
                buf, size = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        _check(lib, lib.cfa_linear_async(pack(buf, size), handle))
    return out


def route(logits, top_k, *, scoring="softmax", bias=None, groups=1, top_groups=1,
          renormalize=True, scale=1.0, out=None, stream=None):
    """Chooses top_k experts per token: (weights fp32 [..., top_k], ids int32 [..., top_k]).

    logits    [..., E] bf16, fp16 or fp32;  scoring "softmax" or "sigmoid"
    bias      [E] fp32, added to the scores for the choice alone
    groups    only experts of the top_groups best of `groups` groups of neighbours can be chosen; a
              group goes by its best key (softmax) or the sum of its two best (sigmoid)
    renormalize  divides the chosen scores by their sum;  scale multiplies them
    out       (weights, ids) to write into
    Equal keys go to the lowest index; an expert whose logit or key is -inf or NaN is never chosen,
    and places that no expert is left for hold id -1 and weight 0.
    """
    if torch is None:
        _start()
    device = logits.device
    _operands(device, logits=logits, bias=bias)
    e = logits.shape[-1] if logits.dim() else 0
    l2, t, ls = _rows(logits, "logits", e)
    if bias is not None and (bias.shape != (e,) or bias.dtype != torch.float32):
        raise ValueError(f"bias: {bias.dtype} {tuple(bias.shape)}, not float32 ({e},)")
    top_k = int(top_k)
    shape = logits.shape[:-1] + (top_k,)
    lib = _lib.load()
    with _enter(stream, device) as handle:
        if out is None:
            if top_k < 1:
                raise ValueError(f"top_k is {top_k}")
            weights = torch.empty(shape, dtype=torch.float32, device=device)
            ids = torch.empty(shape, dtype=torch.int32, device=device)
        else:
            weights, ids = out
            for o, dt, name in ((weights, torch.float32, "weights"), (ids, torch.int32, "ids")):
                if (o.shape != shape or o.dtype != dt or o.device != device or
                        not o.is_contiguous()):
                    raise ValueError(f"{name}: {o.dtype} {tuple(o.shape)}, not a contiguous {dt} "
                                     f"{tuple(shape)}")
        args = _ROUTE.pack(l2.data_ptr(), 0 if bias is None else bias.data_ptr(),
                           weights.data_ptr(), ids.data_ptr(), t, ls, e, top_k, groups,
                           top_groups, _code(logits, "logits"),
                           _one_of(SCORING, scoring, "scoring"),
                           RENORMALIZE if renormalize else 0, scale)
        _check(lib, lib.cfa_route_async(args, handle))
    return weights, ids


def experts(x, ids, weights, w13, w2, *, activation="silu", first_expert=0, residual=None,
            out=None, workspace=None, stream=None):
    """residual + the sum over each token's choices of weight * w2_e act(gate_e x) * (up_e x).

    x         [..., H] bf16 or fp16;  ids int32 and weights fp32 [..., top_k], as route() gives them
    w13       [E, 2 I, H] (gate rows, then up rows) or [E, I, H] (no gate);  w2 [E, H, I]: the
              experts first_expert .. first_expert + E - 1, as loaded.  Other ids add nothing
    residual  [..., H] of x's dtype; `out` may be the same tensor
    workspace  uint8 tensor of experts_workspace bytes (default: allocated)
    """
    if torch is None:
        _start()
    device = x.device
    _operands(device, x=x, ids=ids, weights=weights, w13=w13, w2=w2, residual=residual, out=out)
    if w13.dim() != 3 or w2.dim() != 3:
        raise ValueError(f"w13 {tuple(w13.shape)} and w2 {tuple(w2.shape)} have three dimensions")
    e, h, i = w2.shape
    gated = w13.shape == (e, 2 * i, h)
    if not gated and w13.shape != (e, i, h):
        raise ValueError(f"w13 {tuple(w13.shape)} does not fit w2 {tuple(w2.shape)}")
    if w13.dtype != x.dtype or w2.dtype != x.dtype:
        raise ValueError(f"w13 is {w13.dtype}, w2 {w2.dtype}, x {x.dtype}")
    if not (w13.is_contiguous() and w2.is_contiguous()):
        raise ValueError("w13 and w2 must be contiguous")
    x2, t, xs = _rows(x, "x", h)
    top_k = ids.shape[-1] if ids.dim() else 0
    if (ids.shape != x.shape[:-1] + (top_k,) or weights.shape != ids.shape or
            ids.dtype != torch.int32 or weights.dtype != torch.float32 or
            not (ids.is_contiguous() and weights.is_contiguous())):
        raise ValueError(f"ids {ids.dtype} {tuple(ids.shape)} and weights {weights.dtype} "
                         f"{tuple(weights.shape)} must be contiguous int32 and float32 "
                         f"{tuple(x.shape[:-1])} + (top_k,)")
    code = _code(x, "x")
    act = _one_of(ACTIVATION, activation, "activation")
    lib = _lib.load()
    with _enter(stream, device) as handle:
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=device)
        elif out.shape != x.shape or out.dtype != x.dtype:
            raise ValueError(f"out: {out.dtype} {tuple(out.shape)}, not {x.dtype} "
                             f"{tuple(x.shape)}")
        o2, _, os_ = _rows(out, "out", h)
        rp = rs = 0
        if residual is not None:
            if residual.shape != x.shape or residual.dtype != x.dtype:
                raise ValueError(f"residual: {residual.dtype} {tuple(residual.shape)}, not "
                                 f"{x.dtype} {tuple(x.shape)}")
            r2, _, rs = _rows(residual, "residual", h)
            rp = r2.data_ptr()

        def pack(buf, size):
            return _EXPERTS.pack(x2.data_ptr(), w13.data_ptr(), w2.data_ptr(), rp, ids.data_ptr(),
                                 weights.data_ptr(), o2.data_ptr(), buf, size, t, h, i, xs, rs,
                                 os_, e, first_expert, top_k, code, act, GATED if gated else 0)
        need = _lib.ctypes.c_uint64()
        _check(lib, lib.cfa_experts_workspace(pack(0, 0), _lib.ctypes.byref(need)))
        workspace = _workspace(workspace, need.value, device)
        _check(lib, lib.cfa_experts_async(
            pack(workspace.data_ptr(), workspace.numel() * workspace.element_size()), handle))
    return out


def op_status():
    """Raises CfaError if a wait inside a product's kernel has run out on the current device since the
    last call (the results since then are not valid).  Call it after waiting for the streams."""
    lib = _lib.load()
    _check(lib, lib.cfa_op_status())
