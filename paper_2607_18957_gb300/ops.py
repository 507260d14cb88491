"""Operators on the loaded layout (cfa_linear_async, cfa_route_async, cfa_experts_async of cfa.h):
the matrix product with a weight in its fused layout, the choice of experts, and the products with
stacked experts.  Forward passes for serving; argument marshalling only.

Every call enqueues on `stream` (a torch stream of the operands' device or a stream's handle; default:
torch's current stream there) and returns at once.  Outputs and
workspaces that a call makes come from torch's allocator, on that stream.  For the handle
cudaStreamPerThread, which torch takes for one stream, the calls and what they allocate are on a stream
of torch's that the thread keeps for it, in the order of the thread's own.  Operands are CUDA tensors
of one device whose last dimension is contiguous; rows may lie any distance apart.
"""
import struct
import threading

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
_CODE = None    # torch dtype -> CFA_DTYPE_*
_DTYPE = None   # dtype name -> torch dtype
_lib_c = None
_LINEAR_BYTES, _EXPERTS_BYTES = {}, {}  # workspace bytes by a call's sizes
_raw_stream = _device = _grad = None


def _start():
    global torch, _CODE, _DTYPE, _lib_c, _raw_stream, _device, _grad
    import torch as t
    _lib_c = _lib.load()
    _DTYPE = {"bf16": t.bfloat16, "f16": t.float16, "f32": t.float32}
    _CODE = {v: _lib.DTYPE[k] for k, v in _DTYPE.items()}
    _raw_stream, _device = t._C._cuda_getCurrentRawStream, t._C._cuda_getDevice
    _grad = t.is_grad_enabled
    torch = t


def _check(st):
    if st != _lib.CFA_OK:
        from . import _check as check
        check(st)


def _on(t, name, device):
    """Refuses an operand that is on another device, not contiguous in its last dimension, or part
    of a graph that a backward pass would need."""
    if device < 0 or t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{device}" if device >= 0 else
                         f"the operators run on CUDA tensors, not on {t.device}")
    if not t.is_contiguous() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    if t.requires_grad and _grad():
        raise ValueError(f"{name} requires a gradient, and the operators have no backward pass: "
                         "call them under torch.no_grad()")


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
    """A tensor [..., cols] as rows: (row count, row stride)."""
    shape = t.shape
    if len(shape) == 2:
        n, c = shape
        stride = t.stride(0)
    elif shape and shape[-1]:
        c = shape[-1]
        n = t.numel() // c
        stride = t.view(n, c).stride(0)  # raises where the rows do not lie evenly
    else:
        raise ValueError(f"{name}: shape {tuple(shape)}")
    if c != cols:
        raise ValueError(f"{name}: rows of {c}, not {cols}")
    return n, stride


PER_THREAD = 2  # cudaStreamPerThread
_thread = threading.local()


class _On:
    """A stream that a call enqueues on, current while the call allocates."""

    def __init__(self, stream, device):
        self.around = None
        if isinstance(stream, int):
            # torch takes the handle 0 for a request of one of its own streams, and does not know 1
            # (cudaStreamLegacy): both are the default stream
            handle, stream = stream, (torch.cuda.default_stream(device) if stream in (0, 1) else
                                      torch.cuda.ExternalStream(stream, device=device))
            if handle == PER_THREAD:
                # One handle, a stream in every thread: torch's allocator would give a thread what
                # another's kernels still use.  A stream of torch's stands in for the thread's own.
                self.around, own = stream, _thread.__dict__
                stream = own.get(device)
                if stream is None:
                    stream = own[device] = torch.cuda.Stream(device)
        self.stream = stream
        self.guard = torch.cuda.stream(stream)

    def __enter__(self):
        if self.around is not None:
            self.stream.wait_stream(self.around)
        self.guard.__enter__()

    def __exit__(self, *exc):
        self.guard.__exit__(*exc)
        if self.around is not None:
            self.around.wait_stream(self.stream)


def _elsewhere(stream, device):
    """The guard of a call that is not for the current device's current stream."""
    if stream is not None and not isinstance(stream, int) and stream.device.index != device:
        raise ValueError(f"the stream is on {stream.device}, the operands on cuda:{device}")
    return torch.cuda.device(device) if stream is None else _On(stream, device)


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
    device = x.get_device()
    if device < 0 or weight.get_device() != device or (
            _grad() and (x.requires_grad or weight.requires_grad)):
        _on(x, "x", device)
        _on(weight, "weight", device)
    if stream is not None or device != _device():
        with _elsewhere(stream, device):
            return linear(x, weight, bias, activation=activation, gated=gated, residual=residual,
                          out=out, out_dtype=out_dtype, workspace=workspace)
    wshape, xshape = weight.shape, x.shape
    if len(wshape) != 2:
        raise ValueError(f"weight: shape {tuple(wshape)}")
    n, k = wshape
    ws, one = weight.stride()
    if one != 1 and k > 1:
        _on(weight, "weight", device)
    if len(xshape) == 2 and xshape[1] == k:
        t = xshape[0]
        xs, one = x.stride()
        if one != 1 and k > 1:
            _on(x, "x", device)
    else:
        _on(x, "x", device)
        t, xs = _rows(x, "x", k)
    dtype = x.dtype
    code = _CODE.get(dtype) or _code(x, "x")
    if weight.dtype is not dtype:
        raise ValueError(f"weight is {weight.dtype}, x {dtype}")
    act = _one_of(ACTIVATION, activation, "activation")
    no = n
    if gated:
        if n % 2:
            raise ValueError(f"a gated weight has an even number of rows, not {n}")
        no = n // 2
    bp = bc = rp = rs = buf = size = 0
    if bias is not None:
        _on(bias, "bias", device)
        if bias.shape != (n,):
            raise ValueError(f"bias: shape {tuple(bias.shape)}, not ({n},)")
        bp, bc = bias.data_ptr(), _code(bias, "bias")
    shape = (t, no) if len(xshape) == 2 else xshape[:-1] + (no,)
    odtype, oc = dtype, code
    if out_dtype is not None:
        odtype = _one_of(_DTYPE, out_dtype, "out_dtype")
        oc = _CODE[odtype]
    if out is None:
        out = torch.empty(shape, dtype=odtype, device=x.device)
        os_ = no
    else:
        _on(out, "out", device)
        if out.shape != shape or (out_dtype is not None and out.dtype is not odtype):
            raise ValueError(f"out: {out.dtype} {tuple(out.shape)}, not {tuple(shape)}")
        odtype, oc = out.dtype, _code(out, "out")
        _, os_ = _rows(out, "out", no)
    if residual is not None:
        _on(residual, "residual", device)
        if residual.shape != shape or residual.dtype is not odtype:
            raise ValueError(f"residual: {residual.dtype} {tuple(residual.shape)}, not {odtype} "
                             f"{tuple(shape)}")
        _, rs = _rows(residual, "residual", no)
        rp = residual.data_ptr()
    xp, wp = x.data_ptr(), weight.data_ptr()
    if (xp | wp | (xs | ws) * 2) & 15:
        sizes = (t, n, k, xs, ws, xp & 15, wp & 15, gated)
        need = _LINEAR_BYTES.get(sizes)  # by the sizes and the alignment alone
        if need is None:
            size = _lib.ctypes.c_uint64()
            _check(_lib_c.cfa_linear_workspace(
                _LINEAR.pack(xp, wp, bp, rp, 0, 0, 0, t, n, k, xs, ws, rs, os_, code, bc, code,
                             act, GATED if gated else 0, 0), _lib.ctypes.byref(size)))
            if len(_LINEAR_BYTES) >= 1024:
                _LINEAR_BYTES.clear()
            need = _LINEAR_BYTES[sizes] = size.value
        size = 0
        if need:
            workspace = _workspace(workspace, need, x.device)
            buf, size = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    st = _lib_c.cfa_linear_async(
        _LINEAR.pack(xp, wp, bp, rp, out.data_ptr(), buf, size, t, n, k, xs, ws, rs, os_, code, bc,
                     oc, act, GATED if gated else 0, 0), _raw_stream(device))
    if st:
        _check(st)
    return out


def route(logits, top_k, *, scoring="softmax", bias=None, groups=1, top_groups=1,
          renormalize=True, scale=1.0, out=None, stream=None):
    """Chooses top_k experts per token: (weights fp32 [..., top_k], ids int32 [..., top_k]).

    logits    [..., E] bf16, fp16 or fp32;  scoring "softmax" or "sigmoid"
    bias      [E] fp32, added to the scores for the choice alone
    groups    only experts of the top_groups best of `groups` groups of neighbours can be chosen; a
              group goes by its best key (softmax) or the sum of its two best (sigmoid), of the
              experts that can be chosen at all
    renormalize  divides the chosen scores by their sum;  scale multiplies them
    out       (weights, ids) to write into
    Equal keys go to the lowest index; an expert whose logit or key is -inf or NaN is never chosen,
    and places that no expert is left for hold id -1 and weight 0.
    """
    if torch is None:
        _start()
    device = logits.get_device()
    if device < 0 or (logits.requires_grad and _grad()):
        _on(logits, "logits", device)
    if stream is not None or device != _device():
        with _elsewhere(stream, device):
            return route(logits, top_k, scoring=scoring, bias=bias, groups=groups,
                         top_groups=top_groups, renormalize=renormalize, scale=scale, out=out)
    lshape = logits.shape
    if len(lshape) == 2 and lshape[1]:
        t, e = lshape
        ls, one = logits.stride()
        if one != 1 and e > 1:
            _on(logits, "logits", device)
    else:
        _on(logits, "logits", device)
        e = lshape[-1] if lshape else 0
        t, ls = _rows(logits, "logits", e)
    bp = 0
    if bias is not None:
        _on(bias, "bias", device)
        if bias.shape != (e,) or bias.dtype is not torch.float32:
            raise ValueError(f"bias: {bias.dtype} {tuple(bias.shape)}, not float32 ({e},)")
        bp = bias.data_ptr()
    top_k = int(top_k)
    if top_k < 1:
        raise ValueError(f"top_k is {top_k}")
    shape = (t, top_k) if len(lshape) == 2 else lshape[:-1] + (top_k,)
    code = _CODE.get(logits.dtype) or _code(logits, "logits")
    score = _one_of(SCORING, scoring, "scoring") if scoring != "softmax" else 0
    if out is None:
        on = logits.device
        weights = torch.empty(shape, dtype=torch.float32, device=on)
        ids = torch.empty(shape, dtype=torch.int32, device=on)
    else:
        weights, ids = out
        for o, dt, name in ((weights, torch.float32, "weights"), (ids, torch.int32, "ids")):
            _on(o, name, device)
            if o.shape != shape or o.dtype is not dt or not o.is_contiguous():
                raise ValueError(f"{name}: {o.dtype} {tuple(o.shape)}, not a contiguous {dt} "
                                 f"{tuple(shape)}")
    st = _lib_c.cfa_route_async(
        _ROUTE.pack(logits.data_ptr(), bp, weights.data_ptr(), ids.data_ptr(), t, ls, e, top_k,
                    groups, top_groups, code, score, RENORMALIZE if renormalize else 0, scale),
        _raw_stream(device))
    if st:
        _check(st)
    return weights, ids


def experts(x, ids, weights, w13, w2, *, activation="silu", first_expert=0, residual=None,
            out=None, workspace=None, stream=None):
    """residual + the sum over each token's choices of weight * w2_e act(gate_e x) * (up_e x).

    x         [..., H] bf16 or fp16;  ids int32 and weights fp32 [..., top_k], as route() gives them
    w13       [E, 2 I, H] (gate rows, then up rows) or [E, I, H] (no gate);  w2 [E, H, I]: the
              experts first_expert .. first_expert + E - 1, as loaded.  Other ids add nothing
    residual  [..., H] of x's dtype; `out` may be the same tensor
    workspace  uint8 tensor (default: allocated; its size is cfa_experts_workspace of cfa.h)
    The values act(gate_e x) * (up_e x) are rounded to x's dtype between the two products (fp16: above
    65,504 they become infinite).
    """
    if torch is None:
        _start()
    device = x.get_device()
    if device < 0 or not (ids.get_device() == weights.get_device() == w13.get_device() ==
                          w2.get_device() == device) or (
            _grad() and (x.requires_grad or weights.requires_grad or w13.requires_grad or
                         w2.requires_grad)):
        for v, name in ((x, "x"), (ids, "ids"), (weights, "weights"), (w13, "w13"), (w2, "w2")):
            _on(v, name, device)
    if stream is not None or device != _device():
        with _elsewhere(stream, device):
            return experts(x, ids, weights, w13, w2, activation=activation,
                           first_expert=first_expert, residual=residual, out=out,
                           workspace=workspace)
    if not (ids.is_contiguous() and weights.is_contiguous() and w13.is_contiguous() and
            w2.is_contiguous()):
        raise ValueError("ids, weights, w13 and w2 must be contiguous")
    shape, ishape, w2shape, w13shape = x.shape, ids.shape, w2.shape, w13.shape
    if len(w2shape) != 3 or len(w13shape) != 3:
        raise ValueError(f"w13 {tuple(w13shape)} and w2 {tuple(w2shape)} have three dimensions")
    e, h, i = w2shape
    gated = w13shape[1] == 2 * i
    if w13shape[0] != e or w13shape[2] != h or not (gated or w13shape[1] == i):
        raise ValueError(f"w13 {tuple(w13shape)} does not fit w2 {tuple(w2shape)}")
    dtype = x.dtype
    if w13.dtype is not dtype or w2.dtype is not dtype:
        raise ValueError(f"w13 is {w13.dtype}, w2 {w2.dtype}, x {dtype}")
    _on(x, "x", device)
    t, xs = _rows(x, "x", h)
    top_k = ishape[-1] if ishape else 0
    if (ishape[:-1] != shape[:-1] or weights.shape != ishape or ids.dtype is not torch.int32 or
            weights.dtype is not torch.float32):
        raise ValueError(f"ids {ids.dtype} {tuple(ishape)} and weights {weights.dtype} "
                         f"{tuple(weights.shape)} must be int32 and float32 {tuple(shape[:-1])} + "
                         "(top_k,)")
    code = _CODE.get(dtype) or _code(x, "x")
    act = 4 if activation == "silu" else _one_of(ACTIVATION, activation, "activation")
    on = x.device
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=on)
        os_ = h
    else:
        _on(out, "out", device)
        if out.shape != shape or out.dtype is not dtype:
            raise ValueError(f"out: {out.dtype} {tuple(out.shape)}, not {dtype} {tuple(shape)}")
        _, os_ = _rows(out, "out", h)
    rp = rs = 0
    if residual is not None:
        _on(residual, "residual", device)
        if residual.shape != shape or residual.dtype is not dtype:
            raise ValueError(f"residual: {residual.dtype} {tuple(residual.shape)}, not {dtype} "
                             f"{tuple(shape)}")
        _, rs = _rows(residual, "residual", h)
        rp = residual.data_ptr()
    ptrs = (x.data_ptr(), w13.data_ptr(), w2.data_ptr(), rp, ids.data_ptr(), weights.data_ptr(),
            out.data_ptr())
    flags = GATED if gated else 0
    sizes = (t, h, i, e, top_k)
    need = _EXPERTS_BYTES.get(sizes)  # by the sizes alone
    if need is None or code not in (2, 3):
        size = _lib.ctypes.c_uint64()
        _check(_lib_c.cfa_experts_workspace(
            _EXPERTS.pack(*ptrs, 0, 0, t, h, i, xs, rs, os_, e, first_expert, top_k, code, act,
                          flags), _lib.ctypes.byref(size)))
        if len(_EXPERTS_BYTES) >= 1024:
            _EXPERTS_BYTES.clear()
        need = _EXPERTS_BYTES[sizes] = size.value
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=on)
    else:
        _workspace(workspace, need, on)
    st = _lib_c.cfa_experts_async(
        _EXPERTS.pack(*ptrs, workspace.data_ptr(), workspace.numel() * workspace.element_size(), t,
                      h, i, xs, rs, os_, e, first_expert, top_k, code, act, flags),
        _raw_stream(device))
    if st:
        _check(st)
    return out


def op_status():
    """Raises CfaError if a wait inside a product's kernel has run out on the current device since the
    calling thread's last call (the results since then are not valid), whichever thread or stream it
    belongs to.  Call it after waiting for the streams."""
    _check(_lib.load().cfa_op_status())
