"""Operators of a decoding step around the products (cfa_norm_async, cfa_append_async, cfa_attend_async
and cfa_logprobs_async of cfa.h): the norms between blocks, the rotation of queries and keys with the way
of keys and values into a paged cache, the attention over that cache, and the log probabilities of
tokens.  Forward passes for serving; argument marshalling only.

As the operators of ops.py, the calls enqueue on `stream` (a torch stream of the operands' device or a
stream's handle; default: torch's current stream there) and return at once; outputs and workspaces that
a call makes come from torch's allocator, on that stream.  attend keeps its workspace for the stream's next
call (a captured call gets one of its own, which the graph keeps).
"""
import math
import struct

from . import _lib, ops
from .ops import ACTIVATION, _check, _code, _elsewhere, _on, _one_of, _rows

__all__ = ["norm", "append", "attend", "logprobs", "rotary_frequencies"]

F8_E4M3 = 9  # CFA_DTYPE_F8_E4M3
INTERLEAVED = 0x1

_NORM = struct.Struct("<7Q7q3iI3fi")
_APPEND = struct.Struct("<7Q9q8iI3f")
_ATTEND = struct.Struct("<9Q10q10iI3f")
_LOGPROBS = struct.Struct("<6Q3q2ifI")
SIZES = {"cfa_norm_args": _NORM.size, "cfa_append_args": _APPEND.size,
         "cfa_attend_args": _ATTEND.size,
         "cfa_logprobs_args": _LOGPROBS.size}
_ATTEND_BYTES = {}  # workspace bytes by a call's sizes
_KEPT = {}          # attend's workspaces, by device and stream of torch's: its calls there follow one another
_FOREIGN = {}       # those of streams that are not torch's, by device and handle: (workspace, last call's end)


def _like(t, name, device, shape, dtype, cols):
    """(address, row stride) of an operand that is shaped and typed like another."""
    if t.get_device() != device or t.requires_grad:
        _on(t, name, device)
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, not {dtype} {tuple(shape)}")
    if t.is_contiguous():
        return t.data_ptr(), cols
    _on(t, name, device)
    return t.data_ptr(), _rows(t, name, cols)[1]


def norm(x, weight, *, residual=None, gate=None, activation="silu", post_weight=None, scale=1.0,
         eps=1e-6, offset=0.0, out=None, stream=None):
    """N(h) * (offset + weight) of h = residual + scale * act(gate) * a, N(v) = v / sqrt(mean(v^2) + eps):
    y, or with a residual (y, h).

    x         [..., C] bf16, fp16 or fp32: what the block gave
    a         x, or with a post_weight (a norm behind the block) N(x) * (offset + post_weight)
    gate      like x, or [C]: multiplies a by activation(gate) ("none", "relu", "gelu", "gelu_tanh",
              "silu")
    residual  like x: the stream that the block adds to
    weight, post_weight  [C], both of x's dtype or both fp32
    out       y, or with a residual (y, h), to write into: each may be x, the residual or a gate like x
    """
    if ops.torch is None:
        ops._start()
    device = x.get_device()
    if device < 0 or weight.get_device() != device or (
            ops._grad() and (x.requires_grad or weight.requires_grad)):
        _on(x, "x", device)
        _on(weight, "weight", device)
    if stream is not None or device != ops._device():
        with _elsewhere(stream, device):
            return norm(x, weight, residual=residual, gate=gate, activation=activation,
                        post_weight=post_weight, scale=scale, eps=eps, offset=offset, out=out)
    shape, dtype = x.shape, x.dtype
    cols = shape[-1] if shape else 0
    if len(shape) == 2 and cols:
        t = shape[0]
        xs, one = x.stride()
        if one != 1 and cols > 1:
            _on(x, "x", device)
    else:
        _on(x, "x", device)
        t, xs = _rows(x, "x", cols)
    code = ops._CODE.get(dtype) or _code(x, "x")
    if weight.shape != (cols,):
        raise ValueError(f"weight: shape {tuple(weight.shape)}, not ({cols},)")
    if not weight.is_contiguous():
        _on(weight, "weight", device)
    wcode = ops._CODE.get(weight.dtype) or _code(weight, "weight")
    pp = rp = rs = gp = gs = hp = hs = act = 0
    if post_weight is not None:
        _on(post_weight, "post_weight", device)
        if post_weight.shape != (cols,) or post_weight.dtype is not weight.dtype:
            raise ValueError(f"post_weight: {post_weight.dtype} {tuple(post_weight.shape)}, not "
                             f"{weight.dtype} ({cols},)")
        pp = post_weight.data_ptr()
    if gate is not None:
        act = _one_of(ACTIVATION, activation, "activation")
        if gate.shape == (cols,) and len(shape) > 1:
            _on(gate, "gate", device)
            if gate.dtype is not dtype:
                raise ValueError(f"gate: {gate.dtype}, not {dtype}")
            gp = gate.data_ptr()
        else:
            gp, gs = _like(gate, "gate", device, shape, dtype, cols)
    if residual is not None:
        rp, rs = _like(residual, "residual", device, shape, dtype, cols)
    y = h = None
    if out is None:
        torch = ops.torch
        y = torch.empty(shape, dtype=dtype, device=x.device)
        ys = cols
        if residual is not None:
            h = torch.empty(shape, dtype=dtype, device=x.device)
            hp, hs = h.data_ptr(), cols
        yp = y.data_ptr()
    else:
        if residual is not None:
            y, h = out
            hp, hs = _like(h, "h", device, shape, dtype, cols)
        else:
            y = out
        yp, ys = _like(y, "y", device, shape, dtype, cols)
    st = ops._lib_c.cfa_norm_async(
        _NORM.pack(x.data_ptr(), rp, gp, weight.data_ptr(), pp, yp, hp, t, cols, xs, rs, gs, ys, hs,
                   code, wcode, act, 0, scale, eps, offset, 0), ops._raw_stream(device))
    if st:
        _check(st)
    return y if residual is None else (y, h)


def rotary_frequencies(dim, base=10000.0, *, scaling=None, factor=1.0, length=None, low=1.0, high=4.0,
                       fast=32.0, slow=1.0, magnitude=None):
    """Frequencies of append() for `dim` rotated values of a head: (a list of dim / 2 radians per
    position, magnitude).  base ** (-2 i / dim), and for contexts `factor` times longer

    scaling   None; "linear": every frequency divided by factor; "base": a larger base, so that the last
              frequency is divided by factor and the first by one; "bands": with t the turns that a
              pair makes within `length` positions, pairs of t >= high keep their frequency, those of
              t <= low have it divided, between them smoothly; "ramp": the same, linear in the pair's
              index from the one that turns `fast` times, rounded down but not below 0, to the one that
              turns `slow` times, rounded up, which may lie behind the last pair; and queries and keys
              grow by `magnitude` (default 0.1 ln factor + 1)
    """
    if dim < 2 or dim % 2:
        raise ValueError(f"{dim} values do not make pairs")
    if not (base > 1.0 and factor >= 1.0):
        raise ValueError(f"base {base}, factor {factor}")
    half = dim // 2
    if scaling == "base" and dim > 2:
        base = base * factor ** (dim / (dim - 2))
    f = [base ** (-i / half) for i in range(half)]
    grow = 1.0
    if scaling == "linear":
        f = [v / factor for v in f]
    elif scaling in ("bands", "ramp"):
        if not length:
            raise ValueError(f"scaling {scaling!r} goes by the length of the original contexts")
        if scaling == "bands":
            if not low < high:
                raise ValueError(f"low {low} turns, high {high}")
            kept = [(length * v / (2 * math.pi) - low) / (high - low) for v in f]
        else:
            def index(turns):
                return half * math.log(length / (turns * 2 * math.pi)) / math.log(base)
            first, last = max(math.floor(index(fast)), 0), math.ceil(index(slow))
            kept = [1.0 - (i - first) / max(last - first, 1e-3) for i in range(half)]
            grow = 0.1 * math.log(factor) + 1.0
        kept = [min(max(k, 0.0), 1.0) for k in kept]
        f = [v * (k + (1.0 - k) / factor) for v, k in zip(f, kept)]
    elif scaling not in (None, "base"):
        raise ValueError(f"unknown scaling {scaling!r}: one of linear, base, bands, ramp")
    return f, grow if magnitude is None else magnitude


def _ints(t, name, device, shape):
    """The address of an int32 operand."""
    if t.get_device() != device:
        _on(t, name, device)
    if t.shape != shape or t.dtype is not ops.torch.int32 or not t.is_contiguous():
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, not a contiguous torch.int32 "
                         f"{tuple(shape)}")
    return t.data_ptr()


def _cache(k, v, dtype, code, device):
    """Checks a paged cache: (its dtype's code, the strides of k and of v)."""
    ks, vs = k.stride(), v.stride()
    if (k.get_device() != device or v.get_device() != device or ks[-1] != 1 or vs[-1] != 1 or
            k.requires_grad or v.requires_grad):
        _on(k, "k_cache", device)
        _on(v, "v_cache", device)
    if len(ks) != 4 or v.shape != k.shape or v.dtype is not k.dtype:
        raise ValueError(f"k_cache {k.dtype} {tuple(k.shape)} and v_cache {v.dtype} {tuple(v.shape)} "
                         "are both [pages, page_size, kv_heads, head_dim]")
    if k.dtype is not dtype:
        if k.dtype is not ops.torch.float8_e4m3fn:
            raise ValueError(f"the cache is {k.dtype}, not {dtype} or torch.float8_e4m3fn")
        code = F8_E4M3
    return code, ks[:3], vs[:3]


def append(qkv, k_cache, v_cache, slots, *, heads, positions=None, frequencies=None,
           interleaved=False, magnitude=1.0, k_scale=1.0, v_scale=1.0, out=None, stream=None):
    """Turns queries and keys by their positions and appends keys and values to a paged cache: the
    turned queries [T, heads, D].

    qkv       [T, (heads + 2 KV) D] bf16 or fp16, as linear() gives it with a fused q/k/v weight
    k_cache, v_cache  [pages, page_size, KV, D] of any strides with D contiguous, of qkv's dtype or
              torch.float8_e4m3fn, which holds values divided by k_scale or v_scale
    slots     [T] int32, page * page_size + place; a token whose slot is negative or behind the last page
              is not appended
    positions [T] int32;  frequencies [R / 2] fp64, radians per position (rotary_frequencies()): the first
              R <= D values of a head turn, in pairs (i, i + R / 2) or, interleaved, (2 i, 2 i + 1),
              and grow by `magnitude`.  Without them nothing turns, and the result is qkv's own part
    out       [T, heads, D] to write the queries into; may be qkv's own part
    """
    if ops.torch is None:
        ops._start()
    torch = ops.torch
    device = qkv.get_device()
    if device < 0 or qkv.requires_grad:
        _on(qkv, "qkv", device)
    if stream is not None or device != ops._device():
        with _elsewhere(stream, device):
            return append(qkv, k_cache, v_cache, slots, heads=heads, positions=positions,
                          frequencies=frequencies, interleaved=interleaved, magnitude=magnitude,
                          k_scale=k_scale, v_scale=v_scale, out=out)
    dtype, shape = qkv.dtype, qkv.shape
    code = ops._CODE.get(dtype) or _code(qkv, "qkv")
    ccode, ks, vs = _cache(k_cache, v_cache, dtype, code, device)
    pages, page_size, kv, dim = k_cache.shape
    if heads < 1 or len(shape) != 2 or shape[1] != (heads + 2 * kv) * dim:
        raise ValueError(f"qkv: {tuple(shape)}, not rows of ({heads} + 2 * {kv}) * {dim}")
    t = shape[0]
    xs, one = qkv.stride()
    if one != 1:
        _on(qkv, "qkv", device)
    sp = _ints(slots, "slots", device, (t,))
    if (positions is None) != (frequencies is None):
        raise ValueError("positions and frequencies belong together")
    pp = fp = qp = qs = rot = 0
    if positions is not None:
        pp = _ints(positions, "positions", device, (t,))
        if (frequencies.get_device() != device or not frequencies.is_contiguous() or
                frequencies.requires_grad):
            _on(frequencies, "frequencies", device)
        pairs = frequencies.shape
        if frequencies.dtype is not torch.float64 or len(pairs) != 1:
            raise ValueError(f"frequencies: {frequencies.dtype} {tuple(pairs)}, not torch.float64 "
                             "(R / 2,)")
        rot = 2 * pairs[0]
        fp = frequencies.data_ptr()
    shape = (t, heads, dim)
    if out is not None:
        _on(out, "out", device)
        if out.shape != shape or out.dtype is not dtype or (heads > 1 and out.stride(1) != dim):
            raise ValueError(f"out: {out.dtype} {tuple(out.shape)}, not {dtype} {shape} with rows of "
                             f"{heads * dim}")
        q, qp, qs = out, out.data_ptr(), out.stride(0)
    elif rot:
        q = torch.empty(shape, dtype=dtype, device=qkv.device)
        qp, qs = q.data_ptr(), heads * dim
    else:
        q = qkv[:, :heads * dim].unflatten(1, (heads, dim))
    st = ops._lib_c.cfa_append_async(
        _APPEND.pack(qkv.data_ptr(), pp, sp, fp, qp, k_cache.data_ptr(), v_cache.data_ptr(), t, xs, qs,
                     *ks, *vs, pages, page_size, heads, kv, dim, rot, code, ccode,
                     INTERLEAVED if interleaved else 0, magnitude, k_scale, v_scale),
        ops._raw_stream(device))
    if st:
        _check(st)
    return q


def _kept(device, on, need):
    """A workspace for calls on the current stream, whose handle is `on`, that has none large enough:
    (the workspace, an event to record behind the call or None).

    torch's streams live as long as the process.  Any other's handle may be another stream's by now,
    while the first one's last call is still under way: calls there wait for the one before."""
    torch, key = ops.torch, (device, on)
    stream = torch.cuda.current_stream(device)

    def empty():
        return torch.empty(need, dtype=torch.uint8, device=stream.device)
    if not on or stream.stream_id != on:
        if len(_KEPT) >= 64:
            _KEPT.clear()
        workspace = _KEPT[key] = empty()
        return workspace, None
    workspace, last = _FOREIGN.get(key, (None, None))
    if last is not None:
        stream.wait_event(last)
    else:
        last = torch.cuda.Event()
        if len(_FOREIGN) >= 64:  # the oldest one's memory is free once its last call is over
            old, end = _FOREIGN.pop(list(_FOREIGN)[0], (None, None))
            if old is not None:
                stream.wait_event(end)
                old.record_stream(stream)
    if workspace is None or workspace.numel() < need:
        workspace = empty()
    _FOREIGN[key] = workspace, last
    return workspace, last


def attend(q, k_cache, v_cache, pages, lengths, *, scale=None, window=0, k_scale=1.0, v_scale=1.0,
           lse=False, out=None, workspace=None, stream=None):
    """Attention of new tokens over a paged cache that holds their keys and values already: like q, or
    with lse=True (that, log of the sum of the exponentials fp32 [B, (N,) heads]).

    q         [B, heads, D], one new token of each of B sequences, or [B, N, heads, D], a few; bf16 or
              fp16, D 64, 96, 128 or 256
    k_cache, v_cache  as append() fills them; 8-bit values count k_scale and v_scale times
    pages     [B, P] int32: key j of a sequence is in page pages[b, j // page_size] at place j % page_size.
              The keys of a page whose number is not in the cache are not there
    lengths   [B] int32: keys of each sequence, the new tokens' among them.  Token i of N sees those up to
              lengths - N + i, with a window only the last `window` of them; one that sees none gets 0
              and -inf
    scale     of the scores (default: D ** -0.5)
    out       like q; with lse=True (out, lse)
    workspace  uint8 tensor (default: the stream's; its size is cfa_attend_workspace of cfa.h), of which
              calls that may overlap need one each
    """
    if ops.torch is None:
        ops._start()
    torch = ops.torch
    device = q.get_device()
    if device < 0 or q.requires_grad:
        _on(q, "q", device)
    if stream is not None or device != ops._device():
        with _elsewhere(stream, device):
            return attend(q, k_cache, v_cache, pages, lengths, scale=scale, window=window,
                          k_scale=k_scale, v_scale=v_scale, lse=lse, out=out, workspace=workspace)
    on = ops._raw_stream(device)
    if on == ops.PER_THREAD:  # torch's current stream: its workspace is to be the thread's all the same
        return attend(q, k_cache, v_cache, pages, lengths, scale=scale, window=window, k_scale=k_scale,
                      v_scale=v_scale, lse=lse, out=out, workspace=workspace, stream=on)
    shape, dtype = q.shape, q.dtype
    code = ops._CODE.get(dtype) or _code(q, "q")
    ccode, ks, vs = _cache(k_cache, v_cache, dtype, code, device)
    cache_pages, page_size, kv, dim = k_cache.shape
    if len(shape) == 3:
        (b, heads, d), new = shape, 1
    elif len(shape) == 4:
        b, new, heads, d = shape
    else:
        raise ValueError(f"q: shape {tuple(shape)}")
    if d != dim:
        raise ValueError(f"q has heads of {d}, the cache of {dim}")
    if q.is_contiguous():
        qs = heads * dim
    else:
        _on(q, "q", device)
        if heads > 1 and q.stride(-2) != dim:
            raise ValueError("q: the heads of a token must lie side by side")
        qs = (q if len(shape) == 3 else q.view(b * new, heads, d)).stride(0)
    table = pages.shape
    if pages.get_device() != device or not pages.is_contiguous():
        _on(pages, "pages", device)
    if len(table) != 2 or table[0] != b or pages.dtype is not torch.int32:
        raise ValueError(f"pages: {pages.dtype} {tuple(table)}, not torch.int32 ({b}, P)")
    np_ = _ints(lengths, "lengths", device, (b,))
    lp, sums = 0, None
    if out is None:
        o = torch.empty(shape, dtype=dtype, device=q.device)
        os_ = heads * dim
        if lse:
            sums = torch.empty(shape[:-1], dtype=torch.float32, device=q.device)
    else:
        if lse:
            o, sums = out
            _on(sums, "lse", device)
            if (sums.shape != shape[:-1] or sums.dtype is not torch.float32 or
                    not sums.is_contiguous()):
                raise ValueError(f"lse: {sums.dtype} {tuple(sums.shape)}, not a contiguous "
                                 f"torch.float32 {tuple(shape[:-1])}")
        else:
            o = out
        _on(o, "out", device)
        if o.shape != shape or o.dtype is not dtype or (heads > 1 and o.stride(-2) != dim):
            raise ValueError(f"out: {o.dtype} {tuple(o.shape)}, not {dtype} {tuple(shape)} with the heads "
                             "of a token side by side")
        os_ = (o if len(shape) == 3 else o.view(b * new, heads, dim)).stride(0)
    if lse:
        lp = sums.data_ptr()
    if scale is None:
        scale = dim ** -0.5

    sizes = (new, heads, kv, dim)
    need = _ATTEND_BYTES.get(sizes)
    args = (b, qs, os_, pages.stride(0), *ks, *vs, new, table[1], cache_pages, page_size, heads, kv,
            dim, window, code, ccode, 0, scale, k_scale, v_scale)
    ptrs = (q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), pages.data_ptr(), np_, o.data_ptr(), lp)
    if need is None:
        size = _lib.ctypes.c_uint64()
        _check(ops._lib_c.cfa_attend_workspace(_ATTEND.pack(*ptrs, 0, 0, *args),
                                               _lib.ctypes.byref(size)))
        if len(_ATTEND_BYTES) >= 1024:
            _ATTEND_BYTES.clear()
        need = _ATTEND_BYTES[sizes] = size.value
    last = None
    if workspace is not None:
        ops._workspace(workspace, need, q.device)
        need = workspace.numel() * workspace.element_size()
    elif torch.cuda.is_current_stream_capturing():
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    else:
        workspace = _KEPT.get((device, on))
        if workspace is None or workspace.numel() < need:
            workspace, last = _kept(device, on, need)
    st = ops._lib_c.cfa_attend_async(_ATTEND.pack(*ptrs, workspace.data_ptr(), need, *args), on)
    if last is not None:
        last.record(torch.cuda.current_stream(device))
    if st:
        _check(st)
    return (o, sums) if lse else o


def logprobs(logits, tokens, *, top=0, scale=1.0, out=None, stream=None):
    """Log probabilities of a token per row under softmax(scale * logits): (logprobs, entropy), fp32
    [...]; with top > 0 also (.., top_logprobs fp32 [..., top], top_ids int32 [..., top]), the largest
    logits in descending order, equal ones by their index.

    logits    [..., V] bf16, fp16 or fp32;  tokens [...] int32: below 0 gives 0 (a padded row)
    top       0 to 32;  scale  the inverse temperature
    out       the same tuple to write into
    """
    if ops.torch is None:
        ops._start()
    torch = ops.torch
    device = logits.get_device()
    if device < 0 or logits.requires_grad:
        _on(logits, "logits", device)
    if stream is not None or device != ops._device():
        with _elsewhere(stream, device):
            return logprobs(logits, tokens, top=top, scale=scale, out=out)
    shape = logits.shape
    if len(shape) == 2 and shape[1]:
        rows, cols = shape
        xs, one = logits.stride()
        if one != 1 and cols > 1:
            _on(logits, "logits", device)
    else:
        _on(logits, "logits", device)
        cols = shape[-1] if shape else 0
        rows, xs = _rows(logits, "logits", cols)
    code = ops._CODE.get(logits.dtype) or _code(logits, "logits")
    lead = shape[:-1]
    tp = _ints(tokens, "tokens", device, lead)
    top = int(top)
    if out is None:
        on, f32 = logits.device, torch.float32
        out = (torch.empty(lead, dtype=f32, device=on), torch.empty(lead, dtype=f32, device=on))
        if top:
            if top < 0:
                raise ValueError(f"top is {top}")
            best = lead + (top,)
            out += (torch.empty(best, dtype=f32, device=on),
                    torch.empty(best, dtype=torch.int32, device=on))
    else:
        out = tuple(out)
        want = [(lead, torch.float32), (lead, torch.float32)]
        if top:
            want += [(lead + (top,), torch.float32), (lead + (top,), torch.int32)]
        if len(out) != len(want):
            raise ValueError(f"out: {len(out)} tensors, not {len(want)}")
        for o, (sh, dt) in zip(out, want):
            _on(o, "out", device)
            if o.shape != sh or o.dtype is not dt or not o.is_contiguous():
                raise ValueError(f"out: {o.dtype} {tuple(o.shape)}, not a contiguous {dt} {tuple(sh)}")
    st = ops._lib_c.cfa_logprobs_async(
        _LOGPROBS.pack(logits.data_ptr(), tp, out[0].data_ptr(), out[1].data_ptr(),
                       out[2].data_ptr() if top else 0, out[3].data_ptr() if top else 0, rows, cols, xs,
                       code, top, scale, 0), ops._raw_stream(device))
    if st:
        _check(st)
    return out
