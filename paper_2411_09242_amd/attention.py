"""Token-by-token generation beside the planned graphs: a paged key/value
cache held in 4 bits, attention over it, attention with a sliding window
and a few first tokens that stay visible, linear attention with a decay, and
rotary positions (ctypes binding of include/fluid_attention.h).

    kv_write(pool, pages, k, v, start, count)   quantise new tokens into the cache
    kv_read(pool, pages, start, k, v, count)    its values as ordinary tensors
    kv_attention(pool, pages, q, kv_len, ...)   queries over the cache
    attention(q, k, v, ...)                     queries over ordinary keys and values
    KvCache                                     pool, page table and lengths of a batch
    linear_attention(q, k, v, decay, ...)       attention with a state instead of a cache
    Rotary, rotary(turns, q, k, ...)            queries and keys turned by their positions

Tensors of tokens are torch tensors [batch, tokens, heads, head_dim] in fp32
or bf16 on the GPU, with any strides and contiguous channels; lengths, starts
and page tables are int32 tensors on the GPU.  Calls enqueue kernels on
torch's current stream, or on ``stream`` (a torch stream or a raw handle), and
return without waiting.  With ``stream`` the caller orders the call behind what
makes its tensors and before what uses the result (``wait_stream``); the tensors'
memory is not handed out again before the call has run.  Arguments that cannot be right raise ``FluidError``
before anything is launched, and so do tensors that want gradients.  What a window has left behind may be freed: page
table entries outside the pool hold no tokens.
"""
from __future__ import annotations

import ctypes as C
import math

from . import fluid

_VP, _I32, _U64 = C.c_void_p, C.c_int32, C.c_uint64

PAGE_TOKENS = (32, 64, 128, 256, 512, 1024)


class Tokens(C.Structure):
    _fields_ = [("dtype", _I32), ("batch", _I32), ("tokens", _I32), ("heads", _I32), ("head_dim", _I32),
                ("stride", C.c_int64 * 3)]


class CacheDesc(C.Structure):
    _fields_ = [("n_pages", _I32), ("page_tokens", _I32), ("kv_heads", _I32), ("head_dim", _I32), ("batch", _I32),
                ("max_pages", _I32), ("table_stride", C.c_int64)]


class Opts(C.Structure):
    _fields_ = [("scale", C.c_float), ("causal", _I32), ("window", _I32), ("sinks", _I32)]


class RotaryDesc(C.Structure):
    _fields_ = [("dim", _I32), ("interleaved", _I32), ("scaling", _I32), ("amplitude", C.c_float)] + [
        (name, C.c_double) for name in ("base", "factor", "length", "low", "high")]


_PROTOS = {
    "fluid_kv_pool_bytes": [_VP, _VP],
    "fluid_kv_write": [_VP] * 10,
    "fluid_kv_read": [_VP] * 10,
    "fluid_kv_attention_workspace": [_VP, _VP, _I32, _VP, _VP],
    "fluid_kv_attention": [_VP, _VP, _VP, _VP, _I32, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _U64, _VP],
    "fluid_attention_workspace": [_VP] * 4,
    "fluid_attention": [_VP] * 12 + [_U64, _VP],
    "fluid_rotary_turns": [_VP] * 2,
    "fluid_rotate": [_VP] * 4 + [C.c_int64, _VP, _I32] + [_VP] * 9,
    "fluid_linear_attention_workspace": [_VP] * 3,
    "fluid_linear_attention": [C.c_float] + [_VP] * 14 + [_U64, _VP],
}
SYMBOLS = tuple(_PROTOS)

_bound = None


def _lib():
    """The library that ``fluid.load`` chose, with this header's prototypes."""
    global _bound
    lib = fluid._L()
    if _bound is not lib:
        for name, args in _PROTOS.items():
            f = getattr(lib, name)
            f.restype = C.c_int
            f.argtypes = args
        _bound = lib
    return lib


def _refuse(msg):
    raise fluid.FluidError(-1, msg)


def _torch():
    import torch
    return torch


def _describe(t, name, device):
    """fluid_tokens of a tensor, or a refusal."""
    torch = _torch()
    if t.dim() != 4:
        _refuse(f"{name}: a tensor [batch, tokens, heads, head_dim] is needed, got {t.dim()} dimensions")
    if t.get_device() != device:
        _refuse(f"{name}: on {t.device}, not on GPU {device}")
    if t.dtype not in (torch.float32, torch.bfloat16):
        _refuse(f"{name}: dtype must be float32 or bfloat16, got {t.dtype}")
    shape, stride = t.shape, t.stride()
    if stride[3] != 1 and shape[3] > 1:
        _refuse(f"{name}: channels must be contiguous")
    if max(shape) >= 1 << 31:
        _refuse(f"{name}: too large")
    return Tokens(fluid.F32 if t.dtype == torch.float32 else fluid.BF16, *shape, (C.c_int64 * 3)(*stride[:3]))


def _check_ints(t, name, n, device):
    """Refuses what is no int32 tensor of n values; None is none."""
    if t is None:
        return
    if (t.dtype != _torch().int32 or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1)
            or t.get_device() != device):
        _refuse(f"{name}: {n} contiguous int32 values on GPU {device} are needed")


def _describe_cache(pool, pages, head_dim, device):
    torch = _torch()
    if pool.dim() != 3 or pool.dtype != torch.uint8 or not pool.is_contiguous():
        _refuse("pool: a contiguous uint8 tensor [pages, kv_heads, block] is needed")
    if pages.dim() != 2 or pages.dtype != torch.int32 or (pages.shape[1] > 1 and pages.stride(1) != 1):
        _refuse("pages: an int32 tensor [batch, max_pages] with contiguous rows is needed")
    if pool.get_device() != device or pages.get_device() != device:
        _refuse(f"pool, pages: on {pool.device} and {pages.device}, not on GPU {device}")
    n, heads, block = pool.shape
    tokens = block * 4 // (5 * head_dim) if head_dim else 0
    if block * 4 != 5 * head_dim * tokens or tokens not in PAGE_TOKENS:
        _refuse(f"pool: a block of {block} bytes is no page of head_dim {head_dim}")
    stride = pages.stride(0) if pages.shape[0] > 1 else pages.shape[1]
    return CacheDesc(n, tokens, heads, head_dim, pages.shape[0], pages.shape[1], stride)


def _describe_opts(scale, causal, window, sinks, head_dim):
    for name, v in (("window", window), ("sinks", sinks)):
        if not 0 <= v < 1 << 31:
            _refuse(f"{name}: {v} is out of range")
    return Opts(1.0 / math.sqrt(head_dim) if scale is None else scale, 1 if causal else 0, window, sinks)


# A call's checks and descriptions depend on its tensors' types, shapes,
# strides and devices and on its numbers alone, and a decoding loop makes the
# same few calls over and over: they are made once for each such set.  (Filling
# and checking them takes 9 us, as long as a small kernel; finding them, 2.)
# kv_max, which grows from step to step, is no part of the set: it decides the
# workspace alone, whose size is asked for again where kv_max is another.
_calls = {}


def _form(t):
    return None if t is None else (t.dtype, t.shape, t.stride(), t.get_device())


def _keep(key, made):
    if len(_calls) >= 4096:
        _calls.clear()
    _calls[key] = made
    return made


def _check_grad(*tensors):
    """Refuses tensors that want gradients, which no call here computes."""
    if any(t.requires_grad for t in tensors) and _torch().is_grad_enabled():
        _refuse("a tensor requires gradients, and there is no backward pass: detach it, or call under torch.no_grad()")


def _device_of(t, name):
    if not t.is_cuda:
        _refuse(f"{name}: a tensor on the GPU is needed, got {t.device}")
    return t.get_device()


def _as_stream(stream, device):
    return stream if hasattr(stream, "cuda_stream") else _torch().cuda.ExternalStream(stream, device=device)


def _record(stream, device, *tensors):
    """Keeps tensors that their owner drops until `stream` is done with them:
    torch hands memory out again in the order of its own stream alone."""
    s = _as_stream(stream, device)
    for t in tensors:
        if t is not None:
            t.record_stream(s)


def _stream(stream, device):
    if stream is None:
        return _torch().cuda.current_stream(device).cuda_stream
    return getattr(stream, "cuda_stream", stream)


try:  # the same handle without a Stream object around it
    from torch._C import _cuda_getCurrentRawStream as _raw_stream
except ImportError:
    def _raw_stream(device):
        return _stream(None, device)


try:
    from torch._C import _cuda_getDevice as _current_device
except ImportError:
    def _current_device():
        return _torch().cuda.current_device()


def _launch(f, device, *args):
    """f(*args) with the tensors' GPU as the current one, as launches need it."""
    if _current_device() == device:
        st = f(*args)
    else:
        with _torch().cuda.device(device):
            st = f(*args)
    if st:
        fluid._check(st)


def _addr(d):
    return C.addressof(d)


def pool_block(page_tokens, head_dim):
    """Bytes of one page of one kv head."""
    return 5 * head_dim * page_tokens // 4


def _io_call(pool, pages, k, v, start, count):
    dev = _device_of(pool, "pool")
    kd, vd = _describe(k, "k", dev), _describe(v, "v", dev)
    c = _describe_cache(pool, pages, k.shape[3], dev)
    _check_ints(start, "start", pages.shape[0], dev)
    _check_ints(count, "count", pages.shape[0], dev)
    if start is None:
        _refuse("start: needed")
    return (_lib(), dev, _addr(c), _addr(kd), _addr(vd), (c, kd, vd))


def _io(write, pool, pages, k, v, start, count, stream):
    _check_grad(k, v)
    key = (fluid._lib, pool.shape, pool.stride(), pool.dtype, pool.get_device(), pages.shape, pages.stride(), pages.dtype,
           pages.get_device(), k.dtype, k.shape, k.stride(), k.get_device(), v.dtype, v.shape, v.stride(),
           v.get_device(), _form(start), None if count is None else _form(count))
    made = _calls.get(key)
    if made is None:
        made = _keep(key, _io_call(pool, pages, k, v, start, count))
    lib, dev, c, kd, vd, _ = made
    _launch(lib.fluid_kv_write if write else lib.fluid_kv_read, dev,
            c, pool.data_ptr(), pages.data_ptr(), kd, k.data_ptr(), vd, v.data_ptr(), start.data_ptr(),
            None if count is None else count.data_ptr(), _raw_stream(dev) if stream is None else _stream(stream, dev))
    if stream is not None:
        _record(stream, dev, pool, pages, k, v, start, count)


def kv_write(pool, pages, k, v, start, count=None, stream=None):
    """Quantise tokens k, v [batch, T, kv_heads, head_dim] into the cache: row
    i of sequence b becomes token start[b] + i, for i < count[b] (None: all)."""
    _io(True, pool, pages, k, v, start, count, stream)


def kv_read(pool, pages, start, k, v, count=None, stream=None):
    """The cache's values of tokens start[b] .. of every sequence into k, v
    [batch, T, kv_heads, head_dim], count[b] of them (None: T); rows past that
    are left as they are."""
    _io(False, pool, pages, k, v, start, count, stream)


def _workspace(need, workspace, device, stream):
    """(tensor to keep for the call, address, bytes)."""
    torch = _torch()
    if workspace is None:
        # torch hands a freed block out again only in the order of the stream
        # it was allocated on, so it is allocated on the call's own
        if stream is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
        else:
            with torch.cuda.stream(_as_stream(stream, device)):
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
    elif workspace.get_device() != device or not workspace.is_contiguous():
        _refuse(f"workspace: a contiguous tensor on GPU {device} is needed")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _kv_call(pool, pages, q, kv_len, q_len, scale, window, sinks, out):
    dev = _device_of(pool, "pool")
    qd = _describe(q, "q", dev)
    od = qd if out is None else _describe(out, "out", dev)
    D, n = q.shape[3], pages.shape[0]
    c, o = _describe_cache(pool, pages, D, dev), _describe_opts(scale, True, window, sinks, D)
    _check_ints(kv_len, "kv_len", n, dev)
    _check_ints(q_len, "q_len", n, dev)
    # the last is (kv_max, bytes of workspace) of the latest call
    return [_lib(), dev, _addr(c), _addr(o), _addr(qd), _addr(od), c.max_pages * c.page_tokens, (c, o, qd, od), (None, 0)]


def _kv_need(made, kv_max):
    """Bytes of workspace for a described call and this bound."""
    lib, _, c, o, qd, _, _, _, (most, need) = made
    if most != kv_max:
        n = _U64()
        fluid._check(lib.fluid_kv_attention_workspace(c, o, kv_max, qd, C.byref(n)))
        need = n.value
        made[8] = kv_max, need
    return need


def kv_attention_workspace(pool, pages, q, kv_max=None, scale=None, window=0, sinks=0):
    """Bytes of workspace that ``kv_attention`` needs for these arguments."""
    made = _kv_call(pool, pages, q, None, None, scale, window, sinks, None)
    return _kv_need(made, made[6] if kv_max is None else kv_max)


def kv_attention(pool, pages, q, kv_len, q_len=None, kv_max=None, scale=None, window=0, sinks=0, out=None,
                 workspace=None, stream=None):
    """Causal attention of q [batch, T, heads, head_dim] over the cache.

    Sequence b has kv_len[b] tokens in the cache, the newest q_len[b] (None: T)
    of which are the queries' own; with a ``window`` a query sees the last
    ``window`` tokens up to its own and the first ``sinks`` ones.  scale: of
    q . k, 1 / sqrt(head_dim) by default.  kv_max: the largest kv_len to
    expect, which sizes the split of long caches over the GPU (by default all
    that a row of the table can name; caches far shorter than it are slower than
    with a bound near their length).  out: where to write (rows past q_len
    are left as they are; allocated as zeros by default).  Returns out."""
    if out is None:
        out = _zeros(q, stream)
    _check_grad(q, out)
    key = (fluid._lib, pool.shape, pool.stride(), pool.dtype, pool.get_device(), pages.shape, pages.stride(), pages.dtype,
           pages.get_device(), q.dtype, q.shape, q.stride(), q.get_device(), out.dtype, out.shape, out.stride(),
           out.get_device(), _form(kv_len), None if q_len is None else _form(q_len), scale, window, sinks)
    made = _calls.get(key)
    if made is None:
        if kv_len is None:
            _refuse("kv_len: needed")
        made = _keep(key, _kv_call(pool, pages, q, kv_len, q_len, scale, window, sinks, out))
    lib, dev, c, o, qd, od, most, _, _ = made
    if kv_max is None:
        kv_max = most
    need = _kv_need(made, kv_max)
    keep, ws, ws_bytes = _workspace(need, workspace, dev, stream) if need else (None, None, 0)
    _launch(lib.fluid_kv_attention, dev,
            c, pool.data_ptr(), pages.data_ptr(), o, kv_max, qd, q.data_ptr(), None if q_len is None else q_len.data_ptr(),
            kv_len.data_ptr(), od, out.data_ptr(), ws, ws_bytes, _raw_stream(dev) if stream is None else _stream(stream, dev))
    if stream is not None:
        _record(stream, dev, pool, pages, q, q_len, kv_len, out, workspace)
    del keep
    return out


def _zeros(q, stream):
    """Zeros of q's shape, filled on the call's stream."""
    torch = _torch()
    if stream is None or not q.is_cuda:
        return torch.zeros(q.shape, dtype=q.dtype, device=q.device)
    with torch.cuda.stream(_as_stream(stream, q.device)):
        return torch.zeros(q.shape, dtype=q.dtype, device=q.device)


def _dense_call(q, k, v, q_len, kv_len, scale, causal, window, sinks, out):
    dev = _device_of(q, "q")
    qd, kd, vd = _describe(q, "q", dev), _describe(k, "k", dev), _describe(v, "v", dev)
    od = _describe(out, "out", dev)
    B, D = q.shape[0], q.shape[3]
    o = _describe_opts(scale, causal, window, sinks, D)
    _check_ints(q_len, "q_len", B, dev)
    _check_ints(kv_len, "kv_len", B, dev)
    need = _U64()
    fluid._check(_lib().fluid_attention_workspace(_addr(o), _addr(qd), _addr(kd), C.byref(need)))
    return (_lib(), dev, _addr(o), _addr(qd), _addr(kd), _addr(vd), _addr(od), need.value, (o, qd, kd, vd, od))


def attention(q, k, v, q_len=None, kv_len=None, scale=None, causal=True, window=0, sinks=0, out=None,
              workspace=None, stream=None):
    """Attention of q [batch, T, heads, head_dim] over k, v [batch, N,
    kv_heads, head_dim] (heads a multiple of kv_heads), all of one dtype.

    Sequence b has kv_len[b] tokens (None: N), the newest q_len[b] (None: T) of
    which are the queries' own.  With a ``window`` a query sees the tokens less
    than ``window`` from its own (up to its own if causal) and the first
    ``sinks`` ones.  Rows that see nothing are zeros.  Returns out, as
    ``kv_attention`` does."""
    if out is None:
        out = _zeros(q, stream)
    _check_grad(q, k, v, out)
    key = (fluid._lib, q.dtype, q.shape, q.stride(), q.get_device(), k.dtype, k.shape, k.stride(), k.get_device(),
           v.dtype, v.shape, v.stride(), v.get_device(), out.dtype, out.shape, out.stride(), out.get_device(),
           None if q_len is None else _form(q_len), None if kv_len is None else _form(kv_len), scale, causal, window,
           sinks)
    made = _calls.get(key)
    if made is None:
        made = _keep(key, _dense_call(q, k, v, q_len, kv_len, scale, causal, window, sinks, out))
    lib, dev, o, qd, kd, vd, od, need, _ = made
    keep, ws, ws_bytes = _workspace(need, workspace, dev, stream) if need else (None, None, 0)
    _launch(lib.fluid_attention, dev,
            o, qd, q.data_ptr(), kd, k.data_ptr(), vd, v.data_ptr(), None if q_len is None else q_len.data_ptr(),
            None if kv_len is None else kv_len.data_ptr(), od, out.data_ptr(), ws, ws_bytes,
            _raw_stream(dev) if stream is None else _stream(stream, dev))
    if stream is not None:
        _record(stream, dev, q, k, v, q_len, kv_len, out, workspace)
    del keep
    return out


def _linear_call(q, k, v, decay, state, count, out, state_out):
    torch = _torch()
    dev = _device_of(q, "q")
    qd, kd, vd = _describe(q, "q", dev), _describe(k, "k", dev), _describe(v, "v", dev)
    od = _describe(out, "out", dev)
    B, T, Hk, D = k.shape
    if decay.dtype != torch.float32 or tuple(decay.shape) not in ((Hk,), (B, T, Hk)) or decay.get_device() != dev:
        _refuse(f"decay: fp32 [{Hk}] or [{B}, {T}, {Hk}] on GPU {dev} is needed")
    stride = (C.c_int64 * 3)(*((0, 0) + decay.stride() if decay.dim() == 1 else decay.stride()))
    for name, t in (("state", state), ("state_out", state_out)):
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (B, Hk, D, D) or not t.is_contiguous()
                              or t.get_device() != dev):
            _refuse(f"{name}: contiguous fp32 [{B}, {Hk}, {D}, {D}] on GPU {dev} is needed")
    _check_ints(count, "count", B, dev)
    need = _U64()
    fluid._check(_lib().fluid_linear_attention_workspace(_addr(qd), _addr(kd), C.byref(need)))
    return (_lib(), dev, _addr(qd), _addr(kd), _addr(vd), _addr(od), _addr(stride), need.value, (qd, kd, vd, od, stride))


def linear_attention(q, k, v, decay, state=None, count=None, scale=None, out=None, state_out=None, workspace=None,
                     stream=None):
    """Attention whose memory is a state S [head_dim, head_dim] of every kv
    head: token after token S = exp(decay) S + k v^T, out = scale S^T q.

    q [batch, T, heads, head_dim], k and v [batch, T, kv_heads, head_dim] (heads
    a multiple of kv_heads) of one dtype; decay: its logarithm in fp32, at most 0,
    [kv_heads] or one a token [batch, T, kv_heads].  state: fp32 [batch, kv_heads,
    head_dim, head_dim] to start from (None: zeros); state_out: where to leave the
    last one, which may be ``state`` (allocated by default).  count[b] (None: T)
    tokens of sequence b are there; out's rows behind them are left as they are, and
    out must not overlap an input.
    scale: 1 / sqrt(head_dim) by default.  A prompt and the single tokens behind
    it are calls that hand the state on.  Returns (out, state_out)."""
    if out is None:
        out = _zeros(q, stream)
    if state_out is None:
        state_out = _new_state(k, stream)
    if (q.requires_grad or k.requires_grad or v.requires_grad or decay.requires_grad or out.requires_grad
            or state_out.requires_grad or (state is not None and state.requires_grad)):
        _check_grad(q, k, v, decay, out, state_out, *(() if state is None else (state,)))
    key = (fluid._lib, q.dtype, q.shape, q.stride(), q.get_device(), k.dtype, k.shape, k.stride(), k.get_device(),
           v.dtype, v.shape, v.stride(), v.get_device(), out.dtype, out.shape, out.stride(), out.get_device(),
           decay.dtype, decay.shape, decay.stride(), decay.get_device(), None if state is None else _form(state),
           state_out.dtype, state_out.shape, state_out.stride(), state_out.get_device(),
           None if count is None else _form(count), "linear")
    made = _calls.get(key)
    if made is None:
        made = _keep(key, _linear_call(q, k, v, decay, state, count, out, state_out))
    lib, dev, qd, kd, vd, od, stride, need, _ = made
    keep, ws, ws_bytes = _workspace(need, workspace, dev, stream) if need else (None, None, 0)
    _launch(lib.fluid_linear_attention, dev,
            q.shape[3] ** -0.5 if scale is None else scale, qd, q.data_ptr(), kd, k.data_ptr(), vd, v.data_ptr(),
            decay.data_ptr(), stride, None if state is None else state.data_ptr(),
            None if count is None else count.data_ptr(), od, out.data_ptr(), state_out.data_ptr(), ws, ws_bytes,
            _raw_stream(dev) if stream is None else _stream(stream, dev))
    if stream is not None:
        _record(stream, dev, q, k, v, decay, state, count, out, state_out, workspace)
    del keep
    return out, state_out


def linear_attention_workspace(q, k):
    """Bytes of workspace that ``linear_attention`` needs for these tensors."""
    dev = _device_of(q, "q")
    qd, kd, need = _describe(q, "q", dev), _describe(k, "k", dev), _U64()
    fluid._check(_lib().fluid_linear_attention_workspace(_addr(qd), _addr(kd), C.byref(need)))
    return need.value


def _new_state(k, stream):
    """A state for k's sequences and heads, allocated on the call's stream."""
    torch = _torch()
    if k.dim() != 4:
        _refuse(f"k: a tensor [batch, tokens, heads, head_dim] is needed, got {k.dim()} dimensions")
    shape = (k.shape[0], k.shape[2], k.shape[3], k.shape[3])
    if stream is None or not k.is_cuda:
        return torch.empty(shape, dtype=torch.float32, device=k.device)
    with torch.cuda.stream(_as_stream(stream, k.device)):
        return torch.empty(shape, dtype=torch.float32, device=k.device)


SCALINGS = {"none": 0, "linear": 1, "base": 2, "ramp": 3}


class Rotary:
    """How positions turn a head's first ``dim`` channels: frequencies
    base^(-2 i / dim) of pairs (i, i + dim / 2), or (2 i, 2 i + 1) if
    ``interleaved``, for contexts ``factor`` times as long by one of
    ``scaling``:

        "linear"  all frequencies divided by factor
        "base"    base * factor^(dim / (dim - 2))
        "ramp"    frequencies that make ``high`` turns or more over ``length``
                  tokens stay, those of ``low`` or fewer are divided, the others
                  mixed in proportion

    Turned channels are multiplied by ``amplitude``.  ``turns`` holds the pairs'
    turns a token on the GPU, made once."""

    def __init__(self, dim, base=10000.0, interleaved=False, scaling="none", factor=1.0, length=0.0, low=1.0, high=32.0,
                 amplitude=1.0, device="cuda"):
        torch = _torch()
        if scaling not in SCALINGS:
            _refuse(f"scaling: one of {', '.join(SCALINGS)} is needed, got {scaling!r}")
        self.desc = RotaryDesc(dim, 1 if interleaved else 0, SCALINGS[scaling], amplitude, base, factor, length, low, high)
        if not 2 <= dim <= 1024:
            _refuse(f"dim: {dim} does not lie in 2 .. 1024")
        turns = torch.empty(dim // 2, dtype=torch.int64)
        fluid._check(_lib().fluid_rotary_turns(_addr(self.desc), turns.data_ptr()))
        self.dim = dim
        self.turns = turns.to(device)


def _rotary_call(turns, q, k, start, positions, count, q_out, k_out):
    torch = _torch()
    dev = _device_of(q, "q")
    if not isinstance(turns, Rotary):
        _refuse("turns: a Rotary is needed")
    if turns.turns.get_device() != dev:
        _refuse(f"turns: on {turns.turns.device}, not on GPU {dev}")
    qd, qod = _describe(q, "q", dev), _describe(q_out, "q_out", dev)
    kd = kod = None
    if k is not None:
        kd, kod = _describe(k, "k", dev), _describe(k_out, "k_out", dev)
    elif k_out is not None:
        _refuse("k_out: there is no k")
    B, T = q.shape[:2]
    _check_ints(start, "start", B, dev)
    _check_ints(count, "count", B, dev)
    stride = 0
    if positions is not None:
        if (positions.dtype != torch.int32 or tuple(positions.shape) != (B, T) or positions.get_device() != dev
                or (T > 1 and positions.stride(1) != 1)):
            _refuse(f"positions: int32 [{B}, {T}] with contiguous rows on GPU {dev} is needed")
        stride = positions.stride(0)
    refs = [None if d is None else _addr(d) for d in (qd, qod, kd, kod)]
    return (_lib(), dev, *refs, stride, (qd, qod, kd, kod))


def rotary(turns, q, k=None, start=None, positions=None, count=None, inverse=False, q_out=None, k_out=None, stream=None):
    """q [batch, T, heads, head_dim] and k [batch, T, kv_heads, head_dim] (None:
    q alone) turned by their positions as ``turns``, a Rotary, says.

    Row i of sequence b is at position start[b] + i (None: i), or at positions[b,
    i].  Rows from count[b] on (None: T) are left as they are.  inverse: turned
    back, times the amplitude as well: the transpose, which is the gradient.  q_out,
    k_out: where to write, which may be q and k themselves (allocated as zeros by
    default).  Returns (q_out, k_out), or q_out without a k."""
    if q_out is None:
        q_out = _zeros(q, stream)
    if k is not None and k_out is None:
        k_out = _zeros(k, stream)
    if q.requires_grad or q_out.requires_grad or (k is not None and (k.requires_grad or k_out.requires_grad)):
        _check_grad(q, q_out, *(() if k is None else (k, k_out)))
    on = turns.turns.get_device() if isinstance(turns, Rotary) else None
    key = (fluid._lib, q.dtype, q.shape, q.stride(), q.get_device(), q_out.dtype, q_out.shape, q_out.stride(),
           q_out.get_device(), None if k is None else _form(k), None if k_out is None else _form(k_out),
           None if start is None else _form(start), None if positions is None else _form(positions),
           None if count is None else _form(count), on, "rotary")
    made = _calls.get(key)
    if made is None:
        made = _keep(key, _rotary_call(turns, q, k, start, positions, count, q_out, k_out))
    lib, dev, qd, qod, kd, kod, stride, _ = made
    _launch(lib.fluid_rotate, dev, C.addressof(turns.desc), turns.turns.data_ptr(),
            None if start is None else start.data_ptr(), None if positions is None else positions.data_ptr(), stride,
            None if count is None else count.data_ptr(), 1 if inverse else 0, qd, q.data_ptr(), qod, q_out.data_ptr(),
            kd, None if k is None else k.data_ptr(), kod, None if k_out is None else k_out.data_ptr(),
            _raw_stream(dev) if stream is None else _stream(stream, dev))
    if stream is not None:
        _record(stream, dev, q, k, start, positions, count, q_out, k_out, turns.turns)
    return q_out if k is None else (q_out, k_out)


class KvCache:
    """The cache of a batch of sequences: pool, page table and lengths.

    Pages are handed out on the host as sequences grow and given back when a
    window has left them behind (``trim``) or a sequence ends (``clear``).
    ``lengths`` is the host's copy; ``kv_len`` the device's.  Every change copies
    the whole table and the lengths to the device, which takes host time in
    proportion to batch x max_tokens / page_tokens.  Methods run on torch's
    current stream; ``attend`` takes ``stream``, to be ordered by the caller."""

    def __init__(self, batch, kv_heads, head_dim, max_tokens, n_pages=None, page_tokens=64, device="cuda"):
        torch = self.torch = _torch()
        per = -(-max_tokens // page_tokens)
        n_pages = batch * per if n_pages is None else n_pages
        desc = CacheDesc(n_pages, page_tokens, kv_heads, head_dim, batch, per, per)
        n = _U64()
        fluid._check(_lib().fluid_kv_pool_bytes(C.byref(desc), C.byref(n)))
        block = pool_block(page_tokens, head_dim)
        assert n.value == n_pages * kv_heads * block
        self.page_tokens, self.max_tokens = page_tokens, per * page_tokens
        self.pool = torch.zeros(n_pages, kv_heads, block, dtype=torch.uint8, device=device)
        self.table = [[-1] * per for _ in range(batch)]
        self.pages = torch.full((batch, per), -1, dtype=torch.int32, device=device)
        self.free = list(range(n_pages - 1, -1, -1))
        self.lengths = [0] * batch
        self.kv_len = torch.zeros(batch, dtype=torch.int32, device=device)

    def _push(self):
        """Host copies to the device, behind what the current stream runs."""
        self.pages.copy_(self.torch.tensor(self.table, dtype=self.torch.int32))
        self.kv_len.copy_(self.torch.tensor(self.lengths, dtype=self.torch.int32))

    def append(self, k, v, counts=None):
        """Write tokens k, v [batch, T, kv_heads, head_dim] behind what every
        sequence holds (counts: how many of each, on the host)."""
        batch = len(self.lengths)
        if k.dim() != 4 or k.shape[0] != batch:
            _refuse(f"k: a tensor [{batch}, tokens, heads, head_dim] is needed, got {tuple(k.shape)}")
        counts = [k.shape[1]] * batch if counts is None else list(counts)
        if len(counts) != batch:
            _refuse(f"counts: {batch} are needed, got {len(counts)}")
        start = list(self.lengths)
        for b, n in enumerate(counts):
            if not 0 <= n <= k.shape[1] or start[b] + n > self.max_tokens:
                _refuse(f"sequence {b}: {start[b]} + {n} tokens do not fit {self.max_tokens}")
        new = [(b, i) for b, n in enumerate(counts) if n
               for i in range(start[b] // self.page_tokens, (start[b] + n - 1) // self.page_tokens + 1)
               if self.table[b][i] < 0]
        if len(new) > len(self.free):
            _refuse(f"the pool has {len(self.free)} free pages, {len(new)} are needed")
        for b, i in new:
            self.table[b][i] = self.free.pop()
        self.lengths = [s + n for s, n in zip(start, counts)]
        at = self.kv_len.clone()
        self._push()
        try:
            kv_write(self.pool, self.pages, k, v, at, self.kv_len - at)
        except Exception:  # nothing was written: as if not called
            for b, i in reversed(new):
                self.free.append(self.table[b][i])
                self.table[b][i] = -1
            self.lengths = start
            self._push()
            raise

    def attend(self, q, q_len=None, **kw):
        """``kv_attention`` of q over the cache."""
        return kv_attention(self.pool, self.pages, q, self.kv_len, q_len=q_len, kv_max=max(max(self.lengths), 1), **kw)

    def read(self, k, v):
        """All tokens' values into k, v [batch, T, ...]; T at least the longest
        sequence."""
        kv_read(self.pool, self.pages, self.torch.zeros_like(self.kv_len), k, v, self.kv_len)

    def trim(self, window, sinks=0):
        """Give back the pages that no query from the newest token on sees: none
        without a window (0)."""
        if window < 0 or sinks < 0:
            _refuse(f"window, sinks: {window}, {sinks} must not be negative")
        if window == 0:
            return
        for b, n in enumerate(self.lengths):
            for i in range(max(0, n - window) // self.page_tokens):
                if i * self.page_tokens >= sinks and self.table[b][i] >= 0:
                    self.free.append(self.table[b][i])
                    self.table[b][i] = -1
        self._push()

    def clear(self, b):
        """Forget sequence b."""
        self.free += [p for p in self.table[b] if p >= 0]
        self.table[b] = [-1] * len(self.table[b])
        self.lengths[b] = 0
        self._push()
