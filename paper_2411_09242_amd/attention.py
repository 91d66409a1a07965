"""Token-by-token generation beside the planned graphs: a paged key/value
cache held in 4 bits, attention over it, and attention with a sliding window
and a few first tokens that stay visible (ctypes binding of
include/fluid_attention.h).

    kv_write(pool, pages, k, v, start, count)   quantise new tokens into the cache
    kv_read(pool, pages, start, k, v, count)    its values as ordinary tensors
    kv_attention(pool, pages, q, kv_len, ...)   queries over the cache
    attention(q, k, v, ...)                     queries over ordinary keys and values
    KvCache                                     pool, page table and lengths of a batch

Tensors of tokens are torch tensors [batch, tokens, heads, head_dim] in fp32
or bf16 on the GPU, with any strides and contiguous channels; lengths, starts
and page tables are int32 tensors on the GPU.  Calls enqueue kernels on
torch's current stream, or on ``stream`` (a torch stream or a raw handle), and
return without waiting; arguments that cannot be right raise ``FluidError``
before anything is launched.  What a window has left behind may be freed: page
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


_PROTOS = {
    "fluid_kv_pool_bytes": [_VP, _VP],
    "fluid_kv_write": [_VP] * 10,
    "fluid_kv_read": [_VP] * 10,
    "fluid_kv_attention_workspace": [_VP, _VP, _I32, _VP, _VP],
    "fluid_kv_attention": [_VP, _VP, _VP, _VP, _I32, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _U64, _VP],
    "fluid_attention_workspace": [_VP] * 4,
    "fluid_attention": [_VP] * 12 + [_U64, _VP],
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


# Descriptions by what they describe (type, shape, strides): a decoding loop
# makes the same few over and over, and filling a ctypes structure takes as
# long as a small launch.
_descs = {}


def _tokens(t, name, device):
    if t.dim() != 4:
        _refuse(f"{name}: a tensor [batch, tokens, heads, head_dim] is needed, got {t.dim()} dimensions")
    if t.device != device:
        _refuse(f"{name}: on {t.device}, not on {device}")
    shape, stride = t.shape, t.stride()
    key = (t.dtype, shape, stride)
    d = _descs.get(key)
    if d is None:
        torch = _torch()
        if t.dtype not in (torch.float32, torch.bfloat16):
            _refuse(f"{name}: dtype must be float32 or bfloat16, got {t.dtype}")
        if stride[3] != 1 and shape[3] > 1:
            _refuse(f"{name}: channels must be contiguous")
        if max(shape) >= 1 << 31:
            _refuse(f"{name}: too large")
        if len(_descs) > 4096:
            _descs.clear()
        d = Tokens(fluid.F32 if t.dtype == torch.float32 else fluid.BF16, *shape, (C.c_int64 * 3)(*stride[:3]))
        d = _descs[key] = (C.addressof(d), d)
    return d[0]


def _torch():
    import torch
    return torch


def _ints(t, name, n, device):
    """Address of an int32 tensor of n values; None stays None."""
    if t is None:
        return None
    if t.dtype != _torch().int32 or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1) or t.device != device:
        _refuse(f"{name}: {n} contiguous int32 values on {device} are needed")
    return t.data_ptr()


def _cache(pool, pages, head_dim):
    if pool.dim() != 3 or pool.element_size() != 1 or not pool.is_contiguous():
        _refuse("pool: a contiguous uint8 tensor [pages, kv_heads, block] is needed")
    if pages.dim() != 2 or pages.dtype != _torch().int32 or (pages.shape[1] > 1 and pages.stride(1) != 1):
        _refuse("pages: an int32 tensor [batch, max_pages] with contiguous rows is needed")
    if pages.device != pool.device:
        _refuse(f"pages: on {pages.device}, not on {pool.device}")
    key = (pool.shape, pages.shape, pages.stride(), head_dim)
    d = _descs.get(key)
    if d is None:
        n, heads, block = pool.shape
        tokens = block * 4 // (5 * head_dim)
        if block * 4 != 5 * head_dim * tokens or tokens not in PAGE_TOKENS:
            _refuse(f"pool: a block of {block} bytes is no page of head_dim {head_dim}")
        if len(_descs) > 4096:
            _descs.clear()
        stride = pages.stride(0) if pages.shape[0] > 1 else pages.shape[1]
        d = CacheDesc(n, tokens, heads, head_dim, pages.shape[0], pages.shape[1], stride)
        d = _descs[key] = (C.addressof(d), d)
    return d[0]


def _opts(scale, causal, window, sinks, head_dim):
    key = (scale, causal, window, sinks, head_dim)
    d = _descs.get(key)
    if d is None:
        for name, v in (("window", window), ("sinks", sinks)):
            if not 0 <= v < 1 << 31:
                _refuse(f"{name}: {v} is out of range")
        if len(_descs) > 4096:
            _descs.clear()
        d = Opts(1.0 / math.sqrt(head_dim) if scale is None else scale, 1 if causal else 0, window, sinks)
        d = _descs[key] = (C.addressof(d), d)
    return d[0]


def _stream(stream, device):
    if stream is None:
        stream = _torch().cuda.current_stream(device)
    return getattr(stream, "cuda_stream", stream)


def _on_gpu(t, name):
    if not t.is_cuda:
        _refuse(f"{name}: a tensor on the GPU is needed, got {t.device}")
    return t.device


def pool_block(page_tokens, head_dim):
    """Bytes of one page of one kv head."""
    return 5 * head_dim * page_tokens // 4


def kv_write(pool, pages, k, v, start, count=None, stream=None):
    """Quantise tokens k, v [batch, T, kv_heads, head_dim] into the cache: row
    i of sequence b becomes token start[b] + i, for i < count[b] (None: all)."""
    dev = _on_gpu(pool, "pool")
    kd, vd = _tokens(k, "k", dev), _tokens(v, "v", dev)
    n = pages.shape[0]
    fluid._check(_lib().fluid_kv_write(
        _cache(pool, pages, k.shape[3]), pool.data_ptr(), pages.data_ptr(), kd, k.data_ptr(), vd, v.data_ptr(),
        _ints(start, "start", n, dev), _ints(count, "count", n, dev), _stream(stream, dev)))


def kv_read(pool, pages, start, k, v, count=None, stream=None):
    """The cache's values of tokens start[b] .. of every sequence into k, v
    [batch, T, kv_heads, head_dim], count[b] of them (None: T); rows past that
    are left as they are."""
    dev = _on_gpu(pool, "pool")
    kd, vd = _tokens(k, "k", dev), _tokens(v, "v", dev)
    n = pages.shape[0]
    fluid._check(_lib().fluid_kv_read(
        _cache(pool, pages, k.shape[3]), pool.data_ptr(), pages.data_ptr(), kd, k.data_ptr(), vd, v.data_ptr(),
        _ints(start, "start", n, dev), _ints(count, "count", n, dev), _stream(stream, dev)))


def _workspace(need, workspace, device, stream):
    """(tensor to keep for the call, address, bytes)."""
    if need == 0:
        return None, None, 0
    torch = _torch()
    if workspace is None:
        # torch hands a freed block out again only in the order of the stream
        # it was allocated on, so it is allocated on the call's own
        if stream is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
        else:
            s = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(stream, device=device)
            with torch.cuda.stream(s):
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def kv_attention_workspace(pool, pages, q, kv_max=None, scale=None, window=0, sinks=0):
    """Bytes of workspace that ``kv_attention`` needs for these arguments."""
    dev = pool.device
    D = q.shape[3]
    c, o, qd = _cache(pool, pages, D), _opts(scale, True, window, sinks, D), _tokens(q, "q", dev)
    if kv_max is None:
        kv_max = pages.shape[1] * (pool.shape[2] * 4 // (5 * D))
    n = _U64()
    fluid._check(_lib().fluid_kv_attention_workspace(c, o, kv_max, qd, C.byref(n)))
    return n.value


def kv_attention(pool, pages, q, kv_len, q_len=None, kv_max=None, scale=None, window=0, sinks=0, out=None,
                 workspace=None, stream=None):
    """Causal attention of q [batch, T, heads, head_dim] over the cache.

    Sequence b has kv_len[b] tokens in the cache, the newest q_len[b] (None: T)
    of which are the queries' own; with a ``window`` a query sees the last
    ``window`` tokens up to its own and the first ``sinks`` ones.  scale: of
    q . k, 1 / sqrt(head_dim) by default.  kv_max: the largest kv_len to
    expect, which sizes the split of long caches over the GPU (by default all
    that a row of the table can name).  out: where to write (rows past q_len
    are left as they are; allocated as zeros by default).  Returns out."""
    dev = _on_gpu(pool, "pool")
    qd, D, n = _tokens(q, "q", dev), q.shape[3], pages.shape[0]
    c, o = _cache(pool, pages, D), _opts(scale, True, window, sinks, D)
    if kv_max is None:
        kv_max = pages.shape[1] * (pool.shape[2] * 4 // (5 * D))
    if out is None:
        out = _torch().zeros_like(q, memory_format=_torch().contiguous_format)
    od = _tokens(out, "out", dev)
    lib = _lib()
    need = _U64()
    fluid._check(lib.fluid_kv_attention_workspace(c, o, kv_max, qd, C.byref(need)))
    keep, ws, ws_bytes = _workspace(need.value, workspace, dev, stream)
    if kv_len is None:
        _refuse("kv_len: needed")
    fluid._check(lib.fluid_kv_attention(
        c, pool.data_ptr(), pages.data_ptr(), o, kv_max, qd, q.data_ptr(), _ints(q_len, "q_len", n, dev),
        _ints(kv_len, "kv_len", n, dev), od, out.data_ptr(), ws, ws_bytes, _stream(stream, dev)))
    del keep
    return out


def attention(q, k, v, q_len=None, kv_len=None, scale=None, causal=True, window=0, sinks=0, out=None,
              workspace=None, stream=None):
    """Attention of q [batch, T, heads, head_dim] over k, v [batch, N,
    kv_heads, head_dim] (heads a multiple of kv_heads), all of one dtype.

    Sequence b has kv_len[b] tokens (None: N), the newest q_len[b] (None: T) of
    which are the queries' own.  With a ``window`` a query sees the tokens less
    than ``window`` from its own (up to its own if causal) and the first
    ``sinks`` ones.  Rows that see nothing are zeros.  Returns out, as
    ``kv_attention`` does."""
    dev = _on_gpu(q, "q")
    qd, kd, vd = _tokens(q, "q", dev), _tokens(k, "k", dev), _tokens(v, "v", dev)
    B, D = q.shape[0], q.shape[3]
    o = _opts(scale, causal, window, sinks, D)
    if out is None:
        out = _torch().zeros_like(q, memory_format=_torch().contiguous_format)
    od = _tokens(out, "out", dev)
    lib = _lib()
    need = _U64()
    fluid._check(lib.fluid_attention_workspace(o, qd, kd, C.byref(need)))
    keep, ws, ws_bytes = _workspace(need.value, workspace, dev, stream)
    fluid._check(lib.fluid_attention(
        o, qd, q.data_ptr(), kd, k.data_ptr(), vd, v.data_ptr(), _ints(q_len, "q_len", B, dev),
        _ints(kv_len, "kv_len", B, dev), od, out.data_ptr(), ws, ws_bytes, _stream(stream, dev)))
    del keep
    return out


class KvCache:
    """The cache of a batch of sequences: pool, page table and lengths.

    Pages are handed out on the host as sequences grow and given back when a
    window has left them behind (``trim``) or a sequence ends (``clear``).
    ``lengths`` is the host's copy; ``kv_len`` the device's."""

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
        counts = [k.shape[1]] * len(self.lengths) if counts is None else list(counts)
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
        kv_write(self.pool, self.pages, k, v, at, self.kv_len - at)

    def attend(self, q, q_len=None, **kw):
        """``kv_attention`` of q over the cache."""
        return kv_attention(self.pool, self.pages, q, self.kv_len, q_len=q_len, kv_max=max(max(self.lengths), 1), **kw)

    def read(self, k, v):
        """All tokens' values into k, v [batch, T, ...]; T at least the longest
        sequence."""
        kv_read(self.pool, self.pages, self.torch.zeros_like(self.kv_len), k, v, self.kv_len)

    def trim(self, window, sinks=0):
        """Give back the pages that no query from the newest token on sees."""
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
