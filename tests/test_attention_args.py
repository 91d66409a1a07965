"""Entry points of fluid_attention.h without a GPU: both libraries export
them, what cannot be right is refused with a cause before any launch, and what
is right reaches the (here missing) GPU; workspace sizes; the oracle's own
pins."""
import ctypes as C
import os
import re

import numpy as np
import pytest

from oracle import attention as OA
from paper_2411_09242_amd import attention as A
from paper_2411_09242_amd import fluid as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, TOO_SMALL = -1, -2, -4


@pytest.fixture(scope="module", autouse=True)
def host_lib():
    F.load(host_only=True)
    yield
    F.load(host_only=True)


@pytest.mark.parametrize("name", ["libfluid_host.so", "libfluid.so"])
def test_libraries_export_every_declared_symbol(name):
    lib = C.CDLL(os.path.join(F.LIBDIR, name))
    src = open(os.path.join(ROOT, "include", "fluid_attention.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    syms = set(re.findall(r"\b(fluid_[a-z_]+)\s*\(", src))
    assert syms == set(A.SYMBOLS)
    for s in syms:
        assert hasattr(lib, s), s


ADDR = 1 << 20  # a plausible, 256-byte aligned address; never read on the host


def tokens(dtype=F.BF16, batch=2, tokens=5, heads=4, head_dim=64, stride=None):
    stride = stride or (tokens * heads * head_dim, heads * head_dim, head_dim)
    return A.Tokens(dtype, batch, tokens, heads, head_dim, (C.c_int64 * 3)(*stride))


def cache(n_pages=9, page_tokens=64, kv_heads=2, head_dim=64, batch=2, max_pages=4, table_stride=4):
    return A.CacheDesc(n_pages, page_tokens, kv_heads, head_dim, batch, max_pages, table_stride)


def opts(scale=0.125, causal=1, window=0, sinks=0):
    return A.Opts(scale, causal, window, sinks)


def ref(x):
    return None if x is None else C.byref(x)


def io(c=None, kd=None, vd=None, pool=ADDR, pages=ADDR, k=ADDR, v=ADDR, start=ADDR, count=None, write=True):
    lib = A._lib()
    c, kd = c or cache(), kd or tokens(heads=2)
    vd = vd or tokens(heads=2)
    f = lib.fluid_kv_write if write else lib.fluid_kv_read
    return f(ref(c), pool, pages, ref(kd), k, ref(vd), v, start, count, None), lib.fluid_last_error().decode()


def kv(c=None, o=None, kv_max=200, qd=None, od=None, pool=ADDR, pages=ADDR, q=ADDR, kv_len=ADDR, out=ADDR, ws=ADDR,
       ws_bytes=1 << 40):
    lib = A._lib()
    c, o, qd = c or cache(), o or opts(), qd or tokens()
    od = od or tokens()
    return (lib.fluid_kv_attention(ref(c), pool, pages, ref(o), kv_max, ref(qd), q, None, kv_len, ref(od), out, ws,
                                   ws_bytes, None), lib.fluid_last_error().decode())


def dense(o=None, qd=None, kd=None, vd=None, od=None, q=ADDR, k=ADDR, v=ADDR, out=ADDR, ws=ADDR, ws_bytes=1 << 40):
    lib = A._lib()
    o, qd, kd = o or opts(), qd or tokens(), kd or tokens(heads=2, tokens=9)
    vd, od = vd or tokens(heads=2, tokens=9), od or tokens()
    return (lib.fluid_attention(ref(o), ref(qd), q, ref(kd), k, ref(vd), v, None, None, ref(od), out, ws, ws_bytes,
                                None), lib.fluid_last_error().decode())


def test_what_is_right_reaches_the_gpu_part():
    for st, msg in (io(), io(write=False), kv(), dense(), dense(o=opts(causal=0, window=7, sinks=2))):
        assert st == UNSUPPORTED, msg
        assert "host-only" in msg


@pytest.mark.parametrize("bad, word", [
    (dict(c=cache(head_dim=48), kd=tokens(heads=2, head_dim=48), vd=tokens(heads=2, head_dim=48)), "head_dim"),
    (dict(c=cache(page_tokens=16)), "page_tokens"), (dict(c=cache(page_tokens=48)), "page_tokens"),
    (dict(c=cache(page_tokens=2048)), "page_tokens"), (dict(c=cache(n_pages=0)), "n_pages"),
    (dict(c=cache(max_pages=0)), "max_pages"), (dict(c=cache(table_stride=3)), "table_stride"),
    (dict(c=cache(max_pages=1 << 25, table_stride=1 << 25)), "2^30"),
    (dict(pool=None), "NULL"), (dict(pool=ADDR + 8), "aligned"), (dict(pages=None), "NULL"), (dict(k=None), "NULL"),
    (dict(v=None), "NULL"), (dict(start=None), "start"), (dict(k=ADDR + 1), "misaligned"),
    (dict(kd=tokens(heads=3)), "kv_heads"), (dict(kd=tokens(heads=2, batch=3)), "batch"),
    (dict(kd=tokens(heads=2, tokens=0)), "at least 1"), (dict(kd=tokens(heads=2, dtype=2)), "dtype"),
    (dict(kd=tokens(heads=2, dtype=F.F32)), "one dtype"), (dict(vd=tokens(heads=2, tokens=6)), "as many tokens"),
    (dict(kd=tokens(heads=2, stride=(-640, 128, 64))), "stride"),
])
def test_cache_refusals(bad, word):
    for write in (True, False):
        st, msg = io(write=write, **bad)
        assert st == INVALID and word in msg, (st, msg)


@pytest.mark.parametrize("bad, word", [
    (dict(o=opts(scale=0.0)), "scale"), (dict(o=opts(scale=-1.0)), "scale"), (dict(o=opts(scale=float("nan"))), "scale"),
    (dict(o=opts(scale=float("inf"))), "scale"), (dict(o=opts(window=-1)), "window"), (dict(o=opts(sinks=-1)), "sinks"),
    (dict(o=opts(causal=2)), "causal"), (dict(qd=tokens(heads=3), od=tokens(heads=3)), "multiple"),
    (dict(od=tokens(tokens=4)), "out"), (dict(od=tokens(dtype=F.F32)), "out"), (dict(q=None), "NULL"),
    (dict(out=None), "NULL"), (dict(qd=tokens(batch=3), od=tokens(batch=3)), "batch"),
    (dict(qd=tokens(head_dim=32), od=tokens(head_dim=32)), "head_dim"),
])
def test_attention_refusals(bad, word):
    for call in (kv, dense):
        st, msg = call(**bad)
        assert st == INVALID and word in msg, (st, msg)


def test_scales_whose_log2_form_is_no_number_are_refused():
    for call in (kv, dense):
        assert call(o=opts(scale=2.0 ** 127))[0] == UNSUPPORTED
        for scale in (2.4e38, 3.4e38):  # times log2(e): past fp32
            st, msg = call(o=opts(scale=scale))
            assert st == INVALID and "scale" in msg, (st, msg)


def test_what_no_launch_can_hold_is_refused():
    """A launch has fewer than 2^32 threads: 256 (or more) to four octets of
    tokens, to 128 rows of a kv head, to 16 rows over the cache."""
    def many(batch, tokens_=1, heads=128):  # one token's data for all
        return tokens(batch=batch, tokens=tokens_, heads=heads, head_dim=32, stride=(0, 0, 0))

    def out(batch, heads=128):
        return tokens(batch=batch, tokens=1, heads=heads, head_dim=32, stride=(32 * heads, 32, 32))
    for batch, st_ in ((1 << 17, UNSUPPORTED), (1 << 20, INVALID)):  # 2^24 and 2^27 octets
        c = cache(kv_heads=128, head_dim=32, batch=batch)
        st, msg = io(c=c, kd=many(batch), vd=many(batch))
        assert st == st_ and ("too large" in msg) == (st_ == INVALID), (batch, st, msg)
    for batch, st_ in ((1 << 16, UNSUPPORTED), (1 << 18, INVALID)):  # 2^23 and 2^25 kv heads
        c = cache(kv_heads=128, head_dim=32, batch=batch)
        for st, msg in (kv(c=c, qd=many(batch), od=out(batch)), dense(qd=many(batch), kd=many(batch), vd=many(batch), od=out(batch))):
            assert st == st_ and ("too large" in msg) == (st_ == INVALID), (batch, st, msg)
    most = (1 << 31) - 1  # counts whose product is past 64 bits
    c = cache(kv_heads=most, head_dim=32, batch=most)
    q = tokens(batch=most, tokens=1 << 30, heads=most, head_dim=32, stride=(0, 0, 0))
    o = tokens(batch=most, tokens=1 << 30, heads=most, head_dim=32, stride=(1 << 40, 1 << 40, 32))
    for st, msg in (io(c=c, kd=q, vd=q), kv(c=c, qd=q, od=o), dense(qd=q, kd=q, vd=q, od=o)):
        assert st == INVALID and "too large" in msg, (st, msg)
    c, n = cache(kv_heads=most, n_pages=most), C.c_uint64()
    assert A._lib().fluid_kv_pool_bytes(ref(c), C.byref(n)) == INVALID


def test_more_refusals():
    for st, msg, word in ((*kv(o=opts(causal=0)), "causal"), (*kv(kv_max=0), "kv_max"), (*kv(kv_len=None), "kv_len"),
                          (*kv(pool=ADDR + 4), "aligned"), (*dense(k=None), "NULL"),
                          (*dense(vd=tokens(heads=2, tokens=8)), "one dtype and shape"),
                          (*dense(kd=tokens(heads=2, tokens=9, dtype=F.F32)), "dtype"),
                          (*dense(qd=tokens(tokens=1 << 29, stride=(0, 0, 64)), od=tokens(tokens=1 << 29, stride=(0, 0, 64)),
                                  kd=tokens(heads=1), vd=tokens(heads=1)), "2^30 rows")):
        assert st == INVALID and word in msg, (st, msg)


def test_outputs_that_repeat_elements_are_refused():
    for stride in ((0, 128, 64), (640, 0, 64), (640, 128, 0), (640, 128, 32)):
        kd = tokens(heads=2, stride=stride)
        q = tokens(heads=2, stride=stride)
        assert io(kd=kd, vd=kd)[0] == UNSUPPORTED  # as inputs they may
        for st, msg in (io(kd=kd, write=False), io(vd=kd, write=False), kv(qd=q, od=q), dense(qd=q, od=q)):
            assert st == INVALID and "head_dim" in msg, (stride, st, msg)
    one = tokens(heads=2, batch=1, stride=(0, 128, 64))  # a stride that is never used
    assert io(c=cache(batch=1), kd=one, vd=one, write=False)[0] == UNSUPPORTED


def test_workspace_is_checked_and_only_needed_for_long_caches():
    lib, n = A._lib(), C.c_uint64()
    c, q = cache(max_pages=512, table_stride=512), tokens(tokens=1)
    assert lib.fluid_kv_attention_workspace(ref(c), ref(opts()), 100, ref(q), C.byref(n)) == 0 and n.value == 0
    assert kv(c=c, kv_max=100, qd=q, od=q, ws=None, ws_bytes=0)[0] == UNSUPPORTED
    assert lib.fluid_kv_attention_workspace(ref(c), ref(opts()), 32768, ref(q), C.byref(n)) == 0 and n.value > 0
    long = dict(c=c, kv_max=32768, qd=q, od=q)
    assert kv(**long, ws=ADDR, ws_bytes=n.value)[0] == UNSUPPORTED
    for bad in (dict(ws=ADDR, ws_bytes=n.value - 1), dict(ws=None, ws_bytes=n.value)):
        st, msg = kv(**long, **bad)
        assert st == TOO_SMALL and "workspace" in msg
    st, msg = kv(**long, ws=ADDR + 16, ws_bytes=n.value)
    assert st == INVALID and "aligned" in msg
    # a window bounds what is read, whatever the cache's length
    w = opts(window=64, sinks=4)
    assert lib.fluid_kv_attention_workspace(ref(c), ref(w), 32768, ref(q), C.byref(n)) == 0 and n.value == 0


def test_pool_bytes():
    lib, n = A._lib(), C.c_uint64()
    assert lib.fluid_kv_pool_bytes(ref(cache(head_dim=128, page_tokens=128, n_pages=1 << 20, kv_heads=8)),
                                   C.byref(n)) == 0
    assert n.value == (1 << 20) * 8 * A.pool_block(128, 128)
    assert lib.fluid_kv_pool_bytes(None, C.byref(n)) == INVALID


def test_binding_refuses_tensors_that_cannot_be_right():
    torch = pytest.importorskip("torch")
    cpu = torch.zeros(1, 4, 2, 64)
    pages = torch.zeros(1, 2, dtype=torch.int32)
    pool = torch.zeros(2, 2, A.pool_block(32, 64), dtype=torch.uint8)
    one = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: A.attention(cpu, cpu, cpu), lambda: A.kv_write(pool, pages, cpu, cpu, one),
                 lambda: A.kv_read(pool, pages, one, cpu, cpu), lambda: A.kv_attention(pool, pages, cpu, one)):
        with pytest.raises(F.FluidError, match="GPU"):
            call()
    dev = cpu.get_device()
    for bad, word in ((cpu[0], "dimensions"), (cpu.half(), "dtype"), (cpu.transpose(2, 3), "contiguous")):
        with pytest.raises(F.FluidError, match=word):
            A._describe(bad, "q", dev)
    with pytest.raises(F.FluidError, match="not on GPU 3"):
        A._describe(cpu, "q", 3)
    for bad in (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32),
                torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(F.FluidError, match="int32"):
            A._check_ints(bad, "start", 2, dev)
    for bad_pool, bad_pages, word in ((torch.zeros(2, 2, 100, dtype=torch.uint8), pages, "block"),
                                      (torch.zeros(2, 200, dtype=torch.uint8), pages, "pool"), (pool.float(), pages, "pool"),
                                      (pool, pages.long(), "pages"), (pool, pages[0], "pages")):
        with pytest.raises(F.FluidError, match=word):
            A._describe_cache(bad_pool, bad_pages, 64, dev)
    for window, sinks, word in ((-1, 0, "window"), (0, -1, "sinks"), (1 << 31, 0, "window")):
        with pytest.raises(F.FluidError, match=word):
            A._describe_opts(None, True, window, sinks, 64)


def test_calls_run_with_their_tensors_gpu_current(monkeypatch):
    """A default stream's handle is 0 on every GPU: without this the kernels of
    tensors on GPU 1 would run on GPU 0."""
    torch = pytest.importorskip("torch")
    at, seen = [0], []

    class On:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.was, at[0] = at[0], self.device

        def __exit__(self, *_):
            at[0] = self.was
    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(A, "_current_device", lambda: at[0])
    for device in (1, 0):
        A._launch(lambda *a: seen.append((at[0], a)) or 0, device, 5, 6)
    assert seen == [(1, (5, 6)), (0, (5, 6))] and at == [0]
    with pytest.raises(F.FluidError):
        A._launch(lambda: INVALID, 1)
    assert at == [0]


def test_tensors_that_want_gradients_are_refused():
    """There is no backward pass: the result would be detached without a word."""
    torch = pytest.importorskip("torch")
    x, want = torch.zeros(1, 4, 2, 64), torch.zeros(1, 4, 2, 64, requires_grad=True)
    pages, one = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    pool = torch.zeros(2, 2, A.pool_block(32, 64), dtype=torch.uint8)
    calls = [lambda a, b: A.attention(a, b, b), lambda a, b: A.attention(b, a, b), lambda a, b: A.attention(b, b, a),
             lambda a, b: A.attention(b, b, b, out=a), lambda a, b: A.kv_attention(pool, pages, a, one),
             lambda a, b: A.kv_attention(pool, pages, b, one, out=a), lambda a, b: A.kv_write(pool, pages, a, b, one),
             lambda a, b: A.kv_write(pool, pages, b, a, one), lambda a, b: A.kv_read(pool, pages, one, a, b),
             lambda a, b: A.kv_read(pool, pages, one, b, a)]
    for call in calls:
        with pytest.raises(F.FluidError, match="gradient"):
            call(want, x)
        with torch.no_grad(), pytest.raises(F.FluidError, match="GPU"):  # on to the next check
            call(want, x)


# ------------------------------------------------------- pins of the oracle
def test_quantised_values_are_near_and_exact_where_they_can_be():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((50, 64)) * np.exp(rng.standard_normal((50, 1)))).astype(np.float32)
    n, s, b = OA.quantise(x)
    assert n.min() == 0 and n.max() == 15
    y = OA.values(n, s, b)
    half = np.repeat(s.astype(np.float64), 32, -1)
    # half a step, b's rounding to f16 (its size is below 16 s + |x|), the value's
    assert (np.abs(y - x) <= 0.5 * half + 2.0 ** -11 * (16 * half + 2 * np.abs(x)) + 2.0 ** -24).all()
    flat = np.full((1, 32), 0.375, np.float32)
    assert (OA.values(*OA.quantise(flat)) == 0.375).all()
    ramp = np.arange(32, dtype=np.float32)[None] % 16 * 0.25 - 1
    assert (OA.values(*OA.quantise(ramp)) == ramp).all()


def test_oracle_cache_reads_what_it_wrote_and_keeps_neighbours():
    rng = np.random.default_rng(2)
    pool = np.zeros((2, 1, A.pool_block(32, 64)), np.uint8)
    c = OA.Cache(pool, 32, 64)
    x = rng.standard_normal((32, 2, 64)).astype(np.float32)
    for t in rng.permutation(32):
        c.write(1, 0, int(t), x[t, 0], x[t, 1])
    for t in range(32):
        k, v = c.read(1, 0, t)
        assert (k == OA.values(*OA.quantise(x[t, 0]))).all() and (v == OA.values(*OA.quantise(x[t, 1]))).all()
    assert not pool[0].any()


def test_oracle_attention_against_plain_sums():
    rng = np.random.default_rng(3)
    q, k, v = (rng.standard_normal((n, 8)) for n in (5, 9, 9))
    for causal, window, sinks in ((True, 0, 0), (True, 3, 1), (False, 2, 0), (False, 0, 0)):
        out, mass, _ = OA.attention(q, k, v, 0.3, causal, window, sinks)
        for i in range(5):
            w = [np.exp(0.3 * q[i] @ k[j]) if OA.sees(4 + i, j, 9, causal, window, sinks) else 0.0 for j in range(9)]
            assert np.allclose(out[i], sum(a * x for a, x in zip(w, v)) / sum(w), atol=1e-12)
            assert (mass[i] >= np.abs(out[i]) - 1e-12).all()
    out, _, _ = OA.attention(np.ones((3, 8)), np.ones((1, 8)), np.ones((1, 8)), 1.0)
    assert (out[:2] == 0).all() and (out[2] == 1).all()  # the first two rows sit before the only token
