"""Rotary positions, linear attention and 4-bit matrices without a GPU: both
libraries export the calls, what cannot be right is refused with a cause before
any launch, what is right reaches the (here missing) GPU; turns; the oracle's own
pins."""
import ctypes as C
import math
import os
import re

import numpy as np
import pytest

from oracle import decoder_layers as O
from paper_2411_09242_amd import attention as A
from paper_2411_09242_amd import fluid as F
from paper_2411_09242_amd import w4 as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, TOO_SMALL = -1, -2, -4
ADDR = 1 << 20  # a plausible, 256-byte aligned address; never read on the host


@pytest.fixture(scope="module", autouse=True)
def host_lib():
    F.load(host_only=True)
    yield
    F.load(host_only=True)


@pytest.mark.parametrize("name", ["libfluid_host.so", "libfluid.so"])
def test_libraries_export_every_declared_symbol(name):
    lib = C.CDLL(os.path.join(F.LIBDIR, name))
    src = open(os.path.join(ROOT, "include", "fluid_w4.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    syms = set(re.findall(r"\b(fluid_[a-z0-9_]+)\s*\(", src))
    assert syms == set(W.SYMBOLS)
    for s in syms:
        assert hasattr(lib, s), s


def ref(x):
    return None if x is None else C.byref(x)


def error():
    return A._lib().fluid_last_error().decode()


def tokens(dtype=F.BF16, batch=2, tokens=5, heads=4, head_dim=64, stride=None):
    stride = stride or (tokens * heads * head_dim, heads * head_dim, head_dim)
    return A.Tokens(dtype, batch, tokens, heads, head_dim, (C.c_int64 * 3)(*stride))


# ------------------------------------------------------------------ rotary
def desc(dim=64, interleaved=0, scaling=0, amplitude=1.0, base=10000.0, factor=1.0, length=0.0, low=1.0, high=32.0):
    return A.RotaryDesc(dim, interleaved, scaling, amplitude, base, factor, length, low, high)


def rotate(r=None, turns=ADDR, start=None, positions=None, pstride=5, count=None, inverse=0, qd=None, q=ADDR, qod=None,
           qo=ADDR + 4096, kd=None, k=ADDR + 8192, kod=None, ko=ADDR + 12288, no_r=False):
    qd = qd or tokens()
    qod = qod or qd
    st = A._lib().fluid_rotate(None if no_r else ref(r or desc()), turns, start, positions, pstride, count, inverse, ref(qd),
                               q, ref(qod), qo, ref(kd), k, ref(kod or kd), ko, None)
    return st, error()


def test_right_rotary_calls_reach_the_gpu_part():
    for kw in (dict(), dict(kd=tokens(heads=2)), dict(start=ADDR), dict(positions=ADDR), dict(qo=ADDR),
               dict(qd=tokens(head_dim=80), r=desc(dim=40)), dict(qd=tokens(head_dim=7), r=desc(dim=6, interleaved=1)),
               dict(qd=tokens(dtype=F.F32, head_dim=1024), r=desc(dim=1024)), dict(inverse=1, count=ADDR)):
        st, msg = rotate(**kw)
        assert st == UNSUPPORTED and "host-only" in msg, (kw, msg)


@pytest.mark.parametrize("bad, word", [
    (dict(no_r=True), "NULL"), (dict(r=desc(dim=0)), "dim"), (dict(r=desc(dim=63)), "dim"), (dict(r=desc(dim=1026)), "dim"),
    (dict(r=desc(dim=66)), "larger than head_dim"), (dict(r=desc(interleaved=2)), "interleaved"),
    (dict(r=desc(scaling=4)), "scaling"), (dict(r=desc(scaling=-1)), "scaling"), (dict(r=desc(amplitude=math.inf)), "amplitude"),
    (dict(r=desc(base=0.5)), "base"), (dict(r=desc(base=math.nan)), "base"), (dict(r=desc(scaling=1, factor=0.0)), "factor"),
    (dict(r=desc(scaling=1, factor=math.nan)), "factor"), (dict(r=desc(dim=2, scaling=2, factor=2.0)), "at least 4"),
    (dict(r=desc(scaling=3, factor=2.0)), "length"), (dict(r=desc(scaling=3, length=9.0, low=4.0, high=4.0)), "low"),
    (dict(turns=None), "turns"), (dict(turns=ADDR + 4), "turns"), (dict(start=ADDR, positions=ADDR), "only one"),
    (dict(inverse=2), "inverse"), (dict(q=None), "NULL"), (dict(qo=None), "NULL"), (dict(kd=tokens(heads=2), k=None), "NULL"),
    (dict(kd=tokens(heads=2), ko=None), "NULL"), (dict(qod=tokens(heads=3)), "shape"), (dict(qod=tokens(dtype=F.F32)), "dtype"),
    (dict(kd=tokens(heads=2, tokens=6)), "one dtype"), (dict(kd=tokens(dtype=F.F32)), "one dtype"),
    (dict(kd=tokens(head_dim=128)), "one dtype"), (dict(q=ADDR + 1), "misaligned"), (dict(qd=tokens(tokens=0)), "at least 1"),
    (dict(qd=tokens(head_dim=1025), r=desc(dim=64)), "head_dim"), (dict(qd=tokens(stride=(-64, 64, 64))), "stride"),
    (dict(qod=tokens(stride=(1280, 256, 63))), "head_dim"), (dict(qo=ADDR, qod=tokens(stride=(2560, 256, 64))), "strides"),
    (dict(positions=ADDR, pstride=-1), "position_stride"),
    (dict(qd=tokens(batch=1 << 20, tokens=1 << 20, stride=(0, 0, 64)), qod=tokens(batch=1 << 20, tokens=1 << 20,
                                                                                  stride=(1 << 30, 256, 64))), "too large"),
])
def test_rotary_refusals(bad, word):
    st, msg = rotate(**bad)
    assert st == INVALID and word in msg, (st, msg)


@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling="linear", factor=4.0), dict(scaling="linear", factor=0.1),
                                dict(scaling="base", factor=8.0), dict(scaling="ramp", factor=8.0, length=8192, low=1.0, high=4.0),
                                dict(scaling="ramp", factor=32.0, length=4096, low=1.0, high=32.0), dict(base=1.0)])
@pytest.mark.parametrize("dim", [4, 64, 128, 1024])
def test_turns_are_the_frequencies(kw, dim):
    opt = dict(kw, scaling=A.SCALINGS[kw.get("scaling", "none")])
    turns = (C.c_uint64 * (dim // 2))()
    assert A._lib().fluid_rotary_turns(ref(desc(dim, **opt)), turns) == 0
    want = O.frequencies(dim, **kw) / (2 * O.PI)
    for t, w in zip(turns, want):
        part = w - np.floor(w)
        off = abs(int(t) - int(np.floor(np.ldexp(part, 64))))
        assert min(off, 2 ** 64 - off) <= 4 + 64 * float(w), (t, w)  # a few units of the long float's last place


def test_rotary_object_refuses():
    pytest.importorskip("torch")
    for kw, word in ((dict(dim=64, scaling="other"), "scaling"), (dict(dim=0), "dim"), (dict(dim=5), "even"),
                     (dict(dim=64, base=0.0), "base")):
        with pytest.raises(F.FluidError, match=word):
            A.Rotary(device="cpu", **kw)


def test_oracle_rotation_pins():
    x = np.arange(8, dtype=np.float64).reshape(1, 1, 8)
    theta = O.frequencies(4, base=4.0)
    assert np.allclose(theta.astype(float), [1.0, 0.5])
    y = O.rotate(x, [3], theta)
    c, s = np.cos([3, 1.5]), np.sin([3, 1.5])
    assert np.allclose(y[0, 0], [0 * c[0] - 2 * s[0], 1 * c[1] - 3 * s[1], 2 * c[0] + 0 * s[0], 3 * c[1] + 1 * s[1], 4, 5, 6, 7])
    z = O.rotate(x, [3], theta, interleaved=True, amplitude=2.0)
    assert np.allclose(z[0, 0, :4], [2 * (0 * c[0] - 1 * s[0]), 2 * (1 * c[0]), 2 * (2 * c[1] - 3 * s[1]), 2 * (3 * c[1] + 2 * s[1])])
    assert np.allclose(O.rotate(y, [3], theta, inverse=True), x)


# -------------------------------------------------------- linear attention
def linear(scale=0.5, qd=None, q=ADDR, kd=None, k=ADDR, vd=None, v=ADDR, decay=ADDR, stride=(0, 0, 1), state=ADDR, count=None,
           od=None, out=ADDR + (1 << 24), state_out=ADDR, ws=ADDR, ws_bytes=1 << 40):
    qd = qd or tokens()
    kd = kd or tokens(heads=2)
    stride = None if stride is None else (C.c_int64 * 3)(*stride)
    st = A._lib().fluid_linear_attention(scale, ref(qd), q, ref(kd), k, ref(vd or kd), v, decay, stride, state, count,
                                         ref(od or qd), out, state_out, ws, ws_bytes, None)
    return st, error()


def test_right_linear_calls_reach_the_gpu_part():
    for kw in (dict(), dict(state=None, state_out=None), dict(count=ADDR),
               dict(state_out=ADDR + 2 * 2 * 64 * 64 * 4), dict(state=ADDR + 2 * 2 * 64 * 64 * 4), dict(stride=(10, 2, 1)), dict(scale=-1.0),
               dict(qd=tokens(tokens=3000), kd=tokens(tokens=3000, heads=1)),
               dict(qd=tokens(dtype=F.F32, head_dim=128), kd=tokens(dtype=F.F32, head_dim=128, heads=4))):
        st, msg = linear(**kw)
        assert st == UNSUPPORTED and "host-only" in msg, (kw, msg)


@pytest.mark.parametrize("bad, word", [
    (dict(scale=math.inf), "scale"), (dict(scale=math.nan), "scale"), (dict(q=None), "NULL"), (dict(k=None), "NULL"),
    (dict(v=None), "NULL"), (dict(out=None), "NULL"), (dict(decay=None), "decay"), (dict(decay=ADDR + 2), "decay"),
    (dict(stride=None), "decay_stride"), (dict(stride=(0, -1, 0)), "decay"), (dict(state=ADDR + 4), "aligned"),
    (dict(state_out=ADDR + 8), "aligned"), (dict(kd=tokens(heads=3)), "multiple"), (dict(kd=tokens(heads=2, tokens=6)), "one dtype"),
    (dict(kd=tokens(heads=2, dtype=F.F32)), "one dtype"), (dict(vd=tokens(heads=1)), "one dtype and shape"),
    (dict(od=tokens(tokens=6)), "out"), (dict(od=tokens(stride=(1280, 0, 64))), "head_dim"),
    *((dict(out=ADDR + (2 << 24), **{name: ADDR + (2 << 24)}), "must not be q, k or v") for name in "qkv"),
    (dict(state_out=ADDR + 2 * 2 * 64 * 64 * 4 - 16), "apart"), (dict(state=ADDR + 16), "apart"),
    (dict(qd=tokens(head_dim=48), kd=tokens(head_dim=48, heads=2)), "head_dim"), (dict(qd=tokens(tokens=0)), "at least 1"),
    (dict(qd=tokens(batch=1 << 20, heads=64, stride=(0, 0, 0)), kd=tokens(batch=1 << 20, heads=64, stride=(0, 0, 0)),
          od=tokens(batch=1 << 20, heads=64, stride=(1 << 20, 1 << 14, 64))), "too large"),
])
def test_linear_attention_refusals(bad, word):
    st, msg = linear(**bad)
    assert st == INVALID and word in msg, (st, msg)


def test_linear_attention_workspace_is_checked():
    n = C.c_uint64()
    qd, kd = tokens(batch=1, tokens=8192, heads=4, head_dim=128), tokens(batch=1, tokens=8192, heads=4, head_dim=128)
    assert A._lib().fluid_linear_attention_workspace(ref(qd), ref(kd), C.byref(n)) == 0
    if n.value:
        assert linear(qd=qd, kd=kd, ws_bytes=n.value)[0] == UNSUPPORTED
        for bad in (dict(ws_bytes=n.value - 1), dict(ws=None)):
            st, msg = linear(qd=qd, kd=kd, **bad)
            assert st == TOO_SMALL and "workspace" in msg
        st, msg = linear(qd=qd, kd=kd, ws=ADDR + 64)
        assert st == INVALID and "aligned" in msg
    one = tokens(tokens=1)
    assert A._lib().fluid_linear_attention_workspace(ref(one), ref(one), C.byref(n)) == 0 and n.value == 0
    assert A._lib().fluid_linear_attention_workspace(ref(one), None, C.byref(n)) == INVALID


def test_oracle_linear_attention_against_plain_sums():
    rng = np.random.default_rng(1)
    q, k, v, g = rng.standard_normal((6, 2, 8)), rng.standard_normal((6, 8)), rng.standard_normal((6, 8)), -rng.random(6)
    S0 = rng.standard_normal((8, 8))
    out, last, size, M = O.linear_attention(q, k, v, g, S0, 0.7)
    c = np.cumsum(g)
    for t in range(6):
        for j in range(2):
            w = [np.exp(c[t] - c[i]) * (q[t, j] @ k[i]) for i in range(t + 1)]
            want = 0.7 * (sum(a * v[i] for i, a in enumerate(w)) + np.exp(c[t]) * (q[t, j] @ S0))
            assert np.allclose(out[t, j], want) and (size[t, j] >= np.abs(want) - 1e-12).all()
    assert np.allclose(last, np.exp(c[5]) * S0 + sum(np.exp(c[5] - c[i]) * np.outer(k[i], v[i]) for i in range(6)))
    assert (M >= np.abs(last) - 1e-12).all()


# ---------------------------------------------------------- 4-bit matrices
def shape(rows=40, cols=200, group=64):
    return W.W4Desc(rows, cols, group)


def matrix(rows=3, cols=200, dtype=F.BF16, stride=None):
    return W.Matrix(dtype, rows, cols, cols if stride is None else stride)


def matmul(w=None, packed=ADDR, gate=None, xd=None, x=ADDR, ad=None, add=None, od=None, out=ADDR + 65536, no_w=False,
           ws=ADDR, ws_bytes=1 << 40):
    st = W._lib().fluid_w4_matmul(None if no_w else ref(w or shape()), packed, gate, ref(xd or matrix()), x, ref(ad), add,
                                  ref(od or matrix(cols=40)), out, ws, ws_bytes, None)
    return st, error()


def test_right_products_reach_the_gpu_part():
    for kw in (dict(), dict(gate=ADDR), dict(ad=matrix(cols=40), add=ADDR), dict(ad=matrix(cols=40), add=ADDR + 65536),
               dict(xd=matrix(stride=0)), dict(xd=matrix(stride=203)), dict(xd=matrix(dtype=F.F32), od=matrix(cols=40, dtype=F.F32)),
               dict(w=shape(cols=1, rows=1), xd=matrix(cols=1), od=matrix(cols=1))):
        st, msg = matmul(**kw)
        assert st == UNSUPPORTED and "host-only" in msg, (kw, msg)


@pytest.mark.parametrize("bad, word", [
    (dict(no_w=True), "NULL"), (dict(w=shape(rows=0)), "at least 1"), (dict(w=shape(cols=0)), "at least 1"),
    (dict(w=shape(group=16)), "group"), (dict(w=shape(group=96)), "group"), (dict(packed=None), "NULL"),
    (dict(packed=ADDR + 8), "aligned"), (dict(gate=ADDR + 4), "aligned"), (dict(x=None), "NULL"), (dict(out=None), "NULL"),
    (dict(x=ADDR + 1), "misaligned"), (dict(xd=matrix(cols=201)), "cols"), (dict(xd=matrix(dtype=2)), "dtype"),
    (dict(xd=matrix(rows=0)), "at least 1"), (dict(xd=matrix(stride=-1)), "stride"), (dict(od=matrix(cols=41)), "cols"),
    (dict(od=matrix(cols=40, rows=4)), "out"), (dict(od=matrix(cols=40, dtype=F.F32)), "out"),
    (dict(od=matrix(cols=40, stride=39)), "stride"), (dict(ad=matrix(cols=40, rows=2), add=ADDR), "add"),
    (dict(ad=None, add=ADDR), "add"), (dict(ad=matrix(cols=40, stride=50), add=ADDR + 65536), "stride"), (dict(out=ADDR), "out"),
    (dict(xd=matrix(rows=1 << 24), od=matrix(rows=1 << 24, cols=40)), "too many rows"),
    (dict(w=shape(rows=1 << 27), od=matrix(cols=1 << 27)), "too large"),
])
def test_product_refusals(bad, word):
    st, msg = matmul(**bad)
    assert st == INVALID and word in msg, (st, msg)


def test_product_workspace_is_checked():
    lib, n = W._lib(), C.c_uint64()
    x = lambda rows, dtype=F.BF16: ref(matrix(rows=rows, cols=8192, dtype=dtype))  # noqa: E731
    w = shape(rows=512, cols=8192)
    kw = dict(w=w, xd=matrix(rows=40, cols=8192), od=matrix(rows=40, cols=512))
    assert lib.fluid_w4_matmul_workspace(ref(w), x(40), 0, C.byref(n)) == 0 and n.value > 0
    assert matmul(**kw, ws_bytes=n.value)[0] == UNSUPPORTED
    for bad in (dict(ws_bytes=n.value - 1), dict(ws=None)):
        st, msg = matmul(**kw, **bad)
        assert st == TOO_SMALL and "workspace" in msg
    st, msg = matmul(**kw, ws=ADDR + 16)
    assert st == INVALID and "aligned" in msg
    assert lib.fluid_w4_matmul_workspace(ref(w), x(40), 1, C.byref(n)) == 0 and matmul(**kw, gate=ADDR, ws_bytes=n.value)[0] == UNSUPPORTED
    for rows, dtype in ((16, F.BF16), (16, F.F32), (32, F.BF16)):
        assert lib.fluid_w4_matmul_workspace(ref(w), x(rows, dtype), 0, C.byref(n)) == 0 and n.value == 0
    assert lib.fluid_w4_matmul_workspace(ref(w), x(32, F.F32), 0, C.byref(n)) == 0 and n.value > 0
    kw = dict(w=w, xd=matrix(rows=16, cols=8192), od=matrix(rows=16, cols=512))
    assert matmul(**kw, ws=None, ws_bytes=0)[0] == UNSUPPORTED
    for bad in ((w, x(0), 0), (w, x(40), 2), (shape(group=5), x(40), 0), (w, None, 0), (w, x(40, 2), 0),
                (w, ref(matrix(rows=40, cols=8191)), 0)):
        assert lib.fluid_w4_matmul_workspace(ref(bad[0]), bad[1], bad[2], C.byref(n)) == INVALID
    assert lib.fluid_w4_matmul_workspace(ref(w), x(40), 0, None) == INVALID


def test_packing_and_reading_refusals():
    lib = W._lib()
    m = matrix(rows=40)
    assert lib.fluid_w4_pack(ref(shape()), ref(m), ADDR, ADDR, None) == UNSUPPORTED
    assert lib.fluid_w4_read(ref(shape()), ADDR, ref(m), ADDR, None) == UNSUPPORTED
    for f in (lambda w, d, x, p: lib.fluid_w4_pack(ref(w), ref(d), x, p, None),
              lambda w, d, x, p: lib.fluid_w4_read(ref(w), p, ref(d), x, None)):
        for bad, word in (((shape(rows=41), m, ADDR, ADDR), "rows"), ((shape(cols=199), m, ADDR, ADDR), "cols"),
                          ((shape(), m, None, ADDR), "NULL"), ((shape(), m, ADDR, None), "NULL"),
                          ((shape(), m, ADDR, ADDR + 2), "aligned"), ((shape(), None, ADDR, ADDR), "NULL"),
                          ((shape(rows=1 << 29, cols=1 << 20), matrix(rows=1 << 29, cols=1 << 20), ADDR, ADDR), "too large")):
            assert f(*bad) == INVALID and word in error(), (word, error())
    assert lib.fluid_w4_read(ref(shape()), ADDR, ref(matrix(rows=40, stride=199)), ADDR, None) == INVALID
    n = C.c_uint64()
    assert lib.fluid_w4_bytes(ref(shape()), C.byref(n)) == 0 and n.value == 3 * 2 * (1024 + 128)
    assert lib.fluid_w4_bytes(ref(shape()), None) == INVALID


def test_bindings_refuse_tensors_that_cannot_be_right():
    torch = pytest.importorskip("torch")
    x, w = torch.zeros(3, 200), W.W4(torch.zeros(W.w4_bytes(40, 200, 64), dtype=torch.uint8), 40, 200, 64)
    t, rot, g = torch.zeros(1, 4, 2, 64), A.Rotary(64, device="cpu"), torch.zeros(2)
    for call in (lambda: W.w4_matmul(x, w), lambda: W.w4_pack(x), lambda: W.w4_read(w), lambda: A.rotary(rot, t),
                 lambda: A.linear_attention(t, t, t, g)):
        with pytest.raises(F.FluidError, match="GPU"):
            call()
    for bad, word in ((torch.zeros(5, dtype=torch.uint8), "bytes"), (torch.zeros(W.w4_bytes(40, 200, 64)), "bytes")):
        with pytest.raises(F.FluidError, match=word):
            W.W4(bad, 40, 200, 64)
    dev = x.get_device()
    for bad, word in ((torch.zeros(200), "two dimensions"), (x.half(), "dtype"), (x.t(), "contiguous"),
                      (torch.zeros(2, 3, 8)[:, :2], "one distance")):
        with pytest.raises(F.FluidError, match=word):
            W._matrix(bad, "x", dev)
    m = W._matrix(torch.zeros(2, 3, 4, 8)[..., :5], "x", dev)
    assert (m.rows, m.cols, m.stride) == (24, 5, 8)
    m = W._matrix(torch.zeros(1, 1, 8), "x", dev)
    assert (m.rows, m.cols) == (1, 8)
    want = x.clone().requires_grad_()
    tw = t.clone().requires_grad_()
    for call in (lambda: W.w4_matmul(want, w), lambda: W.w4_matmul(x, w, add=want), lambda: W.w4_pack(want),
                 lambda: A.rotary(rot, tw), lambda: A.rotary(rot, t, tw), lambda: A.linear_attention(tw, t, t, g),
                 lambda: A.linear_attention(t, t, t, g.clone().requires_grad_())):
        with pytest.raises(F.FluidError, match="gradient"):
            call()


def test_oracle_bytes_and_values():
    rng = np.random.default_rng(2)
    w = rng.standard_normal((18, 150)).astype(np.float32)
    n, s, b = O.quantise(w, 32)
    step = np.repeat(s.astype(np.float64), 32, 1)[:, :150]
    assert (np.abs(O.values(n, s, b, 32) - w) <= 0.5 * step + 2.0 ** -11 * (32 * step + 2 * np.abs(w)) + 2.0 ** -23).all()
    packed = O.pack(n, s, b, 32)
    assert packed.size == W.w4_bytes(18, 150, 32)
    words = packed[:2 * 2 * 1024].view(np.uint32).reshape(2, 2, 64, 4)
    # row 17, channel 130: the second tiles, inside 2: word 0 of place 0 + 1, element 2 at nibble 1
    assert (words[1, 1, 1, 0] >> 4) & 15 == n[17, 130]
    y, size = O.product(rng.standard_normal((3, 150)), n, s, b, 32)
    assert (size >= np.abs(y)).all()


# --------------------------------------- bounds that the headers state, and sizes
def exact_frequencies(dim, base=10000.0, scaling="none", factor=1.0, length=0.0, low=1.0, high=32.0):
    """theta_i / (2 pi) and theta_i, in 60 digits."""
    from decimal import Decimal as D, getcontext
    getcontext().prec = 60
    tau = 2 * D("3.14159265358979323846264338327950288419716939937510582097494")
    base, factor = D(base), D(factor)
    if scaling == "base":
        base = base * factor ** (D(dim) / D(dim - 2))
    for i in range(dim // 2):
        theta = base ** (D(-2 * i) / D(dim))
        if scaling == "linear":
            theta /= factor
        if scaling == "ramp":
            kept = min(D(1), max(D(0), (D(length) * theta / tau - D(low)) / (D(high) - D(low))))
            theta = kept * theta + (1 - kept) * theta / factor
        yield theta / tau, theta


@pytest.mark.parametrize("kw", [
    dict(), dict(base=500000.0), dict(base=1.0), dict(base=1e300), dict(scaling="linear", factor=4.0),
    dict(scaling="base", factor=8.0), dict(scaling="base", base=500000.0, factor=2.5),
    dict(scaling="ramp", factor=8.0, length=8192, low=1.0, high=4.0),
    dict(scaling="ramp", factor=32.0, length=4096, low=1.0, high=32.0),
    dict(scaling="linear", factor=0.1), dict(scaling="linear", factor=1e-3), dict(scaling="linear", factor=1e-6),
    dict(scaling="base", factor=0.01), dict(scaling="ramp", factor=0.25, length=8192, low=1.0, high=4.0)])
@pytest.mark.parametrize("dim", [4, 30, 64, 128, 1024])
def test_turns_are_within_the_units_that_the_header_states(kw, dim):
    opt = dict(kw, scaling=A.SCALINGS[kw.get("scaling", "none")])
    turns = (C.c_uint64 * (dim // 2))()
    assert A._lib().fluid_rotary_turns(ref(desc(dim, **opt)), turns) == 0
    for t, (turn, theta) in zip(turns, exact_frequencies(dim, **kw)):
        off = abs(int(t) - (turn % 1) * 2 ** 64)
        assert min(off, 2 ** 64 - off) <= max(1, theta), (t, turn, float(off))


def linear_need(qd, kd):
    n = C.c_uint64()
    assert A._lib().fluid_linear_attention_workspace(ref(qd), ref(kd), C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("shape, heads, places", [
    (dict(batch=1, tokens=8192, head_dim=128), (4, 4), None),          # runs
    (dict(batch=1, tokens=1200, head_dim=128), (2, 2), None),
    (dict(batch=1, tokens=1200, head_dim=64, dtype=F.F32), (8, 2), None),
    (dict(batch=3, tokens=40, head_dim=64), (4, 2), 1),                # one run of shared heads: a state each
    (dict(batch=3, tokens=40, head_dim=64), (2, 2), 0),                # nothing is read by others than write it
    (dict(batch=3, tokens=2, head_dim=64), (4, 2), 0)])
def test_linear_attention_workspace_is_there_and_enough(shape, heads, places):
    qd, kd = (tokens(**shape, heads=h, stride=(1 << 30, 1 << 16, 128)) for h in heads)
    n, state = linear_need(qd, kd), shape["batch"] * heads[1] * (shape["head_dim"] ** 2 + 1) * 4
    assert n % state == 0 and (n // state >= 2 if places is None else n == places * state)
    if n:
        assert linear(qd=qd, kd=kd, ws_bytes=n)[0] == UNSUPPORTED
        for bad in (dict(ws_bytes=n - 1), dict(ws=None)):
            st, msg = linear(qd=qd, kd=kd, **bad)
            assert st == TOO_SMALL and "workspace" in msg
        st, msg = linear(qd=qd, kd=kd, ws=ADDR + 64)
        assert st == INVALID and "aligned" in msg


@pytest.mark.parametrize("bad, word", [
    (dict(ko=ADDR + 4096), "same"), (dict(q=ADDR, k=ADDR, qo=ADDR, ko=ADDR), "same"), (dict(qo=ADDR + 8192), "q_out must not be k"),
    (dict(ko=ADDR), "k_out must not be q"), (dict(k=ADDR, qo=ADDR), "q_out must not be k")])
def test_rotary_refuses_outputs_that_others_read_or_write(bad, word):
    st, msg = rotate(kd=tokens(), **bad)
    assert st == INVALID and word in msg, (st, msg)


def test_rotary_of_one_tensor_twice_and_in_place():
    for kw in (dict(k=ADDR), dict(qo=ADDR, ko=ADDR + 8192), dict(qo=ADDR), dict(ko=ADDR + 8192)):
        st, msg = rotate(kd=tokens(), **kw)
        assert st == UNSUPPORTED and "host-only" in msg, (kw, msg)
