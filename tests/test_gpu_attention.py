"""The 4-bit cache, attention over it, and windowed attention on the GPU
against plain NumPy in 64 bits (oracle/attention.py).

Tolerances.  With u = 2^-24 the fp32 rounding unit, a dot product of n fp32
terms is off by at most n u times the sum of its terms' sizes.  A score's error
is therefore at most (D + 8) u S, with S the largest sum of |q k| scale a row
sees (the 8 for the scale, the maximum's subtraction and the exponential's own
rounding), an attention weight's relative error twice that plus that of the
sum over N tokens, and an output's error the weights' error times M = sum of
p |v|, with N u again for its own sum.  On top of that:
  * bf16 tensors: attention rounds the weights to bf16 (8 bits: 2^-8), the
    cache's to f16 (11 bits: 2^-11) and its queries to f16 below 2^-14 of a
    row's largest (2^-25 of it: D 2^-25 of S at most); the output is rounded
    to bf16 (2^-8 of it);
  * fp32 tensors over the cache: queries and weights are two f16 parts each
    (2^-22 of the value, 2^-25 of the largest query).
"""
import itertools

import numpy as np
import pytest

from oracle import attention as OA

torch = pytest.importorskip("torch")
from paper_2411_09242_amd import attention as A  # noqa: E402
from paper_2411_09242_amd import fluid as F  # noqa: E402

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def gpu_lib():
    F.load()
    yield


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rand(seed, *shape, dtype="f32", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(DT[dtype]).cuda()


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


def laid_out(t, how):
    """The same values in other strides: heads before tokens, rows padded (16
    bytes kept or broken), or an odd start."""
    B, T, H, D = t.shape
    if how == "heads_first":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    pad = {"padded": 16, "odd": 3}[how]
    buf = torch.full((B, T, H, D + pad), 7.0, dtype=t.dtype, device=t.device)
    off = 1 if how == "odd" else 0
    buf[..., off:off + D] = t
    return buf[..., off:off + D]


class Paged:
    """A pool with shuffled pages for `lens` tokens a sequence."""

    def __init__(self, lens, H, D, P, seed=0, spare=3, fill=None):
        per = max(1, max(-(-n // P) for n in lens))
        n = len(lens) * per + spare
        perm = np.random.default_rng(seed).permutation(n)[:len(lens) * per].reshape(len(lens), per)
        self.table = perm
        self.pages = torch.tensor(perm, dtype=torch.int32, device="cuda")
        self.pool = torch.zeros(n, H, A.pool_block(P, D), dtype=torch.uint8, device="cuda")
        if fill is not None:
            self.pool.fill_(fill)
        self.P, self.D, self.H = P, D, H

    def mirror(self):
        return OA.Cache(self.pool.cpu().numpy().copy(), self.P, self.D)

    def put(self, mirror, b, h, pos, k, v):
        mirror.write(self.table[b][pos // self.P], h, pos % self.P, k, v)


# ------------------------------------------------------------- write, read
IO = [("bf16", 32, 32, 2, [0, 3], [1, 1]), ("bf16", 64, 64, 1, [5, 62], [11, 3]), ("bf16", 128, 32, 2, [0, 31], [37, 9]),
      ("f32", 32, 64, 1, [7, 0], [2, 8]), ("f32", 64, 32, 2, [0, 17], [33, 16]), ("f32", 128, 128, 1, [120, 1], [20, 6])]


@pytest.mark.parametrize("dtype, D, P, H, start, count", IO)
@pytest.mark.parametrize("how", [None, "heads_first", "padded", "odd"])
def test_write_makes_the_formats_bytes_and_read_gives_their_values(dtype, D, P, H, start, count, how):
    lens = [s + c for s, c in zip(start, count)]
    pg = Paged(lens, H, D, P, fill=0xA5)
    T = max(count) + 1
    k, v = rand(1, 2, T, H, D, dtype=dtype), rand(2, 2, T, H, D, dtype=dtype, scale=3.0)
    if how:
        k, v = laid_out(k, how), laid_out(v, how)
    m = pg.mirror()
    A.kv_write(pg.pool, pg.pages, k, v, ints(start), ints(count))
    hk, hv = host(k).astype(np.float32), host(v).astype(np.float32)
    for b, h in itertools.product(range(2), range(H)):
        for i in range(count[b]):
            pg.put(m, b, h, start[b] + i, hk[b, i, h], hv[b, i, h])
    assert (pg.pool.cpu().numpy() == m.pool).all()
    ko, vo = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    if how:
        ko, vo = laid_out(ko, how), laid_out(vo, how)
    A.kv_read(pg.pool, pg.pages, ints(start), ko, vo, ints(count))
    for b, h, i in itertools.product(range(2), range(H), range(T)):
        if i >= count[b]:
            assert (host(ko)[b, i, h] == 9.0).all() and (host(vo)[b, i, h] == 9.0).all()
            continue
        pos = start[b] + i
        want = m.read(pg.table[b][pos // P], h, pos % P)
        for got, w in zip((ko, vo), want):
            assert (host(got)[b, i, h] == host(torch.tensor(w).to(DT[dtype]))).all()


def test_every_group_of_many_is_rounded_as_the_format_says():
    """Pairs that one rounding more or less changes are one group in thousands."""
    T, H, D = 2048, 16, 128
    for dtype in ("f32", "bf16"):
        k = rand(1, 1, T, H, D) * torch.exp(2 * rand(3, 1, T, H, 1)) + rand(4, 1, 1, H, D)
        v = rand(2, 1, T, H, D).abs() * 100
        k, v = k.to(DT[dtype]), v.to(DT[dtype])
        pg = Paged([T], H, D, 256)
        A.kv_write(pg.pool, pg.pages, k, v, ints([0]))
        ko, vo = torch.empty(1, T, H, D, device="cuda"), torch.empty(1, T, H, D, device="cuda")
        A.kv_read(pg.pool, pg.pages, ints([0]), ko, vo)
        for x, got in ((k, ko), (v, vo)):
            assert (host(got) == OA.values(*OA.quantise(host(x).astype(np.float32)))).all()


@pytest.mark.parametrize("D", [32, 64, 128])
def test_token_by_token_writes_the_bytes_of_one_call(D):
    k, v = rand(3, 1, 45, 2, D, dtype="bf16"), rand(4, 1, 45, 2, D, dtype="bf16")
    one, many = Paged([45], 2, D, 32), Paged([45], 2, D, 32)
    A.kv_write(one.pool, one.pages, k, v, ints([0]))
    order = np.random.default_rng(5).permutation(45)
    for t in order:
        A.kv_write(many.pool, many.pages, k[:, t:t + 1], v[:, t:t + 1], ints([t]))
    assert torch.equal(one.pool, many.pool)


def test_special_groups():
    x = torch.zeros(1, 9, 1, 64)
    x[0, 0] = 0.375                                  # equal values are exact
    x[0, 1, 0, 3] = float("inf")                     # one group odd, its neighbour not
    x[0, 2, 0, 40] = float("nan")
    x[0, 3] = torch.linspace(-1e6, 1e6, 64)          # past the limit
    x[0, 4] = torch.randn(64, generator=torch.Generator().manual_seed(1)) * 1e-6  # float16's subnormal range
    x[0, 5, 0, 7] = -0.0
    x[0, 6] = 3e38
    x[0, 7, 0, :32] = torch.arange(32) % 16 * 0.25   # on the grid: exact
    x[0, 8, 0, 63] = float("-inf")
    pg = Paged([9], 1, 64, 32)
    k = x.cuda()
    A.kv_write(pg.pool, pg.pages, k, k, ints([0]))
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    A.kv_read(pg.pool, pg.pages, ints([0]), ko, vo)
    got = host(ko)[0, :, 0]
    assert np.array_equal(got, host(vo)[0, :, 0], equal_nan=True)
    n, s, b = OA.quantise(x[0, :, 0].numpy())
    assert np.array_equal(got, OA.values(n, s, b), equal_nan=True)
    assert (got[0] == 0.375).all() and (got[6] == 16384).all()
    assert np.isnan(got[1, :32]).all() and (got[1, 32:] == 0).all()
    assert (got[2, :32] == 0).all() and np.isnan(got[2, 32:]).all() and np.isnan(got[8, 32:]).all()
    assert (got[7, :32] == np.arange(32) % 16 * 0.25).all()


def test_positions_and_pages_out_of_range_touch_nothing():
    D, P, H = 64, 32, 2
    pg = Paged([64, 64, 64, 64], H, D, P)
    pg.pages[0, 1] = -1                 # freed
    pg.pages[1, 0] = pg.pool.shape[0]   # past the pool
    pg.pages[1, 1] = 1 << 30
    before = pg.pool.clone()
    k = rand(5, 4, 70, H, D)
    start, count = ints([30, 0, -5, 60]), ints([70, 70, 70, 1 << 30])
    A.kv_write(pg.pool, pg.pages, k, k, start, count)
    m = OA.Cache(before.cpu().numpy().copy(), P, D)
    for b, s in enumerate([30, 0, -5, 60]):
        for i in range(70):
            pos = s + i
            if 0 <= pos < 64 and 0 <= int(pg.pages[b, pos // P]) < pg.pool.shape[0]:
                for h in range(H):
                    m.write(int(pg.pages[b, pos // P]), h, pos % P, host(k)[b, i, h].astype(np.float32),
                            host(k)[b, i, h].astype(np.float32))
    assert (pg.pool.cpu().numpy() == m.pool).all()
    for s, c in (([30, 0, -5, 60], [0, -3, 0, 0]), ([1 << 30, -(1 << 30), 64, 200], [70, 70, 70, 70])):
        A.kv_write(pg.pool, pg.pages, k, k, ints(s), ints(c))
        assert (pg.pool.cpu().numpy() == m.pool).all()
    out = torch.full_like(k, 5.0)
    A.kv_read(pg.pool, pg.pages, start, out, out.clone(), count)
    o = host(out)
    assert (o[0, 2:] == 5).all() and (o[1] == 5).all() and (o[2, :5] == 5).all() and (o[2, 69:] == 5).all()
    assert (o[3, 4:] == 5).all() and (o[0, :2] != 5).all() and (o[2, 5:69] != 5).all()


# --------------------------------------------------------------- attention
def bound(dtype, cached, D, N, out, mass, size):
    weight = 2 * (D + 8) * U * size[:, None] + 3 * N * U
    if cached:
        weight = weight + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -21) + 2 * D * 2.0 ** -25 * size[:, None]
    elif dtype == "bf16":
        weight = weight + 2.0 ** -8
    last = 2.0 ** -8 if dtype == "bf16" else 2 * U
    return mass * weight * 1.01 + np.abs(out) * last * 1.01 + 1e-30


def check(got, q, k, v, q_len, kv_len, scale, causal, window, sinks, dtype, cached, left=None):
    """Every row of `got` against the oracle; rows past q_len hold `left`."""
    B, T, H, D = q.shape
    group = H // k.shape[2]
    got, q, k, v = (host(t) if torch.is_tensor(t) else t for t in (got, q, k, v))
    for b in range(B):
        t, n = min(q_len[b], T), kv_len[b]
        for h in range(H):
            out, mass, size = OA.attention(q[b, :t, h], k[b, :n, h // group], v[b, :n, h // group], scale, causal,
                                           window, sinks)
            tol = bound(dtype, cached, D, n, out, mass, size)
            err = np.abs(got[b, :t, h] - out)
            assert (err <= tol).all(), (b, h, np.argwhere(~(err <= tol))[:4], err.max(), (err / tol).max())
            if left is not None:
                assert (got[b, t:, h] == left).all()


DENSE = [  # T, N, q_len, kv_len, heads, kv_heads, causal, window, sinks
    (1, 1, None, None, 1, 1, True, 0, 0),
    (1, 300, None, [300, 1, 0], 4, 2, True, 0, 0),
    (5, 64, [5, 0, 3], [64, 33, 63], 8, 1, True, 20, 3),
    (130, 130, None, None, 2, 2, True, 0, 0),
    (130, 197, [130, 17, 64], [197, 31, 65], 4, 2, True, 33, 4),
    (33, 333, None, [333, 20, 7], 2, 1, True, 64, 1),       # more queries than tokens: rows that see nothing
    (64, 128, None, None, 2, 2, False, 0, 0),
    (97, 161, [97, 50, 1], [161, 3, 128], 3, 3, False, 0, 0),
    (97, 161, None, [161, 40, 100], 3, 1, False, 16, 5),
    (40, 20, None, None, 2, 2, False, 6, 0),                # positions before the first token, both directions
    (2, 1500, None, [1500, 700, 65], 4, 4, True, 1, 0),     # a window of itself alone
    (3, 2000, None, None, 2, 1, True, 0, 0),                # few rows, tokens split over workgroups
    (200, 200, None, None, 1, 1, True, 1 << 30, 1 << 30),   # a window wider than everything
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("T, N, q_len, kv_len, H, Hk, causal, window, sinks", DENSE)
def test_attention(dtype, D, T, N, q_len, kv_len, H, Hk, causal, window, sinks):
    B = 3
    q, k, v = rand(1, B, T, H, D, dtype=dtype), rand(2, B, N, Hk, D, dtype=dtype), rand(3, B, N, Hk, D, dtype=dtype)
    ql, kl = q_len or [T] * B, kv_len or [N] * B
    for b in range(B):  # what lies past a sequence's end must not matter
        k[b, kl[b]:], v[b, kl[b]:] = float("nan"), float("inf")
    out = torch.full_like(q, 4.0)
    r = A.attention(q, k, v, q_len=q_len and ints(q_len), kv_len=kv_len and ints(kv_len), causal=causal, window=window,
                    sinks=sinks, out=out)
    assert r is out
    check(out, q, k, v, ql, kl, D ** -0.5, causal, window, sinks, dtype, False, left=4.0)


MANY = [  # batch, T, N, heads, kv_heads, window, sinks, ragged: hundreds of row tiles, taken in an order of their own
    (1, 700, 700, 48, 48, 0, 0, False),     # up to 64 of them to an XCD
    (4, 600, 650, 16, 16, 0, 0, True),
    (16, 260, 300, 16, 16, 50, 3, True),    # more
    (3, 520, 1030, 32, 8, 0, 0, True),      # shared keys, queries behind them
    (1, 2900, 2900, 12, 12, 100, 2, False),  # heads that do not come out even over the XCDs, up to 512 tiles
    (3, 700, 800, 100, 20, 0, 0, True),     # and more
    (64, 20, 40, 16, 16, 0, 0, True),       # more heads to an XCD than lanes
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B, T, N, H, Hk, window, sinks, ragged", MANY)
def test_attention_of_many_rows(dtype, B, T, N, H, Hk, window, sinks, ragged):
    D = 32
    q, k, v = rand(1, B, T, H, D, dtype=dtype), rand(2, B, N, Hk, D, dtype=dtype), rand(3, B, N, Hk, D, dtype=dtype)
    ql, kl = [T] * B, [N] * B
    if ragged:
        ql = [T * (b * 7 % 5) // 4 for b in range(B)]
        kl = [N - N * (b * 3 % 4) // 4 for b in range(B)]
    out = torch.full_like(q, 4.0)
    A.attention(q, k, v, q_len=ints(ql) if ragged else None, kv_len=ints(kl) if ragged else None, window=window,
                sinks=sinks, out=out)
    check(out, q, k, v, ql, kl, D ** -0.5, True, window, sinks, dtype, False, left=4.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B, T, N, H, Hk, window", [(4, 600, 650, 16, 16, 0), (7, 500, 500, 12, 12, 40), (5, 300, 900, 32, 8, 0)])
def test_attention_of_many_rows_in_both_directions(dtype, B, T, N, H, Hk, window):
    D = 32
    q, k, v = rand(1, B, T, H, D, dtype=dtype), rand(2, B, N, Hk, D, dtype=dtype), rand(3, B, N, Hk, D, dtype=dtype)
    ql = [T * (b * 7 % 5) // 4 for b in range(B)]
    kl = [N - N * (b * 3 % 4) // 4 for b in range(B)]
    kl[-1] = 0
    out = torch.full_like(q, 4.0)
    A.attention(q, k, v, q_len=ints(ql), kv_len=ints(kl), causal=False, window=window, sinks=2, out=out)
    check(out, q, k, v, ql, kl, D ** -0.5, False, window, 2, dtype, False, left=4.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("how", ["heads_first", "padded", "odd"])
@pytest.mark.parametrize("D", [32, 128])
def test_attention_strides(dtype, how, D):
    q, k, v = (rand(i, 2, n, h, D, dtype=dtype) for i, (n, h) in enumerate(((70, 4), (99, 2), (99, 2))))
    out = laid_out(torch.zeros_like(q), how)
    A.attention(laid_out(q, how), laid_out(k, how), laid_out(v, how), window=50, sinks=2, scale=0.3, out=out)
    check(out, q, k, v, [70] * 2, [99] * 2, 0.3, True, 50, 2, dtype, False)
    # one set of keys for every sequence: stride 0
    kb, vb = k[:1].expand(2, -1, -1, -1), v[:1].expand(2, -1, -1, -1)
    check(A.attention(q, kb, vb), q, kb, vb, [70] * 2, [99] * 2, D ** -0.5, True, 0, 0, dtype, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("causal, window, sinks", [(True, 0, 0), (True, 9, 2), (False, 9, 2)])
def test_what_a_row_does_not_see_may_be_anything(dtype, value, causal, window, sinks):
    D, T = 64, 150
    q, k, v = (rand(i, 1, T, 2, D, dtype=dtype) for i in range(3))
    for at in (5, 40, 149):
        k2, v2 = k.clone(), v.clone()
        k2[0, at, 0], v2[0, at, 1, 7] = value, value
        got = host(A.attention(q, k2, v2, causal=causal, window=window, sinks=sinks))
        clean = host(A.attention(q, k, v, causal=causal, window=window, sinks=sinks))
        for i in range(T):
            if OA.sees(i, at, T, causal, window, sinks):
                assert not np.isfinite(got[0, i, 1, 7])
                assert np.isfinite(np.delete(got[0, i, 1], 7)).all()
            else:
                assert np.array_equal(got[0, i], clean[0, i]), (at, i)


PAIRED = [  # T, N, heads, kv_heads, causal, window, sinks: tiles that all rows see whole beside tiles that they do not
    (1, 100, 2, 2, True, 0, 0),       # the last tile is cut off by the length
    (1, 192, 2, 2, True, 100, 0),     # the first by the window
    (1, 300, 4, 1, True, 170, 70),    # the sinks' second tile too
    (64, 384, 4, 1, True, 0, 0),      # the diagonal, behind cached keys
    (70, 333, 4, 1, True, 77, 5),
    (5, 250, 2, 1, False, 101, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("T, N, H, Hk, causal, window, sinks", PAIRED)
def test_what_a_row_sees_is_never_dropped(dtype, value, T, N, H, Hk, causal, window, sinks):
    D = 64
    q, k, v = rand(0, 1, T, H, D, dtype=dtype), rand(1, 1, N, Hk, D, dtype=dtype), rand(2, 1, N, Hk, D, dtype=dtype)
    clean = host(A.attention(q, k, v, causal=causal, window=window, sinks=sinks))
    for at in sorted({*range(5, N, 32), N - 1}):
        v2 = v.clone()
        v2[0, at, 0, 7] = value
        got = host(A.attention(q, k, v2, causal=causal, window=window, sinks=sinks))
        for i in range(T):
            for h in range(H // Hk):
                if OA.sees(N - T + i, at, N, causal, window, sinks):
                    assert not np.isfinite(got[0, i, h, 7]), (at, i, h)
                    assert np.isfinite(np.delete(got[0, i, h], 7)).all()
                else:
                    assert np.array_equal(got[0, i, h], clean[0, i, h]), (at, i, h)


def test_large_and_small_scores():
    for dtype in ("bf16", "f32"):
        q, k, v = (rand(i, 1, 90, 2, 64, dtype=dtype) for i in range(3))
        for scale in (1e-6, 1.0, 30.0):
            check(A.attention(q, k, v, scale=scale), q, k, v, [90], [90], scale, True, 0, 0, dtype, False)
        big = (q.float() * 1e18).to(q.dtype), (k.float() * 1e-18).to(k.dtype), (v.float() * 1e30).to(v.dtype)
        check(A.attention(*big), *big, [90], [90], 0.125, True, 0, 0, dtype, False)


SCORES = [1e6, 1e10, 1e20, 1e36]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SCORES + [-x for x in SCORES])
def test_scores_of_any_size(dtype, size):
    """Scores of `size` times 1 .. 100 / 64, far further apart than their
    rounding: a row is the value of its highest alone (1e36: scores up to
    1.6e36, sums within fp32)."""
    D, N = 64, 100
    q, k, v = torch.zeros(1, N, 1, D), torch.zeros(1, N, 1, D), rand(1, 1, N, 1, D, dtype=dtype)
    q[..., 3] = np.sign(size) * 2.0 ** 60 if abs(size) > 1e19 else np.sign(size)
    k[0, :, 0, 3] = (1 + torch.arange(N)) / 64 * (abs(size) / q[..., 3].abs().max())
    q, k = q.to(DT[dtype]).cuda(), k.to(DT[dtype]).cuda()
    for T in (1, 5, N):
        got = A.attention(q[:, N - T:], k, v, scale=1.0)
        want = v[:, N - T:] if size > 0 else v[:, :1].expand(1, T, 1, D)
        # weights cancel but for a few fp32 roundings
        assert ((got.float() - want.float()).abs() <= want.float().abs() * 2.0 ** -20).all(), T


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SCORES + [-x for x in SCORES])
@pytest.mark.parametrize("N", [100, 3000])
def test_scores_of_any_size_over_the_cache(dtype, size, N):
    D = 64
    pg = Paged([N], 1, D, 64)
    k, v = torch.zeros(1, N, 1, D, device="cuda"), rand(1, 1, N, 1, D, dtype=dtype)
    k[0, :, 0, 3] = (1 + torch.arange(N, device="cuda") % 200) / 64
    A.kv_write(pg.pool, pg.pages, k.to(DT[dtype]), v, ints([0]))
    kk, vv = torch.zeros(1, N, 1, D, device="cuda"), torch.zeros(1, N, 1, D, device="cuda")
    A.kv_read(pg.pool, pg.pages, ints([0]), kk, vv)
    kk = host(kk)[0, :, 0, 3]
    for T in (1, 5):
        q = torch.zeros(1, T, 1, D, device="cuda")
        q[..., 3] = size
        got = host(A.kv_attention(pg.pool, pg.pages, q.to(DT[dtype]), ints([N]), scale=1.0))
        for i in range(T):
            x = kk[:N - T + 1 + i] * np.sign(size)
            best = x == x.max()
            # all products are exact but for q's rounding, the same for all: ties have one weight
            want = host(vv)[0, :N - T + 1 + i, 0][best].mean(0)
            tol = np.abs(host(vv)[0, :N - T + 1 + i, 0][best]).mean(0) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -19)
            assert (np.abs(got[0, i, 0] - want) <= tol + 1e-30).all(), (T, i)


def test_scores_down_to_the_lowest_are_seen():
    """Rows whose scores are all the same, down to -2.3e38, are means of what
    they see; those of minus infinity alone are zeros."""
    D, N = 32, 40
    for dtype in ("bf16", "f32"):
        v = torch.ones(1, N, 1, D, dtype=DT[dtype], device="cuda")
        for score in (1e37, -1e37, -2.2e38, -2.3e38):
            q, k = torch.zeros(1, N, 1, D, device="cuda"), torch.zeros(1, N, 1, D, device="cuda")
            q[..., 0], k[..., 0] = 1e19, score / 1e19
            for T in (1, N):
                got = A.attention(q[:, :T].to(DT[dtype]), k.to(DT[dtype]), v, scale=1.0)
                assert ((got.float() - 1).abs() <= 2.0 ** -20).all(), (score, T)
        k[..., 0] = -float("inf")
        assert (A.attention(q.to(DT[dtype]), k.to(DT[dtype]), v, scale=1.0) == 0).all()


TOP = 3.4028234663852886e38


@pytest.mark.parametrize("value", [TOP, -TOP, 3.3962e38, -3.3962e38, 3.39e38, float("inf")])
@pytest.mark.parametrize("T, N, causal, window, sinks", [(150, 150, True, 9, 2), (150, 150, True, 0, 0), (3, 100, True, 0, 0),
                                                        (150, 150, False, 9, 2)])
def test_fp32_values_and_keys_to_the_end_of_the_range(value, T, N, causal, window, sinks):
    """Past bf16's largest.  A row that does not see them is as without them; a
    row that does has their weighted value, or overflows: 2^8 is the largest
    weight before the division."""
    D, at = 64, N - 40
    kw = dict(causal=causal, window=window, sinks=sinks)
    q, k, v = rand(0, 1, T, 2, D), rand(1, 1, N, 2, D), rand(2, 1, N, 2, D)
    clean = host(A.attention(q, k, v, **kw))
    v2 = v.clone()
    v2[0, at, 1, 7] = value
    got = host(A.attention(q, k, v2, **kw))
    for i in range(T):
        rest = np.array_equal(np.delete(got[0, i, 1], 7), np.delete(clean[0, i, 1], 7))
        assert rest and np.array_equal(got[0, i, 0], clean[0, i, 0])
        if not OA.sees(N - T + i, at, N, causal, window, sinks):
            assert got[0, i, 1, 7] == clean[0, i, 1, 7]
            continue
        p = host(k)[0, :, 1] @ host(q)[0, i, 1] * D ** -0.5
        see = [OA.sees(N - T + i, j, N, causal, window, sinks) for j in range(N)]
        p = np.exp(np.where(see, p, -np.inf) - p[see].max())
        want = p[at] / p.sum() * value
        x = got[0, i, 1, 7]
        assert np.isinf(want) and x == want or abs(x - want) <= 1e-4 * abs(want) or (np.isinf(x) and x * want > 0), (i, x, want)
    if np.isinf(value):
        return
    # as a key: |q| of a quarter there, so that no score overflows
    q[..., 5] = torch.where(q[..., 5] > 0, 0.25, -0.25)
    k2 = k.clone()
    k2[0, at, :, 5] = value
    got = host(A.attention(q, k2, v, **kw))
    for i in range(T):
        for h in range(2):
            see = np.array([OA.sees(N - T + i, j, N, causal, window, sinks) for j in range(N)])
            if see[at] and host(q)[0, i, h, 5] * value > 0:
                assert np.allclose(got[0, i, h], host(v)[0, at, h], rtol=2.0 ** -22)
            else:
                see[at] = False
                x = host(k)[0, see, h] @ host(q)[0, i, h] * D ** -0.5
                x = np.exp(x - x.max())
                assert np.allclose(got[0, i, h], x / x.sum() @ host(v)[0, see, h], atol=1e-4)


def test_fp32_queries_to_the_end_of_the_range():
    D, N = 64, 100
    q, k, v = torch.zeros(1, N, 1, D, device="cuda"), torch.zeros(1, N, 1, D, device="cuda"), rand(1, 1, N, 1, D)
    k[0, :, 0, 5] = (1 + torch.arange(N, device="cuda")) / 128
    for value in (TOP, -TOP, 3.3962e38):
        q[..., 5] = value
        got = A.attention(q, k, v)
        want = v if value > 0 else v[:, :1].expand(1, N, 1, D)
        assert ((got - want).abs() <= want.abs() * 2.0 ** -20).all()


CACHED = [  # T, heads, kv_heads, kv_len, q_len, window, sinks, page
    (1, 2, 2, [1, 0, 31], None, 0, 0, 32),
    (1, 8, 2, [33, 300, 64], None, 0, 0, 64),
    (1, 16, 1, [500, 32, 77], None, 40, 4, 32),
    (1, 20, 1, [500, 2, 77], None, 0, 0, 128),
    (5, 4, 2, [100, 5, 3], [5, 2, 5], 0, 0, 32),        # a sequence with more queries than tokens
    (4, 8, 1, [400, 90, 33], [4, 0, 1], 17, 3, 32),
    (9, 8, 1, [700, 257, 9], None, 100, 70, 256),       # three tiles of rows
    (3, 4, 4, [260, 129, 1], None, 1, 0, 64),
    (2, 4, 2, [1000, 999, 513], None, 64, 1000, 1024),  # sinks past the window
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("T, H, Hk, kv_len, q_len, window, sinks, P", CACHED)
def test_kv_attention(dtype, D, T, H, Hk, kv_len, q_len, window, sinks, P):
    B = 3
    pg = Paged(kv_len, Hk, D, P, fill=0xFF)  # NaN pairs wherever nothing is written
    N = max(kv_len)
    k, v = rand(2, B, N, Hk, D, dtype=dtype), rand(3, B, N, Hk, D, dtype=dtype)
    A.kv_write(pg.pool, pg.pages, k, v, ints([0] * B), ints(kv_len))
    ko, vo = torch.zeros(B, N, Hk, D, device="cuda"), torch.zeros(B, N, Hk, D, device="cuda")
    A.kv_read(pg.pool, pg.pages, ints([0] * B), ko, vo, ints(kv_len))
    q = rand(4, B, T, H, D, dtype=dtype)
    out = torch.full_like(q, 4.0)
    kw = dict(q_len=q_len and ints(q_len), window=window, sinks=sinks)
    A.kv_attention(pg.pool, pg.pages, q, ints(kv_len), out=out, kv_max=N, **kw)
    check(out, q, ko, vo, q_len or [T] * B, kv_len, D ** -0.5, True, window, sinks, dtype, True, left=4.0)
    if T == 1 or q_len:
        # a bound that proves too low or too high changes the split, not the values' meaning
        for most in (1, 1 << 20):
            r = A.kv_attention(pg.pool, pg.pages, q, ints(kv_len), kv_max=most, **kw)
            check(r, q, ko, vo, q_len or [T] * B, kv_len, D ** -0.5, True, window, sinks, dtype, True, left=0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_kv_attention_split_over_workgroups(dtype):
    B, H, Hk, D, P, lens = 2, 8, 2, 128, 64, [5000, 1400]
    pg = Paged(lens, Hk, D, P)
    k, v = rand(2, B, 5000, Hk, D, dtype=dtype), rand(3, B, 5000, Hk, D, dtype=dtype)
    A.kv_write(pg.pool, pg.pages, k, v, ints([0, 0]), ints(lens))
    ko, vo = torch.zeros(B, 5000, Hk, D, device="cuda"), torch.zeros(B, 5000, Hk, D, device="cuda")
    A.kv_read(pg.pool, pg.pages, ints([0, 0]), ko, vo, ints(lens))
    for T in (1, 3, 5):
        q = rand(4, B, T, H, D, dtype=dtype)
        assert A.kv_attention_workspace(pg.pool, pg.pages, q, 5000) > 0
        first = A.kv_attention(pg.pool, pg.pages, q, ints(lens), kv_max=5000)
        check(first, q, ko, vo, [T] * 2, lens, D ** -0.5, True, 0, 0, dtype, True)
        assert torch.equal(first, A.kv_attention(pg.pool, pg.pages, q, ints(lens), kv_max=5000))  # same bits again
        r = A.kv_attention(pg.pool, pg.pages, q, ints(lens), kv_max=1500, window=1200, sinks=64)
        check(r, q, ko, vo, [T] * 2, lens, D ** -0.5, True, 1200, 64, dtype, True)


def test_kv_attention_queries_of_all_sizes_and_strides():
    D, lens = 64, [90, 41]
    pg = Paged(lens, 2, D, 32)
    k, v = rand(2, 2, 90, 2, D), rand(3, 2, 90, 2, D)
    A.kv_write(pg.pool, pg.pages, k, v, ints([0, 0]), ints(lens))
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    A.kv_read(pg.pool, pg.pages, ints([0, 0]), ko, vo, ints(lens))
    for dtype in ("bf16", "f32"):
        q = rand(5, 2, 3, 4, D, dtype=dtype)
        for size in (1e-30, 1e-3, 1.0, 1e4, 1e30):
            x = (q.float() * size).to(q.dtype)
            scale = 0.2 / size
            if not 1e-38 < scale < 1e38:
                continue
            check(A.kv_attention(pg.pool, pg.pages, x, ints(lens), scale=scale), x, ko, vo, [3] * 2, lens, scale, True, 0,
                  0, dtype, True)
        for how in ("heads_first", "padded", "odd"):
            out = laid_out(torch.zeros_like(q), how)
            A.kv_attention(pg.pool, pg.pages, laid_out(q, how), ints(lens), out=out)
            check(out, q, ko, vo, [3] * 2, lens, D ** -0.5, True, 0, 0, dtype, True)
        assert (A.kv_attention(pg.pool, pg.pages, torch.zeros_like(q), ints(lens)).isfinite()).all()
        q[0, 1, 2, 5] = float("nan")  # one row's own business
        r = A.kv_attention(pg.pool, pg.pages, q, ints(lens))
        assert r[0, 1, 2].isnan().all() and r.isnan().sum() == D


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_that_leave_the_range_of_fp32_with_a_rows_size(dtype):
    D, lens = 64, [90]
    pg = Paged(lens, 2, D, 32)
    k, v = rand(2, 1, 90, 2, D) * 1e-3, rand(3, 1, 90, 2, D)
    A.kv_write(pg.pool, pg.pages, k, v, ints([0]))
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    A.kv_read(pg.pool, pg.pages, ints([0]), ko, vo)
    q = rand(5, 1, 3, 4, D, dtype=dtype)
    tiny = (q.float() * 2.0 ** -125).to(q.dtype)
    for scale in (1e-10, 1e-30):  # scores of 0: means
        check(A.kv_attention(pg.pool, pg.pages, tiny, ints(lens), scale=scale), tiny, ko, vo, [3], lens, scale, True, 0, 0,
              dtype, True)
    huge = torch.zeros_like(q)
    huge[..., 5] = 1e36  # the largest key of channel 5 alone
    got = host(A.kv_attention(pg.pool, pg.pages, huge, ints(lens), scale=1000.0))
    for i in range(3):
        for h in range(4):
            x = host(ko)[0, :88 + i, h // 2, 5]
            want = host(vo)[0, :88 + i, h // 2][x == x.max()].mean(0)
            assert (np.abs(got[0, i, h] - want) <= np.abs(want) * 2.0 ** -8 + 2.0 ** -10).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window, sinks", [(0, 0), (6, 2)])
def test_kv_attention_unseen_tokens_may_be_odd_and_pages_gone(dtype, window, sinks):
    D, T, n = 64, 6, 100
    pg = Paged([n], 1, D, 32)
    k, v = rand(2, 1, n, 1, D, dtype=dtype), rand(3, 1, n, 1, D, dtype=dtype)
    q = rand(4, 1, T, 3, D, dtype=dtype)
    A.kv_write(pg.pool, pg.pages, k, v, ints([0]))
    clean = host(A.kv_attention(pg.pool, pg.pages, q, ints([n]), window=window, sinks=sinks))
    for at in (1, 93, 97, 99):
        k2, v2 = k.clone(), v.clone()
        k2[0, at], v2[0, at, 0, 40] = float("nan"), float("inf")
        A.kv_write(pg.pool, pg.pages, k2, v2, ints([0]))
        got = host(A.kv_attention(pg.pool, pg.pages, q, ints([n]), window=window, sinks=sinks))
        for i in range(T):
            if OA.sees(n - T + i, at, n, True, window, sinks):
                assert np.isnan(got[0, i]).any()
            else:
                assert np.array_equal(got[0, i], clean[0, i])
    A.kv_write(pg.pool, pg.pages, k, v, ints([0]))
    if window:  # pages 1 is behind the window and holds no sink
        pg.pages[0, 1] = -1
        assert np.array_equal(host(A.kv_attention(pg.pool, pg.pages, q, ints([n]), window=window, sinks=sinks)), clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("fill", [0x70, 0x7B, 0xFB, 0xFF])
def test_kv_attention_over_a_pool_that_was_never_cleared(dtype, D, fill):
    """Pairs of any bytes: 0x70 and 0x7B are finite, their values past float16."""
    H, P, lens = 2, 64, [101, 1, 37]
    k, v = rand(2, 3, 101, H, D, dtype=dtype), rand(3, 3, 101, H, D, dtype=dtype)
    pools = [Paged(lens, H, D, P, fill=f) for f in (0, fill)]
    for T, window, sinks in ((1, 0, 0), (5, 0, 0), (5, 20, 0), (20, 9, 2)):
        q = rand(4, 3, T, 4, D, dtype=dtype)
        got = []
        for pg in pools:
            A.kv_write(pg.pool, pg.pages, k, v, ints([0] * 3), ints(lens))
            got.append(A.kv_attention(pg.pool, pg.pages, q, ints(lens), window=window, sinks=sinks))
        assert got[0].isfinite().all() and torch.equal(*got)
    # tokens that the window hides were never written, their page is in the table or is not, and page 0 is like that
    for dark in (False, True):
        got = []
        for f in (0, fill):
            pg = Paged([160], H, D, 32, fill=f, spare=1)
            pg.pages.copy_(torch.tensor([[1, 2, 3, 4, 5]], dtype=torch.int32))
            A.kv_write(pg.pool, pg.pages, k[:1, :53], v[:1, :53], ints([107]))
            if dark:
                pg.pages[0, :3] = -1
            q = rand(4, 1, 9, 4, D, dtype=dtype)
            got.append(A.kv_attention(pg.pool, pg.pages, q, ints([160]), window=40))
        assert got[0].isfinite().all() and torch.equal(*got)


def test_pool_and_strides_past_32_bits():
    D, P, H = 128, 64, 8
    n = (5 << 30) // (H * A.pool_block(P, D))
    pool = torch.empty(n, H, A.pool_block(P, D), dtype=torch.uint8, device="cuda")
    pages = torch.tensor([[n - 1, 0], [n // 2 + 1, n - 2]], dtype=torch.int32, device="cuda")
    lens = [100, 77]
    big = torch.empty((5 << 30) // 2, dtype=torch.bfloat16, device="cuda")  # sequences 4 GiB apart
    x = big.as_strided((2, 100, H, D), ((4 << 30) // 2, H * D, D, 1))
    x.copy_(rand(1, 2, 100, H, D, dtype="bf16"))
    A.kv_write(pool, pages, x, x, ints([0, 0]), ints(lens))
    ko, vo = torch.zeros(2, 100, H, D, device="cuda"), torch.zeros(2, 100, H, D, device="cuda")
    A.kv_read(pool, pages, ints([0, 0]), ko, vo, ints(lens))
    for b in range(2):
        w = OA.values(*OA.quantise(host(x)[b, :lens[b]].astype(np.float32)))
        assert (host(ko)[b, :lens[b]] == w).all() and (host(vo)[b, :lens[b]] == w).all()
    q = x[:, 99:100]
    check(A.kv_attention(pool, pages, q, ints(lens)), q, ko, vo, [1, 1], lens, D ** -0.5, True, 0, 0, "bf16", True)
    check(A.attention(q, x, x), q, x, x, [1, 1], [100, 100], D ** -0.5, True, 0, 0, "bf16", False)


# ----------------------------------------------- streams, graphs, the cache
def test_calls_on_another_stream():
    q, k, v = (rand(i, 1, 3, 2, 64) for i in range(3))
    kk, vv = rand(7, 1, 3000, 2, 64), rand(8, 1, 3000, 2, 64)
    want = A.attention(q, kk, vv)
    pg = Paged([3000], 2, 64, 64)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        A.kv_write(pg.pool, pg.pages, kk, vv, ints([0]), stream=stream)
        a = A.attention(q, kk, vv, out=torch.zeros_like(q), stream=stream)
        b = A.kv_attention(pg.pool, pg.pages, q, ints([3000]), out=torch.zeros_like(q), kv_max=3000, stream=stream)
        s.synchronize()
        assert torch.equal(a, want)
        assert torch.equal(b, A.kv_attention(pg.pool, pg.pages, q, ints([3000]), kv_max=3000))


def test_tensors_dropped_behind_a_call_on_another_stream_stay_until_it_has_run():
    q, k, v = rand(1, 1, 3, 2, 64), rand(2, 1, 3000, 2, 64), rand(3, 1, 3000, 2, 64)
    pg = Paged([3000], 2, 64, 64)
    want = A.attention(q, k, v)
    busy = torch.randn(8192, 8192, device="cuda").bfloat16()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        t = [x.clone() for x in (q, k, v)]
        at = ints([0])
        used = {x.data_ptr() for x in (*t, at)}
        out = torch.zeros_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(8):  # some milliseconds
                torch.mm(busy, busy)
        A.attention(*t, out=out, stream=stream)
        A.kv_write(pg.pool, pg.pages, t[1], t[2], at, stream=stream)
        del t, at
        fresh = [torch.full_like(y, float("nan")) for y in (q, k, v)] + [ints([1 << 20])]
        early = not s.query()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert not early or not used & {y.data_ptr() for y in fresh}
        ko, vo = torch.zeros_like(k), torch.zeros_like(v)
        A.kv_read(pg.pool, pg.pages, ints([0]), ko, vo)
        assert np.array_equal(host(ko)[0, :, 0], OA.values(*OA.quantise(host(k)[0, :, 0].astype(np.float32))))


def test_a_captured_decode_step_replays():
    D, H, P, B = 128, 4, 64, 2
    pg = Paged([2000] * B, H, D, P)
    lens = ints([1500, 900])
    A.kv_write(pg.pool, pg.pages, rand(1, B, 1500, H, D, dtype="bf16"), rand(2, B, 1500, H, D, dtype="bf16"), ints([0, 0]))
    q, k, v = (rand(i, B, 1, H, D, dtype="bf16") for i in range(3, 6))
    out = torch.zeros_like(q)
    work = torch.empty(A.kv_attention_workspace(pg.pool, pg.pages, q, 2000) or 1, dtype=torch.uint8, device="cuda")
    kw = dict(kv_max=2000, window=1300, sinks=4)

    def step():
        A.kv_write(pg.pool, pg.pages, k, v, lens)
        lens.add_(1)
        A.kv_attention(pg.pool, pg.pages, q, lens, out=out, workspace=work, **kw)
    copy, at = pg.pool.clone(), lens.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    pg.pool.copy_(copy)
    lens.copy_(at)
    for i in range(4):
        for t, seed in ((q, 10), (k, 20), (v, 30)):
            t.copy_(rand(seed + i, *t.shape, dtype="bf16"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        A.kv_write(copy, pg.pages, k, v, at)
        at.add_(1)
        assert torch.equal(copy, pg.pool) and torch.equal(at, lens)
        assert torch.equal(got, A.kv_attention(copy, pg.pages, q, at, **kw))


def test_cache_object_grows_trims_and_refuses():
    c = A.KvCache(2, 2, 64, 200, n_pages=9, page_tokens=32)
    k, v = rand(1, 2, 150, 2, 64), rand(2, 2, 150, 2, 64)
    c.append(k[:, :70], v[:, :70], [70, 33])
    c.append(k[:, 70:75], v[:, 70:75])
    assert c.lengths == [75, 38] and c.kv_len.tolist() == [75, 38] and len(c.free) == 4
    kk, vv = torch.zeros(2, 75, 2, 64, device="cuda"), torch.zeros(2, 75, 2, 64, device="cuda")
    c.read(kk, vv)
    q = rand(3, 2, 1, 4, 64)
    check(c.attend(q), q, kk, vv, [1, 1], [75, 38], 0.125, True, 0, 0, "f32", True)
    before = c.attend(q, window=10, sinks=0)
    c.trim(10)
    assert len(c.free) == 6 and torch.equal(c.attend(q, window=10, sinks=0), before)
    with pytest.raises(F.FluidError, match="do not fit"):
        c.append(k, v)
    with pytest.raises(F.FluidError, match="free pages"):
        c.append(k[:, :140], v[:, :140], [125, 140])
    c.clear(0)
    assert c.lengths == [0, 38] and len(c.free) == 7
    assert (c.attend(q)[0] == 0).all()


def test_a_refused_append_leaves_the_cache_as_it_was():
    c = A.KvCache(2, 2, 64, 128, page_tokens=32)
    k = rand(1, 2, 40, 2, 64)
    c.append(k[:, :5], k[:, :5])
    was = [list(r) for r in c.table], list(c.free), list(c.lengths), c.pages.clone(), c.pool.clone()
    for bad in (lambda: c.append(k.half(), k.half()), lambda: c.append(k, k[:, :39]), lambda: c.append(k[:1], k[:1]),
                lambda: c.append(k[:, :, :1], k[:, :, :1]), lambda: c.append(k, k, [40]), lambda: c.append(k, k, [1, 1, 1]),
                lambda: c.append(k, k, [-1, 1]), lambda: c.append(k[0], k[0])):
        with pytest.raises(F.FluidError):
            bad()
        assert (c.table, c.free, c.lengths) == was[:3] and torch.equal(c.pages, was[3]) and torch.equal(c.pool, was[4])
        assert c.kv_len.tolist() == c.lengths
    c.append(k, k)
    assert c.lengths == [45, 45]


def test_a_decoding_loop_describes_its_calls_once():
    c = A.KvCache(2, 2, 64, 2100, page_tokens=32)
    k, q = rand(1, 2, 2030, 2, 64, dtype="bf16"), rand(2, 2, 1, 4, 64, dtype="bf16")
    c.append(k, k)
    sizes, needs = [], set()
    for i in range(40):
        c.append(k[:, :1], k[:, :1])
        got = c.attend(q)
        sizes.append(len(A._calls))
        needs.add(A.kv_attention_workspace(c.pool, c.pages, q, max(c.lengths)))
        assert torch.equal(got, A.kv_attention(c.pool, c.pages, q, c.kv_len, kv_max=max(c.lengths)))
    assert len(needs) > 1  # the loop passes a length from which the tokens are split
    assert sizes[0] == sizes[-1]
    with pytest.raises(F.FluidError, match="kv_max"):
        A.kv_attention(c.pool, c.pages, q, c.kv_len, kv_max=0)


def test_trim_without_a_window_gives_nothing_back():
    c = A.KvCache(1, 2, 64, 128, page_tokens=32)
    k = rand(1, 1, 100, 2, 64)
    c.append(k, k)
    q = rand(2, 1, 1, 2, 64)
    before = c.attend(q)
    c.trim(0)
    assert torch.equal(c.attend(q), before) and not c.free
    with pytest.raises(F.FluidError, match="negative"):
        c.trim(-1)


def test_checks_hold_behind_a_call_of_the_same_shapes():
    block = A.pool_block(32, 64)
    pages, at, one = ints([0]).view(1, 1), ints([0]), ints([1])
    k = rand(1, 1, 1, 2, 64, dtype="bf16")
    pool = torch.zeros(2, 2, block, dtype=torch.uint8, device="cuda")
    calls = (lambda p: A.kv_write(p, pages, k, k, at), lambda p: A.kv_read(p, pages, at, k.clone(), k.clone()),
             lambda p: A.kv_attention(p, pages, k, one))
    apart = pool.transpose(0, 1)[:1]
    assert apart.shape == pool[:1].shape and not apart.is_contiguous()
    for call in calls:
        call(pool[:1])
        with pytest.raises(F.FluidError, match="contiguous"):
            call(apart)
