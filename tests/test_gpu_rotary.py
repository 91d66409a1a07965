"""Rotary positions on the GPU against plain NumPy (oracle/decoder_layers.py).

Tolerance.  With u = 2^-24: an angle within an eighth of a turn is off by at
most 2 u (its two conversions and their sum), sine and cosine by that and 3 u of
their series, the amplitude's product by one more; the two products and their
sum by 2 u: 8 u A (|x| + |y|) for a pair (x, y).  A bf16 output is rounded by
2^-8 of itself."""
import numpy as np
import pytest

from oracle import decoder_layers as O

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


def rand(seed, *shape, dtype="f32"):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(DT[dtype]).cuda()


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


def check(got, x, positions, counts, rot, inverse=False, dtype="f32", before=0.0):
    theta, inter, amp = rot
    got, x = host(got), host(x)
    d = 2 * len(theta)
    for b, n in enumerate(counts):
        want = O.rotate(x[b, :n], positions[b][:n], theta, inter, amp, inverse)
        size = np.abs(x[b, :n])
        head = size[..., :d]
        pair = head.reshape(*head.shape[:-1], *((d // 2, 2) if inter else (2, d // 2))).sum(-1 if inter else -2, keepdims=True)
        tol = np.zeros_like(size)
        tol[..., :d] = (8 * U * abs(amp) * np.broadcast_to(
            pair, (*head.shape[:-1], *((d // 2, 2) if inter else (2, d // 2))))).reshape(head.shape)
        if dtype == "bf16":
            tol += 2.0 ** -8 * np.abs(want) * (tol > 0)
        assert (np.abs(got[b, :n] - want) <= tol).all(), np.abs(got[b, :n] - want).max()
        assert (got[b, n:] == before).all()


def laid_out(t, how):
    """The same values in other strides."""
    B, T, H, D = t.shape
    if how == "heads_first":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    pad = {"padded": 16, "odd": 3}[how]
    buf = torch.full((B, T, H, D + pad), 7.0, dtype=t.dtype, device=t.device)
    off = 1 if how == "odd" else 0
    buf[..., off:off + D] = t
    return buf[..., off:off + D]


SCALED = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0, base=500000.0),
          dict(scaling="ramp", factor=8.0, length=4096, low=1.0, high=4.0, amplitude=1.2)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D, d", [(128, 128), (64, 64), (64, 16), (80, 40), (96, 12), (30, 30), (50, 2), (7, 6), (256, 64)])
def test_pairs_turn_by_position_and_the_rest_stays(dtype, inter, D, d):
    for i, how in enumerate((None, "heads_first", "padded", "odd")):
        opt = SCALED[i] if d >= 4 or SCALED[i].get("scaling") != "base" else {}
        rot = A.Rotary(d, interleaved=inter, **opt)
        amp = opt.get("amplitude", 1.0)
        theta = O.frequencies(d, **{k: v for k, v in opt.items() if k != "amplitude"})
        start, count = [5, 0, 100003], [4, 0, 3]
        q, k = rand(1, 3, 4, 6, D, dtype=dtype), rand(2, 3, 4, 2, D, dtype=dtype)
        qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
        if how:
            q, k, qo, ko = (laid_out(t, how) for t in (q, k, qo, ko))
        A.rotary(rot, q, k, start=ints(start), count=ints(count), q_out=qo, k_out=ko)
        pos = [[s + i for i in range(4)] for s in start]
        check(qo, q, pos, count, (theta, inter, amp), dtype=dtype, before=9.0)
        check(ko, k, pos, count, (theta, inter, amp), dtype=dtype, before=9.0)
        if how in ("padded", "odd"):  # nothing beside the rows
            base = qo._base
            assert (base[..., D + (1 if how == "odd" else 0):] == 7.0).all()


@pytest.mark.parametrize("dtype, D, H, Hk, T", [("bf16", 128, 32, 8, 700), ("f32", 64, 12, 12, 513), ("bf16", 96, 7, 1, 1300)])
def test_long_prompts_whose_threads_take_several_heads(dtype, D, H, Hk, T):
    rot = A.Rotary(D, base=500000.0)
    q, k = rand(1, 4, T, H, D, dtype=dtype), rand(2, 4, T, Hk, D, dtype=dtype)
    qo, ko = A.rotary(rot, q, k)
    pos = [range(T)] * 4
    check(qo, q, pos, [T] * 4, (O.frequencies(D, 500000.0), False, 1.0), dtype=dtype)
    check(ko, k, pos, [T] * 4, (O.frequencies(D, 500000.0), False, 1.0), dtype=dtype)


@pytest.mark.parametrize("inter", [False, True])
def test_far_and_negative_positions_given_one_by_one(inter):
    rot = A.Rotary(64, interleaved=inter)
    pos = [[0, -1, 2 ** 31 - 1, -2 ** 31], [12345678, 1 << 30, 1, 99]]
    q = rand(3, 2, 4, 5, 64)
    wide = torch.zeros(2, 9, dtype=torch.int32, device="cuda")
    wide[:, :4] = ints(pos)
    out = A.rotary(rot, q, positions=wide[:, :4])
    check(out, q, pos, [4, 4], (O.frequencies(64), inter, 1.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_back(dtype):
    for inter, D, d in ((False, 128, 128), (True, 64, 16), (False, 30, 10)):
        rot = A.Rotary(d, interleaved=inter)
        q, k = rand(5, 2, 9, 4, D, dtype=dtype), rand(6, 2, 9, 2, D, dtype=dtype)
        a, b = A.rotary(rot, q, k, start=ints([7, 3000]))
        q1, k1 = q.clone(), k.clone()
        got = A.rotary(rot, q1, k1, start=ints([7, 3000]), q_out=q1, k_out=k1)
        assert got[0] is q1 and torch.equal(q1, a) and torch.equal(k1, b)
        A.rotary(rot, q1, start=ints([7, 3000]), inverse=True, q_out=q1)
        pos = [[s + i for i in range(9)] for s in (7, 3000)]
        check(q1, a, pos, [9, 9], (O.frequencies(d), inter, 1.0), inverse=True, dtype=dtype)
        # q in place beside a k that is not: its tail is copied, q's stays
        q2, k2 = q.clone(), torch.zeros_like(k)
        A.rotary(rot, q2, k, start=ints([7, 3000]), q_out=q2, k_out=k2)
        assert torch.equal(q2, a) and torch.equal(k2, b)


def test_the_inverse_is_the_gradient():
    """<rotate(x), y> = <x, inverse(y)>, as of any linear map and its gradient;
    and the map's differences are those of the formula."""
    rot = A.Rotary(32, interleaved=True, amplitude=1.3)
    x, y, dx = rand(1, 1, 5, 2, 48), rand(2, 1, 5, 2, 48), rand(3, 1, 5, 2, 48)
    s = ints([17])
    f = lambda t, **kw: host(A.rotary(rot, t, start=s, **kw))  # noqa: E731
    left, right = (f(x) * host(y)).sum(), (host(x) * f(y, inverse=True)).sum()
    size = 2.6 * (np.abs(host(x)) * np.abs(host(y))).sum() + 2.6 * np.abs(host(x)).sum() * np.abs(host(y)).max()
    assert abs(left - right) <= 16 * U * size
    step = f(x + dx) - f(x)
    want = O.rotate(host(dx)[0], [17 + i for i in range(5)], O.frequencies(32), True, 1.3)
    assert np.abs(step[0] - want).max() <= 32 * U * 2.6 * np.abs(host(torch.cat([x, dx]))).max()


def test_not_a_number_stays_in_its_pair():
    x = rand(1, 1, 2, 2, 64)
    x[0, 0, 0, 3] = float("nan")
    x[0, 0, 0, 60] = float("inf")
    y = host(A.rotary(A.Rotary(32), x, start=ints([4])))
    bad = ~np.isfinite(y)
    assert bad[0, 0, 0, 3] and bad[0, 0, 0, 19] and bad[0, 0, 0, 60] and bad.sum() == 3


def test_a_graph_replays_with_the_positions_of_the_time():
    rot = A.Rotary(64)
    q, k = rand(1, 2, 1, 4, 64, dtype="bf16"), rand(2, 2, 1, 2, 64, dtype="bf16")
    qo, ko, start = torch.zeros_like(q), torch.zeros_like(k), ints([3, 9])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        A.rotary(rot, q, k, start=start, q_out=qo, k_out=ko)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        A.rotary(rot, q, k, start=start, q_out=qo, k_out=ko)
    for step in range(4):
        q.copy_(rand(10 + step, 2, 1, 4, 64, dtype="bf16"))
        start.add_(1)
        g.replay()
        a, b = A.rotary(rot, q, k, start=start)
        torch.cuda.synchronize()
        assert torch.equal(a, qo) and torch.equal(b, ko)


def test_on_another_stream():
    rot, q = A.Rotary(64), rand(1, 2, 33, 4, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = A.rotary(rot, q, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, A.rotary(rot, q))


@pytest.mark.parametrize("inter", [False, True])
def test_the_inverse_has_the_amplitude_too(inter):
    """Turned and turned by the transpose, a pair comes back times amplitude^2: each
    turn is off by 8 u A (|x| + |y|), the second also turns the first one's error."""
    rot, x, s = A.Rotary(64, interleaved=inter, amplitude=1.5), rand(1, 1, 9, 2, 64), ints([1000])
    got = host(A.rotary(rot, A.rotary(rot, x, start=s), start=s, inverse=True))
    size = np.abs(host(x)).reshape(1, 9, 2, *((32, 2) if inter else (2, 32))).sum(-1 if inter else -2, keepdims=True)
    tol = np.broadcast_to(32 * U * 2.25 * size, (1, 9, 2, *((32, 2) if inter else (2, 32)))).reshape(got.shape)
    assert (np.abs(got - 2.25 * host(x)) <= tol).all()


@pytest.mark.parametrize("dtype, D, H, Hk, T", [("f32", 64, 12, 12, 800), ("bf16", 96, 7, 1, 2800), ("f32", 128, 5, 3, 1100),
                                                ("bf16", 64, 9, 2, 2800)])
@pytest.mark.parametrize("how", [None, "odd"])
def test_threads_of_several_heads(dtype, D, H, Hk, T, how):
    """131072 threads with four heads each, or with those that are left."""
    inter = D == 128
    el = 2 if dtype == "bf16" else 4
    assert 4 * T * (D * el // 16 // (1 if inter else 2)) * ((H + Hk + 3) // 4) >= 131072
    rot = A.Rotary(D, base=500000.0, interleaved=inter)
    q, k = rand(1, 4, T, H, D, dtype=dtype), rand(2, 4, T, Hk, D, dtype=dtype)
    if how:
        q, k = laid_out(q, how), laid_out(k, how)
    qo, ko = A.rotary(rot, q, k, count=ints([T, T - 1, 1, 0]))
    pos, counts = [range(T)] * 4, [T, T - 1, 1, 0]
    check(qo, q, pos, counts, (O.frequencies(D, 500000.0), inter, 1.0), dtype=dtype)
    check(ko, k, pos, counts, (O.frequencies(D, 500000.0), inter, 1.0), dtype=dtype)
