"""4-bit matrices on the GPU against plain NumPy (oracle/decoder_layers.py).

Tolerance of a product.  With u = 2^-24 a sum of n fp32 terms is off by at most
n u times the sum of their sizes.  A group's sum of x (16 + n) has G terms of at
most 31 |x| (fp32 x in parts that leave u of it), x's own G of |x|; s and b enter
in fp32, and the groups are summed: (G + groups + 8) u times the sum of
(31 |s| + |b|) |x|, twice that for matrix cores that cut a sum's last bit off.
SiLU has a slope of at most 1.1 and rounds by 4 u; a bf16 output by 2^-8."""
import numpy as np
import pytest

from oracle import decoder_layers as O

torch = pytest.importorskip("torch")
from paper_2411_09242_amd import fluid as F  # noqa: E402
from paper_2411_09242_amd import w4 as W  # noqa: E402

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def gpu_lib():
    F.load()
    yield


def rand(seed, *shape, dtype="f32", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(DT[dtype]).cuda()


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


def matrix(seed, N, K, group):
    """A matrix in 4 bits, made by the oracle's bytes; levels and pairs."""
    w = (host(rand(seed, N, K)) * np.exp(0.3 * host(rand(seed + 1, N, 1))) / K ** 0.5).astype(np.float32)
    n, s, b = O.quantise(w, group)
    return n, s, b


def held(n, s, b, group):
    """The bytes, by whole arrays."""
    N, K = n.shape
    tiles, blocks = -(-N // 16), -(-K // 128)
    full = np.zeros((tiles * 16, blocks * 128), np.uint32)
    full[:N, :K] = n
    full = full.reshape(tiles, 16, blocks, 4, 4, 8).transpose(0, 2, 4, 1, 3, 5)
    words = np.zeros(full.shape[:-1], np.uint32)
    for e in range(8):
        words |= full[..., e] << np.uint32(4 * O.NIBBLE[e])
    pairs = np.zeros((tiles * 16, blocks * 128 // group, 2), np.float16)
    pairs[:N, :s.shape[1], 0], pairs[:N, :s.shape[1], 1] = s, b
    pairs = pairs.reshape(tiles, 16, blocks, 128 // group, 2).transpose(0, 2, 1, 3, 4)
    return np.concatenate([np.ascontiguousarray(words).reshape(-1).view(np.uint8),
                           np.ascontiguousarray(pairs).reshape(-1).view(np.uint8)])


def w4_of(n, s, b, group):
    return W.W4(torch.from_numpy(held(n, s, b, group)).cuda(), *n.shape, group)


SHAPES = [(16, 128, 128), (1, 1, 32), (17, 129, 64), (40, 300, 32), (33, 200, 128), (5, 40, 64)]


@pytest.mark.parametrize("N, K, group", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packing_makes_the_formats_bytes_and_reading_gives_their_values(N, K, group, dtype):
    m = rand(1, N, K, dtype=dtype) * torch.exp(rand(2, N, 1)).to(DT[dtype])
    m = m.to(DT[dtype])
    if K > 2:
        m[0, :] = 0.375  # a flat group
        m[N // 2, K // 2] = 1e6  # past the limit
    n, s, b = O.quantise(host(m).astype(np.float32), group)
    want = O.pack(n, s, b, group)
    assert (want == held(n, s, b, group)).all()  # the two oracles of the layout
    w = W.w4_pack(m, group)
    assert (w.packed.cpu().numpy() == want).all()
    wide = torch.full((N, K + 3), 7.0, dtype=DT[dtype], device="cuda")
    wide[:, 1:1 + K] = m
    assert torch.equal(W.w4_pack(wide[:, 1:1 + K], group).packed, w.packed)
    values = O.values(n, s, b, group)
    assert (host(W.w4_read(w)) == values.astype(np.float32)).all()
    out = torch.full((N, K + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    W.w4_read(w, out=out[:, 2:2 + K])
    assert (host(out[:, 2:2 + K]) == host(torch.tensor(values.astype(np.float32)).bfloat16())).all()
    assert (out[:, :2] == 7.0).all() and (out[:, 2 + K:] == 7.0).all()


def test_groups_that_hold_no_number():
    m = rand(1, 20, 256)
    m[3, 40] = float("inf")
    m[7, 200] = float("nan")
    w = W.w4_pack(m, 64)
    n, s, b = O.quantise(host(m).astype(np.float32), 64)
    assert (w.packed.cpu().numpy() == held(n, s, b, 64)).all()
    v = host(W.w4_read(w))
    assert np.isnan(v[3, :64]).all() and np.isnan(v[7, 192:]).all() and np.isnan(v).sum() == 128
    y = host(W.w4_matmul(rand(2, 3, 256), w))
    assert np.isnan(y[:, [3, 7]]).all() and np.isfinite(np.delete(y, [3, 7], 1)).all()


def check(got, x, parts, group, dtype, gate=None, add=None):
    n, s, b = parts
    K = n.shape[1]
    x = host(x).reshape(-1, K)
    terms = 2 * (group + -(-K // group) + 8) * U
    want, size = O.product(x, n, s, b, group)
    tol = terms * size
    if gate is not None:
        z, zs = O.product(x, *gate, group)
        with np.errstate(over="ignore"):
            silu = z / (1 + np.exp(-z))
        tol = tol * (np.abs(silu) + 1.1 * terms * zs) + np.abs(want) * (1.1 * terms * zs + 4 * U * np.abs(silu))
        want = want * silu
        tol = tol + U * np.abs(want)
    if add is not None:
        want = want + host(add).reshape(want.shape)
        tol = tol + U * np.abs(want)
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    got = host(got).reshape(want.shape)
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / np.maximum(tol, 1e-30)).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", [1, 2, 5, 16, 17, 32, 40, 64, 70])
def test_products(dtype, group, M):
    for N, K in ((48, 256), (777, 1000), (17, 129), (1, 8), (130, 2100)):
        parts, gate = matrix(1, N, K, group), matrix(5, N, K, group)
        x, add = rand(9, M, K, dtype=dtype), rand(11, M, N, dtype=dtype)
        w, g = w4_of(*parts, group), w4_of(*gate, group)
        check(W.w4_matmul(x, w), x, parts, group, dtype)
        check(W.w4_matmul(x, w, add=add), x, parts, group, dtype, add=add)
        check(W.w4_matmul(x, w, gate=g), x, parts, group, dtype, gate)
        check(W.w4_matmul(x, w, gate=g, add=add), x, parts, group, dtype, gate, add)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_rows_and_many_tiles(dtype):
    for N, K, group, M in ((64, 16000, 128, 1), (5000, 640, 32, 3), (16, 11008, 64, 33)):
        parts = matrix(1, N, K, group)
        x = rand(9, M, K, dtype=dtype)
        check(W.w4_matmul(x, w4_of(*parts, group)), x, parts, group, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_dimensions_and_outputs(dtype):
    N, K, group = 50, 200, 64
    parts = matrix(1, N, K, group)
    w = w4_of(*parts, group)
    for off, pad in ((0, 8), (1, 3)):
        buf = torch.full((2, 3, K + pad), float("nan"), dtype=DT[dtype], device="cuda")
        x = buf[..., off:off + K]
        x.copy_(rand(3, 2, 3, K, dtype=dtype))
        out = torch.full((2, 3, N + 5), 7.0, dtype=DT[dtype], device="cuda")
        res = out[..., 2:2 + N]
        res.copy_(rand(4, 2, 3, N, dtype=dtype))
        add = res.clone()
        got = W.w4_matmul(x, w, add=res, out=res)  # the residual in place
        assert got is res
        check(got, x, parts, group, dtype, add=add)
        assert (out[..., :2] == 7.0).all() and (out[..., 2 + N:] == 7.0).all()
    one = rand(5, 1, K, dtype=dtype)
    y = W.w4_matmul(one.expand(4, K), w)  # a row repeated
    assert torch.equal(y, W.w4_matmul(one, w).expand(4, N))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 4, 5, 16, 20, 32, 33])
def test_two_tiles_to_a_workgroup(dtype, M):
    """So many rows of the matrix that workgroups have two tiles; the last has one."""
    N, group = 16 * 513 - 3, 64
    for K, pad in ((300, 0), (301, 0), (1500, 7)):
        parts = matrix(K, N, K, group)
        x = rand(3, M, K + pad, dtype=dtype)[:, :K]
        check(W.w4_matmul(x, w4_of(*parts, group)), x, parts, group, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 3, 16, 21, 40])
def test_rows_of_every_length_and_alignment(dtype, M):
    """Pieces of eight channels that end with the row, words that start between two
    rows; what lies beside the rows is no number."""
    N, group = 19, 32
    for K in (1, 5, 7, 8, 9, 15, 16, 100, 127, 131, 136, 255):
        parts = matrix(K, N, K, group)
        w = w4_of(*parts, group)
        for off, pad in ((0, 0), (1, 2), (2, 5), (3, 4)):
            buf = torch.full((M * (K + pad) + 8,), float("nan"), dtype=DT[dtype], device="cuda")
            x = buf[off:off + M * (K + pad)].view(M, K + pad)[:, :K]
            x.copy_(rand(3 + K, M, K, dtype=dtype))
            check(W.w4_matmul(x, w), x, parts, group, dtype)


def test_rows_do_not_touch_each_other():
    """A row that is no number makes none of the others so, and a row's result
    does not depend on what is beside it."""
    N, K = 40, 300
    parts = matrix(1, N, K, 32)
    w = w4_of(*parts, 32)
    for dtype in DT:
        x = rand(3, 20, K, dtype=dtype)
        y = W.w4_matmul(x, w)
        x[7, 5], x[11, 299] = float("nan"), float("inf")
        z = W.w4_matmul(x, w)
        rest = [i for i in range(20) if i not in (7, 11)]
        assert torch.equal(y[rest], z[rest]) and not z[[7, 11]].isfinite().any()


def test_a_graph_replays():
    parts, gate = matrix(1, 96, 512, 128), matrix(3, 96, 512, 128)
    w, g = w4_of(*parts, 128), w4_of(*gate, 128)
    x, out = rand(1, 1, 512, dtype="bf16"), torch.zeros(1, 96, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        W.w4_matmul(x, w, gate=g, out=out)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        W.w4_matmul(x, w, gate=g, out=out)
    for i in range(4):
        x.copy_(rand(20 + i, 1, 512, dtype="bf16"))
        graph.replay()
        want = W.w4_matmul(x, w, gate=g)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_on_another_stream():
    m, x = rand(1, 100, 300), rand(2, 4, 300)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    w = W.w4_pack(m, 32, stream=s)
    y, v = W.w4_matmul(x, w, stream=s), W.w4_read(w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    w1 = W.w4_pack(m, 32)
    assert torch.equal(w.packed, w1.packed) and torch.equal(y, W.w4_matmul(x, w1)) and torch.equal(v, W.w4_read(w1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 2, 4, 5])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_an_output_head_of_few_rows(dtype, M, group):
    """1025 tiles: from 1024 on up to four rows too have two tiles to a workgroup."""
    N = 16 * 1025 - 3
    for K, pad in ((300, 0), (301, 0), (520, 7)):
        parts = matrix(K, N, K, group)
        x, add = rand(3, M, K + pad, dtype=dtype)[:, :K], rand(5, M, N, dtype=dtype)
        add = add if K == 301 else None
        check(W.w4_matmul(x, w4_of(*parts, group), add=add), x, parts, group, dtype, add=add)


@pytest.mark.parametrize("M, group", [(6, 32), (20, 128)])
def test_two_tiles_in_other_groups(M, group):
    N = 16 * 513 - 3
    for dtype in DT:
        parts = matrix(7, N, 301, group)
        x = rand(3, M, 301, dtype=dtype)
        check(W.w4_matmul(x, w4_of(*parts, group)), x, parts, group, dtype)


@pytest.mark.parametrize("dtype, M", [("bf16", 40), ("bf16", 70), ("f32", 17)])
@pytest.mark.parametrize("gated", [False, True])
def test_graphs_of_products_in_runs_replay(dtype, M, gated):
    """Products in two launches with a workspace: one graph with its own, two that
    share the caller's, eager calls between the replays."""
    N, K = 96, 4096
    w, g = w4_of(*matrix(1, N, K, 64), 64), w4_of(*matrix(3, N, K, 64), 64) if gated else None
    x, add = rand(1, M, K, dtype=dtype), rand(2, M, N, dtype=dtype)
    need = W.w4_matmul_workspace(x, w, gated)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros(M, N, dtype=DT[dtype], device="cuda") for _ in range(3)]
    W.w4_matmul(x, w, gate=g, add=add, out=outs[0])
    graphs = []
    for i, out in enumerate(outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            W.w4_matmul(x, w, gate=g, add=add if i < 2 else None, out=out, workspace=ws if i else None)
    for i in range(4):
        x.copy_(rand(20 + i, M, K, dtype=dtype))
        for out in outs:
            out.fill_(7.0)
        ws.fill_(255)
        for graph in graphs:
            graph.replay()
        want, plain = W.w4_matmul(x, w, gate=g, add=add), W.w4_matmul(x, w, gate=g, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want) and torch.equal(outs[2], plain)
    with pytest.raises(F.FluidError, match="workspace"):
        W.w4_matmul(x, w, gate=g, workspace=ws[:need - 256])
