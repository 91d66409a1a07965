"""Linear attention on the GPU: precision, norm over norm, where bounds of single
values that grow with the tokens would let a lost part pass.

Tolerances.  u = 2^-24.  Sums that cancel: with integers that fp32 and bf16 hold
whole, and decays and a scale of 1, the exact result is 0.  What is left are fp32
roundings of partial sums: of n terms of size t, n u / 2 of at most sqrt(n) t each
where signs are random, which add up as random errors do: u n t / 2, so u times the
sum of sizes.  Factors in two bf16 parts (16 bits) leave 10 to 21 u of it.

Long prompts with random values, whose memories of 512 tokens reach over several runs.
What a chunk of 64 tokens (fp32: 32) keeps of a state is within 2 u, the same at each
chunk, and what counts at the end has passed half of a memory's 8 (16) chunks: 16 u =
2^-20, beside which the roundings of sums, some u in all, are small.  A state rounded to
bf16 is off by 1.7e-3, values in two bf16 parts by 5e-6.  bf16 rows are rounded
by at most 2^-8 of their binade's least value, 2^-8 / sqrt(3) in the mean square, and the
values of a binade are 1.47 of it: 2^-9 of themselves with what the sizes' spread adds."""
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


def rand(seed, *shape, dtype="f32"):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(DT[dtype]).cuda()


def whole(seed, most, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).float()


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


SIGNS = torch.tensor([1.0, 1.0, 1.0, -1.0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("T", [3, 64, 300])
def test_rows_of_a_state_that_cancel(dtype, D, T):
    """Every fourth row of the state is the sum of the three before it, its query
    channel their channel's negative; keys and values are 0."""
    B, H = 2, 4
    S = whole(1, 2 ** 22, B, H, D // 4, 3, D)
    S = torch.cat([S, S.sum(3, keepdim=True)], 3).reshape(B, H, D, D) / 2 ** 20
    q = (rand(2, B, T, H, D // 4, 1, dtype=dtype).cpu() * SIGNS).to(DT[dtype]).reshape(B, T, H, D).cuda()
    zero = torch.zeros(B, T, H, D, dtype=DT[dtype], device="cuda")
    out, last = A.linear_attention(q, zero, zero, torch.zeros(H, device="cuda"), state=S.cuda(), scale=1.0)
    size = np.einsum("bthk,bhkd->bthd", np.abs(host(q)), np.abs(host(S)))
    assert np.linalg.norm(host(out)) <= U * np.linalg.norm(size)
    assert torch.equal(last.cpu(), S)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("group", [1, 3])
def test_tokens_that_cancel(dtype, D, group):
    """Every fourth token's key is the sum of the three before it, its value their
    value's negative: rows that see whole fours are 0."""
    B, T, H = 2, 64, 2
    k = whole(1, 40, B, T // 4, 3, H, D)
    k = torch.cat([k, k.sum(2, keepdim=True)], 2).reshape(B, T, H, D).to(DT[dtype]).cuda()
    v = rand(2, B, T // 4, 1, H, D, dtype=dtype).cpu() * SIGNS.view(4, 1, 1)
    v = v.to(DT[dtype]).reshape(B, T, H, D).cuda()
    q = rand(3, B, T, H * group, D, dtype=dtype)
    out, last = A.linear_attention(q, k, v, torch.zeros(H, device="cuda"), scale=1.0)
    w = np.einsum("bihgd,bjhd->bhgij", host(q).reshape(B, T, H, group, D), host(k))
    size = np.einsum("bhgij,bjhd->bihgd", np.abs(np.tril(w)), np.abs(host(v))).reshape(B, T, H * group, D)
    at = slice(3, T, 4)
    assert np.linalg.norm(host(out)[:, at]) <= U * np.linalg.norm(size[:, at])
    most = np.einsum("bjhk,bjhd->bhkd", np.abs(host(k)), np.abs(host(v)))
    assert np.linalg.norm(host(last)) <= U * np.linalg.norm(most)


@pytest.mark.parametrize("dtype, T, H, Hk, D", [
    ("bf16", 2048, 4, 4, 128), ("bf16", 2048, 2, 2, 32), ("f32", 1111, 4, 2, 128), ("f32", 2000, 2, 2, 32),  # runs folded
    ("bf16", 1500, 8, 2, 64), ("bf16", 2048, 8, 1, 128), ("f32", 2000, 8, 2, 64)])  # runs added up by a launch
@pytest.mark.parametrize("per_token", [False, True])
def test_long_memories_keep_their_precision(dtype, T, H, Hk, D, per_token):
    q, k, v = rand(1, 1, T, H, D, dtype=dtype), rand(2, 1, T, Hk, D, dtype=dtype), rand(3, 1, T, Hk, D, dtype=dtype)
    g = torch.full((Hk,), -1 / 512).cuda()
    if per_token:
        g = (g * (0.5 + torch.rand(1, T, Hk, generator=torch.Generator().manual_seed(4)).cuda())).contiguous()
    state = rand(5, 1, Hk, D, D) * 16
    out, last = A.linear_attention(q, k, v, g, state=state, scale=0.125)
    decay = np.broadcast_to(host(g).reshape(-1, Hk), (T, Hk))
    for h in range(Hk):
        rows = slice(h * H // Hk, (h + 1) * H // Hk)
        o, S, _, _ = O.linear_attention(host(q)[0, :, rows], host(k)[0, :, h], host(v)[0, :, h], decay[:, h],
                                        host(state)[0, h], 0.125)
        off = np.linalg.norm(host(last)[0, h] - S) / np.linalg.norm(S)
        assert off <= 2.0 ** -20, ("state", h, off)
        off = np.linalg.norm(host(out)[0, :, rows] - o) / np.linalg.norm(o)
        assert off <= (2.0 ** -9 if dtype == "bf16" else 2.0 ** -20), ("out", h, off)
