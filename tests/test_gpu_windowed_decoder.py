"""The example that runs the cache, the attention over it and windowed
attention between planned graphs: tokens one by one against the same tokens at
once, and against a plain forward pass over the cache's own values."""
import os
import sys

import numpy as np
import pytest

from oracle import attention as OA

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def make(**kw):
    import windowed_decoder as W
    return W.Decoder(layers=2, hidden=128, heads=4, kv_heads=2, head_dim=32, ffn=192, window=24, sinks=3, batch=2,
                     max_tokens=128, page_tokens=32, **kw)


def test_one_by_one_is_as_all_at_once():
    """Both see the same cached values; what differs is where bf16 roundings of
    weights and sums fall, a few units of 2^-8 of rows of size about 1."""
    a, b = make(), make()
    x = torch.randn(2, 50, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    assert torch.equal(a.prompt(x[:, :40]), b.prompt(x[:, :40]))
    one = torch.cat([a.step(x[:, i:i + 1].contiguous()).clone() for i in range(40, 50)], 1)
    many = b.extend(x[:, 40:])
    assert a.caches[0].lengths == b.caches[0].lengths == [50, 50]
    # the first layer's keys come from the same inputs: the pools hold the same values
    k = [torch.zeros(2, 50, 2, 32, device="cuda") for _ in range(4)]
    a.caches[0].read(k[0], k[1])
    b.caches[0].read(k[2], k[3])
    assert torch.equal(k[0], k[2]) and torch.equal(k[1], k[3])
    err = (one.float() - many.float()).norm() / many.float().norm()
    assert err < 2.0 ** -8 * 4, float(err)


def test_a_step_against_a_plain_forward_pass():
    d = make()
    x = torch.randn(2, 41, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).bfloat16()
    d.prompt(x[:, :40])
    got = d.step(x[:, 40:].contiguous()).double().cpu().numpy()
    norm = lambda h: h / np.sqrt((h * h).mean(-1, keepdims=True) + 1e-5)  # noqa: E731
    h = x[:, 40].double().cpu().numpy()
    for (proj, fin), cache in zip(d.weights, d.caches):
        proj, fin = ([w.double().cpu().numpy() for w in part] for part in (proj, fin))
        k, v = (torch.zeros(2, 41, 2, 32, device="cuda") for _ in range(2))
        cache.read(k, v)
        k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
        q = (norm(h) @ proj[1]).reshape(2, 4, 32)
        a = np.stack([[OA.attention(q[b, i][None], k[b, :, i // 2], v[b, :, i // 2], 32 ** -0.5, True, 24, 3)[0][0]
                       for i in range(4)] for b in range(2)])
        h = h + a.reshape(2, 128) @ fin[0]
        n = norm(h)
        gate = n @ fin[2]
        h = h + (gate / (1 + np.exp(-gate)) * (n @ fin[3])) @ fin[4]
    # two layers of about ten bf16 roundings each, 2^-9 apiece on average, adding up as random errors do
    err = np.linalg.norm(got[:, 0] - h) / np.linalg.norm(h)
    assert err < 2.0 ** -9 * np.sqrt(20) * 2, err


def test_generation_runs_and_gives_pages_back():
    d = make()
    x = torch.randn(2, 40, 128, device="cuda").bfloat16()
    y = d.generate(x, 48)
    assert y.shape == (2, 48, 128) and y.isfinite().all()
    for c in d.caches:
        assert c.lengths == [88, 88] and len(c.free) > 0


def test_command_line(capsys):
    import windowed_decoder as W
    W.main(["--hidden", "256", "--heads", "4", "--kv-heads", "2", "--head-dim", "64", "--ffn", "512", "--prompt", "70",
            "--steps", "4", "--window", "32"])
    assert "last output finite: True" in capsys.readouterr().out


def test_a_second_prompt_behind_cached_tokens_is_refused():
    """It would not see them."""
    d = make()
    x = torch.randn(2, 40, 128, device="cuda").bfloat16()
    first = d.prompt(x).clone()
    with pytest.raises(ValueError, match="extend"):
        d.prompt(x)
    for c in d.caches:
        assert c.lengths == [40, 40]
        c.clear(0), c.clear(1)
    assert torch.equal(d.prompt(x), first)
