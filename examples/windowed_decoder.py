"""A small bf16 decoder that generates behind a prompt: planned graphs for the
dense layers, and between them attention with a window and a few first tokens,
a key/value cache held in 4 bits, and attention over it.

    python examples/windowed_decoder.py [--layers 2 --hidden 1024 --heads 8 --kv-heads 2 --prompt 512 --steps 32]
        [--rotary] [--four-bit] [--linear-every 2]

Random weights; a layer's last output stands for the next token's embedding.
With ``rotary`` queries and keys are turned by their positions; with
``four_bit`` single tokens run products with 4-bit copies of the weights instead of
the planned graphs; with ``linear_every`` n every n-th layer has linear attention
with a state in the place of a cache.
Prompt: ``attention`` over the prompt's own keys and values, which then go into
the cache (``KvCache.append``).  Steps: one token appended and attended over the
cache (``KvCache.attend``), pages that the window has left behind given back
(``KvCache.trim``).  ``extend`` takes several tokens at once as a second chunk
of a prompt would: the cache read back, and ``attention`` over that.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

EPS = 1e-5


def project_desc(B, T, C, q, kv):
    """x -> RMSNorm -> queries, keys, values."""
    w = lambda k, n: {"role": "weight", "shape": [k, n], "dtype": "bf16"}  # noqa: E731
    mm = lambda i, c, n: {"op": "matmul", "ins": [i, ~c], "out_shape": [B, T, n]}  # noqa: E731
    return {"dtype": "bf16", "inputs": [[B, T, C]],
            "consts": [{"role": "gamma", "shape": [C], "dtype": "bf16"}, w(C, q), w(C, kv), w(C, kv)],
            "nodes": [{"op": "rmsnorm", "ins": [0, ~0], "out_shape": [B, T, C], "fattr": EPS},
                      mm(1, 1, q), mm(1, 2, kv), mm(1, 3, kv)],
            "outputs": [2, 3, 4]}


def finish_desc(B, T, C, q, ffn):
    """x, attention -> output product, residual, SwiGLU block."""
    w = lambda k, n: {"role": "weight", "shape": [k, n], "dtype": "bf16"}  # noqa: E731
    node = lambda op, ins, n, **kw: {"op": op, "ins": ins, "out_shape": [B, T, n], **kw}  # noqa: E731
    return {"dtype": "bf16", "inputs": [[B, T, C], [B, T, q]],
            "consts": [w(q, C), {"role": "gamma", "shape": [C], "dtype": "bf16"}, w(C, ffn), w(C, ffn), w(ffn, C)],
            "nodes": [node("matmul", [1, ~0], C), node("add", [2, 0], C), node("rmsnorm", [3, ~1], C, fattr=EPS),
                      node("matmul", [4, ~2], ffn), node("silu", [5], ffn), node("matmul", [4, ~3], ffn),
                      node("mul", [6, 7], ffn), node("matmul", [8, ~4], C), node("add", [9, 3], C)],
            "outputs": [10]}


class Decoder:
    def __init__(self, layers=2, hidden=1024, heads=8, kv_heads=2, head_dim=128, ffn=2816, window=256, sinks=4,
                 batch=1, max_tokens=4096, page_tokens=64, seed=0, rotary=False, four_bit=False, linear_every=0):
        import torch
        from paper_2411_09242_amd import attention as A
        from paper_2411_09242_amd import fluid as F
        from paper_2411_09242_amd import w4
        F.load()
        self.torch, self.A, self.F, self.w4 = torch, A, F, w4
        self.B, self.C, self.H, self.Hk, self.D = batch, hidden, heads, kv_heads, head_dim
        self.ffn, self.window, self.sinks = ffn, window, sinks
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda k, n: (torch.randn(k, n, generator=g, device="cuda") / k ** 0.5).bfloat16()  # noqa: E731
        one = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
        q, kv = heads * head_dim, kv_heads * head_dim
        self.weights = [([one, w(hidden, q), w(hidden, kv), w(hidden, kv)],
                         [w(q, hidden), one, w(hidden, ffn), w(hidden, ffn), w(ffn, hidden)]) for _ in range(layers)]
        # what a layer keeps of the tokens so far: a cache, or a state
        self.memory = [torch.zeros(batch, kv_heads, head_dim, head_dim, device="cuda")
                       if linear_every and (i + 1) % linear_every == 0 else
                       A.KvCache(batch, kv_heads, head_dim, max_tokens, page_tokens=page_tokens) for i in range(layers)]
        self.caches = [m for m in self.memory if isinstance(m, A.KvCache)]
        self.seen = torch.zeros(batch, dtype=torch.int32, device="cuda")  # tokens so far
        # states remember some 16 to 500 tokens, by head
        self.decay = torch.log1p(-torch.exp2(-torch.linspace(4, 9, kv_heads, device="cuda")))
        self.rot = A.Rotary(head_dim) if rotary else None
        self.small = [self._four_bit(*w) for w in self.weights] if four_bit else None
        self.runs = {}

    plans = {}  # of all decoders, by graph

    def _plan(self, desc):
        """Graph, layouts and arena.  A plan follows measured times: another
        measurement may choose other kernels, which round elsewhere, so a graph
        is measured once and decoders of the same shapes give the same bits."""
        F, key = self.F, repr(desc)
        if key not in self.plans:
            graph = F.Graph.from_desc(desc)
            plan = F.LayoutPlan(graph, F.CostTable.measure(graph))
            self.plans[key] = graph, plan, F.ArenaPlan(graph, plan)
        return self.plans[key]

    def _runs(self, T):
        """Executors of both graphs for every layer, for T tokens a sequence."""
        if T not in self.runs:
            F, torch = self.F, self.torch
            q, kv = self.H * self.D, self.Hk * self.D

            def make(desc, consts):
                graph, plan, arena = self._plan(desc)
                return [F.Executor(graph, plan, arena, c, [torch.zeros(s) for s in desc["inputs"]]) for c in consts]
            self.runs[T] = list(zip(
                make(project_desc(self.B, T, self.C, q, kv), [a for a, _ in self.weights]),
                make(finish_desc(self.B, T, self.C, q, self.ffn), [b for _, b in self.weights])))
        return self.runs[T]

    def _four_bit(self, project, finish):
        """A layer's matrices in 4 bits: q, k and v in one, the others; outputs
        first, as products take them."""
        pack = lambda *m: self.w4.w4_pack(self.torch.cat([t.t() for t in m]).contiguous(), 64)  # noqa: E731
        return [pack(*project[1:])] + [pack(m) for m in (finish[0], *finish[2:])]

    def _norm(self, x):
        f = x.float()
        return (f * (f.square().mean(-1, keepdim=True) + EPS).rsqrt()).bfloat16()

    def _small_layer(self, layer, x, attend):
        """A layer of single tokens with 4-bit products."""
        B, T, _ = x.shape
        mul, (qkv, o, gate, up, down) = self.w4.w4_matmul, self.small[layer]
        heads = mul(self._norm(x), qkv).view(B, T, self.H + 2 * self.Hk, self.D)
        q, k, v = heads.split([self.H, self.Hk, self.Hk], 2)
        a = self.torch.empty(B, T, self.H, self.D, dtype=x.dtype, device=x.device)
        attend(layer, q, k, v, a)
        x = mul(a.view(B, T, -1), o, add=x)
        return mul(mul(self._norm(x), up, gate=gate), down, add=x)

    def _forward(self, x, attend):
        """All layers on x [batch, T, hidden]; attend(layer, q, k, v, out)."""
        B, T, _ = x.shape

        def mix(layer, q, k, v, out):
            if self.rot is not None:
                self.A.rotary(self.rot, q, k, start=self.seen, q_out=q, k_out=k)
            state = self.memory[layer]
            if isinstance(state, self.A.KvCache):
                attend(state, q, k, v, out)
            else:
                self.A.linear_attention(q, k, v, self.decay, state=state, state_out=state, out=out)
        if self.small is not None and T == 1:
            for layer in range(len(self.weights)):
                x = self._small_layer(layer, x, mix)
        else:
            for layer, (project, finish) in enumerate(self._runs(T)):
                project.inputs[0].copy_(x)
                q, k, v = project.run()
                finish.inputs[0].copy_(x)
                mix(layer, q.view(B, T, self.H, self.D), k.view(B, T, self.Hk, self.D), v.view(B, T, self.Hk, self.D),
                    finish.inputs[1].view(B, T, self.H, self.D))
                x = finish.run()[0]
        self.seen += T
        return x

    def prompt(self, x):
        """The prompt's hidden states; its keys and values go into the cache,
        which has to be empty: ``extend`` takes what comes behind."""
        if any(n for c in self.caches for n in c.lengths):
            raise ValueError("a prompt sees its own tokens alone, and the cache holds some: use extend, or clear it")
        self.seen.zero_()
        for m in self.memory:
            if not isinstance(m, self.A.KvCache):
                m.zero_()

        def attend(cache, q, k, v, out):
            self.A.attention(q, k, v, window=self.window, sinks=self.sinks, out=out)
            cache.append(k, v)
        return self._forward(x, attend)

    def step(self, x):
        """One token of every sequence behind what the cache holds."""
        def attend(cache, q, k, v, out):
            cache.append(k, v)
            cache.attend(q, window=self.window, sinks=self.sinks, out=out)
        return self._forward(x, attend)

    def extend(self, x):
        """Several tokens at once, over the cache read back."""
        def attend(cache, q, k, v, out):
            cache.append(k, v)
            n = max(cache.lengths)
            keys = k.new_empty(self.B, n, self.Hk, self.D)
            values = torch.empty_like(keys)
            cache.read(keys, values)
            self.A.attention(q, keys, values, kv_len=cache.kv_len, window=self.window, sinks=self.sinks, out=out)
        torch = self.torch
        return self._forward(x, attend)

    def generate(self, x, steps):
        """The prompt and `steps` tokens behind it: [batch, steps, hidden]."""
        x = self.prompt(x)[:, -1:].clone()
        out = []
        for i in range(steps):
            x = self.step(x).clone()
            out.append(x)
            if i % 16 == 15:
                for c in self.caches:
                    c.trim(self.window, self.sinks)
        return self.torch.cat(out, 1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, v in (("layers", 2), ("hidden", 1024), ("heads", 8), ("kv-heads", 2), ("head-dim", 128), ("ffn", 2816),
                    ("window", 256), ("sinks", 4), ("batch", 1), ("prompt", 512), ("steps", 32)):
        ap.add_argument("--" + name, type=int, default=v)
    ap.add_argument("--linear-every", type=int, default=0)
    for name in ("rotary", "four-bit"):
        ap.add_argument("--" + name, action="store_true")
    a = vars(ap.parse_args(argv))
    prompt, steps = a.pop("prompt"), a.pop("steps")
    d = Decoder(max_tokens=prompt + 2 * steps, **a)
    torch = d.torch
    x = torch.randn(a["batch"], prompt, a["hidden"], device="cuda").bfloat16()
    for n in {prompt} if d.small else {prompt, 1}:
        d._runs(n)  # plans are made ahead of time
    torch.cuda.synchronize()
    t = time.perf_counter()
    y = d.generate(x, steps)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    held = sum(c.pool.numel() for c in d.caches)
    print(f"{a['batch']} x {prompt} prompt tokens and {steps} steps of {a['layers']} layers: {t * 1e3:.1f} ms, "
          f"cache {held / 1e6:.1f} MB, {sum(len(c.free) for c in d.caches)} pages free, "
          f"last output finite: {bool(y.isfinite().all())}")


if __name__ == "__main__":
    main()
