"""A small bf16 decoder that generates behind a prompt: planned graphs for the
dense layers, and between them attention with a window and a few first tokens,
a key/value cache held in 4 bits, and attention over it.

    python examples/windowed_decoder.py [--layers 2 --hidden 1024 --heads 8 --kv-heads 2 --prompt 512 --steps 32]

Random weights; a layer's last output stands for the next token's embedding.
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
                 batch=1, max_tokens=4096, page_tokens=64, seed=0):
        import torch
        from paper_2411_09242_amd import attention as A
        from paper_2411_09242_amd import fluid as F
        F.load()
        self.torch, self.A, self.F = torch, A, F
        self.B, self.C, self.H, self.Hk, self.D = batch, hidden, heads, kv_heads, head_dim
        self.ffn, self.window, self.sinks = ffn, window, sinks
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda k, n: (torch.randn(k, n, generator=g, device="cuda") / k ** 0.5).bfloat16()  # noqa: E731
        one = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
        q, kv = heads * head_dim, kv_heads * head_dim
        self.weights = [([one, w(hidden, q), w(hidden, kv), w(hidden, kv)],
                         [w(q, hidden), one, w(hidden, ffn), w(hidden, ffn), w(ffn, hidden)]) for _ in range(layers)]
        self.caches = [A.KvCache(batch, kv_heads, head_dim, max_tokens, page_tokens=page_tokens) for _ in range(layers)]
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

    def _forward(self, x, attend):
        """All layers on x [batch, T, hidden]; attend(layer, q, k, v, out)."""
        B, T, _ = x.shape
        for layer, (project, finish) in enumerate(self._runs(T)):
            project.inputs[0].copy_(x)
            q, k, v = project.run()
            finish.inputs[0].copy_(x)
            attend(layer, q.view(B, T, self.H, self.D), k.view(B, T, self.Hk, self.D), v.view(B, T, self.Hk, self.D),
                   finish.inputs[1].view(B, T, self.H, self.D))
            x = finish.run()[0]
        return x

    def prompt(self, x):
        """The prompt's hidden states; its keys and values go into the cache,
        which has to be empty: ``extend`` takes what comes behind."""
        if any(n for c in self.caches for n in c.lengths):
            raise ValueError("a prompt sees its own tokens alone, and the cache holds some: use extend, or clear it")
        def attend(layer, q, k, v, out):
            self.A.attention(q, k, v, window=self.window, sinks=self.sinks, out=out)
            self.caches[layer].append(k, v)
        return self._forward(x, attend)

    def step(self, x):
        """One token of every sequence behind what the cache holds."""
        def attend(layer, q, k, v, out):
            cache = self.caches[layer]
            cache.append(k, v)
            cache.attend(q, window=self.window, sinks=self.sinks, out=out)
        return self._forward(x, attend)

    def extend(self, x):
        """Several tokens at once, over the cache read back."""
        def attend(layer, q, k, v, out):
            cache = self.caches[layer]
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
    a = vars(ap.parse_args(argv))
    prompt, steps = a.pop("prompt"), a.pop("steps")
    d = Decoder(max_tokens=prompt + 2 * steps, **a)
    torch = d.torch
    x = torch.randn(a["batch"], prompt, a["hidden"], device="cuda").bfloat16()
    d._runs(prompt), d._runs(1)  # plans are made ahead of time
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
