"""Cases of what a decoder's layers need beside attention over the cache:
rotary positions, products with 4-bit weights, and linear attention with a
decay.

Kinds of case:
  * ``rotary``: queries and keys turned by their positions, in one call;
  * ``w4``: rows times a matrix held in 4 bits, with a residual added or a
    gate's product in the same call;
  * ``linear``: linear attention from a state on, which single tokens and
    whole prompts share.

Rotary.  Pair i of the first d channels turns by the angle p theta_i at
position p, theta_i = base^(-2i / d); it is channels (i, i + d / 2), or
(2i, 2i + 1) where interleaved.  A longer context divides theta_i by a factor:
all of them (``linear``), through the base, base * factor^(d / (d - 2))
(``base``), or those that turn less than ``low`` times over ``length`` tokens
and none of those that turn more than ``high`` times, in proportion between
(``ramp``).  ``amplitude`` multiplies the turned channels.

Weights in 4 bits.  A matrix [N, K] has groups of G channels of a row, with a
pair of float16 (s, b) each; the nibble n stands for b + s (16 + n);
s = f16((max - min) / 15), b = f16(min - 16 s), n = rint((x - b) / s) - 16
within 0 .. 15.  In bytes: for every 16 rows and 128 channels (the last ones
padded) 64 x 4 words, word j of place 16 g + r with the channels 32 j + 8 g ..
+ 7 of row r, element e at nibble (e >> 1) + 4 (e & 1); behind all of them, for
the same tiles, 16 rows x 128 / G words with s in the low half, b in the high.

Linear attention.  S_t = exp(g_t) S_{t-1} + k_t v_t^T and
o_t = scale S_t^T q_t for every head, g_t the logarithm of the head's decay
(fixed, or one a token), S [dim, dim] in fp32.
"""
import math

import torch

own = False

LIMIT = 16384.0  # weights beyond it are stored as it
CHUNK = 64       # tokens that the plain linear attention takes together


# ------------------------------------------------------------------ cases
def _rotary(name, dtype, batch, tokens, q_heads, kv_heads, dim, part, far, interleaved=False, scaling="none",
            ragged=False):
    c = dict(kind="rotary", dtype=dtype, batch=batch, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, dim=dim,
             part=part, far=far, interleaved=interleaved, scaling=scaling, ragged=ragged)
    return dict(c, name=name) if name else c


def _w4(name, dtype, rows, k, n, group, gate=False, add=False):
    c = dict(kind="w4", dtype=dtype, rows=rows, k=k, n=n, group=group, gate=gate, add=add)
    return dict(c, name=name) if name else c


def _linear(name, dtype, batch, tokens, q_heads, kv_heads, dim, fixed=True, ragged=False):
    c = dict(kind="linear", dtype=dtype, batch=batch, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, dim=dim,
             fixed=fixed, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's decode step far into a scaled context: latency counts
        _rotary("rotary-one", "bf16", 1, 1, 32, 8, 128, 128, 100000, scaling="ramp"),
        # five drafted tokens of each of eight sequences, fp32 heads of 64
        _rotary("rotary-draft", "f32", 8, 5, 12, 12, 64, 64, 1000, ragged=True),
        # a long bf16 prompt, four query heads to a key head
        _rotary("rotary-prompt", "bf16", 1, 8192, 32, 8, 128, 128, 8192),
        # second chunks of ragged prompts, a quarter of the head turned, pairs
        # interleaved
        _rotary("rotary-part", "f32", 8, 500, 16, 16, 64, 16, 20000, interleaved=True, scaling="base", ragged=True),
        # one token's output product with the residual
        _w4("w4-one", "bf16", 1, 4096, 4096, 128, add=True),
        # one token's gated half of the feed-forward block
        _w4("w4-gate", "bf16", 1, 4096, 11008, 128, gate=True),
        # the other half for a served batch
        _w4("w4-batch", "bf16", 32, 11008, 4096, 64, add=True),
        # five tokens in fp32, odd sizes, the smallest groups
        _w4("w4-odd", "f32", 5, 1000, 777, 32),
        # one user's decode step: the states of 32 heads
        _linear("linear-one", "bf16", 1, 1, 32, 32, 128),
        # a served batch's decode step, a decay for every token
        _linear("linear-batch", "bf16", 64, 1, 32, 32, 128, fixed=False),
        # a long prompt
        _linear("linear-prompt", "bf16", 1, 8192, 32, 32, 128),
        # fp32 prompts of up to 512 tokens, odd lengths, shared keys
        _linear("linear-ragged", "f32", 8, 512, 16, 4, 64, fixed=False, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


_MOST = {}


def _most(kind):
    if not _MOST:
        for c in listed():
            _MOST[c["kind"]] = max(_MOST.get(c["kind"], 0.0), _cost(c))
    return _MOST[kind]


def draw(rng):
    while True:
        kind = rng.choice(["rotary", "w4", "linear"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if kind == "w4":
            c = _w4("", dtype, rng.choice([1, 1, _log(rng, 1, 64)]), _log(rng, 64, 16384), _log(rng, 16, 32768),
                    rng.choice([32, 64, 128, 128]), rng.random() < 0.3, rng.random() < 0.4)
        else:
            kv_heads = rng.choice([1, 2, 4, 8, 8, 12, 16, 32])
            q_heads = kv_heads * rng.choice([1, 1, 2, 4, 7])
            batch, tokens = _log(rng, 1, 64), rng.choice([1, _log(rng, 1, 8192), _log(rng, 16, 8192)])
            ragged = rng.random() < 0.5
            if kind == "rotary":
                dim = rng.choice([64, 128, 128, 80, 96, 256])
                part = rng.choice([dim, dim, dim // 2, dim // 4])
                c = _rotary("", dtype, batch, tokens, q_heads, kv_heads, dim, part, _log(rng, 1, 1000000),
                            rng.random() < 0.4, rng.choice(["none", "linear", "base", "ramp"]), ragged)
            else:
                c = _linear("", dtype, batch, tokens, q_heads, kv_heads, rng.choice([32, 64, 128, 128]),
                            rng.random() < 0.5, ragged)
        if _cost(c) <= _most(kind):
            return c


def _counts(case):
    """Tokens of every sequence; the first has all."""
    t = case["tokens"]
    if not case["ragged"]:
        return [t] * case["batch"]
    return [t - int(0.7 * (t - 1) * math.modf(b * 0.7548776662466927)[0]) for b in range(case["batch"])]


def work(case):
    el = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "w4":
        M, K, N, mats = case["rows"], case["k"], case["n"], 2 if case["gate"] else 1
        held = mats * N * (K / 2 + 4 * -(-K // case["group"]))
        return {"bytes": held + el * M * (K + N * (2 if case["add"] else 1)), "flops": 2.0 * mats * M * N * K}
    H, Hk, D, tokens = case["q_heads"], case["kv_heads"], case["dim"], sum(_counts(case))
    if case["kind"] == "rotary":
        return {"bytes": 2.0 * el * tokens * (H + Hk) * D, "flops": 3.0 * tokens * (H + Hk) * case["part"]}
    state = 8.0 * case["batch"] * Hk * D * D  # read once, written once
    return {"bytes": el * tokens * (2.0 * H + 2.0 * Hk) * D + state, "flops": 2.0 * D * D * (H + Hk) * tokens}


# ----------------------------------------------------------------- inputs
def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _scaling(case):
    """Base, factor, length and amplitude as models of such contexts have them."""
    kind = case["scaling"]
    factor = 1.0 if kind == "none" else 8.0
    return dict(base=10000.0 if kind == "none" else 500000.0, scaling=kind, factor=factor, length=8192, low=1.0, high=4.0,
                amplitude=0.1 * math.log(factor) + 1.0 if kind == "ramp" else 1.0)


def _pack(w, G):
    """A matrix [N, K] in 4 bits, as bytes; all torch, a row's groups at a time."""
    N, K = w.shape
    tiles, blocks = -(-N // 16), -(-K // 128)
    kg = -(-K // G)
    # a short last group is filled with its own last value
    g = torch.cat([w, w[:, -1:].expand(N, kg * G - K)], 1).view(N, kg, G).clamp(-LIMIT, LIMIT)
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    s = ((hi - lo) / torch.full_like(hi, 15)).half().float()
    b = (lo - 16 * s).half().float()
    n = torch.where(s > 0, (torch.round((g - b) / s) - 16).clamp(0, 15), torch.zeros_like(g)).view(N, kg * G)
    n[:, K:] = 0
    level = torch.zeros(tiles * 16, blocks * 128, dtype=torch.int32, device=w.device)
    level[:N, :min(kg * G, blocks * 128)] = n[:, :blocks * 128].to(torch.int32)
    # [tile, row, block, word, place, element] to [tile, block, place, row, word, element]
    level = level.view(tiles, 16, blocks, 4, 4, 8).permute(0, 2, 4, 1, 3, 5)
    e = torch.arange(8, device=w.device)
    words = (level << (4 * ((e >> 1) + 4 * (e & 1)))).sum(-1, dtype=torch.int32)
    pairs = torch.zeros(tiles * 16, blocks * (128 // G), 2, dtype=torch.float16, device=w.device)
    pairs[:N, :kg, 0], pairs[:N, :kg, 1] = s.squeeze(-1).half(), b.squeeze(-1).half()
    pairs = pairs.view(tiles, 16, blocks, 128 // G, 2).transpose(1, 2).contiguous()
    return torch.cat([words.flatten().view(torch.uint8), pairs.flatten().view(torch.uint8)])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s = dict(case=case, dt=dt)
    if case["kind"] == "w4":
        M, K, N = case["rows"], case["k"], case["n"]
        s["x"] = _rand(gen, M, K).to(dt)
        for name in ("w", "gate") if case["gate"] else ("w",):
            # rows and channels of different sizes, as trained matrices have them
            w = _rand(gen, N, K) * torch.exp(0.3 * _rand(gen, N, 1)) * torch.exp(0.3 * _rand(gen, 1, K)) / math.sqrt(K)
            s[name] = _pack(w, case["group"])
        s["add"] = _rand(gen, M, N).to(dt) if case["add"] else None
        s["out"] = torch.zeros(M, N, dtype=dt, device="cuda")
        if own:
            from paper_2411_09242_amd import w4
            for name in ("w", "gate") if case["gate"] else ("w",):
                s["own_" + name] = w4.W4(s[name], N, K, case["group"])
        return s
    B, T, H, Hk, D = (case[k] for k in ("batch", "tokens", "q_heads", "kv_heads", "dim"))
    counts = _counts(case)
    s["counts"] = counts
    s["count"] = torch.tensor(counts, dtype=torch.int32, device="cuda")
    # the real rows of a padded batch, which the host program knows
    s["rows"] = torch.tensor([b * T + i for b, t in enumerate(counts) for i in range(t)], device="cuda")
    s["q"], s["k"] = _rand(gen, B, T, H, D).to(dt), _rand(gen, B, T, Hk, D).to(dt)
    if case["kind"] == "rotary":
        # every sequence is somewhere else in its context
        far = torch.rand(B, generator=gen, device="cuda") * 0.7 + 0.3
        s["start"] = (far * case["far"]).to(torch.int32) - 1
        s["start"].clamp_(min=0)
        s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
        if own:
            from paper_2411_09242_amd import attention as A
            s["turns"] = A.Rotary(case["part"], interleaved=case["interleaved"], **_scaling(case))
        return s
    s["v"] = _rand(gen, B, T, Hk, D).to(dt)
    s["scale"] = 1.0 / math.sqrt(D)
    # memories of 20 to some thousand tokens, or gates that tokens set
    if case["fixed"]:
        s["decay"] = torch.log1p(-torch.exp2(-4.0 - 7.0 * torch.rand(Hk, generator=gen, device="cuda")))
    else:
        s["decay"] = -torch.nn.functional.softplus(_rand(gen, B, T, Hk) - 2.0 - 3.0 * torch.rand(Hk, generator=gen,
                                                                                               device="cuda"))
    s["state"] = 4.0 * _rand(gen, B, Hk, D, D)
    s["state_out"] = torch.zeros_like(s["state"])
    s["out"] = torch.zeros(B, T, H, D, dtype=dt, device="cuda")
    return s


# ------------------------------------------------------------ plain forms
def _frequencies(case):
    o, d = _scaling(case), case["part"]
    base = o["base"] * o["factor"] ** (d / (d - 2)) if o["scaling"] == "base" else o["base"]
    theta = base ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    if o["scaling"] == "linear":
        theta = theta / o["factor"]
    if o["scaling"] == "ramp":
        kept = ((o["length"] * theta / (2 * math.pi) - o["low"]) / (o["high"] - o["low"])).clamp(0, 1)
        theta = kept * theta + (1 - kept) * theta / o["factor"]
    return theta, o["amplitude"]


def _plain_rotary(x, c, s, d, interleaved):
    """x [rows, heads, dim] in fp32, c and s [rows, 1, d / 2]."""
    y = x.clone()
    a, b = (slice(0, d, 2), slice(1, d, 2)) if interleaved else (slice(0, d // 2), slice(d // 2, d))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def _plain_weights(packed, N, K, G):
    """The matrix [N, K] in fp32."""
    tiles, blocks = -(-N // 16), -(-K // 128)
    words = packed[:tiles * blocks * 1024].view(torch.int32).view(tiles, blocks, 4, 16, 4, 1)
    pairs = packed[tiles * blocks * 1024:].view(torch.float16).view(tiles, blocks, 16, 128 // G, 2).float()
    e = torch.arange(8, device=packed.device)
    n = ((words >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15).permute(0, 3, 1, 4, 2, 5)   # tile, row, block, word, place, e
    n = n.reshape(tiles, 16, blocks, 128 // G, G)
    p = pairs.transpose(1, 2)[..., None, :]
    return (p[..., 1] + p[..., 0] * (16 + n)).reshape(tiles * 16, blocks * 128)[:N, :K]


def _plain_linear(q, k, v, decay, state, count, scale):
    """q [B, T, H, D], k and v [B, T, Hk, D] and decay [B, T, Hk], in chunks."""
    B, T, H, D = q.shape
    Hk = k.shape[2]
    real = (torch.arange(T, device=q.device) < count[:, None])[:, :, None]
    q = q.view(B, T, Hk, H // Hk, D).permute(0, 2, 3, 1, 4)                # [B, Hk, group, T, D]
    k, v = (torch.where(real[..., None], x, torch.zeros_like(x)).transpose(1, 2) for x in (k, v))
    g = torch.where(real, decay.double(), torch.zeros_like(decay, dtype=torch.float64)).transpose(1, 2)
    out = torch.empty(B, Hk, H // Hk, T, D, dtype=torch.float32, device=q.device)
    S = state
    for at in range(0, T, CHUNK):
        to = min(at + CHUNK, T)
        qc, kc, vc, c = q[:, :, :, at:to], k[:, :, at:to], v[:, :, at:to], g[:, :, at:to].cumsum(-1)
        low = torch.ones(to - at, to - at, dtype=torch.bool, device=q.device).tril()
        weight = torch.exp((c[..., :, None] - c[..., None, :]).masked_fill(~low, -math.inf)).float()
        score = torch.matmul(qc, kc.transpose(-1, -2).contiguous()[:, :, None]) * weight[:, :, None]
        o = torch.matmul(score, vc[:, :, None]) + torch.exp(c).float()[:, :, None, :, None] * torch.matmul(qc, S[:, :, None])
        out[:, :, :, at:to] = scale * o
        left = torch.exp(c[..., -1:] - c).float()[..., None]
        S = torch.exp(c[..., -1]).float()[..., None, None] * S + torch.matmul((kc * left).transpose(-1, -2).contiguous(), vc)
    return out.permute(0, 3, 1, 2, 4).reshape(B, T, H, D), S


def run(state):
    case, s = state["case"], state
    if case["kind"] == "rotary":
        if own:
            from paper_2411_09242_amd import attention as A
            A.rotary(s["turns"], s["q"], s["k"], start=s["start"], count=s["count"], q_out=s["q_out"], k_out=s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        T, rows = case["tokens"], s["rows"]
        theta, amplitude = _frequencies(case)
        angle = (s["start"].double()[rows // T] + rows % T)[:, None] * theta
        c, sn = ((amplitude * f(angle)).float()[:, None] for f in (torch.cos, torch.sin))
        for name in ("q", "k"):
            y = _plain_rotary(s[name].flatten(0, 1)[rows].float(), c, sn, case["part"], case["interleaved"])
            s[name + "_out"].flatten(0, 1)[rows] = y.to(s["dt"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if case["kind"] == "w4":
        if own:
            from paper_2411_09242_amd import w4
            w4.w4_matmul(s["x"], s["own_w"], gate=s.get("own_gate"), add=s["add"], out=s["out"])
            return {"out": s["out"]}
        N, K, G = case["n"], case["k"], case["group"]
        x = s["x"].float()
        y = x @ _plain_weights(s["w"], N, K, G).T
        if case["gate"]:
            z = x @ _plain_weights(s["gate"], N, K, G).T
            y = y * (z / (1 + torch.exp(-z)))
        if case["add"]:
            y = y + s["add"].float()
        s["out"].copy_(y.to(s["dt"]))
        return {"out": s["out"]}
    if own:
        from paper_2411_09242_amd import attention as A
        A.linear_attention(s["q"], s["k"], s["v"], s["decay"], state=s["state"], count=s["count"], scale=s["scale"],
                           out=s["out"], state_out=s["state_out"])
        return {"out": s["out"], "state": s["state_out"]}
    B, T, Hk = case["batch"], case["tokens"], case["kv_heads"]
    o, last = _plain_linear(s["q"].float(), s["k"].float(), s["v"].float(), s["decay"].expand(B, T, Hk), s["state"],
                            s["count"], s["scale"])
    s["out"].flatten(0, 1)[s["rows"]] = o.to(s["dt"]).flatten(0, 1)[s["rows"]]
    s["state_out"].copy_(last)
    return {"out": s["out"], "state": s["state_out"]}


# ------------------------------------------------------- results in 64 bits
def _exact_rotary(case, s):
    o, d, T = _scaling(case), case["part"], case["tokens"]
    base, f = o["base"], o["factor"]
    if o["scaling"] == "base":
        base = base * math.pow(f, d / (d - 2))
    freq = []
    for i in range(d // 2):
        t = math.exp(-2.0 * i / d * math.log(base))
        if o["scaling"] == "linear":
            t /= f
        elif o["scaling"] == "ramp":
            turns = o["length"] * t / (2.0 * math.pi)
            share = min(1.0, max(0.0, (turns - o["low"]) / (o["high"] - o["low"])))
            t = t * (share + (1.0 - share) / f)
        freq.append(t)
    freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
    out = {}
    for name in ("q", "k"):
        y = s[name + "_out"].double()
        for b, n in enumerate(s["counts"]):
            p = int(s["start"][b]) + torch.arange(n, dtype=torch.float64, device="cuda")
            turn = torch.polar(torch.full((n, d // 2), o["amplitude"], dtype=torch.float64, device="cuda"),
                               torch.outer(p, freq))[:, None]
            x = s[name][b, :n].double()
            y[b, :n] = x
            head = x[..., :d].unflatten(-1, (-1, 2) if case["interleaved"] else (2, -1))
            pair = head if case["interleaved"] else head.transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            y[b, :n, :, :d] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        out[name] = y
    return out


def _exact_weights(packed, N, K, G):
    """Byte by byte: row r, channel c."""
    blocks = -(-K // 128)
    area = -(-N // 16) * blocks * 1024
    r = torch.arange(N, device="cuda")[:, None]
    c = torch.arange(K, device="cuda")[None]
    inside = c % 128
    tile = (r // 16) * blocks + c // 128
    word = tile * 256 + (16 * ((inside % 32) // 8) + r % 16) * 4 + inside // 32
    e = inside % 8
    nibble = (e // 2) + 4 * (e % 2)
    byte = packed[4 * word + nibble // 2].to(torch.int16)
    level = torch.where(nibble % 2 == 1, torch.div(byte, 16, rounding_mode="floor"), byte % 16).double()
    pair = packed[area:].view(torch.float16).double()
    at = 2 * (tile * (16 * (128 // G)) + (r % 16) * (128 // G) + inside // G)
    return pair[at + 1] + pair[at] * (level + 16.0)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_rotary(case, s)
    if case["kind"] == "w4":
        N, K, G = case["n"], case["k"], case["group"]
        y = torch.mm(s["x"].double(), _exact_weights(s["w"], N, K, G).t())
        if case["gate"]:
            z = torch.mm(s["x"].double(), _exact_weights(s["gate"], N, K, G).t())
            y = y * z * torch.sigmoid(z)
        return {"out": y if s["add"] is None else y + s["add"].double()}
    # token after token
    B, T, H, Hk, D = (case[k] for k in ("batch", "tokens", "q_heads", "kv_heads", "dim"))
    S = s["state"].double()
    out = s["out"].double()
    g = s["decay"].double() if s["decay"].dim() == 3 else s["decay"].double().view(1, 1, Hk).repeat(B, T, 1)
    for t in range(T):
        live = torch.tensor([t < n for n in s["counts"]], device="cuda")
        step = torch.exp(g[:, t])[:, :, None, None] * S + s["k"][:, t].double()[..., :, None] * s["v"][:, t].double()[..., None, :]
        S = step if all(t < n for n in s["counts"]) else torch.where(live[:, None, None, None], step, S)
        o = torch.matmul(s["q"][:, t].double().view(B, Hk, H // Hk, D), S).reshape(B, H, D) * s["scale"]
        out[:, t] = torch.where(live[:, None, None], o, out[:, t])
    return {"out": out, "state": S}
