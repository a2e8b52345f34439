"""Rotary positions and linear attention with a decay for each head: what the library is timed and checked on.

Every case is one user-level call of ``paper_2606_01294_gb300.ops``: the rotation of a layer's queries and keys by
their positions and its gradient; the attention over prompts (a batch, one long document, a new turn on a carried
state, packed sequences), its gradients, and its step for one token of every sequence of a batch.  ``run`` computes them
either in a plain form of elementary torch operations in 32 bits, or, where ``own`` is true, through the library.  Sizes
are those of the repository's workloads (a 2048-wide layer of 16 heads of 128, T = 4096 and 20480, decode batch 256, 64
packed prompts) and the ranges around them.
"""
import math
import random

import torch

own = False

BF16, FP32 = "bf16", "fp32"
DTYPE = {BF16: torch.bfloat16, FP32: torch.float32}
SIZE = {BF16: 2, FP32: 4}

#: Tokens of a chunk in the plain form of the attention.
CHUNK = 64


def listed():
    return [
        # One token for a full serving batch at positions all over a long context (YaRN): latency.
        dict(name="rotary_decode_b256", op="rotary", B=256, T=1, heads=16, kv=16, d=128, part=128, dtype=BF16,
             interleaved=False, scaling="yarn", factor=8.0),
        # The queries and keys of a batch of 4K prompts, slices of one projection.
        dict(name="rotary_prefill_4k", op="rotary", B=8, T=4096, heads=16, kv=16, d=128, part=128, dtype=BF16,
             interleaved=False, scaling="none", factor=1.0),
        # The gradient of an odd number of tokens, pairs side by side in half of each head, fewer key heads.
        dict(name="rotary_bwd_part", op="rotary_bwd", B=3, T=3001, heads=12, kv=4, d=128, part=64, dtype=BF16,
             interleaved=True, scaling="linear", factor=4.0),
        # A new turn of one conversation on its carried state: short, ragged.
        dict(name="attend_turn", op="attend", B=1, T=1000, heads=16, kv=16, d=128, dtype=BF16, resumed=True, packed=False),
        # A batch of 4K prompts.
        dict(name="attend_4k", op="attend", B=8, T=4096, heads=16, kv=16, d=128, dtype=BF16, resumed=False, packed=False),
        # One long document: few heads, many chunks.
        dict(name="attend_20k", op="attend", B=1, T=20480, heads=16, kv=16, d=128, dtype=BF16, resumed=False,
             packed=False),
        # A serving mix: 64 prompts of very different lengths in one call.
        dict(name="attend_packed_64", op="attend", B=64, T=4000, heads=16, kv=16, d=128, dtype=BF16, resumed=True,
             packed=True),
        # Full-precision evaluation of a small model.
        dict(name="attend_fp32", op="attend", B=4, T=777, heads=4, kv=4, d=64, dtype=FP32, resumed=False, packed=False),
        # One token for two interactive sessions: latency.
        dict(name="step_b2", op="step", B=2, heads=16, kv=16, d=128, dtype=BF16, pool=0),
        # One token for a full serving batch, whose states lie anywhere in a pool.
        dict(name="step_b256", op="step", B=256, heads=16, kv=16, d=128, dtype=BF16, pool=300),
        # The gradients of a training step at 4K.
        dict(name="attend_bwd_4k", op="attend_bwd", B=4, T=4096, heads=16, kv=16, d=128, dtype=BF16, resumed=False,
             packed=False),
        # Heads of 64 that share keys and values in fours, odd length, a state before and a gradient after the batch's end.
        dict(name="attend_bwd_shared", op="attend_bwd", B=3, T=1501, heads=16, kv=4, d=64, dtype=BF16, resumed=True,
             packed=False),
    ]


#: Elements of q (of the states for a step) of the largest listed case of each operator: a drawn one has no more.
MOST = {"rotary": 8 * 4096 * 2048, "rotary_bwd": 8 * 4096 * 2048, "attend": 8 * 4096 * 2048, "attend_bwd": 4 * 4096 * 2048,
        "step": 256 * 16 * 128 * 128}


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "rotary", "rotary_bwd", "attend", "attend", "attend", "attend", "attend_bwd", "attend_bwd",
                     "attend_bwd", "step", "step"])
    heads = rng.choice([2, 4, 8, 12, 16, 16])
    kv = rng.choice([heads, heads, heads // 2, 1])
    if op in ("rotary", "rotary_bwd"):
        d, part = rng.choice([(64, 64), (128, 128), (128, 64), (128, 32), (96, 96), (80, 20), (256, 256), (66, 66)])
        T = _log_int(rng, 1, 20000)
        scaling, factor = rng.choice([("none", 1.0), ("linear", 4.0), ("ntk", 4.0), ("yarn", 16.0), ("yarn", 4.0)])
        return dict(op=op, B=_log_int(rng, 1, max(1, min(256, MOST[op] // (T * heads * d)))), T=T, heads=heads, kv=kv, d=d,
                    part=part, dtype=rng.choice([BF16, BF16, FP32]), interleaved=rng.random() < 0.5, scaling=scaling,
                    factor=factor)
    d = rng.choice([64, 128, 128])
    if op == "step":
        B = _log_int(rng, 1, min(256, MOST[op] // (heads * d * d)))
        return dict(op=op, B=B, heads=heads, kv=kv, d=d, dtype=rng.choice([BF16, BF16, FP32]),
                    pool=rng.choice([0, B, B + rng.randrange(40)]))
    dtype = rng.choice([BF16, BF16, BF16, FP32])
    most = MOST[op] // (heads * d) // (4 if dtype == FP32 else 1)
    if rng.random() < 0.3:
        B, T = _log_int(rng, 2, 64), _log_int(rng, 30, 4000)
        return dict(op=op, B=min(B, max(1, most // T)), T=T, heads=heads, kv=kv, d=d, dtype=dtype,
                    resumed=rng.random() < 0.5, packed=True)
    T = _log_int(rng, 2, 20480 if op == "attend" else 8192)
    return dict(op=op, B=_log_int(rng, 1, max(1, min(32, most // T))), T=min(T, most), heads=heads, kv=kv, d=d,
                dtype=dtype, resumed=rng.random() < 0.5, packed=False)


def _lengths(case):
    """Tokens of each sequence: all T, or, packed, spread from none to T with the longest first or last."""
    B, T = case["B"], case["T"]
    if not case["packed"]:
        return [T] * B
    rng = random.Random(1000003 * B + T)
    spread = [int(round(math.exp(rng.uniform(math.log(T / 40 + 1), math.log(T + 1))))) - 1 for _ in range(B - 1)]
    return [T] + spread if B % 2 else spread + [T]


def _frequencies(case):
    """Radians a position for each pair, and the factor of cosine and sine, in 64 bits: a base of 10000, with positions
    divided by a factor (linear), the base raised so that the slowest pair is stretched by it (ntk), or the slow pairs
    stretched and the fast ones kept (yarn; a context of 4096 before)."""
    R, factor = case["part"], case["factor"]
    base = 10000.0 * (factor ** (R / (R - 2)) if case["scaling"] == "ntk" else 1.0)
    f = base ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "yarn":
        pair = lambda turns: R * math.log(4096 / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), R - 1)
        keep = 1 - ((torch.arange(R // 2, dtype=torch.float64) - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    r = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    op, H, K, d, dtype = case["op"], case["heads"], case["kv"], case["d"], DTYPE[case["dtype"]]
    s = {"case": dict(case)}
    if op in ("rotary", "rotary_bwd"):
        B, T = case["B"], case["T"]
        # q, k (and v, which the rotation leaves) of one projection
        qkv = r(B, T, (H + 2 * K) * d).to(dtype)
        s["q"] = qkv[..., :H * d].unflatten(-1, (H, d))
        s["k"] = qkv[..., H * d:(H + K) * d].unflatten(-1, (K, d))
        begin = torch.randint(0, 30000, (B, 1), device="cuda", generator=gen)
        s["positions"] = begin + torch.arange(T, device="cuda")
        freqs, s["amplitude"] = _frequencies(case)
        s["freqs"] = freqs.cuda()
        return s
    # from about 32 tokens of memory to 4096
    bits = 5 + 7 * torch.arange(H, dtype=torch.float64) / max(1, H - 1)
    s["log_decay"] = torch.log1p(-torch.exp2(-bits)).float().cuda()
    if op == "step":
        B = case["B"]
        s["q"], s["k"], s["v"] = (r(B, n, d).to(dtype) for n in (H, K, K))
        s["state"] = 3 * r(case["pool"] or B, H, d, d)
        s["slots"] = torch.randperm(case["pool"], device="cuda", generator=gen)[:B].int() if case["pool"] else None
        return s
    lengths = _lengths(case)
    rows = (1, sum(lengths)) if case["packed"] else (case["B"], case["T"])
    qkv = r(*rows, (H + 2 * K) * d).to(dtype)
    s["q"], s["k"], s["v"] = (t.unflatten(-1, (-1, d)) for t in qkv.split([H * d, K * d, K * d], -1))
    s["cu"] = torch.tensor([0] + lengths, device="cuda").cumsum(0) if case["packed"] else None
    s["state"] = 3 * r(case["B"], H, d, d) if case["resumed"] else None
    if op == "attend_bwd":
        s["dout"] = r(*rows, H, d).to(dtype)
        s["dstate"] = 0.1 * r(case["B"], H, d, d) if case["resumed"] else None
    return s


# ---------------------------------------------------------------- the plain forms


def _plain_rotary(s):
    c = s["case"]
    R = c["part"]
    angle = s["positions"][..., None, None].double() * s["freqs"]
    cos, sin = ((s["amplitude"] * f(angle)).float() for f in (torch.cos, torch.sin))
    if c["op"] == "rotary_bwd":
        sin = -sin

    def rotate(x):
        y = x.float()
        if c["interleaved"]:
            a, b = y[..., 0:R:2], y[..., 1:R:2]
            turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = y[..., :R // 2], y[..., R // 2:R]
            turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        return torch.cat([turned, y[..., R:]], -1).to(x.dtype)

    return {"q": rotate(s["q"]), "k": rotate(s["k"])}


def _padded(s):
    """How the sequences' tokens lie in a batch of whole chunks: (row of each place, whether it holds one, lengths)."""
    c = s["case"]
    most = -(-c["T"] // CHUNK) * CHUNK
    at = torch.arange(most, device="cuda")
    if s["cu"] is None:
        n = torch.full((c["B"], 1), c["T"], device="cuda")
        begin = torch.arange(c["B"], device="cuda")[:, None] * c["T"]
    else:
        n, begin = (s["cu"][1:] - s["cu"][:-1])[:, None], s["cu"][:-1, None]
    held = at < n
    return torch.where(held, begin + at, 0), held, n


def _spread(s, x, rows, held):
    """[B, heads, time, d] in 32 bits, zero where no token is, each head with its own copy."""
    y = x.flatten(0, 1)[rows].float() * held[..., None, None]
    return y.transpose(1, 2).repeat_interleave(s["case"]["heads"] // x.shape[2], 1)


def _gather(x, s, held):
    """The tokens of [B, heads, time, d] as they lay."""
    y = x.transpose(1, 2)
    return (y[:, :s["case"]["T"]] if s["cu"] is None else y[held][None]).contiguous()


def _power(s, n):
    """decay ** n for each head, n >= 0: [..., heads, time] from [..., 1, time]."""
    return torch.exp(s["log_decay"].double()[:, None] * n.double()).float()


def _within(s):
    """decay ** (i - j) of a chunk for j <= i, and 0."""
    i = torch.arange(CHUNK, device="cuda")
    gap = i[:, None] - i
    return _power(s, gap.clamp(min=0).view(1, -1)).view(-1, CHUNK, CHUNK) * (gap >= 0)


def _between(s, chunks):
    """decay ** (CHUNK (r - s - 1)) for chunks s < r, and 0."""
    r = torch.arange(chunks, device="cuda")
    gap = r[:, None] - r - 1
    return _power(s, (CHUNK * gap.clamp(min=0)).view(1, -1)).view(-1, chunks, chunks) * (gap >= 0)


def _chunks(x):
    return x.unflatten(2, (-1, CHUNK))


def _attend(s, q, k, v, reverse):
    """sum over j <= i (or j >= i) of decay ** |i - j| (q_i . k_j) v_j."""
    i = torch.arange(CHUNK, device="cuda")[None]
    q, k, v = _chunks(q), _chunks(k), _chunks(v)
    mask, chain = _within(s), _between(s, q.shape[2])
    far, near = (_power(s, CHUNK - 1 - i), _power(s, i + 1))
    if reverse:
        mask, chain, far, near = mask.transpose(1, 2), chain.transpose(1, 2), near, far
    own_part = ((q @ k.transpose(-1, -2)) * mask[:, None]) @ v
    steps = (k * far[:, None, :, None]).transpose(-1, -2) @ v
    states = (chain @ steps.flatten(3)).view(steps.shape)
    return (own_part + (q * near[:, None, :, None]) @ states).flatten(2, 3)


def _plain_attend(s):
    c = s["case"]
    rows, held, n = _padded(s)
    q, k, v = (_spread(s, s[name], rows, held) for name in ("q", "k", "v"))
    scale = c["d"] ** -0.5
    at = torch.arange(q.shape[2], device="cuda")
    left = (_power(s, (n - 1 - at).clamp(min=0)[:, None]) * held[:, None])[..., None]  # to the sequence's end
    since = _power(s, at[None] + 1)[..., None]
    S0 = s["state"]
    whole = _power(s, n[:, None])[..., None]
    if c["op"] == "attend":
        o = _attend(s, q, k, v, False)
        state = (k * left).transpose(-1, -2) @ v
        if S0 is not None:
            o = o + (q * since) @ S0
            state = state + whole * S0
        return {"o": _gather(o * scale, s, held).to(s["q"].dtype), "state": state}
    do = _spread(s, s["dout"], rows, held) * scale
    dq = _attend(s, do, v, k, False)
    dk = _attend(s, v, do, q, True)
    dv = _attend(s, k, q, do, True)
    out = {}
    if S0 is not None:
        dq = dq + (do * since) @ S0.transpose(-1, -2)
        dk = dk + (v * left) @ s["dstate"].transpose(-1, -2)
        dv = dv + (k * left) @ s["dstate"]
        out["dstate"] = (q * since).transpose(-1, -2) @ do + whole * s["dstate"]
    shared = lambda x, name: x.unflatten(1, (s[name].shape[2], -1)).sum(2)  # noqa: E731
    for name, x in (("q", dq), ("k", dk), ("v", dv)):
        out["d" + name] = _gather(shared(x, name), s, held).to(s[name].dtype)
    return out


def _plain_step(s):
    c = s["case"]
    H = c["heads"]
    q, k, v = (s[n].float().repeat_interleave(H // s[n].shape[1], 1) for n in ("q", "k", "v"))
    state = s["state"] if s["slots"] is None else s["state"][s["slots"]]
    state = state * torch.exp(s["log_decay"])[:, None, None] + k[..., None] * v[:, :, None]
    o = (q[..., None] * state).sum(2) * c["d"] ** -0.5
    if s["slots"] is None:
        s["state"].copy_(state)
    else:
        s["state"][s["slots"]] = state
    return {"o": o.to(s["q"].dtype), "state": s["state"]}


# ---------------------------------------------------------------- the library's calls


def _own(s):
    from paper_2606_01294_gb300 import ops
    c = s["case"]
    if c["op"] in ("rotary", "rotary_bwd"):
        call = ops.rotary if c["op"] == "rotary" else ops.rotary_bwd
        q, k = call(s["q"], s["k"], s["positions"], s["freqs"], interleaved=c["interleaved"], amplitude=s["amplitude"])
        return {"q": q, "k": k}
    if c["op"] == "step":
        o = ops.decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], slots=s["slots"])
        return {"o": o, "state": s["state"]}
    if c["op"] == "attend":
        o, state = ops.decay_attention(s["q"], s["k"], s["v"], s["log_decay"], state=s["state"], cu_seqlens=s["cu"])
        return {"o": o, "state": state}
    g = ops.decay_attention_bwd(s["q"], s["k"], s["v"], s["log_decay"], s["dout"], state=s["state"],
                                dfinal_state=s["dstate"], cu_seqlens=s["cu"])
    return {name: g[name] for name in (("dstate",) if s["state"] is not None else ()) + ("dq", "dk", "dv")}


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    if op in ("rotary", "rotary_bwd"):
        return _plain_rotary(s)
    return _plain_step(s) if op == "step" else _plain_attend(s)


def work(case):
    """Bytes: every input and output once.  Flops: of the attention's chunkwise form with chunks of 128 (within a chunk
    j <= i alone), a product and a sum as two."""
    op, size, H, K, d = case["op"], SIZE[case["dtype"]], case["heads"], case["kv"], case["d"]
    if op in ("rotary", "rotary_bwd"):
        n = case["B"] * case["T"]
        return {"bytes": n * (2 * (H + K) * d * size + 8) + 4 * case["part"], "flops": 3 * n * (H + K) * case["part"]}
    if op == "step":
        B = case["B"]
        return {"bytes": B * (8 * H * d * d + (2 * H + 2 * K) * d * size), "flops": 5 * B * H * d * d}
    n = sum(_lengths(case))
    states = 4 * case["B"] * H * d * d
    if op == "attend":
        return {"bytes": n * (2 * H + 2 * K) * d * size + states * (1 + case["resumed"]),
                "flops": n * H * (2 * 128 * d + 4 * d * d)}
    return {"bytes": n * (3 * H + 4 * K) * d * size + 3 * states * case["resumed"],
            "flops": 3 * n * H * (2 * 128 * d + 4 * d * d)}


# ---------------------------------------------------------------- 64 bits, from the definitions


def _exact_rotary(s):
    c = s["case"]
    R = c["part"]
    turn = s["positions"].double()[..., None] * s["freqs"] * (-1.0 if c["op"] == "rotary_bwd" else 1.0)
    turn = torch.polar(torch.full_like(turn, s["amplitude"]), turn)[:, :, None]
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        pairs = x[..., :R].unflatten(-1, (R // 2, 2)) if c["interleaved"] else x[..., :R].unflatten(-1, (2, R // 2)).mT
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        x[..., :R] = y.flatten(-2) if c["interleaved"] else y.mT.flatten(-2)
        out[name] = x
    return out


def _exact_step(s):
    slots = torch.arange(s["case"]["B"], device="cuda") if s["slots"] is None else s["slots"].long()
    state, H = s["state"].double(), s["case"]["heads"]
    gamma = s["log_decay"].double().exp()
    q, k, v = (s[n].double()[:, torch.arange(H, device="cuda") * s[n].shape[1] // H] for n in ("q", "k", "v"))
    new = torch.einsum("h,bhkv->bhkv", gamma, state[slots]) + torch.einsum("bhk,bhv->bhkv", k, v)
    state[slots] = new
    return {"o": torch.einsum("bhk,bhkv->bhv", q, new) / math.sqrt(s["case"]["d"]), "state": state}


def _exact_attend(s):
    """Token by token: the state's recurrence and its reverse, over all sequences at once."""
    c = s["case"]
    B, T, H, d = c["B"], c["T"], c["heads"], c["d"]
    lengths = _lengths(c)
    starts = [sum(lengths[:b]) for b in range(B)]
    gamma = s["log_decay"].double().exp()[:, None, None]
    n = torch.tensor(lengths, device="cuda")
    first = torch.tensor(starts, device="cuda")
    flat = {x: s[x].flatten(0, 1) for x in ("q", "k", "v", "dout") if x in s}
    scale = 1 / math.sqrt(d)

    def at(name, t):  # token t of every sequence that has one (else of row 0), each head's own
        x = flat[name][torch.where(t < n, first + t, 0)].double()
        return x[:, torch.arange(H, device="cuda") * x.shape[1] // H]

    S = torch.zeros(B, H, d, d, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
    outs = torch.zeros(T, B, H, d, dtype=torch.float64, device="cuda")
    for t in range(T):
        new = torch.addcmul(gamma * S, at("k", t)[..., None], at("v", t)[:, :, None])
        S = torch.where((t < n)[:, None, None, None], new, S) if c["packed"] else new
        if c["op"] == "attend":
            outs[t] = torch.einsum("bhk,bhkv->bhv", at("q", t), S) * scale
        else:
            outs[t] = torch.einsum("bhkv,bhv->bhk", S, at("dout", t)) * scale

    def rows(x):  # [T, B, H, d] as the tokens lie
        x = x.transpose(0, 1)
        return x if not c["packed"] else torch.cat([x[b, :lengths[b]] for b in range(B)])[None]

    if c["op"] == "attend":
        return {"o": rows(outs), "state": S}
    dS = torch.zeros_like(S) if s["dstate"] is None else s["dstate"].double()
    dk, dv = torch.zeros_like(outs), torch.zeros_like(outs)
    for t in reversed(range(T)):
        now = torch.addcmul(dS, at("q", t)[..., None] * scale, at("dout", t)[:, :, None])
        dk[t] = torch.einsum("bhkv,bhv->bhk", now, at("v", t))
        dv[t] = torch.einsum("bhkv,bhk->bhv", now, at("k", t))
        now = gamma * now
        dS = torch.where((t < n)[:, None, None, None], now, dS) if c["packed"] else now
    out = {"dstate": dS} if s["state"] is not None else {}
    for name, x in (("q", outs), ("k", dk), ("v", dv)):
        x = rows(x)
        heads = s[name].shape[2]
        out["d" + name] = sum(x[:, :, j::H // heads] for j in range(H // heads)) if heads < H else x
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("rotary", "rotary_bwd"):
        return _exact_rotary(s)
    return _exact_step(s) if case["op"] == "step" else _exact_attend(s)
