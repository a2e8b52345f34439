"""The operators around the token mixer that the library is timed and checked on.

Every case is one user-level call of ``paper_2606_01294_gb300.ops``: the embedding lookup and its gradient,
the gated group norm after the mixer's read and its gradient, the clipped policy loss with its gradient (or
the token log-probabilities alone), and the AdamW update of many tensors with states in 32 or 8 bits.
``run`` computes them either in a plain form of elementary torch operations in 32 bits, or, where ``own`` is
true, through the library.  Sizes are those of the repository's workloads (a 2048-wide layer of 16 heads of
128, T = 4096, decode batch 256), with generic vocabularies, and the ranges around them.
"""
import math
import random

import torch

own = False

BF16, FP32 = "bf16", "fp32"
DTYPE = {BF16: torch.bfloat16, FP32: torch.float32}
SIZE = {BF16: 2, FP32: 4}

#: Values that share a scale in the 8-bit optimizer state, and the largest finite e4m3 value.
BLOCK = 256
LR, BETAS, EPS, DECAY, STEP = 3e-4, (0.9, 0.95), 1e-8, 0.1, 1000
CLIP, KL, TEMPERATURE = (0.2, 0.25), 0.05, 0.9


def listed():
    return [
        # The input of one decode step of a full serving batch: 256 rows of the table, latency.
        dict(name="embed_decode_b256", op="embed", tokens=256, vocab=32000, width=2048, dtype=BF16),
        # The input of a batch of 4K prompts.
        dict(name="embed_prefill_4k", op="embed", tokens=8 * 4096, vocab=32000, width=2048, dtype=BF16),
        # A training step's gradient of the table: the token frequencies of text (Zipf), fp32 gradient.
        dict(name="embed_grad_4k", op="embed_grad", tokens=4 * 4096, vocab=32000, width=2048, dtype=BF16,
             grad_dtype=FP32, padding=False),
        # The mixer's output of one decode step, normalised per head and gated: latency.
        dict(name="norm_decode_b256", op="norm", tokens=256, heads=16, d=128, dtype=BF16, gate=True, act="silu",
             centered=True),
        # The same over a batch of 4K prompts.
        dict(name="norm_prefill_4k", op="norm", tokens=8 * 4096, heads=16, d=128, dtype=BF16, gate=True, act="silu",
             centered=True),
        # Its gradients (input, gate, weight, bias) in a training step at 4K.
        dict(name="norm_bwd_4k", op="norm_bwd", tokens=4 * 4096, heads=16, d=128, dtype=BF16, gate=True, act="silu",
             centered=True),
        # The log-probabilities of one short answer's tokens under a policy kept in fp32.
        dict(name="logp_short_fp32", op="logp", tokens=77, vocab=32000, dtype=FP32, masked=0),
        # The policy loss and its gradient over the answers of a batch; a quarter of the tokens are prompt.
        dict(name="policy_8k", op="policy", tokens=8192, vocab=32000, dtype=BF16, masked=2048),
        # A large vocabulary of odd size: rows that start on no 16-byte boundary.
        dict(name="policy_wide_odd", op="policy", tokens=1500, vocab=128001, dtype=BF16, masked=100),
        # The small tensors of one layer (norm weights, biases, gate projections): latency.
        dict(name="adamw_small_fp32", op="adamw", layers=1, width=0, dtype=FP32, grad_dtype=FP32, bits=32,
             master=False),
        # Four layers' tensors with everything in fp32.
        dict(name="adamw_fp32", op="adamw", layers=4, width=2048, dtype=FP32, grad_dtype=FP32, bits=32, master=False),
        # Twelve layers of bf16 weights with fp32 masters and 8-bit states.
        dict(name="adamw_8bit_master", op="adamw", layers=12, width=2048, dtype=BF16, grad_dtype=BF16, bits=8,
             master=True),
    ]


#: Bytes of the largest listed case of each operator: a drawn one moves no more.
MOST = {"embed": 265e6, "embed_grad": 325e6, "norm": 400e6, "norm_bwd": 335e6, "policy": 900e6, "logp": 450e6}


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_bwd", "norm_bwd", "policy", "policy", "logp",
                     "adamw", "adamw"])
    dtype = rng.choice([BF16, BF16, FP32])
    size = SIZE[dtype]
    if op in ("embed", "embed_grad"):
        width = rng.choice([64, 256, 500, 768, 1024, 1001, 2048, 4096])
        if op == "embed":
            tokens = _log_int(rng, 1, min(65536, int(MOST[op] / (2 * width * size + 8))))
            return dict(op=op, tokens=tokens, vocab=_log_int(rng, 1000, 100000), width=width, dtype=dtype)
        grad_dtype = rng.choice([dtype, FP32])
        vocab = _log_int(rng, 300, min(200000, int(0.8 * MOST[op] / (width * SIZE[grad_dtype]))))
        left = MOST[op] - vocab * width * SIZE[grad_dtype]
        tokens = _log_int(rng, 1, min(65536, int(left / (width * size + 8))))
        return dict(op=op, tokens=tokens, vocab=vocab, width=width, dtype=dtype, grad_dtype=grad_dtype,
                    padding=rng.random() < 0.4)
    if op in ("norm", "norm_bwd"):
        heads, d = rng.choice([(2, 64), (4, 128), (8, 128), (16, 128), (16, 64), (12, 96), (5, 33), (1, 2048), (4, 500)])
        gate = rng.random() < 0.7
        units = (2 + gate) + (2 * (op == "norm_bwd") if gate else (op == "norm_bwd"))
        tokens = _log_int(rng, 1, int(MOST[op] / (units * heads * d * size)) if heads > 1 else 20000)
        return dict(op=op, tokens=min(tokens, int(MOST[op] / (units * heads * d * size))), heads=heads, d=d,
                    dtype=dtype, gate=gate, act=rng.choice(["silu", "silu", "sigmoid", "none"]),
                    centered=rng.random() < 0.6)
    if op in ("policy", "logp"):
        vocab = _log_int(rng, 500, 260000)
        tokens = _log_int(rng, 1, max(1, min(8192, int(MOST[op] / (vocab * size * (2 if op == "policy" else 1))))))
        return dict(op=op, tokens=tokens, vocab=vocab, dtype=dtype, masked=rng.choice([0, tokens // 4, tokens // 2]))
    dtype, grad_dtype, bits, master = rng.choice([(FP32, FP32, 32, False), (FP32, FP32, 8, False), (FP32, BF16, 32, False),
                                                  (BF16, BF16, 32, True), (BF16, BF16, 8, True),
                                                  (BF16, BF16, 8, False), (BF16, FP32, 8, True)])
    return dict(op=op, layers=_log_int(rng, 1, 4), width=rng.choice([0, 256, 500, 1024, 2048]), dtype=dtype,
                grad_dtype=grad_dtype, bits=bits, master=master)


def _shapes(case):
    """The tensors of ``layers`` layers: projections of queries, keys, values, output gate and output, the per-head gate
    and decay, the norm's weight and bias.  ``width`` 0: only the small ones, of a 2048-wide layer."""
    wide, heads = case["width"] or 2048, max(1, (case["width"] or 2048) // 128)
    small = [(heads, wide), (heads,), (heads, 129), (wide,), (wide,), (wide - 7,), (3,)]
    large = [(wide, wide)] * 5 if case["width"] else []
    return (large + small) * case["layers"]


def _numel(shape):
    return math.prod(shape)


def _flat(case):
    """(offset, elements) of each tensor in the flat buffers that hold them, a multiple of BLOCK apart; the rest is zero."""
    at, places = 0, []
    for shape in _shapes(case):
        places.append((at, _numel(shape)))
        at += -(-_numel(shape) // BLOCK) * BLOCK
    return places, at


def _views(case, flat):
    places, _ = _flat(case)
    return [flat[a:a + n].view(s) for (a, n), s in zip(places, _shapes(case))]


def _prepare_adamw(case, gen):
    places, total = _flat(case)
    held = torch.zeros(total, device="cuda")
    [held[a:a + k].fill_(1) for a, k in places]
    n = lambda scale: torch.randn(total, device="cuda", generator=gen) * held * scale  # noqa: E731
    w = n(0.02)
    # gradients whose size differs from block to block by orders of magnitude, as between layers and rows
    spread = torch.exp(1.5 * torch.randn(total // BLOCK, 1, device="cuda", generator=gen))
    grad = (n(1e-3).view(-1, BLOCK) * spread).view(-1)
    m, v = n(3e-4).view(-1, BLOCK) * spread, (n(1e-3).view(-1, BLOCK) * spread).square()
    s = {"p": w.to(DTYPE[case["dtype"]]), "grad": grad.to(DTYPE[case["grad_dtype"]]),
         "master": w if case["master"] else None, "scale": None,
         "clip": torch.full((1,), 0.7, device="cuda")}
    if case["bits"] == 8:
        root = v.sqrt()
        top = torch.stack([m.abs().amax(1), root.amax(1)], 1)
        s["scale"] = torch.exp2(torch.ceil(torch.log2(top / 448)))
        s["m"] = (m / s["scale"][:, :1]).to(torch.float8_e4m3fn).view(-1)
        s["v"] = ((root / s["scale"][:, 1:]).clamp_min(2.0 ** -9) * held.view(-1, BLOCK)).to(torch.float8_e4m3fn).view(-1)
    else:
        s["m"], s["v"] = m.reshape(-1), v.reshape(-1)
    return s


def _prepare_policy(case, gen):
    N, V = case["tokens"], case["vocab"]
    r = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    logits = (2.5 * r(N, V)).to(DTYPE[case["dtype"]])
    # actions drawn from the policy itself
    logp = torch.log_softmax(logits.float() / TEMPERATURE, -1)
    noise = -torch.log(torch.empty(N, V, device="cuda").exponential_(generator=gen))
    actions = noise.add_(logp).argmax(-1)
    logp = logp.gather(1, actions[:, None])[:, 0]
    # most tokens are near the policy that drew them, an eighth have moved far from it
    moved = 0.5 * torch.sign(r(N)) * (torch.rand(N, device="cuda", generator=gen) < 0.125)
    weights = torch.full((N,), 1.0 / max(1, N - case["masked"]), device="cuda")
    weights[torch.randperm(N, device="cuda", generator=gen)[:case["masked"]]] = 0
    return {"logits": logits, "actions": actions, "old": logp + 0.04 * r(N) + moved, "ref": logp + 0.2 * r(N),
            "adv": 0.4 + r(N), "weights": weights}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, r = case["op"], lambda *shape: torch.randn(*shape, device="cuda", generator=gen)
    if op == "adamw":
        s = _prepare_adamw(case, gen)
    elif op in ("policy", "logp"):
        s = _prepare_policy(case, gen)
    elif op in ("embed", "embed_grad"):
        N, V, D = case["tokens"], case["vocab"], case["width"]
        # ranks of a Zipf distribution
        ids = (torch.exp(torch.rand(N, device="cuda", generator=gen) * math.log(V)).long() - 1).clamp_(0, V - 1)
        s = {"ids": ids, "padding": 0 if case.get("padding") else None}
        if op == "embed":
            s["table"] = (0.02 * r(V, D)).to(DTYPE[case["dtype"]])
        else:
            s["dout"] = r(N, D).to(DTYPE[case["dtype"]])
    else:
        N, C, dtype = case["tokens"], case["heads"] * case["d"], DTYPE[case["dtype"]]
        s = {"x": (0.5 * r(N, C) + 0.1).to(dtype), "weight": (1 + 0.1 * r(C)).to(dtype), "bias": (0.1 * r(C)).to(dtype),
             "gate": r(N, C).to(dtype) if case["gate"] else None}
        if op == "norm_bwd":
            s["dout"] = r(N, C).to(dtype)
    return {"case": dict(case), **s}


# ---------------------------------------------------------------- the plain forms


def _act(name, u):
    """act(u) and its derivative."""
    if name == "none":
        return u, torch.ones_like(u)
    sig = 1 / (1 + torch.exp(-u))
    if name == "sigmoid":
        return sig, sig * (1 - sig)
    return u * sig, sig * (1 + u * (1 - sig))


def _normed(s, dtype):
    c = s["case"]
    x = s["x"].to(dtype).view(c["tokens"], c["heads"], c["d"])
    dev = x - x.mean(-1, keepdim=True) if c["centered"] else x
    rstd = 1 / torch.sqrt(dev.square().mean(-1, keepdim=True) + 1e-5)
    w, b = (s[n].to(dtype).view(c["heads"], c["d"]) for n in ("weight", "bias"))
    return dev * rstd, rstd, w, b


def _plain_norm(s):
    c = s["case"]
    xh, _, w, b = _normed(s, torch.float32)
    u = xh * w + b
    y = u * _act(c["act"], s["gate"].float().view_as(u))[0] if c["gate"] else _act(c["act"], u)[0]
    return {"y": y.view_as(s["x"]).to(s["x"].dtype)}


def _plain_norm_bwd(s):
    c = s["case"]
    xh, rstd, w, b = _normed(s, torch.float32)
    u, dy = xh * w + b, s["dout"].float().view_as(xh)
    out = {}
    if c["gate"]:
        a, da = _act(c["act"], s["gate"].float().view_as(u))
        out["dgate"] = (dy * u * da).view_as(s["x"]).to(s["x"].dtype)
        du = dy * a
    else:
        du = dy * _act(c["act"], u)[1]
    dxh = du * w
    dx = dxh - xh * (dxh * xh).mean(-1, keepdim=True)
    if c["centered"]:
        dx = dx - dxh.mean(-1, keepdim=True)
    out["dx"] = (dx * rstd).view_as(s["x"]).to(s["x"].dtype)
    out["dweight"] = (du * xh).sum(0).view(-1).to(s["weight"].dtype)
    out["dbias"] = du.sum(0).view(-1).to(s["bias"].dtype)
    return out


def _plain_embed_grad(s):
    c = s["case"]
    dout = s["dout"].float() * c["width"] ** 0.5
    if s["padding"] is not None:
        dout = dout * (s["ids"] != s["padding"])[:, None]
    table = torch.zeros(c["vocab"], c["width"], device="cuda").index_add_(0, s["ids"], dout)
    return {"dtable": table.to(DTYPE[c["grad_dtype"]])}


def _plain_logp(s):
    """Shifted exponentials of the rows, their sums and the actions' log-probabilities."""
    z = s["logits"].float() / TEMPERATURE
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    return e, total, (z.gather(1, s["actions"][:, None]) - top - torch.log(total))[:, 0]


def _plain_policy(s):
    e, total, logp = _plain_logp(s)
    w, adv = s["weights"], s["adv"]
    ratio = torch.exp(logp - s["old"])
    free, held = ratio * adv, ratio.clamp(1 - CLIP[0], 1 + CLIP[1]) * adv
    d = s["ref"] - logp
    loss = (w * (KL * (torch.exp(d) - d - 1) - torch.minimum(free, held))).sum()
    slope = w * (KL * (1 - torch.exp(d)) - torch.where(free <= held, free, 0)) / TEMPERATURE
    grad = e * (-slope[:, None] / total)
    grad = grad.scatter_add(1, s["actions"][:, None], slope[:, None])
    return {"loss": loss, "logp": torch.where(w != 0, logp, 0), "dlogits": grad.to(s["logits"].dtype)}


def _encode(x, scale, turn):
    """e4m3 values of x >= 0 over a power-of-two scale, rounded up where the fraction between two neighbours passes
    the threshold ``turn`` (20 bits)."""
    y = x / scale
    bits = (((y.view(torch.int32) + turn) >> 20) - (120 << 3)).clamp(max=127)  # 127: NaN
    small = (y * 512 * 1048576).floor().int().add(turn) >> 20
    return torch.where(y < 2.0 ** -6, small, bits)


def _scale_of(x):
    """The smallest power of two 2^e >= 2^-100 with x <= 448 * 2^e for the finite x of each block."""
    top = torch.where(torch.isfinite(x), x, 0).amax(1, keepdim=True).view(torch.int32)
    return ((((top + 0x1FFFFF) >> 23) - 8).clamp(min=27) << 23).view(torch.float32)


def _plain_adamw(s):
    """All tensors at once: what lies between them in the flat buffers is zero and stays zero."""
    c = s["case"]
    g = s["grad"].float() * s["clip"]
    m, v = s["m"], s["v"]
    if c["bits"] == 8:
        m = (m.float().view(-1, BLOCK) * s["scale"][:, :1]).view(-1)
        v = (v.float().view(-1, BLOCK) * s["scale"][:, 1:]).square().view(-1)
    m = m * BETAS[0] + g * (1 - BETAS[0])
    v = v * BETAS[1] + g * g * (1 - BETAS[1])
    root = torch.sqrt(v)
    p = (s["master"] if c["master"] else s["p"]).float()
    rate = LR / (1 - BETAS[0] ** STEP)
    p = p * (1 - LR * DECAY) - rate * m / (root / (1 - BETAS[1] ** STEP) ** 0.5 + EPS)
    if c["master"]:
        s["master"].copy_(p)
    s["p"].copy_(p)
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return _adamw_state(s)
    # an element's index in its own tensor
    starts, lengths = torch.tensor([(at, -(-n // BLOCK)) for at, n in _flat(c)[0]], device="cuda").T
    index = torch.arange(m.numel(), device="cuda").view(-1, BLOCK) - starts.repeat_interleave(lengths)[:, None]
    turn = (((index * 0x6A09E667 + STEP * 0x9E3779B1) & 0xFFFFFFFF) >> 12).int()
    m, root = m.view(-1, BLOCK), root.view(-1, BLOCK)
    sm, sv = _scale_of(m.abs()), _scale_of(root)
    code = _encode(m.abs(), sm, 0xFFFFF - turn) + 128 * (m < 0)
    level = torch.where(root > 0, _encode(root, sv, turn).clamp(min=1), 0)
    s["m"].copy_(code.view(-1).to(torch.uint8).view(torch.float8_e4m3fn))
    s["v"].copy_(level.view(-1).to(torch.uint8).view(torch.float8_e4m3fn))
    s["scale"].copy_(torch.cat([sm, sv], 1))
    return _adamw_state(s)


def _adamw_state(s):
    return {k: s[k] for k in ("p", "m", "v", "scale", "master") if s[k] is not None}


# ---------------------------------------------------------------- the library's calls


def _own(s):
    from paper_2606_01294_gb300 import ops
    c = s["case"]
    if c["op"] == "embed":
        return {"out": ops.embed(s["table"], s["ids"], scale=c["width"] ** 0.5)}
    if c["op"] == "embed_grad":
        return {"dtable": ops.embed_grad(s["dout"], s["ids"], c["vocab"], scale=c["width"] ** 0.5,
                                         padding_id=s["padding"], dtype=DTYPE[c["grad_dtype"]])}
    if c["op"] in ("norm", "norm_bwd"):
        how = dict(groups=c["heads"], activation=c["act"], centered=c["centered"], eps=1e-5)
        if c["op"] == "norm":
            return {"y": ops.group_norm(s["x"], s["weight"], s["bias"], s["gate"], **how)}
        return ops.group_norm_bwd(s["x"], s["weight"], s["bias"], s["gate"], s["dout"], **how)
    if c["op"] == "logp":
        return {"logp": ops.token_logp(s["logits"], s["actions"], temperature=TEMPERATURE)}
    if c["op"] == "policy":
        return ops.policy_loss(s["logits"], s["actions"], s["old"], s["adv"], ref_logp=s["ref"], weights=s["weights"],
                               clip=CLIP, kl_coef=KL, temperature=TEMPERATURE)
    places, _ = _flat(c)
    blocks = lambda x: [x[a // BLOCK:a // BLOCK + -(-n // BLOCK)] for a, n in places]  # noqa: E731
    state = ops.AdamWState(m=_views(c, s["m"]), v=_views(c, s["v"]),
                           scale=blocks(s["scale"]) if c["bits"] == 8 else None,
                           master=_views(c, s["master"]) if c["master"] else None)
    ops.adamw_step(_views(c, s["p"]), _views(c, s["grad"]), state, STEP, lr=LR, betas=BETAS, eps=EPS,
                   weight_decay=DECAY, grad_scale=s["clip"])
    return _adamw_state(s)


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    if op == "embed":
        return {"out": (s["table"][s["ids"]].float() * s["case"]["width"] ** 0.5).to(s["table"].dtype)}
    if op == "logp":
        return {"logp": _plain_logp(s)[2]}
    return {"embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "policy": _plain_policy,
            "adamw": _plain_adamw}[op](s)


def work(case):
    """Bytes: every input and output once (rows of zero weight are written, not read).  Flops: the elementary operations
    of the formulas, an exponential or a root as one."""
    op, size = case["op"], SIZE[case["dtype"]]
    if op == "embed":
        n = case["tokens"] * case["width"]
        rows = min(case["tokens"], case["vocab"])
        return {"bytes": n * size + rows * case["width"] * size + 8 * case["tokens"], "flops": n}
    if op == "embed_grad":
        n = case["tokens"] * case["width"]
        return {"bytes": n * size + 8 * case["tokens"] + case["vocab"] * case["width"] * SIZE[case["grad_dtype"]],
                "flops": 2 * n}
    if op in ("norm", "norm_bwd"):
        C = case["heads"] * case["d"]
        n = case["tokens"] * C
        if op == "norm":
            return {"bytes": (2 + case["gate"]) * n * size + 2 * C * size, "flops": 12 * n}
        return {"bytes": (3 + 2 * case["gate"]) * n * size + 4 * C * size, "flops": 30 * n}
    if op in ("policy", "logp"):
        N, V = case["tokens"], case["vocab"]
        if op == "logp":
            return {"bytes": N * V * size + 12 * N, "flops": 4 * N * V}
        return {"bytes": (2 * N - case["masked"]) * V * size + 28 * N, "flops": 7 * (N - case["masked"]) * V}
    n = sum(_numel(s) for s in _shapes(case))
    each = 2 * (4 + 4) if case["bits"] == 32 else 2 * (1 + 1) + 16 / BLOCK
    each += SIZE[case["grad_dtype"]] + (8 + size if case["master"] else 2 * size)
    return {"bytes": n * each, "flops": 16 * n}


# ---------------------------------------------------------------- 64 bits, from the definitions


def _exact_norm(s):
    c = s["case"]
    N, H, d = c["tokens"], c["heads"], c["d"]
    x, w, b = s["x"].double().view(N, H, d), s["weight"].double().view(H, d), s["bias"].double().view(H, d)
    gate = s["gate"].double().view(N, H, d) if c["gate"] else None
    with torch.enable_grad():  # the gradients by reverse mode over the definition
        leaves = [t.clone().requires_grad_() for t in (x, w, b)] + ([gate.clone().requires_grad_()] if c["gate"] else [])
        X, W, B = leaves[:3]
        mean = X.mean(-1, keepdim=True) if c["centered"] else 0.0
        var = ((X - mean) ** 2).mean(-1, keepdim=True)
        u = (X - mean) / (var + 1e-5) ** 0.5 * W + B
        t = leaves[3] if c["gate"] else u
        a = {"none": lambda t: t, "sigmoid": torch.sigmoid, "silu": lambda t: t * torch.sigmoid(t)}[c["act"]](t)
        y = u * a if c["gate"] else a
        if c["op"] == "norm":
            return {"y": y.detach().view_as(s["x"])}
        grads = torch.autograd.grad(y, leaves, s["dout"].double().view(N, H, d), allow_unused=True)
    out = {"dx": grads[0].view_as(s["x"]), "dweight": grads[1].reshape(-1), "dbias": grads[2].reshape(-1)}
    if c["gate"]:
        out["dgate"] = grads[3].view_as(s["x"])
    return out


def _exact_policy(s):
    logps, grads, losses = [], [], []
    for a in range(0, s["case"]["tokens"], 512):
        cut = slice(a, a + 512)
        z = s["logits"][cut].double() / TEMPERATURE
        act, w = s["actions"][cut], s["weights"][cut].double()
        lse = torch.logsumexp(z, -1, keepdim=True)
        lp = z.gather(1, act[:, None])[:, 0] - lse[:, 0]
        if s["case"]["op"] == "logp":
            logps.append(lp)
            continue
        lp.requires_grad_()
        with torch.enable_grad():
            ratio = (lp - s["old"][cut].double()).exp()
            adv = s["adv"][cut].double()
            gain = torch.minimum(ratio * adv, torch.clamp(ratio, 1 - CLIP[0], 1 + CLIP[1]) * adv)
            d = s["ref"][cut].double() - lp
            loss = (w * (KL * (d.exp() - d - 1) - gain)).sum()
        slope = torch.autograd.grad(loss, lp)[0][:, None] / TEMPERATURE
        grad = -slope * (z - lse).exp()
        grad.scatter_add_(1, act[:, None], slope)
        grads.append(grad)
        losses.append(loss.detach())
        logps.append(torch.where(w != 0, lp.detach(), 0))
    if s["case"]["op"] == "logp":
        return {"logp": torch.cat(logps)}
    return {"loss": torch.stack(losses).sum(), "logp": torch.cat(logps), "dlogits": torch.cat(grads)}


def _exact_quantise(x, turn):
    """x >= 0 in blocks to (e4m3 value, scale): neighbours in e4m3 by their spacing, up where the fraction passes 1 - turn."""
    top = x.amax(1, keepdim=True)
    e = torch.clamp(torch.ceil(torch.log2(torch.where(top > 0, top, 2.0 ** -150) / 448)), min=-100)
    y = x / 2.0 ** e
    gap = 2.0 ** (torch.clamp(torch.floor(torch.log2(torch.where(y > 0, y, 2.0 ** -60))), min=-6) - 3)
    return torch.floor(y / gap + turn) * gap, 2.0 ** e


def _exact_adamw(s):
    c, out = s["case"], {k: v.double().clone() for k, v in _adamw_state(s).items()}
    for at, n in _flat(c)[0]:
        cut = slice(at, at + n)
        rows = slice(at // BLOCK, at // BLOCK + -(-n // BLOCK))
        g = s["grad"][cut].double() * s["clip"].double()
        m, v = out["m"][cut], out["v"][cut]
        if c["bits"] == 8:
            per = out["scale"][rows].repeat_interleave(BLOCK, 0)[:n]
            m, v = m * per[:, 0], (v * per[:, 1]) ** 2
        m, v = BETAS[0] * m + (1 - BETAS[0]) * g, BETAS[1] * v + (1 - BETAS[1]) * g ** 2
        p = out["master" if c["master"] else "p"][cut]
        p = p - LR * DECAY * p - LR * (m / (1 - BETAS[0] ** STEP)) / ((v / (1 - BETAS[1] ** STEP)) ** 0.5 + EPS)
        out["p"][cut] = p
        if c["master"]:
            out["master"][cut] = p
        if c["bits"] == 32:
            out["m"][cut], out["v"][cut] = m, v
            continue
        i = torch.arange(-(-n // BLOCK) * BLOCK, device="cuda", dtype=torch.int64)
        word = (i * 1779033703 + STEP * 2654435761) % (1 << 32)
        turn = ((word // 4096).double() / (1 << 20)).view(-1, BLOCK)
        full = lambda x: torch.cat([x, x.new_zeros(-n % BLOCK)]).view(-1, BLOCK)  # noqa: E731
        size, sm = _exact_quantise(full(m.abs()), (1 - 2.0 ** -20) - turn)
        root, sv = _exact_quantise(full(v ** 0.5), turn)
        root = torch.where(full(v) > 0, root.clamp(min=2.0 ** -9), 0.0)
        out["m"][cut] = (size * torch.sign(full(m))).view(-1)[:n]
        out["v"][cut] = root.view(-1)[:n]
        out["scale"][rows] = torch.cat([sm, sv], 1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    if case["op"] in ("policy", "logp"):
        return _exact_policy(s)
    if case["op"] in ("norm", "norm_bwd"):
        return _exact_norm(s)
    scale = math.sqrt(case["width"])
    if case["op"] == "embed":
        return {"out": s["table"].double().index_select(0, s["ids"]) * scale}
    order = torch.argsort(s["ids"], stable=True)
    ids, rows = s["ids"][order], s["dout"].double()[order] * scale
    if s["padding"] is not None:
        rows = torch.where((ids == s["padding"])[:, None], 0.0, rows)
    # the sums of equal tokens as differences of a running sum over the sorted ones
    run_sum = torch.cat([rows.new_zeros(1, rows.shape[1]), rows.cumsum(0)])
    edges = torch.searchsorted(ids, torch.arange(case["vocab"] + 1, device="cuda"))
    return {"dtable": run_sum[edges[1:]] - run_sum[edges[:-1]]}
