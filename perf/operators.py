"""Timed cases of the operators at the output end of a language model: the matrix product that makes rows, and the
verification of drafted tokens against rows.

`cat_linear` is a layer's matrix product with what follows it (bias, activation, residual) in one kernel:
    Y = act(X W^T + b) + R.
`cat_verify_drafts` decides which of the tokens that a quantised network drafted its full-precision counterpart accepts, and
draws the token that follows, from given random numbers.  A sequence without drafts is plain sampling, which is how drafts are
drawn in the first place.

The plain forms below compute the same in elementary torch operations: the product in 32 bits, the verification in 64, because
its outputs are tokens and a sum of a hundred thousand probabilities decides between neighbours.  Inputs are made on the GPU from
the seed alone.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4, "none": 0}
LARGEST = float(torch.finfo(torch.float32).max)
NO_RESIDUAL = 2.0 ** -40      # a residual of less mass than this is what rounding left of none


def listed():
    return [
        # One token through a small classification head, logits in fp32 as cat_apply takes them: launch latency.
        dict(name="linear_head_1", op="linear", rows=1, cols=1000, inner=512, type="bf16", out="fp32", act="none", bias=True, residual=False),
        # One token through a wide layer: the time of reading the weights once.
        dict(name="linear_token_wide", op="linear", rows=1, cols=16384, inner=4096, type="bf16", out="bf16", act="silu", bias=False,
             residual=False),
        # Eight sequences decoding together.
        dict(name="linear_tokens_8", op="linear", rows=8, cols=8192, inner=2048, type="fp16", out="fp16", act="gelu", bias=True, residual=False),
        # A short prompt through a second MLP layer: long inner dimension, residual stream added.
        dict(name="linear_mlp_2k", op="linear", rows=2048, cols=2048, inner=8192, type="bf16", out="bf16", act="none", bias=True, residual=True),
        # The logits of a validation set: the rows that cat_apply corrects.
        dict(name="linear_logits_50k", op="linear", rows=50_000, cols=1000, inner=2048, type="bf16", out="fp32", act="none", bias=True,
             residual=False),
        # No size is a multiple of anything: rows that start on any even address.
        dict(name="linear_ragged", op="linear", rows=4999, cols=2047, inner=1001, type="fp16", out="fp16", act="gelu_tanh", bias=True,
             residual=True),
        # A long prompt through a first MLP layer: bound by the tensor cores.
        dict(name="linear_prompt_16k", op="linear", rows=16384, cols=16384, inner=4096, type="bf16", out="bf16", act="gelu", bias=True,
             residual=False),
        # One sequence, a small vocabulary, three drafts: launch latency.
        dict(name="verify_one", op="verify", seqs=1, drafts=3, vocab=1000, target="fp32", draft="fp32", noise=0.5),
        # A few sequences on a small server.
        dict(name="verify_8", op="verify", seqs=8, drafts=4, vocab=32000, target="bf16", draft="bf16", noise=0.5),
        # The draft's logits corrected by cat_apply (fp32 rows), the target's as the network gave them.
        dict(name="verify_corrected", op="verify", seqs=16, drafts=5, vocab=16384, target="bf16", draft="fp32", noise=0.3),
        # Many sequences sampling without drafts; rows that start on any even address.
        dict(name="verify_sampling", op="verify", seqs=256, drafts=0, vocab=50_001, target="fp16", draft="fp16", noise=0.5),
        # A full server: long drafts over a large vocabulary.
        dict(name="verify_64", op="verify", seqs=64, drafts=7, vocab=128_000, target="bf16", draft="bf16", noise=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        rows, cols, inner = _log_int(rng, 1, 16384), _log_int(rng, 64, 16384), _log_int(rng, 64, 8192)
        if rng.random() < 0.6:       # most layers are multiples of eight wide
            cols, inner = -(-cols // 8) * 8, -(-inner // 8) * 8
        rows = min(rows, max(1, 2 ** 40 // (cols * inner)))
        kind = rng.choice(["bf16", "fp16"])
        return dict(op="linear", rows=rows, cols=cols, inner=inner, type=kind, out=rng.choice([kind, "fp32"]),
                    act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), bias=rng.random() < 0.7, residual=rng.random() < 0.5)
    vocab, drafts = _log_int(rng, 500, 131_072), rng.randint(0, 8)
    seqs = min(_log_int(rng, 1, 256), max(1, 120_000_000 // ((2 * drafts + 1) * vocab)))
    kind = rng.choice(["bf16", "fp16", "fp32"])
    return dict(op="verify", seqs=seqs, drafts=drafts, vocab=vocab, target=kind, draft=rng.choice([kind, "fp32", "none"]),
                noise=rng.choice([0.2, 0.5, 1.0]))


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "linear":
        kind, out = TYPES[case["type"]], TYPES[case["out"]]
        m, n, k = case["rows"], case["cols"], case["inner"]
        # activations with a few large channels, weights of a trained layer's scale
        x = torch.randn((m, k), generator=g, device=DEV)
        x *= 1 + 4 * (torch.rand((k,), generator=g, device=DEV) < 0.01)
        w = torch.randn((n, k), generator=g, device=DEV) * k ** -0.5
        state = dict(op="linear", act=case["act"], out=out, x=x.to(kind), w=w.to(kind), bias=None, residual=None)
        if case["bias"]:
            state["bias"] = (0.5 * torch.randn((n,), generator=g, device=DEV)).to(kind)
        if case["residual"]:
            state["residual"] = torch.randn((m, n), generator=g, device=DEV).to(out)
        return state
    b, s, v = case["seqs"], case["drafts"], case["vocab"]
    # logits whose probabilities fall off like a power of the rank, in an order of the vocabulary that differs from row to row
    base = -1.3 * torch.log(1 + v * torch.rand((b, s + 1, v), generator=g, device=DEV))
    target = base + 0.5 * torch.randn((b, s + 1, v), generator=g, device=DEV)
    target = (target - target.amax(-1, keepdim=True) + 20).to(TYPES[case["target"]])
    temperature = 0.6 + 0.6 * torch.rand((b,), generator=g, device=DEV)
    if b > 1:
        temperature[:: 8] = 0.0      # some sequences decode greedily
    if case["draft"] == "none":      # drafts from a lookup, without probabilities
        draft = None
        guess = target[:, :s].float()
    else:
        draft = (target[:, :s].float() + case["noise"] * torch.randn((b, s, v), generator=g, device=DEV)).to(TYPES[case["draft"]])
        guess = draft.float()
    gumbel = -torch.log(-torch.log(torch.rand((b, s, v), generator=g, device=DEV).clamp(1e-20, 1 - 1e-7)))
    tokens = (guess + temperature[:, None, None] * gumbel).argmax(-1).int()
    lengths = torch.randint(0, s + 1, (b,), generator=g, device=DEV, dtype=torch.int32)
    lengths = torch.where(torch.rand((b,), generator=g, device=DEV) < 0.75, torch.full_like(lengths, s), lengths)
    return dict(op="verify", target=target, draft=draft, tokens=tokens, lengths=lengths, temperature=temperature,
                u_accept=torch.rand((b, s), generator=g, device=DEV), u_sample=torch.rand((b,), generator=g, device=DEV))


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _linear(st):
    z = st["x"].float() @ st["w"].float().t()
    if st["bias"] is not None:
        z = z + st["bias"].float()
    z = _act(z, st["act"])
    if st["residual"] is not None:
        z = z + st["residual"].float()
    return z.to(st["out"])


def _probabilities(logits, temperature):
    """softmax(logits / T) in 64 bits; a row at T <= 0 has all its mass on its largest entry (the first of equals), one without a
    finite entry has none."""
    x = torch.where(torch.isnan(logits), -math.inf, logits.double()).clamp(max=LARGEST)
    top, at = x.max(-1, keepdim=True)
    t = temperature.double()[:, None, None].expand_as(top)
    warm = t > 0
    e = torch.exp((x - top.clamp(min=-LARGEST)) / torch.where(warm, t, torch.ones_like(t)))
    e = torch.where(warm, e, (torch.arange(x.shape[-1], device=x.device) == at).double()) * (top > -math.inf)
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, torch.ones_like(total))


def _verify(st):
    target, draft, tokens = st["target"], st["draft"], st["tokens"].long()
    b, s = tokens.shape
    v = target.shape[-1]
    p = _probabilities(target, st["temperature"])
    inside = (tokens >= 0) & (tokens < v)
    at = tokens.clamp(0, v - 1)[..., None]
    if draft is None:
        q = torch.zeros((b, s, v), dtype=torch.float64, device=p.device).scatter_(2, at, inside[..., None].double())
    else:
        q = _probabilities(draft, st["temperature"])
    px, qx = p[:, :s].gather(2, at)[..., 0] * inside, q.gather(2, at)[..., 0] * inside
    steps = torch.arange(s, device=p.device)
    length = st["lengths"].long().clamp(max=s)
    accept = (st["u_accept"].double() * qx < px) & (steps < length[:, None])
    kept = accept.long().cumprod(1).sum(1)
    row = torch.arange(b, device=p.device)
    last = p[row, kept]
    if s:
        left = (last - q[row, kept.clamp(max=s - 1)]).clamp(min=0)
        refused = (kept < length) & (left.sum(-1) >= NO_RESIDUAL)
        last = torch.where(refused[:, None], left, last)
    mass = last.sum(-1)
    beyond = last.cumsum(-1) > (st["u_sample"].double() * mass)[:, None]
    drawn = torch.where(mass > 0, beyond.long().argmax(-1), torch.full_like(kept, -1))
    slots = torch.arange(s + 1, device=p.device)
    out = torch.cat([tokens, drawn[:, None]], 1)
    out = torch.where(slots < kept[:, None], out, torch.where(slots == kept[:, None], drawn[:, None], torch.full_like(out, -1)))
    return {"tokens": out.int(), "accepted": kept.int()}


def run(state):
    if own:
        from paper_2509_26277_b200 import binding as B
    if state["op"] == "linear":
        if own:
            return B.cat_linear(state["x"], state["w"], bias=state["bias"], residual=state["residual"], activation=state["act"],
                                out_dtype=state["out"])
        return _linear(state)
    if own:
        tokens, accepted = B.cat_verify_drafts(state["target"], state["draft"], state["tokens"], state["u_accept"], state["u_sample"],
                                               draft_lengths=state["lengths"], temperature=state["temperature"])
        return {"tokens": tokens, "accepted": accepted}
    return _verify(state)


def exact(case, seed):
    """The definitions in 64 bits, sequence by sequence for the verification."""
    st = prepare(case, seed)
    if st["op"] == "linear":
        x, w = st["x"].double(), st["w"].double()
        y = torch.empty((x.shape[0], w.shape[0]), dtype=torch.float64, device=DEV)
        for i in range(0, x.shape[0], 4096):
            z = torch.einsum("mk,nk->mn", x[i:i + 4096], w)
            z = z if st["bias"] is None else z + st["bias"].double()
            if st["act"] == "relu":
                z = z * (z > 0)
            elif st["act"] == "gelu":
                z = 0.5 * z * torch.erfc(-z / math.sqrt(2))
            elif st["act"] == "gelu_tanh":
                z = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
            elif st["act"] == "silu":
                z = z * torch.sigmoid(z)
            y[i:i + 4096] = z if st["residual"] is None else z + st["residual"][i:i + 4096].double()
        return y
    b, s = st["tokens"].shape
    v = st["target"].shape[-1]
    tokens, kept = torch.full((b, s + 1), -1, dtype=torch.int32), torch.zeros((b,), dtype=torch.int32)

    def masses(row, t):
        x = row.double()
        if t <= 0:
            one = torch.zeros_like(x)
            one[int((x == x.max()).nonzero()[0])] = 1
            return one
        return torch.softmax(x / t, -1)

    for i in range(b):
        t, length, j = float(st["temperature"][i]), int(st["lengths"][i]), 0
        mass = masses(st["target"][i, 0], t)
        while j < length:
            x = int(st["tokens"][i, j])
            if st["draft"] is None:
                other = torch.zeros_like(mass)
                other[x] = 1
            else:
                other = masses(st["draft"][i, j], t)
            if not float(st["u_accept"][i, j]) * float(other[x]) < float(mass[x]):
                left = (mass - other).clamp(min=0)
                mass = left if float(left.sum()) >= NO_RESIDUAL else mass
                break
            tokens[i, j] = x
            j += 1
            mass = masses(st["target"][i, j], t)
        kept[i] = j
        rising = mass.cumsum(-1)
        tokens[i, j] = min(v - 1, int((rising <= float(st["u_sample"][i]) * float(rising[-1])).sum()))
    return {"tokens": tokens, "accepted": kept}


def work(case):
    if case["op"] == "linear":
        m, n, k = case["rows"], case["cols"], case["inner"]
        small, out = BYTES[case["type"]], BYTES[case["out"]]
        return {"bytes": small * (m * k + n * k + (n if case["bias"] else 0)) + out * m * n * (2 if case["residual"] else 1),
                "flops": 2 * m * n * k}
    # Every row once.  What lies behind a refused draft need not be read, and greedy sequences need no draft rows: a call may
    # take less.
    b, s, v = case["seqs"], case["drafts"], case["vocab"]
    rows = b * ((s + 1) * BYTES[case["target"]] + s * BYTES[case["draft"]])
    return {"bytes": rows * v + 4 * b * (3 * s + 5), "flops": 6 * b * (2 * s + 1) * v}
