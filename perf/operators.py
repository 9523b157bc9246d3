"""What the speed of the operators between two collectives is measured on: AdamW over the shards that a reduce-scatter
leaves and an all-gather sends out, the residual's addition with the root-mean-square norm between the two collectives of
sequence parallelism, and the router's balance loss with the counts that an all-to-all(v) goes by.

Sizes come from the traffic that the repository's workloads are shaped like: GPT-6.7B (hidden 4096, ffn 16384, sequence
2048, bf16, 8 ranks) and DeepSeek-V2-Lite (hidden 2048, 64 experts, top-6 routing, 4096 tokens a rank).
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
_ES = {"bf16": 2, "fp32": 4}
_BLOCK = 128                    # elements that share a scale where something is held in 8 bits
_TOP = 448.0                    # the largest e4m3 value
_TINY = 2.0 ** -100             # a block whose largest magnitude is less is held as zeros
_BETAS, _EPS, _DECAY, _LR = (0.9, 0.95), 1e-8, 0.1, 3e-4
_NORM_EPS = 1e-6
_ALPHA = {"expert_weight": 0.003, "rank_weight": 0.05, "traffic_weight": 0.02}


def listed():
    return [
        # Norm weights and biases of a few layers that one rank keeps whole: the smallest step, all latency.
        {"name": "adamw_norms", "op": "adamw", "layout": "even", "tensors": 8, "total": 8 * 4096, "sizes": 1,
         "param": "fp32", "grad": "fp32", "bits": 32, "copy": False, "scaled": False},
        # One rank's shard of a transformer block (12 h^2 weights over 8 ranks, with its norms and biases): fp32 weights, the
        # reduce-scatter's bf16 gradients, clipped, and the bf16 copies that the all-gather sends out.
        {"name": "adamw_shard", "op": "adamw", "layout": "block", "tensors": 14, "total": 0, "sizes": 4096,
         "param": "fp32", "grad": "bf16", "bits": 32, "copy": True, "scaled": True},
        # The same with states in 8 bits.
        {"name": "adamw_shard_8bit", "op": "adamw", "layout": "block", "tensors": 14, "total": 0, "sizes": 4096,
         "param": "fp32", "grad": "bf16", "bits": 8, "copy": True, "scaled": True},
        # Many uneven tensors back to back in flat buffers, bf16 weights, no copies: fine-tuning with little memory.
        {"name": "adamw_many_8bit", "op": "adamw", "layout": "ragged", "tensors": 150, "total": 9_000_000, "sizes": 7,
         "param": "bf16", "grad": "bf16", "bits": 8, "copy": False, "scaled": False},
        # One token being generated.
        {"name": "rmsnorm_token", "op": "rmsnorm", "rows": 1, "hidden": 4096, "dtype": "bf16", "weight": "bf16",
         "residual": True, "quantize": False},
        # A rank's tokens between the reduce-scatter and the all-gather of sequence parallelism.
        {"name": "rmsnorm_shard", "op": "rmsnorm", "rows": 8192, "hidden": 4096, "dtype": "bf16", "weight": "bf16",
         "residual": True, "quantize": False},
        # The same for the smaller hidden size, the all-gather's payload in 8 bits.
        {"name": "rmsnorm_8bit", "op": "rmsnorm", "rows": 4096, "hidden": 2048, "dtype": "bf16", "weight": "fp32",
         "residual": True, "quantize": True},
        # A hidden size that divides by nothing, in fp32, without a residual.
        {"name": "rmsnorm_odd_fp32", "op": "rmsnorm", "rows": 1001, "hidden": 5003, "dtype": "fp32", "weight": "fp32",
         "residual": False, "quantize": False},
        # The training step's backward pass over eight sequences, the residual's gradient added.
        {"name": "rmsnorm_backward", "op": "rmsnorm_backward", "rows": 16384, "hidden": 4096, "dtype": "bf16",
         "weight": "bf16", "residual": True},
        # The router of one rank's small micro-batch, forward and backward.
        {"name": "balance_small", "op": "balance", "R": 1, "tokens": 512, "ragged": False, "experts": 64, "topk": 6,
         "ranks": 8, "dtype": "fp32", "index": "int64", "padding": 0.0, "backward": True},
        # The counts of the expert-parallel dispatch over eight ranks, and its loss.
        {"name": "balance_dispatch", "op": "balance", "R": 8, "tokens": 4096, "ragged": False, "experts": 64, "topk": 6,
         "ranks": 8, "dtype": "fp32", "index": "int64", "padding": 0.0, "backward": False},
        # A training step over padded batches of uneven length with many experts, forward and backward.
        {"name": "balance_train", "op": "balance", "R": 8, "tokens": 32768, "ragged": True, "experts": 256, "topk": 8,
         "ranks": 16, "dtype": "bf16", "index": "int32", "padding": 0.1, "backward": True},
    ]


def _log(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; half of them are round."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and n >= 512:
        n = n // 128 * 128
    return max(lo, min(hi, n))


def draw(rng):
    op = rng.choice(["adamw"] * 4 + ["rmsnorm"] * 4 + ["rmsnorm_backward"] * 2 + ["balance"] * 3)
    if op == "adamw":
        count = _log(rng, 1, 200)
        param = rng.choice(["fp32", "fp32", "bf16"])
        return {"op": op, "layout": rng.choice(["even", "ragged", "ragged"]), "tensors": count,
                "total": max(count, _log(rng, 2000, 20_000_000)), "sizes": rng.randrange(1 << 20), "param": param,
                "grad": rng.choice(["bf16", "fp32"]), "bits": rng.choice([8, 32]),
                "copy": param == "fp32" and rng.random() < 0.6, "scaled": rng.random() < 0.5}
    if op == "rmsnorm" or op == "rmsnorm_backward":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        hidden = _log(rng, 64, 20000)
        c = {"op": op, "rows": _log(rng, 1, max(1, 60_000_000 // (hidden * _ES[dtype] // 2))), "hidden": hidden,
             "dtype": dtype, "weight": rng.choice([dtype, "fp32"]), "residual": rng.random() < 0.7}
        if op == "rmsnorm":
            c["quantize"] = rng.random() < 0.4
        return c
    ranks = rng.choice([1, 2, 4, 8, 16])
    experts = max(4, ranks * rng.choice([1, 2, 3, 4, 8, 8, 12, 16, 20]))
    experts += -experts % ranks
    R, dtype = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice(["fp32", "bf16"])
    tokens = _log(rng, 1, min(100_000, 40_000_000 // (R * experts * _ES[dtype] // 2)))
    return {"op": op, "R": R, "tokens": tokens, "ragged": rng.random() < 0.5, "experts": experts,
            "topk": rng.randint(1, min(10, experts // 2)), "ranks": ranks, "dtype": dtype,
            "index": rng.choice(["int32", "int64"]), "padding": rng.choice([0.0, 0.15, 0.9]) if tokens > 100 else 0.0,
            "backward": rng.random() < 0.6}


# ---- sizes ---------------------------------------------------------------------


def _sizes(case):
    """Elements of each tensor of an AdamW step."""
    if case["layout"] == "block":
        # One rank's eighth of a transformer block: the weights of attention and of the feed-forward layer, their biases
        # and the two norms.
        h = case["sizes"]
        shares = [3 * h * h, h * h, 4 * h * h, 4 * h * h, 3 * h, h, 4 * h, h, h, h, h, h, 64, 8]
        return [-(-n // 8) for n in shares][: case["tensors"]]
    total, count = case["total"], case["tensors"]
    if case["layout"] == "even":
        return [total // count] * (count - 1) + [total - total // count * (count - 1)]
    rng = random.Random(case["sizes"])
    cuts = [math.exp(rng.uniform(0.0, 7.0)) for _ in range(count)]
    scale = total / sum(cuts)
    return [max(1, int(c * scale)) for c in cuts]


def _tokens(case):
    """Tokens of each rank's batch."""
    if not case["ragged"]:
        return [case["tokens"]] * case["R"]
    rng = random.Random(case["tokens"] * 31 + case["R"])
    return [max(1, int(case["tokens"] * rng.uniform(0.3, 1.0))) for _ in range(case["R"])]


def _cut(flat, sizes):
    return list(torch.split(flat, sizes))


# ---- inputs ----------------------------------------------------------------------


def _to_blocks(x):
    """(blocks of 128 along the last axis, zeros behind the end, and its length)."""
    n = x.shape[-1]
    pad = -n % _BLOCK
    return torch.nn.functional.pad(x, (0, pad)).unflatten(-1, ((n + pad) // _BLOCK, _BLOCK)), n


def _quantize(x, floor):
    """(e4m3 values, fp32 scales) of x by blocks of 128 along its last axis; with `floor`, what is not zero is at least the
    smallest value that is not."""
    b, n = _to_blocks(x)
    top = b.abs().amax(-1)
    some = ~(top < _TINY)
    # Tensors over tensors: where one is a number torch multiplies by a reciprocal, which rounds twice.
    most = torch.full_like(top, _TOP)
    scale = torch.where(some, top / most, torch.zeros_like(top))
    q = b * torch.where(some, most / top, torch.zeros_like(top)).unsqueeze(-1)
    if floor:
        q = torch.where((q > 0) & (q < 2.0 ** -9), torch.full_like(q, 2.0 ** -9), q)
    return q.flatten(-2)[..., :n].to(torch.float8_e4m3fn).contiguous(), scale


def _dequantize(q, scale):
    b, n = _to_blocks(q.float())
    return (b * scale.unsqueeze(-1)).flatten(-2)[..., :n]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    if case["op"] == "adamw":
        sizes = _sizes(case)
        n = sum(sizes)
        # Gradients whose size differs from one tensor to the next and from one row of a weight to the next.
        level = torch.exp(1.5 * normal(n // 1000 + 1)).repeat_interleave(1000)[:n] * 1e-3
        grad = normal(n) * level
        s = {"sizes": sizes, "step": 10, "flat": {"param": (normal(n) * 0.02).to(_DT[case["param"]]),
                                                  "grad": grad.to(_DT[case["grad"]])}}
        m, v = normal(n) * level * 0.3, level.square() * (0.2 + torch.rand(n, generator=g, device="cuda"))
        v[torch.rand(n, generator=g, device="cuda") < 0.01] = 0.0      # rows that have had no gradient yet
        if case["bits"] == 8:
            pairs = [_quantize(x, False) for x in _cut(m, sizes)], [_quantize(x.sqrt(), True) for x in _cut(v, sizes)]
            for name, ps in zip(("m", "v"), pairs):
                s["flat"][name] = torch.cat([q.view(torch.uint8) for q, _ in ps]).view(torch.float8_e4m3fn)
                s["flat"][name + "_scale"] = torch.cat([x for _, x in ps])
        else:
            s["flat"] |= {"m": m, "v": v}
        if case["copy"]:
            s["flat"]["copy"] = torch.empty(n, dtype=torch.bfloat16, device="cuda")
        blocks = [-(-k // _BLOCK) for k in sizes]
        s |= {name: _cut(x, blocks if "scale" in name else sizes) for name, x in s["flat"].items()}
        s["scale"] = torch.rand(1, generator=g, device="cuda") * 0.5 + 0.5 if case["scaled"] else None
        return s
    if case["op"] in ("rmsnorm", "rmsnorm_backward"):
        rows, hidden, dt = case["rows"], case["hidden"], _DT[case["dtype"]]
        # Activations with a few channels far larger than the others.
        loud = torch.where(torch.rand(hidden, generator=g, device="cuda") < 0.01, 20.0, 1.0)
        s = {"x": (normal(rows, hidden) * loud).to(dt),
             "weight": (1.0 + 0.2 * normal(hidden)).to(_DT[case["weight"]]),
             "residual": (normal(rows, hidden) * 2.0).to(dt) if case["residual"] else None}
        if case["op"] == "rmsnorm_backward":
            s["grad"] = (normal(rows, hidden) * 1e-3).to(dt)
        else:
            s["quantize"] = case["quantize"]
        return s
    tokens = _tokens(case)
    E, k = case["experts"], case["topk"]
    # A router that prefers some experts.
    liked = normal(E) * 0.7
    logits = [normal(t, E) * 1.5 + liked for t in tokens]
    experts = [x.topk(k, dim=-1).indices.to(torch.int64 if case["index"] == "int64" else torch.int32) for x in logits]
    if case["padding"]:
        for e in experts:
            t = e.shape[0]
            e[torch.rand(t, generator=g, device="cuda") < case["padding"]] = -1      # padding tokens
            e[torch.rand(t, generator=g, device="cuda") < 0.05, -1] = -1             # a choice past the capacity
    return {"logits": [x.to(_DT[case["dtype"]]) for x in logits], "experts": experts,
            "grad": torch.rand(case["R"], generator=g, device="cuda") + 0.5 if case["backward"] else None,
            "ranks": case["ranks"]}


# ---- the plain forms -----------------------------------------------------------------


def _plain_adamw(s, i, eight):
    b1, b2 = _BETAS
    p, grad = s["param"][i].float(), s["grad"][i].float()
    m = _dequantize(s["m"][i], s["m_scale"][i]) if eight else s["m"][i]
    v = _dequantize(s["v"][i], s["v_scale"][i]).square() if eight else s["v"][i]
    if s["scale"] is not None:
        grad = grad * s["scale"]
    m = m * b1 + grad * (1 - b1)
    v = v * b2 + grad * grad * (1 - b2)
    root = v.sqrt()
    p = p * (1 - _LR * _DECAY) - (_LR / (1 - b1 ** s["step"])) * m / (root / math.sqrt(1 - b2 ** s["step"]) + _EPS)
    s["param"][i].copy_(p)
    if "copy" in s:
        s["copy"][i].copy_(p)
    if eight:
        for name, x, floor in (("m", m, False), ("v", root, True)):
            q, scale = _quantize(x, floor)
            s[name][i].view(torch.uint8).copy_(q.view(torch.uint8))
            s[name + "_scale"][i].copy_(scale)
    else:
        s["m"][i].copy_(m)
        s["v"][i].copy_(v)


def _plain_rmsnorm(s, quantize):
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(h.dtype)
    x = h.float()
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _NORM_EPS) * s["weight"].float()
    out = _quantize(y, False) if quantize else y.to(h.dtype)
    return out if s["residual"] is None else (out, h)


def _plain_rmsnorm_backward(s):
    h, w, dy = s["x"].float(), s["weight"].float(), s["grad"].float()
    r = torch.rsqrt(h.square().mean(-1, keepdim=True) + _NORM_EPS)
    gy = dy * w
    dx = r * (gy - h * (r * r * (gy * h).mean(-1, keepdim=True)))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return dx.to(s["x"].dtype), (dy * h * r).sum(0)


def _plain_balance(logits, experts, grad, D):
    T, E = logits.shape
    k = experts.shape[1]
    index = experts.long()
    some = (index >= 0) & (index < E)
    valid = some.any(-1)
    live = valid.sum().clamp(min=1).double()
    counts = torch.zeros(E + 1, dtype=torch.int32, device=logits.device)
    where = torch.where(some, index, E).flatten()
    counts = counts.scatter_add_(0, where, torch.ones_like(where, dtype=torch.int32))[:E]
    hit = torch.zeros(T, D + 1, dtype=torch.bool, device=logits.device)
    sent = hit.scatter_(1, torch.where(some, index // (E // D), D), True)[:, :D].sum(0).to(torch.int32)
    f = counts.double() * E / (k * live)
    w = _ALPHA["expert_weight"] * f
    w = w + (_ALPHA["rank_weight"] * f.unflatten(0, (D, E // D)).mean(1)
             + _ALPHA["traffic_weight"] * sent.double() * D / (min(k, D) * live)).repeat_interleave(E // D)
    p = torch.where(valid.unsqueeze(-1), torch.softmax(logits.float(), -1), 0.0)
    loss = (w * p.sum(0) / live).sum().float()
    if grad is None:
        return loss, counts, sent
    # A balanced router's weights are nearly the same and its gradient lives on their differences, which are taken in 64
    # bits: as each row of p sums to one, a constant more or less in w changes nothing.
    c = (w - w.mean()).float()
    d = (grad / live.float()) * p * (c - (p * c).sum(-1, keepdim=True))
    return loss, counts, sent, d.to(logits.dtype)


def run(state):
    if "step" in state:
        eight = "m_scale" in state
        if own:
            import paper_2609_34334_amd as hoccl
            hoccl.adamw(state["param"], state["grad"], state["m"], state["v"], state.get("m_scale"), state.get("v_scale"),
                        copies=state.get("copy"), step=state["step"], lr=_LR, betas=_BETAS, eps=_EPS, weight_decay=_DECAY,
                        grad_scale=state["scale"])
        else:
            _ = [_plain_adamw(state, i, eight) for i in range(len(state["sizes"]))]
        return {name: x for name, x in state["flat"].items() if name != "grad"}
    if "experts" in state:
        grad = state["grad"]
        if own:
            import paper_2609_34334_amd as hoccl
            out = hoccl.balance_loss(state["logits"], state["experts"], state["ranks"], **_ALPHA)
            got = {"loss": out.loss, "expert_tokens": out.expert_tokens, "rank_tokens": out.rank_tokens}
            if grad is not None:
                got["grad"] = hoccl.balance_loss_backward(state["logits"], state["experts"], out.coef, grad)
            return got
        outs = [_plain_balance(x, e, None if grad is None else grad[i], state["ranks"])
                for i, (x, e) in enumerate(zip(state["logits"], state["experts"]))]
        cols = list(zip(*outs))
        got = {"loss": torch.stack(cols[0]), "expert_tokens": torch.stack(cols[1]), "rank_tokens": torch.stack(cols[2])}
        return got if grad is None else got | {"grad": list(cols[3])}
    if "grad" in state:
        if own:
            import paper_2609_34334_amd as hoccl
            return hoccl.rmsnorm_backward(state["grad"], state["x"], state["weight"], state["residual"], eps=_NORM_EPS)
        return _plain_rmsnorm_backward(state)
    quantize = state["quantize"]
    if own:
        import paper_2609_34334_amd as hoccl
        return hoccl.rmsnorm(state["x"], state["weight"], state["residual"], eps=_NORM_EPS, quantize=quantize)
    return _plain_rmsnorm(state, quantize)


# ---- what a pass cannot do without -----------------------------------------------------


def work(case):
    if case["op"] == "adamw":
        sizes = _sizes(case)
        n, blocks = sum(sizes), sum(-(-k // _BLOCK) for k in sizes)
        states = 16 * n if case["bits"] == 32 else 4 * n + 16 * blocks
        return {"bytes": 2 * _ES[case["param"]] * n + _ES[case["grad"]] * n + states + (2 * n if case["copy"] else 0),
                "flops": 20 * n}
    if case["op"] in ("rmsnorm", "rmsnorm_backward"):
        rows, hidden, es = case["rows"], case["hidden"], _ES[case["dtype"]]
        n = rows * hidden
        if case["op"] == "rmsnorm_backward":
            return {"bytes": (4 if case["residual"] else 3) * es * n + _ES[case["weight"]] * hidden + 4 * hidden,
                    "flops": 12 * n}
        out = n + 4 * rows * -(-hidden // _BLOCK) if case["quantize"] else es * n
        return {"bytes": (3 if case["residual"] else 1) * es * n + out + _ES[case["weight"]] * hidden, "flops": 6 * n}
    T, E = sum(_tokens(case)), case["experts"]
    index = T * case["topk"] * (8 if case["index"] == "int64" else 4)
    return {"bytes": T * E * _ES[case["dtype"]] * (2 if case["backward"] else 1) + index,
            "flops": T * E * (14 if case["backward"] else 6)}


# ---- the definitions in 64 bits ----------------------------------------------------------


def _shared(x):
    """Per element of the last axis, the scale of its block of 128 (largest magnitude over 448, 0 for next to nothing), and
    the scales."""
    n = x.shape[-1]
    starts = range(0, n, _BLOCK)
    if n % _BLOCK:
        x = torch.cat([x, x.new_zeros(*x.shape[:-1], -n % _BLOCK)], -1)
    top = x.reshape(*x.shape[:-1], len(starts), _BLOCK).abs().max(-1).values
    scale = torch.where(top < _TINY, 0.0, top / _TOP)
    return scale.repeat_interleave(_BLOCK, -1)[..., :n], scale


def _over(x, scale):
    return torch.where(scale > 0, x / torch.where(scale > 0, scale, 1.0), 0.0)


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "adamw":
        sizes = s["sizes"]
        eight = case["bits"] == 8

        def held(name):
            if not eight:
                return s["flat"][name].to(f64)
            return torch.cat([q.float().to(f64) * z.to(f64).repeat_interleave(_BLOCK)[:len(q)]
                              for q, z in zip(s[name], s[name + "_scale"])])

        (b1, b2), t = _BETAS, s["step"]
        g = s["flat"]["grad"].to(f64) * (1.0 if s["scale"] is None else s["scale"].to(f64))
        m = held("m").mul_(b1).add_(g, alpha=1 - b1)
        v = (held("v").square_() if eight else held("v")).mul_(b2).addcmul_(g, g, value=1 - b2)
        root = v.sqrt()
        update = (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + _EPS)
        p = s["flat"]["param"].to(f64)
        p = p - _LR * (update + _DECAY * p)
        got = {"param": p, "m": m, "v": v}
        if eight:
            for name, x in (("m", m), ("v", root)):
                shared = [_shared(y) for y in _cut(x, sizes)]
                q = _over(x, torch.cat([a for a, _ in shared]))
                got[name] = q if name == "m" else torch.where((q > 0) & (q < 2.0 ** -9), 2.0 ** -9, q)
                got[name + "_scale"] = torch.cat([b for _, b in shared])
        return got | {"copy": p} if case["copy"] else got
    if case["op"] == "rmsnorm":
        h = s["x"].to(f64)
        if s["residual"] is not None:
            # bf16 and fp32 sums of two such values are exact in 64 bits; what is kept is rounded to the type.
            h = (h + s["residual"].to(f64)).to(s["x"].dtype).to(f64)
        y = h / (h.pow(2).sum(-1, keepdim=True) / case["hidden"] + _NORM_EPS).sqrt() * s["weight"].to(f64)
        out = y
        if case["quantize"]:
            each, scale = _shared(y)
            out = (_over(y, each), scale)
        return out if s["residual"] is None else (out, h)
    if case["op"] == "rmsnorm_backward":
        h, w, dy = s["x"].to(f64), s["weight"].to(f64), s["grad"].to(f64)
        rms = (h.pow(2).sum(-1, keepdim=True) / case["hidden"] + _NORM_EPS).sqrt()
        unit = h / rms
        along = (dy * w * unit).sum(-1, keepdim=True) / case["hidden"]
        dx = (dy * w - unit * along) / rms
        if s["residual"] is not None:
            dx = dx + s["residual"].to(f64)
        return dx, (dy * unit).sum(0)
    losses, grads = [], []
    E, k, D = case["experts"], case["topk"], case["ranks"]
    for i, (x, e) in enumerate(zip(s["logits"], s["experts"])):
        chosen = torch.zeros(x.shape[0], E, dtype=f64, device=x.device)
        for c in range(k):
            col = e[:, c].long()
            rows = torch.nonzero(col >= 0).squeeze(-1)
            chosen[rows, col[rows]] += 1.0
        live = chosen.sum(1) > 0
        T = max(1, int(live.sum()))
        z = x.to(f64)
        z = (z - z.max(1, keepdim=True).values).exp()
        p = z / z.sum(1, keepdim=True) * live.unsqueeze(1)
        per_rank = chosen.reshape(-1, D, E // D)
        f = chosen.sum(0) * E / (k * T)
        w = _ALPHA["expert_weight"] * f
        w = w + _ALPHA["rank_weight"] * (f.reshape(D, -1).sum(1) * D / E).repeat_interleave(E // D)
        w = w + _ALPHA["traffic_weight"] * ((per_rank.sum(2) > 0).to(f64).sum(0) * D / (min(k, D) * T)).repeat_interleave(E // D)
        losses.append((p.sum(0) / T) @ w)
        if case["backward"]:
            grads.append(s["grad"][i].to(f64) / T * p * (w - (p @ w).unsqueeze(1)))
    got = {"loss": torch.stack(losses), "expert_tokens": None, "rank_tokens": None}
    return got | {"grad": grads} if case["backward"] else got
