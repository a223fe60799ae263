"""Timed cases of the 8-bit MoE layer's operators: the residual norm that writes 8-bit rows, gating by scores with groups
of experts, expert blocks on 8-bit rows and weights, and the conversion to 8 bits, each in a plain form (elementary torch
operations) and as the framework's call.

8-bit tensors are pairs: values [.., n] in e4m3 and scales [.., n / 32] in e8m0, one per 32 neighbours of the last
dimension.  A block's scale is the smallest power of two, at least 2^-126, by which its largest magnitude becomes at
most 448; a block that holds an infinity or a NaN is NaN in all its values and in its scale.

A case is a dict of plain values; "op" says which operator:
  quantize: rows, H
  norm:     T, H; residual (a second input is added), weighted (a learned scale), sum / out / mx (which results are wanted)
  route:    T, H, E, K; score, balance (a bias for the choice alone), groups, top_groups, best (how many of a group's scores
            make its value), renorm, scale
  experts:  T, H, E, K, I; routing "uniform" or "zipf" (a few hot experts)
"""
from __future__ import annotations

import functools
import math

import torch

own = False

# the layer every benchmark workload of this repository uses, and a generic one with a few large experts
LAYER = dict(H=2048, E=60, K=4)
GROUPED = dict(H=2048, E=256, K=8, score="sigmoid", balance=True, groups=8, top_groups=4, best=2, renorm=True, scale=2.5)
PLAIN_SOFTMAX = dict(score="softmax", balance=False, groups=1, top_groups=1, best=1, renorm=False, scale=1.0)
ALL_OUT = dict(residual=True, weighted=True, sum=True, out=True, mx=True)


def listed():
    return [
        # the rows of a small decode step on their way to 8 bits: one short launch
        dict(name="quantize_13", op="quantize", rows=13, H=2048),
        # a projection of every expert of a layer, converted when the weights are loaded
        dict(name="quantize_weights", op="quantize", rows=60 * 1408, H=2048),
        # one request decoding alone: latency
        dict(name="norm_1", op="norm", T=1, H=2048, **ALL_OUT),
        # a chunk of a prompt, ragged, wider rows; the first layer has no second input, and only the 8-bit rows are wanted
        dict(name="norm_777_mx", op="norm", T=777, H=4096, residual=False, weighted=True, sum=False, out=False, mx=True),
        # a large prefill batch: the new residual stream, the router's rows and the experts' rows in one pass
        dict(name="norm_16384", op="norm", T=16384, H=2048, **ALL_OUT),
        # a lightly loaded decode step of the benchmark's layer
        dict(name="route_13", op="route", T=13, **LAYER, **PLAIN_SOFTMAX),
        # a busy decode step of a layer with many experts in groups, an odd number of requests
        dict(name="route_301_groups", op="route", T=301, **GROUPED),
        # a prefill batch of the same layer
        dict(name="route_8192_groups", op="route", T=8192, **GROUPED),
        # one request decoding alone
        dict(name="experts_1", op="experts", T=1, I=1408, routing="uniform", **LAYER),
        # the benchmark's decode step: one token of each of 128 requests
        dict(name="experts_128", op="experts", T=128, I=1408, routing="uniform", **LAYER),
        # the benchmark's prefill batch, its requests favouring the same experts
        dict(name="experts_4096_zipf", op="experts", T=4096, I=1408, routing="zipf", **LAYER),
        # the largest batch of the benchmark's sweep
        dict(name="experts_16384", op="experts", T=16384, I=1408, routing="uniform", **LAYER),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    def most(op, what):
        return max(work(c)[what] for c in listed() if c["op"] == op)

    while True:
        op = rng.choice(["quantize", "norm", "norm", "route", "route", "experts", "experts", "experts"])
        if op == "quantize":
            c = dict(op=op, rows=_log_uniform(rng, 1, 200000), H=64 * _log_uniform(rng, 1, 128))
        elif op == "norm":
            c = dict(op=op, T=_log_uniform(rng, 1, 16384), H=64 * _log_uniform(rng, 1, 128), residual=rng.random() < 0.8,
                     weighted=rng.random() < 0.8, sum=rng.random() < 0.7, out=rng.random() < 0.7, mx=rng.random() < 0.8)
            if not (c["sum"] or c["out"] or c["mx"]):
                continue
        elif op == "route":
            E = rng.choice([8, 16, 60, 64, 96, 128, 160, 200, 256])
            groups = rng.choice([g for g in (1, 1, 1, 2, 4, 8, 16) if E % g == 0 and E // g >= 4])
            top = rng.randint(1, groups)
            c = dict(op=op, T=_log_uniform(rng, 1, 16384), H=64 * _log_uniform(rng, 2, 128), E=E,
                     K=min(rng.choice([1, 2, 4, 6, 8, 8, 10]), top * (E // groups)), score=rng.choice(["softmax", "sigmoid"]),
                     balance=rng.random() < 0.6, groups=groups, top_groups=top, best=rng.choice([1, 2]),
                     renorm=rng.random() < 0.6, scale=rng.choice([1.0, 1.0, 2.5]))
        else:
            kind = rng.random()
            if kind < 0.4:
                layer = dict(I=1408, **LAYER)
            elif kind < 0.6:       # a few large experts
                layer = dict(H=64 * rng.randint(32, 72), E=rng.choice([4, 8, 8, 12]), K=rng.choice([1, 2, 2]), I=64 * rng.randint(32, 112))
            elif kind < 0.9:       # many small experts
                layer = dict(H=64 * rng.randint(12, 40), E=rng.choice([32, 64, 96, 128, 200, 256]), K=rng.choice([4, 6, 8]),
                             I=64 * rng.randint(4, 20))
            else:                  # tiny layers
                layer = dict(H=64 * rng.randint(1, 4), E=rng.choice([1, 4, 8, 16]), K=1, I=64 * rng.randint(1, 4))
            c = dict(op=op, T=_log_uniform(rng, 1, 16384), routing=rng.choice(["uniform", "zipf"]), **layer)
            if c["E"] * c["I"] * c["H"] > 3e8:
                continue
        if all(work(c)[what] <= most(op, what) for what in ("bytes", "flops")):
            return c


def _zipf_logits(E, gen):
    """A router bias of +-2 logits: a few hot experts, in a random order."""
    r = torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32)) * -1.1
    r = (r - r.min()) / (r.max() - r.min()).clamp_min(1e-6) * 4.0 - 2.0
    return r[torch.randperm(E, generator=gen, device="cuda")]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 3)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, dtype=torch.float32, device="cuda").mul_(std)

    def rows(n, H):     # activations: some channels several times as large as the others, as in trained models
        return normal(n, H).mul_(torch.exp(0.7 * normal(H))).to(torch.bfloat16)

    s = dict(case=c)
    if c["op"] == "quantize":
        s["x"] = rows(c["rows"], c["H"])
    elif c["op"] == "norm":
        s["x"] = rows(c["T"], c["H"])
        s["y"] = rows(c["T"], c["H"]) if c["residual"] else None
        s["weight"] = (1.0 + normal(c["H"], std=0.3)).to(torch.bfloat16) if c["weighted"] else None
    elif c["op"] == "route":
        s["x"] = normal(c["T"], c["H"]).to(torch.bfloat16)
        s["Wr"] = normal(c["E"], c["H"], std=0.02).to(torch.bfloat16)
        s["balance"] = normal(c["E"], std=0.05 if c["score"] == "sigmoid" else 0.3 / c["E"]) if c["balance"] else None
    else:
        T, H, E, K, I = (c[k] for k in ("T", "H", "E", "K", "I"))
        s["x"] = _to_blocks(normal(T, H).mul_(torch.exp(0.7 * normal(H))))
        std = 0.02 if H > 256 else 0.1
        for name, n, k in (("Wg", I, H), ("Wu", I, H), ("Wd", H, I)):
            s[name] = _to_blocks(normal(E, n, k, std=std))
        logits = normal(T, E)
        if c["routing"] == "zipf":
            logits += _zipf_logits(E, gen)
        ids = logits.topk(K, dim=1).indices.reshape(-1)
        order = torch.sort(ids, stable=True).indices
        counts = torch.bincount(ids, minlength=E)
        s["src_of_row"] = order.to(torch.int32)
        s["counts"] = counts.tolist()     # (the plain form's sizes; the framework reads the bounds on the device)
        s["expert_offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        s["Yp"] = torch.empty((T * K, H), dtype=torch.bfloat16, device="cuda")
        s["workspace"] = torch.empty(T * K * I * 2 + 256, dtype=torch.uint8, device="cuda")
    return s


def _power(e):
    """2^e in fp32 of whole numbers -126 <= e <= 127, exactly."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _to_blocks(v):
    """fp32 [.., n] -> (e4m3 values [.., n], e8m0 scales [.., n / 32])"""
    b = v.reshape(*v.shape[:-1], v.shape[-1] // 32, 32)
    largest = b.abs().amax(-1)
    bad = ~torch.isfinite(largest)
    m, e = torch.frexp(largest.masked_fill(bad, 1.0).clamp_min(2.0 ** -126))      # largest = m * 2^e, 1/2 <= m < 1
    e = (e - 9 + (m > 0.875).to(e.dtype)).clamp_min(-126)                         # 448 = 0.875 * 2^9
    q = (b * _power(-e)[..., None]).masked_fill(bad[..., None], math.nan).to(torch.float8_e4m3fn)
    scales = (e + 127).masked_fill(bad, 255).to(torch.uint8).view(torch.float8_e8m0fnu)
    return q.reshape(v.shape), scales


def _values(pair):
    """fp32 values of an 8-bit tensor (finite scales)"""
    q, scales = pair
    s = _power(scales.view(torch.uint8).to(torch.int64) - 127)
    return (q.to(torch.float32).reshape(*scales.shape, 32) * s[..., None]).reshape(q.shape)


def _plain_norm(s):
    c = s["case"]
    u = s["x"].float()
    if s["y"] is not None:
        u = u + s["y"].float()
    n = u / torch.sqrt((u * u).mean(-1, keepdim=True) + 1e-6)
    if s["weight"] is not None:
        n = n * s["weight"].float()
    got = {}
    if c["sum"]:
        got["sum"] = u.to(torch.bfloat16)
    if c["out"]:
        got["out"] = n.to(torch.bfloat16)
    if c["mx"]:
        got["q"], got["scales"] = _to_blocks(n)
    return got


def _plain_logits(x, Wr):
    # The router's logits are defined with their order of additions (element h belongs to partial sum (h / 8) mod 64, which
    # takes its elements one by one; the 64 are folded pairwise): the loop is that order, 64 sums at a time.
    T, H = x.shape
    E, n = Wr.shape[0], -(-H // 512)
    xp = torch.nn.functional.pad(x.float(), (0, 512 * n - H)).reshape(T, 1, n, 64, 8)
    wp = torch.nn.functional.pad(Wr.float(), (0, 512 * n - H)).reshape(1, E, n, 64, 8)
    acc = torch.zeros((T, E, 64), dtype=torch.float32, device=x.device)
    for i in range(8 * n):
        acc.addcmul_(xp[:, :, i // 8, :, i % 8], wp[:, :, i // 8, :, i % 8])      # (a product of two bf16 is exact in fp32)
    for _ in range(6):
        acc = acc[..., 0::2] + acc[..., 1::2]
    return acc[..., 0]


def _plain_route(s):
    c = s["case"]
    T, E, G = c["T"], c["E"], c["groups"]
    logits = _plain_logits(s["x"], s["Wr"]).double()      # (scores decide between near ties: 64 bits, rounded once)
    scores = (torch.sigmoid(logits) if c["score"] == "sigmoid" else torch.softmax(logits, -1)).float()
    choice = scores if s["balance"] is None else scores + s["balance"]
    if G > 1:
        best = choice.reshape(T, G, E // G).sort(dim=-1, descending=True).values[..., :c["best"]].sum(-1)
        kept = best.sort(dim=-1, descending=True, stable=True).indices[:, :c["top_groups"]]
        allowed = torch.zeros((T, G), dtype=torch.bool, device=logits.device).scatter_(1, kept, True)
        choice = choice.masked_fill(~allowed.repeat_interleave(E // G, 1), -math.inf)
    ids = choice.sort(dim=-1, descending=True, stable=True).indices[:, :c["K"]]
    w = scores.gather(1, ids)
    if c["renorm"]:
        w = w / (w.sum(-1, keepdim=True) + 1e-20)
    return {"topk_ids": ids.to(torch.int32), "topk_w": w * c["scale"]}


def _plain_experts(s):
    c = s["case"]
    x = _values(s["x"])[(s["src_of_row"] // c["K"]).long()]
    at = 0
    for e, n in enumerate(s["counts"]):      # (an expert's weights multiply its rows: as many products as experts have rows)
        if n:
            r = x[at:at + n]
            g = r @ _values((s["Wg"][0][e], s["Wg"][1][e])).T
            u = r @ _values((s["Wu"][0][e], s["Wu"][1][e])).T
            h = (g / (1.0 + torch.exp(-g)) * u).to(torch.bfloat16).float()     # (the hidden rows are bf16)
            s["Yp"][at:at + n] = (h @ _values((s["Wd"][0][e], s["Wd"][1][e])).T).to(torch.bfloat16)
        at += n
    return {"Yp": s["Yp"]}


def run(state):
    s = state
    c = s["case"]
    if own:
        import paper_2604_26881_amd as moe
        if c["op"] == "quantize":
            q, scales = moe.moe_quantize_mx(s["x"])
            return {"q": q, "scales": scales}
        if c["op"] == "norm":
            got = moe.moe_residual_norm_mx(s["x"], s["y"], s["weight"], eps=1e-6, keep_sum=c["sum"], keep_out=c["out"], quantize=c["mx"])
            return {k: v for k, v in zip(("sum", "out", "q", "scales"), got) if v is not None}
        if c["op"] == "route":
            ids, w = moe.moe_route_scored(s["x"], s["Wr"], s["balance"], c["K"], score=c["score"], groups=c["groups"],
                                          top_groups=c["top_groups"], group_best=c["best"], renorm=c["renorm"], scale=c["scale"])
            return {"topk_ids": ids, "topk_w": w}
        moe.moe_expert_group_forward_mx(0, c["E"], s["x"], s["src_of_row"], c["K"], s["expert_offsets"], s["Wg"], s["Wu"], s["Wd"],
                                        s["Yp"], s["workspace"])
        return {"Yp": s["Yp"]}
    if c["op"] == "quantize":
        q, scales = _to_blocks(s["x"].float())
        return {"q": q, "scales": scales}
    return {"norm": _plain_norm, "route": _plain_route, "experts": _plain_experts}[c["op"]](s)


@functools.lru_cache(maxsize=None)
def _active(T, E, K, routing):
    """Experts that a batch activates, on average, from a sample of the same router logits."""
    g = torch.Generator().manual_seed(1)
    logits = torch.randn((4096, E), generator=g)
    if routing == "zipf" and E > 1:
        r = torch.log(torch.arange(1, E + 1, dtype=torch.float32)) * -1.1
        logits = logits + (r - r.min()) / (r.max() - r.min()) * 4.0 - 2.0
    share = torch.bincount(logits.topk(K, dim=1).indices.reshape(-1), minlength=E).double() / 4096
    return float((1.0 - (1.0 - share).pow(T)).sum())


def work(case):
    c = case
    mx = 1.0 + 1.0 / 32.0        # bytes of an 8-bit value and its share of the scale
    if c["op"] == "quantize":
        return {"bytes": c["rows"] * c["H"] * (2.0 + mx), "flops": 2.0 * c["rows"] * c["H"]}
    if c["op"] == "norm":
        per = 2.0 + 2.0 * c["residual"] + 2.0 * c["sum"] + 2.0 * c["out"] + mx * c["mx"]
        return {"bytes": c["T"] * c["H"] * per + 2.0 * c["H"] * c["weighted"], "flops": 5.0 * c["T"] * c["H"]}
    T, H, E, K = (c[k] for k in ("T", "H", "E", "K"))
    if c["op"] == "route":
        return {"bytes": 2.0 * H * (T + E) + 8.0 * T * K + 4.0 * E * c["balance"], "flops": 2.0 * T * H * E}
    I = c["I"]
    return {"bytes": mx * (T * H + 3.0 * _active(T, E, K, c["routing"]) * I * H) + 2.0 * T * K * H + 4.0 * (T * K + E + 1),
            "flops": 6.0 * T * K * H * I}


# ---- the definitions in 64 bits

def _two_to(e):
    """2^e in 64 bits, exactly, of whole numbers in a 64-bit tensor (the library's power is an ulp off at times)"""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _grid(v):
    """64-bit values to the 8-bit format: (the e4m3 values, the scales), as 64-bit numbers."""
    blocks = torch.stack(v.split(32, dim=-1), dim=-2)
    top = blocks.abs().max(dim=-1).values
    e = torch.ceil(torch.log2(torch.clamp(top, min=2.0 ** -134) / 448.0)).clamp(min=-126.0)
    e = torch.where(top > 448.0 * _two_to(e), e + 1.0, e)                         # (should the logarithm round across a whole number)
    e = torch.where((top <= 448.0 * _two_to(e - 1.0)) & (e > -126.0), e - 1.0, e)
    scale = _two_to(e)
    t = blocks / scale[..., None]
    exponent = torch.frexp(t.abs().clamp(min=2.0 ** -6)).exponent - 1
    step = _two_to(exponent - 3)
    q = torch.round(t / step) * step
    return q.flatten(-2), scale


def _wide(pair):
    """64-bit values of an 8-bit tensor"""
    q, scales = pair
    return q.double() * scales.double().repeat_interleave(32, dim=-1)


def _exact_logits(x, Wr):
    """The defined order of additions in 64-bit arithmetic, each sum rounded to the 24 bits that it is defined with."""
    T, H = x.shape
    x, Wr = x.double(), Wr.double()
    at = torch.arange(H, device=x.device)
    sums = torch.zeros((T, Wr.shape[0], 64), dtype=torch.float64, device=x.device)
    for k in range(0, H, 512):
        here = at[k:k + 512]
        lanes = here.numel() // 8
        for i in range(8):
            h = here[i::8]
            sums[..., :lanes] = (sums[..., :lanes] + x[:, None, h] * Wr[None, :, h]).float().double()
    lane = torch.arange(64, device=x.device)
    for s in (1, 2, 4, 8, 16, 32):
        sums = (sums + sums[..., lane ^ s]).float().double()
    return sums[..., 0]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "quantize":
        q, scales = _grid(s["x"].double())
        return {"q": q, "scales": scales}
    if c["op"] == "norm":
        u = s["x"].double()
        if s["y"] is not None:
            u = u + s["y"].double()
        n = u * torch.rsqrt(u.square().sum(-1, keepdim=True) / c["H"] + 1e-6)
        if s["weight"] is not None:
            n = n * s["weight"].double()
        q, scales = _grid(n) if c["mx"] else (None, None)
        got = {"sum": u if c["sum"] else None, "out": n if c["out"] else None, "q": q, "scales": scales}
        return {k: v for k, v in got.items() if v is not None}
    if c["op"] == "route":
        l = _exact_logits(s["x"], s["Wr"])
        p = 1.0 / (1.0 + torch.exp(-l)) if c["score"] == "sigmoid" else torch.exp(l - torch.logsumexp(l, -1, keepdim=True))
        rank = p.float().double()                # (the choice is defined on scores of 24 bits)
        if s["balance"] is not None:
            rank = (rank + s["balance"].double()).float().double()
        if c["groups"] > 1:
            size = c["E"] // c["groups"]
            value = torch.stack([rank[:, g * size:(g + 1) * size].topk(c["best"], dim=1).values.sum(1).float().double()
                                 for g in range(c["groups"])], 1)
            ahead = (value[:, None, :] > value[:, :, None]).sum(-1)               # groups with a larger value
            tie = (value[:, None, :] == value[:, :, None]) & torch.ones_like(value[0, None, :] * value[0, :, None]).tril(-1).bool()
            kept = ahead + tie.sum(-1) < c["top_groups"]
            rank = rank.where(kept[:, torch.arange(c["E"], device=l.device) // size], torch.full_like(rank, -math.inf))
        ids = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :c["K"]]
        w = torch.take_along_dim(p, ids, 1)
        if c["renorm"]:
            w = w / (w.sum(1, keepdim=True) + 1e-20)
        return {"topk_ids": None, "topk_w": w * c["scale"]}
    x = _wide(s["x"])
    parts = []
    tokens = torch.div(s["src_of_row"].long(), c["K"], rounding_mode="floor").split(s["counts"])
    for e, t in enumerate(tokens):
        if t.numel():
            gate = torch.matmul(x[t], _wide([w[e] for w in s["Wg"]]).T)
            up = torch.matmul(x[t], _wide([w[e] for w in s["Wu"]]).T)
            parts.append(torch.matmul(gate * torch.sigmoid(gate) * up, _wide([w[e] for w in s["Wd"]]).T))
    return {"Yp": torch.cat(parts)}
