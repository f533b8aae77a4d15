"""What a layer of experts needs to be trained and to run in 8 bits throughout, as a measurement takes it: cases, inputs, a plain form and the library's calls.

Five kinds of pass:

  choose     a router's logits: each token's k experts with the largest, their weights (softmax), and the logarithm of the sum of exponentials
  balance    rows per expert, the balance loss and the mean square of that logarithm, and the logits' gradient of those and of the weights
  rows       rows in 8 bits (e4m3) with a power-of-two scale for each 128 columns, laid out by expert on the way
  matrices   the experts' matrices in 8 bits with a scale for each block of 128 x 128, and the same transposed (for the gradient of the rows)
  product    out[p] = x[p] . W[e]^T of such rows and matrices, for the rows p of each expert e

`own` chooses between the plain form (elementary torch operations in 32 bits, rounded once) and the library's entry points.
Both take what prepare() makes.  exact() is the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BLOCK = 128


def listed():
    return [
        # ---- choose
        # a decoding step of a small batch: latency
        dict(name="choose_8x64_k4", op="choose", tokens=8, experts=64, k=4, type="f32", masked=0.0, all=False, pad=0),
        # a prefill in batches that are padded, weights not normalised among the chosen; bf16 has ties
        dict(name="choose_16384x256_k8", op="choose", tokens=16384, experts=256, k=8, type="bf16", masked=0.0625, all=True, pad=0),
        # ---- balance, forward and backward
        # ragged: the pixels of maps, two of sixty experts, some of the slots beyond an expert's capacity
        dict(name="balance_4099x60_k2", op="balance", tokens=4099, experts=60, k=2, type="bf16", masked=0.1, drop=0.0625, all=False, pad=0),
        # a training step
        dict(name="balance_32768x256_k8", op="balance", tokens=32768, experts=256, k=8, type="f32", masked=0.0, drop=0.0, all=False, pad=0),
        # ---- rows in 8 bits
        # odd sizes in 32 bits, rows stay where they are: no row but the first is aligned, the last block of a row is not whole
        dict(name="rows_f32_4099x1001", op="rows", tokens=4099, k=0, experts=1, cols=1001, type="f32", drop=0.0, pad=0),
        # a prefill or training step: four copies of each row
        dict(name="rows_16384x4of64x2048", op="rows", tokens=16384, k=4, experts=64, cols=2048, type="bf16", drop=0.0, pad=0),
        # ---- matrices in 8 bits
        # ragged, master weights in 32 bits
        dict(name="matrices_f32_8x1000x520", op="matrices", experts=8, n=1000, k=520, type="f32", both=True),
        # after a step of training: forward and transposed
        dict(name="matrices_16x4096x2048", op="matrices", experts=16, n=4096, k=2048, type="bf16", both=True),
        # ---- the product
        # a decoding step: 16 rows over 16 experts, bound by the weights
        dict(name="product_16r_16e_1024x2048", op="product", rows=16, experts=16, n=1024, k=2048, scales="e8m0", relu=False, tail=0),
        # ordinary and ragged, scales of weights that were rounded elsewhere
        dict(name="product_4001r_8e_1000x528_f32", op="product", rows=4001, experts=8, n=1000, k=528, scales="f32", relu=True, tail=17),
        # a training step with such scales
        dict(name="product_16384r_8e_2048x4096_f32", op="product", rows=16384, experts=8, n=2048, k=4096, scales="f32", relu=False, tail=0),
        # a large prefill
        dict(name="product_32768r_16e_4096x2048", op="product", rows=32768, experts=16, n=4096, k=2048, scales="e8m0", relu=False, tail=0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high, whole, share):
    """A number of columns: a multiple of `whole` in this share of the draws."""
    v = _log(rng, low, high)
    return (v + whole - 1) // whole * whole if rng.random() < share else v


def draw(rng):
    op = rng.choice(["choose", "choose", "balance", "balance", "rows", "rows", "matrices", "product", "product", "product"])
    if op in ("choose", "balance"):
        experts = _width(rng, 2, 512, 8, 0.6)
        k = min(experts, rng.choice([1, 2, 2, 4, 6, 8, 16]))
        tokens = _log(rng, 1, min(65536, (1 << 23) // experts))
        case = dict(op=op, tokens=tokens, experts=experts, k=k, type=rng.choice(["f32", "bf16"]), masked=rng.choice([0.0, 0.0, 0.0625, 0.5]))
        if op == "balance":
            case["drop"] = rng.choice([0.0, 0.0, 0.0625, 0.5])
        return dict(case, all=rng.random() < 0.4, pad=rng.choice([0, 0, 0, 8, 3]))
    if op == "rows":
        cols = _width(rng, 64, 8192, 16, 0.7)
        k = rng.choice([0, 1, 2, 2, 4, 6, 8])
        experts = max(k, _log(rng, 2, 256)) if k else 1
        tokens = _log(rng, 1, min(65536, (1 << 27) // (cols * max(k, 1))))
        return dict(op=op, tokens=tokens, k=k, experts=experts, cols=cols, type=rng.choice(["bf16", "bf16", "f32"]), drop=rng.choice([0.0, 0.0, 0.0625, 0.5]) if k else 0.0,
                    pad=rng.choice([0, 0, 0, 16, 3]))
    share = rng.choice([0.0, 1.0, 1.0, 1.0])
    n, k = _width(rng, 64, 8192, 16, share), _width(rng, 64, 8192, 16, share)
    if op == "matrices":
        return dict(op=op, experts=_log(rng, 1, max(1, min(64, (1 << 27) // (n * k)))), n=n, k=k, type=rng.choice(["bf16", "f32"]), both=rng.random() < 0.7)
    experts = _log(rng, 1, max(1, min(64, (1 << 28) // (n * k))))
    rows = _log(rng, 1, min(32768, (1 << 37) // (n * k)))
    return dict(op=op, rows=rows, experts=experts, n=n, k=k, scales=rng.choice(["e8m0", "f32"]), relu=rng.random() < 0.3, tail=min(rng.choice([0, 0, 0, 17]), rows // 2))


# ---------------------------------------------------------------- inputs

def _values(g, rows, cols, dtype, pad=0, spread=0.5):
    """Activations: normal, with channels of different strengths, as a view whose rows lie cols + pad apart."""
    strength = torch.exp(spread * torch.randn(cols, generator=g, device="cuda"))
    out = torch.zeros(rows, cols + pad, device="cuda", dtype=dtype)
    out[:, :cols] = (torch.randn(rows, cols, generator=g, device="cuda") * strength).to(dtype)
    return out[:, :cols]


def _exponent(top):
    """e of the least power of two with top <= 448 * 2^e, -126 at least."""
    mantissa, exponent = torch.frexp(torch.clamp(top, min=2.0 ** -126))                   # top = mantissa 2^exponent, 448 = 0.875 2^9
    return torch.clamp(exponent.to(torch.int32) - 9 + (mantissa > 0.875).to(torch.int32), min=-126)


def _power(e):
    return ((e + 127) << 23).view(torch.float32)


def _in_blocks(v):
    """Rows in e4m3 with a scale (float32, a power of two) for each 128 columns."""
    cols = v.shape[-1]
    blocks = (cols + _BLOCK - 1) // _BLOCK
    b = torch.nn.functional.pad(v, (0, blocks * _BLOCK - cols)).view(*v.shape[:-1], blocks, _BLOCK)
    scale = _power(_exponent(b.abs().amax(-1)))
    q = (b / scale[..., None]).to(torch.float8_e4m3fn)
    return q.reshape(*v.shape[:-1], blocks * _BLOCK)[..., :cols].contiguous(), scale


def _tops(W):
    """The largest absolute value of each block of 128 x 128 of [E, n, k]."""
    E, n, k = W.shape
    nb, kb = (n + _BLOCK - 1) // _BLOCK, (k + _BLOCK - 1) // _BLOCK
    b = torch.nn.functional.pad(W, (0, kb * _BLOCK - k, 0, nb * _BLOCK - n)).view(E, nb, _BLOCK, kb, _BLOCK)
    return b.abs().amax((2, 4))


def _spread_blocks(scale, n, k):
    """A scale for each block -> one for each element of [E, n, k]."""
    return scale.repeat_interleave(_BLOCK, 1)[:, :n].repeat_interleave(_BLOCK, 2)[:, :, :k]


def _sorted(chosen, experts):
    """The slots sorted by expert: offsets, the slot of each row (-1: none), the row of each slot (-1: not sent)."""
    key = torch.where(chosen.reshape(-1) < 0, experts, chosen.reshape(-1).long())
    order = torch.argsort(key, stable=True)
    offsets = torch.searchsorted(key[order].contiguous(), torch.arange(experts + 1, device="cuda"))
    n = key.numel()
    place = torch.empty(n, dtype=torch.long, device="cuda")
    place[order] = torch.arange(n, device="cuda")
    position = torch.where(place < offsets[-1], place, -1).to(torch.int32)
    order = torch.where(torch.arange(n, device="cuda") < offsets[-1], order, -1)
    return offsets.to(torch.int32), order, position.view(chosen.shape)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)
    op, s = case["op"], {"case": case}
    if op in ("choose", "balance"):
        tokens, experts, k = case["tokens"], case["experts"], case["k"]
        # logits of a router: some experts in greater demand
        logits = 1.5 * torch.randn(tokens, experts, generator=g, device="cuda") + 0.5 * torch.randn(experts, generator=g, device="cuda")
        held = torch.zeros(tokens, experts + case["pad"], device="cuda", dtype=_TYPES[case["type"]])
        held[:, :experts] = logits.to(held.dtype)
        s["logits"] = held[:, :experts]
        there = torch.rand(tokens, generator=g, device="cuda") >= case["masked"]
        s["mask"] = there.to(torch.uint8) if case["masked"] else None
        s["experts"] = torch.empty(tokens, k, dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty(tokens, k, device="cuda")
        s["lse"] = torch.empty(tokens, device="cuda")
        if op == "balance":
            values, chosen = torch.topk(s["logits"].float(), k, dim=-1)
            s["lse"].copy_(torch.where(there, torch.logsumexp(s["logits"].float(), -1), -math.inf))
            weights = torch.exp(values - s["lse"][:, None]) if case["all"] else torch.softmax(values, -1)
            sent = there[:, None] & (torch.rand(tokens, k, generator=g, device="cuda") >= case["drop"])
            s["experts"].copy_(torch.where(sent, chosen, -1))
            s["weights"].copy_(torch.where(there[:, None], weights, 0.0))
            s["dweights"] = torch.where(sent, torch.randn(tokens, k, generator=g, device="cuda"), 0.0)
            s["dloss"] = torch.tensor([0.01, 0.001], device="cuda") * tokens                     # (so that the parts of the gradient are of one size)
            s["counts"] = torch.empty(experts + 1, dtype=torch.int32, device="cuda")
            s["share"] = torch.empty(experts, device="cuda")
            s["loss"] = torch.empty(2, device="cuda")
            s["dlogits"] = torch.empty(tokens, experts, dtype=_TYPES[case["type"]], device="cuda")
    elif op == "rows":
        tokens, k, experts, cols = case["tokens"], case["k"], case["experts"], case["cols"]
        s["x"] = _values(g, tokens, cols, _TYPES[case["type"]], case["pad"])
        s["position"] = s["offsets"] = s["order"] = None
        if k:
            demand = torch.randn(tokens, experts, generator=g, device="cuda") + 0.5 * torch.randn(experts, generator=g, device="cuda")
            chosen = torch.topk(demand, k, dim=-1).indices.to(torch.int32)
            chosen[torch.rand(tokens, k, generator=g, device="cuda") < case["drop"]] = -1
            s["offsets"], s["order"], s["position"] = _sorted(chosen, experts)
        rows = tokens * max(k, 1)
        s["out"] = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda")
        s["scale"] = torch.empty(rows, (cols + _BLOCK - 1) // _BLOCK, dtype=torch.float8_e8m0fnu, device="cuda")
    elif op == "matrices":
        E, n, k = case["experts"], case["n"], case["k"]
        nb, kb = (n + _BLOCK - 1) // _BLOCK, (k + _BLOCK - 1) // _BLOCK
        strength = torch.exp(0.5 * torch.randn(k, generator=g, device="cuda"))
        s["W"] = (torch.randn(E, n, k, generator=g, device="cuda") * (k ** -0.5 * strength)).to(_TYPES[case["type"]])
        s["out"] = torch.empty(E, n, k, dtype=torch.float8_e4m3fn, device="cuda")
        s["scale"] = torch.empty(E, nb, kb, dtype=torch.float8_e8m0fnu, device="cuda")
        s["out_t"] = torch.empty(E, k, n, dtype=torch.float8_e4m3fn, device="cuda") if case["both"] else None
        s["scale_t"] = torch.empty(E, kb, nb, dtype=torch.float8_e8m0fnu, device="cuda") if case["both"] else None
    else:
        rows, experts, n, k = case["rows"], case["experts"], case["n"], case["k"]
        # experts in different demand, some without a row; the last `tail` rows belong to none
        r = np.random.RandomState(int(seed) % (1 << 31))
        share = np.exp(0.5 * r.standard_normal(experts))
        counts = r.multinomial(rows - case["tail"], share / share.sum())
        s["offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32).cuda()
        s["most"] = int(max(1, counts.max()))
        s["x"], scale = _in_blocks(_values(g, rows, k, torch.float32))
        s["scale"] = scale.to(torch.float8_e8m0fnu)
        W = torch.randn(experts, n, k, generator=g, device="cuda") * k ** -0.5
        top = _tops(W)
        scale = _power(_exponent(top)) if case["scales"] == "e8m0" else top / 448.0
        s["W"] = (W / _spread_blocks(scale, n, k)).to(torch.float8_e4m3fn)
        s["wscale"] = scale.to(torch.float8_e8m0fnu) if case["scales"] == "e8m0" else scale
        s["out"] = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    return s


# ---------------------------------------------------------------- the plain form

def _plain_choose(s):
    case, logits = s["case"], s["logits"].float()
    values, chosen = torch.sort(logits, dim=-1, descending=True, stable=True)             # (equal ones stay in order: the lowest index first)
    values, chosen = values[:, :case["k"]], chosen[:, :case["k"]].to(torch.int32)
    top = values[:, :1]
    lse = top + torch.log(torch.exp(logits - top).sum(-1, keepdim=True))
    if case["all"]:
        weights = torch.exp(values - lse)
    else:
        e = torch.exp(values - top)
        weights = e / e.sum(-1, keepdim=True)
    if s["mask"] is not None:
        there = s["mask"].bool()[:, None]
        chosen, weights, lse = torch.where(there, chosen, -1), torch.where(there, weights, 0.0), torch.where(there, lse, -math.inf)
    return {"experts": chosen, "weights": weights, "lse": lse[:, 0]}


def _plain_balance(s):
    case, E = s["case"], s["case"]["experts"]
    there = s["lse"] > -math.inf
    lse = torch.where(there, s["lse"], 0.0)
    p = torch.where(there[:, None], torch.exp(s["logits"].float() - lse[:, None]), 0.0)
    sent = s["experts"] >= 0
    to = torch.where(sent, s["experts"], E).reshape(-1).long()
    counts = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    counts.scatter_add_(0, to, torch.ones_like(to, dtype=torch.int32))
    tokens = there.sum()
    counts[E] = tokens
    n = torch.clamp(tokens, min=1).double()
    share = (p.double().sum(0) / n).float()                                             # (long sums)
    load = counts[:E].double() * (E / (case["k"] * n))
    loss = torch.stack([(load * share.double()).sum(), lse.double().square().sum() / n]).float()
    # its gradient, and that of the weights
    load, n = load.float(), n.float()
    dlogits = p * (load - (p * load).sum(-1, keepdim=True)) * (s["dloss"][0] / n) + p * (lse[:, None] * (2.0 * s["dloss"][1] / n))
    inner = s["weights"] * s["dweights"]
    if case["all"]:
        direct = inner
        dlogits = dlogits - p * inner.sum(-1, keepdim=True)
    else:
        direct = inner - s["weights"] * inner.sum(-1, keepdim=True)
    wide = torch.zeros(p.shape[0], E + 1, device="cuda")
    wide.scatter_add_(1, to.view(sent.shape), direct)
    return {"counts": counts, "share": share, "loss": loss, "dlogits": (dlogits + wide[:, :E]).to(s["logits"].dtype)}


def _plain_rows(s):
    x = s["x"].float()
    if s["order"] is not None:
        sent = s["order"] >= 0
        x = torch.where(sent[:, None], x[torch.clamp(s["order"], min=0) // s["case"]["k"]], 0.0)
    q, scale = _in_blocks(x)
    if s["order"] is not None:
        scale = torch.where(sent[:, None], scale, 1.0)
    return {"out": q, "scale": scale.to(torch.float8_e8m0fnu)}


def _plain_matrices(s):
    W = s["W"].float()
    scale = _power(_exponent(_tops(W)))
    q = (W / _spread_blocks(scale, W.shape[1], W.shape[2])).to(torch.float8_e4m3fn)
    got = {"out": q, "scale": scale.to(torch.float8_e8m0fnu)}
    if s["out_t"] is not None:
        got["out_t"] = q.view(torch.uint8).transpose(1, 2).contiguous().view(torch.float8_e4m3fn)
        got["scale_t"] = scale.transpose(1, 2).contiguous().to(torch.float8_e8m0fnu)
    return got


def _plain_product(s):
    case, offsets = s["case"], s["offsets"].long()
    rows, E, n, k = case["rows"], case["experts"], case["n"], case["k"]
    x = s["x"].float() * s["scale"].float().repeat_interleave(_BLOCK, 1)[:, :k]
    W = s["W"].float() * _spread_blocks(s["wscale"].float(), n, k)
    # each expert's rows at the same length, zeros behind them; rows of no expert behind all
    p = torch.arange(rows, device="cuda")
    expert = torch.searchsorted(offsets[1:].contiguous(), p, right=True)
    sent = expert < E
    to = torch.where(sent, expert * s["most"] + p - offsets[torch.clamp(expert, max=E - 1)], E * s["most"])
    padded = torch.zeros(E * s["most"] + 1, k, device="cuda")
    padded[to] = x
    out = torch.bmm(padded[:-1].view(E, s["most"], k), W.transpose(1, 2)).reshape(-1, n)
    out = torch.where(sent[:, None], out[torch.clamp(to, max=out.shape[0] - 1)], 0.0)
    if case["relu"]:
        out = torch.clamp(out, min=0.0)
    return {"out": out.to(torch.bfloat16)}


_PLAIN = {"choose": _plain_choose, "balance": _plain_balance, "rows": _plain_rows, "matrices": _plain_matrices, "product": _plain_product}


# ---------------------------------------------------------------- the library's calls

def _library(s):
    from paper_2210_06223_amd import binding as B
    case, op = s["case"], s["case"]["op"]
    if op == "choose":
        B.lasnet_choose_experts(s["logits"], case["k"], mask=s["mask"], experts=s["experts"], weights=s["weights"], lse=s["lse"],
                                flags=B.LASNET_WEIGHTS_OF_ALL if case["all"] else 0)
        return {"experts": s["experts"], "weights": s["weights"], "lse": s["lse"]}
    if op == "balance":
        B.lasnet_balance(s["logits"], s["lse"], s["experts"], counts=s["counts"], share=s["share"], loss=s["loss"])
        B.lasnet_choose_experts_backward(s["logits"], s["lse"], s["experts"], s["weights"], dweights=s["dweights"], counts=s["counts"], dloss=s["dloss"],
                                         dlogits=s["dlogits"], flags=B.LASNET_WEIGHTS_OF_ALL if case["all"] else 0)
        return {"counts": s["counts"], "share": s["share"], "loss": s["loss"], "dlogits": s["dlogits"]}
    if op == "rows":
        B.lasnet_quantize_rows(s["x"], position=s["position"], offsets=s["offsets"], out=s["out"], scale=s["scale"])
        return {"out": s["out"], "scale": s["scale"]}
    if op == "matrices":
        B.lasnet_quantize_matrices(s["W"], out=s["out"], scale=s["scale"], out_t=s["out_t"], scale_t=s["scale_t"])
        got = {"out": s["out"], "scale": s["scale"]}
        if s["out_t"] is not None:
            got["out_t"], got["scale_t"] = s["out_t"], s["scale_t"]
        return got
    B.lasnet_block_product(s["x"], s["scale"], s["offsets"], s["W"], s["wscale"], out=s["out"], flags=B.LASNET_POST_RELU if case["relu"] else 0)
    return {"out": s["out"]}


def run(state):
    return _library(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "choose":
        v = s["logits"].double()
        there = torch.ones(case["tokens"], dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0
        lse = torch.logsumexp(v, 1)
        best = torch.topk(v, case["k"], dim=1).values                 # (which of equal ones is chosen does not change the weights)
        w = torch.exp(best - (lse if case["all"] else torch.logsumexp(best, 1)).unsqueeze(1))
        return {"experts": None, "weights": w * there.unsqueeze(1), "lse": lse.masked_fill(~there, -math.inf)}
    if op == "balance":
        E, k, e = case["experts"], case["k"], s["experts"].long()
        there = torch.isfinite(s["lse"])
        lse = s["lse"].double().masked_fill(~there, 0.0)
        p = torch.exp(s["logits"].double() - lse.unsqueeze(1)) * there.unsqueeze(1)
        T = max(1, int(there.sum()))
        f = torch.bincount(e[e >= 0], minlength=E).double() / (k * T)
        share = p.mean(0) * (case["tokens"] / T)
        a, b = s["dloss"].double().tolist()
        d = a * E / T * (p * f - p * (p @ f).unsqueeze(1)) + 2 * b / T * p * lse.unsqueeze(1)
        w, dw = s["weights"].double(), s["dweights"].double()
        pull = (w * dw).sum(1, keepdim=True)
        if case["all"]:
            d -= p * pull
        for j in range(k):
            t = torch.nonzero(e[:, j] >= 0).flatten()
            d[t, e[t, j]] += w[t, j] * (dw[t, j] if case["all"] else dw[t, j] - pull[t, 0])
        return {"counts": None, "share": share, "loss": torch.stack([E * (f * share).sum(), (lse * lse).sum() / T]), "dlogits": d}
    if op in ("rows", "matrices"):                         # what an element stands for over its scale; the scale itself is no rounded number
        v = (s["x"] if op == "rows" else s["W"]).double()
        out = torch.empty_like(v, memory_format=torch.contiguous_format)
        if op == "rows":
            for c in range(0, case["cols"], _BLOCK):
                top = v[:, c:c + _BLOCK].abs().max(1, keepdim=True).values.clamp(min=2.0 ** -126)
                out[:, c:c + _BLOCK] = v[:, c:c + _BLOCK] * torch.exp2(-torch.ceil(torch.log2(top / 448.0)).clamp(min=-126))
            if s["position"] is not None:
                flat, moved = s["position"].long().reshape(-1), torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
                slots = torch.nonzero(flat >= 0).flatten()
                moved[flat[slots]] = out[slots // case["k"]]
                out = moved
            return {"out": out, "scale": None}
        for i in range(0, case["n"], _BLOCK):
            for c in range(0, case["k"], _BLOCK):
                b = v[:, i:i + _BLOCK, c:c + _BLOCK]
                top = b.abs().amax((1, 2), keepdim=True).clamp(min=2.0 ** -126)
                out[:, i:i + _BLOCK, c:c + _BLOCK] = b * torch.exp2(-torch.ceil(torch.log2(top / 448.0)).clamp(min=-126))
        return {"out": out, "scale": None, "out_t": out.transpose(1, 2), "scale_t": None} if case["both"] else {"out": out, "scale": None}
    ends, k, n = s["offsets"].tolist(), case["k"], case["n"]
    column, row = torch.arange(k, device="cuda") // _BLOCK, torch.arange(n, device="cuda") // _BLOCK
    x = s["x"].double() * s["scale"].double()[:, column]
    out = torch.zeros(case["rows"], n, dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        w = s["W"][e].double() * s["wscale"][e].double()[row][:, column]
        out[ends[e]:ends[e + 1]] = x[ends[e]:ends[e + 1]] @ w.T
    return {"out": out.clamp(min=0.0) if case["relu"] else out}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = {"f32": 4, "bf16": 2}
    op = case["op"]
    if op in ("choose", "balance"):
        slots, cells = case["tokens"] * case["k"], case["tokens"] * case["experts"] * size[case["type"]]
        if op == "choose":
            return {"bytes": cells + 8 * slots + 4 * case["tokens"] + (case["tokens"] if case["masked"] else 0), "flops": 3 * case["tokens"] * case["experts"]}
        return {"bytes": 2 * cells + 12 * slots + 4 * case["tokens"] + 8 * case["experts"], "flops": 8 * case["tokens"] * case["experts"]}
    if op == "rows":
        rows, blocks = case["tokens"] * max(case["k"], 1), (case["cols"] + _BLOCK - 1) // _BLOCK
        return {"bytes": case["tokens"] * case["cols"] * size[case["type"]] + rows * (case["cols"] + blocks) + (4 * rows if case["k"] else 0),
                "flops": 2 * case["tokens"] * case["cols"]}
    if op == "matrices":
        cells = case["experts"] * case["n"] * case["k"]
        return {"bytes": cells * (size[case["type"]] + (2 if case["both"] else 1)), "flops": 2 * cells}
    sent, n, k = case["rows"] - case["tail"], case["n"], case["k"]
    kb, nb = (k + _BLOCK - 1) // _BLOCK, (n + _BLOCK - 1) // _BLOCK
    weights = min(case["experts"], sent) * (n * k + nb * kb * (1 if case["scales"] == "e8m0" else 4))
    return {"bytes": sent * (k + kb) + weights + case["rows"] * n * 2, "flops": 2 * sent * n * k}
