"""The router's choice, the balance of the experts and the logits' gradient, against plain 64-bit definitions.

Tolerances, fixed before the first run.  u = 2^-24 is half a unit in the last place of fp32.  An exponential of a difference of two numbers of size up to m
carries the difference's rounding, m u, and a few units of its own (4 u); a sum of n such terms, all positive, in any order n u more; a quotient or product u each.
So a weight is within (m + n + 16) u of itself, an lse within (n + 8) u + (|lse| + 2 |top|) u, a mean probability within (m + 8) u (its sum is made in 64 bits), and a
gradient within (4 m + n + 32) u of the sum of the sizes of its terms.  A result is rounded to its type: half a unit, 2^-9 of it at least and at most 2^-8 in bf16, u in fp32.
"""
import math

import pytest
import torch

from paper_2210_06223_amd import binding as B
from tests.test_call_streams import CURRENT, SIDE, OnDevice, dev, made  # noqa: F401
from tests.test_row_operators import BF16, F32, HALF, U, close, f64, gen, rand

SHAPES = [(1, 1, 1), (1, 2, 1), (3, 5, 5), (7, 60, 2), (130, 64, 4), (65, 129, 16), (33, 256, 8), (9, 256, 33), (17, 513, 33), (5, 1030, 64), (3, 2500, 8), (3, 4096, 64), (1000, 8, 2),
          (70, 16, 20)]


def values(g, tokens, E, dtype, pad):
    """Logits, some of them equal."""
    t = rand(g, tokens, E, dtype=dtype, pad=pad, scale=2.0)
    return t.copy_((t.float() * 4).round() / 4) if E > 2 and dtype == F32 else t


def choose_ref(l, k, there, of_all):
    """experts, weights, lse and what the sums' sizes are, in 64 bits."""
    v = f64(l)
    T, E = v.shape
    experts, weights, lse = torch.full((T, k), -1, dtype=torch.int32), torch.zeros(T, k, dtype=torch.float64), torch.full((T,), -math.inf, dtype=torch.float64)
    for t in range(T):
        if not there[t]:
            continue
        rows = [(-(math.inf if math.isnan(x) else x), not math.isnan(x), e) for e, x in enumerate(v[t].tolist()) if math.isnan(x) or x > -math.inf]
        if not rows:
            continue
        best = [e for _, _, e in sorted(rows)][:k]
        experts[t, :len(best)] = torch.tensor(best, dtype=torch.int32)
        lse[t] = torch.logsumexp(v[t], 0)
        chosen = v[t][best]
        weights[t, :len(best)] = torch.exp(chosen - lse[t]) if of_all else torch.softmax(chosen, 0)
    return experts, weights, lse


@pytest.mark.gpu
@pytest.mark.parametrize("of_all", [False, True], ids=["chosen", "all"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_choice(dtype, of_all):
    for tokens, E, k in SHAPES:
        for pad in (0, 5):
            print("choose", tokens, E, k, dtype, of_all, pad, flush=True)
            g = gen(tokens * 7 + E)
            l = values(g, tokens, E, dtype, pad)
            mask = torch.rand(tokens, generator=g) > 0.2
            if tokens > 2:
                l[1] = -math.inf                                # a row without a candidate
                l[2, ::2] = -math.inf
            if pad:
                torch.as_strided(l, (tokens, E + pad), (E + pad, 1))[:, E:] = math.nan
            l[~mask.cuda()] = math.nan                         # what is masked may be anything
            experts, weights, lse = B.lasnet_choose_experts(l, k, mask=mask.cuda() if tokens % 2 else mask.to(torch.uint8).cuda(), flags=B.LASNET_WEIGHTS_OF_ALL if of_all else 0)
            want_e, want_w, want_l = choose_ref(l, k, mask, of_all)
            assert torch.equal(experts.cpu(), want_e)
            m = 2 * float(torch.nan_to_num(f64(l), 0.0, 0.0, 0.0).abs().max())
            close(weights, want_w, (m + E + 16) * U * want_w + 1e-38, "weights")
            assert torch.equal(torch.isinf(lse.cpu()), torch.isinf(want_l))
            fine = ~torch.isinf(want_l)
            close(f64(lse)[fine], want_l[fine], (E + 8) * U + (want_l[fine].abs() + m) * U, "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("E", [6, 70, 300, 1200])
def test_not_numbers_and_signed_zeros(E, dtype):
    l = torch.zeros(6, E, dtype=dtype)
    l[0, ::2] = -0.0                                           # equal to 0: the lowest numbers
    l[1] = -1.0
    l[1, E - 1], l[1, 3] = math.inf, math.nan
    l[2] = -math.inf
    l[2, 4] = -3.0e38
    l[3] = -math.inf
    l[4] = torch.finfo(dtype).min                              # the type's lowest values are candidates
    l[5, 2], l[5, 5] = 1e-40 if dtype == F32 else 1e-39, 2e-40 if dtype == F32 else 2e-39       # below the normal numbers
    experts, weights, lse = (t.cpu() for t in B.lasnet_choose_experts(l.cuda(), 3))
    assert experts.tolist() == [[0, 1, 2], [3, E - 1, 0], [4, -1, -1], [-1, -1, -1], [0, 1, 2], [5, 2, 0]]
    assert torch.isnan(weights[1]).all() and torch.isnan(lse[1])
    assert weights[2].tolist() == [1.0, 0.0, 0.0] and weights[3].tolist() == [0.0, 0.0, 0.0]
    assert lse[3] == -math.inf and math.isclose(float(lse[2]), float(l[2, 4]), rel_tol=1e-6)
    close(weights[[0, 4, 5]], torch.full((3, 3), 1 / 3, dtype=torch.float64), (E + 16) * U, "weights")


def balance_ref(l, lse, experts, k):
    """counts, share, loss of 64-bit logits and lse."""
    E = l.shape[1]
    there = lse > -math.inf
    T = int(there.sum())
    p = torch.exp(l[there] - lse[there][:, None])
    e = experts.reshape(-1)
    counts = torch.bincount(e[(e >= 0) & (e < E)].long(), minlength=E)
    if not T:
        return counts, T, torch.zeros(E, dtype=torch.float64), torch.zeros(2, dtype=torch.float64)
    share = p.sum(0) / T
    return counts, T, share, torch.stack([E * (counts.double() / (k * T) * share).sum(), (lse[there] ** 2).mean()])


def balance_inputs(tokens, E, k, dtype, pad):
    g = gen(tokens * 3 + E)
    l = rand(g, tokens, E, dtype=dtype, pad=pad, scale=2.0)
    mask = (torch.rand(tokens, generator=g) > 0.2).cuda()
    l[~mask] = math.nan
    experts, weights, lse = B.lasnet_choose_experts(l, k, mask=mask)
    if tokens > 5:
        experts[3] = experts[3, 0].item()                      # an expert twice, and none
        experts[4, 0] = E + 3
        experts[5, -1] = -7
    return g, l, experts, weights, lse


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_balance(dtype):
    for tokens, E, k in SHAPES + [(20000, 24, 2), (70000, 3, 1), (5000, 300, 6)]:
        for pad in (0, 3):
            print("balance", tokens, E, k, dtype, pad, flush=True)
            _, l, experts, _, lse = balance_inputs(tokens, E, k, dtype, pad)
            counts, share, loss = B.lasnet_balance(l, lse, experts)
            want_c, T, want_s, want_l = balance_ref(f64(l), f64(lse), experts.cpu(), k)
            assert counts.cpu().tolist() == want_c.tolist() + [T]
            m = float(torch.nan_to_num(f64(l), 0.0).abs().max()) * 2
            close(share, want_s, (2 * m + 8) * U * want_s + 1e-38, "share")
            close(loss, want_l, (2 * m + 10) * U * want_l + 1e-38, "loss")
            again = B.lasnet_balance(l, lse, experts)
            assert all(torch.equal(a, b) for a, b in zip((counts, share, loss), again)), "twice the same bits"


@pytest.mark.gpu
def test_balance_of_nothing():
    l = torch.full((5, 7), math.nan, device="cuda")
    for rows in (0, 5):
        experts, weights, lse = B.lasnet_choose_experts(l[:rows], 2, mask=torch.zeros(rows, dtype=torch.uint8, device="cuda"))
        assert (experts == -1).all() and (weights == 0).all() and (lse == -math.inf).all()
        counts, share, loss = B.lasnet_balance(l[:rows], lse, experts)
        assert (counts == 0).all() and (share == 0).all() and (loss == 0).all()
        d = B.lasnet_choose_experts_backward(l[:rows], lse, experts, weights, dweights=torch.ones(rows, 2, device="cuda"), counts=counts, dloss=torch.ones(2, device="cuda"))
        assert (d == 0).all() and d.shape == (rows, 7)


def grad_ref(l, lse, experts, weights, dweights, counts, dloss, of_all):
    """The header's formula in 64 bits, and the sum of the sizes of its terms."""
    (T, E), k = l.shape, experts.shape[1]
    there = lse > -math.inf
    p = torch.where(there[:, None], torch.exp(torch.where(there[:, None], l - lse[:, None], 0.0)), 0.0)
    d, size = torch.zeros_like(p), torch.zeros_like(p)
    if dloss is not None:
        n = max(1, int(counts[E]))
        c = dloss[0] * E * counts[:E].double() / (k * n * n)
        z = torch.where(there, 2 * dloss[1] * torch.where(there, lse, 0.0) / n, 0.0)[:, None]
        d = p * (c - (p * c).sum(1, keepdim=True)) + p * z
        size = p * (c.abs() + (p * c.abs()).sum(1, keepdim=True)) + p * z.abs()
    if dweights is not None:
        s, sa = ((f(weights * dweights)).sum(1, keepdim=True) for f in (lambda v: v, torch.abs))
        if of_all:
            d, size = d - p * s, size + p * sa
        for t in range(T):
            for j in range(k):
                e = int(experts[t, j])
                if there[t] and 0 <= e < E:
                    w = weights[t, j]
                    d[t, e] += w * (dweights[t, j] - (0 if of_all else s[t, 0]))
                    size[t, e] += w * (dweights[t, j].abs() + (0 if of_all else sa[t, 0]))
    return d, size


@pytest.mark.gpu
@pytest.mark.parametrize("of_all", [False, True], ids=["chosen", "all"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_gradient(dtype, of_all):
    for tokens, E, k in SHAPES:
        for pad, parts in ((0, "wb"), (5, "w"), (0, "b")):
            print("gradient", tokens, E, k, dtype, of_all, pad, parts, flush=True)
            g, l, experts, weights, lse = balance_inputs(tokens, E, k, dtype, pad)
            counts, _, _ = B.lasnet_balance(l, lse, experts)
            dw = rand(g, tokens, k) if "w" in parts else None
            dloss = torch.tensor([0.7, -0.3]).cuda() if "b" in parts else None
            flags = B.LASNET_WEIGHTS_OF_ALL if of_all else 0
            if of_all:
                _, weights, _ = B.lasnet_choose_experts(l, k, mask=lse > -math.inf, flags=flags)
            d = B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=dw, counts=counts if "b" in parts else None, dloss=dloss, flags=flags)
            ref, size = grad_ref(f64(l), f64(lse), experts.cpu(), f64(weights), None if dw is None else f64(dw), counts.cpu(), None if dloss is None else f64(dloss), of_all)
            m = 2 * float(torch.nan_to_num(f64(l), 0.0).abs().max())
            close(d, ref, HALF[dtype] * ref.abs() + (4 * m + E + 32) * U * size + 1e-38, "dlogits")
            held = torch.full((tokens, E + 4), 9.0, dtype=dtype, device="cuda")             # in place, and apart
            held[:, :E] = l
            B.lasnet_choose_experts_backward(held[:, :E], lse, experts, weights, dweights=dw, counts=counts if "b" in parts else None, dloss=dloss, dlogits=held[:, :E], flags=flags)
            assert torch.equal(held[:, :E], d) and (held[:, E:] == 9.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("of_all", [False, True], ids=["chosen", "all"])
def test_gradient_against_differences(of_all):
    """Of the 64-bit definition's loss = dloss . loss + dweights . weights (counts held), at a step of 1e-4: the quotient's error is of the order of the step squared and 1e-16 over
    the step, under 1e-7."""
    g = gen(11)
    tokens, E, k = 12, 9, 3
    l, dw, dloss = rand(g, tokens, E), rand(g, tokens, k), torch.tensor([1.3, 0.4]).cuda()
    flags = B.LASNET_WEIGHTS_OF_ALL if of_all else 0
    experts, weights, lse = B.lasnet_choose_experts(l, k, flags=flags)
    counts, _, _ = B.lasnet_balance(l, lse, experts)
    d = f64(B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=dw, counts=counts, dloss=dloss, flags=flags))
    e, D, W = experts.cpu().long(), f64(dloss), f64(dw)

    def value(v):
        s = torch.logsumexp(v, 1)
        w = torch.gather(v, 1, e)
        w = torch.exp(w - s[:, None]) if of_all else torch.softmax(w, 1)
        share = torch.softmax(v, 1).mean(0)
        return D[0] * E * (counts.cpu()[:E].double() / (k * tokens) * share).sum() + D[1] * (s * s).mean() + (W * w).sum()

    v, h = f64(l), 1e-4
    for t in range(tokens):
        for i in range(E):
            up, down = v.clone(), v.clone()
            up[t, i] += h
            down[t, i] -= h
            assert abs(float(value(up) - value(down)) / (2 * h) - float(d[t, i])) < 1e-7 + 64 * U * 4


@pytest.mark.gpu
@pytest.mark.parametrize("of_all", [False, True], ids=["chosen", "all"])
def test_slots_without_weight_add_nothing(of_all):
    """What a slot of expert -1 is given (a token with fewer candidates than slots: nothing ever writes there) reaches no gradient, NaN included."""
    for tokens, E, k in ((7, 5, 8), (3, 40, 20), (4, 20, 33)):
        g = gen(tokens)
        l = rand(g, tokens, E)
        l[0, 2:] = -math.inf
        l[2] = -math.inf
        flags = B.LASNET_WEIGHTS_OF_ALL if of_all else 0
        experts, weights, lse = B.lasnet_choose_experts(l, k, flags=flags)
        dw = rand(g, tokens, k)
        want = B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=dw.masked_fill(experts < 0, 0.0), flags=flags)
        assert torch.isfinite(want).all() and bool((experts < 0).any())
        for other in (math.nan, math.inf):
            assert torch.equal(B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=dw.masked_fill(experts < 0, other), flags=flags), want)


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    """Two graphs, each with a workspace of its own, replayed in turn on new inputs with other work between; and the calls on a stream of their own."""
    tokens, E, k = 3000, 40, 4
    g = gen(5)
    new = lambda: rand(g, tokens, E, dtype=BF16)
    dloss = torch.tensor([0.5, 0.1]).cuda()

    def path(l, dw, stream=None):
        experts, weights, lse = B.lasnet_choose_experts(l, k, stream=stream)
        counts, share, loss = B.lasnet_balance(l, lse, experts, stream=stream)
        return [experts, weights, lse, counts, share, loss, B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=dw, counts=counts, dloss=dloss, stream=stream)]

    dw = rand(g, tokens, k)
    held = [new(), new()]
    side = torch.cuda.Stream()
    path(held[0], dw)
    torch.cuda.synchronize()
    graphs = []
    for l in held:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = path(l, dw)
        graphs.append((graph, out))
    for _ in range(3):
        for l in held:
            l.copy_(new())
        for graph, _ in graphs:
            graph.replay()
        got = [[t.clone() for t in out] for _, out in graphs]
        torch.cuda.synchronize()
        for l, have in zip(held, got):
            want = path(l, dw)
            other = path(l, dw, side)
            side.synchronize()
            assert all(torch.equal(a, b) and torch.equal(c, b) for a, b, c in zip(have, want, other))


# ---------------------------------------------------------------- what is refused (no GPU)

def call(name, *args):
    return getattr(B.lib(), "lasnet_" + name)(*args)


def on_device(monkeypatch):
    """What a call makes is taken for device memory, too."""
    real = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: real(*a, **k).as_subclass(OnDevice))


def rows(n, cols, dtype, at=0x1000, stride=0):
    return B.lasnet_rows(at, n, stride, cols, dtype)


def test_arguments_that_are_refused():
    P = 0x10000
    ref = lambda r: None if r is None else B.ctypes.byref(r)

    def choose(l=rows(4, 8, B.LASNET_F32), k=2, e=P, w=2 * P, lse=3 * P, flags=0, mask=None):
        return call("choose_experts", ref(l), mask, k, e, w, lse, flags, None)
    assert choose(l=None) == B.LASNET_EINVAL and choose(k=0) == B.LASNET_EINVAL and choose(flags=1) == B.LASNET_EINVAL
    assert choose(e=None) == B.LASNET_EINVAL and choose(w=None) == B.LASNET_EINVAL
    assert choose(k=65) == B.LASNET_EUNSUPPORTED and choose(l=rows(4, 4097, B.LASNET_F32)) == B.LASNET_EUNSUPPORTED
    assert choose(l=rows(4, 8, B.LASNET_E4M3)) == B.LASNET_EUNSUPPORTED and choose(l=rows(1 << 30, 8, B.LASNET_F32)) == B.LASNET_EUNSUPPORTED
    assert choose(l=rows(-1, 8, B.LASNET_F32)) == B.LASNET_ESHAPE and choose(l=rows(4, 8, B.LASNET_F32, stride=7)) == B.LASNET_ESHAPE

    def balance(l=rows(4, 8, B.LASNET_F32), lse=P, e=2 * P, k=2, c=3 * P, s=4 * P, loss=5 * P, ws=None, size=0):
        return call("balance", ref(l), lse, e, k, c, s, loss, ws, size, None)
    assert balance(c=None) == balance(s=None) == balance(loss=None) == balance(lse=None) == balance(e=None) == B.LASNET_EINVAL
    many = rows(100000, 8, B.LASNET_F32)
    need = B.lib().lasnet_balance_workspace_bytes(100000, 8)
    assert need > 0 and B.lib().lasnet_balance_workspace_bytes(4, 8) == 0 and B.lib().lasnet_balance_workspace_bytes(4, 5000) == 0
    assert balance(l=many) == balance(l=many, ws=6 * P, size=need - 1) == balance(l=many, ws=6 * P + 128, size=need) == B.LASNET_EINVAL
    assert balance(k=0) == B.LASNET_EINVAL

    def back(l=rows(4, 8, B.LASNET_F32), lse=P, e=2 * P, w=3 * P, k=2, dw=4 * P, c=5 * P, dl=6 * P, d=rows(4, 8, B.LASNET_F32, 7 * P), flags=0):
        return call("choose_experts_backward", ref(l), lse, e, w, k, dw, c, dl, ref(d), flags, None)
    assert back(lse=None) == back(e=None) == back(w=None) == back(c=None) == back(flags=2) == back(d=None) == B.LASNET_EINVAL
    assert back(d=rows(4, 8, B.LASNET_BF16, 7 * P)) == back(d=rows(5, 8, B.LASNET_F32, 7 * P)) == B.LASNET_ESHAPE
    assert back(d=rows(4, 8, B.LASNET_F32, 0x1000, stride=16)) == B.LASNET_EALIAS         # in place is the same rows, not the same address


def test_tensors_that_are_refused(monkeypatch):
    on_device(monkeypatch)
    l, e, w, lse = dev(4, 8), dev(4, 2, dtype=torch.int32), dev(4, 2), dev(4)
    with pytest.raises(ValueError, match="rows"):
        B.lasnet_choose_experts(dev(8), 2)
    with pytest.raises(ValueError, match="mask"):
        B.lasnet_choose_experts(l, 2, mask=dev(3, dtype=torch.uint8))
    with pytest.raises(ValueError, match="mask"):
        B.lasnet_choose_experts(l, 2, mask=dev(4))
    with pytest.raises(ValueError, match="experts"):
        B.lasnet_choose_experts(l, 2, experts=dev(4, 3, dtype=torch.int32))
    with pytest.raises(ValueError, match="weights"):
        B.lasnet_choose_experts(l, 2, weights=dev(4, 2, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="lse"):
        B.lasnet_balance(l, dev(5), e)
    with pytest.raises(ValueError, match="experts"):
        B.lasnet_balance(l, lse, dev(8, dtype=torch.int32))
    with pytest.raises(ValueError, match="experts"):
        B.lasnet_balance(l, lse, dev(5, 2, dtype=torch.int32))
    with pytest.raises(ValueError, match="counts"):
        B.lasnet_balance(l, lse, e, counts=dev(8, dtype=torch.int32))
    with pytest.raises(ValueError, match="counts"):
        B.lasnet_choose_experts_backward(l, lse, e, w, counts=dev(8, dtype=torch.int32), dloss=dev(2))
    with pytest.raises(ValueError, match="dloss"):
        B.lasnet_choose_experts_backward(l, lse, e, w, counts=dev(9, dtype=torch.int32), dloss=dev(3))
    with pytest.raises(ValueError, match="dweights"):
        B.lasnet_choose_experts_backward(l, lse, e, w, dweights=dev(4, 3))


# (see test_row_arguments.py)
F, H, Q = B.LASNET_F32, B.LASNET_BF16, B.LASNET_E4M3
ENTRIES = {
    "choose_experts": ([("logits", "ri", 8, 16, F), ("mask", "i"), 2, ("experts", "o"), ("weights", "o"), ("lse", "o"), 0, None], set()),
    "balance": ([("logits", "ri", 30000, 16, F), ("lse", "i"), ("experts", "i"), 2, ("counts", "o"), ("share", "o"), ("loss", "o"), ("workspace", "o"), 1 << 24, None], set()),
    "choose_experts_backward": ([("logits", "ri", 8, 16, F), ("lse", "i"), ("experts", "i"), ("weights", "i"), 2, ("dweights", "i"), ("counts", "i"), ("dloss", "i"),
                                 ("dlogits", "ro", 8, 16, F), 0, None], {("dlogits", "logits")}),
    "quantize_rows": ([("x", "ri", 8, 16, H), ("position", "i"), ("offsets", "i"), 2, 4, ("out", "ro", 16, 16, Q), ("scale", "o"), None], set()),
    "quantize_matrices": ([("W", "i"), F, 2, 16, 32, ("out", "o"), ("scale", "o"), ("out_t", "o"), ("scale_t", "o"), None], set()),
    "block_product": ([("x", "ri", 8, 16, Q), ("scale", "i"), ("offsets", "i"), 2, ("W", "i"), ("wscale", "i"), B.LASNET_E8M0, ("out", "ro", 8, 16, H), 0, None], set()),
}


def test_an_output_at_the_address_of_another_argument_is_refused(monkeypatch):
    from tests import test_row_arguments
    monkeypatch.setattr(test_row_arguments, "ENTRIES", ENTRIES)
    test_row_arguments.test_an_output_at_the_address_of_another_argument_is_refused()


def test_a_workspace_in_other_memory_is_refused(monkeypatch):
    from tests.test_row_arguments import Recording
    L, real = Recording(), torch.empty
    monkeypatch.setattr(B, "_lib", L)
    monkeypatch.setattr(B, "_marshal", B._AllThroughCtypes)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: real(*a, **k).as_subclass(OnDevice))
    l, lse, e = dev(6, 8), dev(6), dev(6, 2, dtype=torch.int32)
    for kw in (dict(), dict(counts=dev(9, dtype=torch.int32), share=dev(8), loss=dev(2))):
        for ws in (torch.zeros(4096, dtype=torch.uint8), torch.zeros(4096, dtype=torch.uint8, device="meta").as_subclass(OnDevice), dev(64, 128, dtype=torch.uint8)[:, ::2]):
            with pytest.raises(ValueError, match="workspace"):
                B.lasnet_balance(l, lse, e, workspace=ws, **kw)
        assert not L.enqueued
        B.lasnet_balance(l, lse, e, workspace=dev(4096, dtype=torch.uint8), **kw)
        assert L.enqueued.pop() == "lasnet_balance"


def calls(k):
    """name, the call, how many outputs and workspaces it makes"""
    l, lse, e, w = dev(6, 8), dev(6), dev(6, 2, dtype=torch.int32), dev(6, 2)
    yield "choose", lambda: B.lasnet_choose_experts(l, 2, **k), 3, 0
    yield "balance", lambda: B.lasnet_balance(l, lse, e, **k), 3, 1
    yield "backward", lambda: B.lasnet_choose_experts_backward(l, lse, e, w, dweights=w, **k), 1, 0


@pytest.mark.parametrize("which", range(3))
def test_what_a_call_makes_is_memory_of_its_stream(which, made):
    for given in (None, CURRENT, SIDE):
        name, run, outputs, workspaces = list(calls({} if given is None else {"stream": given}))[which]
        made.clear()
        run()
        assert [s for _, s in made] == [given or CURRENT] * (outputs + workspaces), name
        assert [getattr(t, "used_on", []) for t, _ in made] == [[CURRENT] if given is SIDE else []] * outputs + [[]] * workspaces, name


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Of bytes and of elements: 1.1 M tokens of 4096 experts in fp32, the last of which are compared with the same tokens by themselves."""
    tokens, E, k, last = 1100000, 4096, 4, 257
    l = torch.empty(tokens, E, device="cuda")
    l[:] = torch.randn(1000, E, generator=gen(1)).cuda().repeat(1100, 1)
    l[-last:] = torch.randn(last, E, generator=gen(2)).cuda()
    experts, weights, lse = B.lasnet_choose_experts(l, k)
    few = B.lasnet_choose_experts(l[-last:].clone(), k)
    for a, b in zip((experts, weights, lse), few):
        assert torch.equal(a[-last:], b) and torch.equal(a[:1000], a[1000:2000])
    counts, share, loss = B.lasnet_balance(l, lse, experts)
    assert int(counts[E]) == tokens and int(counts[:E].sum()) == tokens * k
    rest = torch.bincount(experts.flatten().long(), minlength=E).int()
    assert torch.equal(counts[:E], rest) and abs(float(share.double().sum()) - 1) < E * U
    dw = torch.randn(tokens, k, generator=gen(3)).cuda()
    d = B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=dw, dlogits=l)
    # (in place: what it read is gone)
    assert torch.equal(d[-last:], B.lasnet_choose_experts_backward(torch.randn(last, E, generator=gen(2)).cuda(), lse[-last:].clone(), experts[-last:].clone(), weights[-last:].clone(),
                                                                   dweights=dw[-last:].clone()))


@pytest.mark.gpu
@pytest.mark.parametrize("E", [7, 8, 31, 32, 33, 64, 65, 257, 340, 512, 513, 1000, 1024, 1025, 2048, 2049])
def test_every_number_of_lanes(E, monkeypatch):
    """Widths on both sides of where a token gets twice the lanes, through all three calls."""
    import tests.test_router as module
    monkeypatch.setattr(module, "SHAPES", [(37, E, k) for k in (1, 3, 7)] + ([(300, E, 8), (37, E, 9)] if E > 8 else []))
    for dtype in (F32, BF16):
        test_choice(dtype, E % 2 == 0)
        test_balance(dtype)
        test_gradient(dtype, E % 2 == 0)


# ---------------------------------------------------------------- slots dropped after the choice

@pytest.mark.gpu
@pytest.mark.parametrize("of_all", [False, True], ids=["chosen", "all"])
@pytest.mark.parametrize("tokens,E,k", [(12, 9, 3), (5, 70, 20), (3, 40, 33)])
def test_gradient_with_dropped_slots_against_differences(tokens, E, k, of_all):
    """The way of a layer with capacities: the list with -1 in the dropped slots' places goes to lasnet_route and lasnet_balance, the list as it was chosen to the gradient, with the dweights that
    lasnet_combine_rows_backward writes (0 for a dropped slot).  Against differences of the 64-bit loss = dloss . loss + dout . out (counts held), where a dropped slot's logit is in the sum that
    the weights are shares of.  At a step of 1e-4 the quotient is within 1e-6 (third derivatives of less than 100, a sixth of them times the step squared; terms of 1e2 and 1e-16 of them over the step); fp32: dweights
    carry C + 2 u and the gradient 4 m + E + 32 u of its terms, together at most w (|dweights| + |s|), so twice the largest of dweights, and the balance's, under 4 here."""
    g, C = gen(tokens + E), 4
    l, dloss = rand(g, tokens, E), torch.tensor([1.3, 0.4]).cuda()
    y, dout = rand(g, tokens * k, C), rand(g, tokens, C)
    flags = B.LASNET_WEIGHTS_OF_ALL if of_all else 0
    experts, weights, lse = B.lasnet_choose_experts(l, k, flags=flags)
    dropped = (torch.rand(tokens, k, generator=g) < 0.3)
    dropped[0, 0] = True
    sent = experts.masked_fill(dropped.cuda(), -1)
    counts, _, _ = B.lasnet_balance(l, lse, sent)
    offsets, _, position = B.lasnet_route(sent, E)
    _, dweights = B.lasnet_combine_rows_backward(dout, y, position, offsets, weights=weights)
    assert (dweights.view(tokens, k).cpu()[dropped] == 0).all()
    d = f64(B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=dweights, counts=counts, dloss=dloss, flags=flags))
    e, p, D, Y, G = experts.cpu().long(), position.cpu().long(), f64(dloss), f64(y), f64(dout)
    rows_ = Y[p.clamp(min=0)] * (~dropped)[..., None]
    n = counts.cpu()[:E].double()

    def value(v):
        s = torch.logsumexp(v, 1)
        w = torch.gather(v, 1, e)
        w = torch.exp(w - s[:, None]) if of_all else torch.softmax(w, 1)
        return D[0] * E * (n / (k * tokens) * torch.softmax(v, 1).mean(0)).sum() + D[1] * (s * s).mean() + (G * (w[..., None] * rows_).sum(1)).sum()

    v, h = f64(l), 1e-4
    slack = 1e-6 + (8 * float(v.abs().max()) + E + 64) * U * (2 * float(f64(dweights).abs().max()) + 4)
    for t in range(tokens):
        for i in range(E):
            up, down = v.clone(), v.clone()
            up[t, i] += h
            down[t, i] -= h
            assert abs(float(value(up) - value(down)) / (2 * h) - float(d[t, i])) < slack, (t, i)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_what_a_slot_without_an_expert_leaves_out(dtype):
    """A slot of weight w whose expert is given as -1 leaves w (dweights - s) out of its logit's gradient (so the row of the weights' part does not add up to zero), and nothing else."""
    for tokens, E, k in ((40, 9, 3), (9, 70, 20), (5, 40, 33)):
        g = gen(tokens + 2 * E)
        l, dw = rand(g, tokens, E, dtype=dtype), rand(g, tokens, k)
        experts, weights, lse = B.lasnet_choose_experts(l, k)
        dropped = torch.rand(tokens, k, generator=g) < 0.4
        dw[dropped.cuda()] = 0.0
        whole = f64(B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=dw))
        given = f64(B.lasnet_choose_experts_backward(l, lse, experts.masked_fill(dropped.cuda(), -1), weights, dweights=dw))
        w, s = f64(weights), (f64(weights) * f64(dw)).sum(1, keepdim=True)
        left = torch.zeros(tokens, E + 1, dtype=torch.float64)
        left.scatter_(1, torch.where(dropped, experts.cpu().long(), E), -w * s)
        size = w.max() * (f64(dw).abs() * w).sum(1, keepdim=True)
        # (the terms' sizes; each side is rounded once to its type)
        close(whole - given, left[:, :E], HALF[dtype] * (1 + 2 ** -7) * (whole.abs() + given.abs()) + (k + 40) * U * (size + whole.abs()) + 1e-38, "left out")
        close(whole.sum(1), torch.zeros(tokens, dtype=torch.float64), HALF[dtype] * (1 + 2 ** -7) * whole.abs().sum(1) + (E + 40) * U * (size[:, 0] * k + whole.abs().sum(1)) + 1e-38, "sum of a row")


# ---------------------------------------------------------------- logits of more than two dimensions

def test_a_workspace_for_logits_of_any_dimensions(monkeypatch):
    """Where the outputs are given and no workspace, one is made for as many tokens as the logits have rows, in two dimensions or four."""
    asked, got = [], []

    class Library:
        at_balance = 0

        def lasnet_balance_workspace_bytes(self, tokens, E):
            asked.append((tokens, E))
            return 512

    class Marshal:
        @staticmethod
        def balance(at, logits, lse, experts, counts, share, loss, workspace):
            got.append(workspace)
            return 0

    monkeypatch.setattr(B, "lib", Library)
    monkeypatch.setattr(B, "_marshal", Marshal)
    outputs = dict(counts=dev(9, dtype=torch.int32), share=dev(8), loss=dev(2))
    for shape in ((6, 8), (2, 3, 8), (1, 3, 2, 8)):
        B.lasnet_balance(dev(*shape), dev(6), dev(6, 2, dtype=torch.int32), **outputs)
        assert asked.pop() == (6, 8) and got.pop().numel() == 512, shape
    for shape in ((), (8,), (6, 0)):                           # (no rows: refused behind, not here)
        B.lasnet_balance(dev(*shape), dev(6), dev(6, 2, dtype=torch.int32), **outputs)
        assert not asked and got.pop() is None, shape


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [2 * 8 * 16, 2 * 32 * 32], ids=["one workgroup", "many"])
def test_logits_of_four_dimensions(tokens):
    """[N, H, W, E] through the three calls, outputs given or not, on both sides of where the balance needs a workspace: the same bits as [N H W, E]."""
    E, k, g = 24, 2, gen(tokens)
    l, dloss = rand(g, tokens, E), torch.tensor([0.5, 0.1]).cuda()
    assert (B.lib().lasnet_balance_workspace_bytes(tokens, E) > 0) == (tokens > 1000)

    def path(l, given):
        new = lambda *s, dtype=F32: torch.empty(*s, dtype=dtype, device="cuda") if given else None
        experts, weights, lse = B.lasnet_choose_experts(l, k, experts=new(tokens, k, dtype=torch.int32), weights=new(tokens, k), lse=new(tokens))
        balance = B.lasnet_balance(l, lse, experts, counts=new(E + 1, dtype=torch.int32), share=new(E), loss=new(2))
        d = B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=weights, counts=balance[0], dloss=dloss, dlogits=torch.empty_like(l) if given else None)
        assert d.shape == l.shape
        return [experts, weights, lse, *balance, d.reshape(tokens, E)]

    want = path(l, False)
    for shape in ((tokens, E), (2, -1, E), (2, -1, 16, E)):
        for given in (False, True):
            assert all(torch.equal(a, b) for a, b in zip(path(l.view(shape), given), want)), (shape, given)


@pytest.mark.gpu
@pytest.mark.parametrize("of_all", [False, True], ids=["chosen", "all"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_tokens_that_take_no_part_get_zeros_whatever_the_loss_is(dtype, of_all):
    """An infinite or NaN gradient of the loss (an overflow of a scaled one), logits and dweights that are NaN: zeros for a token whose lse is -inf, also beside others in its wave."""
    for tokens, E, k in ((50, 8, 2), (50, 60, 2), (9, 200, 6), (7, 500, 8), (5, 1000, 33), (3, 4000, 4)):
        g = gen(E)
        l, dw = rand(g, tokens, E, dtype=dtype), rand(g, tokens, k)
        mask = torch.arange(tokens) % 3 != 1
        l[~mask.cuda()] = math.nan
        dw[~mask.cuda()] = math.nan
        flags = B.LASNET_WEIGHTS_OF_ALL if of_all else 0
        experts, weights, lse = B.lasnet_choose_experts(l, k, mask=mask.cuda(), flags=flags)
        counts, _, _ = B.lasnet_balance(l, lse, experts)
        for dloss in ((math.inf, 0.1), (math.nan, 0.1), (0.1, math.inf), (0.1, math.nan), (-math.inf, math.inf)):
            d = B.lasnet_choose_experts_backward(l, lse, experts, weights, dweights=dw, counts=counts, dloss=torch.tensor(dloss).cuda(), flags=flags)
            assert (d[~mask.cuda()] == 0).all(), (tokens, E, k, dloss)
            assert not torch.isfinite(d[mask.cuda()].float()).all()


# ---------------------------------------------------------------- what the header promises of sums and of tokens that take no part

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_sums_over_tokens_keep_what_32_bits_lose(dtype):
    """A quarter (or one) of the tokens has p = 1, the others about 2^-25, less than half a unit of it: in 64 bits the small ones count, in 32 they would vanish next to a 1.  The bound: of the
    small ones' own exponentials 16 u of them, and the rounding of share, u."""
    for E, tokens in ((2, 256), (2, 4096), (60, 1024), (200, 512), (500, 64), (1500, 40), (4000, 16), (2, 40000)):
        small = -17.25                                         # e^-17.25 = 1.08 2^-25, exact in bf16
        for first in (tokens // 4, 1):
            print("sums", E, tokens, first, dtype, flush=True)
            l = torch.full((tokens, E), small, dtype=dtype, device="cuda")
            l[:first] = 0.0
            lse, experts = torch.zeros(tokens, device="cuda"), torch.zeros(tokens, 1, dtype=torch.int32, device="cuda")
            _, share, loss = B.lasnet_balance(l, lse, experts)
            low = (tokens - first) * math.exp(small) / tokens
            want = first / tokens + low
            assert (f64(share) - want).abs().max() <= U * want + 16 * U * low, (E, tokens, first, float(share[0]) - want)
            assert abs(float(loss[0]) - E * want) <= 2 * U * E * want + 16 * U * E * low
