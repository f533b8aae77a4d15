"""The layer of experts against 64-bit autograd of its definition, on the choices that the library's rows lead to: which experts, and (for
gradients, where a sign that a rounding turns carries a whole gradient) which activations passed the ReLU.

Tolerances, fixed before the first run: every intermediate (h, mid, y, dy, dmid, drows, dh) is rounded to bf16 once, 2^-9 rms of it; a handful of such
roundings in a row stay under 2^-6 of the result's 2-norm.  8 bits: rows and W1 carry 2^-5 rms each at most, under 2^-4 together.
"""
import pytest
import torch

from paper_2210_06223_amd import expert_layer as L


def reference(layer, x, addend, experts, passed=None, dtype=torch.float64):
    p = {n: getattr(layer, n).cpu().to(dtype).requires_grad_() for n in ("g", "R", "W1", "W2")}
    X = x.cpu().to(dtype).reshape(-1, layer.C).requires_grad_()
    s = X if addend is None else X + addend.cpu().to(dtype).reshape(-1, layer.C)
    h = s * torch.rsqrt(s.square().mean(-1, keepdim=True) + 1e-6) * p["g"]
    chosen = torch.gather(h @ p["R"].t(), 1, experts.cpu().long())
    w = torch.softmax(chosen, -1)
    out = s
    for j in range(layer.k):
        e = experts[:, j].cpu().long()
        mid = torch.einsum("tc,tmc->tm", h, p["W1"][e])
        mid = torch.relu(mid) if passed is None else mid * passed[:, j]
        out = out + w[:, j:j + 1] * torch.einsum("tm,tcm->tc", mid, p["W2"][e])
    return X, p, out


def far(got, ref):
    ref = ref.detach()
    return float((got.detach().cpu().double().reshape(ref.shape) - ref).norm() / ref.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("shape,with_addend", [((1,), False), ((37,), True), ((2, 5, 4), False)])
def test_layer(shape, with_addend, monkeypatch):
    layer = L.ExpertLayer(C=96, M=80, E=5, k=2, seed=3)
    g = torch.Generator().manual_seed(len(shape))
    make = lambda: torch.randn(*shape, layer.C, generator=g).bfloat16().cuda()
    x, dout, addend = make(), make(), make() if with_addend else None
    seen = []
    choose = layer.choose
    layer.choose = lambda h: seen.append(choose(h)) or seen[-1]
    mids, sums, product, combine = [], [], L.B.lasnet_expert_product, L.B.lasnet_combine_rows
    monkeypatch.setattr(L.B, "lasnet_expert_product", lambda *a, **k: mids.append(product(*a, **k)) or mids[-1])
    monkeypatch.setattr(L.B, "lasnet_combine_rows", lambda *a, **k: sums.append(a[1]) or combine(*a, **k))
    out, grads = layer.train_step(x, dout, addend)
    passed = (mids[0] > 0).cpu().double()[sums[0].cpu().long()]             # [rows, k, M]
    X, p, ref = reference(layer, x, addend, seen[-1][0], passed)
    (ref * dout.cpu().double().reshape(-1, layer.C)).sum().backward()
    assert out.shape == x.shape and far(out, ref) < 2.0 ** -6
    for name, want in (("x", X.grad), ("g", p["g"].grad), ("R", p["R"].grad), ("W1", p["W1"].grad), ("W2", p["W2"].grad)):
        assert far(grads[name], want) < 2.0 ** -6, name
    served = layer.serve(x, addend)
    assert served.shape == x.shape and far(served, reference(layer, x, addend, seen[-1][0])[2]) < 2.0 ** -4
