"""The layer of experts in 8-bit blocks, with its balance, against 64-bit autograd of its definition, on the choices and the signs behind the ReLU that the library's rows lead to.

Tolerances, fixed before the first run: every operand of a product carries the rounding to e4m3, at most 2^-4 of an element and at most 2^-5 in the mean square, and the bf16 roundings of
2^-9.  A result has up to five of them behind it, independent of each other: under sqrt(5) 2^-5 + 2^-6 < 2^-3 of its 2-norm.  The loss follows from logits of rows in bf16: 2^-6.
"""
import math

import pytest
import torch

from paper_2210_06223_amd import expert_layer as L
from tests.test_expert_layer import far


def reference(layer, x, addend, experts, mask, passed=None):
    p = {n: getattr(layer, n).cpu().double().requires_grad_() for n in ("g", "R", "W1", "W2")}
    X = x.cpu().double().reshape(-1, layer.C).requires_grad_()
    s = X if addend is None else X + addend.cpu().double().reshape(-1, layer.C)
    h = s * torch.rsqrt(s.square().mean(-1, keepdim=True) + 1e-6) * p["g"]
    logits = h @ p["R"].t()
    there = torch.ones(len(h)) if mask is None else mask.cpu().double()
    e = experts.cpu().long()
    w = torch.softmax(torch.gather(logits, 1, e.clamp(min=0)), -1) * there[:, None]
    out = s
    for j in range(layer.k):
        mid = torch.einsum("tc,tmc->tm", h, p["W1"][e[:, j].clamp(min=0)])
        mid = torch.relu(mid) if passed is None else mid * passed[:, j]
        out = out + w[:, j:j + 1] * torch.einsum("tm,tcm->tc", mid, p["W2"][e[:, j].clamp(min=0)])
    counts, T = torch.bincount(e[e >= 0], minlength=layer.E).double(), max(1.0, float(there.sum()))
    share = (torch.softmax(logits, -1) * there[:, None]).sum(0) / T
    lse = torch.logsumexp(logits, -1) * there
    return X, p, out, torch.stack([layer.E * (counts / (layer.k * T) * share).sum(), (lse * lse).sum() / T]), counts


@pytest.mark.gpu
@pytest.mark.parametrize("shape,with_addend,masked", [((1,), False, False), ((37,), True, True), ((2, 5, 4), False, False), ((300,), False, True)])
def test_layer_in_blocks(shape, with_addend, masked, monkeypatch):
    layer = L.ExpertLayer(C=288, M=200, E=5, k=2, seed=4)
    layer.pack_blocks()
    g = torch.Generator().manual_seed(len(shape) + shape[0])
    make = lambda: torch.randn(*shape, layer.C, generator=g).bfloat16().cuda()
    x, dout, addend = make(), make(), make() if with_addend else None
    mask = (torch.rand(math.prod(shape), generator=g) > 0.3).cuda() if masked else None
    a = (3.0, 0.5)
    seen, mids, sums, choose, product, combine = [], [], [], L.B.lasnet_choose_experts, L.B.lasnet_block_product, L.B.lasnet_combine_rows
    monkeypatch.setattr(L.B, "lasnet_choose_experts", lambda *v, **k: seen.append(choose(*v, **k)) or seen[-1])
    monkeypatch.setattr(L.B, "lasnet_block_product", lambda *v, **k: mids.append(product(*v, **k)) or mids[-1])
    monkeypatch.setattr(L.B, "lasnet_combine_rows", lambda *v, **k: sums.append(v[1]) or combine(*v, **k))
    out, grads, loss, counts = layer.train_step_blocks(x, dout, addend, mask=mask, balance=a)
    position = sums[0].cpu().long()
    passed = (mids[0] > 0).cpu().double()[position.clamp(min=0)]            # [rows, k, M]
    X, p, ref, ref_loss, ref_counts = reference(layer, x, addend, seen[0][0], mask, passed)
    (ref * dout.cpu().double().reshape(-1, layer.C)).sum().add(a[0] * ref_loss[0] + a[1] * ref_loss[1]).backward()
    assert out.shape == x.shape and far(out, ref) < 2.0 ** -3
    assert counts.cpu().tolist()[:-1] == ref_counts.long().tolist() and int(counts[-1]) == (int(mask.sum()) if masked else len(position))
    assert ((loss.cpu().double() - ref_loss.detach()).abs() <= 2.0 ** -6 * ref_loss.detach().abs()).all()
    for name, want in (("x", X.grad), ("g", p["g"].grad), ("R", p["R"].grad), ("W1", p["W1"].grad), ("W2", p["W2"].grad)):
        assert far(grads[name], want) < 2.0 ** -3, name
    if masked:                                                              # what takes no part is passed through
        s = x if addend is None else (x.float() + addend.float()).bfloat16()
        assert torch.equal(out[~mask], s[~mask])
    served = layer.serve_blocks(x, addend, mask=mask)
    assert served.shape == x.shape and torch.equal(served, out), "the same calls forward"
