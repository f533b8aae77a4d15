"""A layer of experts over rows, from the library's calls: norm, routing, two products, and the way back into the residual.

Rows are tokens, or the pixels of a feature map [N,H,W,C] (N*H*W rows as they lie in memory).  For every row r of the residual stream x (+ the addend that is due):

  s = x + addend;  h = s / rms(s) * g;  the k experts e of the largest logits h . R^T, weighted by the softmax of those k;
  out = s + sum_e w_e * (ReLU(h W1_e^T) W2_e^T)

serve() runs it with W1 in 8 bits (rows and weights e4m3, as lasnet_norm_rows and pack() write them) and W2 in bfloat16; train_step() in bfloat16, with all
gradients.  Both take any number of rows, one included.  The router's small product, top-k and softmax are torch's.

The router reads the rows as the experts do: in 8 bits in serve(), in bfloat16 in train_step(), so where two logits are closer than that rounding the two may choose
different experts for a row.

`python -m paper_2210_06223_amd.expert_layer` times both on synthetic rows.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import torch

from . import binding as B

_EPS = 1e-6


class ExpertLayer:
    """Weights: g [C] and R [E,C] float32; W1 [E,M,C], W2 [E,C,M] bfloat16."""

    def __init__(self, C: int, M: int, E: int, k: int, seed: int = 0, dev="cuda:0"):
        gen = torch.Generator().manual_seed(seed)
        r = lambda *shape, s: torch.randn(*shape, generator=gen).mul_(s)
        self.C, self.M, self.E, self.k = C, M, E, k
        self.g = (1.0 + r(C, s=0.1)).to(dev)
        self.R = r(E, C, s=C ** -0.5).to(dev)
        self.W1 = r(E, M, C, s=C ** -0.5).to(dev, torch.bfloat16)
        self.W2 = r(E, C, M, s=M ** -0.5).to(dev, torch.bfloat16)
        self.pack()

    def pack(self) -> None:
        """W1 in 8 bits for serve(), with a scale for each output column; to be called again after W1 has changed."""
        w = self.W1.float()
        self.w1_scale = (w.abs().amax(-1) / 448.0).clamp_(min=1e-30).contiguous()
        self.W1_8 = (w / self.w1_scale[..., None]).to(torch.float8_e4m3fn)

    def choose(self, h: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        """(experts int32 [rows,k], weights float32 [rows,k]) of normalised rows."""
        logits, experts = torch.topk(h.reshape(-1, self.C).float() @ self.R.t(), self.k, dim=-1)
        return experts.to(torch.int32), torch.softmax(logits, -1)

    def serve(self, x: torch.Tensor, addend: Optional[torch.Tensor] = None) -> torch.Tensor:
        q, scale, s = B.lasnet_norm_rows(x, self.g, _EPS, residual=addend, out_dtype=torch.float8_e4m3fn)
        h = q.reshape(-1, self.C).float() * scale.float()[:, None]
        experts, weights = self.choose(h)
        offsets, _, position = B.lasnet_route(experts, self.E)
        rows, rows_scale = B.lasnet_dispatch_rows(q, position, offsets, scale=scale)
        mid = B.lasnet_expert_product(rows, offsets, self.W1_8, scale=rows_scale, wscale=self.w1_scale, flags=B.LASNET_POST_RELU)
        y = B.lasnet_expert_product(mid, offsets, self.W2)
        return B.lasnet_combine_rows(y, position, weights=weights, base=x if s is None else s)

    def train_step(self, x: torch.Tensor, dout: torch.Tensor, addend: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Dict[str, torch.Tensor]]:
        """(out, gradients of x (and of the addend: the same), g, R, W1, W2) for the gradient dout of out."""
        rstd = torch.empty(x.numel() // self.C, device=x.device)
        h, _, s = B.lasnet_norm_rows(x, self.g, _EPS, residual=addend, rstd=rstd)
        s = x if s is None else s
        experts, weights = self.choose(h)
        offsets, _, position = B.lasnet_route(experts, self.E)
        rows, _ = B.lasnet_dispatch_rows(h, position, offsets)
        mid = B.lasnet_expert_product(rows, offsets, self.W1, flags=B.LASNET_POST_RELU)
        y = B.lasnet_expert_product(mid, offsets, self.W2)
        out = B.lasnet_combine_rows(y, position, weights=weights, base=s)

        dy, dweights = B.lasnet_combine_rows_backward(dout, y, position, offsets, weights=weights)
        grads = {"W2": B.lasnet_expert_product_dw(dy, mid, offsets, dtype=torch.float32)}
        dmid = B.lasnet_expert_product_dx(dy, offsets, self.W2)
        dmid.mul_(mid > 0)
        grads["W1"] = B.lasnet_expert_product_dw(dmid, rows, offsets, dtype=torch.float32)
        drows = B.lasnet_expert_product_dx(dmid, offsets, self.W1)
        # the router: softmax over the chosen logits, then its product
        dchosen = weights * (dweights - (dweights * weights).sum(-1, keepdim=True))
        dlogits = torch.zeros(dchosen.shape[0], self.E, device=x.device).scatter_(1, experts.long(), dchosen)
        grads["R"] = dlogits.t() @ h.reshape(-1, self.C).float()
        dh = B.lasnet_combine_rows(drows, position, base=(dlogits @ self.R).to(h.dtype))           # dispatch's gradient is the sum of the rows sent
        grads["x"], grads["g"] = B.lasnet_norm_rows_backward(dh.view(x.shape), s, self.g, rstd, dsum=dout)
        return out, grads


def _timed(f, n: int = 20) -> float:
    for _ in range(3):
        f()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    a.record()
    for _ in range(n):
        f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / n * 1e3


def main() -> None:
    layer = ExpertLayer(C=1024, M=1024, E=16, k=2)
    for rows in (1, 16, 196, 25088):                # one token, a small batch, one 14x14 map, 128 of them
        x = torch.randn(rows, layer.C, device="cuda").bfloat16()
        dout = torch.randn_like(x)
        print("%6d rows: serve %8.1f us, training step %8.1f us" % (rows, _timed(lambda: layer.serve(x)), _timed(lambda: layer.train_step(x, dout))), flush=True)


if __name__ == "__main__":
    main()
