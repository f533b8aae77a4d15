"""Scales of e4m3 products over their whole range: 0 to 254 (2^-127 to 2^127), 255 (NaN), with wscale from below fp32's normal numbers to near its end.

The products here are whole multiples of one power of two within an instruction's reach, so the matrix core's sums are exact.  Tolerance, fixed before the first
run: one rounding in fp32 and one to bf16 are within 2^-8 of the result; below the normal numbers, bf16's least step 2^-133.  From 2^128 on the result is infinite, between bf16's
largest number and that it may be either."""
import math

import pytest
import torch

from paper_2210_06223_amd import binding as B

E4M3 = torch.float8_e4m3fn
BYTES = [0, 1, 2, 64, 126, 127, 128, 190, 253, 254, 255]
WSCALE = [2.0 ** -140, 1e-38, 1e-30, 1e-6, 0.7, 0.0, 1.0, 4.0, -3.0, 1e6, 1e30, 3e38, math.inf, math.nan]

# rows, n, k, pad of x: few rows; rows through registers; a tile a workgroup; the reduction shared by groups of waves; 256 x 256 tiles
SIZES = [(60, 64, 128, 0), (60, 67, 100, 0), (700, 130, 144, 3), (700, 144, 144, 0), (300, 64, 2048, 0), (90, 512, 1024, 16), (5000, 4096, 256, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n,k,pad", SIZES)
def test_scales_of_the_whole_range(rows, n, k, pad):
    g = torch.Generator().manual_seed(rows + n + k)
    pick = lambda *shape: torch.where(torch.rand(*shape, generator=g) < 0.4, -1.0, 1.0) * torch.randint(1, 3, shape, generator=g)
    x, W = pick(rows, k), pick(2, n, k)                          # +-1, +-2 ...
    kind = torch.arange(rows) % 3                                # ... as +-224, +-448; +-2^-9, +-2^-8; zeros
    x = x * torch.tensor([224.0, 2.0 ** -9, 0.0])[kind][:, None]
    W = W * torch.tensor([224.0, 2.0 ** -9])[:, None, None]
    scale = torch.tensor(BYTES, dtype=torch.uint8)[torch.randint(0, len(BYTES), (rows,), generator=g)]
    wscale = torch.tensor(WSCALE, dtype=torch.float32)[torch.randint(0, len(WSCALE), (2, n), generator=g)]
    offsets = torch.tensor([0, rows // 2, rows - 5], dtype=torch.int32)
    store = torch.zeros(rows, k + pad, dtype=E4M3, device="cuda")
    store[:, :k] = x.to(E4M3).cuda()
    print("scales", rows, n, k, pad, flush=True)
    for with_w in (True, False):
        for with_s in (True, False):
            got = B.lasnet_expert_product(store[:, :k], offsets.cuda(), W.to(E4M3).cuda(), scale=scale.cuda() if with_s else None,
                                          wscale=wscale.cuda() if with_w else None).cpu().double()
            ref = torch.zeros(rows, n, dtype=torch.float64)
            factor = torch.exp2(scale.double() - 127) if with_s else torch.ones(rows, dtype=torch.float64)
            factor[scale == 255] = math.nan if with_s else 1.0
            for e in range(2):
                s = slice(int(offsets[e]), int(offsets[e + 1]))
                ref[s] = (x[s].double() @ W[e].double().T) * factor[s, None]
                if with_w:
                    ref[s] *= wscale[e].double()
            what = "wscale %s, scale %s" % (with_w, with_s)
            assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
            size = ref.abs()
            finite = size <= float(torch.finfo(torch.bfloat16).max)
            beyond = size >= 2.0 ** 128
            assert torch.equal(got[beyond], torch.sign(ref[beyond]) * math.inf), what
            bad = ~((got - ref).abs() <= 2.0 ** -8 * size + 2.0 ** -133) & finite
            assert not bad.any(), "%s: %d of %d off, first %s" % (what, int(bad.sum()), bad.numel(), [(float(got[bad][0]), float(ref[bad][0]))])
