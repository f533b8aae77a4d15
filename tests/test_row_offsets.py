"""Offsets that do not ascend or lie outside [0, rows], through every kernel of the products (few rows, a tile a workgroup with up to 62 experts and more, a
reduction shared by groups of waves, streaming tiles with up to 63 experts and more, rows through registers, dW in parts): no memory but the outputs and the workspace is
written, and offsets that ascend once they are cut to [0, rows] give the results of the cut ones, with NaN all around the inputs."""
import math

import numpy as np
import pytest
import torch

from paper_2210_06223_amd import binding as B

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
GUARD = 1 << 16                                                  # bytes around each tensor


def between(shape, dtype, fill, values=None):
    """A dense tensor in the middle of a buffer of bytes `fill`, and the buffer."""
    n = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
    n16 = (n + 15) // 16 * 16
    buffer = torch.full((2 * GUARD + n16,), fill, dtype=torch.uint8, device="cuda")
    t = buffer[GUARD:GUARD + n].view(dtype).view(shape)
    if values is not None:
        t.copy_(values)
    return t, (buffer, GUARD, n)


def untouched(guarded, fill, what):
    buffer, at, n = guarded
    assert (buffer[:at] == fill).all() and (buffer[at + n:] == fill).all(), what


def offsets_of(E, rows, seed):
    """name, offsets, whether they ascend once cut"""
    r = np.random.RandomState(seed)
    up = np.sort(r.randint(0, rows + 1, E + 1))
    low, high = up.copy(), up.copy()
    low[0], high[-1] = -2 ** 31, 2 ** 31 - 1
    if E > 3:
        low[1], high[-2] = -7, rows + 5
    yield "below", low, True
    yield "above", high, True
    yield "around", np.concatenate([[-5], up[1:-1], [rows + 1000]]), True
    yield "descending", up[::-1].copy(), False
    yield "to and fro", np.where(np.arange(E + 1) % 2, rows, 0), False
    yield "far to and fro", np.where(np.arange(E + 1) % 2, 2 ** 31 - 1, -2 ** 31), False
    yield "any", r.randint(-rows, 2 * rows + 1, E + 1), False


# rows, experts, n, k
SIZES = [(60, 3, 64, 128), (300, 4, 2048, 2048), (300, 3, 64, 2048), (700, 3, 64, 200), (4000, 5, 512, 136), (1000, 62, 128, 72), (900, 70, 200, 136), (5000, 6, 4096, 256), (2000, 70, 2048, 264),
         (300, 4, 67, 101), (64, 2, 3, 5), (500, 130, 33, 65)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,E,n,k", SIZES)
def test_products(rows, E, n, k):
    g = torch.Generator().manual_seed(rows + E)
    x, _ = between((rows, k), BF16, 255, torch.randn(rows, k, generator=g))       # (bytes 255: NaN in both types)
    W, _ = between((E, n, k), BF16, 255, torch.randn(E, n, k, generator=g))
    dy, _ = between((rows, n), BF16, 255, torch.randn(rows, n, generator=g))
    q, _ = between((rows, k), E4M3, 255, torch.randn(rows, k, generator=g))
    V, _ = between((E, n, k), E4M3, 255, torch.randn(E, n, k, generator=g))
    scale, _ = between((rows,), torch.uint8, 255, torch.randint(120, 130, (rows,), generator=g))
    wscale, _ = between((E, n), F32, 255, torch.rand(E, n, generator=g))
    calls = [("bf16", (rows, n), BF16, lambda o, out: B.lasnet_expert_product(x, o, W, out=out)),
             ("e4m3", (rows, n), BF16, lambda o, out: B.lasnet_expert_product(q, o, V, scale=scale, wscale=wscale, out=out)),
             ("dx", (rows, k), BF16, lambda o, out: B.lasnet_expert_product_dx(dy, o, W, dx=out)),
             ("dW", (E, n, k), BF16, lambda o, out: B.lasnet_expert_product_dw(dy, x, o, dW=out)),
             ("dW f32", (E, n, k), F32, lambda o, out: B.lasnet_expert_product_dw(dy, x, o, dW=out))]
    for name, o, ascends in offsets_of(E, rows, rows):
        given = torch.from_numpy(o.astype(np.int32)).cuda()
        cut = torch.from_numpy(np.clip(o, 0, rows).astype(np.int32)).cuda()
        for what, shape, dtype, call in calls:
            print("offsets", rows, E, n, k, name, what, flush=True)
            out, guarded = between(shape, dtype, 77)
            call(given, out)
            untouched(guarded, 77, (name, what))
            if ascends:
                want, guarded = between(shape, dtype, 77)
                call(cut, want)
                untouched(guarded, 77, (name, what, "cut"))
                first = 0 if what.startswith("dW") else int(cut[0])      # (rows ahead of the first expert's are not spoken of)
                assert torch.equal(out[first:], want[first:]), (name, what)
                assert torch.isfinite(out[first:].float()).all(), (name, what)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,E,n,k", [(13000, 2, 136, 200), (20000, 3, 64, 72)])
def test_weights_gradient_in_parts(rows, E, n, k):
    g = torch.Generator().manual_seed(rows)
    x, _ = between((rows, k), BF16, 255, torch.randn(rows, k, generator=g))
    dy, _ = between((rows, n), BF16, 255, torch.randn(rows, n, generator=g))
    need = B.lib().lasnet_expert_product_dw_workspace_bytes(rows, E, n, k)
    assert need > 0
    for name, o, ascends in offsets_of(E, rows, rows):
        given = torch.from_numpy(o.astype(np.int32)).cuda()
        cut = torch.from_numpy(np.clip(o, 0, rows).astype(np.int32)).cuda()
        for dtype in (BF16, F32):
            print("parts", rows, E, n, k, name, dtype, flush=True)
            out, guarded = between((E, n, k), dtype, 77)
            ws, beside = between((need,), torch.uint8, 255)
            B.lasnet_expert_product_dw(dy, x, given, dW=out, workspace=ws)
            untouched(guarded, 77, name)
            untouched(beside, 255, name)
            if ascends:
                want = torch.empty_like(out)
                B.lasnet_expert_product_dw(dy, x, cut, dW=want, workspace=ws)
                assert torch.equal(out, want) and torch.isfinite(out.float()).all(), name


@pytest.mark.gpu
def test_rows_that_are_moved():
    """Dispatch and the sum's gradient take the end of the rows sent from offsets[E], cut, and positions outside the rows as not sent."""
    tokens, k, E, cols = 50, 3, 4, 200
    g = torch.Generator().manual_seed(3)
    p = torch.randperm(tokens * k, generator=g).to(torch.int32).view(tokens, k)
    p[7], p[9, 1], p[20, 2] = -1, 2 ** 31 - 1, -2 ** 31
    p[30, 0] = tokens * k
    position = p.cuda()
    sent = (p >= 0) & (p < tokens * k)
    x = torch.randn(tokens, cols, generator=g).to(BF16).cuda()
    y, _ = between((tokens * k, cols), BF16, 255, torch.randn(tokens * k, cols, generator=g))
    for last in (-2 ** 31, -1, tokens * k, 2 ** 31 - 1):
        offsets = torch.tensor([0, 1, 2, 3, last], dtype=torch.int32).cuda()
        print("moved", last, flush=True)
        out, guarded = between((tokens * k, cols), BF16, 77)
        B.lasnet_dispatch_rows(x, position, offsets, out=out)
        untouched(guarded, 77, last)
        dy, guarded = between((tokens * k, cols), BF16, 77)
        dw, beside = between((tokens, k), F32, 77)
        B.lasnet_combine_rows_backward(x, y, position, offsets, dy=dy, dweights=dw)
        untouched(guarded, 77, last)
        untouched(beside, 77, last)
        assert (dw.cpu()[~sent] == 0).all() and torch.isfinite(dw).all()
        if last >= tokens * k:
            at = p[sent].long()
            assert torch.equal(out.cpu()[at], x.cpu()[torch.nonzero(sent)[:, 0]]) and torch.equal(dy.cpu()[at], x.cpu()[torch.nonzero(sent)[:, 0]])
    total, guarded = between((tokens, cols), BF16, 77)
    B.lasnet_combine_rows(y, position, out=total)
    untouched(guarded, 77, "sum")
    assert torch.isfinite(total.float()).all() and (total[7] == 0).all()
