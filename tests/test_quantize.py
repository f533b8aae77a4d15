"""Rows and matrices in 8 bits with scales for blocks of 128: bit for bit (the scale is exact, the division by a power of two, too, and one rounding to nearest even is left)."""
import math

import numpy as np
import pytest
import torch

from paper_2210_06223_amd import binding as B
from tests.test_call_streams import CURRENT, SIDE, dev, made  # noqa: F401
from tests.test_router import call, on_device, rows
from tests.test_row_operators import BF16, E4M3, F32, f64, gen, rand, scale_ref


def bits(t):
    return t.cpu().view(torch.uint8)


def blocks_ref(v):
    """(e4m3 bytes, scale bytes) of 64-bit rows [..., cols]."""
    cols = v.shape[-1]
    q, scales = torch.empty(v.shape, dtype=torch.uint8), []
    for c in range(0, cols, 128):
        b = v[..., c:c + 128]
        e = torch.from_numpy(scale_ref(b.abs().amax(-1).numpy()).astype(np.float64))
        scales.append((e + 127).to(torch.uint8))
        q[..., c:c + 128] = (b * torch.exp2(-e)[..., None]).to(F32).to(E4M3).view(torch.uint8)        # (a power of two of an fp32 number is one)
    return q, torch.stack(scales, -1)


def some_rows(g, n, cols, dtype, pad):
    x = rand(g, n, cols, dtype=dtype, pad=pad)
    x *= torch.exp2(torch.randint(-30, 30, (n, 1), generator=g).float()).to(dtype).cuda()
    if n > 2:
        x[1] = 0.0
        x[2, cols // 2:] *= 1e-38                               # down to numbers below the normal ones
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_rows(dtype):
    for n, cols in [(1, 1), (3, 127), (4, 128), (5, 129), (9, 255), (7, 520), (6, 1001), (3, 2048), (5, 4100), (2, 9000), (300, 64)]:
        for pad in (0, 3):
            print("rows", n, cols, dtype, pad, flush=True)
            x = some_rows(gen(n + cols), n, cols, dtype, pad)
            held = torch.full((n, cols + 5), 7.0, device="cuda").to(E4M3)
            q, scale = B.lasnet_quantize_rows(x, out=held[:, :cols])
            want, want_s = blocks_ref(f64(x))
            assert scale.shape == (n, (cols + 127) // 128)
            assert torch.equal(bits(scale), want_s) and torch.equal(bits(held)[:, :cols], want)
            assert (held[:, cols:].float() == 7.0).all()
    x = rand(gen(1), 2, 3, 4, 200, dtype=dtype)                 # a feature map is rows
    q, scale = B.lasnet_quantize_rows(x)
    assert q.shape == x.shape and torch.equal(bits(q), blocks_ref(f64(x))[0]) and scale.shape == (24, 2)
    assert B.lasnet_quantize_rows(torch.empty(0, 8, device="cuda"))[0].shape == (0, 8)


@pytest.mark.gpu
def test_borders_and_not_numbers():
    x = torch.zeros(6, 256)
    x[0, 5], x[0, 130] = 448.0, 448.0 * (1 + 2 ** -20)
    x[1, 0], x[1, 255] = 3e38, 1e-45
    x[2, 3], x[2, 4] = math.nan, 2.0                            # a NaN aside
    x[2, 200] = 5.0
    q, scale = (t.cpu() for t in B.lasnet_quantize_rows(x.cuda()))
    assert bits(scale)[0].tolist() == [127, 128] and bits(scale)[2].tolist() == [120, 121] and bits(scale)[1, 1] == 1 and (bits(scale)[3:] == 1).all()
    assert torch.isnan(q[2, 3].float()) and q[2, 4].float() == 256.0 and not torch.isnan(q[2, 128:].float()).any()
    assert q[0, 5].float() == 448.0 and q[0, 130].float() == 224.0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_rows_laid_out_by_expert(dtype):
    for tokens, k, E, cols in [(1, 1, 1, 64), (5, 2, 3, 130), (40, 4, 7, 1001), (33, 8, 16, 2048), (700, 1, 4, 96), (3, 2, 2, 8200)]:
        for none in (False, True):
            print("by expert", tokens, k, E, cols, dtype, none, flush=True)
            g = gen(tokens + cols)
            x = some_rows(g, tokens, cols, dtype, 3)
            experts = torch.full((tokens, k), -1, dtype=torch.int32) if none else torch.randint(-1, E, (tokens, k), generator=g, dtype=torch.int32)
            offsets, order, position = B.lasnet_route(experts.cuda(), E)
            held = torch.full((tokens * k + 2, cols), 7.0, device="cuda").to(E4M3)
            scale = torch.full(((tokens * k + 2) * ((cols + 127) // 128),), 9, dtype=torch.uint8, device="cuda")
            at = scale[:tokens * k * ((cols + 127) // 128)].view(tokens * k, -1)
            B.lasnet_quantize_rows(x, position=position, offsets=offsets, out=held[:tokens * k], scale=at)
            q, s = blocks_ref(f64(x))
            sent = order.cpu() >= 0
            want_q, want_s = q[order.cpu().clamp(min=0).long() // k], s[order.cpu().clamp(min=0).long() // k]
            want_q[~sent], want_s[~sent] = 0, 127
            assert torch.equal(bits(held)[:tokens * k], want_q) and torch.equal(bits(at), want_s)
            assert (held[tokens * k:].float() == 7.0).all() and (scale[at.numel():] == 9).all()


@pytest.mark.gpu
def test_positions_out_of_range_reach_no_other_memory():
    x, offsets = torch.ones(8, 64, device="cuda"), torch.tensor([0, 100], dtype=torch.int32).cuda()
    held = torch.full((18, 64), 7.0, device="cuda").to(E4M3)
    position = torch.tensor([[99, -5]] * 8, dtype=torch.int32).cuda()
    B.lasnet_quantize_rows(x, position=position, offsets=offsets, out=held[:16])
    assert (held.float() == 7.0).all()
    B.lasnet_quantize_rows(x, position=position, offsets=offsets - 1000, out=held[:16])
    assert (held[:16].float() == 0.0).all() and (held[16:].float() == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_matrices(dtype):
    for E, n, k in [(1, 1, 1), (2, 128, 128), (1, 127, 129), (3, 100, 300), (2, 257, 64), (1, 520, 1000), (5, 8, 513)]:
        print("matrices", E, n, k, dtype, flush=True)
        g = gen(n + k)
        W = rand(g, E, n, k, dtype=dtype)
        W *= torch.exp2(torch.randint(-8, 8, (E, n, 1), generator=g).float()).to(dtype).cuda()
        if n > 128:
            W[0, 128:] = 0.0
        q, scale, q_t, scale_t = B.lasnet_quantize_matrices(W, transposed=True)
        v = f64(W)
        want, want_s = torch.empty(E, n, k, dtype=torch.uint8), torch.empty(E, (n + 127) // 128, (k + 127) // 128, dtype=torch.uint8)
        for i in range(0, n, 128):
            for c in range(0, k, 128):
                b = v[:, i:i + 128, c:c + 128]
                one, s = zip(*(_block(m) for m in b))
                want[:, i:i + 128, c:c + 128] = torch.stack([o.reshape(b.shape[1:]) for o in one])
                want_s[:, i // 128, c // 128] = torch.stack([t.reshape(()) for t in s])
        assert torch.equal(bits(scale), want_s) and torch.equal(bits(q), want)
        assert torch.equal(bits(scale_t), want_s.transpose(1, 2)) and torch.equal(bits(q_t), want.transpose(1, 2))
        again = B.lasnet_quantize_matrices(W)
        assert again[2] is None and again[3] is None and torch.equal(bits(again[0]), want)


def _block(m):
    e = float(scale_ref(float(m.abs().max())))
    return (m * 2.0 ** -e).to(F32).to(E4M3).view(torch.uint8), torch.tensor(int(e + 127), dtype=torch.uint8)


# ---------------------------------------------------------------- what is refused (no GPU)

def test_arguments_that_are_refused():
    P, ref = 0x100000, B.ctypes.byref

    def q(x=rows(4, 200, B.LASNET_BF16), pos=None, off=None, k=2, E=3, out=rows(4, 200, B.LASNET_E4M3, P), scale=2 * P):
        return call("quantize_rows", ref(x), pos, off, k, E, ref(out), scale, None)
    assert q(x=rows(4, 200, B.LASNET_E4M3)) == q(out=rows(4, 200, B.LASNET_BF16, P)) == B.LASNET_EUNSUPPORTED
    assert q(out=rows(8, 200, B.LASNET_E4M3, P)) == q(out=rows(4, 201, B.LASNET_E4M3, P)) == q(pos=3 * P, off=4 * P) == B.LASNET_ESHAPE
    by = rows(8, 200, B.LASNET_E4M3, P)
    assert q(scale=None) == q(pos=3 * P, out=by) == q(off=3 * P) == q(pos=3 * P, off=4 * P, k=0, out=by) == B.LASNET_EINVAL
    assert q(pos=3 * P, off=4 * P, k=65, out=by) == q(pos=3 * P, off=4 * P, E=5000, out=by) == B.LASNET_EUNSUPPORTED
    assert q(scale=0x1000) == q(out=rows(4, 200, B.LASNET_E4M3, 0x1000)) == B.LASNET_EALIAS

    def m(W=P, dtype=B.LASNET_F32, E=2, n=8, k=8, out=2 * P, scale=3 * P, out_t=None, scale_t=None):
        return call("quantize_matrices", W, dtype, E, n, k, out, scale, out_t, scale_t, None)
    assert m(W=None) == m(out=None) == m(scale=None) == m(out_t=4 * P) == m(scale_t=4 * P) == m(dtype=3) == m(E=0) == B.LASNET_EINVAL
    assert m(n=0) == m(k=-1) == B.LASNET_ESHAPE
    assert m(dtype=B.LASNET_E4M3) == m(n=1 << 21) == m(E=4096, n=1 << 20, k=1 << 20) == m(E=5000) == B.LASNET_EUNSUPPORTED
    assert m(out=P) == m(out_t=3 * P, scale_t=5 * P) == B.LASNET_EALIAS


def test_tensors_that_are_refused(monkeypatch):
    on_device(monkeypatch)
    x = dev(4, 200)
    with pytest.raises(ValueError, match="together"):
        B.lasnet_quantize_rows(x, position=dev(4, 2, dtype=torch.int32))
    with pytest.raises(ValueError, match="tokens"):
        B.lasnet_quantize_rows(x, position=dev(5, 2, dtype=torch.int32), offsets=dev(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="scale"):
        B.lasnet_quantize_rows(x, scale=dev(4, 1, dtype=torch.uint8))
    with pytest.raises(ValueError, match="matrices"):
        B.lasnet_quantize_matrices(dev(4, 200))
    with pytest.raises(ValueError, match="matrices"):
        B.lasnet_quantize_matrices(dev(2, 4, 8), out=dev(2, 8, 4).to(E4M3).as_subclass(type(x)))
    with pytest.raises(ValueError, match="together"):
        B.lasnet_quantize_matrices(dev(2, 4, 8), out_t=dev(2, 8, 4).to(E4M3).as_subclass(type(x)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_an_infinity_is_nan_and_spoils_no_neighbour(dtype):
    x = torch.randn(4, 256, generator=gen(1)).to(dtype)
    x[1, 7], x[2, 200] = math.inf, -math.inf
    x[1, 8] = 2.0 ** 121
    clean = [t.cpu() for t in B.lasnet_quantize_rows(x.masked_fill(x.abs() == math.inf, 0).cuda())]
    q, scale = (t.cpu() for t in B.lasnet_quantize_rows(x.cuda()))
    m, ms = (t.cpu() for t in B.lasnet_quantize_matrices(x[None].cuda())[:2])
    assert bits(scale)[1, 0] == 247 and bits(scale)[2, 1] == 247 and (bits(ms) == 247).all()
    assert torch.isnan(q[1, 7].float()) and torch.isnan(q[2, 200].float()) and q[1, 8].float() == 2.0
    assert int(torch.isnan(q.float()).sum()) == 2 and torch.equal(torch.isnan(m[0].float()), torch.isinf(x)) and m[0, 1, 8].float() == 2.0
    keep = torch.ones(4, 256, dtype=torch.bool)
    keep[1, :128] = keep[2, 128:] = False
    assert torch.equal(bits(q)[keep], bits(clean[0])[keep])


def calls(k):
    """name, the call, how many outputs it makes"""
    x, pos, off, W = dev(6, 8, dtype=BF16), dev(6, 2, dtype=torch.int32), dev(4, dtype=torch.int32), dev(3, 8, 16)
    yield "rows", lambda: B.lasnet_quantize_rows(x, **k), 2
    yield "rows by expert", lambda: B.lasnet_quantize_rows(x, pos, off, **k), 2
    yield "matrices", lambda: B.lasnet_quantize_matrices(W, **k), 2
    yield "matrices, transposed, too", lambda: B.lasnet_quantize_matrices(W, transposed=True, **k), 4


@pytest.mark.parametrize("which", range(4))
def test_what_a_call_makes_is_memory_of_its_stream(which, made):
    for given in (None, CURRENT, SIDE):
        name, run, outputs = list(calls({} if given is None else {"stream": given}))[which]
        made.clear()
        run()
        assert [s for _, s in made] == [given or CURRENT] * outputs, name
        assert [getattr(t, "used_on", []) for t, _ in made] == [[CURRENT] if given is SIDE else []] * outputs, name


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Of bytes and of elements: rows, and matrices with their transposes, the last of which are compared with the same ones by themselves."""
    n, cols, last = 600001, 8200, 130
    x = torch.empty(n, cols, dtype=BF16, device="cuda")
    x[:] = torch.randn(1, cols, generator=gen(1)).cuda()
    x[-last:] = torch.randn(last, cols, generator=gen(2)).cuda()
    q, scale = B.lasnet_quantize_rows(x)
    few, few_s = B.lasnet_quantize_rows(x[-last:].clone())
    assert torch.equal(q.view(torch.uint8)[-last:], few.view(torch.uint8)) and torch.equal(scale.view(torch.uint8)[-last:], few_s.view(torch.uint8))
    del q
    position = torch.arange(2 * n, dtype=torch.int32).flip(0).reshape(n, 2).cuda()                   # the last token goes to the first rows
    q, scale = B.lasnet_quantize_rows(x, position, torch.tensor([0, 2 * n], dtype=torch.int32).cuda())
    assert torch.equal(q.view(torch.uint8)[1:2 * last:2].flip(0), few.view(torch.uint8)) and torch.equal(scale.view(torch.uint8)[0:2 * last:2].flip(0), few_s.view(torch.uint8))
    assert bool((q.view(torch.uint8)[2 * last:] == q.view(torch.uint8)[2 * last]).all())
    del q, x
    W = torch.empty(5, 1000, 1000001, dtype=BF16, device="cuda")
    W[:] = torch.randn(1000, 1, generator=gen(3)).cuda()
    W[4, :, -1001:] = torch.randn(1000, 1001, generator=gen(4)).cuda()
    got = B.lasnet_quantize_matrices(W, transposed=True)
    at = 1000001 // 128 * 128 - 896                                                                   # (whole blocks from here)
    want = B.lasnet_quantize_matrices(W[4:, :, at:].contiguous(), transposed=True)
    for have, part in zip((got[0][4:, :, at:], got[1][4:, :, at // 128:], got[2][4:, at:], got[3][4:, at // 128:]), want):
        assert torch.equal(have.view(torch.uint8), part.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("cols", [1024, 1001])
def test_outputs_past_the_caches_and_in_them(cols, dtype):
    """Outputs of 104 and 120 MiB, on both sides of where they go past the caches: the bits of the same rows in small calls, in place and laid out by expert."""
    k, E, g = 4, 8, gen(cols)
    for mib in (104, 120):
        tokens = (mib << 20) // (cols * k)
        x = torch.randn(tokens, cols, generator=g).to(dtype).cuda()
        parts = [B.lasnet_quantize_rows(x[i:i + 4096]) for i in range(0, tokens, 4096)]
        q, s = (torch.cat([p[j].view(torch.uint8) for p in parts]) for j in range(2))
        offsets, _, position = B.lasnet_route(torch.randint(-1, E, (tokens, k), generator=g, dtype=torch.int32).cuda(), E)
        out, scale = B.lasnet_quantize_rows(x, position=position, offsets=offsets)
        at, sent = position.flatten().long(), position.flatten() >= 0
        token = torch.arange(tokens, device="cuda").repeat_interleave(k)
        assert torch.equal(out.view(torch.uint8)[at[sent]], q[token[sent]]) and torch.equal(scale.view(torch.uint8)[at[sent]], s[token[sent]]), mib
        n = int(offsets[E])
        assert n == int(sent.sum()) and not out.view(torch.uint8)[n:].any() and (scale.view(torch.uint8)[n:] == 127).all()
        many = x.repeat(k, 1)
        out, scale = B.lasnet_quantize_rows(many)
        assert torch.equal(out.view(torch.uint8), q.repeat(k, 1)) and torch.equal(scale.view(torch.uint8), s.repeat(k, 1)), mib
