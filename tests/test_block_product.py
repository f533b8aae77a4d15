"""Products of 8-bit rows and matrices with scales for blocks of 128, against the definition in 64 bits.

Tolerances, fixed before the first run, as for the products with a scale a row: fp32 sums of n products (n + 4) u sum|terms|, the matrix core's cut of 2^-13 below the largest
of a group, 128 2^-13 max|x| max|W| for each block with its scales, and the rounding to bf16.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2210_06223_amd import binding as B
from paper_2210_06223_amd import build
from tests.test_call_streams import CURRENT, SIDE, dev, made  # noqa: F401
from tests.test_router import call, on_device, rows
from tests.test_row_operators import BF16, E4M3, F32, HALF, U, close, f64, gen, rand

E8M0 = torch.float8_e8m0fnu


def split(r, n, E, tail, empty=False):
    share = r.dirichlet(np.ones(E))
    if empty:
        share[r.integers(E)] = 0
        share /= max(share.sum(), 1e-9)
    counts = r.multinomial(n - tail, share) if E > 1 else np.array([n - tail])
    return np.concatenate([[0], np.cumsum(counts)])


def make(rows_, E, n, k, floats, tail=0, pad=0, seed=0):
    g, kb, nb = gen(seed + rows_ + n + k), (k + 127) // 128, (n + 127) // 128
    o = split(np.random.default_rng(seed + rows_), rows_, E, tail, True)
    x = (torch.randn(rows_, k + pad, generator=g) * torch.exp(torch.randn(rows_, 1, generator=g))).to(E4M3).cuda()[:, :k]
    scale = torch.randint(120, 134, (rows_, kb), generator=g, dtype=torch.uint8).cuda().view(E8M0)
    W = torch.randn(E, n, k, generator=g).to(E4M3).cuda()
    wscale = (torch.rand(E, nb, kb, generator=g) * 3 + 0.01).cuda() if floats else torch.randint(121, 133, (E, nb, kb), generator=g, dtype=torch.uint8).cuda().view(E8M0)
    return o, torch.from_numpy(o.astype(np.int32)).cuda(), x, scale, W, wscale


def number(scale):
    return f64(scale) if scale.dtype == F32 else torch.exp2(scale.cpu().view(torch.uint8).double() - 127)


def reference(o, x, scale, W, wscale):
    """(result, sum of the terms' sizes, what the matrix core may cut)."""
    (R, k), (E, n, _) = x.shape, W.shape
    s, ws = number(scale), number(wscale)
    ref, size, cut = (torch.zeros(R, n, dtype=torch.float64) for _ in range(3))
    wide = torch.arange(n) // 128
    for e in range(E):
        a, b = int(o[e]), int(o[e + 1])
        if a == b:
            continue
        X, V = f64(x[a:b]), f64(W[e])
        for c in range(0, k, 128):
            f = s[a:b, c // 128][:, None] * ws[e, :, c // 128][wide][None, :]
            ref[a:b] += f * (X[:, c:c + 128] @ V[:, c:c + 128].T)
            size[a:b] += f * (X[:, c:c + 128].abs() @ V[:, c:c + 128].abs().T)
            cut[a:b] += f * 128 * 2.0 ** -13 * X[:, c:c + 128].abs().amax(1)[:, None] * V[:, c:c + 128].abs().amax(1)[None, :]
    return ref, size, cut


# every kind of kernel: few rows; reductions shared by groups of waves; tiles of every size; many tiles; odd widths and alignments; short and ragged reductions
SHAPES = [(1, 1, 1, 1), (1, 1, 64, 128), (1, 1, 300, 2048), (5, 3, 100, 130), (16, 16, 256, 512), (17, 2, 96, 1040), (33, 1, 144, 272), (64, 2, 512, 528), (40, 4, 200, 16),
          (300, 8, 500, 520), (200, 3, 300, 1537), (256, 1, 256, 1792), (500, 2, 512, 1040), (1000, 3, 640, 384), (1500, 4, 1024, 272), (2500, 2, 768, 640), (700, 5, 130, 48),
          (90, 3, 257, 15), (129, 2, 129, 129), (2, 2, 4096, 4096), (30, 30, 512, 1024), (32, 4, 320, 2064), (64, 64, 512, 1024), (60, 5, 1000, 400),
          (1000, 1, 1032, 2320)]
LARGE = [(9000, 3, 1536, 256), (8200, 2, 2048, 512), (14000, 70, 1024, 384), (13000, 4, 1160, 640), (9001, 2, 1540, 784), (8500, 2, 1602, 256), (9000, 3, 1536, 784), (9000, 2, 1544, 1040), (4652, 1, 4096, 400),
         (5164, 1, 4096, 640)]


@pytest.mark.gpu
@pytest.mark.parametrize("floats", [False, True], ids=["e8m0", "f32"])
def test_product(floats):
    for R, E, n, k in SHAPES:
        for tail, pad, relu in ((0, 0, False), (min(R // 2, 7), 16, True), (0, 5, False)):
            print("block product", R, E, n, k, floats, tail, pad, flush=True)
            o, offsets, x, scale, W, wscale = make(R, E, n, k, floats, tail, pad)
            held = torch.full((R + 1, n + 3 + pad), 7.0, dtype=BF16, device="cuda")
            got = B.lasnet_block_product(x, scale, offsets, W, wscale, out=held[:R, :n], flags=B.LASNET_POST_RELU if relu else 0)
            ref, size, cut = reference(o, x, scale, W, wscale)
            ref = ref.clamp(min=0) if relu else ref
            close(got, ref, HALF[BF16] * (1 + 2 ** -8) * ref.abs() + (k + 4) * U * size + cut + 1e-38, "out")
            assert (held[R] == 7.0).all() and (held[:, n:] == 7.0).all()
            assert (got[int(o[-1]):] == 0).all()
            if float(ref.norm()) > 0:
                assert float((f64(got) - ref).norm() / ref.norm()) < 2.0 ** -8
            assert torch.equal(got, B.lasnet_block_product(x, scale, offsets, W, wscale, flags=B.LASNET_POST_RELU if relu else 0)), "twice the same bits, whatever the output's layout"


@pytest.mark.gpu
@pytest.mark.parametrize("floats", [False, True], ids=["e8m0", "f32"])
@pytest.mark.parametrize("shape", LARGE, ids=str)
def test_large_product(shape, floats):
    R, E, n, k = shape
    o, offsets, x, scale, W, wscale = make(R, E, n, k, floats, 300)
    got = B.lasnet_block_product(x, scale, offsets, W, wscale)
    rows_ = torch.unique(torch.cat([torch.from_numpy(np.clip(o[:, None] + np.arange(-3, 4), 0, R - 1).reshape(-1)), torch.arange(0, R, 41)]))      # every expert's first and last, and some
    e = torch.searchsorted(torch.from_numpy(o[1:].copy()), rows_, right=True)
    for i in range(E):
        at = rows_[e == i]
        if len(at):
            ref, size, cut = reference([0, len(at)], x[at.cuda()], scale.view(torch.uint8)[at.cuda()].view(E8M0), W[i:i + 1], wscale[i:i + 1])
            close(f64(got)[at], ref, HALF[BF16] * (1 + 2 ** -8) * ref.abs() + (k + 4) * U * size + cut + 1e-38, "out of expert %d" % i)
    assert (got[int(o[-1]):] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("floats", [False, True], ids=["e8m0", "f32"])
@pytest.mark.parametrize("R,n,k", [(30, 64, 256), (300, 200, 640), (600, 512, 2048), (9000, 2048, 512), (300, 200, 650)])
def test_small_whole_numbers_are_exact(R, n, k, floats):
    """Products and sums of small whole numbers times powers of two that no part of the sum loses: each scale lands on its own block."""
    g, E = gen(R), 3
    o = split(np.random.default_rng(R), R, E, 5)
    offsets = torch.from_numpy(o.astype(np.int32)).cuda()
    kb, nb = (k + 127) // 128, (n + 127) // 128
    x, W = (torch.randint(-1, 2, s, generator=g).float().to(E4M3).cuda() for s in ((R, k), (E, n, k)))
    scale = torch.randint(126, 130, (R, kb), generator=g, dtype=torch.uint8).cuda().view(E8M0)
    ws = torch.randint(126, 130, (E, nb, kb), generator=g, dtype=torch.uint8)
    wscale = torch.exp2(ws.float() - 127).cuda() if floats else ws.cuda().view(E8M0)
    got = B.lasnet_block_product(x, scale, offsets, W, wscale)
    ref, _, _ = reference(o, x, scale, W, wscale)
    assert torch.equal(f64(got), ref.to(F32).to(BF16).double())


@pytest.mark.gpu
@pytest.mark.parametrize("floats", [False, True], ids=["e8m0", "f32"])
@pytest.mark.parametrize("k", [640, 650, 1664])
def test_rows_stay_apart(k, floats):
    """Scales of NaN of one row, of one expert and of rows that no expert has, and NaN in their elements, reach no other output."""
    for R in (40, 300, 9000):
        o, offsets, x, scale, W, wscale = make(R, 3, 1544, k, floats, 20, seed=3)
        clean = B.lasnet_block_product(x, scale, offsets, W, wscale)
        a = int(o[1]) if o[1] > 0 else int(o[2]) - 1
        row = max(a - 1, 0)
        expert = int(np.searchsorted(o[1:], row, side="right"))
        scale.view(torch.uint8)[row, 0] = 255
        scale.view(torch.uint8)[int(o[-1]):] = 255
        x.view(torch.uint8)[int(o[-1]):] = 0x7f
        other = (expert + 1) % 3
        (wscale if floats else wscale.view(torch.uint8))[other, 2, 1] = math.nan if floats else 255
        got = B.lasnet_block_product(x, scale, offsets, W, wscale)
        assert torch.isnan(got[row].float()).all() and (got[int(o[-1]):] == 0).all()
        keep = torch.ones(R, 1544, dtype=torch.bool)
        keep[row] = False
        keep[int(o[other]):int(o[other + 1]), 256:384] = False
        assert torch.isnan(got[int(o[other]):int(o[other + 1]), 256:384].float()).all()
        assert torch.equal(got.cpu()[keep], clean.cpu()[keep])


@pytest.mark.gpu
def test_scales_at_the_ends_of_their_range():
    """The two scales' powers of two are added before they meet the products: 2^127 times 2^-100 is no overflow."""
    for R, n, k in ((4, 64, 256), (300, 128, 256), (300, 128, 250), (9000, 2048, 256)):
        x, W = torch.ones(R, k, device="cuda").to(E4M3), torch.ones(1, n, k, device="cuda").to(E4M3)
        offsets = torch.tensor([0, R], dtype=torch.int32).cuda()
        kb, nb = (k + 127) // 128, (n + 127) // 128
        for sx, sw in ((254, 27), (27, 254), (1, 253), (100, 100)):
            scale = torch.full((R, kb), sx, dtype=torch.uint8, device="cuda")
            wscale = torch.full((1, nb, kb), sw, dtype=torch.uint8, device="cuda")
            got = B.lasnet_block_product(x, scale, offsets, W, wscale)
            assert (got.double() == float(torch.tensor(k * 2.0 ** (sx + sw - 254)).to(BF16))).all(), (R, sx, sw)


@pytest.mark.gpu
def test_offsets_out_of_range_reach_no_other_memory():
    x, W = torch.ones(64, 128, device="cuda").to(E4M3), torch.ones(2, 64, 128, device="cuda").to(E4M3)
    scale, wscale = torch.full((64, 1), 127, dtype=torch.uint8, device="cuda"), torch.ones(2, 1, 1, device="cuda")
    for o in ([-5, 30, 1000], [0, 70, 64], [64, 0, -9]):
        out = torch.full((66, 64), 5.0, dtype=BF16, device="cuda")
        B.lasnet_block_product(x, scale, torch.tensor(o, dtype=torch.int32).cuda(), W, wscale, out=out[:64])
        assert (out[64:] == 5.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("floats", [False, True], ids=["e8m0", "f32"])
def test_counted_barriers_against_the_drained_build(floats):
    """The check build waits for all loads at every barrier: the same bits."""
    check = B.load_library(build.LIB_CHECK)
    for R, E, n, k in [(256, 1, 256, 1792), (500, 2, 512, 1040), (1000, 3, 640, 384), (1500, 4, 1024, 272), (2500, 2, 768, 640), (9000, 3, 1536, 256), (14000, 70, 1024, 384),
                       (16000, 2, 2048, 2048)]:
        o, offsets, x, scale, W, wscale = make(R, E, n, k, floats, 9)
        got = B.lasnet_block_product(x, scale, offsets, W, wscale)
        other = torch.empty_like(got)
        d, out = B._rows(x, "x"), B._rows(other, "out")
        st = check.lasnet_block_product(ctypes.byref(d), scale.data_ptr(), offsets.data_ptr(), E, W.data_ptr(), wscale.data_ptr(), B.LASNET_F32 if floats else B.LASNET_E8M0,
                                        ctypes.byref(out), 0, B._stream(None))
        assert st == B.LASNET_OK
        assert torch.equal(got, other), (R, E, n, k)


@pytest.mark.gpu
def test_a_run_of_them_captured_and_on_another_stream():
    """Rows to experts in blocks, a product, its output in blocks, the second product and the way back, forward and the rows' gradient: in a graph replayed on new inputs, on a
    stream of its own, and eagerly."""
    tokens, k, E, C, M = 700, 2, 6, 384, 264
    g = gen(8)
    x, dout = rand(g, tokens, C, dtype=BF16), rand(g, tokens, C, dtype=BF16)
    l = rand(g, tokens, E)
    W1, W2 = rand(g, E, M, C, dtype=BF16, scale=C ** -0.5), rand(g, E, C, M, dtype=BF16, scale=M ** -0.5)

    def path(s=None):
        q1, s1, t1, ts1 = B.lasnet_quantize_matrices(W1, transposed=True, stream=s)
        q2, s2, t2, ts2 = B.lasnet_quantize_matrices(W2, transposed=True, stream=s)
        experts, weights, _ = B.lasnet_choose_experts(l, k, stream=s)
        offsets, _, position = B.lasnet_route(experts, E, stream=s)
        r, rs = B.lasnet_quantize_rows(x, position=position, offsets=offsets, stream=s)
        mid = B.lasnet_block_product(r, rs, offsets, q1, s1, flags=B.LASNET_POST_RELU, stream=s)
        y = B.lasnet_block_product(*B.lasnet_quantize_rows(mid, stream=s), offsets, q2, s2, stream=s)
        out = B.lasnet_combine_rows(y, position, weights=weights, base=x, stream=s)
        dy, dweights = B.lasnet_combine_rows_backward(dout, y, position, offsets, weights=weights, stream=s)
        dmid = B.lasnet_block_product(*B.lasnet_quantize_rows(dy, stream=s), offsets, t2, ts2, stream=s)
        return [out, dweights, dmid, B.lasnet_block_product(*B.lasnet_quantize_rows(dmid, stream=s), offsets, t1, ts1, stream=s), offsets, position]

    want = path()
    # against the same in 64 bits without rounding: four operands of 2^-4 at most (2^-5.5 rms or less, each) under a sum each, 2^-4 of the norm in all
    offsets, position = want[4].cpu(), want[5].cpu().long()
    X, A, V = f64(x), f64(W1), f64(W2)
    experts, weights, _ = B.lasnet_choose_experts(l, k)
    ref = X.clone()
    for j in range(k):
        e = experts[:, j].cpu().long()
        mid = torch.relu(torch.einsum("tc,tmc->tm", X, A[e]))
        ref += f64(weights)[:, j:j + 1] * torch.einsum("tm,tcm->tc", mid, V[e])
    assert float((f64(want[0]) - ref).norm() / (ref - X).norm()) < 2.0 ** -4
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = path()
    side = torch.cuda.Stream()
    for i in range(3):
        x.copy_(rand(g, tokens, C, dtype=BF16))
        l.copy_(rand(g, tokens, E))
        graph.replay()
        got = [t.clone() for t in held]
        torch.cuda.synchronize()
        want, other = path(), path(side)
        side.synchronize()
        for a, b, c in zip(got, want, other):
            assert torch.equal(a, b) and torch.equal(c, b)


# ---------------------------------------------------------------- what is refused (no GPU)

def test_arguments_that_are_refused():
    P, ref = 0x100000, ctypes.byref

    def product(x=rows(4, 200, B.LASNET_E4M3), scale=P, off=2 * P, E=2, W=3 * P, ws=4 * P, ty=B.LASNET_E8M0, out=rows(4, 64, B.LASNET_BF16, 5 * P), flags=0):
        return call("block_product", ref(x), scale, off, E, W, ws, ty, ref(out), flags, None)
    assert product(x=rows(4, 200, B.LASNET_BF16)) == product(out=rows(4, 64, B.LASNET_F32, 5 * P)) == product(E=5000) == B.LASNET_EUNSUPPORTED
    assert product(out=rows(5, 64, B.LASNET_BF16, 5 * P)) == B.LASNET_ESHAPE
    assert product(scale=None) == product(off=None) == product(W=None) == product(ws=None) == product(ty=B.LASNET_BF16) == product(flags=2) == product(E=0) == B.LASNET_EINVAL
    for at in (0x1000, P, 2 * P, 3 * P, 4 * P):
        assert product(out=rows(4, 64, B.LASNET_BF16, at)) == B.LASNET_EALIAS


def test_tensors_that_are_refused(monkeypatch):
    on_device(monkeypatch)
    eight = lambda *s: dev(*s).to(E4M3).as_subclass(type(dev(1)))
    x, off, W = eight(4, 200), dev(3, dtype=torch.int32), eight(2, 64, 200)
    s, ws = dev(4, 2, dtype=torch.uint8), dev(2, 1, 2)
    for bad in (dict(scale=dev(4, 1, dtype=torch.uint8)), dict(scale=dev(4, 2)), dict(wscale=dev(2, 1, 1)), dict(wscale=dev(2, 1, 2, dtype=BF16)), dict(W=eight(2, 64, 128)),
                dict(W=dev(2, 64, 200)), dict(W=eight(64, 200)), dict(offsets=dev(3)), dict(out=dev(4, 63, dtype=BF16))):
        args = dict(x=x, scale=s, offsets=off, W=W, wscale=ws, **{}) | bad
        with pytest.raises(ValueError):
            B.lasnet_block_product(args["x"], args["scale"], args["offsets"], args["W"], args["wscale"], out=args.get("out"))


@pytest.mark.gpu
@pytest.mark.parametrize("floats", [False, True], ids=["e8m0", "f32"])
def test_an_output_written_past_the_caches(floats):
    """Large outputs are: 26000 x 4096 in bf16, 213 MB.  Whole numbers up to 256, which bf16 holds."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x, W = (torch.randint(-1, 2, s, generator=g, device="cuda").float() for s in ((26000, 256), (1, 4096, 256)))
    scale = torch.full((26000, 2), 127, dtype=torch.uint8, device="cuda")
    wscale = torch.ones(1, 32, 2, device="cuda") if floats else torch.full((1, 32, 2), 127, dtype=torch.uint8, device="cuda")
    offsets = torch.tensor([0, 25990], dtype=torch.int32).cuda()
    got = B.lasnet_block_product(x.to(E4M3), scale, offsets, W.to(E4M3), wscale)
    want = x @ W[0].T
    want[25990:] = 0
    assert torch.equal(got.float(), want)


@pytest.mark.gpu
def test_scales_in_32_bits_are_any_numbers():
    """0, negative, below the normal numbers and large, block by block; W and x of ones and whole scales, so that every sum is exact."""
    some = [0.0, -1.0, 3.0, -0.375, 2.0 ** -126, 2.0 ** 100, 1.0, -2.0]
    for R, n, k in ((4, 64, 1024), (300, 200, 1024), (300, 200, 1023), (9000, 2048, 1024)):
        kb, nb = (k + 127) // 128, (n + 127) // 128
        x, W = torch.ones(R, k, device="cuda").to(E4M3), torch.ones(1, n, k, device="cuda").to(E4M3)
        scale = torch.full((R, kb), 127, dtype=torch.uint8, device="cuda")
        offsets = torch.tensor([0, R], dtype=torch.int32).cuda()
        for b in range(kb):                                    # one block at a time
            for v in some:
                ws = torch.zeros(1, nb, kb)
                ws[:, :, b] = v
                got = B.lasnet_block_product(x, scale, offsets, W, ws.cuda())
                assert (got.double() == float(torch.tensor(min(128, k - 128 * b) * v, dtype=F32).to(BF16))).all(), (R, k, b, v)
        ws = torch.full((1, nb, kb), 1.0)
        ws[:, :, 1] = math.inf
        got = B.lasnet_block_product(x, scale, offsets, W, ws.cuda())
        assert (got.double() == math.inf).all()


@pytest.mark.parametrize("given", [None, CURRENT, SIDE], ids=["none", "current", "other"])
def test_what_a_call_makes_is_memory_of_its_stream(given, made):
    x, W, off = dev(6, 8).to(E4M3).as_subclass(type(dev(1))), dev(3, 16, 8).to(E4M3).as_subclass(type(dev(1))), dev(4, dtype=torch.int32)
    made.clear()
    B.lasnet_block_product(x, dev(6, 1, dtype=torch.uint8), off, W, dev(3, 1, 1), **({} if given is None else {"stream": given}))
    assert [s for _, s in made] == [given or CURRENT] and getattr(made[0][0], "used_on", []) == ([CURRENT] if given is SIDE else [])


@pytest.mark.gpu
@pytest.mark.parametrize("floats", [False, True], ids=["e8m0", "f32"])
@pytest.mark.parametrize("R,n,k", [(600000, 4104, 1040), (4300000, 1024, 640), (560000, 4097, 201)])
def test_offsets_past_32_bits(R, n, k, floats):
    """Of bytes and of elements, of the output and of the rows: the last rows are compared with the same rows by themselves.  (Another kernel may run for so few: bf16 of sums of the same
    whole numbers, which are exact.)"""
    last, kb, nb = 400, (k + 127) // 128, (n + 127) // 128
    some = torch.randint(-2, 3, (997, k), generator=gen(1)).to(E4M3).cuda().view(torch.uint8)
    x = torch.empty(R, k, dtype=torch.uint8, device="cuda")
    x[:R // 997 * 997].view(-1, 997, k)[:] = some
    x[R // 997 * 997 - 997:] = some[:1].expand(R - R // 997 * 997 + 997, k)
    x[-last:] = torch.randint(-2, 3, (last, k), generator=gen(2)).to(E4M3).cuda().view(torch.uint8)
    x = x.view(E4M3)
    W = torch.randint(-2, 3, (2, n, k), generator=gen(3)).to(E4M3).cuda()
    scale = torch.full((R, kb), 127, dtype=torch.uint8, device="cuda")
    wscale = torch.ones(2, nb, kb, device="cuda") if floats else torch.full((2, nb, kb), 127, dtype=torch.uint8, device="cuda")
    got = B.lasnet_block_product(x, scale, torch.tensor([0, 997, R], dtype=torch.int32).cuda(), W, wscale)
    end = B.lasnet_block_product(x[-last:].clone(), scale[-last:].clone(), torch.tensor([0, 0, last], dtype=torch.int32).cuda(), W, wscale)
    assert torch.equal(got[-last:], end)
    assert torch.equal(got[997:1994], got[997 * 400:997 * 401])


# rows that are not whole pieces of 16 bytes, kernel by kernel: few tiles, straight to registers; the reduction shared by four groups and by two; all of it in one
ODD = [(1, 1, 515, 4095), (5, 2, 97, 17), (40, 4, 130, 143), (300, 4, 1001, 1001), (60, 8, 2047, 515), (64, 3, 1900, 1153), (1000, 8, 1023, 1049), (900, 3, 777, 130), (700, 2, 4001, 257),
       (700, 2, 4002, 389), (4000, 8, 1001, 131), (900, 70, 40, 129), (1200, 20, 333, 1001), (256, 1, 4094, 519)]


@pytest.mark.gpu
@pytest.mark.parametrize("floats", [False, True], ids=["e8m0", "f32"])
@pytest.mark.parametrize("shape", ODD, ids=str)
def test_rows_of_any_width_and_address(shape, floats):
    """At every place a word has for a first byte, with NaN on both sides of the rows and of the matrices; rows lie next to each other or apart."""
    R, E, n, k = shape
    o, offsets, x, scale, W, wscale = make(R, E, n, k, floats, min(R // 2, 9))
    ref, size, cut = reference(o, x, scale, W, wscale)
    bound = HALF[BF16] * (1 + 2 ** -8) * ref.abs() + (k + 4) * U * size + cut + 1e-38
    want = None
    for at, pad in ((1, 0), (2, 3), (3, 1), (4, 6)):
        print("odd", shape, floats, at, pad, flush=True)
        held = torch.full((64 + R * (k + pad),), 0x7f, dtype=torch.uint8, device="cuda")
        X = held[at:at + R * (k + pad)].view(R, k + pad)[:, :k]
        X.copy_(x.view(torch.uint8))
        beside = torch.full((64 + E * n * k,), 0x7f, dtype=torch.uint8, device="cuda")
        V = beside[5 - at:5 - at + E * n * k].view(E, n, k)
        V.copy_(W.view(torch.uint8))
        out = torch.full((R + 2, n + pad), 7.0, dtype=BF16, device="cuda")
        got = B.lasnet_block_product(X.view(E4M3), scale, offsets, V.view(E4M3), wscale, out=out[1:R + 1, :n])
        close(got, ref, bound, "out")
        assert (out[0] == 7.0).all() and (out[R + 1] == 7.0).all() and (out[:, n:] == 7.0).all() and (got[int(o[-1]):] == 0).all()
        want = got.clone() if want is None else want
        assert torch.equal(got, want), "the same bits wherever they lie"


@pytest.mark.gpu
def test_scales_in_32_bits_at_the_ends_of_their_range():
    """The same with fp32 scales of the matrices: no part of a scale meets a sum before the row's does.  1.5, 1.25 and the sums are exact; k products of one size, so the result is."""
    one, least = 1.0, 2.0 ** -9                                # (e4m3's smallest number)
    for R, n, k in ((4, 64, 256), (16, 64, 512), (64, 512, 1024), (300, 128, 256), (300, 128, 250), (40, 1536, 650), (9000, 2048, 256), (9000, 2048, 250)):
        offsets = torch.tensor([0, R], dtype=torch.int32).cuda()
        kb, nb = (k + 127) // 128, (n + 127) // 128
        for v, sx, w in ((one, 254, 1.5 * 2.0 ** -100), (one, 27, 1.5 * 2.0 ** 118), (least, 27, 1.5 * 2.0 ** 127), (least, 1, 1.25 * 2.0 ** 126), (one, 100, -1.25 * 2.0 ** 20),
                         (one, 254, 1.25 * 2.0 ** -140), (one, 254, 2.0 ** -149), (one, 254, 0.0), (one, 1, math.inf), (least, 250, -math.inf)):
            print("fp32 scales", R, n, k, v, sx, w, flush=True)
            x, W = torch.full((R, k), v, device="cuda").to(E4M3), torch.full((1, n, k), v, device="cuda").to(E4M3)
            scale = torch.full((R, kb), sx, dtype=torch.uint8, device="cuda")
            wscale = torch.full((1, nb, kb), w, device="cuda")
            got = B.lasnet_block_product(x, scale, offsets, W, wscale)
            want = k * v * v * w * 2.0 ** (sx - 127)
            assert math.isinf(w) or w == 0.0 or 2.0 ** -126 <= abs(want) < 2.0 ** 128
            assert (got.double() == float(torch.tensor(want).to(BF16))).all(), (R, n, k, v, sx, w, float(got[0, 0]), want)


@pytest.mark.gpu
def test_an_infinite_scale_is_no_nan_whatever_shares_the_reduction():
    """A group of waves whose share of the reduction begins behind its end (five or nine steps in four shares, the last not whole) adds nothing: an infinite scale of the last block stays infinite."""
    for R, E, n, k in ((200, 50, 256, 528), (200, 50, 256, 1040), (100, 4, 256, 1552), (32, 4, 2048, 2064), (200, 50, 256, 640), (300, 2, 512, 784), (64, 8, 255, 527), (9000, 1, 1536, 784)):
        print("infinite scale", R, E, n, k, flush=True)
        x, W = torch.ones(R, k, device="cuda").to(E4M3), torch.ones(E, n, k, device="cuda").to(E4M3)
        offsets = (torch.arange(E + 1) * R // E).to(torch.int32).cuda()
        kb, nb = (k + 127) // 128, (n + 127) // 128
        scale, wscale = torch.full((R, kb), 127, dtype=torch.uint8, device="cuda"), torch.ones(E, nb, kb, device="cuda")
        wscale[:, 0, -1] = -math.inf
        got = B.lasnet_block_product(x, scale, offsets, W, wscale)
        assert (got[:, :128] == -math.inf).all(), (R, E, n, k, got[0, 0])
        assert (got[:, 128:].double() == float(torch.tensor(float(k)).to(BF16))).all()
