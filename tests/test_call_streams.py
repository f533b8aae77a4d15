"""A call on another stream than the current one: what it makes (outputs, workspaces) is memory of that stream, so that no work of the current stream is still
at it, and outputs are known to be used on the current stream, too."""
import contextlib

import pytest
import torch

from paper_2210_06223_amd import binding as B

BF16, E4M3, I32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32


class OnDevice(torch.Tensor):
    """A host tensor that the binding's checks take for one in device memory (the calls go to a library that does nothing)."""
    is_cuda = property(lambda self: True)

    def record_stream(self, stream):
        self.used_on = getattr(self, "used_on", []) + [stream]


def dev(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


class NoLibrary:
    def __getattr__(self, name):
        return lambda *a: 512 if name.endswith("_bytes") else 0


def row_calls(k):
    """name, the call, how many outputs and workspaces it makes"""
    x, r, w, q = dev(6, 8, dtype=BF16), dev(6), dev(8), dev(12, 8, dtype=BF16)
    pos, off, W = dev(6, 2, dtype=I32), dev(4, dtype=I32), dev(3, 8, 8, dtype=BF16)
    yield "norm_rows", lambda: B.lasnet_norm_rows(x, w, 1e-6, residual=x, out_dtype=E4M3, **k), 3, 0
    yield "norm_rows_backward", lambda: B.lasnet_norm_rows_backward(x, x, w, r, **k), 2, 1
    yield "route", lambda: B.lasnet_route(pos, 3, **k), 3, 1
    yield "dispatch_rows", lambda: B.lasnet_dispatch_rows(x.to(E4M3).as_subclass(OnDevice), pos, off, scale=dev(6, dtype=torch.uint8), **k), 2, 0
    yield "combine_rows", lambda: B.lasnet_combine_rows(q, pos, **k), 1, 0
    yield "combine_rows_backward", lambda: B.lasnet_combine_rows_backward(x, q, pos, off, **k), 2, 0
    yield "expert_product", lambda: B.lasnet_expert_product(q, off, W, **k), 1, 0
    yield "expert_product_dx", lambda: B.lasnet_expert_product_dx(q, off, W, **k), 1, 0
    yield "expert_product_dw", lambda: B.lasnet_expert_product_dw(q, q, off, **k), 1, 1


def map_calls(k):
    x, f, idx, M, C = dev(1, 4, 4, 64, dtype=BF16), dev(64), dev(4, dtype=I32), 16, 64
    W = (dev(M, C, dtype=BF16), dev(M), dev(M, 3, 3, M, dtype=BF16), dev(M), dev(C, M, dtype=BF16), f)
    yield "masker", lambda: B.lasnet_masker(x, f, 0.0, 2, **k), 3
    yield "masker_ex", lambda: B.lasnet_masker_ex(x, f, 0.0, 2, pass_out=x, **k), 3
    yield "masker_logits", lambda: B.lasnet_masker_logits(x, f, 0.0, 2, **k), 1
    yield "block", lambda: B.lasnet_sparse_bottleneck(x, idx, idx[:1], 2, *W, **k), 1
    yield "dense", lambda: B.lasnet_dense_bottleneck(x, *W, **k), 1
    yield "pack", lambda: B.lasnet_pack_weights(2, W[0], W[2], W[4], **k), 1
    yield "packed", lambda: B.lasnet_sparse_bottleneck_packed(x, idx, idx[:1], 2, M, dev(128), dev(M), dev(M), f, **k), 1


@pytest.fixture
def made(monkeypatch):
    """What is made: (tensor, the stream it is made under)."""
    current, made, empty = [CURRENT], [], torch.empty

    @contextlib.contextmanager
    def switched(s):
        before, current[0] = current[0], s
        yield
        current[0] = before

    def recorded(*a, **k):
        made.append((empty(*a, **k).as_subclass(OnDevice), current[0]))
        return made[-1][0]

    monkeypatch.setattr(torch.cuda, "stream", switched)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[0])
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch._C, "_cuda_setStream", lambda stream_id, device_index, device_type: current.__setitem__(0, _Stream.by_id[stream_id]), raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch, "empty", recorded)
    monkeypatch.setattr(B, "_stream", lambda s: 0 if s is None else s.cuda_stream)
    monkeypatch.setattr(B, "_lib", NoLibrary())
    monkeypatch.setattr(B, "_marshal", B._AllThroughCtypes)
    return made


class _Stream:
    device_index, device_type, by_id = 0, 1, {}

    def __init__(self, handle):
        self.stream_id = self.cuda_stream = handle
        self.by_id[handle] = self


CURRENT, SIDE = _Stream(0x11), _Stream(0x77)


@pytest.mark.parametrize("which", range(9))
def test_rows_what_a_call_makes_is_memory_of_its_stream(which, made):
    for given in (None, CURRENT, SIDE):
        name, call, outputs, workspaces = list(row_calls({} if given is None else {"stream": given}))[which]
        made.clear()
        call()
        assert [s for _, s in made] == [given or CURRENT] * (outputs + workspaces), name
        used = [getattr(t, "used_on", []) for t, _ in made]
        assert used == [[CURRENT] if given is SIDE else []] * outputs + [[]] * workspaces, name


@pytest.mark.parametrize("which", range(7))
def test_maps_what_a_call_makes_is_memory_of_its_stream(which, made):
    for given in (None, CURRENT, SIDE):
        name, call, outputs = list(map_calls({} if given is None else {"stream": given}))[which]
        made.clear()
        call()
        assert [s for _, s in made] == [given or CURRENT] * outputs, name
        assert [getattr(t, "used_on", []) for t, _ in made] == [[CURRENT] if given is SIDE else []] * outputs, name


@pytest.mark.gpu
def test_maps_on_another_stream_while_the_current_one_is_busy():
    """As below, for a masker, its list and a block (its memory beyond the arguments is the library's, one buffer for each stream)."""
    g = torch.Generator().manual_seed(2)
    x, Wm = torch.randn(2, 14, 14, 64, generator=g).to(BF16).cuda(), torch.randn(64, generator=g).cuda()
    W = [torch.randn(*s, generator=g).mul_(0.05).to(BF16 if len(s) > 1 else torch.float32).cuda() for s in ((16, 64), (16,), (16, 3, 3, 16), (16,), (64, 16), (64,))]

    def path(**s):
        mask, idx, count = B.lasnet_masker(x, Wm, 0.0, 2, **s)
        return mask, count, B.lasnet_sparse_bottleneck(x, idx, count, 2, *W, **s)

    want = path()
    side, a, b = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda"), torch.empty(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for i in range(5):
        print("busy", i, flush=True)
        side.wait_stream(torch.cuda.current_stream())
        torch.mm(a, a, out=b)
        blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (98, 392, 4, x.numel() * 2) for _ in range(2)]
        for t in blocks:
            t.fill_(255)
        del blocks, t
        got = path(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        for x1, x2 in zip(got, want):
            assert torch.equal(x1, x2), i


@pytest.mark.gpu
def test_rows_on_another_stream_while_the_current_one_is_busy():
    """Workspaces and outputs of calls on a side stream, made while the current stream still has to write to blocks of their sizes that were freed before: the
    results are those of the default stream, every time."""
    g = torch.Generator().manual_seed(1)
    rows, C, E, k = 13000, 136, 2, 2
    x, dy = (torch.randn(rows, C, generator=g).to(BF16).cuda() for _ in range(2))
    w, e = torch.randn(C, generator=g).cuda(), torch.randint(-1, E, (rows, k), generator=g, dtype=I32).cuda()
    rstd = torch.rsqrt(x.float().square().mean(-1) + 1e-6)
    offsets = torch.tensor([0, 6000, 12500], dtype=I32).cuda()
    L = B.lib()
    sizes = [L.lasnet_norm_rows_backward_workspace_bytes(rows, C), L.lasnet_route_workspace_bytes(rows, k, E), L.lasnet_expert_product_dw_workspace_bytes(rows, E, C, C)]
    assert all(sizes)
    sizes += [x.numel() * 2, C * 4, rows * k * 4, (E + 1) * 4, E * C * C * 2]

    def path(**s):
        return [*B.lasnet_norm_rows_backward(dy, x, w, rstd, **s), *B.lasnet_route(e, E, **s), B.lasnet_expert_product_dw(dy, x, offsets, **s)]

    want = path()
    side, a, b = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda"), torch.empty(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for i in range(5):
        print("busy", i, flush=True)
        side.wait_stream(torch.cuda.current_stream())
        torch.mm(a, a, out=b)                                    # (some 0.2 ms before the blocks below are written)
        blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
        for t in blocks:
            t.fill_(255)
        del blocks, t
        got = path(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        for x1, x2 in zip(got, want):
            assert torch.equal(x1, x2), i
