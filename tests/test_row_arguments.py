"""Arguments of the calls on rows that are refused before anything is enqueued: workspaces in the wrong memory."""
import pytest
import torch

from paper_2210_06223_amd import binding as B
from tests.test_call_streams import NoLibrary, OnDevice, dev

BF16, I32 = torch.bfloat16, torch.int32


def calls(make):
    """name, the call with a workspace, without its outputs and with them; make(*shape, dtype): a tensor"""
    x, r, w, q = make(6, 8, dtype=BF16), make(6), make(8), make(12, 8, dtype=BF16)
    e, off = make(6, 2, dtype=I32), make(4, dtype=I32)
    yield "norm", lambda ws: B.lasnet_norm_rows_backward(x, x, w, r, workspace=ws)
    yield "norm, outputs", lambda ws: B.lasnet_norm_rows_backward(q[:6], x, w, r, dx=make(6, 8, dtype=BF16), dweight=make(8), workspace=ws)
    yield "route", lambda ws: B.lasnet_route(e, 3, workspace=ws)
    yield "route, outputs", lambda ws: B.lasnet_route(e, 3, offsets=make(4, dtype=I32), order=make(12, dtype=I32), position=make(6, 2, dtype=I32), workspace=ws)
    yield "dw", lambda ws: B.lasnet_expert_product_dw(q, q, off, workspace=ws)
    yield "dw, outputs", lambda ws: B.lasnet_expert_product_dw(q, q, off, dW=make(3, 8, 8, dtype=BF16), workspace=ws)


class Recording(NoLibrary):
    def __init__(self):
        self.enqueued = []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda *a: 512
        return lambda *a: self.enqueued.append(name) or 0


@pytest.mark.parametrize("which", range(6))
def test_a_workspace_in_other_memory_is_refused(which, monkeypatch):
    L, real = Recording(), torch.empty
    monkeypatch.setattr(B, "_lib", L)
    monkeypatch.setattr(B, "_marshal", B._AllThroughCtypes)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: real(*a, **k).as_subclass(OnDevice))
    name, call = list(calls(dev))[which]
    elsewhere = torch.zeros(4096, dtype=torch.uint8, device="meta").as_subclass(OnDevice)         # (stands for another GPU)
    for ws in (torch.zeros(4096, dtype=torch.uint8), elsewhere, dev(64, 128, dtype=torch.uint8)[:, ::2], dev(1, dtype=torch.uint8).expand(4096)):
        with pytest.raises(ValueError, match="workspace"):
            call(ws)
    assert not L.enqueued, name
    call(dev(4096, dtype=torch.uint8))
    assert len(L.enqueued) == 1, name


@pytest.mark.gpu
def test_a_host_workspace_is_refused_natively_too():
    """(With the outputs given, the calls are offered to the native marshalling: it leaves them to the checks.)"""
    make = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device="cuda")
    for name, call in calls(make):
        for ws in (torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(1 << 20, dtype=torch.uint8).pin_memory(), make(64, 1 << 16, dtype=torch.uint8)[:, ::2]):
            with pytest.raises(ValueError, match="workspace"):
                call(ws)
        call(make(1 << 20, dtype=torch.uint8))
    torch.cuda.synchronize()
    L, x = B.lib(), make(6, 8, dtype=BF16)
    assert B._marshal.norm_rows_backward(L.at_norm_rows_backward, x, x, make(8), make(6), None, make(6, 8, dtype=BF16), make(8), torch.zeros(1 << 20, dtype=torch.uint8)) is None
