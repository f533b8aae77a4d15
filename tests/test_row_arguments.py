"""Arguments of the calls on rows that are refused before anything is enqueued: workspaces in the wrong memory, outputs at the address of another argument."""
import ctypes

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


def test_tensors_without_rows_are_refused_as_such():
    """(With all outputs given and without.)"""
    x, w, none, i = torch.zeros(2, 4), torch.zeros(4), torch.zeros(()), torch.zeros((), dtype=I32)
    for kw in (dict(), dict(dx=x, dweight=w)):
        with pytest.raises(ValueError, match="rows"):
            B.lasnet_norm_rows_backward(none.as_subclass(OnDevice), none.as_subclass(OnDevice), w, w, **kw)
    for kw in (dict(), dict(offsets=i, order=i, position=i)):
        with pytest.raises(ValueError, match="experts"):
            B.lasnet_route(i, 3, **kw)
    for kw in (dict(), dict(dW=none)):
        with pytest.raises(ValueError, match="rows|offsets"):
            B.lasnet_expert_product_dw(none, none, dev(3, dtype=I32), **kw)


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


# Entries: their arguments in order, (name, kind) of an address ("i": input, "o": output; "ri", "ro": rows, with their numbers of rows and columns and type) or a plain value; and the
# pairs that may be the same rows.
F, H = B.LASNET_F32, B.LASNET_BF16
ENTRIES = {
    "norm_rows": ([("x", "ri", 8, 16, H), ("residual", "ri", 8, 16, H), ("weight", "i"), 1e-6, ("sum_out", "ro", 8, 16, H), ("out", "ro", 8, 16, B.LASNET_E4M3), ("scale", "o"),
                   ("rstd", "o"), None], {("sum_out", "x"), ("sum_out", "residual")}),
    "norm_rows_backward": ([("dy", "ri", 8, 16, H), ("s", "ri", 8, 16, H), ("weight", "i"), ("rstd", "i"), ("dsum", "ri", 8, 16, H), ("dx", "ro", 8, 16, H), ("dweight", "o"),
                            ("workspace", "o"), 1 << 20, None], {("dx", "dy"), ("dx", "dsum")}),
    "route": ([("experts", "i"), 100000, 2, 4, ("offsets", "o"), ("order", "o"), ("position", "o"), ("workspace", "o"), 1 << 24, None], set()),
    "dispatch_rows": ([("x", "ri", 8, 16, B.LASNET_E4M3), ("scale", "i"), ("position", "i"), ("offsets", "i"), 2, 4, ("out", "ro", 16, 16, B.LASNET_E4M3), ("out_scale", "o"), None],
                      set()),
    "combine_rows": ([("y", "ri", 16, 16, F), ("weights", "i"), ("position", "i"), 2, ("base", "ri", 8, 16, F), ("out", "ro", 8, 16, F), None], {("out", "base")}),
    "combine_rows_backward": ([("dout", "ri", 8, 16, F), ("y", "ri", 16, 16, F), ("weights", "i"), ("position", "i"), ("offsets", "i"), 2, 4, ("dy", "ro", 16, 16, F),
                               ("dweights", "o"), None], {("dy", "y")}),
    "expert_product": ([("x", "ri", 8, 16, B.LASNET_E4M3), ("scale", "i"), ("offsets", "i"), 2, ("W", "i"), ("wscale", "i"), ("out", "ro", 8, 16, H), 0, None], set()),
    "expert_product_dx": ([("dy", "ri", 8, 16, H), ("offsets", "i"), 2, ("W", "i"), ("dx", "ro", 8, 16, H), None], set()),
    "expert_product_dw_ex": ([("dy", "ri", 8, 16, H), ("x", "ri", 8, 16, H), ("offsets", "i"), 2, ("dW", "o"), F, ("workspace", "o"), 1 << 20, None], set()),
}

_PROBE = r"""
class Rows(ctypes.Structure):
    _fields_ = [("data", vp), ("rows", ctypes.c_int64), ("stride", ctypes.c_int64), ("cols", ctypes.c_int32), ("dtype", ctypes.c_int32)]
def enter(name, args, same=None):
    # the entry's status; same: two names, the first of which gets the second's address
    at = {a[0]: (i + 1) << 32 for i, a in enumerate(args) if isinstance(a, list)}
    if same:
        at[same[0]] = at[same[1]]
    passed = []
    for a in args:
        if not isinstance(a, list):
            passed.append(ctypes.c_float(a) if isinstance(a, float) else vp(None) if a is None else ctypes.c_longlong(a))
        elif a[1][0] == "r":
            passed.append(ctypes.byref(Rows(at[a[0]], a[2], 0, a[3], a[4])))
        else:
            passed.append(vp(at[a[0]]))
    F.fake_set(-1, 0, 0)
    st = getattr(L, "lasnet_" + name)(*passed)
    return st, sum(l.startswith("launch") for l in F.fake_log().decode().splitlines())
result = {}
for name, (args, pairs) in ENTRIES.items():
    result[name] = {"apart": enter(name, args), "pairs": [[p, enter(name, args, p)] for p in pairs]}
"""


def test_an_output_at_the_address_of_another_argument_is_refused():
    """Of every output with every input and every other output, as the header says; pairs that may be the same rows, and arguments all apart, are enqueued.  (On the
    recording runtime: nothing runs.)"""
    from tests import _fake_hip
    table = {}
    for name, (args, allowed) in ENTRIES.items():
        named = [a for a in args if isinstance(a, tuple)]
        outs = [a[0] for a in named if a[1].endswith("o")]
        table[name] = ([list(a) if isinstance(a, tuple) else a for a in args], [[o, a[0]] for o in outs for a in named if a[0] != o])
    got = _fake_hip.run("ENTRIES = %r\n" % table + _PROBE)
    for name, (args, allowed) in ENTRIES.items():
        st, launches = got[name]["apart"]
        assert st == B.LASNET_OK and launches > 0, name
        for (o, other), (st, launches) in got[name]["pairs"]:
            if (o, other) in allowed or (other, o) in allowed:
                assert st == B.LASNET_OK and launches > 0, (name, o, other)
            else:
                assert st == B.LASNET_EALIAS and launches == 0, (name, o, other, st)
