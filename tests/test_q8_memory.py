"""Which memory the binding hands to a call in 8 bits: pools, streams, devices, sizes, by the stand-ins of test_block_memory.py.  Nothing here
needs a device."""
import pytest
import torch

import paper_2503_14376_amd as tfla
from tests.test_block_memory import BF16, F32, Stream, Tensor, machine, tensors  # noqa: F401

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def calls(M=300, K=333, N=200, device=0):
    """every operator and direction with tensors of its own: name -> (call, its input tensors)"""
    def t(*shape, d=BF16):
        return Tensor(shape, d, device)
    kb, nb = -(-K // 128), -(-N // 128)
    x, r, dy, z, u, res = t(M, K), t(M, K), t(M, N), t(M, N), t(M, N), t(M, N)
    g, n = t(K, d=F32), t(N, d=F32)
    xq, xs = t(M, K, d=E4M3), t(kb, M, d=E8M0)
    w, ws, w2, ws2 = t(N, K, d=E4M3), t(kb, nb, d=E8M0), t(N, K, d=E4M3), t(kb, nb, d=E8M0)
    wt, wst, wt2, wst2 = t(K, N, d=E4M3), t(nb, kb, d=E8M0), t(K, N, d=E4M3), t(nb, kb, d=E8M0)
    return {
        "q8_quant": (lambda **k: tfla.q8_quant(x, want_t=True, **k), [x]),
        "norm_q8_fwd": (lambda **k: tfla.norm_q8_fwd(x, g, g, r, norm_kind=tfla.NORM_LAYER, keep_y=True, **k), [x, g, r]),
        "linear_q8_fwd": (lambda **k: tfla.linear_q8_fwd(xq, xs, w, ws, n, res, act=tfla.ACT_SILU, keep_pre=True, **k), [xq, xs, w, ws, n, res]),
        "linear_q8_bwd": (lambda **k: tfla.linear_q8_bwd(x, wt, wst, dy, z, act=tfla.ACT_SILU, want_db=True, **k), [x, wt, wst, dy, z]),
        "gated_q8_fwd": (lambda **k: tfla.gated_q8_fwd(xq, xs, w, ws, w2, ws2, n, n, keep_pre=True, **k), [xq, xs, w, ws, w2, ws2, n]),
        "gated_q8_bwd": (lambda **k: tfla.gated_q8_bwd(x, wt, wst, wt2, wst2, z, u, dy, want_db=True, **k), [x, wt, wst, wt2, wst2, z, u, dy])}


NAMES = tuple(calls())
WITH_WORKSPACE = NAMES[2:]


@pytest.mark.parametrize("name", NAMES)
def test_streams(machine, name):  # noqa: F811
    """on another stream new memory is that stream's and everything else is recorded on it; on the current one nothing of the kind"""
    side = Stream(77)
    call, inputs = calls()[name]
    o = call(stream=side)
    assert machine.calls[-1][1][-1] == 77 and len(tensors(o)) >= 2
    for k, t in tensors(o).items():
        assert t.pool is side and machine.streams[0] in t.seen, k
    assert all(side in t.seen for t in inputs)
    call, inputs = calls()[name]
    o = call()
    assert machine.calls[-1][1][-1] == 0
    assert all(t.pool is machine.streams[0] and not t.seen for t in tensors(o).values()) and not any(t.seen for t in inputs)
    call(stream=side, out=o)
    assert all(side in t.seen for t in tensors(o).values())


@pytest.mark.parametrize("name", NAMES)
def test_devices(machine, name):  # noqa: F811
    call, _ = calls(device=1)[name]
    machine.streams[1] = Stream(91, 1)
    o = call()
    assert machine.calls[-1][2] == 1 and machine.device == 0 and machine.calls[-1][1][-1] == 91
    assert all(t.get_device() == 1 and t.pool is machine.streams[1] for t in tensors(o).values())
    call, inputs = calls()[name]
    with pytest.raises(ValueError):
        call(stream=Stream(93, 1))
    for t in inputs if len(inputs) > 1 else ():         # (a call with one input runs where that is)
        t.device = torch.device("cuda", 1)
        with pytest.raises(ValueError):
            call()
        t.device = torch.device("cuda", 0)
    o = tensors(call())
    for k in o:
        o[k].device = torch.device("cuda", 1)
        with pytest.raises(ValueError):
            call(out=dict(o))
        o[k].device = torch.device("cuda", 0)
    assert len(machine.calls) == 2


@pytest.mark.parametrize("name", NAMES)
def test_types_and_shapes(machine, name):  # noqa: F811
    """every tensor of the call in another type, with a row more, or with gaps is refused"""
    call, inputs = calls()[name]
    o = {k: t for k, t in tensors(call()).items() if k != "workspace"}
    for t in list(inputs) + list(o.values()):
        dtype, shape = t.dtype, t.shape
        for change in ({"dtype": torch.float16}, {"shape": (shape[0] + 256,) + shape[1:]}, {"is_contiguous": lambda: False}):
            if name == "q8_quant" and t is inputs[0] and "shape" in change:
                continue            # (the one tensor that all the others follow)
            t.__dict__.update(change)
            with pytest.raises(ValueError):
                call(out=dict(o))
            t.dtype, t.shape = dtype, shape
            t.__dict__.pop("is_contiguous", None)
    call(out=dict(o))
    assert len(machine.calls) == 2


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("which", ["M", "K", "N"])
def test_sizes_beyond_32_bits_are_refused(machine, name, which):  # noqa: F811
    if name in ("q8_quant", "norm_q8_fwd") and which == "N":
        which = "K"
    for n in (1 << 31, (1 << 32) + 4):
        with pytest.raises(ValueError):
            calls(**{"M": 2, "K": 3, "N": 2, which: n})[name][0]()
    assert not machine.calls


@pytest.mark.parametrize("name", WITH_WORKSPACE)
def test_workspaces(machine, name):  # noqa: F811
    """a kept one is used again and recorded where it is; a caller's own is not kept; memory that the device cannot use is refused"""
    def given():
        args = machine.calls[-1][1]
        return args[-3], args[-2]
    call, _ = calls()[name]
    o = call()
    ws = o["workspace"]
    assert given() == (ws.address, ws.numel()) and ws.numel() > 0
    side = Stream(81)
    call(stream=side, out=o)
    assert o["workspace"] is ws and side in ws.seen
    mine = Tensor((1 << 24,), torch.uint8)
    p = call(workspace=mine)
    assert given() == (mine.address, 1 << 24) and p["workspace"] is None
    n = len(machine.calls)
    host, gaps = (Tensor((1 << 24,), torch.uint8) for _ in range(2))
    host.get_device = lambda: -1
    gaps.is_contiguous = lambda: False
    for bad in (host, gaps):
        with pytest.raises(ValueError):
            call(workspace=bad)
        with pytest.raises(ValueError):
            call(out={"workspace": bad})
    assert len(machine.calls) == n


def test_backward_calls_take_what_they_read(machine):  # noqa: F811
    M, K, N = 40, 24, 16
    x, dy, a, u = (Tensor(s) for s in ((M, K), (M, N), (M, N), (M, N)))
    w, w2, s, s2 = Tensor((K, N), E4M3), Tensor((K, N), E4M3), Tensor((1, 1), E8M0), Tensor((1, 1), E8M0)
    both = ((lambda x, w, s, **k: tfla.linear_q8_bwd(x, w, s, dy, **k), ("dx", "dw", "db")),
            (lambda x, w, s, **k: tfla.gated_q8_bwd(x, w, s, w and w2, s and s2, a, u, dy, **k), ("dx", "dw_gate", "db_gate")))
    for call, (dx, dw, db) in both:
        o = call(None, w, s, want_dw=False)
        assert o[dx].shape == (M, K) and machine.calls[-1][1][0] is None
        o = call(x, None, None, want_dx=False, want_db=True)
        assert o[dw].shape == (N, K) and machine.calls[-1][1][1] is None
        o = call(None, None, None, want_dx=False, want_dw=False, want_db=True)
        assert o[db].shape == (N,) and dx not in o and dw not in o
        n = len(machine.calls)
        for t, k in (((None, w, s), {}), ((x, None, s), {}), ((x, w, None), {}), ((None, None, None), {"want_dw": False})):
            with pytest.raises(ValueError):
                call(*t, **k)
        assert len(machine.calls) == n
