"""Which memory the binding hands to a call: pools, streams and devices, by stand-ins for device tensors,
streams and the library's launching calls (its workspace queries are the real ones).  Nothing here needs a device."""
import contextlib
import os

import pytest
import torch

import paper_2503_14376_amd as tfla
from paper_2503_14376_amd import binding

F32, BF16 = torch.float32, torch.bfloat16


class Stream:
    def __init__(self, handle, device=0):
        self.cuda_stream, self.device = handle, torch.device("cuda", device)


class Tensor:
    """what the binding asks of a device tensor; `pool`: the stream whose memory it is, `seen`: the streams recorded on it"""
    count = 0

    def __init__(self, shape, dtype=BF16, device=0, pool=None):
        self.shape, self.dtype, self.device, self.pool, self.seen = tuple(shape), dtype, torch.device("cuda", device), pool, set()
        Tensor.count += 1
        self.address = Tensor.count << 40
        self.is_cuda = True

    def get_device(self):
        return self.device.index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.address

    def numel(self):
        n = 1
        for d in self.shape:
            n *= d
        return n

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size() if self.dtype != torch.uint8 else 1

    def record_stream(self, stream):
        self.seen.add(stream)


class Machine:
    """the current stream and device, and what was launched: (name, arguments, device that was current)"""

    def __init__(self, monkeypatch):
        self.device, self.streams, self.calls = 0, [Stream(0, 0), Stream(0, 1)], []
        empty = torch.empty
        real = binding.load_library()

        def new(shape, dtype=None, device=None):
            if device is None:
                return empty(shape, dtype=dtype)
            d = index(device)
            return Tensor((shape,) if isinstance(shape, int) else shape, dtype, d, self.streams[d])

        @contextlib.contextmanager
        def on_stream(s):
            d, before, at = s.device.index, self.streams[s.device.index], self.device
            self.streams[d], self.device = s, d
            yield
            self.streams[d], self.device = before, at

        @contextlib.contextmanager
        def on_device(d):
            before, self.device = self.device, d if isinstance(d, int) else d.index
            yield
            self.device = before

        class Library:
            def __getattr__(lib, name):
                if name.endswith("_bytes"):
                    return getattr(real, name)

                def launch(*args):
                    self.calls.append((name, args, self.device))
                    return 0
                return launch

        def index(device):
            return self.device if device is None else device if isinstance(device, int) else torch.device(device).index

        monkeypatch.setattr(torch, "empty", new)
        monkeypatch.setattr(torch, "empty_like", lambda t: new(t.shape, t.dtype, t.device))
        monkeypatch.setattr(torch.cuda, "stream", on_stream)
        monkeypatch.setattr(torch.cuda, "device", on_device)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.streams[index(device)])
        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.device)
        monkeypatch.setattr(torch.cuda, "device_count", lambda: len(self.streams))
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: self.streams[d].cuda_stream, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.device, raising=False)
        monkeypatch.setattr(binding, "_torch_names", None)
        monkeypatch.setattr(binding, "_lib", Library())


@pytest.fixture
def machine(monkeypatch):
    if not os.path.exists(binding.lib_path()):
        from paper_2503_14376_amd import build
        build.build(verbose=False)
    yield Machine(monkeypatch)


def calls(M=300, K=333, N=200, dtype=BF16, device=0):
    """every operator and direction with tensors of its own: name -> (call, its input tensors)"""
    def t(*shape, d=dtype):
        return Tensor(shape, d, device)
    x, w, w2, y, dy, z = t(M, K), t(N, K), t(N, K), t(M, N), t(M, N), t(M, N)
    g, b, n, stat, mean = t(K, d=F32), t(K, d=F32), t(N, d=F32), t(M, d=F32), t(M, d=F32)
    dx, res = t(M, K), t(M, K)
    return {
        "norm_fwd": (lambda **k: tfla.norm_fwd(x, g, b, norm_kind=tfla.NORM_LAYER, **k), [x, g, b]),
        "norm_bwd": (lambda **k: tfla.norm_bwd(x, dx, stat, mean, g, res, norm_kind=tfla.NORM_LAYER, want_dbeta=True, **k),
                     [x, dx, stat, mean, g, res]),
        "linear_fwd": (lambda **k: tfla.linear_fwd(x, w, n, y, act=tfla.ACT_SILU, keep_pre=True, **k), [x, w, n, y]),
        "linear_bwd": (lambda **k: tfla.linear_bwd(x, w, dy, z, act=tfla.ACT_SILU, want_db=True, **k), [x, w, dy, z]),
        "gated_fwd": (lambda **k: tfla.gated_fwd(x, w, w2, n, n, keep_pre=True, **k), [x, w, w2, n]),
        "gated_bwd": (lambda **k: tfla.gated_bwd(x, w, w2, y, z, dy, want_db=True, **k), [x, w, w2, y, z, dy])}


NAMES = ("norm_fwd", "norm_bwd", "linear_fwd", "linear_bwd", "gated_fwd", "gated_bwd")


def tensors(o):
    return {k: v for k, v in o.items() if v is not None}


@pytest.mark.parametrize("name", NAMES)
def test_a_call_on_another_stream_takes_memory_of_that_stream(machine, name):
    """new outputs and workspaces come from the pool of the stream that writes them, and the current stream may drop them at any time"""
    side = Stream(77)
    call, inputs = calls()[name]
    o = call(stream=side)
    assert machine.calls[-1][1][-1] == 77
    assert len(tensors(o)) >= 2
    for k, t in tensors(o).items():
        assert t.pool is side, k
        assert machine.streams[0] in t.seen, k
    for t in inputs:
        assert side in t.seen
    assert machine.streams[0].cuda_stream == 0


@pytest.mark.parametrize("name", NAMES)
def test_a_call_on_the_current_stream_takes_its_memory(machine, name):
    call, inputs = calls()[name]
    o = call()
    assert machine.calls[-1][1][-1] == 0
    for t in list(tensors(o).values()):
        assert t.pool is machine.streams[0] and not t.seen
    assert not any(t.seen for t in inputs)


@pytest.mark.parametrize("name", NAMES)
def test_outputs_used_on_another_stream_are_recorded_there(machine, name):
    side = Stream(78)
    call, _ = calls()[name]
    o = call()
    call(stream=side, out=o)
    for k, t in tensors(o).items():
        if k != "workspace":
            assert side in t.seen, k


# ---- the workspace that `out` keeps ---------------------------------------------------------------------------------
WITH_WORKSPACE = ("norm_bwd", "linear_fwd", "linear_bwd", "gated_fwd", "gated_bwd")


def workspace_of(machine, name):
    """address and size that the last call was given"""
    where = {"norm_bwd": 13, "linear_fwd": 11, "linear_bwd": 12, "gated_fwd": 13, "gated_bwd": 16}[name]
    n, args, _ = machine.calls[-1]
    assert n == "tfla_" + name
    return args[where], args[where + 1]


@pytest.mark.parametrize("name", WITH_WORKSPACE)
def test_the_kept_workspace_is_recorded_on_every_stream_that_uses_it(machine, name):
    side = Stream(81)
    call, _ = calls()[name]
    o = call()
    ws = o["workspace"]
    assert workspace_of(machine, name) == (ws.address, ws.numel())
    call(stream=side, out=o)
    assert o["workspace"] is ws and side in ws.seen
    # and back: a later use on the current stream, which is another one now
    machine.streams[0] = other = Stream(82)
    call(out=o)
    assert other in ws.seen
    # no second look at a stream it knows
    ws.seen.clear()
    call(out=o)
    assert not ws.seen


@pytest.mark.parametrize("name", WITH_WORKSPACE)
def test_a_workspace_that_became_too_small_stays_alive(machine, name):
    """a graph that was captured with it holds its address for as long as the caller keeps `out`"""
    import gc
    import weakref
    call, _ = calls()[name]
    o = call()
    ws = weakref.ref(o["workspace"])
    keep = {"workspace": o.pop("workspace")}
    del o
    big = calls(M=4000, K=2001, N=1203)[name][0](out=keep)
    assert big["workspace"].numel() > ws().numel()
    assert workspace_of(machine, name)[0] == big["workspace"].address
    del big
    gc.collect()
    assert ws() is not None
    keep.clear()
    gc.collect()
    assert ws() is None


@pytest.mark.parametrize("name", WITH_WORKSPACE)
def test_a_callers_workspace_is_not_kept(machine, name):
    side = Stream(83)
    call, _ = calls()[name]
    mine = Tensor((1 << 24,), torch.uint8, pool=machine.streams[0])
    o = call(workspace=mine, stream=side)
    assert workspace_of(machine, name) == (mine.address, 1 << 24) and side in mine.seen
    assert o["workspace"] is None
    call(out=o)
    assert o["workspace"] is not mine and workspace_of(machine, name)[0] == o["workspace"].address
    # its size counts in bytes
    call(workspace=Tensor((1 << 20,), F32))
    assert workspace_of(machine, name)[1] == 4 << 20


# ---- devices --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("name", NAMES)
def test_a_call_runs_on_its_tensors_device(machine, name):
    """the handle of a default stream is 0 on every device: it means the current one's, which has to be the tensors'"""
    call, _ = calls(device=1)[name]
    o = call()
    _, args, device = machine.calls[-1]
    assert device == 1 and machine.device == 0
    for t in tensors(o).values():
        assert t.get_device() == 1 and t.pool is machine.streams[1]
    machine.streams[1] = Stream(91, 1)
    call()
    assert machine.calls[-1][1][-1] == 91
    side = Stream(92, 1)
    o = call(stream=side)
    assert machine.calls[-1][1][-1] == 92 and machine.calls[-1][2] == 1
    for t in tensors(o).values():
        assert t.pool is side and machine.streams[1] in t.seen


@pytest.mark.parametrize("name", NAMES)
def test_tensors_and_streams_of_other_devices_are_refused(machine, name):
    call, inputs = calls()[name]
    with pytest.raises(ValueError):
        call(stream=Stream(93, 1))
    for t in inputs:
        t.device = torch.device("cuda", 1)
        with pytest.raises(ValueError):
            call()
        t.device = torch.device("cuda", 0)
    o = tensors(call())
    for k in o:
        if k != "workspace":
            o[k].device = torch.device("cuda", 1)
            with pytest.raises(ValueError):
                call(out=dict(o))
            o[k].device = torch.device("cuda", 0)
    assert len(machine.calls) == 1


# ---- sizes of 2^31 and more, which ctypes would cut off --------------------------------------------------------------
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("which", ["M", "K", "N"])
def test_sizes_beyond_32_bits_are_refused(machine, name, which):
    import ctypes
    assert ctypes.c_int((1 << 32) + 4).value == 4
    if name.startswith("norm") and which == "N":
        which = "K"
    sizes = {"M": 2, "K": 3, "N": 2}
    for n in (1 << 31, (1 << 32) + 4):
        sizes[which] = n
        with pytest.raises(ValueError):
            calls(**sizes)[name][0]()
    assert not machine.calls


@pytest.mark.parametrize("name", WITH_WORKSPACE)
def test_a_workspace_that_the_device_cannot_use_is_refused(machine, name):
    """host memory, memory of another device, or a tensor with gaps"""
    call, _ = calls()[name]
    host, other, gaps = (Tensor((1 << 24,), torch.uint8) for _ in range(3))
    host.get_device = lambda: -1
    other.device = torch.device("cuda", 1)
    gaps.is_contiguous = lambda: False
    for bad in (host, other, gaps):
        with pytest.raises(ValueError):
            call(workspace=bad)
        with pytest.raises(ValueError):
            call(out={"workspace": bad})
    assert not machine.calls


# ---- the cell's calls: memory and streams ---------------------------------------------------------------------------
def cell_calls(B=1, H=2, T=128, k=64, v=64):
    def t(*shape, d=BF16):
        return Tensor(shape, d)
    q, kk, u, o, dy, y = t(B, H, T, k), t(B, H, T, k), t(B, H, T, v), t(B, H, T, v), t(B, H, T, v), t(B, H, T, v)
    i, f, n, m = (t(B, H, T, d=F32) for _ in range(4))
    g, C, nn, mm = t(H, v, d=F32), t(B, H, k, v, d=F32), t(B, H, k, d=F32), t(B, H, d=F32)
    q1, k1, u1, o1, i1, f1 = t(B, H, k), t(B, H, k), t(B, H, v), t(B, H, v), t(B, H, d=F32), t(B, H, d=F32)
    outs = {"H": t(B, H, T, v), "Cn": t(B, H, k, v, d=F32), "nn": t(B, H, k, d=F32), "mn": t(B, H, d=F32), "n_out": t(B, H, T, d=F32),
            "m_out": t(B, H, T, d=F32)}

    def static(**kw):
        return tfla.mlstm_fwd_static(q, kk, u, i, f, C, nn, mm, chunk=64, **{"out": outs, **kw})
    return {
        "fwd": (lambda **kw: tfla.mlstm_fwd(q, kk, u, i, f, C, nn, mm, chunk=64, **kw), [q, kk, u, i, f, C, nn, mm]),
        "static": (static, [q, kk, u, i, f, C, nn, mm] + list(outs.values())),
        "bwd": (lambda **kw: tfla.mlstm_bwd(q, kk, u, i, f, dy, n, m, C, nn, mm, chunk=64, **kw), [q, kk, u, i, f, dy, n, m, C, nn, mm]),
        "step": (lambda **kw: tfla.mlstm_step(q1, k1, u1, i1, f1, C, nn, mm, **kw), [q1, k1, u1, i1, f1, C, nn, mm]),
        "layer_fwd": (lambda **kw: tfla.mlstm_layer_fwd(q, kk, u, i, f, o, g, g, C, nn, mm, chunk=64, **kw), [q, kk, u, i, f, o, g, C, nn, mm]),
        "layer_bwd": (lambda **kw: tfla.mlstm_layer_bwd(q, kk, u, i, f, y, dy, o, g, g, n, m, C, nn, mm, chunk=64, **kw),
                      [q, kk, u, i, f, y, dy, o, g, n, m, C, nn, mm]),
        "layer_step": (lambda **kw: tfla.mlstm_layer_step(q1, k1, u1, i1, f1, C, nn, mm, o1, g, g, **kw), [q1, k1, u1, i1, f1, o1, g, C, nn, mm]),
        "gain": (lambda **kw: dict(enumerate(tfla.transfer_gain(u, y, **kw))), [u, y])}


@pytest.mark.parametrize("name", list(cell_calls()))
def test_the_cells_calls_on_another_stream(machine, name):
    """as above: new memory from the stream's pool, everything else recorded on it; on the current stream nothing of the kind"""
    side = Stream(95)
    call, inputs = cell_calls()[name]
    o = call(stream=side)
    assert machine.calls[-1][1][-1] == 95
    for k, t in tensors(o).items():
        assert t in inputs or (t.pool is side and machine.streams[0] in t.seen), k
    for t in inputs:
        assert side in t.seen
    if name not in ("gain", "static"):
        call, _ = cell_calls()[name]
        o = call()
        for t in tensors(o).values():
            assert t.pool is machine.streams[0] and not t.seen
        kept = {k: t for k, t in tensors(o).items() if k != "workspace"}
        call(stream=side, out=dict(kept))
        assert all(side in t.seen for t in kept.values())
    call, inputs = cell_calls()[name]
    call()
    assert machine.calls[-1][1][-1] == 0 and not any(t.seen for t in inputs)


# ---- backward calls need the tensors that they read -----------------------------------------------------------------
def test_backward_calls_take_what_they_read(machine):
    M, K, N = 40, 24, 16
    x, w, w2, dy, a, u = (Tensor(s) for s in ((M, K), (N, K), (N, K), (M, N), (M, N), (M, N)))
    both = ((lambda x, w, **k: tfla.linear_bwd(x, w, dy, **k), ("dx", "dw", "db")),
            (lambda x, w, **k: tfla.gated_bwd(x, w, None if w is None else w2, a, u, dy, **k), ("dx", "dw_gate", "db_gate")))
    for call, (dx, dw, db) in both:
        o = call(None, w, want_dw=False)
        assert o[dx].shape == (M, K) and machine.calls[-1][1][0] is None
        o = call(x, None, want_dx=False, want_db=True)
        assert o[dw].shape == (N, K) and machine.calls[-1][1][1] is None
        o = call(None, None, want_dx=False, want_dw=False, want_db=True)
        assert o[db].shape == (N,) and dx not in o and dw not in o
        n = len(machine.calls)
        for bad in (dict(x=None, w=w), dict(x=x, w=None), dict(x=None, w=None, want_dw=False), dict(x=None, w=None, want_dx=False)):
            with pytest.raises(ValueError):
                call(bad.pop("x"), bad.pop("w"), **bad)
        assert len(machine.calls) == n


@pytest.mark.parametrize("name", ("linear_fwd", "layer_fwd"))
def test_a_stream_may_be_anything_with_a_handle(machine, monkeypatch, name):
    class Handle:
        cuda_stream = 96
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    call, _ = {**calls(), **cell_calls()}[name]
    o = call(stream=Handle())
    assert machine.calls[-1][1][-1] == 96 and all(t.pool.cuda_stream == 96 for t in tensors(o).values())
