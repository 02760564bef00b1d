"""Host-side checks of the entry points in 8 bits: invalid arguments come back as the documented codes before anything is launched, the
workspace queries agree with the calls, and the binding refuses tensors that are not what a call needs.  No compute call is made
here: every call below fails its checks, or has no work."""
import pytest
import torch

from tests.test_block_arguments import ENUM, NULL, P, SHAPE, WORKSPACE, lib  # noqa: F401


def quant(lib, M=4, K=64, dtype=1, rows=1, x=P, q=P, s=P, qt=None, st=None):
    return lib.tfla_q8_quant(x, M, K, dtype, rows, q, s, qt, st, None)


@pytest.mark.parametrize("kw,rc", [(dict(M=-1), SHAPE), (dict(M=(1 << 24) + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=(1 << 20) + 1), SHAPE),
                                   (dict(M=1 << 24, K=1 << 13), SHAPE), (dict(dtype=2), ENUM), (dict(rows=0), ENUM), (dict(rows=64), ENUM),
                                   (dict(x=None), NULL), (dict(s=None), NULL), (dict(q=None), NULL), (dict(qt=P), NULL), (dict(st=P), NULL)])
def test_quantiser_refusals(lib, kw, rc):  # noqa: F811
    assert quant(lib, **kw) == rc


def norm(lib, M=4, D=64, dtype=1, kind=0, eps=1e-6, x=P, q=P, s=P):
    return lib.tfla_norm_q8_fwd(x, None, None, None, M, D, dtype, kind, eps, q, s, None, None, None, None, None)


@pytest.mark.parametrize("kw,rc", [(dict(M=-1), SHAPE), (dict(M=(1 << 24) + 1), SHAPE), (dict(D=0), SHAPE), (dict(D=16385), SHAPE),
                                   (dict(dtype=2), ENUM), (dict(kind=2), ENUM), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
                                   (dict(x=None), NULL), (dict(q=None), NULL), (dict(s=None), NULL)])
def test_norm_refusals(lib, kw, rc):  # noqa: F811
    assert norm(lib, **kw) == rc


def lin_fwd(lib, M=4, K=64, N=64, act=0, x=P, xs=P, w=P, s=P, y=P, ws=None, wsb=0):
    return lib.tfla_linear_q8_fwd(x, xs, w, s, None, None, M, K, N, act, y, None, ws, wsb, None)


def lin_bwd(lib, M=4, K=64, N=64, act=0, x=P, w=P, s=P, dy=P, z=None, dx=P, dw=P, ws=None, wsb=0):
    return lib.tfla_linear_q8_bwd(x, w, s, dy, z, M, K, N, act, dx, dw, P, ws, wsb, None)


def gat_fwd(lib, M=4, K=64, N=64, act=1, x=P, xs=P, wg=P, sg=P, wu=P, su=P, h=P, hs=P, ws=None, wsb=0):
    return lib.tfla_gated_q8_fwd(x, xs, wg, sg, wu, su, None, None, M, K, N, act, h, hs, None, None, None, ws, wsb, None)


def gat_bwd(lib, M=4, K=64, N=64, act=1, x=P, wg=P, sg=P, wu=P, su=P, a=P, u=P, dh=P, dx=P, dwg=P, dwu=P, ws=None, wsb=0):
    return lib.tfla_gated_q8_bwd(x, wg, sg, wu, su, a, u, dh, M, K, N, act, dx, dwg, dwu, P, P, ws, wsb, None)


DIMS = [(dict(M=-1), SHAPE), (dict(M=(1 << 24) + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=(1 << 20) + 1), SHAPE), (dict(N=-3), SHAPE),
        (dict(N=1 << 20, K=1 << 17), SHAPE), (dict(M=1 << 24, K=1 << 13), SHAPE), (dict(act=4), ENUM), (dict(act=-1), ENUM)]


@pytest.mark.parametrize("f", [lin_fwd, lin_bwd, gat_fwd, gat_bwd])
@pytest.mark.parametrize("kw,rc", DIMS)
def test_dimensions_are_refused(lib, f, kw, rc):  # noqa: F811
    assert f(lib, **kw) == rc


def test_backward_calls_take_fewer_tokens(lib):  # noqa: F811
    """offsets within a tile of the transposed operands are 32-bit"""
    for f in (lin_bwd, gat_bwd):
        assert f(lib, M=(1 << 21) + 1) == SHAPE and f(lib, M=1 << 21) == WORKSPACE
    for q in (lib.tfla_linear_q8_workspace_bytes, lib.tfla_gated_q8_workspace_bytes):
        assert q(1, (1 << 21) + 1, 64, 64, 0, 0) == 0 and q(1, 1 << 21, 64, 64, 0, 0) > 0


@pytest.mark.parametrize("f,names", [(lin_fwd, ("x", "xs", "w", "s", "y")), (lin_bwd, ("x", "w", "s", "dy")),
                                     (gat_fwd, ("x", "xs", "wg", "sg", "wu", "su", "h", "hs")), (gat_bwd, ("x", "wg", "sg", "wu", "su", "a", "u", "dh", "dwu"))])
def test_missing_tensors_are_refused(lib, f, names):  # noqa: F811
    for n in names:
        assert f(lib, **{n: None}) == NULL, n


def test_activations_need_what_the_forward_call_stored(lib):  # noqa: F811
    assert lin_bwd(lib, act=1) == NULL


@pytest.mark.parametrize("f,query", [(lin_fwd, "tfla_linear_q8_workspace_bytes"), (gat_fwd, "tfla_gated_q8_workspace_bytes")])
def test_a_workspace_is_asked_for_and_checked(lib, f, query):  # noqa: F811
    q = getattr(lib, query)
    need = q(0, 300, 333, 200, 1, 0)
    assert need >= 300 * 336                           # rows of 333 codes are copied into aligned ones
    kw = dict(M=300, K=333, N=200, act=1)
    assert f(lib, **kw) == WORKSPACE
    assert f(lib, ws=P, wsb=need - 1, **kw) == WORKSPACE
    assert f(lib, ws=P + 128, wsb=need, **kw) == WORKSPACE
    assert q(0, 300, 512, 256, 1, 1) >= q(0, 300, 512, 256, 1, 0) + 512 * (300 + 256)
    assert f(lib, M=300, K=512, N=256, x=P + 2, ws=P, wsb=q(0, 300, 512, 256, 1, 0)) == WORKSPACE
    for bad in ((2, 3, 64, 64, 0, 0), (0, -1, 64, 64, 0, 0), (1, 3, 0, 64, 0, 0), (1, 3, 64, 64, 9, 0)):
        assert q(*bad) == 0


def test_backward_workspaces(lib):  # noqa: F811
    for f, q, pair in ((lin_bwd, lib.tfla_linear_q8_workspace_bytes, 1), (gat_bwd, lib.tfla_gated_q8_workspace_bytes, 2)):
        need = q(1, 300, 512, 256, 0, 0)
        assert need >= pair * 2 * 300 * 256 + 512 * 300
        assert q(1, 300, 512, 256, 0, 1) >= need + pair * 512 * 256
        assert f(lib, M=300, K=512, N=256, ws=P, wsb=need - 1) == WORKSPACE and f(lib, ws=None, wsb=1 << 30) == WORKSPACE


def test_no_tokens_is_no_work(lib):  # noqa: F811
    assert quant(lib, M=0, x=None) == 0 and quant(lib, q=None, s=None, x=None) == 0 and norm(lib, M=0, x=None) == 0
    assert lin_fwd(lib, M=0, x=None) == 0 and gat_fwd(lib, M=0, x=None) == 0


def test_the_binding_refuses_what_is_not_a_dense_device_tensor(lib):  # noqa: F811
    import paper_2503_14376_amd as tfla
    x, q = torch.zeros(4, 8), torch.zeros(4, 8).to(torch.float8_e4m3fn)
    s = torch.ones(1, 4).to(torch.float8_e8m0fnu)
    for call in (lambda: tfla.q8_quant(x), lambda: tfla.q8_quant(x.to(torch.float16)), lambda: tfla.norm_q8_fwd(x),
                 lambda: tfla.linear_q8_fwd(q, s, q, s), lambda: tfla.linear_q8_fwd(x, s, q, s), lambda: tfla.linear_q8_bwd(x, q, s, x),
                 lambda: tfla.gated_q8_fwd(q, s, q, s, q, s), lambda: tfla.gated_q8_bwd(x, q, s, q, s, x, x, x)):
        with pytest.raises(ValueError):
            call()
