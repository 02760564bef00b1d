"""Host-side checks of the residual block's entry points: invalid arguments come back as the documented codes before anything is
launched, the workspace queries agree with the calls, and the binding refuses tensors that are not what a call needs.  No compute
call is made here: every call below fails its checks."""
import itertools

import pytest
import torch

SHAPE, NULL, ENUM, WORKSPACE = -2, -1, -4, -5
P = 1 << 20      # an address that is never followed: the call fails before


@pytest.fixture(scope="module")
def lib():
    import os
    import paper_2503_14376_amd as pkg
    if not os.path.exists(pkg.lib_path()):
        from paper_2503_14376_amd import build
        build.build(verbose=False)
    return pkg.load_library()


def norm_fwd(lib, M=4, D=64, dtype=1, kind=0, eps=1e-6, x=P, y=P):
    return lib.tfla_norm_fwd(x, None, None, M, D, dtype, kind, eps, y, None, None, None)


def norm_bwd(lib, M=40, D=64, dtype=1, kind=0, x=P, dy=P, rstd=P, mean=None, dx=P, dgamma=P, ws=None, wsb=0):
    return lib.tfla_norm_bwd(x, dy, rstd, mean, None, None, M, D, dtype, kind, dx, dgamma, None, ws, wsb, None)


@pytest.mark.parametrize("kw,rc", [(dict(M=-1), SHAPE), (dict(M=(1 << 24) + 1), SHAPE), (dict(D=0), SHAPE), (dict(D=16385), SHAPE),
                                   (dict(dtype=2), ENUM), (dict(kind=2), ENUM), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
                                   (dict(x=None), NULL), (dict(y=None), NULL)])
def test_norm_fwd_refusals(lib, kw, rc):
    assert norm_fwd(lib, **kw) == rc


@pytest.mark.parametrize("kw,rc", [(dict(M=-1), SHAPE), (dict(D=0), SHAPE), (dict(dtype=-1), ENUM), (dict(kind=5), ENUM),
                                   (dict(x=None), NULL), (dict(dy=None), NULL), (dict(rstd=None), NULL), (dict(dx=None), NULL),
                                   (dict(kind=1), NULL), (dict(), WORKSPACE), (dict(ws=P, wsb=16), WORKSPACE), (dict(ws=P + 8, wsb=1 << 30), WORKSPACE)])
def test_norm_bwd_refusals(lib, kw, rc):
    assert norm_bwd(lib, **kw) == rc


def lin_fwd(lib, M=4, K=64, N=64, act=0, dtype=1, x=P, w=P, y=P, ws=None, wsb=0):
    return lib.tfla_linear_fwd(x, w, None, None, M, K, N, act, dtype, y, None, ws, wsb, None)


def lin_bwd(lib, M=4, K=64, N=64, act=0, dtype=1, x=P, w=P, dy=P, z=None, dx=P, dw=P, ws=None, wsb=0):
    return lib.tfla_linear_bwd(x, w, dy, z, M, K, N, act, dtype, dx, dw, P, ws, wsb, None)


def gat_fwd(lib, M=4, K=64, N=64, act=1, dtype=1, x=P, wg=P, wu=P, h=P, ws=None, wsb=0):
    return lib.tfla_gated_fwd(x, wg, wu, None, None, M, K, N, act, dtype, h, None, None, ws, wsb, None)


def gat_bwd(lib, M=4, K=64, N=64, act=1, dtype=1, x=P, wg=P, wu=P, a=P, u=P, dh=P, dx=P, dwg=P, dwu=P, ws=None, wsb=0):
    return lib.tfla_gated_bwd(x, wg, wu, a, u, dh, M, K, N, act, dtype, dx, dwg, dwu, P, P, ws, wsb, None)


DIMS = [(dict(M=-1), SHAPE), (dict(M=(1 << 24) + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=(1 << 20) + 1), SHAPE), (dict(N=-3), SHAPE),
        (dict(N=1 << 20, K=1 << 17), SHAPE), (dict(M=1 << 24, K=1 << 13), SHAPE), (dict(dtype=2), ENUM), (dict(act=4), ENUM), (dict(act=-1), ENUM)]


@pytest.mark.parametrize("f", [lin_fwd, lin_bwd, gat_fwd, gat_bwd])
@pytest.mark.parametrize("kw,rc", DIMS)
def test_dimensions_are_refused(lib, f, kw, rc):
    assert f(lib, **kw) == rc


@pytest.mark.parametrize("f,names", [(lin_fwd, ("x", "w", "y")), (lin_bwd, ("x", "w", "dy")), (gat_fwd, ("x", "wg", "wu", "h")),
                                     (gat_bwd, ("x", "wg", "wu", "a", "u", "dh", "dwu"))])
def test_missing_tensors_are_refused(lib, f, names):
    for n in names:
        assert f(lib, **{n: None}) == NULL, n


def test_activations_need_what_the_forward_call_stored(lib):
    assert lin_bwd(lib, act=1) == NULL


@pytest.mark.parametrize("f,query", [(lin_fwd, "tfla_linear_workspace_bytes"), (gat_fwd, "tfla_gated_workspace_bytes")])
def test_a_workspace_is_asked_for_and_checked(lib, f, query):
    q = getattr(lib, query)
    need = q(0, 300, 333, 200, 1, 1, 0)
    assert need >= 2 * 300 * 336                       # rows of 333 values are copied into aligned ones
    kw = dict(M=300, K=333, N=200, act=1)
    assert f(lib, **kw) == WORKSPACE
    assert f(lib, ws=P, wsb=need - 1, **kw) == WORKSPACE
    assert f(lib, ws=P + 128, wsb=need, **kw) == WORKSPACE
    # tensors at odd addresses: more where the rows themselves are fine
    assert q(0, 300, 512, 256, 1, 1, 1) >= q(0, 300, 512, 256, 1, 1, 0) + 2 * 512 * (300 + 256)
    assert f(lib, M=300, K=512, N=256, x=P + 2, ws=P, wsb=q(0, 300, 512, 256, 1, 1, 0)) == WORKSPACE


def test_few_tokens_through_many_weights(lib):
    """up to 32 tokens are taken by either kernel: a query with an unaligned tensor covers the call whichever tensor that is"""
    asked = 0
    for q, f, names in ((lib.tfla_linear_workspace_bytes, lin_fwd, ("x", "w")), (lib.tfla_gated_workspace_bytes, gat_fwd, ("x", "wg"))):
        for M, K, N in itertools.product((1, 4, 5, 8, 16, 17, 24, 32, 33), (512, 4096, 10944), (512, 1024, 4096)):
            need, off = q(0, M, K, N, 1, 1, 0), q(0, M, K, N, 1, 1, 1)
            assert off >= need and (need == 0 or M > 4)
            if need > 0:
                asked += M <= 32
                assert f(lib, M=M, K=K, N=N, act=1) == WORKSPACE
                assert f(lib, M=M, K=K, N=N, act=1, ws=P, wsb=need - 1) == WORKSPACE
            if M > 32:                                     # (below, an unaligned operand needs none and the call would run)
                for name in names:
                    assert f(lib, M=M, K=K, N=N, act=1, ws=P, wsb=0, **{name: P + 2}) == WORKSPACE
    assert asked > 0


def test_backward_workspaces(lib):
    for q, pair in ((lib.tfla_linear_workspace_bytes, 1), (lib.tfla_gated_workspace_bytes, 2)):
        assert q(1, 300, 512, 256, 1, 1, 0) >= pair * 2 * 300 * 256
        assert q(1, 300, 512, 256, 1, 1, 1) > q(1, 300, 512, 256, 1, 1, 0)
        assert q(1, 0, 512, 256, 1, 1, 0) >= 0
        for bad in ((2, 3, 64, 64, 0, 1, 0), (0, -1, 64, 64, 0, 1, 0), (1, 3, 0, 64, 0, 1, 0), (1, 3, 64, 64, 9, 1, 0), (1, 3, 64, 64, 0, 7, 0)):
            assert q(*bad) == 0
    assert lin_bwd(lib, ws=P, wsb=0) == WORKSPACE and gat_bwd(lib, ws=None, wsb=1 << 30) == WORKSPACE
    assert lib.tfla_norm_workspace_bytes(0, 100, 64, 1, 0) == 0 and lib.tfla_norm_workspace_bytes(1, 100, 64, 1, 0) >= 2 * 64 * 4
    assert lib.tfla_norm_workspace_bytes(1, 100, 0, 1, 0) == 0 and lib.tfla_norm_workspace_bytes(3, 100, 64, 1, 0) == 0


def test_no_tokens_is_no_work(lib):
    assert norm_fwd(lib, M=0, x=None, y=None) == 0
    assert lin_fwd(lib, M=0, x=None) == 0 and gat_fwd(lib, M=0, x=None) == 0


def test_the_binding_refuses_what_is_not_a_dense_device_tensor(lib):
    import paper_2503_14376_amd as tfla
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        tfla.norm_fwd(x)
    with pytest.raises(ValueError):
        tfla.linear_fwd(x.to(torch.float16), x)
    with pytest.raises(ValueError):
        tfla.gated_fwd(x.view(2, 2, 8), x, x)
