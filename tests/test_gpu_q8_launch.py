"""Calls in 8 bits of so many tiles that one launch cannot start them all (2^32 threads): 2^22 tiles of 128 x 128 values, 2^24
of 64 x 64 results.  Tensors are zero but in
some rows, at both ends and round the places where a launch ends; outputs hold other bytes before the call."""
import pytest
import torch

from tests.q8_util import E4M3, E8M0
from tests.test_gpu_block import BF16, F32
from tests.test_gpu_block_far import freed, tfla, whole  # noqa: F401

pytestmark = pytest.mark.gpu
F64 = torch.float64


def room(gigabytes):
    free = torch.cuda.mem_get_info()[0]
    if free < gigabytes * 10 ** 9:
        pytest.skip("%d GB of the device are wanted, %d are free" % (gigabytes, free // 10 ** 9))


def some_rows(rows):
    """both ends of the matrix and of each 32nd of it (an XCD's share of a launch is a 16th)"""
    at = {0, 1, 126, 127, 128, 129, rows - 1, rows - 2}
    for i in range(1, 32):
        at |= {rows * i // 32 + d for d in (-129, -1, 0, 1, 128)}
    return sorted(at)


def sparse(seed, rows, cols):
    """zero but in some rows, which hold small whole numbers; those rows"""
    t = torch.zeros((rows, cols), dtype=BF16, device="cuda")
    at = some_rows(rows)
    few = whole(seed, len(at), cols, BF16)
    for i, r in enumerate(at):
        t[r].copy_(few[i])
    return t, at, few


def nothing_but(t, at, empty=0):
    """all other rows of bytes are `empty`; those rows are overwritten"""
    t = t.view(torch.uint8)
    for r in at:
        t[r].fill_(empty)
    for lo in range(0, t.shape[0], 1 << 18):
        assert bool((t[lo:lo + (1 << 18)] == empty).all()), lo


def test_quantiser(tfla):  # noqa: F811
    M, K = 1 << 24, 3969                 # 2^17 x 32 tiles
    room(205)
    print("quantiser", M, K, flush=True)
    x, at, few = sparse(1, M, K)
    q = torch.full((M, K), 0x55, dtype=torch.uint8, device="cuda").view(E4M3)
    scale = torch.full((32, M), 0x55, dtype=torch.uint8, device="cuda").view(E8M0)
    tfla.q8_quant(x, out={"q": q, "scale": scale})
    want = tfla.q8_quant(few)
    rows = torch.tensor(at, device="cuda")
    assert torch.equal(scale.view(torch.uint8)[:, rows], want["scale"].view(torch.uint8))
    assert torch.equal(torch.stack([q[r].view(torch.uint8) for r in at]), want["q"].view(torch.uint8))
    s = scale.view(torch.uint8)
    s[:, rows] = 0
    assert not bool(s.any())
    nothing_but(q, at)


def test_bias_gradient(tfla):  # noqa: F811
    M, N = 1 << 21, 1 << 15              # 2^14 x 2^8 tiles
    room(145)
    print("bias gradient", M, N, flush=True)
    dy, at, few = sparse(2, M, N)
    db = torch.full((N,), float("nan"), device="cuda")
    tfla.linear_q8_bwd(None, None, None, dy, want_dx=False, want_dw=False, want_db=True, out={"db": db})
    assert torch.equal(db, few.to(F64).sum(0).to(F32))


def test_one_token_back_through_the_largest_weights(tfla):  # noqa: F811
    """dx and dw in one launch would be 2^24 tiles"""
    K = N = 1 << 18
    room(210)
    print("largest weights", K, N, flush=True)
    at = some_rows(K)
    wt, few = torch.zeros((K, N), dtype=torch.uint8, device="cuda"), whole(3, len(at), N, BF16, 1)
    codes = few.to(E4M3).view(torch.uint8)                  # (0 and +-1 are codes)
    for i, k in enumerate(at):
        wt[k].copy_(codes[i])
    scale = torch.full((N // 128, K // 128), 127, dtype=torch.uint8, device="cuda").view(E8M0)
    x, dy = torch.zeros((1, K), dtype=BF16, device="cuda"), torch.zeros((1, N), dtype=BF16, device="cuda")
    rows = torch.tensor(at, device="cuda")
    x[:, rows], dy[:, rows] = whole(4, 1, len(at), BF16), whole(5, 1, len(at), BF16)
    dw = torch.full((N, K), float("nan"), dtype=BF16, device="cuda")
    o = tfla.linear_q8_bwd(x, wt.view(E4M3), scale, dy, want_db=True, out={"dw": dw})
    assert torch.equal(o["dx"][:, rows], (dy.to(F64) @ few.to(F64).t()).to(BF16))
    o["dx"][:, rows] = 0
    assert not bool(o["dx"].any()) and torch.equal(o["db"], dy[0].float())
    for n in at:
        assert torch.equal(dw[n], dy[0, n] * x[0]), n
        dw[n] = 0
    for lo in range(0, N, 1 << 14):
        assert not bool(dw[lo:lo + (1 << 14)].any()), lo
