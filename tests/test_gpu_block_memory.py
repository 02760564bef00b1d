"""What the residual block's operators write: outputs and workspaces inside larger allocations of a known pattern, which has to stay."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def tfla():
    import paper_2503_14376_amd as pkg
    pkg.load_library()
    return pkg


def normal(gen, *shape, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N", [(20, 256), (3000, 256), (3000, 333)])
@pytest.mark.parametrize("pair", [False, True])
def test_bias_gradients_alone_store_only_sums(tfla, dtype, M, N, pair):
    """the workspace holds partial sums of rows (four at least) and nothing of the size of the tensors"""
    print("bias gradients", M, N, dtype, pair, flush=True)
    gen, K = generator(M + N), 72
    x, w, w2, z, u, dy = (normal(gen, *s, dtype=dtype) for s in ((M, K), (N, K), (N, K), (M, N), (M, N), (M, N)))
    query = tfla.gated_workspace_bytes if pair else tfla.linear_workspace_bytes
    code = tfla.BF16 if dtype == BF16 else tfla.F32
    ws = torch.full((query(1, M, K, N, tfla.ACT_SILU, code, True),), 0xA5, dtype=torch.uint8, device="cuda")
    kw = dict(act=tfla.ACT_SILU, want_db=True)
    if pair:
        full = tfla.gated_bwd(x, w, w2, z, u, dy, **kw)
        one = tfla.gated_bwd(x, w, w2, z, u, dy, want_dx=False, want_dw=False, workspace=ws, **kw)
        names = ("db_gate", "db_up")
    else:
        full = tfla.linear_bwd(x, w, dy, z, **kw)
        one = tfla.linear_bwd(x, w, dy, z, want_dx=False, want_dw=False, workspace=ws, **kw)
        names = ("db",)
    for n in names:
        assert torch.equal(one[n], full[n])
    written = int((ws != 0xA5).sum())
    sums = 0 if M <= 32 else (M + 3) // 4 * ((N + 7) // 8 * 8) * 4 * len(names)
    assert written <= sums, (written, sums)
    ws.fill_(0xA5)
    if pair:
        tfla.gated_bwd(x, w, w2, z, u, dy, want_dx=False, want_dw=False, workspace=ws, act=tfla.ACT_SILU)
    else:
        tfla.linear_bwd(x, w, dy, z, want_dx=False, want_dw=False, workspace=ws, act=tfla.ACT_SILU)
    assert bool((ws == 0xA5).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,N", [(20, 72, 88), (300, 333, 129)])
def test_gradients_without_the_tensors_that_they_do_not_read(tfla, dtype, M, K, N):
    print("without", M, K, N, dtype, flush=True)
    gen = generator(M + N)
    x, w, w2, z, u, dy = (normal(gen, *s, dtype=dtype) for s in ((M, K), (N, K), (N, K), (M, N), (M, N), (M, N)))
    kw = dict(act=tfla.ACT_SILU, want_db=True)
    full = tfla.linear_bwd(x, w, dy, z, **kw)
    for o in (tfla.linear_bwd(None, w, dy, z, want_dw=False, **kw), tfla.linear_bwd(x, None, dy, z, want_dx=False, **kw),
              tfla.linear_bwd(None, None, dy, z, want_dx=False, want_dw=False, **kw)):
        assert all(torch.equal(o[k], full[k]) for k in o if k != "workspace")
    full = tfla.gated_bwd(x, w, w2, z, u, dy, **kw)
    for o in (tfla.gated_bwd(None, w, w2, z, u, dy, want_dw=False, **kw), tfla.gated_bwd(x, None, None, z, u, dy, want_dx=False, **kw),
              tfla.gated_bwd(None, None, None, z, u, dy, want_dx=False, want_dw=False, **kw)):
        assert all(torch.equal(o[k], full[k]) for k in o if k != "workspace")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_dropped_tensor_is_not_written_from_another_stream(tfla, dtype):
    """work on the current stream still reads a tensor that was dropped; a call on another stream, whose output has that tensor's size,
    must not be given its memory"""
    print("dropped", dtype, flush=True)
    gen = generator(5)
    M, K, N = 2048, 256, 2056
    x, w = normal(gen, M, K, dtype=dtype), normal(gen, N, K, std=0.1, dtype=dtype)
    want = tfla.linear_fwd(x, w)["y"]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()                             # (no other block that the current stream's pool could give)
    old, kept, total = (torch.empty((M, N), dtype=d, device="cuda") for d in (dtype, dtype, F32))
    old.normal_(generator=gen)
    kept.copy_(old)
    total.zero_()
    torch.cuda.synchronize()
    for _ in range(50):
        total += old
    address = old.data_ptr()
    del old
    o = tfla.linear_fwd(x, w, stream=side)
    assert o["y"].data_ptr() != address
    again = torch.empty((M, N), dtype=dtype, device="cuda")
    assert again.data_ptr() == address                   # (the current stream may well use it again)
    torch.cuda.synchronize()
    assert torch.equal(o["y"], want)
    ref = torch.zeros((M, N), device="cuda")
    for _ in range(50):
        ref += kept
    assert torch.equal(total, ref)
