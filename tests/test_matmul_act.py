"""The product with bias, activation, gate and residual (nm_matmul_act) against its definition in 64 bits."""
import ctypes

import pytest
import torch

from ffn_util import (BF16, COL, F16, GELU, GELU_TANH, NONE, RELU, ROW, SILU, TORCH, assert_within, hidden64, randn, rounded, stored)


def make(M, N, K, dtype, gated, seed, bias=True, residual=True):
    wide = N * (2 if gated else 1)
    t = TORCH[dtype]
    return (randn(M, K, seed=seed, dtype=t), randn(K, wide, seed=seed + 1, scale=K ** -0.5, dtype=t),
            randn(wide, seed=seed + 2, dtype=t) if bias else None, randn(M, N, seed=seed + 3, dtype=t) if residual else None)


def expected(A, W, bias, residual, act, gated, dtype):
    z, t = hidden64(A.double(), W.double(), act, gated, None if bias is None else bias.double())
    if residual is not None:
        z = z + residual.double()
        t = t + 2.0 ** -23 * (z.abs() + residual.double().abs())
    return z, rounded(z, t, dtype)


def run(A, W, bias, residual, act, gated, dtype, layout, lda=None, ldc=None, ldr=None, shift=0, workspace=None):
    import paper_2609_16009_b200 as nm
    M, K = A.shape
    N = W.shape[1] // (2 if gated else 1)
    lda, ldc, ldr, t = lda or K, ldc or N, ldr or N, TORCH[dtype]
    dA = torch.full((M * lda + shift,), float("nan"), dtype=t, device="cuda")
    torch.as_strided(dA, (M, K), (lda, 1), shift).copy_(A)
    dW = stored(W, layout).cuda()
    db = None if bias is None else bias.cuda()
    dr = None
    if residual is not None:
        dr = torch.full((M, ldr), float("nan"), dtype=t, device="cuda")
        dr[:, :N] = residual.cuda()
    ws = nm.new_workspace(nm.nm_matmul_act_workspace_bytes(M, N, K, gated, dtype)) if workspace is None else workspace
    outs = []
    for _ in range(2):
        C = torch.full((M + 2, ldc), 77.0, dtype=t, device="cuda")
        nm.nm_matmul_act(dA[shift:], dW, C[1:], M, N, K, act, dtype, layout, ws, gated=gated, bias=db, residual=dr, lda=lda, ldc=ldc, ld_residual=ldr)
        outs.append(C)
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16)), "equal calls give equal bits"
    nm.nm_check_status()
    c = outs[0]
    assert (c[0] == 77).all() and (c[-1] == 77).all() and (c[:, N:] == 77).all(), "written outside C"
    return c[1:M + 1, :N]


SIZES = [(1, 1, 1), (1, 8, 8), (1, 16, 64), (2, 17, 63), (3, 127, 72), (5, 128, 64), (7, 129, 136), (16, 256, 512), (17, 257, 520), (31, 640, 1000), (33, 72, 2048), (64, 1000, 264), (65, 136, 4104),
         (100, 384, 128), (128, 520, 576), (129, 200, 72), (300, 264, 200), (1, 4096, 1536), (16, 24, 18432), (1, 576, 7168)]


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [ROW, COL])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(M, N, K, gated, dtype, layout):
    act = (NONE, RELU, SILU, GELU, GELU_TANH)[(M + N + K) % 5]
    A, W, bias, residual = make(M, N, K, dtype, gated, M + N + K)
    got = run(A, W, bias, residual, act, gated, dtype, layout)
    assert_within(got, *expected(A, W, bias, residual, act, gated, dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("act", [NONE, RELU, SILU, GELU, GELU_TANH])
@pytest.mark.parametrize("gated", [False, True])
def test_epilogues(act, gated, bias, residual):
    A, W, b, r = make(20, 200, 256, BF16, gated, act, bias, residual)
    got = run(A, 3 * W, b, r, act, gated, BF16, COL)
    assert_within(got, *expected(A, 3 * W, b, r, act, gated, BF16))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [ROW, COL])
@pytest.mark.parametrize("lda,ldc,ldr,shift", [(264, 208, 216, 0), (259, 203, 201, 0), (256, 200, 200, 1), (256, 200, 200, 4), (256, 201, 200, 8)])
def test_strides_and_alignment(lda, ldc, ldr, shift, layout):
    A, W, b, r = make(9, 200, 256, BF16, True, 3)
    got = run(A, W, b, r, SILU, True, BF16, layout, lda, ldc, ldr, shift)
    assert_within(got, *expected(A, W, b, r, SILU, True, BF16))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [ROW, COL])
def test_unaligned_weights(layout):
    import paper_2609_16009_b200 as nm
    A, W, _, _ = make(4, 64, 128, BF16, False, 4, False, False)
    flat = torch.zeros(64 * 128 + 1, dtype=torch.bfloat16, device="cuda")
    flat[1:] = stored(W, layout).reshape(-1).cuda()
    C = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    nm.nm_matmul_act(A.cuda(), flat[1:], C, 4, 64, 128, RELU, BF16, layout, nm.new_workspace(nm.nm_matmul_act_workspace_bytes(4, 64, 128)))
    assert_within(C, *expected(A, W, None, None, RELU, False, BF16))


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 40, 200])
def test_onto_the_residual_in_place(M):
    import paper_2609_16009_b200 as nm
    A, W, _, r = make(M, 520, 1024, BF16, False, 5, False)
    C = r.cuda()
    nm.nm_matmul_act(A.cuda(), stored(W, COL).cuda(), C, M, 520, 1024, NONE, BF16, COL, nm.new_workspace(nm.nm_matmul_act_workspace_bytes(M, 520, 1024)), residual=C)
    assert_within(C, *expected(A, W, None, r, NONE, False, BF16))


@pytest.mark.gpu
def test_small_integers_are_exact():
    g = torch.Generator().manual_seed(7)
    A, W = (torch.randint(-2, 3, s, generator=g).to(torch.bfloat16) for s in ((13, 7168), (7168, 96)))
    got = run(A, W, None, None, NONE, False, BF16, ROW)
    assert torch.equal(got.cpu().double(), (A.double() @ W.double()).to(torch.bfloat16).double())


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [ROW, COL])
def test_a_bad_row_and_a_bad_column_stay_where_they_are(layout):
    """An infinity or a NaN in a row of A, or in a column of B, reaches nothing else."""
    A, W, b, r = make(20, 264, 200, BF16, True, 8)
    clean = run(A, W, b, r, SILU, True, BF16, layout)
    bad_A, bad_W = A.clone(), W.clone()
    bad_A[3, 5], bad_A[17, 199] = float("inf"), float("nan")
    bad_W[7, 11], bad_W[0, 264 + 250] = float("nan"), float("inf")
    got = run(bad_A, bad_W, b, r, SILU, True, BF16, layout)
    rows = [m for m in range(20) if m not in (3, 17)]
    cols = [n for n in range(264) if n not in (11, 250)]
    assert torch.equal(got[rows][:, cols], clean[rows][:, cols])
    assert got[17].isnan().all() and got[:, 11].isnan().all()


@pytest.mark.gpu
def test_fp16_result_beyond_its_range_is_infinite():
    A, W = torch.full((2, 64), 30.0, dtype=torch.float16), torch.full((64, 16), 60.0, dtype=torch.float16)
    assert torch.isposinf(run(A, W, None, None, NONE, False, F16, COL)).all()


@pytest.mark.gpu
def test_captured_replayed_and_on_another_stream():
    import paper_2609_16009_b200 as nm
    M, N, K = 5, 520, 2048
    A, W, b, r = make(M, N, K, BF16, True, 9)
    dA, dW, db, dr = A.cuda(), stored(W, COL).cuda(), b.cuda(), r.cuda()
    C = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    ws = nm.new_workspace(nm.nm_matmul_act_workspace_bytes(M, N, K, True))
    torch.cuda.synchronize()

    def call(stream=None):
        nm.nm_matmul_act(dA, dW, C, M, N, K, SILU, BF16, COL, ws, gated=True, bias=db, residual=dr, stream=stream)
    call(s)
    torch.cuda.synchronize()
    assert_within(C, *expected(A, W, b, r, SILU, True, BF16))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    A2 = randn(M, K, seed=99, dtype=torch.bfloat16)
    dA.copy_(A2)
    for _ in range(3):
        C.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert_within(C, *expected(A2, W, b, r, SILU, True, BF16))


@pytest.mark.gpu
@pytest.mark.parametrize("programmatic", [False, True])
def test_two_products_behind_each_other(programmatic):
    """The second reads what the first wrote, through one workspace, also where its weights are read ahead of the wait."""
    import paper_2609_16009_b200 as nm
    M, d, inter = 3, 512, 1000
    x, W1, _, _ = make(M, inter, d, BF16, True, 10, False, False)
    W2 = randn(inter, d, seed=20, scale=inter ** -0.5, dtype=torch.bfloat16)
    dx, d1, d2 = x.cuda(), stored(W1, COL).cuda(), stored(W2, ROW).cuda()
    h, y = torch.zeros(M, inter, dtype=torch.bfloat16, device="cuda"), torch.zeros(M, d, dtype=torch.bfloat16, device="cuda")
    ws = nm.new_workspace(max(nm.nm_matmul_act_workspace_bytes(M, inter, d, True), nm.nm_matmul_act_workspace_bytes(M, d, inter)))
    torch.cuda.synchronize()
    nm.nm_set_programmatic_launch(programmatic)
    try:
        for _ in range(20):
            h.zero_()
            nm.nm_matmul_act(dx, d1, h, M, inter, d, SILU, BF16, COL, ws, gated=True)
            nm.nm_matmul_act(h, d2, y, M, d, inter, NONE, BF16, ROW, ws, residual=dx)
    finally:
        nm.nm_set_programmatic_launch(False)
    assert_within(h, *expected(x, W1, None, None, SILU, True, BF16))
    assert_within(y, *expected(h.cpu(), W2, None, x, NONE, False, BF16))


@pytest.fixture(scope="module")
def lib():
    from paper_2609_16009_b200 import build
    return ctypes.CDLL(build.build())


def test_refusals_need_no_device(lib):
    vp, i, l, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_long, ctypes.c_size_t
    lib.nm_matmul_act.argtypes = [vp, l, vp, vp, vp, l, vp, l] + [i] * 7 + [vp, sz, vp]
    lib.nm_matmul_act_workspace_bytes.restype = sz
    need = lib.nm_matmul_act_workspace_bytes(4, 64, 128, 0, 1)
    assert need >= 65536

    def status(A=256, lda=128, B=512, bias=None, residual=None, ldr=64, C=1024, ldc=64, M=4, N=64, K=128, act=0, gated=0, dtype=1, layout=1, ws=4096, bytes_=1 << 40):
        return lib.nm_matmul_act(A, lda, B, bias, residual, ldr, C, ldc, M, N, K, act, gated, dtype, layout, ws, bytes_, None)
    assert status(A=None) == status(B=None) == status(C=None) == -1
    assert status(M=0) == status(N=0) == status(K=0) == status(M=65537) == status(K=-1) == -1
    assert status(lda=127) == status(ldc=63) == status(residual=256, ldr=63) == -1
    assert status(dtype=0) == status(dtype=2) == status(layout=2) == status(act=5) == status(act=-1) == -2
    assert status(A=257) == status(B=513) == status(C=1025) == status(bias=257) == status(residual=257) == status(ws=4097) == -3
    assert status(ws=None) == status(bytes_=need - 1) == -4
    assert lib.nm_matmul_act_workspace_bytes(0, 1, 1, 0, 1) == lib.nm_matmul_act_workspace_bytes(1, 1, 1, 0, 0) == 0
