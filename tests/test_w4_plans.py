"""Every split of the 4-bit product, forced one after another: warps across the columns and along k, CTAs along k, tokens in pieces."""
import ctypes

import pytest
import torch

from test_w4 import BF16, BF16_F32OUT, F16, assert_close, case, pack, pack_scales


@pytest.fixture
def plan():
    import paper_2609_16009_b200 as nm
    yield nm.nm_debug_set_w4_plan
    nm.nm_debug_set_w4_plan()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,group", [(BF16, 32), (BF16_F32OUT, 128), (F16, 64), (F16, 32)])
@pytest.mark.parametrize("M,N,K", [(1, 200, 1400), (3, 300, 1399), (8, 97, 1400), (9, 200, 1400), (16, 290, 1399)])
def test_every_split(plan, M, N, K, group, dtype):
    """The same product, to the tolerance of its sums, whichever way it is split; calls with the same split have the same bits."""
    import paper_2609_16009_b200 as nm
    A, codes, sc, ref, size = case(M, N, K, group, dtype, M + N)
    dA, packed, scales = A.cuda(), torch.from_numpy(pack(codes)).cuda(), pack_scales(sc).cuda()
    out_type = torch.float32 if dtype == BF16_F32OUT else dA.dtype
    seen = {}
    for warps in (1, 2, 4, 8, 16):
        for ctas in range(1, 9):
            for piece in (0, 1, 2, 3, 5):
                plan(warps, ctas, piece)
                C = torch.full((M + 2, N), 77.0, dtype=out_type, device="cuda")
                nm.nm_matmul_w4(dA, packed, scales, C[1:], M, N, K, group, dtype)
                seen[warps, ctas, piece] = C
    torch.cuda.synchronize()
    for key, C in seen.items():
        c = C.double().cpu().numpy()
        assert (c[0] == 77).all() and (c[-1] == 77).all(), (key, "written outside C")
        try:
            assert_close(c[1:M + 1], ref, size, dtype)
        except AssertionError as e:
            raise AssertionError(f"warps across, CTAs along k, blocks of a piece: {key}: {e}")
    if dtype == BF16_F32OUT:
        assert len({C.cpu().numpy().tobytes() for C in seen.values()}) > 10, "the splits are really different ones"


@pytest.mark.gpu
def test_a_split_that_cannot_be_is_left_to_the_planner(plan):
    import paper_2609_16009_b200 as nm
    M, N, K = 4, 40, 64                                            # one block of k: no two CTAs along it
    A, codes, sc, ref, size = case(M, N, K, 64, BF16, 1)
    packed, scales = torch.from_numpy(pack(codes)).cuda(), pack_scales(sc).cuda()
    for forced in ((16, 8, 0), (1, 8, 3), (0, 2, 0), (16, 0, 1)):
        plan(*forced)
        C = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
        nm.nm_matmul_w4(A.cuda(), packed, scales, C, M, N, K, 64, BF16)
        assert_close(C.double().cpu().numpy(), ref, size, BF16)


def test_refusals():
    import paper_2609_16009_b200 as nm
    for bad in ((3, 0, 0), (32, 0, 0), (-1, 0, 0), (0, 9, 0), (0, -1, 0), (0, 0, -1), (0, 0, 1 << 16)):
        assert nm._lib.nm_debug_set_w4_plan(*(ctypes.c_int(x) for x in bad)) == -1, bad
