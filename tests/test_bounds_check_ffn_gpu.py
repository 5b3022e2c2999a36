"""The feed-forward operators in the debug build (libnm_check.so): every hand-indexed access against the extent of its operand, over ragged shapes.
Clean, and the bits of the normal build."""
import ctypes as C

import pytest
import torch

import test_moe_ffn as moe_tests
from ffn_util import BF16, COL, F16, ROW, SILU, TORCH, stored
from test_bounds_check_storage_gpu import same_in_both
from test_matmul_act import make as make_act

pytestmark = pytest.mark.gpu
NAMES = ("nm_moe_route", "nm_matmul_act", "nm_matmul_act_workspace_bytes", "nm_moe_ffn", "nm_moe_ffn_workspace_bytes", "nm_check_status", "nm_workspace_init", "nm_debug_set_ffn_cut")


@pytest.fixture(scope="module")
def check():
    import paper_2609_16009_b200 as nm
    from paper_2609_16009_b200 import build
    lib = C.CDLL(build.build(check=True))
    assert lib.nm_debug_bounds_checked() == 1
    for name in NAMES:
        getattr(lib, name).argtypes = getattr(nm._lib, name).argtypes
        getattr(lib, name).restype = getattr(nm._lib, name).restype
    return lib


@pytest.mark.parametrize("T,E,k,groups,keep,best,dtype", [(1, 1, 1, 1, 1, 1, 0), (5, 33, 7, 1, 1, 1, 1), (9, 160, 6, 8, 3, 2, 0), (3, 1000, 32, 20, 7, 1, 3), (70, 96, 4, 32, 5, 2, 0)])
def test_route(check, T, E, k, groups, keep, best, dtype):
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, E, generator=g).to({0: torch.float32, 1: torch.bfloat16, 3: torch.float16}[dtype])
    x[::4, ::3] = float("-inf")
    x, bias = x.cuda(), (0.1 * torch.randn(E, generator=g)).cuda()

    def call(nm):
        outs = []
        for score in (0, 1):
            for b in (None, bias):
                e, w = torch.zeros(T, k, dtype=torch.int32, device="cuda"), torch.zeros(T, k, device="cuda")
                nm.nm_moe_route(x, b, e, w, T, E, k, dtype, score, groups=groups, keep_groups=keep, group_best=best)
                outs += [e, w]
        return outs
    same_in_both(call, check)


@pytest.mark.parametrize("layout", [ROW, COL])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("M,N,K,gated,parts", [(1, 1, 1, False, 0), (3, 17, 63, True, 0), (5, 136, 264, True, 0), (16, 2600, 520, False, 3), (33, 72, 2048, False, 7), (100, 264, 1032, True, 2), (129, 520, 72, False, 0)])
def test_product(check, M, N, K, gated, parts, dtype, layout):
    A, W, b, r = (v.cuda() for v in make_act(M, N, K, dtype, gated, M + N))
    W = stored(W.cpu(), layout).cuda()

    def call(nm):
        ws = nm.new_workspace(nm.nm_matmul_act_workspace_bytes(M, N, K, gated, dtype))
        out = torch.full((M, N + 2), 7.0, dtype=TORCH[dtype], device="cuda")
        nm.nm_debug_set_ffn_cut(parts)
        try:
            nm.nm_matmul_act(A, W, out, M, N, K, SILU, dtype, layout, ws, gated=gated, bias=b, residual=r, ldc=N + 2)
        finally:
            nm.nm_debug_set_ffn_cut(0)
        return [out]
    same_in_both(call, check)


@pytest.mark.parametrize("layout", [ROW, COL])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T,d,inter,E,k,parts", [(1, 8, 8, 1, 1, 0), (3, 63, 65, 4, 2, 0), (9, 264, 136, 5, 3, 2), (40, 520, 264, 6, 2, 5), (150, 136, 200, 3, 2, 2), (260, 128, 72, 9, 3, 0)])
def test_experts(check, T, d, inter, E, k, parts, dtype, layout):
    c = moe_tests.make(T, d, inter, E, k, dtype, T + d)
    c["experts"][T // 2] = -1
    dev = moe_tests.place(c, layout)

    def call(nm):
        out = torch.full((T, d), 7.0, dtype=TORCH[dtype], device="cuda")
        nm.nm_debug_set_ffn_cut(parts)
        try:
            moe_tests.call(nm, c, SILU, True, dtype, layout, out, moe_tests.workspace(nm, c, dtype), dev=dev)
        finally:
            nm.nm_debug_set_ffn_cut(0)
        return [out]
    same_in_both(call, check)
