"""The token maps of the feed-forward products in the debug build, which looks at the map that it asks for before anything else: for every box height that a call's
rows can have there is one, and it is the one that is brought in."""
import pytest
import torch

import test_moe_ffn as moe_tests
from ffn_util import BF16, COL, SILU, stored
from test_bounds_check_ffn_gpu import check  # noqa: F401  (the fixture)
from test_bounds_check_storage_gpu import same_in_both
from test_matmul_act import make as make_act

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [1, 8, 9, 16, 17, 24, 25, 32, 33, 48, 49, 64, 65, 96, 97, 100, 128, 129, 161, 200, 256])
def test_rows_of_a_product(check, M):  # noqa: F811
    A, W, b, r = (v.cuda() for v in make_act(M, 264, 136, BF16, False, M))
    W = stored(W.cpu(), COL).cuda()

    def call(nm):
        out = torch.full((M, 264), 7.0, dtype=torch.bfloat16, device="cuda")
        nm.nm_matmul_act(A, W, out, M, 264, 136, SILU, BF16, COL, nm.new_workspace(nm.nm_matmul_act_workspace_bytes(M, 264, 136)), bias=b, residual=r)
        return [out]
    same_in_both(call, check)


@pytest.mark.parametrize("T", [1, 7, 30, 100, 300])
def test_rows_of_experts(check, T):  # noqa: F811
    c = moe_tests.make(T, 136, 72, 5, 2, BF16, T)
    dev = moe_tests.place(c, COL)

    def call(nm):
        out = torch.full((T, 136), 7.0, dtype=torch.bfloat16, device="cuda")
        moe_tests.call(nm, c, SILU, True, BF16, COL, out, moe_tests.workspace(nm, c, BF16), dev=dev)
        return [out]
    same_in_both(call, check)
