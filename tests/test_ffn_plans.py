"""Feed-forward products: every cut of the items, sizes at the borders of the tiles, operands beyond 32-bit offsets, and calls beside each other."""
import pytest
import torch

import test_matmul_act as act_tests
import test_moe_ffn as moe_tests
from ffn_util import BF16, COL, F16, NONE, ROW, SILU, assert_within, hidden64, randn, rounded, stored

pytestmark = pytest.mark.gpu


@pytest.fixture
def cut():
    import paper_2609_16009_b200 as nm
    yield nm.nm_debug_set_ffn_cut
    nm.nm_debug_set_ffn_cut(0)


@pytest.mark.parametrize("parts", [1, 2, 3, 5, 7, 16, 33, 200])
@pytest.mark.parametrize("M,N,K,gated,dtype,layout", [(1, 300, 2048, False, BF16, COL), (4, 136, 1000, True, F16, ROW), (5, 2600, 520, False, BF16, ROW), (16, 136, 4096, True, BF16, COL),
                                                      (17, 2304, 1032, False, F16, COL), (64, 264, 2056, True, BF16, ROW), (100, 128, 1600, False, F16, COL), (128, 2304, 320, False, BF16, COL),
                                                      (200, 520, 704, True, BF16, COL)])
def test_products_in_parts(cut, parts, M, N, K, gated, dtype, layout):
    A, W, b, r = act_tests.make(M, N, K, dtype, gated, M + N + K)
    cut(parts)
    got = act_tests.run(A, W, b, r, SILU, gated, dtype, layout)
    assert_within(got, *act_tests.expected(A, W, b, r, SILU, gated, dtype))


@pytest.mark.parametrize("parts", [1, 2, 3, 8, 32])
@pytest.mark.parametrize("T,d,inter,E,k,dtype,layout", [(1, 1024, 520, 8, 3, BF16, COL), (7, 2304, 264, 5, 2, F16, ROW), (33, 512, 1024, 6, 3, BF16, ROW), (90, 264, 512, 4, 2, F16, COL),
                                                        (300, 256, 200, 5, 3, BF16, COL)])
def test_experts_in_parts(cut, parts, T, d, inter, E, k, dtype, layout):
    c = moe_tests.make(T, d, inter, E, k, dtype, T + d)
    cut(parts)
    assert_within(moe_tests.run(c, SILU, True, dtype, layout), *moe_tests.expected(c, SILU, True, dtype))


@pytest.mark.parametrize("rows", [1, 3, 4, 5, 7, 8, 9, 12, 13, 15, 16, 17, 24, 25, 31, 32, 33, 47, 48, 49, 63, 64, 65, 95, 96, 97, 127, 128, 129, 255, 257])
def test_every_number_of_rows_of_an_expert(rows):
    """Row counts around the accumulator's steps and the tiles' borders, through both products and with a neighbour that has other rows."""
    T = rows + 3
    c = moe_tests.make(T, 264, 136, 3, 1, BF16, rows)
    c["experts"][:] = 1
    c["experts"][::max(1, T // 3)][:3] = 2
    assert_within(moe_tests.run(c, SILU, True, BF16, COL), *moe_tests.expected(c, SILU, True, BF16))
    A, W, b, r = act_tests.make(rows, 200, 136, BF16, False, rows)
    assert_within(act_tests.run(A, W, b, r, SILU, False, BF16, ROW), *act_tests.expected(A, W, b, r, SILU, False, BF16))


@pytest.mark.parametrize("K", [63, 1001, 2050])
def test_one_row_of_any_length(K):
    """The pitch of a single row is no pitch: row-major weights take the tensor-core kernel with any K."""
    A, W, b, r = act_tests.make(1, 264, K, BF16, True, K)
    assert_within(act_tests.run(A, W, b, r, SILU, True, BF16, ROW), *act_tests.expected(A, W, b, r, SILU, True, BF16))
    c = moe_tests.make(1, K, 72, 5, 2, BF16, K)
    assert_within(moe_tests.run(c, SILU, True, BF16, ROW), *moe_tests.expected(c, SILU, True, BF16))


def test_many_pairs():
    """More pairs than a plan keeps in shared memory, and an expert that takes most of them."""
    T, d, inter, E, k = 5000, 64, 64, 20, 2
    c = moe_tests.make(T, d, inter, E, k, BF16, 3)
    c["experts"][: 3 * T // 4, 0] = 5
    assert_within(moe_tests.run(c, SILU, True, BF16, COL), *moe_tests.expected(c, SILU, True, BF16))


@pytest.mark.parametrize("T,E,k", [(1, 40, 6), (20, 40, 6), (21, 40, 6), (22, 40, 6), (128, 64, 1), (129, 64, 1), (64, 64, 2), (2, 200, 64), (43, 1000, 3)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_plans_around_the_pairs_a_block_plans_itself(T, E, k, dtype):
    c = moe_tests.make(T, 136, 72, E, k, dtype, T + E)
    c["experts"][T // 2] = -1
    c["experts"][-1, 0] = E
    for skewed in (False, True):
        if skewed:
            c["experts"][: 3 * T // 4 + 1, 0] = E - 1              # several tiles of one expert
        assert_within(moe_tests.run(c, SILU, True, dtype, COL), *moe_tests.expected(c, SILU, True, dtype))


def test_one_workspace_for_experts_of_all_sizes(cut):
    """Calls that plan themselves and calls that do not, cut and whole, through one workspace: the counters are left as they were found."""
    import paper_2609_16009_b200 as nm
    ws = nm.new_workspace(128 << 20)
    for i, (T, d, inter, E, k, parts) in enumerate([(1, 1024, 264, 8, 2, 3), (300, 256, 136, 5, 2, 2), (2, 4096, 128, 50, 6, 0), (20, 264, 520, 40, 6, 5), (40, 264, 136, 3, 3, 0), (1, 72, 64, 4, 1, 0)]):
        cut(parts)
        c = moe_tests.make(T, d, inter, E, k, BF16, 80 + i)
        out = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
        for _ in range(3):
            moe_tests.call(nm, c, SILU, True, BF16, COL, out, ws)
        assert_within(out, *moe_tests.expected(c, SILU, True, BF16))
        assert int(ws[:65536].count_nonzero()) == 0


def test_many_experts_few_tokens():
    c = moe_tests.make(3, 72, 64, 1024, 32, BF16, 4)
    assert_within(moe_tests.run(c, SILU, True, BF16, ROW), *moe_tests.expected(c, SILU, True, BF16))


def test_weights_of_experts_beyond_32_bit_offsets():
    import paper_2609_16009_b200 as nm
    T, d, inter, E, k = 3, 7168, 2560, 70, 1
    up, down = torch.empty(E, 2 * inter, d, dtype=torch.bfloat16, device="cuda"), torch.empty(E, d, inter, dtype=torch.bfloat16, device="cuda")
    assert up.numel() > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    up[-1] = torch.randn(2 * inter, d, generator=g, device="cuda").bfloat16() * d ** -0.5
    down[-1] = torch.randn(d, inter, generator=g, device="cuda").bfloat16() * inter ** -0.5
    y = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    nm.nm_moe_ffn(x, torch.full((T, 1), E - 1, dtype=torch.int32, device="cuda"), None, up, down, y, T, d, inter, E, k, SILU, BF16, COL,
                  nm.new_workspace(nm.nm_moe_ffn_workspace_bytes(T, d, inter, E, k)))
    c = dict(x=x.cpu(), up=up[-1:].transpose(1, 2).cpu(), down=down[-1:].transpose(1, 2).cpu(), experts=torch.zeros(T, 1, dtype=torch.int32), weights=None, residual=None)
    assert_within(y, *moe_tests.expected(c, SILU, True, BF16, residual=False))


@pytest.mark.parametrize("layout", [ROW, COL])
def test_a_matrix_and_rows_beyond_32_bit_offsets(layout):
    import paper_2609_16009_b200 as nm
    M, N, K, pitch = 3, 300000, 8192, 2 ** 30 + 8
    B = torch.empty((K, N) if layout == ROW else (N, K), dtype=torch.bfloat16, device="cuda")
    B.normal_(std=K ** -0.5, generator=torch.Generator(device="cuda").manual_seed(2))
    A = randn(M, K, seed=3, dtype=torch.bfloat16).cuda()
    C = torch.empty(2 * pitch + N, dtype=torch.bfloat16, device="cuda")
    nm.nm_matmul_act(A, B, C, M, N, K, NONE, BF16, layout, nm.new_workspace(nm.nm_matmul_act_workspace_bytes(M, N, K)), ldc=pitch)
    for cols in (slice(0, 200), slice(150000, 150200), slice(N - 200, N)):
        W = (B[:, cols] if layout == ROW else B[cols].T).double().cpu()
        z, t = hidden64(A.double().cpu(), W, NONE, False)
        got = torch.stack([C[m * pitch:m * pitch + N][cols] for m in range(M)])
        assert_within(got, z, rounded(z, t, BF16))


def test_calls_on_two_streams_at_once():
    """Workspaces of their own, and nothing else shared."""
    import paper_2609_16009_b200 as nm
    cases = [moe_tests.make(9 + 30 * i, 512, 256, 7, 3, BF16, 50 + i) for i in range(2)]
    dev = [moe_tests.place(c, COL) for c in cases]
    ws = [moe_tests.workspace(nm, c, BF16) for c in cases]
    outs = [[torch.zeros_like(d["x"]) for _ in range(10)] for d in dev]
    A, W, b, r = act_tests.make(5, 2600, 1024, BF16, False, 60)
    dA, dW, db, dr, aws = A.cuda(), stored(W, COL).cuda(), b.cuda(), r.cuda(), nm.new_workspace(nm.nm_matmul_act_workspace_bytes(5, 2600, 1024))
    Cs = [torch.zeros(5, 2600, dtype=torch.bfloat16, device="cuda") for _ in range(10)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for j in range(10):
        for i in range(2):
            moe_tests.call(nm, cases[i], SILU, True, BF16, COL, outs[i][j], ws[i], dev=dev[i], stream=streams[i])
        nm.nm_matmul_act(dA, dW, Cs[j], 5, 2600, 1024, SILU, BF16, COL, aws, bias=db, residual=dr, stream=streams[2])
    torch.cuda.synchronize()
    for i in range(2):
        ref, tol = moe_tests.expected(cases[i], SILU, True, BF16)
        for o in outs[i]:
            assert_within(o, ref, tol)
            assert torch.equal(o, outs[i][0])
    ref, tol = act_tests.expected(A, W, b, r, SILU, False, BF16)
    for o in Cs:
        assert_within(o, ref, tol)


def test_one_workspace_for_products_of_all_sizes(cut):
    """The counters are left as they were found: products of other sizes and cuts follow each other through one workspace."""
    import paper_2609_16009_b200 as nm
    ws = nm.new_workspace(64 << 20)
    for i, (M, N, K, gated, parts) in enumerate([(1, 576, 2048, False, 0), (40, 40000, 64, False, 0), (3, 300, 4096, True, 11), (16, 45000, 128, False, 2), (1, 8, 64, False, 0), (128, 2304, 512, False, 3)]):
        cut(parts)
        A, W, b, r = act_tests.make(M, N, K, BF16, gated, 70 + i)
        assert_within(act_tests.run(A, W, b, r, SILU, gated, BF16, COL, workspace=ws), *act_tests.expected(A, W, b, r, SILU, gated, BF16))
    assert int(ws[:65536].count_nonzero()) == 0
