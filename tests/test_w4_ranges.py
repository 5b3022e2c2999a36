"""The 4-bit product at the ends of what its operands can hold, and over more k than a CTA's tokens fit; against a plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from test_w4 import BF16, BF16_F32OUT, F16, TORCH, product  # noqa: F401


def close(got, A, codes, sc, group):
    """As test_w4's assert_close for fp32 output, with what the tokens lose in fp16 (2^-39 of the row's largest)."""
    s = np.repeat(sc.double().numpy(), group, axis=1)[:, :codes.shape[1]]
    a = A.double().numpy()
    ref, size = a @ ((codes - 8) * s).T, np.abs(a) @ (23 * s).T
    lost = 2.0 ** -39 * np.abs(a).max(1, keepdims=True) * (15 * s).sum(1)
    most = float(np.finfo(np.float32).max)
    assert np.abs(ref).max() < most / 2
    tol = 160 * 2.0 ** -23 * size * (1 + 2.0 ** -23) + lost + 2.0 ** -23 * np.abs(ref) + 2.0 ** -149
    err = np.abs(got - ref)
    assert np.all(err <= tol), f"worst {np.nanmax(err / tol):.3f} of the tolerance, {np.count_nonzero(~np.isfinite(got))} not finite"


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5, 16])
@pytest.mark.parametrize("group", [32, 64])
@pytest.mark.parametrize("token,scale", [(2.0 ** 118, 0.005), (2.0 ** 119, 0.005), (2.0 ** 127, 2.0 ** -11), (1.99 * 2.0 ** 127, 2.0 ** -20), (2.0 ** 116, 0.1),
                                         (2.0 ** -126, 0.005), (2.0 ** -126, 2.0 ** 30), (2.0 ** -60, 2.0 ** 60), (2.0 ** 100, 2.0 ** -120), (2.0 ** 60, 2.0 ** 54)])
def test_large_and_small_tokens_of_one_sign(token, scale, group, M):
    """Tokens of one size with codes of one sign: every sum is as large as it gets.  Columns 8 to 15 of a strip hold their codes 16 times as high."""
    import paper_2609_16009_b200 as nm
    N, K = 48, 192
    A = torch.full((M, K), token, dtype=torch.bfloat16)
    codes = np.zeros((N, K), dtype=np.int64)
    codes[1::3], codes[2::3] = 15, np.arange(K) % 16
    sc = torch.full((N, -(-K // group)), scale, dtype=torch.bfloat16)
    close(product(nm, A, codes, sc, M, N, K, group, BF16_F32OUT), A, codes, sc, group)


@pytest.mark.gpu
def test_a_large_token_beside_ordinary_ones():
    """One finite token of the largest size leaves the rows beside it alone, and counts in its own."""
    import paper_2609_16009_b200 as nm
    M, N, K = 3, 32, 256
    g = torch.Generator().manual_seed(2)
    A = torch.randn(M, K, generator=g).to(torch.bfloat16)
    codes = np.random.default_rng(2).integers(0, 16, (N, K))
    sc = torch.full((N, K // 64), 2.0 ** -6, dtype=torch.bfloat16)
    plain = product(nm, A, codes, sc, M, N, K, 64, BF16_F32OUT)
    A[1, 70] = torch.finfo(torch.bfloat16).max
    got = product(nm, A, codes, sc, M, N, K, 64, BF16_F32OUT)
    assert np.array_equal(got[[0, 2]], plain[[0, 2]])
    close(got, A, codes, sc, 64)
