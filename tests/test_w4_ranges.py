"""The 4-bit product at the ends of what its operands can hold, and over more k than a CTA's tokens fit; against a plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from test_w4 import BF16, BF16_F32OUT, F16, TORCH, case, product, unpack, unpack_scales


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


def close_long(got, A, w, s, dtype, K):
    """Sums over many k: four matrix products of 17 additions per scale, one addition per block of 64 k - all of them, if one warp had them - and
    23 joins, each off by 2^-23 of the sum of magnitudes at most; half a step of the output, fp16's absolute one below its normal range."""
    half = {BF16: 2.0 ** -8, BF16_F32OUT: 2.0 ** -24, F16: 2.0 ** -11}[dtype]
    a = A.double().numpy()
    ref, size = a @ w.T, np.abs(a) @ (23 * s).T
    tol = (68 + -(-K // 64) + 23) * 2.0 ** -23 * size * (1 + half) + half * np.abs(ref) + (2.0 ** -25 if dtype == F16 else 0)
    err = np.abs(got - ref)
    assert np.all(err <= tol), f"worst {np.nanmax(err / tol):.3f} of the tolerance"


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,group,dtype", [(16, 33, 100000, 32, BF16), (16, 200, 30000, 32, F16), (13, 100, 60001, 32, F16), (9, 48, 100000, 32, BF16), (16, 17, 100000, 256, BF16_F32OUT),
                                               (8, 33, 100000, 32, BF16), (3, 40, 200001, 64, BF16), (1, 16, 400000, 32, BF16_F32OUT)])
def test_more_k_than_the_tokens_of_a_cta_fit(M, N, K, group, dtype):
    """Up to eight CTAs share k; with their part over 50 to 300 blocks of 64 (by the number of tokens) its tokens come in several pieces."""
    import paper_2609_16009_b200 as nm
    A, codes, sc, _, _ = case(M, N, K, group, dtype, M + K)
    sc = (sc.float() / 16).to(sc.dtype)
    s = np.repeat(sc.double().numpy(), group, axis=1)[:, :K]
    close_long(product(nm, A, codes, sc, M, N, K, group, dtype), A, (codes - 8) * s, s, dtype, K)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("M,N,K,group", [(16, 18427, 7168, 32), (11, 18432, 7168, 32), (16, 7168, 18432, 32)])
def test_tokens_in_pieces_over_many_columns(M, N, K, group, dtype):
    """Wide matrices whose split along k leaves a CTA more tokens than fit: some of the 16-column strips, the first and the last among them."""
    import paper_2609_16009_b200 as nm
    t, nb, G = TORCH[dtype], -(-N // 16), K // group
    g = torch.Generator(device="cuda").manual_seed(N)
    packed = torch.randint(0, 256, (nm.nm_w4_packed_bytes(N, K),), generator=g, device="cuda", dtype=torch.uint8)
    scales = ((0.5 + torch.rand(nm.nm_w4_scale_count(N, K, group), generator=g, device="cuda")) * 0.005).to(t)
    A = torch.randn(M, K, generator=g, device="cuda").to(t)
    out = torch.zeros(M, N, dtype=t, device="cuda")
    nm.nm_matmul_w4(A, packed, scales, out, M, N, K, group, dtype)
    got, per = out.double().cpu().numpy(), K // 64 * 512
    for strip in (0, 1, nb // 2, nb - 2, nb - 1):
        n = min(16, N - 16 * strip)
        codes = unpack(packed[strip * per:(strip + 1) * per].cpu().numpy(), n, K)
        sc = unpack_scales(scales.view(G, nb, 16)[:, strip].cpu().reshape(-1), n, G)
        s = np.repeat(sc.double().numpy(), group, axis=1)
        close_long(got[:, 16 * strip:16 * strip + n], A.cpu(), (codes - 8) * s, s, dtype, K)
