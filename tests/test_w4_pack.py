"""Weights to 4 bits where the type ends."""
import numpy as np
import pytest
import torch

from test_w4 import BF16, COL, F16, ROW, TORCH, unpack, unpack_scales


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("layout", [ROW, COL])
@pytest.mark.parametrize("group", [32, 256])
def test_infinite_weights_keep_their_sign(group, layout, dtype):
    import paper_2609_16009_b200 as nm
    N, K, t = 40, 520, TORCH[dtype]
    g = torch.Generator().manual_seed(group)
    W = torch.randn(N, K, generator=g).to(t)
    plus, minus, nan = (3, 7), (4, 300), (5, 519)
    W[plus], W[minus], W[nan] = float("inf"), -float("inf"), float("nan")
    W[6, 40], W[6, 41] = float("inf"), -float("inf")
    W[7, 256:288] = float("nan")                                   # with groups of 32 a group of nothing else: its scale is 0
    B = (W if layout == COL else W.T).contiguous().cuda()
    packed = torch.zeros(nm.nm_w4_packed_bytes(N, K), dtype=torch.uint8, device="cuda")
    scales = torch.zeros(nm.nm_w4_scale_count(N, K, group), dtype=t, device="cuda")
    back = torch.zeros_like(B)
    nm.nm_w4_quantize(B, packed, scales, N, K, group, dtype, layout)
    nm.nm_w4_dequantize(packed, scales, back, N, K, group, dtype, layout)
    codes, sc = unpack(packed.cpu().numpy(), N, K), unpack_scales(scales.cpu(), N, -(-K // group)).repeat_interleave(group, 1)[:, :K]
    back = (back if layout == COL else back.T).float().cpu()
    assert codes[plus] == 15 and codes[minus] == 0 and codes[nan] == 0 and codes[6, 40] == 15 and codes[6, 41] == 0
    assert (codes[7, 256:288] == (8 if group == 32 else 0)).all()
    assert back[plus] == back[6, 40] == float("inf") and back[minus] == back[6, 41] == -float("inf")
    finite, lost = W.isfinite(), sc.isinf()
    assert lost.sum() == sum(min(group, K - k // group * group) for k in (7, 300, 40))
    assert (codes[(finite & lost).numpy()] == 8).all() and back[finite & lost].isnan().all()
    w, s = W.float()[finite & ~lost], sc.float()[finite & ~lost]
    want = torch.clamp(torch.round(w / s), -8, 7)
    assert np.array_equal(codes[(finite & ~lost).numpy()] - 8, want.numpy()), "the other groups are what they are without"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,power", [(F16, 0), (F16, 10), (F16, -9), (BF16, 0), (BF16, -61), (BF16, 59), (BF16, -118), (BF16, 100)])
def test_every_quotient_of_two_significands(dtype, power):
    """Weights of every significand over scales of (nearly) every significand: the codes of the exactly rounded quotients, ties among them."""
    import paper_2609_16009_b200 as nm
    t, n = TORCH[dtype], 1024 if dtype == F16 else 128
    scale = (n + np.arange(n)) / n * 2.0 ** power                  # one for each column
    top = torch.from_numpy(7 * scale).to(t)                        # the largest of each of its groups
    w = np.concatenate([(n + np.arange(n)) / n * 2.0 ** (power + e) for e in (-1, 0, 1, 2)])
    groups = -(-len(w) // 31)
    W = np.zeros((n, groups, 32))
    W[:, :, 1:] = np.resize(w, groups * 31).reshape(groups, 31) * (1 - 2 * (np.arange(31) % 2))
    W = np.where(np.abs(W) <= top.double().numpy()[:, None, None], W, 0)
    W[:, :, 0] = top.double().numpy()[:, None]
    W = torch.from_numpy(W.reshape(n, -1))
    assert torch.equal(W.to(t).double(), W)
    N, K = W.shape
    packed = torch.zeros(nm.nm_w4_packed_bytes(N, K), dtype=torch.uint8, device="cuda")
    scales = torch.zeros(nm.nm_w4_scale_count(N, K, 32), dtype=t, device="cuda")
    nm.nm_w4_quantize(W.to(t).cuda(), packed, scales, N, K, 32, dtype, COL)
    sc = unpack_scales(scales.cpu(), N, groups)
    assert torch.equal(sc, (top.float() / 7).to(t)[:, None].expand(N, groups))
    want = np.clip(np.rint(W.numpy() / sc.double().repeat_interleave(32, 1).numpy()), -8, 7) + 8     # (a tie's quotient is exact in 64 bits)
    codes = unpack(packed.cpu().numpy(), N, K)
    assert len(np.unique(codes)) >= 15 and np.array_equal(codes, want)
