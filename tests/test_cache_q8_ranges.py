"""Rows of the quantised cache whose values stand at the ends of bf16's range."""
import numpy as np
import pytest
import torch

from test_cache_q8 import records, rounded_to_e4m3, rows_in


@pytest.mark.gpu
@pytest.mark.parametrize("kv", [512, 1024])
@pytest.mark.parametrize("power,eps", [(125, 1e-6), (51, 1e-6), (49, 0.0), (-49, 0.0), (-51, 0.0), (-126, 0.0), (-130, 0.0), (-130, 1e-30)])
def test_write_normalises_rows_at_the_ends_of_the_range(power, eps, kv):
    """The normalised row is ordinary; nothing on the way to it leaves fp32."""
    import paper_2609_16009_b200 as nm
    rope = 64
    x, gamma, _ = rows_in(3, kv, rope, 11, std=2.0 ** power)
    x[1, 5] = 0.0
    if power == 125:
        x[2, 7] = torch.finfo(torch.bfloat16).max
    assert x.isfinite().all() and (x[:, :kv] != 0).sum() > 2 * kv
    gamma = gamma * 3
    cache = torch.zeros(3, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8, device="cuda")
    nm.nm_mla_cache_write_q8(x.cuda(), gamma.cuda(), None, None, cache, 3, 3, kv, rope, eps)
    v = x[:, :kv].double().numpy()
    y = v / np.sqrt((v ** 2).mean(1, keepdims=True) + np.float64(np.float32(eps))) * gamma.double().numpy()
    codes, _, s = records(cache.cpu().numpy(), kv, rope)
    top = np.abs(y).max(1)
    assert (top <= 448 * s[:, 0] * (1 + 2.0 ** -20)).all() and ((top >= 224 * s[:, 0] * (1 - 2.0 ** -20)) | (s[:, 0] == 2.0 ** -32)).all()
    want = np.clip(y / s, -448, 448)
    # half a step of e4m3: 2^-4 of the value, 2^-10 below its normal range; fp32 arithmetic before it 2^-20
    assert np.all(np.abs(codes - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) * (1 + 2.0 ** -15))


@pytest.mark.gpu
def test_codes_next_to_ties():
    """8 million values: every code is the one of the value in 64 bits, those within fp32's rounding of a tie of e4m3 among them; a value that is not
    told apart from a tie at 2^-40 of itself may fall either way."""
    import paper_2609_16009_b200 as nm
    kv, rope, T = 512, 64, 16000
    x, gamma, _ = rows_in(T, kv, rope, 5)
    cache = torch.zeros(T, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8, device="cuda")
    nm.nm_mla_cache_write_q8(x.cuda(), gamma.cuda(), None, None, cache, T, T, kv, rope, 1e-6)
    codes, _, s = records(cache.cpu().numpy(), kv, rope)
    v = x[:, :kv].double().numpy()
    y = v / np.sqrt((v ** 2).mean(1, keepdims=True) + np.float64(np.float32(1e-6))) * gamma.double().numpy()
    want = rounded_to_e4m3(y / s)
    off = codes != want
    near = np.abs(y / s - (codes + want) / 2) <= 2.0 ** -40 * np.abs(want)
    assert not (off & ~near).any(), f"{(off & ~near).sum()} codes on the wrong side of a tie"
    # the row's power of two is the least that holds it
    top = np.abs(y).max(1)
    assert (top <= 448 * s[:, 0] * (1 + 2.0 ** -40)).all() and (top > 224 * s[:, 0] * (1 - 2.0 ** -40)).all()


@pytest.mark.gpu
def test_a_largest_value_just_above_448():
    """Rows whose largest normalised value is 448 up to fp32's rounding: the power of two goes by the value itself."""
    import paper_2609_16009_b200 as nm
    kv, rope = 16, 0
    g = torch.Generator().manual_seed(3)
    x = torch.randn(4096, kv, generator=g).to(torch.bfloat16)
    gamma = torch.full((kv,), 448.0, dtype=torch.bfloat16)
    x[:, 0] = 1.0
    x[:, 1:] = (1 + torch.randint(-2, 3, (4096, kv - 1), generator=g) * 2.0 ** -7).to(torch.bfloat16) * torch.sign(x[:, 1:].float()).to(torch.bfloat16)
    v = x.double().numpy()
    for eps in (0.0, 1e-6, 1e-12):
        cache = torch.zeros(4096, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8, device="cuda")
        nm.nm_mla_cache_write_q8(x.cuda(), gamma.cuda(), None, None, cache, 4096, 4096, kv, rope, eps)
        codes, _, s = records(cache.cpu().numpy(), kv, rope)
        y = v / np.sqrt((v ** 2).mean(1, keepdims=True) + np.float64(np.float32(eps))) * 448.0
        top = np.abs(y).max(1)
        assert (top <= 448 * s[:, 0] * (1 + 2.0 ** -40)).all() and (top > 224 * s[:, 0] * (1 - 2.0 ** -40)).all()
        want = rounded_to_e4m3(y / s)
        assert not ((codes != want) & (np.abs(y / s - (codes + want) / 2) > 2.0 ** -40 * np.abs(want))).any()


@pytest.mark.gpu
def test_values_that_are_ties():
    """Rows of one magnitude without eps: the normaliser is exact, and values that are ties of e4m3, or 448, are taken for what they are."""
    import paper_2609_16009_b200 as nm
    kv, rope = 64, 0
    ties = torch.tensor([1.0625, 1.1875, 17.0, 34.0, 2.0 ** -10, 3 * 2.0 ** -10, 15 * 2.0 ** -10, 0.0, 448.0, 416.0, 1.0, 240.0, 0.53125, 2.0 ** -6, 232.0, 0.0625])
    gamma = ties.repeat(4).to(torch.bfloat16)
    assert torch.equal(gamma.float(), ties.repeat(4))
    size = torch.tensor([1.0, 2.0 ** 20, 2.0 ** -30, 3.0, 1.5, 2.0 ** 60, 2.0 ** -60, 7.0])
    x = (size[:, None] * (1 - 2 * (torch.arange(kv) % 3 == 0).float())).to(torch.bfloat16)
    cache = torch.zeros(8, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8, device="cuda")
    nm.nm_mla_cache_write_q8(x.cuda(), gamma.cuda(), None, None, cache, 8, 8, kv, rope, 0.0)
    codes, _, s = records(cache.cpu().numpy(), kv, rope)
    y = torch.sign(x.float()).double().numpy() * gamma.double().numpy()
    # the normaliser of 1, 2^20 and their like is a power of two; 1 / 3 and its like have no end in binary, and their products are ties to 2^-44 of
    # themselves only
    exact = [0, 1, 2, 5, 6]
    assert (s[exact, 0] == 1).all() and np.isin(s[:, 0], (1, 2)).all()
    assert np.array_equal(codes[exact], rounded_to_e4m3(y[exact]))
    assert np.all(np.abs(codes * s - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * s))


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [1e-6, 0.0])
def test_zeros_in_and_as_rows(eps):
    """A zero stays one beside other values, and a row of zeros has scale 1."""
    import paper_2609_16009_b200 as nm
    kv, rope, T = 272, 8, 5
    x, gamma, _ = rows_in(T, kv, rope, 8)
    x[:, 10:30], x[1, :kv] = 0.0, 0.0
    gamma[40] = 0.0
    x[2, :kv] = 0.0
    x[2, 7] = 1.0
    cache = torch.zeros(T, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8, device="cuda")
    nm.nm_mla_cache_write_q8(x.cuda(), gamma.cuda(), None, None, cache, T, T, kv, rope, eps)
    codes, _, s = records(cache.cpu().numpy(), kv, rope)
    keep = [0, 2, 3, 4] + ([1] if eps else [])                     # (without eps a row of zeros is 0 / 0)
    assert not codes[keep][:, 10:30].any() and not codes[keep][:, 40].any()
    assert (codes[2] != 0).sum() == 1
    if eps:
        assert s[1, 0] == 1 and not codes[1].any()
    else:
        assert np.isnan(codes[1]).all()
