"""Quantised latent cache: rows normalised, rotated, quantised and stored, and read back, against a plain implementation in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

EPS = 1e-6


def e4m3_value(code):
    """The value of e4m3 codes (uint8 array), from the format's definition."""
    c = code.astype(np.int64)
    exp, man = (c >> 3) & 15, c & 7
    v = np.where(exp == 0, man * 2.0 ** -9, (8 + man) * 2.0 ** (exp - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >> 7, -v, v)


def records(cache, kv, rope):
    """uint8 [n][bytes] -> (latent codes' values, key part, scales) in 64 bits."""
    a = np.ascontiguousarray(cache)
    key = np.ascontiguousarray(a[:, kv:kv + 2 * rope]).view(np.uint16).astype(np.uint32) << 16
    s = np.ascontiguousarray(a[:, kv + 2 * rope:kv + 2 * rope + 4]).view(np.float32).astype(np.float64)
    assert not a[:, kv + 2 * rope + 4:].any()
    return e4m3_value(a[:, :kv]), key.view(np.float32).astype(np.float64).reshape(len(a), rope), s


def rounded_to_e4m3(x):
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    return np.clip(np.rint(x / 2.0 ** (e - 3)) * 2.0 ** (e - 3), -448, 448)


def reference(x, gamma, cs, kv, rope):
    x = x.astype(np.float64)
    y, r = x[:, :kv], x[:, kv:]
    if gamma is not None:
        y = y / np.sqrt((y ** 2).mean(1, keepdims=True) + EPS) * gamma
    if cs is not None:
        a, b, c, s = r[:, 0::2], r[:, 1::2], cs[:, 0::2].astype(np.float64), cs[:, 1::2].astype(np.float64)
        r = np.stack((a * c - b * s, a * s + b * c), -1).reshape(len(x), rope)
    return y, r


def rows_in(T, kv, rope, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, kv + rope, generator=g) * std).to(torch.bfloat16)
    gamma = (1 + 0.1 * torch.randn(kv, generator=g)).to(torch.bfloat16)
    ang = torch.rand(T, max(rope // 2, 1), generator=g, dtype=torch.float64) * 6.283
    cs = torch.stack((ang.cos(), ang.sin()), -1).reshape(T, -1).float()[:, :rope].contiguous()
    return x, gamma, cs


@pytest.mark.gpu
@pytest.mark.parametrize("normed,rotated", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("T,kv,rope,stride", [(1, 512, 64, 576), (5, 512, 64, 2112), (33, 512, 64, 576), (3, 16, 8, 24), (7, 528, 0, 528), (4, 1024, 256, 1288), (9, 272, 24, 296)])
def test_write(T, kv, rope, stride, normed, rotated):
    import paper_2609_16009_b200 as nm
    x, gamma, cs = rows_in(T, kv, rope, T + kv)
    nbytes, n = nm.nm_mla_q8_row_bytes(kv, rope), 2 * T + 3
    assert nbytes == kv + 2 * rope + 16
    wide = torch.full((T, stride), float("nan"), dtype=torch.bfloat16)
    wide[:, :kv + rope] = x
    order = torch.from_numpy(np.random.default_rng(T).permutation(n)[:T].astype(np.int64))
    skipped = T // 2 if T > 2 else None
    if skipped is not None:
        order[skipped] = -1
        if T > 4:
            order[0] = n
    cache = torch.full((n, nbytes), 0xA5, dtype=torch.uint8, device="cuda")
    nm.nm_mla_cache_write_q8(wide.cuda(), gamma.cuda() if normed else None, cs.cuda() if rotated and rope else None, order.cuda(), cache, n, T, kv, rope, EPS,
                             ckr_stride=stride)
    got = cache.cpu().numpy()
    kept = [t for t in range(T) if 0 <= order[t] < n]
    untouched = sorted(set(range(n)) - {int(order[t]) for t in kept})
    assert (got[untouched] == 0xA5).all(), "a row that was not named is left as it was"
    y, r = reference(x.double().numpy(), gamma.double().numpy() if normed else None, cs.numpy() if rotated else None, kv, rope)
    codes, key, s = records(got[order[kept].numpy()], kv, rope)
    y, r = y[kept], r[kept]
    e = np.log2(s[:, 0])
    top = np.abs(y).max(1)
    # the least power of two that holds the row; fp32 may see the largest value 2^-20 off
    assert np.array_equal(e, np.rint(e)) and (top <= 448 * s[:, 0] * (1 + 2.0 ** -20)).all() and (top >= 224 * s[:, 0] * (1 - 2.0 ** -20)).all()
    # half a step of e4m3: 2^-4 of the value, 2^-10 below its normal range; fp32 arithmetic before it 2^-20
    want = np.clip(y / s, -448, 448)
    assert np.all(np.abs(codes - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) * (1 + 2.0 ** -15))
    if not normed:
        assert np.array_equal(codes, rounded_to_e4m3(want)), "without a norm nothing comes before the one rounding"
    # half a step of bf16: 8 significant bits, steps of 2^-7 of the binade, so 2^-8 of the value; fp32 products of two terms before it
    size = np.repeat(np.abs(r).reshape(len(kept), rope // 2, 2).max(2), 2, axis=1) if rope else r
    assert np.all(np.abs(key * s - r) <= 2.0 ** -8 * np.abs(r) + 2.0 ** -22 * 2 * size)


@pytest.mark.gpu
def test_write_at_the_ends_of_the_range():
    """Zeros, tiny and huge rows, a NaN, an infinity; codes at and beyond the format's ties."""
    import paper_2609_16009_b200 as nm
    kv, rope = 64, 8
    x = torch.zeros(8, kv + rope, dtype=torch.bfloat16)
    x[1, :kv] = 2.0 ** -100
    x[2, :kv] = 2.0 ** 60
    x[3, 0], x[3, 1] = float("nan"), 3.0
    x[4, 0], x[4, 1] = float("inf"), 3.0
    x[5, :6] = torch.tensor([448.0, 1.0625, 1.1875, 2.0 ** -9, 2.0 ** -10, 0.75 * 2.0 ** -9])      # ties to even, subnormals
    x[6, 0], x[7, 0] = 450.0, 449.0 * 2.0 ** -20
    x[:, kv:] = 5.0
    cache = torch.zeros(8, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8, device="cuda")
    nm.nm_mla_cache_write_q8(x.cuda(), None, None, None, cache, 8, 8, kv, rope, EPS)
    codes, key, s = records(cache.cpu().numpy(), kv, rope)
    # (449 lies half way between the bf16 numbers 448 and 450 and becomes the even one, 448: still within 448 * 2^-20)
    assert s[:, 0].tolist() == [1.0, 2.0 ** -32, 2.0 ** 32, 2.0 ** -7, 2.0 ** 32, 1.0, 2.0, 2.0 ** -20]
    assert not codes[0].any() and not codes[1].any() and (codes[2] == 448).all()
    assert np.isnan(codes[3, 0]) and codes[3, 1] == 384 and codes[4, 0] == 448
    assert codes[5, :6].tolist() == [448.0, 1.0, 1.25, 2.0 ** -9, 0.0, 2.0 ** -9]
    assert np.array_equal(key * s, np.full((8, rope), 5.0)), "the key part survives any scale exactly"


@pytest.mark.gpu
@pytest.mark.parametrize("power", [-12, 70, 100])
def test_write_normalises_rows_of_any_size(power):
    """Squares beyond fp32's range belong to the norm all the same."""
    import paper_2609_16009_b200 as nm
    kv, rope = 512, 64
    x, gamma, _ = rows_in(3, kv, rope, 11, std=2.0 ** power)
    x[1, 5] = 0.0
    cache = torch.zeros(3, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8, device="cuda")
    nm.nm_mla_cache_write_q8(x.cuda(), gamma.cuda(), None, None, cache, 3, 3, kv, rope, EPS)
    y, _ = reference(x.double().numpy(), gamma.double().numpy(), None, kv, rope)
    codes, _, s = records(cache.cpu().numpy(), kv, rope)
    assert (np.abs(y).max(1) <= 448 * s[:, 0] * (1 + 2.0 ** -20)).all()
    want = np.clip(y / s, -448, 448)
    # half a step of e4m3: 2^-4 of the value, 2^-10 below its normal range; fp32 arithmetic before it 2^-20
    assert np.all(np.abs(codes - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) * (1 + 2.0 ** -15))


@pytest.mark.gpu
@pytest.mark.parametrize("n,kv,rope,stride", [(1, 512, 64, 576), (130, 512, 64, 584), (9, 16, 8, 24), (5, 1024, 256, 1280), (6, 528, 0, 536)])
def test_read(n, kv, rope, stride):
    import paper_2609_16009_b200 as nm
    g = torch.Generator().manual_seed(n)
    rows = 40
    cache = torch.zeros(rows, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8)
    codes = torch.randint(0, 256, (rows, kv), generator=g, dtype=torch.uint8)
    codes[(codes & 127) == 127] = 0
    cache[:, :kv] = codes
    cache[:, kv:kv + 2 * rope] = torch.randn(rows, rope, generator=g).to(torch.bfloat16).view(torch.uint8).view(rows, 2 * rope)
    cache[:, kv + 2 * rope:kv + 2 * rope + 4] = torch.exp2(torch.randint(-32, 33, (rows, 1), generator=g).float()).view(torch.uint8)
    index = torch.randint(0, rows, (n,), generator=g)
    if n > 4:
        index[1], index[2], index[3] = -1, rows, index[4]           # none, none, the same row twice
    out = torch.full((n + 1, stride), 9.0, dtype=torch.bfloat16, device="cuda")
    nm.nm_mla_cache_read_q8(cache.cuda(), rows, index.cuda(), out, n, kv, rope, out_stride=stride)
    v, key, s = records(cache.numpy(), kv, rope)
    want = np.concatenate((v, key), 1) * s
    got = out.double().cpu().numpy()
    assert (got[n] == 9).all() and (got[:, kv + rope:] == 9).all(), "written outside the rows"
    for i in range(n):
        r = int(index[i])
        assert np.array_equal(got[i, :kv + rope], want[r] if 0 <= r < rows else np.zeros(kv + rope)), "reading back is exact"


@pytest.mark.gpu
def test_rows_without_an_index_streams_and_graph():
    import paper_2609_16009_b200 as nm
    kv, rope, T = 512, 64, 50
    x, gamma, cs = (t.cuda() for t in rows_in(T, kv, rope, 1))
    cache, other = (torch.zeros(T, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8, device="cuda") for _ in range(2))
    back, again = (torch.zeros(T, kv + rope, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    nm.nm_mla_cache_write_q8(x, gamma, cs, None, cache, T, T, kv, rope, EPS, stream=s)
    nm.nm_mla_cache_read_q8(cache, T, None, back, T, kv, rope, stream=s)
    torch.cuda.synchronize()
    zeros = torch.zeros_like(x)
    g = torch.cuda.CUDAGraph()
    nm.nm_set_programmatic_launch(True)
    try:
        with torch.cuda.graph(g):
            nm.nm_mla_cache_write_q8(zeros, gamma, cs, None, other, T, T, kv, rope, EPS)
            nm.nm_mla_cache_read_q8(other, T, None, again, T, kv, rope)
    finally:
        nm.nm_set_programmatic_launch(False)
    zeros.copy_(x)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(cache, other) and torch.equal(back, again) and back.abs().sum() > 0


def test_refusals():
    import paper_2609_16009_b200 as nm
    vp, lib = ctypes.c_void_p, nm._lib

    def write(x=256, stride=576, gamma=512, cs=1024, rows=2048, cache=4096, n=8, T=2, kv=512, rope=64):
        return lib.nm_mla_cache_write_q8(vp(x), stride, vp(gamma), vp(cs), vp(rows), vp(cache), n, T, kv, rope, 1e-6, None)

    def read(cache=256, n_rows=8, rows=512, out=1024, stride=576, n=2, kv=512, rope=64):
        return lib.nm_mla_cache_read_q8(vp(cache), n_rows, vp(rows), vp(out), stride, n, kv, rope, None)

    for bad in (dict(x=None), dict(cache=None), dict(T=0), dict(T=(1 << 30) + 1), dict(n=0), dict(stride=575)):
        assert write(**bad) == -1, bad
    for bad in (dict(kv=8, rope=64), dict(kv=520, stride=584), dict(kv=1040, stride=4096), dict(rope=12), dict(rope=-8), dict(rope=264, stride=4096)):
        assert write(**bad) == -2, bad
        assert nm.nm_mla_q8_row_bytes(bad.get("kv", 512), bad.get("rope", 64)) == 0
    for bad in (dict(x=264), dict(stride=580), dict(cache=4104), dict(gamma=520), dict(cs=1028), dict(rows=2052)):
        assert write(**bad) == -3, bad
    for bad in (dict(cache=None), dict(out=None), dict(n=0), dict(n=(1 << 30) + 1), dict(n_rows=0), dict(stride=575)):
        assert read(**bad) == -1, bad
    for bad in (dict(kv=500), dict(rope=4)):
        assert read(**bad) == -2, bad
    for bad in (dict(cache=264), dict(out=1032), dict(stride=577), dict(rows=516)):
        assert read(**bad) == -3, bad
    assert nm.nm_mla_q8_row_bytes(512, 64) == 656
