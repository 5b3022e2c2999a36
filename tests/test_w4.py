"""4-bit weights: the narrow product nm_matmul_w4 and the packing entry points, against a plain implementation in 64 bits that
places every nibble by the storage formula of include/nm.h."""
import ctypes

import numpy as np
import pytest
import torch

BF16, BF16_F32OUT, F16, ROW, COL = 1, 2, 3, 0, 1
TORCH = {BF16: torch.bfloat16, BF16_F32OUT: torch.bfloat16, F16: torch.float16}


def strips(N):
    return -(-N // 16)


def blocks(K):
    return -(-K // 64)


def pack(codes):
    """codes [N][K] (0..15) -> packed bytes, by the formula; places beyond N and K get code 5."""
    N, K = codes.shape
    nb, kb = strips(N), blocks(K)
    full = np.full((nb * 16, kb * 64), 5, dtype=np.uint8)
    full[:N, :K] = codes
    out = np.zeros(nb * kb * 512, dtype=np.uint8)
    g, t, j, b = np.meshgrid(np.arange(8), np.arange(4), np.arange(4), np.arange(4), indexing="ij")
    at = 4 * (4 * (4 * g + t) + j) + b
    k = 32 * (j >> 1) + 8 * t + 4 * (j & 1) + 2 * (b & 1) + (b >> 1)
    for s in range(nb):
        for c in range(kb):
            cell = full[16 * s:16 * s + 16, 64 * c:64 * c + 64]
            out[(s * kb + c) * 512 + at] = cell[g, k] | (cell[g + 8, k] << 4)
    return out


def unpack(packed, N, K):
    nb, kb = strips(N), blocks(K)
    g, t, j, b = np.meshgrid(np.arange(8), np.arange(4), np.arange(4), np.arange(4), indexing="ij")
    at = 4 * (4 * (4 * g + t) + j) + b
    k = 32 * (j >> 1) + 8 * t + 4 * (j & 1) + 2 * (b & 1) + (b >> 1)
    full = np.zeros((nb * 16, kb * 64), dtype=np.int64)
    for s in range(nb):
        for c in range(kb):
            v = packed[(s * kb + c) * 512 + at]
            full[16 * s + g, 64 * c + k] = v & 15
            full[16 * s + g + 8, 64 * c + k] = v >> 4
    return full[:N, :K]


def pack_scales(sc):
    """scales [N][G] (tensor) -> storage order; columns beyond N get NaN, which nothing may read into a result."""
    N, G = sc.shape
    nb = strips(N)
    full = torch.full((nb * 16, G), float("nan"), dtype=sc.dtype)
    full[:N] = sc
    return full.view(nb, 2, 8, G).permute(3, 0, 2, 1).contiguous().reshape(-1)


def unpack_scales(flat, N, G):
    nb = strips(N)
    return flat.view(G, nb, 8, 2).permute(1, 3, 2, 0).reshape(nb * 16, G)[:N]


def case(M, N, K, group, dtype, seed, lda=None):
    rng = np.random.default_rng(seed)
    t = TORCH[dtype]
    codes = rng.integers(0, 16, (N, K))
    sc = torch.from_numpy(rng.uniform(0.5, 1.5, (N, -(-K // group))) * 0.005).to(t)
    A = torch.from_numpy(rng.standard_normal((M, K))).to(t)
    w = (codes - 8) * np.repeat(sc.double().numpy(), group, axis=1)[:, :K]
    a = A.double().numpy()
    # sizes of the terms that are added: a times a code 0..15, and 8 a taken off again
    return A, codes, sc, a @ w.T, np.abs(a) @ (23 * np.repeat(sc.double().numpy(), group, axis=1)[:, :K]).T


def assert_close(got, ref, size, dtype):
    # fp32 sums: at most four matrix products of 17 additions per scale, then one addition per block of a warp's run of k and
    # fifteen joins - below 160 additions for the lengths tested, each off by at most 2^-23 of the sum of magnitudes - and
    # half a step of the output type, with fp16's absolute step below its normal range
    half = {BF16: 2.0 ** -9, BF16_F32OUT: 2.0 ** -24, F16: 2.0 ** -12}[dtype]
    tol = 160 * 2.0 ** -23 * size * (1 + half) + 2 * half * np.abs(ref) + (2.0 ** -25 if dtype == F16 else 0)
    err = np.abs(got - ref)
    assert np.all(err <= tol), f"worst {np.max(err / np.maximum(tol, 1e-300)):.3f} of the tolerance"


def product(nm, A, codes, sc, M, N, K, group, dtype, lda=None, ldc=None, shift=0):
    lda, ldc = lda or K, ldc or N
    out = torch.float32 if dtype == BF16_F32OUT else TORCH[dtype]
    dA = torch.full((M * lda + shift,), float("nan"), dtype=TORCH[dtype], device="cuda")
    dA[shift:].view(M, lda)[:, :K] = A.cuda()
    packed, scales = torch.from_numpy(pack(codes)).cuda(), pack_scales(sc).cuda()
    C = torch.full((M + 2, ldc), 77.0, dtype=out, device="cuda")
    nm.nm_matmul_w4(dA[shift:], packed, scales, C[1:], M, N, K, group, dtype, lda=lda, ldc=ldc)
    again = torch.full((M, ldc), 77.0, dtype=out, device="cuda")
    nm.nm_matmul_w4(dA[shift:], packed, scales, again, M, N, K, group, dtype, lda=lda, ldc=ldc)
    bits = torch.int32 if out == torch.float32 else torch.int16
    assert torch.equal(C[1:M + 1].view(bits), again.view(bits)), "equal calls give equal bits"
    c = C.double().cpu().numpy()
    assert (c[0] == 77).all() and (c[-1] == 77).all() and (c[:, N:] == 77).all(), "written outside C"
    return c[1:M + 1, :N]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, BF16_F32OUT, F16])
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 64), (3, 17, 63), (8, 31, 65), (9, 33, 257), (16, 100, 1000), (2, 576, 2048), (16, 48, 4104), (5, 2500, 136)])
def test_product(M, N, K, group, dtype):
    import paper_2609_16009_b200 as nm
    A, codes, sc, ref, size = case(M, N, K, group, dtype, M * 1000 + N + K)
    assert_close(product(nm, A, codes, sc, M, N, K, group, dtype), ref, size, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("M", range(1, 17))
def test_every_token_count(M):
    import paper_2609_16009_b200 as nm
    A, codes, sc, ref, size = case(M, 208, 1536, 64, BF16, 50 + M)
    assert_close(product(nm, A, codes, sc, M, 208, 1536, 64, BF16), ref, size, BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 7168, 512), (4, 19001, 200), (16, 576, 7168), (7, 16, 18432), (12, 6000, 1024)])
def test_every_split(M, N, K):
    """Wide, long and small products: warps side by side over the columns, along k, and clusters along k."""
    import paper_2609_16009_b200 as nm
    A, codes, sc, ref, size = case(M, N, K, 128, BF16_F32OUT, N + K)
    assert_close(product(nm, A, codes, sc, M, N, K, 128, BF16_F32OUT), ref, size, BF16_F32OUT)


@pytest.mark.gpu
@pytest.mark.parametrize("lda,ldc,shift", [(1024, 320, 0), (1000, 301, 0), (1003, 307, 0), (1000, 300, 1), (1000, 300, 8)])
def test_strides_and_alignment(lda, ldc, shift):
    """Rows of A and C inside wider ones, starting on any element; what lies between the rows is NaN and stays out."""
    import paper_2609_16009_b200 as nm
    A, codes, sc, ref, size = case(11, 300, 1000, 64, F16, 9)
    assert_close(product(nm, A, codes, sc, 11, 300, 1000, 64, F16, lda=lda, ldc=ldc, shift=shift), ref, size, F16)


@pytest.mark.gpu
def test_codes_are_exact_integers():
    """One-hot tokens read single weights: (code - 8) * scale to the last bit, every code.  A token row with an infinity or a NaN
    gives NaN and leaves the other rows alone."""
    import paper_2609_16009_b200 as nm
    N, K = 32, 128
    codes = np.arange(N * K).reshape(N, K) % 16
    sc = torch.from_numpy(np.linspace(0.01, 0.02, N * 2).reshape(N, 2)).to(torch.bfloat16)
    for k in (0, 1, 17, 63, 64, 100, 127):
        for dtype in (BF16_F32OUT, F16):
            for big in (1.0, 0.25, 448.0):
                A = torch.zeros(3, K, dtype=TORCH[dtype])
                A[0, k], A[1, k], A[2, 5] = big, float("inf"), float("nan")
                got = product(nm, A, codes, sc.to(TORCH[dtype]), 3, N, K, 64, dtype)
                want = torch.from_numpy((codes[:, k] - 8) * sc.to(TORCH[dtype]).double().numpy()[:, k // 64] * big)
                assert np.array_equal(got[0], (want if dtype == BF16_F32OUT else want.half()).double().numpy())
                assert np.isnan(got[1:]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("low,high", [(-30, 10), (-126, -100), (95, 118), (-3, 3)])
def test_wide_ranges_of_tokens(low, high):
    """bf16 tokens of very different sizes in one row, and rows at the ends of the type's range."""
    import paper_2609_16009_b200 as nm
    M, N, K = 3, 64, 640
    A, codes, sc, _, _ = case(M, N, K, 64, BF16_F32OUT, 77)
    e = torch.randint(low, high + 1, (M, K), generator=torch.Generator().manual_seed(3)).double()
    A = (A.double().clamp(-1, 1) * 2.0 ** e).to(torch.bfloat16)
    w = (codes - 8) * np.repeat(sc.double().numpy(), 64, axis=1)
    a = A.double().numpy()
    got = product(nm, A, codes, sc, M, N, K, 64, BF16_F32OUT)
    # as assert_close, with sums of terms up to 15 |a| (see the kernel), and the tokens' absolute step: 2^-40 of the row's largest
    s = np.repeat(sc.double().numpy(), 64, axis=1)
    size = np.abs(a) @ (23 * s).T
    tol = 160 * 2.0 ** -23 * size + 2.0 ** -40 * np.abs(a).max(1, keepdims=True) * (15 * s).sum(1) + 2.0 ** -149
    assert np.all(np.abs(got - a @ w.T) <= tol)


@pytest.mark.gpu
def test_streams_graph_and_programmatic_launch():
    """Two calls on two streams share nothing; a captured product replays with new tokens; programmatic launch changes no bit."""
    import paper_2609_16009_b200 as nm
    M, N, K = 4, 512, 7168
    A, codes, sc, ref, size = case(M, N, K, 128, BF16, 4)
    packed, scales, dA = torch.from_numpy(pack(codes)).cuda(), pack_scales(sc).cuda(), A.cuda()
    outs = [torch.zeros(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        nm.nm_matmul_w4(dA, packed, scales, outs[0], M, N, K, 128, BF16, stream=s1)
        nm.nm_matmul_w4(dA, packed, scales, outs[1], M, N, K, 128, BF16, stream=s2)
    torch.cuda.synchronize()
    x = torch.zeros_like(dA)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nm.nm_matmul_w4(x, packed, scales, outs[2], M, N, K, 128, BF16)
    x.copy_(dA)
    g.replay()
    nm.nm_set_programmatic_launch(True)
    try:
        for _ in range(3):
            nm.nm_matmul_w4(dA, packed, scales, outs[3], M, N, K, 128, BF16)
    finally:
        nm.nm_set_programmatic_launch(False)
    torch.cuda.synchronize()
    assert_close(outs[0].double().cpu().numpy(), ref, size, BF16)
    assert all(torch.equal(outs[0], o) for o in outs[1:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("layout", [ROW, COL])
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 64), (65, 255), (70, 257), (200, 600), (128, 1024)])
def test_quantise_and_back(N, K, group, layout, dtype):
    import paper_2609_16009_b200 as nm
    rng = np.random.default_rng(N * K + group)
    t = TORCH[dtype]
    W = torch.from_numpy(rng.standard_normal((N, K)) * 0.02).to(t)
    W[0, : min(K, group)] = 0                                       # a group of zeros
    G = -(-K // group)
    wide = np.zeros((N, G * group), dtype=np.float32)
    wide[:, :K] = W.float().numpy()
    amax = np.abs(wide.reshape(N, G, group)).max(2)
    sc = torch.from_numpy(amax / np.float32(7)).to(t)
    s32 = np.repeat(sc.float().numpy(), group, axis=1)[:, :K]
    w32 = W.float().numpy()
    with np.errstate(divide="ignore", invalid="ignore"):
        codes = np.where(s32 > 0, np.clip(np.rint(w32 / s32), -8, 7), 0).astype(np.int64) + 8
    back = torch.from_numpy((codes - 8).astype(np.float32) * s32).to(t)
    B = (W if layout == COL else W.T).contiguous().cuda()
    packed = torch.full((nm.nm_w4_packed_bytes(N, K) + 64,), 0xEE, dtype=torch.uint8, device="cuda")
    scales = torch.full((nm.nm_w4_scale_count(N, K, group) + 16,), 3.0, dtype=t, device="cuda")
    out = torch.full((B.numel() + 16,), 3.0, dtype=t, device="cuda")
    nm.nm_w4_quantize(B, packed, scales, N, K, group, dtype, layout)
    nm.nm_w4_dequantize(packed, scales, out, N, K, group, dtype, layout)
    torch.cuda.synchronize()
    assert (packed[-64:] == 0xEE).all() and (scales[-16:] == 3).all() and (out[-16:] == 3).all(), "written outside"
    assert np.array_equal(unpack(packed.cpu().numpy()[:-64], N, K), codes)
    assert torch.equal(unpack_scales(scales.cpu()[:-16], N, G), sc)
    got = out[:-16].view(B.shape).cpu()
    assert torch.equal(got if layout == COL else got.T, back)


@pytest.mark.gpu
def test_quantise_strange_weights():
    """NaN becomes code 0, an infinite group keeps to the codes' range: no undefined conversion."""
    import paper_2609_16009_b200 as nm
    W = torch.ones(16, 64, dtype=torch.bfloat16)
    W[0, 3], W[1, 5], W[2, :] = float("nan"), float("inf"), 1e-38
    packed = torch.zeros(512, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(16, dtype=torch.bfloat16, device="cuda")
    nm.nm_w4_quantize(W.cuda(), packed, scales, 16, 64, 64, BF16, COL)
    codes = unpack(packed.cpu().numpy(), 16, 64)
    assert codes[0, 3] == 0 and (np.delete(codes[0], 3) == 15).all()
    assert (codes[3:] == 15).all() and codes.min() >= 0
    assert unpack_scales(scales.cpu(), 16, 1)[1].item() == float("inf")


@pytest.mark.gpu
def test_weights_beyond_32_bit_offsets():
    """Weights of 17 GB, 4 GB packed, zeros but for the last sixteen columns: quantised, multiplied and brought back as those alone are."""
    import paper_2609_16009_b200 as nm
    N, K, group = 16 * 8193, 65536, 256
    assert nm.nm_w4_packed_bytes(N, K) > 2 ** 32
    g = torch.Generator().manual_seed(5)
    last = torch.randn(16, K, generator=g).to(torch.bfloat16).cuda()
    B = torch.zeros(N, K, dtype=torch.bfloat16, device="cuda")
    B[-16:] = last
    one, many = ((torch.zeros(nm.nm_w4_packed_bytes(n, K), dtype=torch.uint8, device="cuda"),
                  torch.zeros(nm.nm_w4_scale_count(n, K, group), dtype=torch.bfloat16, device="cuda")) for n in (16, N))
    nm.nm_w4_quantize(last, *one, 16, K, group, BF16, COL)
    nm.nm_w4_quantize(B, *many, N, K, group, BF16, COL)
    assert torch.equal(many[0][-one[0].numel():], one[0]) and (many[0][:-one[0].numel()] == 0x88).all()
    assert torch.equal(many[1].view(K // group, -1)[:, -16:].reshape(-1), one[1])
    A = torch.randn(2, K, generator=g).to(torch.bfloat16).cuda()
    C, c = torch.full((2, N), 7.0, device="cuda"), torch.zeros(2, 16, device="cuda")
    nm.nm_matmul_w4(A, *many, C, 2, N, K, group, BF16_F32OUT)
    nm.nm_matmul_w4(A, *one, c, 2, 16, K, group, BF16_F32OUT)
    assert (C[:, :-16].abs() <= 0).all()
    # both are sums of K terms in fp32, split differently: 2^-23 a step and eight-block runs, of the size of the terms (code and 8 apart: 23 / 8)
    back = torch.zeros(16, K, dtype=torch.bfloat16, device="cuda")
    nm.nm_w4_dequantize(*one, back, 16, K, group, BF16, COL)
    size = A.double().abs() @ back.double().abs().T + A.double().abs().sum(1, keepdim=True) * back.double().abs().max()
    assert ((C[:, -16:].double() - c.double()).abs() <= 2 * 160 * 2.0 ** -23 * 3 * size).all() and c.abs().sum() > 0
    nm.nm_w4_dequantize(*many, B, N, K, group, BF16, COL)
    assert torch.equal(B[-16:], back) and not B[:-16].any()


def test_refusals():
    """Bad arguments are refused before anything is enqueued: no device is needed."""
    import paper_2609_16009_b200 as nm
    vp, lib = ctypes.c_void_p, nm._lib
    ok = dict(A=256, p=512, s=1024, C=2048, M=1, N=32, K=64, g=64, lda=64, ldc=32, d=BF16)

    def call(**kw):
        a = dict(ok, **kw)
        return lib.nm_matmul_w4(vp(a["A"]), vp(a["p"]), vp(a["s"]), vp(a["C"]), a["M"], a["N"], a["K"], a["g"], a["lda"], a["ldc"], a["d"], None)

    for bad in (dict(A=None), dict(p=None), dict(s=None), dict(C=None), dict(M=0), dict(M=17), dict(N=0), dict(K=0), dict(lda=63), dict(ldc=31)):
        assert call(**bad) == -1, bad
    for bad in (dict(d=0), dict(d=9), dict(g=0), dict(g=48), dict(g=512), dict(g=-64), dict(K=(1 << 30) + 1, lda=1 << 31)):
        assert call(**bad) == -2, bad
    for bad in (dict(A=257), dict(p=520), dict(s=1026), dict(C=2049), dict(C=2050, d=BF16_F32OUT)):
        assert call(**bad) == -3, bad
    assert nm.nm_w4_packed_bytes(17, 65) == 2 * 2 * 512 and nm.nm_w4_packed_bytes(0, 5) == 0
    assert nm.nm_w4_scale_count(17, 65, 32) == 32 * 3 and nm.nm_w4_scale_count(17, 65, 33) == 0
    for fn in (lib.nm_w4_quantize, lib.nm_w4_dequantize):
        assert fn(None, vp(512), vp(1024), 16, 64, 64, BF16, ROW, None) == -1
        assert fn(vp(256), vp(512), vp(1024), 0, 64, 64, BF16, ROW, None) == -1
        assert fn(vp(256), vp(512), vp(1024), 16, 64, 64, 0, ROW, None) == -2
        assert fn(vp(256), vp(512), vp(1024), 16, 64, 100, BF16, ROW, None) == -2
        assert fn(vp(256), vp(512), vp(1024), 16, 64, 64, BF16, 2, None) == -2
        assert fn(vp(256), vp(512), vp(1024), 64 * 65535 + 1, 64, 64, BF16, ROW, None) == -2
        assert fn(vp(256), vp(512), vp(1024), 16, (1 << 30) + 1, 64, BF16, ROW, None) == -2
        assert fn(vp(256), vp(512), vp(1025), 16, 64, 64, BF16, ROW, None) == -3


def test_pack_formula_round_trip():
    codes = np.random.default_rng(1).integers(0, 16, (21, 130))
    assert np.array_equal(unpack(pack(codes), 21, 130), codes)
