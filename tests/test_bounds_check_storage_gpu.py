"""The kernels on compressed storage in the debug build (libnm_check.so): every hand-indexed access against the extent of its operand, over the
ragged shapes at which such arithmetic goes wrong.  Clean, and the bits of the normal build."""
import ctypes as C

import numpy as np
import pytest
import torch

from test_attention_q8 import KV, REC, ROPE, SCALE, case as batch_case
from test_cache_q8 import rows_in
from test_w4 import BF16, BF16_F32OUT, COL, F16, ROW, TORCH, case, pack, pack_scales

pytestmark = pytest.mark.gpu
NAMES = ("nm_matmul_w4", "nm_w4_quantize", "nm_w4_dequantize", "nm_mla_cache_write_q8", "nm_mla_cache_read_q8", "nm_mla_attention_q8", "nm_check_status",
         "nm_mla_attention_q8_workspace_bytes")


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


def same_in_both(call, check):
    """call(): the outputs of one run through the binding.  Returns the normal build's."""
    import paper_2609_16009_b200 as nm
    normal, outs = nm._lib, []
    for lib in (normal, check):
        nm._lib = lib
        try:
            out = call(nm)
            torch.cuda.synchronize()
            assert lib.nm_check_status(None) == 0, "an access outside its operand (or an expired wait) was reported"
        finally:
            nm._lib = normal
        outs.append(out)
    for a, b in zip(*outs):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), "the checked build computes different bits"
    return outs[0]


@pytest.mark.parametrize("dtype,group", [(BF16, 32), (BF16_F32OUT, 64), (F16, 128), (BF16, 256), (F16, 32)])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 64), (3, 17, 63), (8, 31, 65), (9, 33, 257), (16, 100, 1000), (2, 576, 2048), (16, 48, 4104), (5, 2500, 136), (7, 16, 18432),
                                   (12, 6000, 1024), (16, 200, 30000)])
def test_product(check, M, N, K, group, dtype):
    A, codes, sc, _, _ = case(M, N, K, group, dtype, M + N + K)
    packed, scales = torch.from_numpy(pack(codes)).cuda(), pack_scales(sc).cuda()
    for lda, shift in ((K, 0), (K + 3, 1)):
        dA = torch.full((M * lda + shift,), float("nan"), dtype=TORCH[dtype], device="cuda")
        torch.as_strided(dA, (M, K), (lda, 1), shift).copy_(A)

        def call(nm):
            out = torch.full((M, N + 2), 7.0, dtype=torch.float32 if dtype == BF16_F32OUT else TORCH[dtype], device="cuda")
            nm.nm_matmul_w4(dA[shift:], packed, scales, out, M, N, K, group, dtype, lda=lda, ldc=N + 2)
            return [out]
        same_in_both(call, check)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("layout", [ROW, COL])
@pytest.mark.parametrize("group", [32, 128, 256])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 64), (65, 255), (70, 257), (200, 600), (128, 1024)])
def test_packing(check, N, K, group, layout, dtype):
    B = torch.randn(N * K, generator=torch.Generator().manual_seed(N)).to(TORCH[dtype]).cuda()

    def call(nm):
        packed = torch.zeros(nm.nm_w4_packed_bytes(N, K), dtype=torch.uint8, device="cuda")
        scales = torch.zeros(nm.nm_w4_scale_count(N, K, group), dtype=TORCH[dtype], device="cuda")
        back = torch.zeros_like(B)
        nm.nm_w4_quantize(B, packed, scales, N, K, group, dtype, layout)
        nm.nm_w4_dequantize(packed, scales, back, N, K, group, dtype, layout)
        return [packed, scales, back]
    same_in_both(call, check)


@pytest.mark.parametrize("normed,rotated", [(True, True), (False, False)])
@pytest.mark.parametrize("T,kv,rope,stride", [(1, 512, 64, 576), (5, 512, 64, 2112), (33, 512, 64, 576), (3, 16, 8, 24), (7, 528, 0, 528), (4, 1024, 256, 1288), (9, 272, 24, 296)])
def test_cache(check, T, kv, rope, stride, normed, rotated):
    x, gamma, cs = rows_in(T, kv, rope, T + kv)
    wide = torch.full((T * stride,), float("nan"), dtype=torch.bfloat16, device="cuda")
    torch.as_strided(wide, (T, kv + rope), (stride, 1)).copy_(x)
    n = 2 * T + 3
    order = torch.from_numpy(np.random.default_rng(T).permutation(n)[:T].astype(np.int64))
    order[T // 2] = -1
    order[0] = n if T > 4 else n - 1
    order, gamma, cs = order.cuda(), gamma.cuda() if normed else None, cs.cuda() if rotated and rope else None

    def call(nm):
        cache = torch.zeros(n, nm.nm_mla_q8_row_bytes(kv, rope), dtype=torch.uint8, device="cuda")
        out = torch.zeros(T, stride, dtype=torch.bfloat16, device="cuda")
        plain = torch.zeros(n, kv + rope, dtype=torch.bfloat16, device="cuda")
        nm.nm_mla_cache_write_q8(wide, gamma, cs, order, cache, n, T, kv, rope, 1e-6, ckr_stride=stride)
        nm.nm_mla_cache_read_q8(cache, n, order, out, T, kv, rope, out_stride=stride)
        nm.nm_mla_cache_read_q8(cache, n, None, plain, n, kv, rope)
        return [cache, out, plain]
    same_in_both(call, check)


@pytest.mark.parametrize("T,H,prefix,lens", [(1, 1, 0, [1]), (1, 16, 0, [97]), (2, 24, 0, [0, 300]), (3, 128, 97, [0, 1, 200]), (5, 24, 200, [3, 0, 96, 97, 11]),
                                             (4, 33, 1000, [0, 0, 0, 0]), (2, 128, 0, [0, 0]), (64, 2, 500, [t % 5 for t in range(64)]), (11, 110, 300, [40 * t for t in range(11)])])
def test_attention(check, T, H, prefix, lens):
    Q, pre, own = batch_case(T, H, prefix, lens, T + H)
    step = max(max(lens), 1)
    cache = torch.zeros(T, step, REC, dtype=torch.uint8)
    for t, o in enumerate(own):
        cache[t, :len(o)] = o
    Q, pre, cache = Q.cuda(), pre.cuda(), cache.cuda()

    def call(nm):
        o16, o32 = (torch.full((T, H, KV), 7.0, dtype=d, device="cuda") for d in (torch.bfloat16, torch.float32))
        lse = torch.full((T, H), 7.0, device="cuda")
        ws = torch.full((nm.nm_mla_attention_q8_workspace_bytes(T, H),), 0xFF, dtype=torch.uint8, device="cuda")
        nm.nm_mla_attention_q8(Q, pre, prefix, cache, step * REC, lens, o16, o32, lse, H, KV, ROPE, SCALE, ws)
        return [o16, o32, lse]
    same_in_both(call, check)
