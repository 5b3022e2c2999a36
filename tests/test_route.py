"""Routing of tokens to experts (nm_moe_route) against a plain implementation in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

F32, BF16, F16 = 0, 1, 3
TORCH = {F32: torch.float32, BF16: torch.bfloat16, F16: torch.float16}
SOFTMAX, SIGMOID = 0, 1


def reference(x, bias, k, score, groups=1, keep=1, best=1, renorm=True, scale=1.0):
    """x: fp64 logits [T][E] -> (experts, weights), by the definition, NaN and infinities included."""
    x = np.where(np.isnan(x), -np.inf, x)
    T, E = x.shape
    with np.errstate(all="ignore"):
        if score == SOFTMAX:
            m = x.max(1, keepdims=True)
            e = np.where(np.isposinf(m), np.isposinf(x).astype(float), np.where(np.isneginf(x), 0.0, np.exp(x - np.where(np.isneginf(m), 0.0, m))))
            total = e.sum(1, keepdims=True)
            s = e / np.where(total == 0, 1.0, total)
        else:
            s = 1 / (1 + np.exp(-x))
        key = s if bias is None else s + bias
        key = np.where(np.isnan(key), -np.inf, key)
        allowed = np.ones((T, E), dtype=bool)
        if groups > 1:
            by = key.reshape(T, groups, E // groups)
            of = np.sort(by, 2)[:, :, ::-1][:, :, :best].sum(2)
            of = np.where(np.isnan(of), -np.inf, of)
            order = np.argsort(-of, axis=1, kind="stable")[:, :keep]
            kept = np.zeros((T, groups), dtype=bool)
            np.put_along_axis(kept, order, True, 1)
            allowed = np.repeat(kept, E // groups, axis=1)
        # what may not be chosen comes behind everything else, minus infinity included
        chosen = np.stack([np.lexsort((np.arange(E), -key[t], ~allowed[t]))[:k] for t in range(T)])
        w = np.take_along_axis(s, chosen, 1)
        if renorm:
            total = w.sum(1, keepdims=True)
            w = np.where(total > 0, w / np.where(total > 0, total, 1.0), 0.0)
    return chosen, w * float(np.float32(scale))                                      # the scale is an fp32 argument


def run(x, bias, k, dtype, score, groups=1, keep=1, best=1, renorm=True, scale=1.0, ld=None):
    import paper_2609_16009_b200 as nm
    T, E = x.shape
    ld = ld or E
    wide = torch.full((T, ld), float("inf"), dtype=TORCH[dtype], device="cuda")      # what lies between the rows would win if it were read
    wide[:, :E] = x.cuda()
    b = None if bias is None else bias.cuda()
    experts = torch.full((T + 2, k), -7, dtype=torch.int32, device="cuda")
    weights = torch.full((T + 2, k), -7.0, device="cuda")
    nm.nm_moe_route(wide, b, experts[1:], weights[1:], T, E, k, dtype, score, groups=groups, keep_groups=keep, group_best=best, renormalise=renorm, scale=scale, ld_logits=ld)
    e, w = experts.cpu().numpy(), weights.cpu().double().numpy()
    assert (e[0] == -7).all() and (e[-1] == -7).all() and (w[0] == -7).all() and (w[-1] == -7).all(), "written outside the outputs"
    return e[1:-1], w[1:-1]


def check(x, bias, k, dtype, score, groups=1, keep=1, best=1, renorm=True, scale=1.0, ld=None):
    e, w = run(x, bias, k, dtype, score, groups, keep, best, renorm, scale, ld)
    re, rw = reference(x.double().numpy(), None if bias is None else bias.double().numpy(), k, score, groups, keep, best, renorm, scale)
    assert np.array_equal(e, re)
    # fp64 throughout (a few steps of 2^-53), one rounding to fp32: half a step, and fp32's absolute step below its normal range
    assert np.all(np.abs(w - rw) <= 1.0001 * 2.0 ** -24 * np.abs(rw) + 2.0 ** -150)


@pytest.mark.gpu
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 2, 2), (3, 31, 5), (4, 32, 32), (5, 33, 7), (1, 64, 6), (7, 65, 1), (16, 97, 4), (130, 128, 8), (33, 129, 9), (9, 256, 8), (2, 257, 32),
                                   (6, 512, 12), (3, 1000, 20), (2, 1024, 32), (5003, 40, 3)])
def test_top_k(T, E, k, dtype, score):
    g = torch.Generator().manual_seed(T * E + k)
    x = (2 * torch.randn(T, E, generator=g)).to(TORCH[dtype])
    check(x, None, k, dtype, score)
    check(x, 0.3 * torch.randn(E, generator=g), k, dtype, score, renorm=False, scale=2.5, ld=E + 3)


@pytest.mark.gpu
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("T,E,groups,keep,k", [(1, 4, 2, 1, 2), (3, 64, 8, 3, 6), (16, 160, 8, 3, 6), (17, 320, 10, 4, 8), (5, 96, 32, 5, 4), (4, 512, 4, 4, 8), (2, 1024, 32, 2, 32),
                                               (9, 30, 15, 7, 14), (300, 60, 4, 2, 11)])
def test_groups(T, E, groups, keep, k, best):
    g = torch.Generator().manual_seed(T * E + k)
    x, bias = torch.randn(T, E, generator=g), 0.2 * torch.randn(E, generator=g)
    check(x, bias, k, F32, SIGMOID, groups, keep, best, scale=1.7)
    check(x, None, k, F32, SOFTMAX, groups, keep, best, renorm=False)
    check(x, bias - 5, k, F32, SIGMOID, groups, keep, best)                          # every key negative: what may not be chosen is still below


@pytest.mark.gpu
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("groups,keep,best", [(1, 1, 1), (8, 3, 1), (8, 3, 2)])
def test_ties_go_to_the_lowest_index(score, groups, keep, best):
    g = torch.Generator().manual_seed(5)
    x = torch.randint(0, 3, (200, 64), generator=g).float()
    check(x, None, 6, F32, score, groups, keep, best)
    check(x, torch.randint(0, 2, (64,), generator=g).float(), 6, F32, score, groups, keep, best)
    check(torch.zeros(3, 64), None, 6, F32, score, groups, keep, best)
    check(torch.full((3, 64), 200.0), None, 6, F32, score, groups, keep, best)           # a saturated sigmoid
    check(torch.tensor([[0.0, -0.0] * 32]), None, 6, F32, score, groups, keep, best)
    check(torch.tensor([[-1.0, 1.0] * 32]), torch.tensor([0.0, -0.0] * 32), 6, F32, score, groups, keep, best)


@pytest.mark.gpu
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("groups,keep,best", [(1, 1, 1), (4, 2, 2)])
def test_infinities_and_nan(score, groups, keep, best):
    inf, nan = float("inf"), float("nan")
    g = torch.Generator().manual_seed(6)
    x = torch.randn(12, 40, generator=g)
    x[0] = -inf                                   # every expert masked
    x[1, 5:] = -inf                               # fewer left than are chosen
    x[2] = nan
    x[3, ::2] = nan
    x[4, 7] = inf
    x[5, [3, 9, 30]] = inf
    x[6, 0], x[6, 1] = inf, nan
    x[7] = torch.finfo(torch.float32).min         # masked by the lowest value
    x[8, 4:] = torch.finfo(torch.float32).min
    x[9] = torch.finfo(torch.float32).max
    x[10] *= 1e30
    for renorm in (True, False):
        check(x, None, 6, F32, score, groups, keep, best, renorm)
        check(x, torch.randn(40, generator=g), 6, F32, score, groups, keep, best, renorm)
    bias = torch.zeros(40)
    bias[::3], bias[1::3] = -inf, nan
    check(x, bias, 15, F32, score, groups, keep, 1)


@pytest.mark.gpu
def test_scores_that_fp32_cannot_tell_apart():
    """Keys that differ by less than a step of fp32 keep their order."""
    x = torch.zeros(4, 64)
    bias = torch.zeros(64)
    x[0, 50], x[0, 20] = 1e-7, 5e-8
    x[1] = 30.0 + torch.arange(64) * 1e-5          # sigmoid within 1e-13 of 1
    x[2] = -60.0 - torch.arange(64) * 1e-5
    bias[10] = 2.0 ** -30
    for score in (SOFTMAX, SIGMOID):
        check(x, bias, 8, F32, score)
        check(x, None, 8, F32, score, 8, 2, 2)


@pytest.mark.gpu
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("groups,keep,best", [(1, 1, 1), (8, 3, 1), (8, 3, 2), (16, 5, 2)])
def test_keys_near_each_other(score, groups, keep, best):
    """Logits and biases a few steps of fp32 apart, or less than fp64 scores tell apart (ties then), from far below to far above."""
    g = torch.Generator().manual_seed(8)
    pick = torch.randint(-3, 4, (160, 64), generator=g).float()
    base = torch.tensor([0.0, 1e-30, 1e-8, 0.37, -5.0, 7.99, 9.0, 40.0, -40.0, -300.0, -650.0, -720.0, -745.0, 700.0, 1e5, -1e5]).repeat(10)[:, None]
    x = base + pick * torch.where(base == 0, torch.tensor(1e-32), torch.finfo(torch.float32).eps * base.abs())
    x[::5, ::7] = float("-inf")
    for bias in (None, torch.zeros(64), 1e-7 * torch.randint(-2, 3, (64,), generator=g).float(), 1000 + 1e-4 * torch.randint(-2, 3, (64,), generator=g).float(),
                 0.5 * torch.randn(64, generator=g)):
        check(x, bias, 6, F32, score, groups, keep, best)
        check(x + torch.randn(160, 64, generator=g), bias, 6, F32, score, groups, keep, best, renorm=False)


@pytest.mark.gpu
def test_equal_calls_and_programmatic_launch_give_equal_bits():
    import paper_2609_16009_b200 as nm
    x = torch.randn(77, 200, generator=torch.Generator().manual_seed(1))
    first = run(x, None, 5, F32, SOFTMAX)
    nm.nm_set_programmatic_launch(True)
    try:
        second = run(x, None, 5, F32, SOFTMAX)
    finally:
        nm.nm_set_programmatic_launch(False)
    assert all(np.array_equal(a, b) for a, b in zip(first, second))


@pytest.fixture(scope="module")
def lib():
    from paper_2609_16009_b200 import build
    return ctypes.CDLL(build.build())


def test_refusals_need_no_device(lib):
    vp, i, l, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_long, ctypes.c_float
    lib.nm_moe_route.argtypes = [vp, l, vp, vp, vp] + [i] * 9 + [f, vp]

    def status(logits=256, ld=64, bias=None, experts=512, weights=1024, T=4, E=64, k=6, dtype=F32, score=0, groups=1, keep=1, best=1):
        return lib.nm_moe_route(logits, ld, bias, experts, weights, T, E, k, dtype, score, groups, keep, best, 1, 1.0, None)
    assert status(logits=None) == status(experts=None) == status(weights=None) == -1
    assert status(T=0) == status(E=0) == status(k=0) == status(k=65) == status(ld=63) == -1
    assert status(groups=0) == status(groups=5) == status(groups=8, keep=9) == status(groups=8, keep=0) == status(groups=16, keep=1) == -1
    assert status(best=0) == status(best=3) == -1
    assert status(groups=32, keep=8, best=2, E=32, ld=32) == -1, "no two experts in a group"
    assert status(score=2) == -1
    assert status(E=1025, ld=1025) == status(E=64, k=33) == status(groups=64, keep=8) == -2
    assert status(dtype=2) == status(dtype=7) == -2
    assert status(logits=258) == status(bias=2) == status(experts=514) == status(weights=1026) == -3
    assert status(logits=257, dtype=BF16) == -3
