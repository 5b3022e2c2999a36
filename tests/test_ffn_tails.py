"""Activations far below zero, where the exponential leaves fp32's range or its inverse does: the values that bf16 and fp32 still hold are not lost.

An activation is fp32: to a few steps of itself, and below fp32's normal range to a few of its steps of 2^-149 there (2^-146 in all: erfc comes with half of one, times up to 8)."""
import math

import pytest
import torch

from ffn_util import BF16, COL, GELU, GELU_TANH, ROW, SILU, assert_within, rounded

pytestmark = pytest.mark.gpu
RANGES = {SILU: (-128.0, -70.0), GELU: (-15.0, -11.0), GELU_TANH: (-11.0, -8.5)}


def values(act):
    """Every bf16 value of the range, and their mirror images."""
    lo, hi = RANGES[act]
    every = torch.arange(2 ** 15, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    v = every[(every.float() >= -hi) & (every.float() <= -lo)]
    return torch.cat([-v, v])


def activation(act, z):
    """The value in 64 bits, to its last digits far below zero too, and what fp32 may be off by: the exponent's own size times a few roundings."""
    if act == GELU:
        a, exponent = 0.5 * z * torch.special.erfc(-math.sqrt(0.5) * z), 0.5 * z * z
    else:
        exponent = z if act == SILU else 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        a = z * torch.special.expit(exponent)
    return a, (8 + 4 * exponent.abs().clamp(max=150)) * 2.0 ** -23 * a.abs() + 2.0 ** -146


def expected(act, g, u):
    a, t = activation(act, g)
    return a * u, rounded(a * u, t * u.abs() + 2.0 ** -23 * (a * u).abs(), BF16)


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("layout", [ROW, COL])
@pytest.mark.parametrize("act", [SILU, GELU, GELU_TANH])
@pytest.mark.parametrize("up", [None, 1.0, 2.0 ** 20, -2.0 ** 100])
def test_a_product_keeps_them(act, layout, up, aligned):
    """The product is one value of B, the gate a constant: what comes out is the activation's."""
    import paper_2609_16009_b200 as nm
    g = values(act)
    N, gated = len(g), up is not None
    W = torch.zeros(8, N * (2 if gated else 1), dtype=torch.bfloat16)
    W[0, :N] = g
    if gated:
        W[1, N:] = up
    flat = torch.zeros(W.numel() + 1, dtype=torch.bfloat16, device="cuda")
    dW = flat[:-1] if aligned else flat[1:]
    dW.copy_((W.T if layout == COL else W).reshape(-1))
    A = torch.zeros(3, 8, dtype=torch.bfloat16)
    A[:, :2] = 1
    C = torch.full((3, N), 77.0, dtype=torch.bfloat16, device="cuda")
    nm.nm_matmul_act(A.cuda(), dW, C, 3, N, 8, act, BF16, layout, nm.new_workspace(nm.nm_matmul_act_workspace_bytes(3, N, 8, gated)), gated=gated)
    ref, tol = expected(act, g.double(), torch.full((N,), 1.0 if up is None else up, dtype=torch.float64))
    assert_within(C, ref.expand(3, N), tol.expand(3, N))


@pytest.mark.parametrize("act", [SILU, GELU_TANH])
def test_an_expert_keeps_them(act):
    """The same as hidden values: one goes out alone each time, in the 16 bits that are kept of it."""
    import paper_2609_16009_b200 as nm
    g = values(act)
    inter = len(g) // 8 * 8
    g = g[:inter]
    up, down = torch.zeros(1, 2 * inter, 8, dtype=torch.bfloat16), torch.zeros(1, inter, inter, dtype=torch.bfloat16)
    up[0, :inter, 0], up[0, inter:, 1] = g, 2.0 ** 100
    down[0].fill_diagonal_(1.0)
    d = max(8, inter)
    wide = torch.zeros(1, 2 * inter, d, dtype=torch.bfloat16)
    wide[:, :, :8] = up
    x = torch.zeros(2, d, dtype=torch.bfloat16)
    x[:, :2] = 1
    y = torch.full((2, d), 77.0, dtype=torch.bfloat16, device="cuda")
    nm.nm_moe_ffn(x.cuda(), torch.zeros(2, 1, dtype=torch.int32, device="cuda"), None, wide.cuda(), down.cuda(), y, 2, d, inter, 1, 1, act, BF16, COL,
                  nm.new_workspace(nm.nm_moe_ffn_workspace_bytes(2, d, inter, 1, 1)))
    ref, tol = expected(act, g.double(), torch.full((inter,), 2.0 ** 100, dtype=torch.float64))
    assert_within(y, ref.expand(2, inter), (tol + 2.0 ** -16 * ref.abs()).expand(2, inter))


@pytest.mark.parametrize("act", [SILU, GELU, GELU_TANH])
def test_the_ends(act):
    """Zero, the largest values and infinities: nothing but minus infinity (0 times infinity) gives a NaN."""
    import paper_2609_16009_b200 as nm
    big = torch.finfo(torch.bfloat16).max
    g = torch.tensor([0.0, 1.0, -1.0, big, -big, float("inf"), float("-inf"), float("nan"), 1e13, -1e13, 1e20, -1e20, 2.0 ** -133, -2.0 ** -133, 88.0, -300.0], dtype=torch.bfloat16)
    C = torch.full((1, 16), 77.0, dtype=torch.bfloat16, device="cuda")
    W = torch.zeros(16, 8, dtype=torch.bfloat16)
    nm.nm_matmul_act(torch.zeros(1, 8, dtype=torch.bfloat16, device="cuda"), W.cuda(), C, 1, 16, 8, act, BF16, COL, nm.new_workspace(nm.nm_matmul_act_workspace_bytes(1, 16, 8)), bias=g.cuda())
    got = C[0].cpu().double()
    assert got[5] == float("inf") and got[7].isnan() and got[6].isnan()
    keep = torch.tensor([i for i in range(16) if i not in (5, 6, 7)])
    ref, tol = activation(act, g.double()[keep])
    assert_within(got[keep], ref, rounded(ref, tol, BF16))
