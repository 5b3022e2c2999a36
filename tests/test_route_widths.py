"""Routing at the borders of the numbers of experts that its kernels are made for, and at numbers of choices around those that all fit a warp's candidates."""
import pytest
import torch

from test_route import BF16, F32, SIGMOID, SOFTMAX, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E", [63, 64, 65, 128, 129, 160, 191, 192, 193, 256, 257, 320, 321, 384, 385, 447, 448, 449, 512, 513, 640, 767, 768, 769, 1023, 1024])
def test_numbers_of_experts(E):
    g = torch.Generator().manual_seed(E)
    x, bias = 2 * torch.randn(37, E, generator=g), 0.3 * torch.randn(E, generator=g)
    for k in (1, 8, 31):
        check(x, None, k, F32, SOFTMAX)
        check(x, bias, k, F32, SIGMOID, renorm=False)
        check(x.bfloat16(), None, k, BF16, SIGMOID)
    for groups in (2, 3, 8):
        if E % groups == 0:
            check(x, bias, 8, F32, SIGMOID, groups, 2 if groups > 2 else 1, 2)
            check(x, None, 8, F32, SOFTMAX, groups, 2 if groups > 2 else 1, 1, renorm=False)


@pytest.mark.parametrize("k", [15, 16, 17, 20, 23, 24, 28, 32])
@pytest.mark.parametrize("E", [40, 128, 256, 512])
def test_numbers_of_choices(E, k):
    """From about twenty on, more keys than lanes pass the bound of the first selection for some tokens, from 24 on for nearly all."""
    g = torch.Generator().manual_seed(E + k)
    x, bias = 2 * torch.randn(200, E, generator=g), 0.3 * torch.randn(E, generator=g)
    check(x, None, k, F32, SOFTMAX)
    check(x, bias, k, F32, SIGMOID, scale=1.5)
    check(x.round(), None, k, F32, SOFTMAX)                        # many equal keys
