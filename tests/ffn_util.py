"""Definitions in 64 bits of the feed-forward operators, and how far a correct kernel may be from them."""
import torch

BF16, F16, ROW, COL = 1, 3, 0, 1
TORCH = {BF16: torch.bfloat16, F16: torch.float16}
HALF = {BF16: 2.0 ** -9, F16: 2.0 ** -12}         # half a step, relative to the power of two below the value; the value itself is at most twice that
NONE, RELU, SILU, GELU, GELU_TANH = range(5)
SLOPE = 1.13                                      # no activation is steeper (silu 1.10, gelu 1.129)
TINY = {BF16: 2.0 ** -134, F16: 2.0 ** -25}


def act64(act, x):
    if act == RELU:
        return x.clamp(min=0)
    if act == SILU:
        return x * torch.special.expit(x)
    if act == GELU:
        return x * torch.special.ndtr(x)
    if act == GELU_TANH:
        return x * torch.special.expit(2 * (2 / torch.pi) ** 0.5 * (x + 0.044715 * x ** 3))
    return x


def sum_error(K):
    """An fp32 sum of K exact products, relative to the sum of their magnitudes: the matrix unit adds 16 (or fewer) at a time to a running sum
    and may cut it off, a step of 2^-23 each; up to 152 partial sums (one a multiprocessor, and the epilogue's few) are joined."""
    return (K / 16 + 160) * 2.0 ** -23


def act_error(z):
    """fp32 arithmetic of the activation and the gate: a few steps; the exponent of exp and the square in erfc magnify the rounding of their
    arguments (relative error of exp(x) is x times that of x)."""
    return (8 + 2 * z.abs().clamp(max=100)) * 2.0 ** -23


def product64(x, W, tx=0.0):
    """x [m][k] (fp64, each value off by at most tx) times W [k][n]: the product and the bound on a kernel's error."""
    z = x @ W
    size = x.abs() @ W.abs()
    more = tx @ W.abs() if torch.is_tensor(tx) else 0.0
    return z, sum_error(x.shape[1]) * size + more


def hidden64(x, W, act, gated, bias=None):
    """act(x Wg + bg) o (x Wu + bu) and its bound; W [k][n or 2n]."""
    z, t = product64(x, W)
    if bias is not None:
        z = z + bias
        t = t + 2.0 ** -23 * (z.abs() + bias.abs())
    if gated:
        n = W.shape[1] // 2
        g, u, tg, tu = z[:, :n], z[:, n:], t[:, :n], t[:, n:]
    else:
        g, u, tg, tu = z, torch.ones_like(z), t, torch.zeros_like(z)
    a = act64(act, g)
    ta = SLOPE * tg + (0 if act in (NONE, RELU) else act_error(g) * a.abs())
    return a * u, (ta * u.abs() + a.abs() * tu + ta * tu) + 2.0 ** -23 * (a * u).abs()


def rounded(ref, t, dtype):
    """The bound after one rounding to the 16-bit type."""
    return t + 2 * HALF[dtype] * (ref.abs() + t) + TINY[dtype]


def assert_within(got, ref, tol, what=""):
    err = (got.double().cpu() - ref.cpu()).abs()
    bad = ~(err <= tol.cpu())
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside; worst {(err / tol.cpu().clamp(min=1e-300)).nan_to_num(1e9).max():.3f} of the tolerance"


def randn(*shape, seed, scale=1.0, dtype=torch.float32):
    return (scale * torch.randn(*shape, generator=torch.Generator().manual_seed(seed))).to(dtype)


def stored(W, layout):
    """Logical [..][k][n] as it lies in memory."""
    return W.transpose(-1, -2).contiguous() if layout == COL else W.contiguous()
