"""One workspace through calls of every kind and size: a prompt through the experts, decode steps, products, narrow products.  No call finds anything of the one before it."""
import pytest
import torch

import test_matmul_act as act_tests
import test_moe_ffn as moe_tests
from ffn_util import BF16, COL, F16, ROW, SILU, TORCH, assert_within, product64, randn, rounded, stored

pytestmark = pytest.mark.gpu
# 40 experts of 1032 x 520: a tile of 128 rows each for 300 tokens, so 200 items of the first product and 360 of the second, more than there are multiprocessors.
D, INTER, E, K = 1032, 520, 40, 6


class Program:
    """What keeps one workspace: layers of a model, a call at a time.  Everything but the counters is poisoned before each call, and the counters are zero after it."""

    def __init__(self, nm, dtype):
        self.nm, self.dtype = nm, dtype
        self.ws = nm.new_workspace(160 << 20)
        self.base = moe_tests.make(1, D, INTER, E, K, dtype, 1)
        self.dev = moe_tests.place(self.base, COL)
        self.A, self.W, self.b, self.r = act_tests.make(5, 21000, 512, dtype, False, 2)       # 83 items in two parts: 166 chunks
        self.dact = self.A.cuda(), stored(self.W, COL).cuda(), self.b.cuda(), self.r.cuda()
        self.N = randn(1024, 520, seed=3, scale=1024 ** -0.5, dtype=torch.bfloat16), randn(3, 1024, seed=4, dtype=torch.bfloat16)
        self.dN = tuple(t.cuda() for t in self.N)

    def poison(self):
        self.ws[self.nm.WS_COUNTER_BYTES:].fill_(0xFF)

    def counters_are_zero(self):
        self.nm.nm_check_status()
        assert int(self.ws[:self.nm.WS_COUNTER_BYTES].count_nonzero()) == 0, "the counters are left as they were found"

    def tokens(self, T, seed):
        g = torch.Generator().manual_seed(seed)
        return dict(self.base, x=randn(T, D, seed=seed, dtype=TORCH[self.dtype]), residual=randn(T, D, seed=seed + 1, dtype=TORCH[self.dtype]),
                    experts=torch.rand(T, E, generator=g).topk(K, 1).indices.to(torch.int32), weights=torch.softmax(torch.randn(T, K, generator=g), 1))

    def experts(self, T, parts, seed):
        nm, c = self.nm, self.tokens(T, seed)
        dev = dict(self.dev, **{n: c[n].cuda() for n in ("x", "residual", "experts", "weights")})
        out = torch.full((T, D), 77.0, dtype=TORCH[self.dtype], device="cuda")
        self.poison()
        nm.nm_debug_set_ffn_cut(parts)
        moe_tests.call(nm, c, SILU, True, self.dtype, COL, out, self.ws, dev=dev)
        nm.nm_debug_set_ffn_cut(0)
        self.counters_are_zero()
        assert_within(out, *moe_tests.expected(c, SILU, True, self.dtype), f"{T} tokens in {parts} parts")

    def product(self, parts):
        nm = self.nm
        A, W, b, r = self.dact
        out = torch.full((5, 21000), 77.0, dtype=TORCH[self.dtype], device="cuda")
        self.poison()
        nm.nm_debug_set_ffn_cut(parts)
        nm.nm_matmul_act(A, W, out, 5, 21000, 512, SILU, self.dtype, COL, self.ws, bias=b, residual=r)
        nm.nm_debug_set_ffn_cut(0)
        self.counters_are_zero()
        assert_within(out, *act_tests.expected(self.A, self.W, self.b, self.r, SILU, False, self.dtype), f"product in {parts} parts")

    def narrow(self):
        """A narrow product whose k-splits count their arrivals in the same words."""
        nm = self.nm
        B, A = self.dN
        out = torch.full((3, 520), 77.0, dtype=torch.bfloat16, device="cuda")
        self.poison()
        nm.nm_debug_set_kernel(0, 0)
        nm.nm_debug_set_plan(0, 4)
        nm.nm_matmul_ws(A, B, out, 3, 520, 1024, BF16, ROW, self.ws)
        nm.nm_debug_set_plan(0, 0)
        nm.nm_debug_set_kernel(-1, 0)
        self.counters_are_zero()
        z, t = product64(self.N[1].double(), self.N[0].double())
        assert_within(out, z, rounded(z, t, BF16), "narrow product")


@pytest.fixture
def nm():
    import paper_2609_16009_b200 as nm
    yield nm
    nm.nm_debug_set_ffn_cut(0)
    nm.nm_debug_set_plan(0, 0)
    nm.nm_debug_set_kernel(-1, 0)


FOLLOWERS = {"one token": lambda p: p.experts(1, 5, 20), "a narrow batch": lambda p: p.experts(16, 0, 30), "a product": lambda p: p.product(2), "a narrow product": lambda p: p.narrow(),
             "another prompt": lambda p: p.experts(130, 0, 40)}


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("parts", [0, 1, 2])
@pytest.mark.parametrize("follower", list(FOLLOWERS))
def test_a_prompt_and_what_follows_it(nm, follower, parts, dtype):
    p = Program(nm, dtype)
    p.experts(300, parts, 10)
    FOLLOWERS[follower](p)
    p.experts(300, parts, 11)
    FOLLOWERS[follower](p)


@pytest.mark.parametrize("programmatic", [False, True])
def test_decode_steps_between_prompts_without_a_pause(nm, programmatic):
    """The same without looking at the counters in between: every call is under way when the next is made."""
    p = Program(nm, BF16)
    calls = [(300, 0), (1, 0), (16, 0), (300, 2), (1, 5), (300, 1), (16, 0)]
    cases = [p.tokens(T, 50 + i) for i, (T, _) in enumerate(calls)]
    devs = [dict(p.dev, **{n: c[n].cuda() for n in ("x", "residual", "experts", "weights")}) for c in cases]
    outs = [torch.full((T, D), 77.0, dtype=torch.bfloat16, device="cuda") for T, _ in calls]
    p.poison()
    torch.cuda.synchronize()
    nm.nm_set_programmatic_launch(programmatic)
    try:
        for c, dev, out, (T, parts) in zip(cases, devs, outs, calls):
            nm.nm_debug_set_ffn_cut(parts)
            moe_tests.call(nm, c, SILU, True, BF16, COL, out, p.ws, dev=dev)
    finally:
        nm.nm_set_programmatic_launch(False)
        nm.nm_debug_set_ffn_cut(0)
    p.counters_are_zero()
    for c, out, (T, _) in zip(cases, outs, calls):
        assert_within(out, *moe_tests.expected(c, SILU, True, BF16), f"{T} tokens")


def test_a_decode_step_captured_before_a_prompt(nm):
    """A graph of one token's step, replayed behind a prompt that went through its workspace in between."""
    p = Program(nm, BF16)
    c = p.tokens(1, 60)
    dev = dict(p.dev, **{n: c[n].cuda() for n in ("x", "residual", "experts", "weights")})
    out = torch.zeros(1, D, dtype=torch.bfloat16, device="cuda")
    nm.nm_debug_set_ffn_cut(5)
    moe_tests.call(nm, c, SILU, True, BF16, COL, out, p.ws, dev=dev)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe_tests.call(nm, c, SILU, True, BF16, COL, out, p.ws, dev=dev)
    nm.nm_debug_set_ffn_cut(0)
    for i in range(2):
        p.experts(300, 0, 70 + i)
        p.poison()
        out.fill_(77.0)
        graph.replay()
        p.counters_are_zero()
        assert_within(out, *moe_tests.expected(c, SILU, True, BF16), "replayed")
