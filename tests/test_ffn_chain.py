"""Routing and experts behind each other many times with programmatic launches, through one buffer of choices that every step writes anew: each step computes with its own."""
import pytest
import torch

import test_moe_ffn as moe_tests
from ffn_util import BF16, COL, F16, SILU, TORCH, assert_within, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T", [1, 16, 40])
def test_choices_written_anew_every_step(T, dtype, captured):
    import paper_2609_16009_b200 as nm
    d, inter, E, k, steps = 1024, 264, 24, 4, 40
    c = moe_tests.make(T, d, inter, E, k, dtype, T)
    dev, ws = moe_tests.place(c, COL), moe_tests.workspace(nm, c, dtype)
    logits = randn(steps, T, E, seed=T + 1).cuda()
    want = []
    for programmatic in (False, True):
        nm.nm_set_programmatic_launch(programmatic)
        try:
            outs, chosen = torch.zeros(steps, T, d, dtype=TORCH[dtype], device="cuda"), torch.zeros(steps, T, k, dtype=torch.int32, device="cuda")

            def steps_():
                for i in range(steps):
                    nm.nm_moe_route(logits[i], None, dev["experts"], dev["weights"], T, E, k, nm.F32)
                    moe_tests.call(nm, c, SILU, True, dtype, COL, outs[i], ws, dev=dev)
            if captured:
                dev["experts"].fill_(-1)
                s = torch.cuda.Stream()
                with torch.cuda.stream(s):                         # (everything is loaded before the capture)
                    steps_()
                torch.cuda.synchronize()
                outs.zero_()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    steps_()
                for _ in range(3):
                    graph.replay()
            else:
                steps_()
            torch.cuda.synchronize()
        finally:
            nm.nm_set_programmatic_launch(False)
        nm.nm_check_status()
        want.append(outs)
    assert torch.equal(want[0].view(torch.int16), want[1].view(torch.int16))
    for i in (0, 1, steps - 1):
        nm.nm_moe_route(logits[i], None, chosen[i], dev["weights"], T, E, k, nm.F32)
        one = dict(c, experts=chosen[i].cpu(), weights=dev["weights"].cpu())
        assert_within(want[1][i], *moe_tests.expected(one, SILU, True, dtype), f"step {i}")
