"""The feed-forward products in the debug build with threads held up at named places: for some microseconds, and nothing changes; for longer than the others wait,
and they give up, what is under way ends, and the call after the next initialisation of the workspace is right."""
import ctypes as C
import time

import pytest
import torch

import test_moe_ffn as moe_tests
from ffn_util import BF16, COL, SILU, stored
from test_bounds_check_ffn_gpu import NAMES
from test_matmul_act import make as make_act

PLACES = {"copy": 1, "passing on": 2, "products": 3, "giving back": 4, "counting": 5, "taking": 6}


@pytest.fixture(scope="module")
def check():
    import paper_2609_16009_b200 as nm
    from paper_2609_16009_b200 import build
    lib = C.CDLL(build.build(check=True))
    for name in NAMES:
        getattr(lib, name).argtypes = getattr(nm._lib, name).argtypes
        getattr(lib, name).restype = getattr(nm._lib, name).restype
    lib.nm_debug_set_ffn_pause.argtypes = [C.c_int, C.c_uint]
    return lib


def test_the_pause_belongs_to_the_debug_build(check):
    import paper_2609_16009_b200 as nm
    assert nm._lib.nm_debug_set_ffn_pause(1, 1000) == -2
    for bad in ((-1, 0), (7, 0), (1, 2_000_000_001)):
        assert check.nm_debug_set_ffn_pause(*bad) == -1, bad


class Product:
    """352 chunks of 16 steps, two an item: longer than the ring, more than one for most CTAs, all of them joined."""
    M, N, K = 16, 45000, 2048

    def __init__(self):
        import paper_2609_16009_b200 as nm
        A, W, b, r = make_act(self.M, self.N, self.K, BF16, False, 5)
        self.A, self.W, self.b, self.r = A.cuda(), stored(W, COL).cuda(), b.cuda(), r.cuda()
        self.ws = nm.new_workspace(nm.nm_matmul_act_workspace_bytes(self.M, self.N, self.K))

    def call(self, lib, where=0, ns=0):
        import paper_2609_16009_b200 as nm
        out = torch.zeros(self.M, self.N, dtype=torch.bfloat16, device="cuda")
        normal, nm._lib = nm._lib, lib
        try:
            nm.nm_debug_set_ffn_cut(2)
            if where:
                assert lib.nm_debug_set_ffn_pause(where, ns) == 0
            nm.nm_matmul_act(self.A, self.W, out, self.M, self.N, self.K, SILU, BF16, COL, self.ws, bias=self.b, residual=self.r)
            torch.cuda.synchronize()
        finally:
            if where:
                assert lib.nm_debug_set_ffn_pause(0, 0) == 0
            nm.nm_debug_set_ffn_cut(0)
            nm._lib = normal
        return out


@pytest.fixture(scope="module")
def product():
    return Product()


@pytest.mark.gpu
@pytest.mark.parametrize("where", list(PLACES))
def test_threads_held_up_change_nothing(check, product, where):
    import paper_2609_16009_b200 as nm
    want = product.call(nm._lib)
    got = product.call(check, PLACES[where], 20_000)
    assert check.nm_check_status(None) == 0, "a wait ran out"
    assert torch.equal(want.view(torch.int16), got.view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("where", list(PLACES))
def test_experts_with_threads_held_up(check, where):
    import paper_2609_16009_b200 as nm
    c = moe_tests.make(20, 1024, 520, 40, 6, BF16, 9)
    dev, ws, outs = moe_tests.place(c, COL), moe_tests.workspace(nm, c, BF16), []
    normal = nm._lib
    for lib, ns in ((normal, 0), (check, 20_000)):
        out = torch.zeros(20, 1024, dtype=torch.bfloat16, device="cuda")
        nm._lib = lib
        try:
            nm.nm_debug_set_ffn_cut(3)
            if ns:
                assert lib.nm_debug_set_ffn_pause(PLACES[where], ns) == 0
            moe_tests.call(nm, c, SILU, True, BF16, COL, out, ws, dev=dev)
            torch.cuda.synchronize()
        finally:
            if ns:
                assert lib.nm_debug_set_ffn_pause(0, 0) == 0
            nm.nm_debug_set_ffn_cut(0)
            nm._lib = normal
        outs.append(out)
    assert check.nm_check_status(None) == 0
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("where", ["copy", "passing on", "products", "giving back"])
def test_an_expired_wait_ends_in_order(check, product, where):
    import paper_2609_16009_b200 as nm
    want = product.call(nm._lib)
    product.call(check)                                            # (its code is loaded)
    assert check.nm_check_status(None) == 0
    t0 = time.monotonic()
    product.call(check, PLACES[where], 1_300_000_000)
    took = time.monotonic() - t0
    print("took %.3f s" % took)
    assert 1.0 <= took < 10
    assert check.nm_check_status(None) == -6 and check.nm_check_status(None) == 0
    nm.nm_workspace_init(product.ws)
    got = product.call(check)
    assert check.nm_check_status(None) == 0
    assert torch.equal(want.view(torch.int16), got.view(torch.int16))
