"""The order in which the warps of the quantised attention tell each other things.

On the CPU: a model of one pair of CTAs' control flow - the issuing warp, the matrix unit, the two threads of a query row - walked through every
interleaving.  A wait by parity passes when the phases completed and the phase waited for differ in their last bit, as the hardware's does.  The
model is told how many buffers and barriers there are, so that the forms that depend on the warps' pace show as such.

On the GPU: the debug build holds one warp up at a named place, many times longer than a tile takes; the bits have to be those of the normal build."""
import ctypes as C
import time

import pytest
import torch

from test_attention_q8 import KV, REC, ROPE, SCALE, case


# ---- the model ------------------------------------------------------------------------------------------------------------

def programs(items, rescale, pair_buffers):
    """The operations of the issuing warp and of a row's two threads, in program order.  items: tiles of each item; rescale: whether a thread waits
    for the P * V of the tile before, as it does when a maximum grows."""
    issue, rows, g0 = [], ([], []), 0
    for i, n in enumerate(items):
        issue += [("wait", "q", i), ("S", g0)]
        for t in range(n):
            issue += ([("S", g0 + t + 1)] if t + 1 < n else []) + [("wait", "p", g0 + t), ("PV", g0 + t)]
        for own in (0, 1):
            r = rows[own]
            r += [("tell", "q", i), ("meet", f"table {i}")]
            for t in range(n):
                g = g0 + t
                r += [("wait", "s", g), ("write", t % pair_buffers, g), ("meet", f"tile {g}"), ("read", t % pair_buffers, g)]
                if t and rescale[own]:
                    r.append(("wait", "pv", g - 1))
                r.append(("tell", "p", g))
            last = g0 + n - 1
            r += ([("wait", "pv", last - 1)] if n > 1 else []) + [("wait", "pv", last)]
            r += [("meet", f"end {i}"), ("write", 0, f"sum {i}"), ("meet", f"sum {i}"), ("read", 0, f"sum {i}")]
        g0 += n
    return [issue, *rows]


def faults(items, rescale=(True, True), pair_buffers=2, pv_barriers=2):
    """Every fault that some interleaving reaches."""
    prog = programs(items, rescale, pair_buffers)
    bars = {"q": 1, "p": 2, "s": 2, "pv": pv_barriers}
    met = [{op[1]: at for at, op in enumerate(p) if op[0] == "meet"} for p in prog]
    work = [op for op in prog[0] if op[0] in ("S", "PV")]          # what the matrix unit does, in this order

    def completed(kind, bar, pc, done):
        """Phases completed of a barrier: two arrivals each of the row's threads, one of the matrix unit."""
        if kind in ("s", "pv"):
            return sum(1 for op in work[:done] if op[0].lower() == kind and op[1] % bars[kind] == bar)
        told = sum(1 for p, at in zip(prog[1:], pc[1:]) for op in p[:at] if op[0] == "tell" and op[1] == kind and op[2] % bars[kind] == bar)
        return told // 2

    found, seen = set(), set()
    todo = [((0, 0, 0), 0, (None,) * 4)]                           # where each program is, what the matrix unit has done, s_pair[buffer][set]
    while todo:
        state = todo.pop()
        if state in seen:
            continue
        seen.add(state)
        pc, done, pair = state
        moves = []
        if done < sum(1 for op in prog[0][:pc[0]] if op[0] in ("S", "PV")):
            moves.append((pc, done + 1, pair))
        for who in range(3):
            if pc[who] == len(prog[who]):
                continue
            op, after, new = prog[who][pc[who]], pc[:who] + (pc[who] + 1,) + pc[who + 1:], pair
            if op[0] == "wait":
                n = bars[op[1]]
                phase, have = op[2] // n, completed(op[1], op[2] % n, pc, done)
                if have % 2 == phase % 2:
                    continue
                if have <= phase:
                    found.add("early")                             # passed for an older phase's sake
                    continue
            elif op[0] == "meet" and pc[3 - who] < met[3 - who][op[1]]:
                continue
            elif op[0] == "write":
                at = 2 * op[1] + who - 1
                new = pair[:at] + (op[2],) + pair[at + 1:]
            elif op[0] == "read" and pair[2 * op[1]:2 * op[1] + 2] != (op[2],) * 2:
                found.add("another tile's")
                continue
            moves.append((after, done, new))
        if not moves and pc != tuple(len(p) for p in prog):
            found.add("stuck")
        todo += moves
    return found


ITEMS = [[1], [2], [3], [5], [1, 3], [2, 1, 2], [4, 4]]
RESCALE = [(False, False), (True, False), (False, True), (True, True)]


@pytest.mark.parametrize("rescale", RESCALE)
@pytest.mark.parametrize("items", ITEMS)
def test_model_maxima_are_those_of_the_tile(items, rescale):
    assert "another tile's" not in faults(items, rescale)


def test_model_sees_the_maximum_of_the_next_tile():
    """With one buffer a thread may write its next maximum before the other one has read this one."""
    assert "another tile's" in faults([2], pair_buffers=1)


@pytest.mark.parametrize("rescale", RESCALE)
@pytest.mark.parametrize("items", ITEMS)
def test_model_every_wait_ends_and_none_too_early(items, rescale):
    assert not faults(items, rescale)


@pytest.mark.parametrize("rescale", RESCALE)
def test_model_sees_a_wait_that_comes_too_late(rescale):
    """With one barrier for the P * V of all tiles a thread that finds the last two through waits for a third."""
    assert faults([2, 1], rescale, pv_barriers=1) == {"stuck"}


# ---- the debug build, a warp held up ---------------------------------------------------------------------------------------

PAUSES = {"maxima": 1, "weights": 2, "product": 3, "copy": 4}


def _declare(lib):
    vp, i, long = C.c_void_p, C.c_int, C.c_long
    lib.nm_mla_attention_q8.argtypes = [vp, long, vp, long, vp, long, vp, vp, vp, vp, i, i, i, i, C.c_float, vp, C.c_size_t, vp]
    lib.nm_debug_set_attention_q8_pause.argtypes = [i, i, C.c_uint]
    lib.nm_check_status.argtypes = [vp]
    return lib


@pytest.fixture(scope="module")
def libs():
    import paper_2609_16009_b200 as nm
    from paper_2609_16009_b200 import build
    normal, check = _declare(C.CDLL(nm.LIB_PATH)), _declare(C.CDLL(build.build(check=True)))
    yield normal, check
    assert check.nm_debug_set_attention_q8_pause(0, 0, 0) == 0
    assert check.nm_check_status(None) == 0 and normal.nm_check_status(None) == 0


class Batch:
    """A batch whose pairs of CTAs walk over several items, the maxima moving from tile to tile."""

    def __init__(self, T=40, H=128, prefix=0, rows=300, seed=5, std=6.0):
        import paper_2609_16009_b200 as nm
        Q, pre, own = case(T, H, prefix, [rows - (7 * (t % 9) if prefix == 0 else 0) for t in range(T)], seed, std)
        self.lens = (C.c_int * T)(*[len(o) for o in own])
        cache = torch.zeros(T, rows, REC, dtype=torch.uint8)
        for t, o in enumerate(own):
            cache[t, :len(o)] = o
        self.T, self.H, self.n_prefix, self.stride = T, H, prefix, rows * REC
        self.Q, self.cache, self.prefix = Q.cuda(), cache.cuda(), pre.cuda()
        self.ws = torch.empty(nm.nm_mla_attention_q8_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")

    def call(self, lib):
        o = torch.full((self.T, self.H, KV), 7.0, device="cuda")
        lse = torch.full((self.T, self.H), 7.0, device="cuda")
        self.ws.fill_(0xFF)
        torch.cuda.synchronize()
        rc = lib.nm_mla_attention_q8(self.Q.data_ptr(), self.H * (KV + ROPE), self.prefix.data_ptr() if self.n_prefix else None, self.n_prefix, self.cache.data_ptr(),
                                     self.stride, self.lens, None, o.data_ptr(), lse.data_ptr(), self.T, self.H, KV, ROPE, SCALE, self.ws.data_ptr(), self.ws.numel(),
                                     None)
        assert rc == 0
        torch.cuda.synchronize()
        return o, lse


@pytest.fixture(scope="module", params=["short", "long"])
def batch(request):
    """Items of one and two tiles; items of 9 and 17, and six of 2, on a pair of CTAs."""
    return Batch() if request.param == "short" else Batch(T=16, prefix=12000, rows=150)


def paused(lib, where, warp, ns, fn):
    assert lib.nm_debug_set_attention_q8_pause(PAUSES[where], warp, ns) == 0
    try:
        return fn()
    finally:
        assert lib.nm_debug_set_attention_q8_pause(0, 0, 0) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("warp", [2, 5, 6, 9])
def test_a_thread_late_to_read_the_maxima_changes_nothing(libs, batch, warp):
    normal, check = libs
    want = batch.call(normal)
    assert torch.isfinite(want[0]).all() and normal.nm_check_status(None) == 0
    for ns in (0, 20_000):
        got = paused(check, "maxima", warp, ns, lambda: batch.call(check))
        assert check.nm_check_status(None) == 0
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.gpu
@pytest.mark.parametrize("where,warp", [("weights", 2), ("weights", 5), ("weights", 8), ("product", 1)])
def test_both_last_products_through_or_neither(libs, batch, where, warp):
    """A softmax warp held up until the last two P * V are through finds them so; an issuing warp held up ahead of each finds nobody gone on."""
    normal, check = libs
    want = batch.call(normal)
    got = paused(check, where, warp, 20_000, lambda: batch.call(check))
    assert check.nm_check_status(None) == 0, "a wait ran out"
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.gpu
@pytest.mark.parametrize("where,warp", [("maxima", 7), ("copy", 0), ("product", 1)])
def test_an_expired_wait_ends_in_order(libs, batch, where, warp):
    """A warp held up for longer than the others wait: they give up, what is under way ends, the kernel returns.  The call is disowned once, and the
    next one is right."""
    normal, check = libs
    want = batch.call(normal)
    paused(check, where, warp, 0, lambda: batch.call(check))
    assert check.nm_check_status(None) == 0
    t0 = time.monotonic()
    paused(check, where, warp, 1_300_000_000, lambda: batch.call(check))
    print("took %.3f s" % (time.monotonic() - t0))
    assert 1.3 <= time.monotonic() - t0 < 10
    assert check.nm_check_status(None) == -6 and check.nm_check_status(None) == 0
    got = batch.call(check)
    assert check.nm_check_status(None) == 0
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_the_pause_belongs_to_the_debug_build():
    import paper_2609_16009_b200 as nm
    from paper_2609_16009_b200 import build
    assert nm._lib.nm_debug_set_attention_q8_pause(1, 2, 1000) == -2
    check = _declare(C.CDLL(build.build(check=True)))
    for bad in ((-1, 2, 0), (99, 2, 0), (1, -1, 0), (1, 10, 0), (1, 2, 2_000_000_001)):
        assert check.nm_debug_set_attention_q8_pause(*bad) == -1, bad
