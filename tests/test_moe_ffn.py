"""The chosen experts' products and their weighted sum (nm_moe_ffn) against the definition in 64 bits."""
import ctypes

import pytest
import torch

from ffn_util import (BF16, COL, F16, GELU, GELU_TANH, RELU, ROW, SILU, TORCH, assert_within, hidden64, product64, randn, rounded, stored)


def make(T, d, inter, E, k, dtype, seed, gated=True):
    t = TORCH[dtype]
    g = torch.Generator().manual_seed(seed)
    wide = inter * (2 if gated else 1)
    return dict(x=randn(T, d, seed=seed, dtype=t), up=randn(E, d, wide, seed=seed + 1, scale=d ** -0.5, dtype=t), down=randn(E, inter, d, seed=seed + 2, scale=inter ** -0.5, dtype=t),
                experts=torch.rand(T, E, generator=g).topk(k, 1).indices.to(torch.int32), weights=torch.softmax(torch.randn(T, k, generator=g), 1), residual=randn(T, d, seed=seed + 3, dtype=t))


def expected(c, act, gated, dtype, first=0, residual=True):
    E, inter, d = c["down"].shape
    T, k = c["experts"].shape
    y = c["residual"].double().clone() if residual else torch.zeros(T, d, dtype=torch.float64)
    size, t = y.abs(), torch.zeros_like(y)
    for e in range(E):
        rows, j = (c["experts"] == e + first).nonzero(as_tuple=True)
        if not len(rows):
            continue
        h, th = hidden64(c["x"][rows].double(), c["up"][e].double(), act, gated)
        # h is kept in two 16-bit terms: 2^-16 of itself, and of a row's largest 2^-24 (fp16 terms have an absolute step)
        th = th + 2.0 ** -16 * h.abs() + 2.0 ** -24 * h.abs().amax(1, keepdim=True)
        z, tz = product64(h, c["down"][e].double(), th)
        w = c["weights"][rows, j].double()[:, None] if c["weights"] is not None else 1.0
        y.index_add_(0, rows, w * z)
        t.index_add_(0, rows, abs(w) * tz)
        size.index_add_(0, rows, abs(w) * z.abs())
    return y, rounded(y, t + (k + 2) * 2.0 ** -23 * size, dtype)


def call(nm, c, act, gated, dtype, layout, out, ws, first=0, residual=True, dev=None, stream=None, **strides):
    dev = dev or place(c, layout)
    T, k = c["experts"].shape
    E, inter, d = c["down"].shape
    nm.nm_moe_ffn(dev["x"], dev["experts"], dev["weights"], dev["up"], dev["down"], out, T, d, inter, E, k, act, dtype, layout, ws, gated=gated,
                  residual=dev["residual"] if residual else None, first_expert=first, stream=stream, **strides)


def place(c, layout):
    return {n: None if v is None else (stored(v, layout) if n in ("up", "down") else v).cuda() for n, v in c.items()}


def workspace(nm, c, dtype):
    T, k = c["experts"].shape
    E, inter, d = c["down"].shape
    ws = torch.full((nm.nm_moe_ffn_workspace_bytes(T, d, inter, E, k, dtype),), 0xFF, dtype=torch.uint8, device="cuda")
    nm.nm_workspace_init(ws[:nm.WS_COUNTER_BYTES])                 # the counters; the rest may hold anything
    return ws


def run(c, act, gated, dtype, layout, first=0, residual=True):
    import paper_2609_16009_b200 as nm
    T, d = c["x"].shape
    ws, outs, dev = workspace(nm, c, dtype), [], place(c, layout)
    for _ in range(2):
        out = torch.full((T + 2, d), 77.0, dtype=TORCH[dtype], device="cuda")
        call(nm, c, act, gated, dtype, layout, out[1:], ws, first, residual, dev)
        outs.append(out)
    nm.nm_check_status()
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16)), "equal calls give equal bits"
    assert (outs[0][0] == 77).all() and (outs[0][-1] == 77).all(), "written outside the result"
    return outs[0][1:-1]


SIZES = [(1, 8, 8, 1, 1), (1, 64, 128, 4, 2), (2, 72, 136, 5, 3), (3, 63, 65, 4, 2), (5, 130, 64, 3, 1), (16, 512, 256, 64, 6), (17, 264, 520, 9, 4), (40, 1024, 72, 6, 3), (64, 256, 384, 16, 8),
         (100, 200, 264, 3, 2), (130, 136, 1000, 2, 1), (257, 128, 128, 40, 5), (300, 256, 192, 2, 2), (1, 2048, 1024, 32, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [ROW, COL])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("T,d,inter,E,k", SIZES)
def test_experts(T, d, inter, E, k, gated, dtype, layout):
    act = (SILU, GELU, GELU_TANH, RELU)[(T + d) % 4]
    c = make(T, d, inter, E, k, dtype, T + d + inter, gated)
    assert_within(run(c, act, gated, dtype, layout), *expected(c, act, gated, dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("kind", ["padding", "shard", "one expert", "nobody", "twice", "outside"])
def test_lists_of_experts(kind, dtype):
    T, d, inter, E, k, first = 50, 256, 136, 8, 3, 0
    c = make(T, d, inter, E, k, dtype, 11)
    if kind == "padding":
        c["experts"][::3] = -1                     # tokens of a padded batch
        c["experts"][1::3, 1] = -1
    elif kind == "shard":
        first = 5
        c["experts"] = torch.randint(0, 20, (T, k), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    elif kind == "one expert":
        c["experts"][:] = 6
    elif kind == "nobody":
        c["experts"][:] = -1
    elif kind == "twice":
        c["experts"][:, 1] = c["experts"][:, 0]
    else:
        c["experts"][::2, 0], c["experts"][1::2, 0] = 2 ** 31 - 1, -2 ** 31
        first = 1
    for residual in (True, False):
        assert_within(run(c, SILU, True, dtype, COL, first, residual), *expected(c, SILU, True, dtype, first, residual))


@pytest.mark.gpu
def test_shards_add_up():
    """The experts held in two places: the parts of both, the residual given to one, are the whole."""
    T, d, inter, E, k = 9, 128, 64, 6, 3
    c = make(T, d, inter, E, k, BF16, 12)
    lower, upper = dict(c, up=c["up"][:2], down=c["down"][:2]), dict(c, up=c["up"][2:], down=c["down"][2:])
    y0, y1 = run(lower, SILU, True, BF16, COL, 0, True), run(upper, SILU, True, BF16, COL, 2, False)
    r0, t0 = expected(lower, SILU, True, BF16, 0, True)
    r1, t1 = expected(upper, SILU, True, BF16, 2, False)
    assert_within(y0.double() + y1.double(), expected(c, SILU, True, BF16)[0], t0 + t1)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [ROW, COL])
def test_what_was_not_chosen_is_not_read(layout):
    c = make(20, 256, 128, 10, 2, BF16, 13)
    c["experts"] = c["experts"] % 4 * 2            # the even ones alone
    ref, tol = expected(c, SILU, True, BF16)
    for e in range(1, 10, 2):
        c["up"][e], c["down"][e] = float("nan"), float("nan")
    c["up"][8], c["down"][8] = float("inf"), float("nan")
    assert_within(run(c, SILU, True, BF16, layout), ref, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_a_bad_token_and_a_bad_expert_stay_where_they_are(dtype):
    c = make(30, 128, 72, 6, 2, dtype, 14)
    clean = run(c, SILU, True, dtype, COL)
    c["x"][4, 7], c["x"][20, 100] = float("nan"), float("inf")
    c["down"][3, 5, :] = float("nan")
    got = run(c, SILU, True, dtype, COL)
    fine = [t for t in range(30) if t not in (4, 20) and not (c["experts"][t] == 3).any()]
    assert len(fine) > 5 and torch.equal(got[fine], clean[fine])
    assert got[4].isnan().all()


@pytest.mark.gpu
def test_hidden_values_beyond_fp16():
    """act(g) * u beyond fp16's largest value, and below its smallest: neither is lost."""
    c = make(6, 64, 64, 3, 2, F16, 15)
    c["x"][:3] = (c["x"][:3].float() * 400).half()
    c["up"] = (c["up"].float() * 8).half()
    c["down"] = (c["down"].float() * 2.0 ** -9).half()
    c["x"][3:] = (c["x"][3:].float() * 2.0 ** -12).half()
    c["residual"] = (c["residual"].float() * 2.0 ** -12).half()
    h, _ = hidden64(c["x"][:3].double(), c["up"][0].double(), SILU, True)
    assert h.abs().max() > 2 * 65504
    assert_within(run(c, SILU, True, F16, COL), *expected(c, SILU, True, F16))


@pytest.mark.gpu
def test_without_weights_they_are_one():
    c = make(7, 64, 72, 5, 3, BF16, 16, False)
    c["weights"] = None
    assert_within(run(c, GELU, False, BF16, ROW), *expected(c, GELU, False, BF16))


@pytest.mark.gpu
@pytest.mark.parametrize("ldx,ldo,ldr", [(272, 264, 280), (259, 257, 261)])
def test_strides(ldx, ldo, ldr):
    import paper_2609_16009_b200 as nm
    T, d = 21, 256
    c = make(T, d, 128, 7, 2, BF16, 17)
    dev = place(c, COL)
    for name, ld in (("x", ldx), ("residual", ldr)):
        wide = torch.full((T, ld), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, :d] = dev[name]
        dev[name] = wide
    out = torch.full((T, ldo), 77.0, dtype=torch.bfloat16, device="cuda")
    call(nm, c, SILU, True, BF16, COL, out, workspace(nm, c, BF16), dev=dev, ldx=ldx, ldo=ldo, ld_residual=ldr)
    assert (out[:, d:] == 77).all()
    assert_within(out[:, :d], *expected(c, SILU, True, BF16))


@pytest.mark.gpu
@pytest.mark.parametrize("onto", ["x", "residual"])
def test_in_place(onto):
    import paper_2609_16009_b200 as nm
    c = make(33, 264, 128, 7, 3, BF16, 18)
    dev = place(c, ROW)
    call(nm, c, SILU, True, BF16, ROW, dev[onto], workspace(nm, c, BF16), dev=dev)
    assert_within(dev[onto], *expected(c, SILU, True, BF16))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_captured_replayed_and_on_another_stream(dtype):
    """A graph computes with the experts that stand in its buffers when it is replayed."""
    import paper_2609_16009_b200 as nm
    a, b = make(12, 256, 136, 9, 3, dtype, 19), make(12, 256, 136, 9, 3, dtype, 20)
    b["up"], b["down"] = a["up"], a["down"]
    b["experts"][3:7] = 4
    dev, ws = place(a, COL), workspace(nm, a, dtype)
    out = torch.zeros(12, 256, dtype=TORCH[dtype], device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(nm, a, SILU, True, dtype, COL, out, ws, dev=dev, stream=s)
    torch.cuda.synchronize()
    assert_within(out, *expected(a, SILU, True, dtype))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(nm, a, SILU, True, dtype, COL, out, ws, dev=dev)
    for c in (b, a, b):
        for n in ("x", "experts", "weights", "residual"):
            dev[n].copy_(c[n])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert_within(out, *expected(c, SILU, True, dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("programmatic", [False, True])
def test_layer_by_layer(programmatic):
    """Router product, routing, shared expert and experts, one layer behind the other through one workspace: each layer against the definition
    for the rows it was given."""
    import paper_2609_16009_b200 as nm
    T, d, inter, E, k = 6, 512, 128, 16, 4
    layers = [make(T, d, inter, E, k, BF16, 30 + i) for i in range(3)]
    routers = [randn(d, E, seed=40 + i, scale=d ** -0.5, dtype=torch.bfloat16) for i in range(3)]
    dev, router = [place(c, COL) for c in layers], [w.cuda() for w in routers]
    shared = [(randn(d, 2 * inter, seed=50 + i, scale=d ** -0.5, dtype=torch.bfloat16), randn(inter, d, seed=60 + i, scale=inter ** -0.5, dtype=torch.bfloat16)) for i in range(3)]
    dshared = [(stored(a, COL).cuda(), stored(b, COL).cuda()) for a, b in shared]
    ws = workspace(nm, layers[0], BF16)
    small = nm.new_workspace(max(nm.nm_matmul_act_workspace_bytes(T, inter, d, True), nm.nm_matmul_act_workspace_bytes(T, d, inter), nm.nm_matmul_workspace_bytes(T, E, d, 1, 2)))
    xs = [layers[0]["x"].cuda()] + [torch.zeros(T, d, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    logits, h, mid = torch.zeros(3, T, E, device="cuda"), torch.zeros(T, inter, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, T, d, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    nm.nm_set_programmatic_launch(programmatic)
    try:
        for i in range(3):
            nm.nm_matmul_ws(xs[i], router[i], logits[i], T, E, d, nm.BF16_F32OUT, ROW, small)
            nm.nm_moe_route(logits[i], None, dev[i]["experts"], dev[i]["weights"], T, E, k, nm.F32, nm.SCORE_SIGMOID, groups=4, keep_groups=2, group_best=2, scale=1.5)
            nm.nm_matmul_act(xs[i], dshared[i][0], h, T, inter, d, SILU, BF16, COL, small, gated=True)
            nm.nm_matmul_act(h, dshared[i][1], mid[i], T, d, inter, 0, BF16, COL, small, residual=xs[i])
            nm.nm_moe_ffn(xs[i], dev[i]["experts"], dev[i]["weights"], dev[i]["up"], dev[i]["down"], xs[i + 1], T, d, inter, E, k, SILU, BF16, COL, ws, residual=mid[i])
    finally:
        nm.nm_set_programmatic_launch(False)
    nm.nm_check_status()
    from test_route import SIGMOID, reference
    for i in range(3):
        x = xs[i].cpu()
        lg, tl = product64(x.double(), routers[i].double())
        assert_within(logits[i], lg, tl + 1e-6)
        e, w = reference(logits[i].cpu().double().numpy(), None, k, SIGMOID, 4, 2, 2, True, 1.5)
        assert torch.equal(dev[i]["experts"].cpu().long(), torch.from_numpy(e))
        hs, th = hidden64(x.double(), shared[i][0].double(), SILU, True)
        th = rounded(hs, th, BF16)                 # the shared expert's hidden values go through bf16
        z, tz = product64(hs, shared[i][1].double(), th)
        z = z + x.double()
        assert_within(mid[i], z, rounded(z, tz + 2.0 ** -22 * z.abs(), BF16))
        c = dict(layers[i], x=x, experts=dev[i]["experts"].cpu(), weights=dev[i]["weights"].cpu(), residual=mid[i].cpu())
        assert_within(xs[i + 1], *expected(c, SILU, True, BF16))


@pytest.fixture(scope="module")
def lib():
    from paper_2609_16009_b200 import build
    return ctypes.CDLL(build.build())


def test_refusals_need_no_device(lib):
    vp, i, l, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_long, ctypes.c_size_t
    lib.nm_moe_ffn.argtypes = [vp, l, vp, vp, vp, vp, vp, l, vp, l] + [i] * 10 + [vp, sz, vp]
    lib.nm_moe_ffn_workspace_bytes.restype = sz
    need = lib.nm_moe_ffn_workspace_bytes(4, 64, 32, 8, 2, 1)
    assert need > 0

    def status(x=256, ldx=64, experts=512, weights=1024, up=2048, down=4096, residual=None, ldr=64, out=8192, ldo=64, T=4, d=64, inter=32, E=8, k=2, first=0, act=2, gated=1, dtype=1,
               layout=1, ws=16384, bytes_=1 << 40):
        return lib.nm_moe_ffn(x, ldx, experts, weights, up, down, residual, ldr, out, ldo, T, d, inter, E, k, first, act, gated, dtype, layout, ws, bytes_, None)
    assert status(x=None) == status(experts=None) == status(up=None) == status(down=None) == status(out=None) == -1
    assert status(T=0) == status(d=0) == status(inter=0) == status(E=0) == status(k=0) == status(first=-1) == -1
    assert status(ldx=63) == status(ldo=63) == status(residual=256, ldr=63) == -1
    assert status(dtype=0) == status(dtype=2) == status(layout=2) == status(act=5) == status(E=1025) == status(T=1 << 22, k=2) == -2
    assert status(x=257) == status(up=2049) == status(down=4097) == status(out=8193) == status(residual=257) == status(experts=514) == status(weights=1026) == status(ws=16385) == -3
    assert status(ws=None) == status(bytes_=need - 1) == -4
    assert lib.nm_moe_ffn_workspace_bytes(0, 1, 1, 1, 1, 1) == lib.nm_moe_ffn_workspace_bytes(1, 1, 1, 1, 1, 0) == 0
