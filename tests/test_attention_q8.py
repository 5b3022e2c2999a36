"""Latent attention of a batch over the quantised cache with a shared prefix, against a plain implementation in 64 bits; and a run of the
operators for compressed storage together, as a decode loop uses them."""
import ctypes

import numpy as np
import pytest
import torch

from test_cache_q8 import e4m3_value, records

KV, ROPE, REC = 512, 64, 656
SCALE = 192 ** -0.5


def make_records(n, g, spread=2):
    """Records of n rows ~ N(0, 1), each with a power of two of its own, as the writer leaves them."""
    x = torch.randn(n, KV + ROPE, generator=g) * torch.exp2(torch.randint(-spread, spread + 1, (n, 1), generator=g).float())
    s = torch.exp2(torch.ceil(torch.log2(x[:, :KV].abs().amax(1, keepdim=True) / 448)))
    rec = torch.zeros(n, REC, dtype=torch.uint8)
    if n:
        rec[:, :KV] = (x[:, :KV] / s).to(torch.float8_e4m3fn).view(torch.uint8)
        rec[:, KV:KV + 2 * ROPE] = (x[:, KV:] / s).to(torch.bfloat16).view(torch.uint8).view(n, 2 * ROPE)
        rec[:, KV + 2 * ROPE:KV + 2 * ROPE + 4] = s.view(torch.uint8).view(n, 4)
    return rec


def rows_of(rec):
    if not len(rec):
        return np.zeros((0, KV + ROPE))
    v, key, s = records(rec.numpy(), KV, ROPE)
    return np.concatenate((v, key), 1) * s


def check(Q, scale, prefix, own, o16, o32, lse):
    """Every head of every sequence.  A weight goes to fp16 (2^-11) and to three e5m2 terms (2^-9 of it at most); its score is off by what
    the queries' second term drops (2^-10 where the largest is over 224) and by fp32 sums of 64 terms' depth; 2^-22 each for the
    exponential and the sums.  bf16 output: 2^-8 of the value."""
    pre = rows_of(prefix)
    for t in range(len(own)):
        rows = np.concatenate((pre, rows_of(own[t])))
        q = Q[t].double().numpy()
        if not len(rows):
            assert not o32[t].any() and not o16[t].any() and np.isneginf(lse[t]).all()
            continue
        x = q @ rows.T * scale
        m = x.max(1, keepdims=True)
        p = np.exp(x - m)
        total = p.sum(1, keepdims=True)
        p /= total
        ref = p @ rows[:, :KV]
        size = p @ np.abs(rows[:, :KV])
        drop = abs(scale) * (np.abs(q[:, :KV]).max(1, keepdims=True) * 2.0 ** -17.8 * np.abs(rows[:, :KV]).sum(1).max()
                             + (np.abs(q) @ np.abs(rows).T).max(1, keepdims=True) * 64 * 2.0 ** -23) + np.abs(x).max() * 2.0 ** -21
        tol = size * (2.0 ** -9 + 2.0 ** -11 + 2.0 ** -20 + 2 * drop) + 2.0 ** -24 * np.abs(rows).max()
        err = np.abs(o32[t] - ref)
        assert np.all(err <= tol), f"sequence {t}: {np.max(err / tol):.2f} of the tolerance"
        assert np.all(np.abs(o16[t] - ref) <= tol + 2.0 ** -8 * (np.abs(ref) + tol))
        want = (m + np.log(total))[:, 0]
        assert np.all(np.abs(lse[t] - want) <= drop[:, 0] + 2.0 ** -18 + 2.0 ** -22 * np.abs(want)), f"sequence {t}: log-sum-exp"


def run(nm, Q, scale, prefix, own, garbage=0xFF, stream=None, q_stride=None, out=None):
    """The call, with garbage (NaN records) behind every sequence's rows and canaries around the outputs."""
    T, H = Q.shape[:2]
    lens = [len(o) for o in own]
    step = max(max(lens), 1) + 3
    cache = torch.full((T, step, REC), garbage, dtype=torch.uint8)
    for t, o in enumerate(own):
        cache[t, :len(o)] = o
    shared = torch.full((len(prefix) + 2, REC), garbage, dtype=torch.uint8)
    shared[:len(prefix)] = prefix
    stride = q_stride or H * (KV + ROPE)
    dQ = torch.full((T, stride), float("nan"), dtype=torch.bfloat16)
    dQ[:, :H * (KV + ROPE)] = Q.reshape(T, -1)
    dQ, cache, shared = dQ.cuda(), cache.cuda(), shared.cuda()
    o16 = torch.full((T * H + 2, KV), 7.0, dtype=torch.bfloat16, device="cuda")
    o32 = torch.full((T * H + 2, KV), 7.0, dtype=torch.float32, device="cuda")
    lse = torch.full((T * H + 2,), 7.0, dtype=torch.float32, device="cuda")
    ws = torch.full((nm.nm_mla_attention_q8_workspace_bytes(T, H),), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    call = lambda: nm.nm_mla_attention_q8(dQ, shared, len(prefix), cache, step * REC, lens, o16[1:], o32[1:], lse[1:], H, KV, ROPE, scale, ws,  # noqa: E731
                                          q_stride=stride, stream=stream)
    call()
    torch.cuda.synchronize()
    nm.nm_check_status()
    for o in (o16, o32, lse):
        assert (o[0] == 7).all() and (o[-1] == 7).all(), "written outside"
    first = [o[1:-1].clone() for o in (o16, o32, lse)]
    call()
    torch.cuda.synchronize()
    assert all(torch.equal(x.view(torch.uint8), y[1:-1].contiguous().view(torch.uint8)) for x, y in zip(first, (o16, o32, lse))), "equal calls give equal bits"
    return (first[0].double().cpu().numpy().reshape(T, H, KV), first[1].double().cpu().numpy().reshape(T, H, KV),
            first[2].double().cpu().numpy().reshape(T, H))


def case(T, H, prefix, lens, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    Q = (torch.randn(T, H, KV + ROPE, generator=g) * std).to(torch.bfloat16)
    return Q, make_records(prefix, g), [make_records(n, g) for n in lens]


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,prefix,lens", [
    (1, 1, 0, [1]), (1, 128, 0, [1]), (1, 16, 0, [95]), (1, 16, 0, [96]), (1, 7, 0, [97]), (1, 128, 0, [192]), (2, 24, 0, [0, 300]),
    (1, 128, 1, [0]), (3, 128, 97, [0, 1, 200]), (5, 24, 200, [3, 0, 96, 97, 11]), (4, 33, 1000, [0, 0, 0, 0]), (3, 1, 5, [2, 0, 1]), (2, 128, 0, [0, 0])])
def test_small(T, H, prefix, lens):
    import paper_2609_16009_b200 as nm
    Q, pre, own = case(T, H, prefix, lens, T * 100 + H + prefix)
    check(Q, SCALE, pre, own, *run(nm, Q, SCALE, pre, own))


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,prefix,lens", [(1, 128, 0, [9001]), (16, 8, 3000, [1 + 37 * t for t in range(16)]), (64, 2, 500, [t % 5 for t in range(64)]),
                                             (3, 100, 5000, [2000, 1, 700])])
def test_longer(T, H, prefix, lens):
    """Several parts a unit, several waves, the largest batch."""
    import paper_2609_16009_b200 as nm
    Q, pre, own = case(T, H, prefix, lens, T + H)
    check(Q, SCALE, pre, own, *run(nm, Q, SCALE, pre, own))


@pytest.mark.gpu
@pytest.mark.parametrize("std,scale", [(0.0, SCALE), (8.0, SCALE), (1.0, -SCALE), (1e-3, 3.0), (1e20, 1e-21)])
def test_flat_and_sharp_scores(std, scale):
    """All weights alike, one weight alone (the maximum moves from tile to tile), a negative scale, queries of extreme sizes."""
    import paper_2609_16009_b200 as nm
    Q, pre, own = case(2, 20, 400, [500, 30], 5, std)
    check(Q, scale, pre, own, *run(nm, Q, scale, pre, own))


@pytest.mark.gpu
def test_many_small_weights_beside_a_large_one():
    """One row holds most of the weight, thousands of equal ones the rest, each 2^-20 of it: they count with their full weight."""
    import paper_2609_16009_b200 as nm
    n = 6000
    rec = torch.zeros(n, REC, dtype=torch.uint8)
    one = torch.tensor([1.0]).to(torch.float8_e4m3fn).view(torch.uint8)
    rec[:, 5] = one                                                # every row: value 1 in column 5
    rec[:, KV + 2 * ROPE:KV + 2 * ROPE + 4] = torch.ones(n, 1).view(torch.uint8)
    rec[4000, 5], rec[4000, 9] = 0, one                            # one row: in column 9 instead
    Q = torch.zeros(1, 4, KV + ROPE, dtype=torch.bfloat16)
    Q[:, :, 9] = 14.0                                              # its score is larger by 14: e^14 = 2^20
    o16, o32, lse = run(nm, Q, 1.0, rec[:0], [rec])
    check(Q, 1.0, rec[:0], [rec], o16, o32, lse)
    rest = (n - 1) / (n - 1 + np.exp(14.0))
    assert np.all(np.abs(o32[0, :, 5] - rest) <= rest * 2.0 ** -8), "2^-9 and 2^-11 on each side of the quotient at most"


@pytest.mark.gpu
def test_scales_of_very_different_rows():
    """Rows whose powers of two differ by 2^40: each keeps its weight and its size."""
    import paper_2609_16009_b200 as nm
    g = torch.Generator().manual_seed(8)
    rec = make_records(300, g)
    rec[:, KV + 2 * ROPE:KV + 2 * ROPE + 4] = torch.exp2(torch.randint(-32, 9, (300, 1), generator=g).float()).view(torch.uint8)
    Q = (torch.randn(1, 16, KV + ROPE, generator=g) * 2.0 ** -12).to(torch.bfloat16)
    check(Q, SCALE, rec[:100], [rec[100:]], *run(nm, Q, SCALE, rec[:100], [rec[100:]]))


@pytest.mark.gpu
def test_records_of_zeros_have_their_weight():
    import paper_2609_16009_b200 as nm
    Q, _, own = case(1, 3, 0, [40], 12)
    zero = torch.zeros(60, REC, dtype=torch.uint8)
    rec = torch.cat((own[0], zero))
    check(Q, SCALE, zero[:0], [rec], *run(nm, Q, SCALE, zero[:0], [rec]))


@pytest.mark.gpu
def test_nan_stays_with_its_head_and_its_sequence():
    import paper_2609_16009_b200 as nm
    Q, pre, own = case(3, 20, 150, [120, 130, 0], 3)
    clean = run(nm, Q, SCALE, pre, own)
    Q[1, 4, 100], Q[2, 7, KV + 3] = float("nan"), float("inf")
    own[0][50, 17] = 0x7F                                          # a NaN code in one record of sequence 0
    got = run(nm, Q, SCALE, pre, own)
    bad = np.zeros((3, 20), dtype=bool)
    bad[0], bad[1, 4], bad[2, 7] = True, True, True
    for c, x in zip(clean, got):
        assert np.isnan(x[bad]).all()
        assert np.array_equal(c[~bad], x[~bad]), "nobody else notices"


@pytest.mark.gpu
def test_strides_streams_and_graph():
    import paper_2609_16009_b200 as nm
    Q, pre, own = case(4, 32, 300, [100, 0, 250, 96], 21)
    ref = run(nm, Q, SCALE, pre, own)
    wide = run(nm, Q, SCALE, pre, own, q_stride=32 * 576 + 64, stream=torch.cuda.Stream())
    assert all(np.array_equal(x, y) for x, y in zip(ref, wide))
    lens, step = [len(o) for o in own], 250
    cache = torch.zeros(4, step, REC, dtype=torch.uint8)
    for t, o in enumerate(own):
        cache[t, :len(o)] = o
    cache, shared, dQ = cache.cuda(), pre.cuda(), Q.cuda()
    outs = [torch.zeros(4, 32, KV, dtype=torch.float32, device="cuda") for _ in range(3)]
    ws = [torch.empty(nm.nm_mla_attention_q8_workspace_bytes(4, 32), dtype=torch.uint8, device="cuda") for _ in range(3)]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):                                            # two streams, a workspace each
        nm.nm_mla_attention_q8(dQ, shared, 300, cache, step * REC, lens, None, outs[0], None, 32, KV, ROPE, SCALE, ws[0], stream=s1)
        nm.nm_mla_attention_q8(dQ, shared, 300, cache, step * REC, lens, None, outs[1], None, 32, KV, ROPE, SCALE, ws[1], stream=s2)
    torch.cuda.synchronize()
    late = torch.zeros_like(dQ)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nm.nm_mla_attention_q8(late, shared, 300, cache, step * REC, lens, None, outs[2], None, 32, KV, ROPE, SCALE, ws[2])
    late.copy_(dQ)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert np.array_equal(o.double().cpu().numpy(), ref[1])
    nm.nm_check_status()


@pytest.mark.gpu
def test_decode_from_compressed_storage():
    """A decode step's KV chain and attention on compressed storage, token after token: the projection from 4-bit weights, the row
    normalised, rotated and quantised into the cache, the attention over prefix and own rows, the output projection - each
    operator against the plain form of its own input."""
    import paper_2609_16009_b200 as nm
    g = torch.Generator().manual_seed(31)
    T, H, d, prefix, room = 3, 16, 640, 200, 8
    W_kv, W_o = ((torch.randn(n, k, generator=g) * 0.05).to(torch.bfloat16) for n, k in ((KV + ROPE, d), (d, H * KV)))
    packs = []
    for W in (W_kv, W_o):
        N, K = W.shape
        packed = torch.zeros(nm.nm_w4_packed_bytes(N, K), dtype=torch.uint8, device="cuda")
        scales = torch.zeros(nm.nm_w4_scale_count(N, K, 64), dtype=torch.bfloat16, device="cuda")
        back = torch.zeros(N, K, dtype=torch.bfloat16, device="cuda")
        nm.nm_w4_quantize(W.cuda(), packed, scales, N, K, 64, nm.BF16, nm.COL_MAJOR)
        exact = torch.zeros(N, K, device="cuda")
        eye = torch.eye(K, dtype=torch.bfloat16, device="cuda")
        for k in range(0, K, 16):                                   # the weights as the product sees them, sixteen k at a time
            m = min(16, K - k)
            col = torch.zeros(m, N, dtype=torch.float32, device="cuda")
            nm.nm_matmul_w4(eye[k:k + m], packed, scales, col, m, N, K, 64, nm.BF16_F32OUT)
            exact[:, k:k + m] = col.T
        nm.nm_w4_dequantize(packed, scales, back, N, K, 64, nm.BF16, nm.COL_MAJOR)
        assert torch.equal(exact.to(torch.bfloat16), back)
        packs.append((packed, scales, exact.double().cpu().numpy()))
    gamma = (1 + 0.1 * torch.randn(KV, generator=g)).to(torch.bfloat16)
    shared = make_records(prefix, g)
    cache = torch.full((T * room, REC), 0xFF, dtype=torch.uint8, device="cuda")
    ws = torch.empty(nm.nm_mla_attention_q8_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    table = torch.zeros(room, ROPE, device="cuda")
    nm.nm_rope_table(table, prefix, room, ROPE)
    for step in range(3):
        h = torch.randn(T, d, generator=g).to(torch.bfloat16)
        Q = torch.randn(T, H, KV + ROPE, generator=g).to(torch.bfloat16)
        ckr = torch.zeros(T, KV + ROPE, dtype=torch.bfloat16, device="cuda")
        o = torch.zeros(T, H, KV, dtype=torch.bfloat16, device="cuda")
        o32, lse = torch.zeros(T, H, KV, device="cuda"), torch.zeros(T, H, device="cuda")
        out = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
        rows = torch.arange(T, device="cuda") * room + step
        cs = table[step].repeat(T, 1)
        nm.nm_matmul_w4(h.cuda(), packs[0][0], packs[0][1], ckr, T, KV + ROPE, d, 64, nm.BF16)
        nm.nm_mla_cache_write_q8(ckr, gamma.cuda(), cs, rows, cache, T * room, T, KV, ROPE, 1e-6)
        nm.nm_mla_attention_q8(Q.cuda(), shared.cuda(), prefix, cache, room * REC, [step + 1] * T, o, o32, lse, H, KV, ROPE, SCALE, ws)
        nm.nm_matmul_w4(o, packs[1][0], packs[1][1], out, T, d, H * KV, 64, nm.BF16)
        torch.cuda.synchronize()
        nm.nm_check_status()
        # products: sums of K terms of size 23 / 8 |a w| at most in fp32, 2^-8 for the output
        for a, w, got in ((h, packs[0][2], ckr), (o.cpu().reshape(T, -1), packs[1][2], out)):
            a, got = a.double().numpy(), got.double().cpu().numpy()
            ref, size = a @ w.T, np.abs(a) @ np.abs(w).T + np.abs(a).sum(1, keepdims=True) * np.abs(w).max()
            assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 160 * 2.0 ** -23 * 3 * size)
        x = ckr.double().cpu().numpy()
        y = x[:, :KV] / np.sqrt((x[:, :KV] ** 2).mean(1, keepdims=True) + 1e-6) * gamma.double().numpy()
        codes, key, s = records(cache[rows].cpu().numpy(), KV, ROPE)
        assert np.all(np.abs(codes * s - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * s) * (1 + 2.0 ** -15))
        own = [cache[t * room:t * room + step + 1].cpu() for t in range(T)]
        check(Q, SCALE, shared, own, o.double().cpu().numpy(), o32.double().cpu().numpy(), lse.double().cpu().numpy())


@pytest.mark.gpu
def test_rows_beyond_32_bit_offsets():
    """A prefix of more than 4 GB and sequences as far apart: rows of zeros (weight 1 each) and 24 that matter at the very end."""
    import paper_2609_16009_b200 as nm
    n, H = 6_600_000, 16
    assert n * REC > 2 ** 32
    g = torch.Generator().manual_seed(41)
    last = make_records(24, g, spread=0)
    Q = (torch.randn(2, H, KV + ROPE, generator=g)).to(torch.bfloat16)
    cache = torch.zeros(n, REC, dtype=torch.uint8, device="cuda")
    x = torch.randn(24, KV + ROPE, generator=g).to(torch.bfloat16)
    nm.nm_mla_cache_write_q8(x.cuda(), None, None, torch.arange(n - 24, n, device="cuda"), cache, n, 24, KV, ROPE)
    back = torch.zeros(24, KV + ROPE, dtype=torch.bfloat16, device="cuda")
    nm.nm_mla_cache_read_q8(cache, n, torch.arange(n - 24, n, device="cuda"), back, 24, KV, ROPE)
    # a value to e4m3 and back: 2^-4 of it, 2^-10 of the row's scale (4 / 448 < 2^-6) below the normal range
    x = x.double()
    assert ((back.cpu().double() - x).abs() <= x.abs() * 2.0 ** -4 * (1 + 2.0 ** -7) + 2.0 ** -16).all()
    cache[n - 24:] = last.cuda()
    rows = rows_of(last)
    o32, lse = torch.zeros(2, H, KV, device="cuda"), torch.zeros(2, H, device="cuda")
    ws = torch.empty(nm.nm_mla_attention_q8_workspace_bytes(2, H), dtype=torch.uint8, device="cuda")
    scale = 0.7                                                    # scores of about 17, e^17 = 24e6
    for prefix, lens in ((n, [0, 0]), (0, [0, 24])):
        if prefix:
            nm.nm_mla_attention_q8(Q.cuda(), cache, n, None, 0, lens, None, o32, lse, H, KV, ROPE, scale, ws)
        else:                                                      # the second sequence starts 4 GB behind the first
            nm.nm_mla_attention_q8(Q.cuda(), None, 0, cache, (n - 24) * REC, lens, None, o32, lse, H, KV, ROPE, scale, ws)
        torch.cuda.synchronize()
        nm.nm_check_status()
        for t in range(2):
            if not prefix and t == 0:
                assert not o32[0].any() and torch.isneginf(lse[0]).all()
                continue
            q = Q[t].double().numpy()
            s = q @ rows.T * scale
            zeros = n - 24 if prefix else 0
            m = np.maximum(s.max(1, keepdims=True), 0)
            p = np.exp(s - m)
            total = p.sum(1, keepdims=True) + zeros * np.exp(-m)
            ref, size = (p / total) @ rows[:, :KV], (p / total) @ np.abs(rows[:, :KV])
            # as in check; the sum of the zeros' weights is one of 22000 equal terms a thread at most: 2^-10 of them in fp32
            drop = scale * (np.abs(q[:, :KV]).max(1, keepdims=True) * 2.0 ** -17.8 * np.abs(rows[:, :KV]).sum(1).max()
                            + (np.abs(q) @ np.abs(rows).T).max(1, keepdims=True) * 64 * 2.0 ** -23) + np.abs(s).max() * 2.0 ** -21
            tol = size * (2.0 ** -9 + 2.0 ** -11 + 2.0 ** -20 + 2 * drop + 2.0 ** -10) + 2.0 ** -24 * np.abs(rows).max()
            assert np.all(np.abs(o32[t].double().cpu().numpy() - ref) <= tol)
            want = (m + np.log(total))[:, 0]
            assert np.all(np.abs(lse[t].double().cpu().numpy() - want) <= drop[:, 0] + 2.0 ** -10 + 2.0 ** -22 * np.abs(want))


@pytest.mark.gpu
def test_chain_launched_programmatically():
    """Projection, cache write, attention and output projection behind each other, each starting while the one before it ends: the
    bits of the plain order, in a graph and step after step."""
    import paper_2609_16009_b200 as nm
    g = torch.Generator().manual_seed(43)
    T, H, d, room, steps = 8, 32, 1024, 8, 6
    packs = []
    for N, K in ((KV + ROPE, d), (d, H * KV)):
        packs.append((torch.randint(0, 256, (nm.nm_w4_packed_bytes(N, K),), dtype=torch.uint8, generator=g).cuda(),
                      torch.full((nm.nm_w4_scale_count(N, K, 128),), 0.01, dtype=torch.bfloat16, device="cuda")))
    gamma, prefix = torch.ones(KV, dtype=torch.bfloat16, device="cuda"), make_records(150, g).cuda()
    Q = torch.randn(steps, T, H, KV + ROPE, generator=g).to(torch.bfloat16).cuda()
    h0 = torch.randn(T, d, generator=g).to(torch.bfloat16).cuda()
    h, ckr = torch.zeros_like(h0), torch.zeros(T, KV + ROPE, dtype=torch.bfloat16, device="cuda")
    o = torch.zeros(T, H, KV, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(nm.nm_mla_attention_q8_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    cache = torch.zeros(T * room, REC, dtype=torch.uint8, device="cuda")
    rows = [torch.arange(T, device="cuda") * room + i for i in range(steps)]

    def run_all():
        h.copy_(h0)
        for i in range(steps):                                     # each step's output is the next one's token
            nm.nm_matmul_w4(h, *packs[0], ckr, T, KV + ROPE, d, 128, nm.BF16)
            nm.nm_mla_cache_write_q8(ckr, gamma, None, rows[i], cache, T * room, T, KV, ROPE)
            nm.nm_mla_attention_q8(Q[i], prefix, 150, cache, room * REC, [i + 1] * T, o, None, None, H, KV, ROPE, SCALE, ws)
            nm.nm_matmul_w4(o, *packs[1], h, T, d, H * KV, 128, nm.BF16)

    run_all()
    torch.cuda.synchronize()
    want = (h.clone(), o.clone(), cache.clone())
    assert want[0].isfinite().all() and want[0].abs().sum() > 0
    graph = torch.cuda.CUDAGraph()
    nm.nm_set_programmatic_launch(True)
    try:
        for _ in range(3):
            cache.zero_()
            run_all()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (h, o, cache)))
        with torch.cuda.graph(graph):
            run_all()
    finally:
        nm.nm_set_programmatic_launch(False)
    for _ in range(3):
        cache.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (h, o, cache)))
    nm.nm_check_status()


def test_refusals():
    import paper_2609_16009_b200 as nm
    vp, lib = ctypes.c_void_p, nm._lib
    need = nm.nm_mla_attention_q8_workspace_bytes(2, 16)
    assert need > 0 and nm.nm_mla_attention_q8_workspace_bytes(0, 16) == 0 and nm.nm_mla_attention_q8_workspace_bytes(65, 16) == 0
    assert nm.nm_mla_attention_q8_workspace_bytes(1, 129) == 0

    def call(Q=256, qs=16 * 576, pre=4096, n_pre=5, cache=8192, cs=656 * 10, lens=(3, 4), o16=512, o32=1024, lse=2048, T=None, H=16, kv=512, rope=64, ws=65536, wb=need):
        arr = (ctypes.c_int * max(len(lens), 1))(*lens) if lens is not None else None
        return lib.nm_mla_attention_q8(vp(Q), qs, vp(pre), n_pre, vp(cache), cs, arr, vp(o16), vp(o32), vp(lse), len(lens) if T is None else T, H, kv, rope, 0.1,
                                       vp(ws), wb, None)

    for bad in (dict(Q=None), dict(lens=None, T=2), dict(T=0), dict(lens=(1,) * 65), dict(H=0), dict(n_pre=-1), dict(pre=None), dict(lens=(3, -1)), dict(cache=None),
                dict(lens=(3, 11)), dict(qs=16 * 576 - 8), dict(n_pre=(1 << 30) + 1)):
        assert call(**bad) == -1, bad
    for bad in (dict(kv=256), dict(rope=32), dict(H=129, qs=129 * 576)):
        assert call(**bad) == -2, bad
    for bad in (dict(Q=264), dict(qs=16 * 576 + 4), dict(pre=4104), dict(cache=8200), dict(cs=6568), dict(o16=516), dict(o32=1032), dict(lse=2050), dict(ws=65544)):
        assert call(**bad) == -3, bad
    for bad in (dict(ws=None), dict(wb=need - 1)):
        assert call(**bad) == -4, bad


def test_the_decoder_of_this_file_knows_the_format():
    every = torch.arange(256, dtype=torch.uint8)
    ref = every.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(e4m3_value(every.numpy()), ref, equal_nan=True)
