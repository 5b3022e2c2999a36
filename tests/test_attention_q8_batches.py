"""The quantised attention at the sizes of a decode batch: more heads than the merge gives four threads a column, pairs of CTAs that walk over several
items of several tiles, and queries with an outlier; and the rotated part of the rows that a decode step writes.  Against 64 bits."""
import numpy as np
import pytest
import torch

import oracle
from test_attention_q8 import KV, REC, ROPE, SCALE, case, check, run
from test_cache_q8 import records


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,prefix,lens", [
    (10, 128, 0, [700 - 30 * t for t in range(10)]),               # 1280 query rows: one thread a column in the merge; one tile an item
    (64, 128, 200, [30 * (t % 7) for t in range(64)]),             # 8192 query rows; items of 3 and 2, 1 and 3, 1, 2 and 1 tiles on a pair
    (16, 128, 3000, [100 + 37 * t for t in range(16)]),            # items of 10 and 12 tiles, 2 and 3 on a pair; a start worth three tiles
    (16, 128, 12000, [150] * 16),                                  # items of 9 and 17 tiles on a pair, six of 2, 9 and four of 2
    (12, 100, 700, [97 * t for t in range(12)])])                  # query tiles that end inside a sequence's heads
def test_batches(T, H, prefix, lens):
    import paper_2609_16009_b200 as nm
    Q, pre, own = case(T, H, prefix, lens, T + H + prefix)
    check(Q, SCALE, pre, own, *run(nm, Q, SCALE, pre, own))


@pytest.mark.gpu
def test_maxima_that_move_in_a_later_item():
    """Sharp scores over several items of several tiles: O is rescaled in the second item and beyond."""
    import paper_2609_16009_b200 as nm
    Q, pre, own = case(16, 128, 3000, [100 + 37 * t for t in range(16)], 77, std=8.0)
    check(Q, SCALE, pre, own, *run(nm, Q, SCALE, pre, own))


@pytest.mark.gpu
@pytest.mark.parametrize("outlier", [64.0, 256.0])
def test_a_head_with_an_outlier(outlier):
    """One query element far above the others, over cache rows that are zero there: what the others lose beside it is all that shows."""
    import paper_2609_16009_b200 as nm
    Q, pre, own = case(2, 24, 100, [300, 40], 9)
    for rec in (pre, *own):
        rec[:, 3] = 0
    plain = run(nm, Q, SCALE, pre, own)
    Q[1, :, 3] = outlier
    got = run(nm, Q, SCALE, pre, own)
    check(Q, SCALE, pre, own, *got)
    assert all(np.array_equal(a[0], b[0]) for a, b in zip(plain, got)), "the other sequence's queries have exponents of their own"


@pytest.mark.gpu
def test_the_rotated_part_of_rows_written_by_a_step():
    """Key parts rotated by rows of nm_rope_table for the sequences' own positions, as a decode step writes them."""
    import paper_2609_16009_b200 as nm
    T, first = 7, 30000
    positions = [first + 13 * t for t in range(T)]
    x = torch.randn(T, KV + ROPE, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    table = torch.zeros(13 * T, ROPE, device="cuda")
    nm.nm_rope_table(table, first, 13 * T, ROPE)
    cs = table[::13].contiguous()
    cache = torch.zeros(T, REC, dtype=torch.uint8, device="cuda")
    nm.nm_mla_cache_write_q8(x.cuda(), torch.ones(KV, dtype=torch.bfloat16, device="cuda"), cs, None, cache, T, T, KV, ROPE)
    _, key, s = records(cache.cpu().numpy(), KV, ROPE)
    k = x[:, KV:].double().numpy()
    want = np.stack([oracle.rope(k[t], positions[t]) for t in range(T)])
    # half a step of bf16, 2^-8; the table's own rounding of cosine and sine, 2^-23, and two fp32 products of the pair before it
    size = np.repeat(np.abs(k).reshape(T, ROPE // 2, 2).sum(2), 2, axis=1)
    assert np.all(np.abs(key * s - want) <= 2.0 ** -8 * np.abs(want) + size * (2.0 ** -23 + 2.0 ** -22))
