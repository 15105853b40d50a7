"""The division of paged_attn_forward among workgroups: shares are alike, by the tiles of keys that they load, also where the new tokens themselves are most of the
keys (fp32 and wide groups, whose blocks have few tokens, prefills from nothing, chunks of several lengths), and what PagedAttnPlan.schedule refuses."""
import numpy as np
import pytest

import paper_2507_07966_amd as pa

CALLS = [
    ("f32", (8, 2), 128, [2100], [2048]), ("f32", (28, 4), 128, [1300], [1200]), ("f32", (14, 2), 64, [2000], [1900]),
    ("f32", (8, 2), 128, [4096], [4096]), ("f32", (32, 1), 128, [2048], [2048]), ("f32", (8, 8), 64, [2900, 700], [2900, 650]),
    ("bf16", (32, 1), 128, [4096], [4096]), ("bf16", (40, 1), 128, [4096], [4096]), ("bf16", (28, 4), 128, [8192], [8192]),
    ("bf16", (300, 1), 64, [2999], [2999]), ("bf16", (14, 2), 64, [3000, 900, 77, 4000], [3000, 900, 77, 4000]),
    ("bf16", (28, 4), 128, [34816], [2048]),
]


@pytest.mark.parametrize("dtype,heads,dim,lens,new", CALLS, ids=lambda v: "-".join(map(str, v)) if isinstance(v, (tuple, list)) else str(v))
def test_shares_of_prefills_are_balanced(dtype, heads, dim, lens, new):
    tokens, page = sum(new), 64
    p = pa.paged_attn_plan(*heads, dim, page, 100000, -(-max(lens) // page), len(lens), tokens, 0.1, dtype=dtype, device=-1)
    groups, _, tile = p.schedule_shape(len(lens), tokens)
    pieces = p.schedule(lens, np.concatenate([[0], np.cumsum(new)]), tokens)
    p.destroy()
    tiles = np.maximum(0, -(-(pieces[:, 6] - pieces[:, 5]) // tile))
    load = np.bincount(pieces[:, 0], weights=tiles, minlength=groups)
    # A share of w keys' cost has at most w / tile tiles and one more for each end that rounding moves.  It holds that many where it starts no block, and by
    # up to 384 keys (start_keys of the chunks, the larger) fewer for each block that it starts: 384 / tile above the mean, where that mean is of shares
    # that start one each.  15 % for what is not worth counting: blocks' last, partly visible tiles.
    most = 1.15 * load.mean() + 384 / tile + 2
    print(f"most {load.max():.0f} of a mean of {load.mean():.1f}, bound {most:.1f}")
    assert load.max() <= most


@pytest.mark.parametrize("lens,cu,tokens,shared,status", [
    ([50, 60], [0, 1], 2, -1, 2), ([50, 60], [0], 2, -1, 2), ([50], [0, 1, 2], 2, -1, 2), ([50], 1, 1, -1, 2), ([[50]], [[0, 1]], 1, -1, 2),
    ([], [], 1, -1, 2), ([1 << 32], [0, 1], 1, -1, 2), ([50], [0, 1 << 31], 1, -1, 2), ([50], [0, 1], 1 << 64, -1, 3), ([50], [0, 1], 1 << 33, -1, 2),
    ([50], [0, 1], 1, 1 << 32, 2), ([50.5], [0, 1], 1, -1, 3), ([50], [0, 1], 1.0, -1, 3),
])
def test_schedule_refuses_arrays_that_do_not_fit(lens, cu, tokens, shared, status):
    """The library reads n lengths and n + 1 ends: shorter arrays were read beyond their end, and wider numbers wrapped."""
    p = pa.paged_attn_plan(4, 2, 64, 16, 100, 8, 8, 64, 0.1, device=-1)
    with pytest.raises(pa.PrefixAttnError) as e:
        p.schedule(lens, cu, tokens, shared)
    assert e.value.status == status
    assert len(p.schedule(np.array([50, 7]), np.array([0, 1, 2]), 2)) > 0
    p.destroy()


def test_numbers_beyond_32_bits_do_not_wrap():
    for head_dim in ((1 << 32) + 64, (1 << 64) + 64, 64 - (1 << 32)):   # each is 64 in 32 bits
        with pytest.raises(pa.PrefixAttnError):
            pa.rope_axes((32,), head_dim, rotary_dim=64)
    p = pa.paged_attn_plan(4, 2, 64, 16, 100, 8, 8, 64, 0.1, device=-1)
    for seqs, tokens in (((1 << 32) + 1, 1), (1, (1 << 64) + 1), (9, 1), (1, 65), (0, 1), (1, 0)):
        with pytest.raises(pa.PrefixAttnError) as e:
            p.schedule_shape(seqs, tokens)
        assert e.value.status == 2
    assert p.schedule_shape(8, 64) and p.schedule_shape(1, 1)
    p.destroy()


@pytest.mark.parametrize("dtype,heads,new,shares", [
    ("bf16", (28, 4), 1, True), ("bf16", (28, 4), 8, True), ("bf16", (28, 4), 9, False), ("bf16", (28, 4), 10, False),
    ("bf16", (4, 4), 56, True), ("bf16", (4, 4), 57, False), ("f32", (8, 2), 14, True), ("f32", (8, 2), 16, False),
])
def test_shared_keys_are_a_segment_where_that_saves_passes(dtype, heads, new, shares):
    """Up to 56 rows a sequence: fuller blocks of one sequence's rows lose more than they save (63 rows: 132 us shared, 110 not)."""
    lens, cu = [9000 + 10 * i for i in range(8)], np.arange(9) * new
    p = pa.paged_attn_plan(*heads, 128, 64, 100000, 150, 8, 8 * new, 0.1, dtype=dtype, device=-1)
    assert (p.schedule(lens, cu, 8 * new, 8192)[:, 1] == -1).any() == shares
    p.destroy()
