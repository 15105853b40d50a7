"""The division of paged_attn_forward among workgroups, on the CPU by the functions that the kernels use: every visible (row, key) pair is covered
exactly once, shares are balanced, cuts fall on tiles, and no length makes the schedule leave its bounds."""
import numpy as np
import pytest

import paper_2507_07966_amd as pa


def plan(dtype="bf16", heads=(28, 4), dim=128, page=64, width=600, seqs=64, tokens=8192):
    return pa.paged_attn_plan(*heads, dim, page, 100000, width, seqs, tokens, 0.1, dtype=dtype, device=-1)


def check(p, lens, new, shared=-1, balanced=True):
    lens, cu = np.asarray(lens, dtype=np.int64), np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    tokens = int(cu[-1])
    group, cap, page = p.num_q_heads // p.num_kv_heads, p.max_pages_per_seq * p.page_size, p.page_size
    groups, block, tile = p.schedule_shape(len(lens), tokens, shared >= 0)
    pieces = p.schedule(lens, cu, tokens, shared)
    used = max(0, min(shared, cap)) // page * page if (pieces[:, 1] == -1).any() else 0
    first = lens - np.diff(cu)
    cover, load = {}, np.zeros(groups, dtype=np.int64)
    for share, b, c, row0, rows, k0, k1, whole in pieces.tolist():
        assert 0 <= share < groups and 0 <= c < p.num_kv_heads and row0 % block == 0 and 1 <= rows <= block
        total = (tokens if b < 0 else cu[b + 1] - cu[b]) * group
        assert row0 + rows == min(row0 + block, total)
        key0 = 0 if b < 0 else used
        assert k0 >= key0 and (k0 - key0) % tile == 0 and k1 >= k0 - tile
        cover.setdefault((b, c, row0), []).append((share, k0, max(k0, k1), whole))
        load[share] += max(0, k1 - k0)
    for b in range(-1 if used else 0, len(lens)):
        n = tokens if b < 0 else int(cu[b + 1] - cu[b])
        for c in range(p.num_kv_heads):
            for row0 in range(0, n * group, block):
                last = (min(row0 + block, n * group) - 1) // group
                end = used if b < 0 else max(used, min(cap + 1, max(0, int(first[b]) + last + 1)))
                parts = cover.pop((b, c, row0))
                assert len(parts) == 1 or not any(w for *_, w in parts)
                assert [s for s, *_ in parts] == list(range(parts[0][0], parts[0][0] + len(parts)))   # consecutive shares
                at = 0 if b < 0 else used
                for _, k0, k1, _ in parts:
                    if k1 > k0:
                        assert k0 == at
                        at = k1
                assert at == end, (b, c, row0, parts, end)
    assert not cover
    return pieces, load


CASES = [
    ("bf16", (28, 4), 128, [1100], [1], -1), ("bf16", (28, 4), 128, [1] * 40, [1] * 40, -1), ("bf16", (28, 4), 128, [33000 + 100 * i for i in range(8)], [1] * 8, 32768),
    ("bf16", (28, 4), 128, [700 + 250 * i for i in range(60)], [1] * 60, -1), ("bf16", (28, 4), 128, [34816], [2048], -1), ("bf16", (28, 4), 128, [2500], [2500], -1),
    ("bf16", (14, 2), 64, [400, 9000, 0, 77, 5000], [300, 1, 0, 77, 200], -1), ("f32", (8, 2), 128, [200, 4100, 3000], [130, 3, 77], -1),
    ("f32", (4, 4), 64, [400, 350, 321], [1, 2, 1], 320), ("bf16", (40, 1), 128, [300, 77], [1, 1], -1), ("bf16", (600, 1), 64, [900, 12], [3, 12], -1),
    ("bf16", (28, 4), 128, [50, 3, 20], [70, 3, 30], -1), ("bf16", (8, 8), 128, [38400, 39000], [1, 1], -1), ("bf16", (8, 2), 128, [100, 700], [1, 1], 64),
    ("bf16", (28, 4), 128, [9000, 7000, 3100, 8200, 40, 6000], [1, 18, 900, 19, 1, 400], -1),   # blocks of half the cost beside whole ones
    ("bf16", (14, 2), 64, [9000 + 17 * i for i in range(30)], [2000] + [1] * 29, -1),
]


@pytest.mark.parametrize("dtype,heads,dim,lens,new,shared", CASES)
def test_every_pair_is_covered_once(dtype, heads, dim, lens, new, shared):
    p = plan(dtype, heads, dim)
    check(p, lens, new, shared)
    p.destroy()


def test_random_calls():
    rng = np.random.default_rng(0)
    for i in range(120):
        hkv = int(rng.choice([1, 2, 4, 8]))
        p = plan(str(rng.choice(["bf16", "f32"])), (hkv * int(rng.choice([1, 4, 7, 20])), hkv), int(rng.choice([64, 128])),
                 page=int(rng.choice([16, 64, 256])), width=int(rng.integers(1, 200)), seqs=400)
        n = int(np.exp(rng.uniform(0, np.log(400))))
        new = rng.integers(0, max(2, int(np.exp(rng.uniform(0, np.log(8192 / n))))), size=n)
        new = new if new.any() else new + 1
        lens = new + np.exp(rng.uniform(0, np.log(20000), size=n)).astype(np.int64) - rng.integers(0, 3, size=n) * new
        check(p, lens, new, int(rng.integers(0, 2000)) if i % 3 == 0 else -1)
        p.destroy()


def test_shares_are_balanced():
    p = plan()
    for lens, new in (([700 + 250 * i for i in range(64)], [1] * 64), ([34816], [2048]), ([120000 // 4], [1])):
        _, load = check(p, lens, new)
        assert load.max() <= 1.2 * load.sum() / len(load) + 512
    p.destroy()


def test_lengths_that_make_no_sense_stay_in_bounds():
    """cu_new that falls, starts below 0 or ends behind the rows, and lengths of any size: shares, heads, rows and keys stay in range."""
    rng = np.random.default_rng(1)
    big = (1 << 31) - 1
    for i in range(200):
        p = plan("bf16" if i % 2 else "f32", (7, 1), 64, page=16, width=int(rng.integers(1, 50)), seqs=16, tokens=500)
        n, tokens = int(rng.integers(1, 17)), int(rng.integers(1, 501))
        cu = rng.choice([0, -5, big, -big, 100, 499, 3, tokens], size=n + 1)
        lens = rng.choice([0, -1, big, -big, 100, 5000, 17], size=n)
        cap = p.max_pages_per_seq * 16
        groups, block, _ = p.schedule_shape(n, tokens, True)
        for share, b, c, row0, rows, k0, k1, _ in p.schedule(lens, cu, tokens, int(rng.choice([-1, 0, big, 100]))).tolist():
            lo, hi = (0, min(max(int(cu[n]), 0), tokens)) if b < 0 else (min(max(int(cu[b]), 0), tokens), min(max(int(cu[b + 1]), 0), tokens))
            assert 0 <= share < groups and c == 0 and 0 <= row0 and 1 <= rows <= block and row0 + rows <= (hi - lo) * 7
            assert 0 <= k0 and k1 <= cap + 1
        p.destroy()


def test_schedule_refuses():
    p = plan(seqs=4, tokens=10)
    for lens, tokens in (([1] * 5, 5), ([1], 11), ([1], 0)):
        with pytest.raises(pa.PrefixAttnError):
            p.schedule(lens, np.arange(len(lens) + 1), tokens)
    p.destroy()
