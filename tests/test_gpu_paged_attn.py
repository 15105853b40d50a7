"""paged_attn_forward on the GPU against the definition in float64."""
import numpy as np
import pytest

from tests.sampling_util import Paged, gpu, host, round_to

pytestmark = pytest.mark.gpu

CASES = {
    # name: dtype, heads, D, page, lens, new, shared
    "one_key": ("bf16", (1, 1), 64, 16, [1], [1], 0),
    "one_token": ("bf16", (28, 4), 128, 16, [1100], [1], 0),
    "tokens_ragged": ("bf16", (28, 4), 128, 64, [1, 63, 64, 65, 700, 2049], [1] * 6, 0),
    "tokens_d64": ("bf16", (14, 2), 64, 32, [5, 1000, 333], [1] * 3, 0),
    "tokens_wide_group": ("bf16", (40, 1), 128, 128, [300, 77], [1, 1], 0),
    "idle_sequences": ("bf16", (8, 2), 128, 64, [200, 0, 900, 64, 31], [1, 0, 1, 0, 1], 0),
    "few_tokens": ("bf16", (28, 4), 128, 16, [130, 17, 4, 555], [4, 3, 4, 2], 0),
    "more_tokens": ("bf16", (12, 2), 128, 32, [130, 517], [7, 9], 0),
    "chunk": ("bf16", (28, 4), 128, 64, [700], [333], 0),
    "chunk_from_nothing": ("bf16", (4, 4), 64, 16, [401], [401], 0),
    "chunk_d64": ("bf16", (14, 2), 64, 64, [1500, 90], [130, 90], 0),
    "mixed": ("bf16", (28, 4), 128, 64, [600, 311, 64, 900, 100], [200, 1, 1, 77, 100], 0),
    "many_chunks": ("bf16", (4, 1), 64, 16, [20 + i % 21 for i in range(600)], [17] * 600, 0),
    "tokens_of_two_blocks": ("bf16", (32, 2), 128, 64, [700, 65], [2, 1], 0),
    "many_sequences": ("bf16", (2, 2), 64, 16, list(range(1, 301)), [1] * 300, 0),
    "shared": ("bf16", (28, 4), 128, 64, [1050, 1100, 1025, 1400], [1] * 4, 1024),
    "shared_few": ("bf16", (14, 2), 64, 16, [700, 660, 671], [4, 1, 3], 640),
    "shared_chunk": ("bf16", (8, 2), 128, 32, [700, 460], [200, 40], 320),
    "wide_group_chunk": ("bf16", (300, 1), 64, 16, [90, 40], [2, 1], 0),   # a token's rows fill more than a block
    "f32_wide_group": ("f32", (40, 1), 64, 16, [90, 40], [2, 1], 0),
    "f32_token": ("f32", (8, 2), 128, 16, [1, 600, 130], [1] * 3, 0),
    "f32_chunk": ("f32", (8, 2), 128, 32, [330, 100], [130, 100], 0),
    "f32_d64": ("f32", (14, 2), 64, 64, [500, 65], [9, 1], 0),
    "f32_shared": ("f32", (4, 4), 64, 16, [400, 350, 321], [1, 2, 1], 320),
}


@pytest.mark.parametrize("name", CASES)
def test_attention_is_the_definition(name):
    dtype, heads, dim, page, lens, new, shared = CASES[name]
    x = Paged(dtype, heads, dim, page, lens, new, shared, pad=3, seed=sorted(CASES).index(name))
    want = x.oracle()
    x.check(*x.attend(), want)
    if shared:
        x.check(*x.attend(shared_len=shared + page // 2), want)   # rounded down to whole pages
        x.check(*x.attend(shared_len=page), want)


@pytest.mark.parametrize("heads,dim,page,lens,new", [((28, 4), 128, 64, [900, 2500, 70, 1300, 4100], [1, 400, 18, 1, 19]),
                                                     ((14, 2), 64, 32, [3000, 700, 900, 5000, 33], [1, 300, 1, 9, 2])])
@pytest.mark.parametrize("late", [False, True])
def test_tokens_beside_a_chunk(heads, dim, page, lens, new, late):
    """Blocks of few rows, in which some wavefronts have none, in a call of chunks; `late`: with scores of hundreds, the largest last."""
    x = Paged("bf16", heads, dim, page, lens, new, pad=3, seed=30 + late)
    if late:
        grow = np.zeros((x.pages, 1, x.page, 1))
        for b, n in enumerate(x.lens):
            for j in range(n):
                grow[x.table[b, j // x.page], 0, j % x.page, 0] = 8.0 * j / n
        x.k = round_to(x.k * grow, "bf16")
        x.q = round_to(x.q * 4.0, "bf16")
    x.check(*x.attend())


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("new", [[1, 1, 1], [90, 3, 1]])
def test_nothing_behind_the_last_key_reaches_a_result(dtype, dim, new):
    """Keys and values that no row sees, in pages in use and others, are NaN and infinity."""
    x = Paged(dtype, (8, 2), dim, 32, [100, 33, 257], new, seed=6)
    want = x.oracle()
    used = np.zeros((x.pages, x.page), dtype=bool)
    for b, n in enumerate(x.lens):
        for j in range(n):
            used[x.table[b, j // x.page], j % x.page] = True
    hole = ~used[:, None, :, None]
    x.k = np.where(hole, np.nan, x.k)
    x.v = np.where(hole, np.inf, x.v)
    x.check(*x.attend(), want)


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("new", [[1, 1, 1, 1, 1], [70, 1, 33, 40, 2], [70, 31, 33, 40, 60]])
def test_rows_without_keys_and_keys_without_pages(dtype, dim, new):
    """A sequence shorter than its new tokens: zeros and -inf; a missing page, a length beyond the table: NaN for the rows that see it only."""
    lens = [50 if new[0] > 1 else 0, 300, 40, 45, 70]
    x = Paged(dtype, (16, 2) if dtype == "bf16" else (4, 2), dim, 16, lens, new, pad=2, seed=7, wide=0)
    x.lens[0] = 45 if new[0] > 1 else 0       # 70 new tokens, 45 in all: 25 rows see nothing
    x.table[1, 3] = -5
    x.table[2, 1] = x.pages
    x.table[3, :] = np.where(np.arange(x.table.shape[1]) < 3, x.table[3], -1)
    x.lens[4] = x.table.shape[1] * 16 + 9
    out, lse = x.attend()
    want = x.oracle()
    x.check(out, lse, want)
    lost = np.isnan(want[0]).all(axis=(1, 2))
    lost[x.cu[-1]:] = False
    assert lost.any() and np.isnan(out[lost]).all() and np.isnan(lse[:, lost]).all()
    if new[0] > 1:
        assert np.isneginf(lse[:, :25]).all() and (out[:25] == 0).all()
    assert np.isneginf(lse[:, 0]).all()


@pytest.mark.parametrize("dtype,dim,new", [("bf16", 64, 1), ("bf16", 64, 120), ("f32", 64, 5), ("bf16", 128, 12), ("bf16", 128, 30), ("bf16", 128, 150)])
def test_large_and_late_scores(dtype, dim, new):
    """Scores of hundreds, the largest last: the running maximum moves at every tile, and chunks are done again with their true maxima."""
    x = Paged(dtype, (4, 2), dim, 64, [800, 330], [new, new], seed=8)
    grow = np.zeros((x.pages, 1, x.page, 1))
    for b, n in enumerate(x.lens):
        for j in range(n):
            grow[x.table[b, j // x.page], 0, j % x.page, 0] = 8.0 * j / n
    from tests.sampling_util import round_to
    x.k = round_to(x.k * grow, dtype)
    x.q = round_to(x.q * 4.0, dtype)
    x.check(*x.attend())


def test_strided_queries_and_no_lse():
    import torch
    import paper_2507_07966_amd as pa
    x = Paged("bf16", (8, 2), 128, 32, [100, 400], [3, 2], seed=9)
    fused = torch.randn(x.tokens, 12, 128, device="cuda").bfloat16()
    fused[:, :8] = gpu(x.q, "bf16")
    out, lse = x.attend(q=fused[:, :8])
    x.check(out, lse)
    plan = x.plan()
    o = torch.empty(x.tokens, 8, 128, device="cuda", dtype=torch.bfloat16)
    pa.paged_attn_forward(plan, fused[:, :8], *x.upload(), o, None, torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda"))
    assert np.array_equal(host(o), out)
    plan.destroy()


def test_bad_lengths_stay_inside_the_rows():
    """cu_new and seq_lens that make no sense: other rows keep their results, nothing outside the packed rows is written."""
    x = Paged("bf16", (4, 2), 64, 16, [100, 50], [2, 3], pad=4, seed=10)
    good = x.attend()
    x.cu = np.array([0, 2, 1000], dtype=np.int32)   # the second sequence is said to reach far behind the rows
    x.lens[1] = -7
    out, lse = x.attend()
    assert np.array_equal(out[:2], good[0][:2]) and np.array_equal(lse[:, :2], good[1][:, :2])
    assert np.isneginf(lse[:, 2:]).all() and (out[2:] == 0).all()


@pytest.mark.parametrize("dtype,lens,new,shared", [("bf16", [900, 300, 1], [1, 1, 1], 0), ("bf16", [900, 300], [150, 40], 0),
                                                   ("bf16", [900, 800], [1, 1], 512), ("f32", [500, 100], [3, 1], 0)])
def test_a_captured_call_follows_the_lengths(dtype, lens, new, shared):
    """Captured once and replayed on other lengths, tables and queries, with the program's own work between: every replay is the eager call bit for bit."""
    import torch
    import paper_2507_07966_amd as pa
    x = Paged(dtype, (8, 2), 64, 32, lens, new, shared, seed=11, wide=4)
    plan = x.plan()
    q, dev = gpu(x.q, dtype), list(x.upload())
    out, lse = torch.zeros_like(q), torch.zeros(8, x.tokens, device="cuda")
    ws = torch.zeros(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    sh = gpu(np.array([shared], dtype=np.int32)) if shared else None
    call = lambda o, l: pa.paged_attn_forward(plan, q, *dev, o, l, ws, shared_len=sh)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, lse)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse)
    rng = np.random.default_rng(12)
    for step in range(3):
        q.copy_(gpu(rng.standard_normal(x.q.shape), dtype))
        dev[3].copy_(gpu((x.lens - step * (x.lens > 40) * 7).astype(np.int32)))
        if step == 2 and shared:
            sh.fill_(shared // 2)
        eager = torch.zeros_like(out), torch.zeros_like(lse)
        call(*eager)
        torch.cuda.synchronize()
        ws.fill_(0x7f)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
    plan.destroy()


def test_two_streams_with_workspaces_of_their_own():
    import torch
    import paper_2507_07966_amd as pa
    x = Paged("bf16", (28, 4), 128, 64, [5000, 3500, 900], [1, 1, 1], seed=13)
    plan, dev = x.plan(), x.upload()
    streams = [torch.cuda.Stream() for _ in range(2)]
    qs = [torch.randn(x.tokens, 28, 128, device="cuda").bfloat16() for _ in streams]
    wss = [torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda") for _ in streams]
    want = [torch.empty_like(qs[0]) for _ in streams]
    for i in range(2):
        pa.paged_attn_forward(plan, qs[i], *dev, want[i], None, wss[i])
    got = [torch.zeros_like(qs[0]) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            pa.paged_attn_forward(plan, qs[i], *dev, got[i], None, wss[i], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    plan.destroy()


def test_results_are_reproducible():
    x = Paged("bf16", (28, 4), 128, 64, [9000, 333, 4000], [1, 1, 1], seed=14)
    y = Paged("bf16", (28, 4), 128, 64, [2000, 900], [260, 200], seed=15)
    for z in (x, y):
        a, b = z.attend(), z.attend()
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_lengths_that_fall_and_empty_calls_compute_nothing():
    import torch
    import paper_2507_07966_amd as pa
    for shared in (None, 16):
        x = Paged("bf16", (4, 2), 64, 16, [100, 50, 70], [2, 3, 1], seed=16)
        x.cu = np.array([0, 4, 2, 6], dtype=np.int32)
        out, lse = x.attend(shared_len=shared)
        assert (out == 7).all() and (lse == 7).all()
    plan = x.plan()
    dev = x.upload()
    out = torch.full((0, 4, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    pa.paged_attn_forward(plan, out, *dev, out, None, torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda"))
    q = torch.full((3, 4, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    none = dev[0], dev[1], dev[2][:0], dev[3][:0], dev[4][:1]
    pa.paged_attn_forward(plan, q, *none, q, None, torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert (q == 7).all()
    plan.destroy()


@pytest.mark.parametrize("dtype,new", [("bf16", [1, 1]), ("bf16", [90, 40]), ("f32", [1, 2])])
def test_caches_beyond_four_gibibytes(dtype, new):
    """Pages at the end of caches of more than 2^32 bytes each, appended to and read."""
    import torch
    import paper_2507_07966_amd as pa
    x = Paged(dtype, (8, 2), 128, 64, [200, 130], new, seed=17)
    size = 2 if dtype == "bf16" else 4
    many = (1 << 32) // (2 * 64 * 128 * size) + x.pages + 5
    shift = many - x.pages
    plan = x.plan(num_pages=many)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    kc, vc = (torch.empty(many, 2, 64, 128, dtype=tdt, device="cuda") for _ in range(2))
    kc[shift:], vc[shift:] = gpu(x.k, dtype), gpu(x.v, dtype)
    rows = [(t, b, int(x.lens[b] - x.cu[b + 1] + t)) for b in range(2) for t in range(x.cu[b], x.cu[b + 1])]
    k = np.stack([x.k[x.table[b, p // 64], :, p % 64] for _, b, p in rows])
    v = np.stack([x.v[x.table[b, p // 64], :, p % 64] for _, b, p in rows])
    for _, b, p in rows:   # wiped, and appended again
        kc[shift + int(x.table[b, p // 64]), :, p % 64] = 9
        vc[shift + int(x.table[b, p // 64]), :, p % 64] = 9
    table = gpu(np.where(x.table >= 0, x.table + shift, -1).astype(np.int32))
    args = kc, vc, table, gpu(x.lens), gpu(x.cu)
    pa.paged_kv_append(plan, gpu(k, dtype), gpu(v, dtype), *args)
    out, lse = torch.empty(x.tokens, 8, 128, dtype=tdt, device="cuda"), torch.empty(8, x.tokens, device="cuda")
    pa.paged_attn_forward(plan, gpu(x.q, dtype), *args, out, lse, torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda"))
    assert np.array_equal(host(kc[shift:]), x.k) and np.array_equal(host(vc[shift:]), x.v)
    x.check(host(out), host(lse))
    plan.destroy()
