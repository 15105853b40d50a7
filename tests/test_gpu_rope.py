"""rope_axes_forward / _backward and paged_kv_append(_rope) on the GPU against the definitions in float64."""
import numpy as np
import pytest

from oracle import ref_sampling as ref
from tests.sampling_util import STEP, U32, Paged, gpu, host, round_to

pytestmark = pytest.mark.gpu


def bound(x, y, pair_axis, positions, inv_freq, layout, dtype):
    """Error of one turned element: sine and cosine err by at most 4 units of 2^-24 (the reduced angle, |x| <= pi / 4, by three
    roundings, the polynomial by 1.5; the first left-out terms are far below) and by 2^-52 of the angle; two products and their sum round three more times;
    then one rounding to the data type."""
    n = len(pair_axis)
    both = np.abs(x).astype(np.float64)
    out = STEP[dtype] * np.abs(y)
    for i in range(n):
        a, b = (i, i + n) if layout == "halves" else (2 * i, 2 * i + 1)
        angle = np.abs(positions[pair_axis[i]].astype(np.float64) * inv_freq[i])[:, None]
        e = (both[:, :, a] + both[:, :, b]) * (7 * U32 + 4 * 2.0 ** -52 * angle)
        out[:, :, a] += e
        out[:, :, b] += e
    return out * (1 + 2.0 ** -7)


CASES = [  # dtype, T, Hq, Hk, D, rotary, sections, layout, interleaved
    ("bf16", 1, 28, 4, 128, 128, (16, 24, 24), "halves", False),
    ("bf16", 37, 28, 4, 128, 128, (24, 20, 20), "halves", True),
    ("bf16", 301, 14, 2, 64, 46, (11, 12), "halves", False),       # an odd number of pairs: vectors and single ones
    ("bf16", 300, 5, 1, 80, 80, (20, 20), "halves", False),
    ("bf16", 65, 3, 0, 72, 26, (5, 4, 3, 1), "pairs", True),       # no k, pairs that end inside a vector
    ("bf16", 9, 2, 2, 9, 2, (1,), "halves", False),                # an odd head, one pair
    ("bf16", 3000, 28, 4, 128, 128, (16, 24, 24), "pairs", False),  # several heads to a thread
    ("bf16", 2111, 28, 4, 128, 118, (16, 24, 19), "halves", False),
    ("bf16", 8300, 28, 4, 128, 118, (16, 24, 19), "halves", False),  # more heads to a thread
    ("f32", 1, 8, 2, 128, 128, (64,), "halves", False),
    ("f32", 77, 14, 2, 64, 46, (11, 12), "pairs", False),
    ("f32", 130, 3, 1, 256, 256, (0, 100, 28), "halves", True),
    ("f32", 2500, 14, 2, 64, 50, (9, 8, 8), "halves", False),
    ("f32", 33, 1, 1, 2, 2, (1,), "pairs", False),
]


def make(case, seed=0, far=1 << 20):
    import paper_2507_07966_amd as pa
    dtype, T, Hq, Hk, D, R, sections, layout, inter = case
    rng = np.random.default_rng(seed)
    rope = pa.rope_axes(sections, D, rotary_dim=R, layout=layout, interleaved=inter)
    pos = rng.integers(-far, far, size=(len(sections), T)).astype(np.int32)
    freq = (10000.0 ** (-np.arange(R // 2) / (R // 2))).astype(np.float32)
    return rope, pos, freq, round_to(rng.standard_normal((T, Hq, D)), dtype), round_to(rng.standard_normal((T, Hk, D)), dtype)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}x{c[2]}+{c[3]}x{c[4]}-{c[5]}-{c[7]}")
def test_rope_is_the_definition(case, backward):
    import torch
    import paper_2507_07966_amd as pa
    dtype, T, Hq, Hk, D = case[:5]
    rope, pos, freq, q, k = make(case)
    qd, kd = gpu(q, dtype), gpu(k, dtype) if Hk else None
    qo, ko = torch.full_like(qd, 7), torch.full_like(kd, 7) if Hk else None
    call = pa.rope_axes_backward if backward else pa.rope_axes_forward
    call(rope, qd, kd, gpu(pos), gpu(freq), qo, ko)
    for x, y in ((q, qo), (k, ko)):
        if y is None:
            continue
        want = ref.rope(x, pos, freq, rope.pair_axis, rope.layout, -1.0 if backward else 1.0)
        err, most = np.abs(host(y) - want), bound(x, want, rope.pair_axis, pos, freq, rope.layout, dtype)
        print(f"error / bound {float((err / np.maximum(most, 1e-30)).max()):.3f}", flush=True)
        assert (err <= most).all()
        assert np.array_equal(host(y)[:, :, rope.rotary_dim:], x[:, :, rope.rotary_dim:])


@pytest.mark.parametrize("case", [CASES[1], CASES[2], CASES[10]], ids=lambda c: f"{c[0]}-{c[1]}")
def test_rope_of_slices_in_place_and_of_far_positions(case):
    """Slices of a fused projection that start at any element, results over the inputs, positions up to 2^31, and nothing beside the
    slices written."""
    import torch
    import paper_2507_07966_amd as pa
    dtype, T, Hq, Hk, D = case[:5]
    rope, pos, freq, q, k = make(case, seed=1, far=(1 << 31) - 1)
    width = (Hq + Hk + 1) * D + 3
    whole = torch.full((T, width), 7.0, device="cuda").to(gpu(q[:1], dtype).dtype)
    qs = whole.as_strided((T, Hq, D), (width, D, 1), 1)
    ks = whole.as_strided((T, Hk, D), (width, D, 1), 1 + Hq * D)
    qs.copy_(gpu(q, dtype))
    ks.copy_(gpu(k, dtype))
    pa.rope_axes_forward(rope, qs, ks, gpu(pos), gpu(freq), qs, ks)
    for x, y in ((q, qs), (k, ks)):
        want = ref.rope(x, pos, freq, rope.pair_axis, rope.layout)
        assert (np.abs(host(y) - want) <= bound(x, want, rope.pair_axis, pos, freq, rope.layout, dtype)).all()
    assert (whole[:, 0] == 7).all() and (whole[:, 1 + (Hq + Hk) * D:] == 7).all()


def test_rope_backward_is_the_gradient():
    """Against differences of the forward: L = <g, y(x)> is linear in x, so L(x + d) - L(x) = <dx, d> for any step."""
    import torch
    import paper_2507_07966_amd as pa
    case = ("f32", 21, 4, 2, 64, 46, (8, 8, 7), "halves", False)
    rope, pos, freq, q, k = make(case, seed=2)
    rng = np.random.default_rng(3)
    g, d = rng.standard_normal(q.shape).astype(np.float32), rng.standard_normal(q.shape).astype(np.float32)

    def loss(x):
        y = torch.empty(q.shape, device="cuda")
        pa.rope_axes_forward(rope, gpu(x, "f32"), None, gpu(pos), gpu(freq), y, None)
        return float((host(y) * g).sum())

    dx = torch.empty(q.shape, device="cuda")
    pa.rope_axes_backward(rope, gpu(g), None, gpu(pos), gpu(freq), dx, None)
    want, got = loss(q + d) - loss(q), float((host(dx) * d).sum())
    # each of the three rotations errs by at most 7 units (above) of (|x0| + |x1|), the sums here are in float64; the steps q + d are rounded once
    most = 8 * U32 * 2 * float((np.abs(g) * (np.abs(q + d) + np.abs(q) + np.abs(d)) * 2).sum())
    assert abs(want - got) <= most and abs(want) > 10 * most


def test_no_tokens_and_one_device():
    import torch
    import paper_2507_07966_amd as pa
    rope = pa.rope_axes((32,), 64)
    e = torch.empty(0, 4, 64, device="cuda")
    pa.rope_axes_forward(rope, e, None, torch.empty(1, 0, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda"), e, None)
    with pytest.raises(pa.PrefixAttnError):
        pa.rope_axes_forward(rope, e, None, torch.empty(1, 0, dtype=torch.int32), torch.ones(32, device="cuda"), e, None)


@pytest.mark.parametrize("dtype,heads,dim,page,lens,new,rotated", [
    ("bf16", (28, 4), 128, 64, [500, 64, 65, 2000], [1, 1, 1, 1], True),
    ("bf16", (28, 4), 128, 16, [40, 3, 0, 17, 33], [40, 3, 0, 2, 0], True),
    ("bf16", (14, 2), 64, 32, [1200, 900], [1100, 900], True),
    ("bf16", (28, 4), 128, 64, [7800, 900], [7600, 800], True),
    ("bf16", (4, 4), 64, 256, [300, 7], [290, 7], False),
    ("f32", (8, 2), 128, 16, [16, 1, 50], [16, 1, 35], True),
    ("f32", (2, 1), 64, 64, [130] * 300, [1] * 300, False),
])
def test_append_is_the_definition(dtype, heads, dim, page, lens, new, rotated):
    """New rows land in their slots, everything else in the caches keeps its bits, also behind the last sequence (5 padding rows) and where a token has no page."""
    import torch
    import paper_2507_07966_amd as pa
    x = Paged(dtype, heads, dim, page, lens, new, pad=5, seed=4)
    hq, hkv = heads
    rng = np.random.default_rng(5)
    if len(lens) > 1:
        x.table[1, 0] = -1                      # no page
        x.table[-1, -1] = x.pages               # nor this
    fused = round_to(rng.standard_normal((x.tokens, hq + 2 * hkv, dim)), dtype)
    q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    fd = gpu(fused, dtype)
    qd, kd, vd = fd[:, :hq], fd[:, hq:hq + hkv], fd[:, hq + hkv:]
    kc, vc, table, lens_d, cu = x.upload()
    plan = x.plan()
    kw = k
    if rotated:
        rope = pa.rope_axes((dim // 4, dim // 8, dim // 8 - 3), dim, rotary_dim=dim - 6)
        pos = rng.integers(0, 50000, size=(3, x.tokens)).astype(np.int32)
        freq = (10000.0 ** (-np.arange(dim // 2 - 3) / (dim // 2 - 3))).astype(np.float32)
        qo = torch.full((x.tokens, hq, dim), 7.0, device="cuda", dtype=fd.dtype)
        pa.paged_kv_append_rope(plan, rope, qd, kd, vd, gpu(pos), gpu(freq), qo, kc, vc, table, lens_d, cu)
        kw = ref.rope(k, pos, freq, rope.pair_axis, "halves")
        qw = ref.rope(q, pos, freq, rope.pair_axis, "halves")
        n = int(x.cu[-1])
        assert (np.abs(host(qo) - qw)[:n] <= bound(q, qw, rope.pair_axis, pos, freq, "halves", dtype)[:n]).all()
        assert (qo[n:] == 7).all()
    else:
        pa.paged_kv_append(plan, kd, vd, kc, vc, table, lens_d, cu)
    want_k, want_v = ref.append(x.k, kw, x.table, x.lens, x.cu), ref.append(x.v, v, x.table, x.lens, x.cu)
    assert np.array_equal(host(vc), want_v)
    got = host(kc)
    old = np.array([[p, j % page] for p, j in written(x)])
    mask = np.zeros(x.k.shape, dtype=bool)
    mask[old[:, 0], :, old[:, 1]] = True
    assert np.array_equal(got[~mask], x.k[~mask])
    if rotated:   # one rounding, and 7 units of the pair (at most 2 |x| sqrt 2 of it): |k| <= 6 here
        assert (np.abs(got - want_k)[mask] <= STEP[dtype] * np.abs(want_k)[mask] + 7 * U32 * 12 + 1e-10).all()
    else:
        assert np.array_equal(got, want_k)
    plan.destroy()


def written(x):
    for t, b, pos in ref.new_rows(x.lens, x.cu, x.tokens):
        p = ref.page_of(x.table, b, pos, x.page, x.pages)
        if p >= 0:
            yield p, pos
