"""The sampling phase's operators together, as a serving loop uses them: a video's tokens are rotated and appended chunk by chunk, its pages are
shared by several rollouts, and these go on token by token, all steps after the first replayed from a captured graph."""
import numpy as np
import pytest

from tests.sampling_util import Paged, gpu, host, round_to

pytestmark = pytest.mark.gpu

HQ, HKV, D, PAGE = 28, 4, 128, 64
VIDEO, ROLLOUTS, STEPS = 640, 5, 4          # video tokens (whole pages), rollouts, generated tokens
PROMPT = [37, 1, 90, 64, 5]                 # each rollout's own tokens before the first generated one


def positions(video, own):
    """Time, height and width of 8 x 8 tokens a frame, then one position on all axes for text."""
    i = np.arange(video)
    grid = np.stack([i // 64, i // 8 % 8, i % 8])
    text = grid.max() + 1 + np.arange(own)
    return np.concatenate([grid, np.stack([text] * 3)], axis=1).astype(np.int32)


def test_rollouts_over_a_shared_video():
    import torch
    import paper_2507_07966_amd as pa
    rng = np.random.default_rng(0)
    total = [VIDEO + p + STEPS for p in PROMPT]
    x = Paged("bf16", (HQ, HKV), D, PAGE, total, [1] * ROLLOUTS, shared=VIDEO, seed=20)
    rope = pa.rope_axes((16, 24, 24), D)
    freq = gpu((10000.0 ** (-np.arange(64) / 64)).astype(np.float32))
    # fused projections of the video and of each rollout's own tokens
    video = torch.from_numpy(rng.standard_normal((VIDEO, HQ + 2 * HKV, D)).astype(np.float32)).cuda().bfloat16()
    own = [torch.from_numpy(rng.standard_normal((p + STEPS, HQ + 2 * HKV, D)).astype(np.float32)).cuda().bfloat16() for p in PROMPT]
    pos = [gpu(positions(VIDEO, p + STEPS)) for p in PROMPT]
    kc, vc = (torch.full((x.pages, HKV, PAGE, D), float("nan"), device="cuda").bfloat16() for _ in range(2))
    table = gpu(x.table)
    plan = x.plan(max_tokens=1024)
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    split = lambda f: (f[:, :HQ], f[:, HQ:HQ + HKV], f[:, HQ + HKV:])

    def step(fused, at, lens, cu, tables, out, lse, shared=None):
        q, k, v = split(fused)
        qr = torch.empty(fused.shape[0], HQ, D, device="cuda", dtype=torch.bfloat16)
        pa.paged_kv_append_rope(plan, rope, q, k, v, at, freq, qr, kc, vc, tables, lens, cu)
        pa.paged_attn_forward(plan, qr, kc, vc, tables, lens, cu, out, lse, ws, shared_len=shared)

    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    # the video, in chunks of 300 tokens, through the first rollout's table
    video_out, video_lse = [], []
    for a in range(0, VIDEO, 300):
        b = min(VIDEO, a + 300)
        out, lse = torch.empty(b - a, HQ, D, device="cuda", dtype=torch.bfloat16), torch.empty(HQ, b - a, device="cuda")
        step(video[a:b], pos[0][:, a:b].contiguous(), i32([b]), i32([0, b - a]), table[:1], out, lse)
        video_out.append(out)
        video_lse.append(lse)
    # the prompts of all rollouts in one call
    prompt = torch.cat([o[:p] for o, p in zip(own, PROMPT)])
    cu = np.concatenate([[0], np.cumsum(PROMPT)])
    prompt_out, prompt_lse = torch.empty(cu[-1], HQ, D, device="cuda", dtype=torch.bfloat16), torch.empty(HQ, cu[-1], device="cuda")
    at = torch.cat([s[:, VIDEO:VIDEO + p] for s, p in zip(pos, PROMPT)], dim=1).contiguous()
    step(prompt, at, i32([VIDEO + p for p in PROMPT]), i32(cu), table, prompt_out, prompt_lse, shared=i32([VIDEO]))
    # token by token; the buffers of a step are filled, and the captured step is replayed
    fused = torch.empty(ROLLOUTS, HQ + 2 * HKV, D, device="cuda", dtype=torch.bfloat16)
    at, lens, ones = torch.empty(3, ROLLOUTS, dtype=torch.int32, device="cuda"), i32([0] * ROLLOUTS), i32(list(range(ROLLOUTS + 1)))
    out, lse, shared = torch.empty(ROLLOUTS, HQ, D, device="cuda", dtype=torch.bfloat16), torch.empty(HQ, ROLLOUTS, device="cuda"), i32([VIDEO])
    steps, graph = [], None
    for s in range(STEPS):
        fused.copy_(torch.stack([o[p + s] for o, p in zip(own, PROMPT)]))
        at.copy_(torch.stack([q[:, VIDEO + p + s] for q, p in zip(pos, PROMPT)], dim=1))
        lens.copy_(i32([VIDEO + p + s + 1 for p in PROMPT]))
        if s == 0:
            step(fused, at, lens, ones, table, out, lse, shared)
        else:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                torch.cuda.synchronize()
                with torch.cuda.graph(graph):
                    step(fused, at, lens, ones, table, out, lse, shared)
            graph.replay()
        torch.cuda.synchronize()
        steps.append((out.clone(), lse.clone()))

    # The same through the prefill: every rollout's whole sequence rotated, causal attention of it alone
    for g, p in enumerate(PROMPT):
        q, k, v = (t.contiguous() for t in split(torch.cat([video, own[g]])))
        pa.rope_axes_forward(rope, q, k, pos[g], freq, q, k)
        n = VIDEO + p + STEPS
        whole = pa.prefix_attn_plan(HQ, HKV, D, 0, [n], D ** -0.5)
        want, want_lse = torch.empty_like(q), torch.empty(HQ, n, device="cuda")
        wws = torch.empty(whole.workspace_bytes, dtype=torch.uint8, device="cuda")
        pa.prefix_attn_forward(whole, q, None, None, k, v, want, wws)
        pa.prefix_attn_lse(whole, wws, want_lse)
        got = torch.cat([*(video_out if g == 0 else []), prompt_out[cu[g]:cu[g + 1]], *[o[g:g + 1] for o, _ in steps]])
        got_lse = torch.cat([*(video_lse if g == 0 else []), prompt_lse[:, cu[g]:cu[g + 1]], *[l[:, g:g + 1] for _, l in steps]], dim=1)
        first = 0 if g == 0 else VIDEO
        # Both sides round the same keys, queries and probabilities: each result errs by at most 2^-8 of sum w |v| (probabilities) and 2^-8 of
        # itself (its own rounding); values are N(0, 1), sum w |v| is below the largest of them, 5.2, and the mean error far below
        err = np.abs(host(got) - host(want[first:]))
        print(f"rollout {g}: largest difference {err.max():.2e}, mean {err.mean():.2e}, LSE {np.abs(host(got_lse) - host(want_lse[:, first:])).max():.2e}", flush=True)
        assert err.max() <= 2 * (5.2 + 5.2) * 2.0 ** -8 and err.mean() <= 2e-3
        assert np.abs(host(got_lse) - host(want_lse[:, first:])).max() <= 1e-3
        whole.destroy()
    plan.destroy()


def test_a_training_step_through_the_rotation():
    """rope_axes_forward, prefix_attn_forward / _backward and rope_axes_backward in a row: the gradients of the projections before the rotation equal
    those that the definitions give in float64."""
    import torch
    import paper_2507_07966_amd as pa
    hq, hkv, d, n = 4, 2, 64, 96
    rng = np.random.default_rng(1)
    q, k, v, g = (rng.standard_normal((n, h, d)) for h in (hq, hkv, hkv, hq))
    rope = pa.rope_axes((10, 6), d, rotary_dim=32, layout="pairs", interleaved=True)
    pos, freq = rng.integers(0, 9000, size=(2, n)).astype(np.int32), (100.0 ** (-np.arange(16) / 16)).astype(np.float32)
    qd, kd, vd, gd = (gpu(a, "f32") for a in (q, k, v, g))
    qr, kr = torch.empty_like(qd), torch.empty_like(kd)
    pa.rope_axes_forward(rope, qd, kd, gpu(pos), gpu(freq), qr, kr)
    plan = pa.prefix_attn_plan(hq, hkv, d, 0, [n], d ** -0.5, dtype="f32")
    out, lse = torch.empty_like(qd), torch.empty(hq, n, device="cuda")
    ws = torch.empty(max(16, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
    pa.prefix_attn_forward(plan, qr, None, None, kr, vd, out, ws)
    pa.prefix_attn_lse(plan, ws, lse)
    dq, dk, dv = torch.empty_like(qd), torch.empty_like(kd), torch.empty_like(vd)
    pa.prefix_attn_backward(plan, qr, None, None, kr, vd, out, gd, lse, dq, None, None, dk, dv,
                            torch.empty(max(16, plan.backward_workspace_bytes), dtype=torch.uint8, device="cuda"))
    pa.rope_axes_backward(rope, dq, dk, gpu(pos), gpu(freq), dq, dk)
    torch.cuda.synchronize()
    plan.destroy()
    # torch's float64 autograd through the definitions, on the CPU
    tq, tk, tv = (torch.from_numpy(np.float32(a).astype(np.float64)).requires_grad_() for a in (q, k, v))
    angle = torch.from_numpy(pos[list(rope.pair_axis)].T.astype(np.float64) * freq.astype(np.float64))[:, None]

    def turn(x):
        a, b = x[..., 0:32:2], x[..., 1:32:2]
        y = torch.stack([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], dim=-1).flatten(-2)
        return torch.cat([y, x[..., 32:]], dim=-1)

    kk, vv = turn(tk).repeat_interleave(hq // hkv, dim=1), tv.repeat_interleave(hq // hkv, dim=1)
    s = torch.einsum("ihd,jhd->hij", turn(tq), kk) * d ** -0.5
    s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -float("inf"))
    o = torch.einsum("hij,jhd->ihd", s.softmax(-1), vv)
    o.backward(torch.from_numpy(np.float32(g).astype(np.float64)))
    for name, got, want in (("dq", dq, tq.grad), ("dk", dk, tk.grad), ("dv", dv, tv.grad)):
        w = want.numpy()
        err, rms = np.abs(host(got) - w), np.sqrt((w ** 2).mean())
        print(name, err.max() / rms, flush=True)
        assert err.max() <= 1e-4 * np.abs(w).max() + 1e-4 * rms   # fp32 throughout, as the fp32 gradients of the attention alone
