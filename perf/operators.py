"""Cases on which the operators of the sampling phase are measured: rollouts over a long video are generated token by token
(or prefilled in chunks) on a paged cache of keys and values, with rotary positions that have a time, a height and a width.

A case names what one pass does ("do"):
  rope           rotation of queries and keys by multi-axis positions (rope_axes_forward)
  rope_backward  the gradient of that rotation (rope_axes_backward)
  append         new keys (rotated) and values into the pages of their sequences, new queries rotated
                 (paged_kv_append_rope)
  attend         attention of each sequence's new tokens over its pages (paged_attn_forward)
`run` computes them in plain tensor operations, or with `own` set through the entry points of `paper_2507_07966_amd`.

Queries, keys, values and gradients are N(0, 1), rounded to the case's data type.  Sequence b of a call has
`new_lo` .. `new_hi` new tokens and, with them, `keys_lo` .. `keys_hi` tokens in all (both drawn from `lens_seed`); its pages
are scattered over the cache.  With `shared` tokens, the first that many tokens of all sequences are one video's, in pages
that all tables name.
"""
import math

import numpy as np
import torch

own = False

TORCH_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
LAYER = (28, 4)      # query and key/value heads of the 7B-class decoder layer that the repository's workloads use
VIDEO = (16, 24, 24)  # rotated pairs of a 128-channel head that follow time, height and width
BASE = 10000.0       # of the rotary frequencies


def _rope(name, do, dtype, heads, head_dim, tokens, sections, layout="halves"):
    """`sections`: how many pairs of channels each axis turns; the other channels pass through."""
    case = {"do": do, "dtype": dtype, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "tokens": tokens,
            "layout": layout}
    for a, n in enumerate(sections):
        case[f"axis{a}"] = n
    return dict(case, name=name) if name else case


def _paged(name, do, dtype, heads, head_dim, page, seqs, new_lo, new_hi, keys_lo, keys_hi, shared=0, lens_seed=0,
           sections=()):
    case = {"do": do, "dtype": dtype, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "page": page,
            "seqs": seqs, "new_lo": new_lo, "new_hi": new_hi, "keys_lo": keys_lo, "keys_hi": keys_hi, "shared": shared,
            "lens_seed": lens_seed}
    if do == "append":
        case["layout"] = "halves"
        for a, n in enumerate(sections):
            case[f"axis{a}"] = n
    return dict(case, name=name) if name else case


def listed():
    return [
        # One step of eight rollouts: the smallest rotation, all latency.
        _rope("rope_step", "rope", "bf16", LAYER, 128, 8, VIDEO),
        # The tokens of a 512-frame video, once per layer in the prefill: the largest rotation.
        _rope("rope_video", "rope", "bf16", LAYER, 128, 32768, VIDEO),
        # The policy's training step over eight rollouts of 2,304 tokens: gradients of queries and keys back through it.
        _rope("rope_train", "rope_backward", "bf16", LAYER, 128, 18432, VIDEO),
        # A smaller model in full precision, neighbouring channels paired, part of a head rotated, nothing a round number.
        _rope("rope_train_f32", "rope_backward", "f32", (14, 2), 64, 5377, (11, 12), layout="pairs"),
        # One step of sixteen rollouts: their new keys and values into the cache.
        _paged("append_step", "append", "bf16", LAYER, 128, 64, 16, 1, 1, 500, 2000, sections=VIDEO),
        # A chunk of a long video's prefill into the cache.
        _paged("append_chunk", "append", "bf16", LAYER, 128, 64, 2, 4000, 4096, 6000, 9000, lens_seed=1, sections=VIDEO),
        # One user's short conversation, one token: the smallest attention call, all latency.
        _paged("attend_token", "attend", "bf16", LAYER, 128, 16, 1, 1, 1, 1100, 1100),
        # One step of eight rollouts over one 512-frame video (the headline workload of this repository, sampled).
        _paged("attend_video", "attend", "bf16", LAYER, 128, 64, 8, 1, 1, 33000, 35000, shared=32768, lens_seed=2),
        # One step of a full server: sixty-four sequences of nothing in common.
        _paged("attend_batch", "attend", "bf16", LAYER, 128, 64, 64, 1, 1, 700, 17000, lens_seed=3),
        # The last chunk of a long video's prefill: the largest call.
        _paged("attend_chunk", "attend", "bf16", LAYER, 128, 64, 1, 2048, 2048, 34816, 34816),
        # A smaller model's server: chunks of prompts beside single tokens, small pages, odd lengths.
        _paged("attend_mixed", "attend", "bf16", (14, 2), 64, 16, 24, 1, 301, 400, 9000, lens_seed=4),
        # A check in full precision on a small layer: chunks of odd lengths.
        _paged("attend_f32", "attend", "f32", (8, 2), 128, 32, 5, 3, 130, 200, 4100, lens_seed=5),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# The dearest listed passes: a drawn case stays below them (fp32 far below: its operations cost more).
MOST_FLOPS = 9e11
MOST_BYTES = 8e8


def draw(rng):
    """One more case of the same ranges."""
    while True:
        do = rng.choice(("rope", "rope_backward", "append", "attend", "attend", "attend"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        heads = rng.choice((LAYER, (14, 2), (12, 2), (16, 8), (8, 2), (4, 4), (16, 2)))
        head_dim = rng.choice((64, 128, 128))
        pairs = head_dim // 2 if rng.random() < 0.6 else rng.randint(head_dim // 8, head_dim // 2)
        axes = rng.randint(1, 4)
        cuts = sorted(rng.sample(range(1, pairs), axes - 1))
        sections = [b - a for a, b in zip([0, *cuts], [*cuts, pairs])]
        if do in ("rope", "rope_backward"):
            case = _rope(None, do, dtype, heads, head_dim, _log_uniform(rng, 1, 32768), sections, rng.choice(("halves", "pairs")))
        else:
            page = rng.choice((16, 32, 64, 128, 256))
            seqs = _log_uniform(rng, 1, 96)
            if do == "append":
                hi = _log_uniform(rng, 1, 8192 // seqs)
                lo, keys_lo = rng.randint(1, hi), hi
                keys_hi = keys_lo + _log_uniform(rng, 1, 4000)
                case = _paged(None, do, dtype, heads, head_dim, page, seqs, lo, hi, keys_lo, keys_hi,
                              lens_seed=rng.randint(0, 1 << 20), sections=sections)
            else:
                kind = rng.choice(("token", "token", "few", "chunk", "mixed", "shared"))
                hi = {"few": rng.randint(2, 8), "chunk": _log_uniform(rng, 16, 2048), "mixed": _log_uniform(rng, 16, 600),
                      "shared": rng.choice((1, 1, 1, 2, 4))}.get(kind, 1)
                lo = 1 if kind != "chunk" else rng.randint(max(1, hi // 2), hi)
                shared = page * max(1, _log_uniform(rng, 256, 32768) // page) if kind == "shared" else 0
                keys_lo = shared + hi + _log_uniform(rng, 1, 2000 if shared else 20000)
                keys_hi = keys_lo + _log_uniform(rng, 1, 2000 if shared else 20000)
                case = _paged(None, do, dtype, heads, head_dim, page, seqs, lo, hi, keys_lo, keys_hi, shared,
                              rng.randint(0, 1 << 20))
        need = work(case)
        slow = 0.01 if dtype == "f32" and do == "attend" else 1.0
        _, keys = _lens(case) if "seqs" in case else (None, np.zeros(1, dtype=np.int64))
        # `keys`: the plain form gathers every sequence's own copy of shared pages
        cache = 2 * int(keys.sum()) * case["kv_heads"] * head_dim * 4
        if need["flops"] <= slow * MOST_FLOPS and need["bytes"] <= MOST_BYTES and cache <= 4e9:
            return case


def _sections(case):
    return [case[f"axis{a}"] for a in range(4) if f"axis{a}" in case]


def _lens(case):
    """New tokens and all tokens of each sequence."""
    rng = np.random.default_rng(case["lens_seed"])
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=case["seqs"])
    keys = rng.integers(case["keys_lo"], case["keys_hi"] + 1, size=case["seqs"])
    return new, np.maximum(keys, new)


def _tables(case):
    """Page table [seqs, pages of the longest], -1 where a sequence has no page, and the number of pages of the cache."""
    _, keys = _lens(case)
    page = case["page"]
    need = (keys + page - 1) // page
    common = case["shared"] // page
    total = common + int((need - common).sum())
    order = np.random.default_rng(case["lens_seed"] + 1).permutation(total)
    table = np.full((case["seqs"], int(need.max())), -1, dtype=np.int32)
    at = common
    for b, n in enumerate(need):
        table[b, :common] = order[:common]
        table[b, common:n] = order[at:at + n - common]
        at += n - common
    return table, total


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dtype = TORCH_DTYPE[case["dtype"]]
    hq, hkv, dim = case["q_heads"], case["kv_heads"], case["head_dim"]

    def normal(*shape):
        flat = torch.empty(math.prod(shape), dtype=dtype, device="cuda")
        step = 1 << 26
        for i in range(0, flat.numel(), step):   # in pieces: the fp32 values before rounding need not all be held
            part = flat[i:i + step]
            part.copy_(torch.randn(part.shape, generator=gen, dtype=torch.float32, device="cuda"))
        return flat.view(shape)

    state = {"case": case}
    if own:
        import paper_2507_07966_amd as pa
        state["pa"] = pa
    if "axis0" in case:
        sections = _sections(case)
        pairs = sum(sections)
        exponent = torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs
        state["inv_freq"] = torch.pow(torch.tensor(BASE, dtype=torch.float64, device="cuda"), -exponent).float()
        state["axis"] = torch.repeat_interleave(torch.arange(len(sections), device="cuda"), torch.tensor(sections, device="cuda"))
        if own:
            state["rope"] = pa.rope_axes(sections, dim, rotary_dim=2 * pairs, layout=case["layout"])

    if case["do"] in ("rope", "rope_backward"):
        tokens = case["tokens"]
        # A video of 8 x 8 tokens a frame that starts anywhere in the sequence: time first, then height and width.
        start = torch.randint(0, 500000, (1,), generator=gen, device="cuda")
        i = torch.arange(tokens, device="cuda")
        axes = [i // 64, i // 8 % 8, i % 8, i][:len(_sections(case))]
        state["positions"] = torch.stack([start + a for a in axes]).to(torch.int32)
        # Forward: slices of the projection's output [queries | keys | values]; backward: gradients, each of its own.
        if case["do"] == "rope":
            qkv = normal(tokens, hq + 2 * hkv, dim)
            state["q"], state["k"] = qkv[:, :hq], qkv[:, hq:hq + hkv]
        else:
            state["q"], state["k"] = normal(tokens, hq, dim), normal(tokens, hkv, dim)
        state["q_out"] = torch.empty(tokens, hq, dim, dtype=dtype, device="cuda")
        state["k_out"] = torch.empty(tokens, hkv, dim, dtype=dtype, device="cuda")
        return state

    new, keys = _lens(case)
    table, pages = _tables(case)
    tokens = int(new.sum())
    state["k_cache"] = normal(pages, hkv, case["page"], dim)
    state["v_cache"] = normal(pages, hkv, case["page"], dim)
    state["new"], state["keys"] = new.tolist(), keys.tolist()
    state["page_table"] = torch.from_numpy(table).cuda()
    state["seq_lens"] = torch.from_numpy(keys.astype(np.int32)).cuda()
    state["cu_new"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    if own:
        state["plan"] = pa.paged_attn_plan(hq, hkv, dim, case["page"], pages, table.shape[1], case["seqs"], tokens,
                                           1.0 / math.sqrt(dim), dtype=case["dtype"])
    if case["do"] == "append":
        qkv = normal(tokens, hq + 2 * hkv, dim)
        state["q"], state["k"], state["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        state["q_out"] = torch.empty(tokens, hq, dim, dtype=dtype, device="cuda")
        # A generated token is text and has one position on all axes; chunks are video tokens, 8 x 8 a frame.
        at = np.concatenate([np.arange(n - m, n) for m, n in zip(new, keys)])
        axes = [at] * 4 if case["new_hi"] == 1 else [at // 64, at // 8 % 8, at % 8, at]
        state["positions"] = torch.from_numpy(np.stack(axes[:len(_sections(case))]).astype(np.int32)).cuda()
        return state
    state["q"] = normal(tokens, hq, dim)
    state["out"] = torch.empty(tokens, hq, dim, dtype=dtype, device="cuda")
    state["lse"] = torch.empty(hq, tokens, dtype=torch.float32, device="cuda")
    if own:
        state["workspace"] = torch.empty(max(16, state["plan"].workspace_bytes), dtype=torch.uint8, device="cuda")
        state["shared_len"] = torch.tensor([case["shared"]], dtype=torch.int32, device="cuda") if case["shared"] else None
    return state


def _rotate(x, positions, inv_freq, axis, layout, sign):
    """Pair i of every head of token t turned by sign * positions[axis[i], t] * inv_freq[i]."""
    angle = positions[axis].T.double() * inv_freq.double()      # [tokens, pairs]; 64 bits: positions reach far
    cos, sin = torch.cos(angle).float().unsqueeze(1), sign * torch.sin(angle).float().unsqueeze(1)
    pairs = inv_freq.numel()
    y = x.float()
    if layout == "halves":
        a, b = y[..., :pairs], y[..., pairs:2 * pairs]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([turned, y[..., 2 * pairs:]], dim=-1).to(x.dtype)


def _plain_append(state):
    case, page = state["case"], state["case"]["page"]
    args = state["positions"], state["inv_freq"], state["axis"], case["layout"], 1.0
    state["q_out"].copy_(_rotate(state["q"], *args))
    k, at = _rotate(state["k"], *args), 0
    for b, (n, total) in enumerate(zip(state["new"], state["keys"])):
        slot = torch.arange(total - n, total, device="cuda")
        where = state["page_table"][b].long()[slot // page]
        state["k_cache"][where, :, slot % page] = k[at:at + n]
        state["v_cache"][where, :, slot % page] = state["v"][at:at + n]
        at += n
    return state["q_out"], state["k_cache"], state["v_cache"]


def _plain_attend(state):
    case = state["case"]
    hkv, dim, page = case["kv_heads"], case["head_dim"], case["page"]
    group = case["q_heads"] // hkv
    out, lse, at = state["out"], state["lse"], 0
    for b, (n, total) in enumerate(zip(state["new"], state["keys"])):
        pages = state["page_table"][b, :(total + page - 1) // page].long()
        i = torch.arange(n, device="cuda").repeat_interleave(group)
        hidden = torch.arange(total, device="cuda") > (total - n + i).unsqueeze(1)
        for c in range(hkv):
            k = state["k_cache"][pages, c].reshape(-1, dim)[:total].float()
            v = state["v_cache"][pages, c].reshape(-1, dim)[:total].float()
            q = state["q"][at:at + n, c * group:(c + 1) * group].float().reshape(-1, dim)
            s = (q @ k.T).mul_(1.0 / math.sqrt(dim)).masked_fill_(hidden, -math.inf)
            top = s.amax(dim=1, keepdim=True)
            p = s.sub_(top).exp_()
            total_p = p.sum(dim=1, keepdim=True)
            out[at:at + n, c * group:(c + 1) * group] = (p @ v / total_p).view(n, group, dim).to(out.dtype)
            lse[c * group:(c + 1) * group, at:at + n] = (top + total_p.log()).view(n, group).T
        at += n
    return out, lse


def run(state):
    case = state["case"]
    do, pa = case["do"], state.get("pa")
    if do in ("rope", "rope_backward"):
        if own:
            call = pa.rope_axes_forward if do == "rope" else pa.rope_axes_backward
            call(state["rope"], state["q"], state["k"], state["positions"], state["inv_freq"], state["q_out"], state["k_out"])
        else:
            args = state["positions"], state["inv_freq"], state["axis"], case["layout"], 1.0 if do == "rope" else -1.0
            state["q_out"].copy_(_rotate(state["q"], *args))
            state["k_out"].copy_(_rotate(state["k"], *args))
        return state["q_out"], state["k_out"]
    if not own:
        return _plain_append(state) if do == "append" else _plain_attend(state)
    cache = state["k_cache"], state["v_cache"], state["page_table"], state["seq_lens"], state["cu_new"]
    if do == "append":
        pa.paged_kv_append_rope(state["plan"], state["rope"], state["q"], state["k"], state["v"], state["positions"],
                                state["inv_freq"], state["q_out"], *cache)
        return state["q_out"], state["k_cache"], state["v_cache"]
    pa.paged_attn_forward(state["plan"], state["q"], *cache, state["out"], state["lse"], state["workspace"],
                          shared_len=state["shared_len"])
    return state["out"], state["lse"]


def work(case):
    """What one pass cannot do without: every input read once (a page that several sequences name, once), every output
    written once; 4 D operations for each pair of a query row and a key that it sees, 6 for each rotated pair of channels."""
    size = 2 if case["dtype"] == "bf16" else 4
    hq, hkv, dim = case["q_heads"], case["kv_heads"], case["head_dim"]
    sections = _sections(case)
    if case["do"] in ("rope", "rope_backward"):
        tokens = case["tokens"]
        return {"bytes": 2 * size * tokens * (hq + hkv) * dim + 4 * tokens * len(sections) + 4 * sum(sections),
                "flops": 6 * tokens * (hq + hkv) * sum(sections)}
    new, keys = _lens(case)
    tokens, tables = int(new.sum()), 4 * int(((keys + case["page"] - 1) // case["page"]).sum()) + 8 * case["seqs"] + 4
    if case["do"] == "append":   # queries, keys and values in; queries out, the new slots of the cache written
        return {"bytes": 2 * size * tokens * (hq + 2 * hkv) * dim + 4 * tokens * len(sections) + 4 * sum(sections) + 12 * case["seqs"],
                "flops": 6 * tokens * (hq + hkv) * sum(sections)}
    stored = case["shared"] + int((keys - case["shared"]).sum())
    pairs = hq * int((new * (keys - new) + new * (new + 1) // 2).sum())
    return {"bytes": 2 * size * (tokens * hq + stored * hkv) * dim + 4 * tokens * hq + tables, "flops": 4 * dim * pairs}


def exact(case, seed):
    """The operators' definitions in 64 bits: rotation as a product of complex numbers, attention row by row of each head
    as weights e^(s - LSE) over the visible keys."""
    s = prepare(case, seed)
    if "axis0" in case:
        axes = torch.stack([s["positions"][a].double() for a in s["axis"].tolist()], dim=1)
        turn = torch.polar(torch.ones_like(axes), axes * s["inv_freq"].double() * (-1 if case["do"] == "rope_backward" else 1))

        def rotated(x):
            y, n = x.double().clone(), turn.shape[1]
            first, second = (slice(0, n), slice(n, 2 * n)) if case["layout"] == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
            z = torch.complex(y[:, :, first], y[:, :, second]) * turn[:, None, :]
            y[:, :, first], y[:, :, second] = z.real, z.imag
            return y

    if case["do"] in ("rope", "rope_backward"):
        return rotated(s["q"]), rotated(s["k"])
    page, ends = case["page"], np.cumsum(s["new"])
    if case["do"] == "append":
        k, v = rotated(s["k"]), s["v"].double()
        k_cache, v_cache, table = s["k_cache"].double(), s["v_cache"].double(), s["page_table"].cpu().numpy()
        place = [(int(table[b, j // page]), j % page) for b, (n, total) in enumerate(zip(s["new"], s["keys"]))
                 for j in range(total - n, total)]
        pages, slots = torch.tensor(place, device="cuda").unbind(1)
        k_cache[pages, :, slots], v_cache[pages, :, slots] = k, v
        return rotated(s["q"]), k_cache, v_cache
    hq, hkv, dim = case["q_heads"], case["kv_heads"], case["head_dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(hq, s["q"].shape[0], dtype=torch.float64, device="cuda")
    for b, (n, total) in enumerate(zip(s["new"], s["keys"])):
        rows = slice(int(ends[b]) - n, int(ends[b]))
        used = s["page_table"][b, :-(-total // page)].long()
        late = torch.ones(n, total, dtype=torch.bool, device="cuda").triu(diagonal=total - n + 1)
        for h in range(hq):
            c = h // (hq // hkv)
            k = s["k_cache"][used, c].double().flatten(0, 1)[:total]
            score = (s["q"][rows, h].double() @ k.T) / math.sqrt(dim)
            score[late] = -math.inf
            lse[h, rows] = torch.logsumexp(score, dim=1)
            weight = torch.exp(score - lse[h, rows, None])
            out[rows, h] = weight @ s["v_cache"][used, c].double().flatten(0, 1)[:total]
    return out, lse
