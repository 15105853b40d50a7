"""Seeded inputs of the sampling phase's tests, as numpy and on the GPU."""
import math

import numpy as np

from oracle import ref_sampling as ref

U32 = 2.0 ** -24
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # half a unit in the last place, relative


def round_to(x, dtype):
    """x in float64, rounded to the data type."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    return (t.bfloat16().float() if dtype == "bf16" else t).numpy().astype(np.float64)


def gpu(x, dtype=None):
    import torch
    if dtype is None:
        return torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to({"bf16": torch.bfloat16, "f32": torch.float32}[dtype])


def host(t):
    return t.double().cpu().numpy()


class Paged:
    """A cache and a call on it.  lens[b] tokens of sequence b, new[b] of them new; pages scattered; `shared` leading tokens of all
    sequences in the same pages; `pad` packed rows behind the last sequence."""

    def __init__(self, dtype, heads, dim, page, lens, new, shared=0, pad=0, spare=3, seed=0, wide=0):
        rng = np.random.default_rng(seed)
        self.dtype, self.heads, self.dim, self.page, self.shared = dtype, heads, dim, page, shared
        hq, hkv = heads
        lens, new = np.asarray(lens), np.asarray(new)
        need = (np.maximum(lens, 0) + page - 1) // page
        common = shared // page
        width = max(1, int(need.max(initial=1))) + wide
        self.pages = common + int(np.maximum(need - common, 0).sum()) + spare
        order = rng.permutation(self.pages)
        self.table = np.full((len(lens), width), -1, dtype=np.int32)
        at = common
        for b, n in enumerate(need):
            self.table[b, :min(common, n)] = order[:min(common, n)]
            own = max(0, n - common)
            self.table[b, common:common + own] = order[at:at + own]
            at += own
        self.lens = lens.astype(np.int32)
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.tokens = int(self.cu[-1]) + pad
        self.k = round_to(rng.standard_normal((self.pages, hkv, page, dim)), dtype)
        self.v = round_to(rng.standard_normal((self.pages, hkv, page, dim)), dtype)
        self.q = round_to(rng.standard_normal((self.tokens, hq, dim)), dtype)
        self.scale = 1.0 / math.sqrt(dim)

    def plan(self, device=0, **kw):
        import paper_2507_07966_amd as pa
        args = dict(num_q_heads=self.heads[0], num_kv_heads=self.heads[1], head_dim=self.dim, page_size=self.page,
                    num_pages=self.pages, max_pages_per_seq=self.table.shape[1], max_seqs=max(1, len(self.lens)),
                    max_tokens=max(1, self.tokens), softmax_scale=self.scale, dtype=self.dtype, device=device)
        args.update(kw)
        return pa.paged_attn_plan(**args)

    def upload(self):
        return gpu(self.k, self.dtype), gpu(self.v, self.dtype), gpu(self.table), gpu(self.lens), gpu(self.cu)

    def attend(self, shared_len=None, q=None):
        """paged_attn_forward on the GPU: out and LSE in float64; rows of no sequence keep the 7 they were filled with."""
        import torch
        import paper_2507_07966_amd as pa
        plan = self.plan()
        qd = gpu(self.q, self.dtype) if q is None else q
        out = torch.full((self.tokens, self.heads[0], self.dim), 7.0, device="cuda", dtype=qd.dtype)
        lse = torch.full((self.heads[0], self.tokens), 7.0, device="cuda")
        ws = torch.full((plan.workspace_bytes,), 0x7f, dtype=torch.uint8, device="cuda")   # fp32 3.4e38: nothing may be read before it is written
        pa.paged_attn_forward(plan, qd, *self.upload(), out, lse, ws, shared_len=None if shared_len is None else gpu(np.array([shared_len], dtype=np.int32)))
        torch.cuda.synchronize()
        plan.destroy()
        return host(out), host(lse)

    def oracle(self):
        return ref.paged_attention(self.q, self.k, self.v, self.table, self.lens, self.cu, self.scale)

    def check(self, out, lse, want=None):
        """Against the definition.  A score's fp32 error is at most D + 2 roundings of sum |q_d k_d| scale (eps); it moves LSE by eps
        and every weight by 2 eps relative; sums over n keys, kept per lane and stage, add at most n / 4 + 16 roundings; exp2 and
        log each err by a few units (8 here), exp2 with an argument of up to |s - m| log2 e, itself rounded: reach roundings
        each.  bf16: the probabilities are rounded to bf16 for their product with V, at most 2^-8 of sum w |v|.  The result
        is rounded once."""
        ro, rl, mass, reach, keys = self.oracle() if want is None else want
        rows = ~np.isnan(reach).any(axis=1) & (np.arange(self.tokens) < self.cu[-1])
        eps = (self.dim + 8) * U32 * reach[rows] + (keys[rows, None] / 4 + 24) * U32
        soft = 2 * eps + (2.0 ** -8 if self.dtype == "bf16" else 0.0)
        bound = mass[rows] * (soft[:, :, None] * (1 + 2.0 ** -7)) + STEP[self.dtype] * np.abs(ro[rows]) + 1e-30
        err = np.abs(out[rows] - ro[rows])
        worst = float((err / bound).max()) if err.size else 0.0
        dead = np.isneginf(rl[:, rows].T)
        lerr = np.abs(np.where(dead, 0.0, lse[:, rows].T) - np.where(dead, 0.0, rl[:, rows].T))
        lbound = eps + 4 * U32 * np.abs(np.where(dead, 0.0, rl[:, rows].T))
        print(f"out error / bound {worst:.3f}, LSE {float((lerr / lbound).max()) if lerr.size else 0.0:.3f}", flush=True)
        assert (err <= bound).all() and (lerr <= lbound).all()
        assert (np.isneginf(lse[:, rows].T) == dead).all()
        assert (out[self.cu[-1]:] == 7).all() and (lse[:, self.cu[-1]:] == 7).all()   # padding stays
