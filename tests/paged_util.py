"""Problems for lsa_kv_append and lsa_paged_attn on a device, their oracle results and error bounds."""
from __future__ import annotations

import math

import numpy as np
import torch

from oracle import lsa_oracle as orc
from paper_2608_01662_b200 import binding

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}   # half a step, relative to the value


def to_np(t):
    return t.detach().double().cpu().numpy()


def table_of(lengths, page, rng, spare=3, width=None):
    """(page table [batch, width] with the pages that the lengths need, -1 elsewhere; number of pages)."""
    need = [-(-n // page) for n in lengths]
    n_pages = sum(need) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(lengths), width or max(1, max(need))), -1, np.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    return table, n_pages


class Cache:
    """A pool of pages, filled with normal values (or garbage where nobody may look)."""

    def __init__(self, lengths, shape, page, dtype="bf16", e4m3=False, device="cuda:0", seed=0, poison=False, pad=0, width=None, scale=1.0):
        self.lengths, self.page, self.dtype, self.e4m3 = list(lengths), page, dtype, e4m3
        self.H, self.G, self.d, self.dv = shape
        self.latent = self.d == 576
        rng = np.random.default_rng(seed)
        self.table, self.n_pages = table_of(lengths, page, rng, width=width)
        gen = torch.Generator(device).manual_seed(seed + 1)
        rows = self.n_pages * page
        self.device = device

        def pool(width):
            x = torch.randn(rows, width + pad, generator=gen, device=device, dtype=torch.float32) * scale
            if not e4m3:
                return x.to(DTYPES[dtype])[:, :width], None
            y = x[:, :width].reshape(rows, self.G, -1)
            s = (y.abs().amax(-1) / 448).clamp(min=1e-30)
            codes = (y / s[..., None]).to(torch.float8_e4m3fn).view(torch.uint8).reshape(rows, width)
            wide = torch.zeros(rows, width + pad, dtype=torch.uint8, device=device)
            wide[:, :width] = codes
            return wide[:, :width], s.contiguous()

        self.k, self.k_scale = pool(self.G * self.d)
        self.v, self.v_scale = (None, None) if self.latent else pool(self.G * self.dv)
        self.page_table = torch.from_numpy(self.table).to(device)
        self.ctx_len = torch.tensor(self.lengths, dtype=torch.int32, device=device)
        self.q = torch.randn(len(lengths), self.H, self.d, generator=gen, device=device, dtype=torch.float32).mul(2).to(DTYPES[dtype])
        if poison:
            self.poison()

    def used_rows(self, sink=0, window=0):
        used = [orc.paged_rows(orc.seen_tokens(n, sink, window), self.table[b], self.page) for b, n in enumerate(self.lengths)]
        return np.unique(np.concatenate(used)) if used else np.zeros(0, np.int64)

    def poison(self, sink=0, window=0):
        """NaN and infinities in every row that no query sees."""
        free = torch.ones(self.n_pages * self.page, dtype=torch.bool)
        free[torch.from_numpy(self.used_rows(sink, window))] = False
        free = free.to(self.device)
        for t, s in ((self.k, self.k_scale), (self.v, self.v_scale)):
            if t is None:
                continue
            if self.e4m3:
                t[free] = 0x7f
                s[free] = math.nan
            else:
                t[free] = math.nan
                t[free, ::3] = math.inf

    def params(self, **kw):
        return binding.make_kv_params(self.H, self.G, self.d, self.dv, self.page, latent=self.latent, dtype=self.dtype, e4m3=self.e4m3, **kw)

    def values(self):
        """(keys [rows, G, d], values [rows, G, dv]) as the real numbers that the pool stands for."""
        def real(t, s, d):
            if not self.e4m3:
                return to_np(t).reshape(-1, self.G, d)
            return orc.e4m3_decode(t.cpu().numpy()).reshape(-1, self.G, d) * to_np(s)[..., None]
        k = real(self.k, self.k_scale, self.d)
        return (k, k[..., :self.dv]) if self.latent else (k, real(self.v, self.v_scale, self.dv))


def many_small_weights(shape, page, device):
    """fp16 sequences of 4096 tokens whose first weighs 1 and has no value, the others 2^-26 each with values of 2^10."""
    c = Cache([4096] * 40, shape, page, "fp16", False, device, seed=21)
    c.q[:] = 0
    c.q[..., 0] = 1
    c.k[:] = 0
    if c.v is None:
        c.k[:, 1:512] = 1024
    else:
        c.v[:] = 1024
    first = torch.from_numpy(c.table[:, 0].astype(np.int64) * page).to(device)
    c.k[first] = 0
    c.k[first, ::c.d] = 26 * math.log(2) * c.d ** 0.5
    if c.v is not None:
        c.v[first] = 0
    return c


def attend(cache, ctx=None, out=None, lse=None, **kw):
    ctx = ctx or binding.Context(None, 0, 0, len(cache.lengths), device=cache.device, kv=cache.params(**kw))
    B = len(cache.lengths)
    out = torch.full((B, cache.H, cache.dv), 7.0, dtype=DTYPES[cache.dtype], device=cache.device) if out is None else out
    lse = torch.full((B, cache.H), 7.0, dtype=torch.float32, device=cache.device) if lse is None else lse
    ctx.paged_attn(cache.q, cache.k, cache.v, cache.page_table, cache.ctx_len, out, lse, k_scale=cache.k_scale, v_scale=cache.v_scale)
    return ctx, out, lse


def check_attend(cache, out, lse, sink=0, window=0, sequences=None):
    """Every element against the oracle, within what the roundings of the method allow.

    With u_p the rounding of a weight to 16 bits (bf16 where the cache is e4m3), u_o that of the result, and weights p, values v:
      |out - ref| <= (u_p + 2 e) sum_s p_s |v_s| + u_o |ref|   (+ 2^-32 sum_s |v_s| where weights are fp16: a weight below 2^-14
    is rounded to a multiple of 2^-24; the largest weight of a part is at least 2^7 before the division)
    e4m3 caches: weights times value scales are rounded to fp16, the largest of a part at least 2^7 when the others are: u_p is fp16's, and
    2^-32 max_s (p_s scale_s) sum_s |code_s| is added for those that become subnormal.
    where e is the relative error of a weight before that rounding: that of its score, (d + 8) roundings of fp32 of products whose
    absolute sum is at most sum_i |q_i k_i| (a tree or a chain of fp32 additions, in log2 units, times ln 2), 2^-21 for exp2 and
    (n / 8 + 512) roundings for the chains of sums.  The log-sum-exp carries the score's error and the sum's.
    """
    k, v = cache.values()
    q = to_np(cache.q)
    got, got_lse = to_np(out), to_np(lse)
    scale = cache.d ** -0.5
    u_o = UNIT[cache.dtype]
    u_p = UNIT["fp16" if cache.e4m3 else cache.dtype]
    group = cache.H // cache.G
    worst = 0.0
    for b in range(len(cache.lengths)) if sequences is None else sequences:
        n = cache.lengths[b]
        ref, ref_lse = orc.paged_attend(q[b], k, v, cache.table[b], n, cache.page, cache.G, sink=sink, window=window, sm_scale=scale)
        pos = orc.seen_tokens(n, sink, window)
        if len(pos) == 0:
            assert np.all(got[b] == 0) and np.all(np.isneginf(got_lse[b])), (b, n)
            continue
        rows = orc.paged_rows(pos, cache.table[b], cache.page)
        for h in range(cache.H):
            g = h // group
            z = scale * (k[rows, g] @ q[b, h])
            p = np.exp(z - ref_lse[h])
            mass = p @ np.abs(v[rows, g])
            e_z = scale * (cache.d + 8) * 2.0 ** -24 * (np.abs(k[rows, g]) @ np.abs(q[b, h])).max()
            e = e_z + 2.0 ** -21 + (len(pos) / 8 + 512) * 2.0 ** -24
            tol = (u_p + 2 * e) * mass + u_o * np.abs(ref[h]) * (1 + u_p)
            if cache.dtype == "fp16" and not cache.e4m3:
                tol = tol + 2.0 ** -32 * np.abs(v[rows, g]).sum(0)
            if cache.e4m3:
                vs = to_np(cache.v_scale)[rows, g]
                tol = tol + 2.0 ** -32 * (p * vs).max() * np.abs(v[rows, g] / vs[:, None]).sum(0)
            if cache.dtype == "fp16":
                tol = tol + 2.0 ** -25   # a result below 2^-14 is rounded to a multiple of 2^-24
            err = np.abs(got[b, h] - ref[h])
            assert np.all(err <= tol), (b, n, h, float((err - tol).max()), float((err / tol).max()))
            worst = max(worst, float((err / tol).max()))
            assert abs(got_lse[b, h] - ref_lse[h]) <= 2 * e + 4 * 2.0 ** -24 * (1 + abs(ref_lse[h])), (b, n, h)
    return worst
