"""lsa_kv_append against the oracle (needs a B200), and a decode loop of append and attention."""
import numpy as np
import pytest
import torch

import paged_util as pu
from oracle import lsa_oracle as orc
from paper_2608_01662_b200 import binding

pytestmark = pytest.mark.gpu

SHAPES = [(32, 8, 128, 128), (16, 1, 128, 128), (10, 2, 64, 64), (3, 3, 64, 64), (64, 1, 576, 512), (5, 1, 576, 512)]


def angles(n_pos, d_rope, device):
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * 1000.0 ** (-torch.arange(d_rope // 2, dtype=torch.float64) * 2 / max(d_rope, 1))
    return torch.cat([a.cos(), a.sin()], 1).float().to(device) if d_rope else None


class Tokens:
    """New tokens of a batch and what the cache has to hold afterwards."""

    def __init__(self, cache, new, decode, d_rope, rope_at, interleaved, seed=0, tail=0, fused=False):
        self.c, self.new, self.d_rope, self.rope_at, self.interleaved = cache, new, d_rope, rope_at, interleaved
        dev, dt = cache.device, pu.DTYPES[cache.dtype]
        gen = torch.Generator(dev).manual_seed(seed + 99)
        n = sum(new) + tail                       # `tail`: padding rows behind the last sequence
        self.n = n
        H, G, d, dv = cache.H, cache.G, cache.d, cache.dv

        def normal(*s):
            return torch.randn(*s, generator=gen, device=dev).to(dt)
        if fused and not cache.latent:
            qkv = normal(n, H + 2 * G, d)
            self.q, self.k, self.v = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
        else:
            self.q, self.k, self.v = normal(n, H, d), normal(n, G, d), None if cache.latent else normal(n, G, dv)
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.start = start
        self.tok_start = None if decode else torch.from_numpy(start).to(dev)
        self.before = torch.tensor([c - k for c, k in zip(cache.lengths, new)], dtype=torch.int32, device=dev)
        self.after = torch.full_like(self.before, -9)
        self.q_out = torch.full((n, H, d), 3.0, dtype=dt, device=dev)
        self.cos_sin = angles(max(cache.lengths), d_rope, dev)

    def params(self):
        return self.c.params(d_rope=self.d_rope, rope_at=self.rope_at, rope_interleaved=self.interleaved)

    def append(self, ctx=None, **kw):
        ctx = ctx or binding.Context(None, 0, 0, len(self.new), device=self.c.device, kv=self.params())
        a = dict(ctx_len=self.before, ctx_len_out=self.after, q=self.q, q_out=self.q_out)
        a.update(kw)
        ctx.kv_append(self.k, self.v, self.c.k, self.c.v, self.c.page_table, a.pop("ctx_len"), a.pop("ctx_len_out"), tok_start=self.tok_start,
                      cos_sin=self.cos_sin, k_scale=self.c.k_scale, v_scale=self.c.v_scale, **a)
        return ctx

    def expected(self):
        """Real values: (q_out, {row: keys [G, d]}, {row: values [G, dv]}) and the largest |a| + |b| of each rotated pair's inputs."""
        q, k = pu.to_np(self.q), pu.to_np(self.k)
        v = None if self.v is None else pu.to_np(self.v)
        cs = None if self.cos_sin is None else pu.to_np(self.cos_sin)
        out, rows = np.full(q.shape, 3.0), []
        kk, vv = np.zeros(k.shape), v
        for b, k_new in enumerate(self.new):
            for i in range(k_new):
                t, pos = int(self.start[b]) + i, self.c.lengths[b] - k_new + i
                rows.append(int(orc.paged_rows([pos], self.c.table[b], self.c.page)[0]))
                half = self.d_rope // 2
                for src, dst in ((q, out), (k, kk)):
                    for h in range(src.shape[1]):
                        dst[t, h] = orc.rotate_pairs(src[t, h], cs[pos, :half], cs[pos, half:], self.rope_at, self.interleaved) if self.d_rope else src[t, h]
        return out, kk, vv, rows

    def mass(self, x):
        """|a cos| + |b sin| is at most |a| + |b|: of each element's pair (only its own magnitude outside the rotated dims)."""
        m = np.abs(x).copy()
        half = self.d_rope // 2
        for j in range(half):
            i0, i1 = (self.rope_at + 2 * j, self.rope_at + 2 * j + 1) if self.interleaved else (self.rope_at + j, self.rope_at + j + half)
            m[..., i0] = m[..., i1] = np.abs(x[..., i0]) + np.abs(x[..., i1])
        return m

    def check(self, old_k, old_v, old_ks=None, old_vs=None):
        c = self.c
        out, kk, vv, rows = self.expected()
        u = pu.UNIT[c.dtype]
        real = len(rows)
        # two products and a sum in fp32 (with or without a fused one): 2 roundings of at most |a| + |b| each, then one to 16 bits;
        # fp16 results below 2^-14 are multiples of 2^-24
        tiny = 2.0 ** -25 if c.dtype == "fp16" else 0.0
        fp32 = 2 * 2.0 ** -24
        got = pu.to_np(self.q_out)
        tol = u * np.abs(out) + (1 + u) * fp32 * self.mass(pu.to_np(self.q)) + tiny
        assert np.all(np.abs(got - out)[:real] <= tol[:real])
        assert np.all(got[real:] == 3.0)                                       # padding rows are left as they were
        assert self.after.tolist() == c.lengths
        keep = np.ones(c.k.shape[0], bool)
        keep[rows] = False
        mass_k = self.mass(pu.to_np(self.k))
        for pool, scale, old, old_s, want, mass in ((c.k, c.k_scale, old_k, old_ks, kk, mass_k), (c.v, c.v_scale, old_v, old_vs, vv, None)):
            if pool is None:
                continue
            same = torch.from_numpy(keep).to(pool.device)
            assert torch.equal(pool[same].view(torch.uint8), old[same].view(torch.uint8))      # nothing else is touched
            w = want[:real]
            err = fp32 * mass[:real] if mass is not None else np.zeros_like(w)
            if not c.e4m3:
                have = pu.to_np(pool)[rows].reshape(w.shape)
                assert np.all(np.abs(have - w) <= u * np.abs(w) + (1 + u) * err + (tiny if mass is not None else 0))
                continue
            assert torch.equal(scale[same], old_s[same])
            have_s = pu.to_np(scale)[rows]
            top = np.abs(w).max(-1)
            assert np.all(np.abs(have_s - np.where(top > 0, top / 448, 1)) <= (err.max(-1) + 2 * 2.0 ** -24 * top) / 448 * (1 + 1e-6))
            # the code is the nearest to value / scale (both as the device has them) up to that value's fp32 error and the quotient's rounding
            have = orc.e4m3_decode(pool.cpu().numpy())[rows].reshape(w.shape)
            x = w / have_s[..., None]
            step = np.maximum(2.0 ** -9, np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -9))) - 3))
            assert np.all(np.abs(have - x) <= step / 2 + err / have_s[..., None] * (1 + 1e-6) + 2.0 ** -23 * np.abs(x))


def make(shape, lengths, new, page, dtype, e4m3, dev, decode=False, d_rope=0, rope_at=0, interleaved=False, seed=0, **kw):
    c = pu.Cache(lengths, shape, page, dtype, e4m3, dev, seed=seed)
    t = Tokens(c, new, decode, d_rope, rope_at, interleaved, seed, **kw)
    old = (c.k.clone(), None if c.v is None else c.v.clone(), None if c.k_scale is None else c.k_scale.clone(),
           None if c.v_scale is None else c.v_scale.clone())
    return c, t, old


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,e4m3", [("bf16", False), ("fp16", False), ("bf16", True), ("fp16", True)])
@pytest.mark.parametrize("rope", ["none", "part", "all"])
def test_decode_step(cuda_device, shape, dtype, e4m3, rope):
    if shape[2] == 576 and e4m3:
        e4m3, dtype = False, "fp16"
    d = shape[2]
    d_rope, at = {"none": (0, 0), "part": (32, d - 32), "all": (64, 512) if d == 576 else (d, 0)}[rope]
    page = 64 if d == 576 else 16
    lengths = [1, 2, page, page + 1, 200, 3 * page]
    c, t, old = make(shape, lengths, [1] * 6, page, dtype, e4m3, cuda_device, True, d_rope, at, sum(shape) % 2 == 0, seed=d_rope)
    ctx = t.append()
    assert ctx.status() == 0
    t.check(*old)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,e4m3", [("bf16", False), ("fp16", True)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("new,lengths", [([5, 0, 1, 40, 17], [5, 9, 30, 41, 200]), ([0, 0, 3], [0, 4, 3]), ([130], [130])])
def test_chunks_of_prompts(cuda_device, shape, dtype, e4m3, interleaved, new, lengths):
    e4m3 = e4m3 and shape[2] != 576
    d_rope, at = (64, 512) if shape[2] == 576 else (48, 16)
    c, t, old = make(shape, lengths, new, 64, dtype, e4m3, cuda_device, False, d_rope, at, interleaved, seed=sum(new), tail=3, fused=True)
    ctx = t.append()
    assert ctx.status() == 0
    t.check(*old)


def test_many_tokens(cuda_device):
    """More tokens than the rule for few of them takes (twice the SMs)."""
    new = [301, 0, 260, 7]
    c, t, old = make((8, 2, 64, 64), [n + i for i, n in enumerate(new)], new, 16, "bf16", True, cuda_device, False, 64, 0, True, seed=5, tail=2)
    ctx = t.append()
    assert ctx.status() == 0
    t.check(*old)


@pytest.mark.parametrize("decode", [True, False])
def test_in_place(cuda_device, decode):
    """q rotated where it lies, lengths updated where they lie: the same values as into buffers of their own."""
    for shape, at, d_rope in (((64, 1, 576, 512), 512, 64), ((8, 2, 64, 64), 0, 32)):
        new = [1, 1, 1] if decode else [4, 0, 70]
        lengths = [9, 64, 300]
        c, t, old = make(shape, lengths, new, 64, "bf16", False, cuda_device, decode, d_rope, at, True, seed=6)
        ctx = t.append()
        k_first, q_first = c.k.clone(), t.q_out.clone()
        for x, o in ((c.k, old[0]), (c.v, old[1])):
            if x is not None:
                x.copy_(o)
        q, lens, launches = t.q.clone(), t.before.clone(), ctx.launch_count()
        t.append(ctx, ctx_len=lens, ctx_len_out=lens, q=q, q_out=q)
        assert ctx.launch_count() == launches + (1 if decode else 2)
        assert ctx.status() == 0 and lens.tolist() == lengths and torch.equal(q, q_first) and torch.equal(c.k, k_first)


@pytest.mark.parametrize("decode", [True, False])
def test_lengths_that_overlap_in_part_are_refused(cuda_device, decode):
    c, t, old = make((8, 2, 64, 64), [9, 64, 300], [1, 1, 1], 64, "bf16", False, cuda_device, decode, 32, 0, False, seed=6)
    ctx = t.append()
    both = torch.zeros(7, dtype=torch.int32, device=cuda_device)
    for out in (both[1:4], both[3:6]):
        with pytest.raises(binding.LsaError) as e:
            t.append(ctx, ctx_len=both[2:5], ctx_len_out=out)
        assert e.value.code == -1
    both[3:6] = t.before
    t.append(ctx, ctx_len=both[3:6], ctx_len_out=both[0:3])
    assert ctx.status() == 0 and both[:3].tolist() == [9, 64, 300]


def test_no_queries_no_lengths_no_tokens(cuda_device):
    c, t, old = make((8, 2, 64, 64), [3, 20], [3, 4], 16, "bf16", False, cuda_device, False, 32, 0, False, seed=7)
    ctx = t.append()
    want = c.k.clone()
    c.k.copy_(old[0])
    t.append(ctx, q=None, q_out=None, ctx_len_out=None)
    assert ctx.status() == 0 and torch.equal(c.k, want)
    # nobody has a new token: the lengths are handed on, and no pool is touched
    c, t, old = make((8, 2, 64, 64), [3, 20], [0, 0], 16, "bf16", False, cuda_device, False, 32, 0, False, seed=7)
    t.append(ctx)
    assert ctx.status() == 0 and t.after.tolist() == [3, 20] and torch.equal(c.k, old[0])


def test_tokens_that_do_not_fit_are_reported_and_skipped(cuda_device):
    lengths = [10, 40, 33, 20]
    c, t, old = make((8, 2, 64, 64), lengths, [1] * 4, 16, "bf16", False, cuda_device, True, 64, 0, False, seed=8)
    ctx = t.append()
    want = (c.k.clone(), c.v.clone(), t.q_out.clone())
    rows = [int(orc.paged_rows([n - 1], c.table[b], 16)[0]) for b, n in enumerate(lengths)]

    def run(spoil):
        c.k.copy_(old[0]), c.v.copy_(old[1]), t.q_out.fill_(3.0)
        c.page_table.copy_(torch.from_numpy(c.table))
        before = t.before.clone()
        spoil(before)
        t.append(ctx, ctx_len=before)
        assert ctx.status() == -7 and ctx.status() == 0
        for b in (0, 2, 3):
            assert torch.equal(c.k[rows[b]], want[0][rows[b]]) and torch.equal(c.v[rows[b]], want[1][rows[b]]) and torch.equal(t.q_out[b], want[2][b])
        others = torch.ones(c.k.shape[0], dtype=torch.bool, device=cuda_device)
        others[[rows[b] for b in (0, 2, 3)]] = False
        assert torch.equal(c.k[others], old[0][others]) and torch.equal(c.v[others], old[1][others])
        assert bool((t.q_out[1] == 3.0).all())

    def page(value):
        def spoil(before):
            c.page_table[1, 39 // 16] = value
        return spoil

    def length(value):
        def spoil(before):
            before[1] = value
        return spoil
    for spoil in (page(-1), page(c.n_pages), page(1 << 30), length(-1), length(c.table.shape[1] * 16), length((1 << 31) - 1)):
        run(spoil)
    # a position without angles
    t.cos_sin = t.cos_sin[:39].contiguous()
    run(lambda before: None)


def test_e4m3_rows_with_infinities_nan_and_extreme_sizes(cuda_device):
    """scale = amax / 448 over the numbers that are ones, code = value / scale: what fp32 division and the format give."""
    n = 8
    c, t, old = make((8, 2, 64, 64), [5] * n, [1] * n, 16, "bf16", True, cuda_device, True, 0, 0, False, seed=19)
    t.v[0, 0, 3] = torch.inf
    t.v[1, 0, 4] = torch.nan
    t.v[2] = t.v[2].float() * 2.0 ** -124      # scales near the smallest numbers: their reciprocals overflow
    t.v[3] = t.v[3].float() * 2.0 ** 126       # scales whose reciprocals are not normal numbers
    t.v[4] = 0
    t.v[5] = t.v[5].float() * 2.0 ** -132
    t.v[6, 1] = -torch.inf
    ctx = t.append()
    assert ctx.status() == 0
    x = t.v.float().cpu()
    top = x.abs().nan_to_num(nan=0.0, posinf=torch.inf).amax(-1)
    scale = torch.where(top / 448 == 0, torch.ones_like(top), top / 448)
    want = (x / scale[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    rows = [int(orc.paged_rows([4], c.table[b], 16)[0]) for b in range(n)]
    got = c.v[rows].view(torch.float8_e4m3fn).reshape(n, 2, 64).cpu()
    assert torch.equal(c.v_scale[rows].cpu(), scale)
    assert torch.equal(got.float().isnan(), want.float().isnan())
    assert torch.equal(got.float().nan_to_num(), want.float().nan_to_num())


def test_token_starts_that_leave_the_tokens_are_reported(cuda_device):
    c, t, old = make((8, 2, 64, 64), [3, 20], [3, 4], 16, "bf16", False, cuda_device, False, 0, 0, False, seed=9)
    ctx = t.append()
    assert ctx.status() == 0
    t.tok_start[2] = 8      # there are seven
    t.append(ctx)
    assert ctx.status() == -7


@pytest.mark.parametrize("shape,e4m3", [((16, 2, 128, 128), False), ((16, 2, 128, 128), True)])
def test_a_decode_loop_in_a_graph(cuda_device, shape, e4m3):
    """Prompts go in as chunks; then append and attention of every step are one captured graph, lengths advancing in place.
    Afterwards the cache is what one append of all tokens gives, bit for bit, and each step's result is the oracle's."""
    _decode_loop(cuda_device, shape, e4m3, 16)


def _decode_loop(dev, shape, e4m3, page):
    H, G, d, dv = shape
    steps, prompts = 9, [30, 0, 63, 7]
    lengths = [p + steps for p in prompts]
    d_rope, at = (64, 512) if d == 576 else (d, 0)
    c, t, old = make(shape, lengths, lengths, page, "bf16", e4m3, dev, False, d_rope, at, False, seed=10)
    t.append()                                  # all at once: what the cache and the queries have to be
    want_k, want_v, want_q = c.k.clone(), None if c.v is None else c.v.clone(), t.q_out.clone()
    c.k.copy_(old[0])
    if c.v is not None:
        c.v.copy_(old[1])
    st = torch.cuda.Stream(dev)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        ctx = binding.Context(None, 0, 0, 4, device=dev, stream=st, kv=t.params())
        lens = torch.zeros(4, dtype=torch.int32, device=dev)
        first = [int(s) for s in t.start[:-1]]
        idx = torch.tensor([first[b] + i for b in range(4) for i in range(prompts[b])], device=dev)
        ts = torch.tensor(np.concatenate([[0], np.cumsum(prompts)]).astype(np.int32), device=dev)
        pools = dict(k_scale=c.k_scale, v_scale=c.v_scale)
        ctx.kv_append(t.k[idx], None if t.v is None else t.v[idx], c.k, c.v, c.page_table, lens, lens, tok_start=ts, cos_sin=t.cos_sin, **pools)
        q, k = torch.empty(4, H, d, dtype=torch.bfloat16, device=dev), torch.empty(4, G, d, dtype=torch.bfloat16, device=dev)
        v = None if c.v is None else torch.empty(4, G, dv, dtype=torch.bfloat16, device=dev)
        out, lse = torch.empty(4, H, dv, dtype=torch.bfloat16, device=dev), torch.empty(4, H, device=dev)
    torch.cuda.synchronize()
    assert ctx.status() == 0 and lens.tolist() == prompts
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        ctx.kv_append(k, v, c.k, c.v, c.page_table, lens, lens, q=q, q_out=q, cos_sin=t.cos_sin, **pools)
        ctx.paged_attn(q, c.k, c.v, c.page_table, lens, out, lse, **pools)
    for s in range(steps):
        at_tok = torch.tensor([first[b] + prompts[b] + s for b in range(4)], device=dev)
        q.copy_(t.q[at_tok]), k.copy_(t.k[at_tok])
        if v is not None:
            v.copy_(t.v[at_tok])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.status() == 0 and lens.tolist() == [p + s + 1 for p in prompts]
        assert torch.equal(q, want_q[at_tok])
        c.lengths, c.q = [p + s + 1 for p in prompts], q
        pu.check_attend(c, out, lse)
    used = torch.from_numpy(c.used_rows()).to(dev)
    assert torch.equal(c.k[used], want_k[used]) and (c.v is None or torch.equal(c.v[used], want_v[used]))
