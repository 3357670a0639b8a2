"""lsa_kv_append and lsa_paged_attn at the ends of their ranges (needs a B200)."""
import numpy as np
import pytest
import torch

import paged_util as pu
from oracle import lsa_oracle as orc
from paper_2608_01662_b200 import binding
from test_gpu_kv_append import make

pytestmark = pytest.mark.gpu


def test_codes_beside_midpoints_for_scales_of_every_size(cuda_device):
    """e4m3 keys whose quotients by the scale lie at midpoints between codes, as near as fp32 values come to them, for scales from the
    subnormal numbers up: the code is that of the fp32 quotient, as IEEE division rounds it.  No value here is rounded before: a key is a
    power of two times an angle's cosine or sine."""
    rng = np.random.default_rng(31)
    exps = list(range(-128, -84)) + list(range(-80, 77, 12))
    n, half = len(exps), 32
    c, t, old = make((8, 2, 64, 64), [b + 1 for b in range(n)], [1] * n, 16, "bf16", True, cuda_device, True, 64, 0, False, seed=31)
    want = np.zeros((n, 64), np.float32)
    mids = np.array([(m + 0.5) / 8 * 2.0 ** e for m in range(8, 16) for e in range(-6, 8)] + [(m + 0.5) * 2.0 ** -9 for m in range(8)])
    for b, e in enumerate(exps):
        top = np.float32(448 * 2.0 ** (e + rng.random()))
        scale = np.float32(top / np.float32(448))
        near = (rng.choice(mids[mids < 440], 63) * np.float64(scale)).astype(np.float32)
        want[b] = np.concatenate([[top], near * rng.choice([-1.0, 1.0], 63).astype(np.float32)])
    up = 2.0 ** 40
    t.k[:, :, :half] = 2.0 ** -40
    t.k[:, :, half:] = 0
    # (halves: dim j becomes x cos_j, dim j + 32 becomes x sin_j)
    t.cos_sin = torch.from_numpy((want.astype(np.float64) * up).astype(np.float32)).to(cuda_device).contiguous()
    ctx = t.append()
    assert ctx.status() == 0
    x = torch.from_numpy(want)
    scale = x.abs().amax(-1) / 448
    codes = (x / scale[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    rows = [int(orc.paged_rows([b], c.table[b], 16)[0]) for b in range(n)]
    for g in range(2):
        assert torch.equal(c.k_scale[rows].cpu()[:, g], scale)
        wrong = (c.k[rows].cpu()[:, 64 * g:64 * g + 64] != codes).any(1)
        assert not bool(wrong.any()), [exps[b] for b in range(n) if wrong[b]]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scales_of_scores_that_underflow(cuda_device, dtype):
    """e4m3: sm_scale times a query's size is far below the smallest fp32 number, so every seen token weighs the same; the hidden ones at
    the end of a strip nothing."""
    c = pu.Cache([1, 50, 77, 300, 2000], (8, 2, 64, 64), 16, dtype, True, cuda_device, seed=32, poison=True)
    c.q *= 2.0 ** (-90 if dtype == "bf16" else -10)
    ctx, out, lse = pu.attend(c, sm_scale=2.0 ** -90)
    assert ctx.status() == 0
    c.q.zero_()      # the same weights: scores of 0
    pu.check_attend(c, out, lse)


def test_append_without_a_workspace_is_refused(cuda_device):
    """Tokens that find no place are reported through words in the workspace: without one nobody would learn of them."""
    import ctypes

    c, t, old = make((8, 2, 64, 64), [9, 20], [1, 1], 16, "bf16", False, cuda_device, True, 32, 0, False, seed=33)
    ctx = t.append()
    bare = ctypes.c_void_p()
    assert binding.lib().lsa_create(ctypes.byref(bare), cuda_device.index or 0, ctypes.c_void_p(ctx.stream.cuda_stream), None, 0) == 0
    with_workspace, ctx.h = ctx.h, bare
    try:
        with pytest.raises(binding.LsaError) as e:
            t.append(ctx)
        assert e.value.code == -3
    finally:
        ctx.h = with_workspace
        binding.lib().lsa_destroy(bare)


def test_sparse_attention_right_after_an_append_of_another_context(cuda_device):
    """The row lists stay, the rows do not: each step's append writes every sequence's last row, and the attention launched right behind
    it, on the lists of the attention before, reads the new one."""
    from paper_2608_01662_b200.configs import CONFIGS
    from paper_2608_01662_b200.workload import DecodeWorkload
    cfg = CONFIGS["cfg4"].replace(batch=64, ctx_lo=300, ctx_hi=3000, M=64, Ksp=1024, R=1)
    wl = DecodeWorkload(cfg, cuda_device)
    wl.prepare()
    wl.step()
    rows = torch.empty((cfg.batch, cfg.S + cfg.Ksp + cfg.W), dtype=torch.int32, device=cuda_device)
    n_rows = torch.empty((cfg.batch,), dtype=torch.int32, device=cuda_device)
    wl.ctx.convert(wl.sparse_idx, wl.n_sparse, 0, cfg.batch, rows, n_rows, None, wl.page_table, wl.ctx_len)
    kv = binding.Context(None, 0, 0, device=cuda_device, kv=binding.make_kv_params(64, 1, 576, 512, cfg.kv_page, latent=True))
    steps, before = 24, wl.ctx_len - 1
    gen = torch.Generator(cuda_device).manual_seed(38)
    new = torch.randn(steps, cfg.batch, 576, generator=gen, device=cuda_device).mul(3).to(torch.bfloat16)
    pool = wl.k[0].view(-1, wl.k[0].shape[-1])

    def step(s, out):
        kv.kv_append(new[s].view(cfg.batch, 1, 576), None, pool, None, wl.page_table, before)
        wl.ctx.sparse_attn(wl.q[0], wl.k[0], wl.v[0], wl.sparse_idx, wl.n_sparse, 0, cfg.batch, 0, out, None, rows, n_rows, wl.ctx_len, cfg.batch)
    outs = torch.empty(2, steps, *wl.out[0].shape, dtype=torch.bfloat16, device=cuda_device)
    torch.cuda.synchronize()
    for s in range(steps):
        step(s, outs[0, s])
    assert wl.ctx.status() == 0 and kv.status() == 0
    for s in range(steps):
        kv.kv_append(new[s].view(cfg.batch, 1, 576), None, pool, None, wl.page_table, before)
        torch.cuda.synchronize()
        step(s, outs[1, s])
        torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    assert not torch.equal(outs[0, 0], outs[0, 1])


def test_one_context_for_the_sparse_and_the_dense_calls(cuda_device):
    """Both take their scratch from one workspace, in turn: neither changes what the other gives."""
    from paper_2608_01662_b200.configs import CONFIGS
    from paper_2608_01662_b200.workload import DecodeWorkload
    cfg = CONFIGS["cfg4"].replace(batch=20, ctx_lo=300, ctx_hi=5000, M=64, Ksp=1024, R=2)
    wl = DecodeWorkload(cfg, cuda_device)
    wl.prepare()
    wl.step()
    want = [x.clone() for x in (*wl.out, *wl.lse, wl.sparse_idx)]
    kv = binding.make_kv_params(64, 1, 576, 512, cfg.kv_page, latent=True, sm_scale=cfg.sm_scale)
    max_ctx = wl.page_table.shape[1] * cfg.kv_page
    wl.ctx = binding.Context(wl.params, cfg.batch, max_ctx, cfg.batch, device=cuda_device, kv=kv)
    alone = binding.Context(None, 0, 0, device=cuda_device, kv=kv)
    pool = wl.k[1].view(-1, wl.k[1].shape[-1])
    dense = [torch.empty_like(wl.out[0]) for _ in range(2)]
    alone.paged_attn(wl.q[1], pool, None, wl.page_table, wl.ctx_len, dense[0])
    row = wl.ctx_len - 1
    for _ in range(5):
        for x in (*wl.out, *wl.lse, wl.sparse_idx):
            x.zero_()
        last = torch.arange(cfg.batch, device=cuda_device)
        rows = wl.page_table[last, row // cfg.kv_page].long() * cfg.kv_page + row % cfg.kv_page
        wl.ctx.kv_append(pool[rows].view(cfg.batch, 1, 576), None, pool, None, wl.page_table, row)   # (what is there already)
        wl.ctx.paged_attn(wl.q[1], pool, None, wl.page_table, wl.ctx_len, dense[1])
        wl.step()
        assert wl.ctx.status() == 0
        assert all(torch.equal(x, y) for x, y in zip((*wl.out, *wl.lse, wl.sparse_idx), want))
        assert torch.equal(dense[0], dense[1])
        dense[1].zero_()


@pytest.mark.parametrize("shape", [(16, 2, 128, 128), (64, 1, 576, 512)])
def test_padded_batches_in_two_graphs_of_one_context(cuda_device, shape):
    """Steps of up to four sequences, two graphs replayed in turn on one workspace: what a place without a sequence holds is neither read
    nor written, its result is 0."""
    H, G, d, dv = shape
    page, steps, places = 64, 6, 4
    lengths = [30 + steps, 400 + steps, 63 + steps]
    c = pu.Cache(lengths, shape, page, "bf16", False, cuda_device, seed=39)
    st = torch.cuda.Stream(cuda_device)
    torch.cuda.synchronize()
    table = torch.full((places, c.table.shape[1]), -1, dtype=torch.int32, device=cuda_device)
    lens = torch.zeros(places, dtype=torch.int32, device=cuda_device)
    starts = torch.zeros(places + 1, dtype=torch.int32, device=cuda_device)
    rows = {}
    gen = torch.Generator(cuda_device).manual_seed(40)
    new_k = torch.randn(places, G, d, generator=gen, device=cuda_device).to(torch.bfloat16)
    new_v = None if c.v is None else torch.randn(places, G, dv, generator=gen, device=cuda_device).to(torch.bfloat16)
    q = torch.randn(places, H, d, generator=gen, device=cuda_device).to(torch.bfloat16)
    graphs, outs = [], []
    with torch.cuda.stream(st):
        ctx = binding.Context(None, 0, 0, device=cuda_device, stream=st, kv=c.params())
        for _ in range(2):
            outs.append((torch.full((places, H, dv), 7.0, dtype=torch.bfloat16, device=cuda_device), torch.full((places, H), 7.0, device=cuda_device)))
    torch.cuda.synchronize()
    for out, lse in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            ctx.kv_append(new_k, new_v, c.k, c.v, table, lens, lens, tok_start=starts)
            ctx.paged_attn(q, c.k, c.v, table, lens, out, lse)
        graphs.append(g)
    full = list(lengths)
    for s in range(steps):
        here = [0, 1, 2] if s % 3 else [1, 2]          # the sequences of this step; the others' places are empty
        table.fill_(-1)
        lens.zero_()
        now = {b: rows.get(b, full[b] - steps) for b in here}
        for place, b in enumerate(here):
            table[place] = c.page_table[b]
            lens[place] = now[b]
        starts.copy_(torch.tensor([min(i, len(here)) for i in range(places + 1)], dtype=torch.int32))
        new_k.normal_(generator=gen)
        if new_v is not None:
            new_v.normal_(generator=gen)
        new_k[len(here):] = float("nan")
        q.normal_(generator=gen)
        q[len(here):] = float("nan")
        torch.cuda.synchronize()
        before = c.k.clone()
        graphs[s % 2].replay()
        torch.cuda.synchronize()
        assert ctx.status() == 0 and lens.tolist() == [now[b] + 1 for b in here] + [0] * (places - len(here))
        written = [int(orc.paged_rows([now[b]], c.table[b], page)[0]) for b in here]
        same = torch.ones(c.k.shape[0], dtype=torch.bool, device=cuda_device)
        same[written] = False
        assert torch.equal(c.k[same], before[same]) and torch.equal(c.k[written], new_k[:len(here)].reshape(len(here), -1))
        out, lse = outs[s % 2]
        c.lengths = [now[b] + 1 if b in now else 0 for b in range(3)]
        order = torch.tensor([here.index(b) if b in here else 3 for b in range(3)], device=cuda_device)   # (place 3 is always empty)
        c.q = q[order]
        pu.check_attend(c, out[order], lse[order], sequences=here)
        assert bool((out[len(here):] == 0).all()) and bool((lse[len(here):] == -torch.inf).all())
        rows.update({b: now[b] + 1 for b in here})


@pytest.mark.parametrize("shape,e4m3", [((16, 2, 128, 128), False), ((16, 2, 128, 128), True), ((24, 1, 576, 512), False)])
def test_sequences_that_share_pages(cuda_device, shape, e4m3):
    """A common beginning is cached once: its pages stand in several rows of the table, and one sequence stands there twice."""
    c = pu.Cache([1000, 700, 900, 1000], shape, 64, "bf16", e4m3, cuda_device, seed=41)
    c.table[1, :8] = c.table[0, :8]
    c.table[2, :3] = c.table[0, :3]
    c.table[3] = c.table[0]
    c.page_table.copy_(torch.from_numpy(c.table))
    c.q[3] = c.q[0]
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
