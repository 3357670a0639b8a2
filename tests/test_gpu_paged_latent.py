"""lsa_paged_attn over latent rows against the oracle (needs a B200)."""
import numpy as np
import pytest
import torch

import paged_util as pu
from paper_2608_01662_b200 import binding
from test_gpu_kv_append import _decode_loop
from test_gpu_paged_attn import RAGGED

pytestmark = pytest.mark.gpu

LATENT = (64, 1, 576, 512)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lengths", [[1], [64], [65], [0], [200], [0, 5, 0], [1000], [63, 64, 65, 128, 1]])
def test_few_tokens(cuda_device, lengths, dtype):
    c = pu.Cache(lengths, LATENT, 64, dtype, False, cuda_device, seed=sum(lengths), poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


@pytest.mark.parametrize("heads", [1, 5, 16, 33, 64])
@pytest.mark.parametrize("page", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_heads_and_pages(cuda_device, heads, page, dtype):
    c = pu.Cache(RAGGED, (heads, 1, 576, 512), page, dtype, False, cuda_device, seed=heads + page, poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


@pytest.mark.parametrize("page", [64, 256])
@pytest.mark.parametrize("sink,window", [(0, 1), (4, 100), (65, 33), (130, 257), (0, 5000)])
def test_sink_and_window(cuda_device, page, sink, window):
    c = pu.Cache(RAGGED, (8, 1, 576, 512), page, "bf16", False, cuda_device, seed=page + sink + window)
    c.poison(sink, window)
    ctx, out, lse = pu.attend(c, sink=sink, window=window)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse, sink, window)


@pytest.mark.parametrize("lengths", [[30000], [40001, 3], [1, 1, 20000, 1, 2], [5000] * 7])
def test_long_sequences_are_split_and_joined(cuda_device, lengths):
    c = pu.Cache(lengths, (20, 1, 576, 512), 64, "bf16", False, cuda_device, seed=len(lengths))
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
    again = pu.attend(c, ctx)[1:]
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("heads", [64, 7])
@pytest.mark.parametrize("lengths", [[130], [250] * 3, [400] * 12, [777] * 10, [1300] * 9, [2000, 70, 900]])
def test_joins_of_few_some_and_many_parts(cuda_device, heads, lengths):
    """Sequences in 2 to 32 parts, alone and several of them."""
    c = pu.Cache(lengths, (heads, 1, 576, 512), 64, "bf16", False, cuda_device, seed=sum(lengths) + heads, poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
    out2 = torch.empty_like(out)
    ctx.paged_attn(c.q, c.k, None, c.page_table, c.ctx_len, out2)
    torch.cuda.synchronize()
    assert torch.equal(out, out2)


def test_many_short_sequences(cuda_device):
    rng = np.random.default_rng(5)
    lengths = [int(x) for x in rng.integers(0, 150, 500)]
    c = pu.Cache(lengths, (3, 1, 576, 512), 64, "bf16", False, cuda_device, seed=6, poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scores_that_grow_along_the_sequence(cuda_device, dtype):
    """Running maxima that move at nearly every tile, by more than the gap that triggers a rescaling; by another amount in each head."""
    c = pu.Cache([900, 12000], (16, 1, 576, 512), 64, dtype, False, cuda_device, seed=8)
    c.q[:] = c.q[:, :, :1].abs().clamp(min=0.5, max=3)
    for b, n in enumerate(c.lengths):
        rows = torch.from_numpy(pu.orc.paged_rows(np.arange(n), c.table[b], c.page)).to(cuda_device)
        c.k[rows] = (torch.linspace(-40, 40, n, device=cuda_device)[:, None] / 8).expand(n, 576).to(c.k.dtype)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


def test_minus_infinite_scores(cuda_device):
    c = pu.Cache([64, 700], (2, 1, 576, 512), 64, "bf16", False, cuda_device, seed=11)
    c.q[:] = 0
    c.q[:, :, 575] = 1                      # a dim that no value has
    plain = c.k.clone()
    for b, n in enumerate(c.lengths):
        rows = torch.from_numpy(pu.orc.paged_rows(np.arange(n), c.table[b], c.page)).to(cuda_device)
        gone = rows[: n - 3] if b else rows[::2]
        c.k[gone, 575] = -torch.inf
        plain[gone, 575] = -3e38
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    c.k = plain
    pu.check_attend(c, out, lse)


def test_nan_stays_with_its_sequence(cuda_device):
    c = pu.Cache([50, 60, 200], (6, 1, 576, 512), 64, "bf16", False, cuda_device, seed=12)
    c.k[int(pu.orc.paged_rows([31], c.table[1], 64)[0]), 570] = torch.nan
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    assert bool(out[1].isnan().all()) and bool(lse[1].isnan().all())
    pu.check_attend(c, out, lse, sequences=[0, 2])


def test_pitches_and_absent_lse(cuda_device):
    c = pu.Cache(RAGGED, (12, 1, 576, 512), 64, "bf16", False, cuda_device, seed=13, pad=64, width=40)
    B = len(RAGGED)
    wide_q = torch.zeros(B, 15, 576, dtype=torch.bfloat16, device=cuda_device)
    wide_q[:, 2:14] = c.q
    c.q = wide_q[:, 2:14]
    wide = torch.full((B, 14, 512), 5.0, dtype=torch.bfloat16, device=cuda_device)
    ctx, out, lse = pu.attend(c, out=wide[:, 1:13])
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
    assert bool((wide[:, 0] == 5).all()) and bool((wide[:, -1] == 5).all())
    ref = out.clone()
    out.zero_()
    ctx.paged_attn(c.q, c.k, None, c.page_table, c.ctx_len, out)
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


def test_bad_pages_and_lengths_are_reported_and_stay_with_their_sequence(cuda_device):
    c = pu.Cache([100, 200, 300, 40], (64, 1, 576, 512), 64, "bf16", False, cuda_device, seed=14)
    ctx = None
    for value in (c.n_pages, -5, 1 << 30):
        c.page_table[1, 1] = value
        ctx, out, lse = pu.attend(c, ctx)
        assert ctx.status() == -7 and ctx.status() == 0
        pu.check_attend(c, out, lse, sequences=[0, 2, 3])
    c.page_table.copy_(torch.from_numpy(c.table))
    c.ctx_len[3] = -1
    c.ctx_len[0] = c.table.shape[1] * 64 + 1
    out, lse = pu.attend(c, ctx)[1:]
    assert ctx.status() == -7
    pu.check_attend(c, out, lse, sequences=[1, 2])
    assert bool((out[3] == 0).all()) and bool((lse[3] == -torch.inf).all())
    c.ctx_len.copy_(torch.tensor(c.lengths, dtype=torch.int32))
    out, lse = pu.attend(c, ctx)[1:]
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


def test_another_stream_and_a_captured_graph(cuda_device):
    st = torch.cuda.Stream(cuda_device)
    c = pu.Cache([300, 1, 5000, 0], LATENT, 64, "bf16", False, cuda_device, seed=16, width=90)
    out, lse = torch.empty(4, 64, 512, dtype=torch.bfloat16, device=cuda_device), torch.empty(4, 64, device=cuda_device)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        ctx = binding.Context(None, 0, 0, 4, device=cuda_device, stream=st, kv=c.params())
        pu.attend(c, ctx, out, lse)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        pu.attend(c, ctx, out, lse)
    for lengths in ([300, 1, 5000, 0], [10, 1, 2999, 0], [0, 0, 17, 0]):
        c.lengths = lengths
        c.ctx_len.copy_(torch.tensor(lengths, dtype=torch.int32))
        c.q.mul_(0.9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.status() == 0
        pu.check_attend(c, out, lse)


def test_a_decode_loop_in_a_graph(cuda_device):
    _decode_loop(cuda_device, LATENT, False, 64)


def test_dense_and_sparse_attention_of_the_same_cache(cuda_device):
    """A budget that covers the context: lsa_layer_group's attention and the dense one see the same tokens."""
    from paper_2608_01662_b200.configs import CONFIGS
    from paper_2608_01662_b200.workload import DecodeWorkload
    cfg = CONFIGS["cfg4"].replace(batch=3, ctx_lo=500, ctx_hi=2000, M=64, Ksp=2048, R=1)
    wl = DecodeWorkload(cfg, cuda_device)
    wl.prepare()
    wl.step()
    assert wl.ctx.status() == 0
    kv = binding.make_kv_params(64, 1, 576, 512, 64, latent=True, sm_scale=cfg.sm_scale)
    ctx = binding.Context(wl.params, cfg.batch, cfg.ctx_hi, cfg.batch, device=cuda_device, kv=kv)
    out, lse = torch.empty_like(wl.out[0]), torch.empty(3, 64, device=cuda_device)
    ctx.paged_attn(wl.q[0], wl.k[0], None, wl.page_table, wl.ctx_len, out, lse)
    assert ctx.status() == 0
    # both within bf16 weights and one rounding of the same sums: two times (2 u) of the mass, whose mean |v| is below 1
    assert float((out.double() - wl.out[0].double()).abs().max()) <= 4 * 2.0 ** -8


def test_many_small_weights(cuda_device):
    c = pu.many_small_weights((64, 1, 576, 512), 64, cuda_device)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse, sequences=[0, 7, 39])


@pytest.mark.parametrize("lengths", [[300] * 64, [400] * 150, [64 * k for k in range(1, 40)], [1000, 0, 1] * 25, [63, 65, 64 * 8, 64 * 7 + 1] * 20])
def test_cuts_near_the_ends_of_sequences(cuda_device, lengths):
    """Lists whose cuts fall near sequences' ends and are moved there, beside others that are not."""
    c = pu.Cache(lengths, (3, 1, 576, 512), 64, "bf16", False, cuda_device, seed=26, poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
