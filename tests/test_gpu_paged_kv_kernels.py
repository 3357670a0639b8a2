"""Every kernel of lsa_kv_append and lsa_paged_attn, on both sides of the rules that choose it (needs a B200)."""
import numpy as np
import pytest
import torch

import paged_util as pu
from paper_2608_01662_b200 import binding
from test_gpu_kv_append import make
from test_gpu_paged_attn import RAGGED

pytestmark = pytest.mark.gpu

FORMS = [("bf16", False), ("fp16", False), ("bf16", True), ("fp16", True)]


# ---- append.  Blocks of 512 threads (latent rows: 576) for as many tokens as there are SMs, if a token has more rows than four trips of
# the smaller block; else of 64 (288).  More rows than a block takes at once: 64 over 8 heads of 128 dims and 72 over 18 of 64 for queries,
# 40 over 20 and 72 over 18 for keys and values.
APPEND_WIDE = [(64, 8, 128, 128), (40, 20, 128, 128), (96, 8, 128, 128), (72, 18, 64, 64), (80, 8, 64, 64)]


@pytest.mark.parametrize("shape", APPEND_WIDE)
@pytest.mark.parametrize("dtype,e4m3", FORMS)
@pytest.mark.parametrize("tokens", [100, 160])
def test_append_of_wide_tokens(cuda_device, shape, dtype, e4m3, tokens):
    """One token each for 100 and 160 sequences: both sides of the number of SMs."""
    assert 100 <= torch.cuda.get_device_properties(cuda_device).multi_processor_count < 160
    lengths = [1 + (7 * b) % 40 for b in range(tokens)]
    c, t, old = make(shape, lengths, [1] * tokens, 16, dtype, e4m3, cuda_device, True, 64, 0, sum(shape) % 3 == 0, seed=tokens)
    ctx = t.append()
    assert ctx.status() == 0
    t.check(*old)


@pytest.mark.parametrize("shape", APPEND_WIDE)
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new", [[60, 0, 1, 39], [150, 3, 0, 58]])
def test_append_of_runs_of_wide_tokens(cuda_device, shape, e4m3, new):
    lengths = [n + 11 * i for i, n in enumerate(new)]
    c, t, old = make(shape, lengths, new, 32, "bf16", e4m3, cuda_device, False, 32, 16, True, seed=sum(new), tail=3, fused=True)
    ctx = t.append()
    assert ctx.status() == 0
    t.check(*old)


@pytest.mark.parametrize("heads", [1, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("new", [[70, 0, 1, 20], [160, 0, 1, 40]])
def test_append_of_runs_of_latent_rows(cuda_device, heads, dtype, new):
    lengths = [n + 50 * i for i, n in enumerate(new)]
    c, t, old = make((heads, 1, 576, 512), lengths, new, 64, dtype, False, cuda_device, False, 64, 512, heads % 2 == 0, seed=heads, tail=2)
    ctx = t.append()
    assert ctx.status() == 0
    t.check(*old)


@pytest.mark.parametrize("shape", [(64, 8, 128, 128), (64, 1, 576, 512), (16, 1, 576, 512)])
def test_append_in_place_and_without_queries(cuda_device, shape):
    """The larger blocks again with q rotated where it lies, and with keys and values only."""
    for tokens in (100, 160):
        at, d_rope = (512, 64) if shape[2] == 576 else (0, 128)
        c, t, old = make(shape, [5] * tokens, [1] * tokens, 64, "bf16", False, cuda_device, True, d_rope, at, True, seed=34)
        ctx = t.append()
        k, v, q_out, q = c.k.clone(), None if c.v is None else c.v.clone(), t.q_out.clone(), t.q.clone()
        for more in (dict(q=q, q_out=q), dict(q=None, q_out=None)):
            for pool, o in ((c.k, old[0]), (c.v, old[1])):
                if pool is not None:
                    pool.copy_(o)
            t.append(ctx, **more)
            assert ctx.status() == 0 and torch.equal(c.k, k) and (v is None or torch.equal(c.v, v)) and torch.equal(q, q_out)


# (4 GB of rows, each filled with one number, so that a row written in the wrong place is one that differs)
@pytest.mark.parametrize("shape", [(16, 8, 128, 128), (16, 1, 576, 512)])
def test_append_past_32_bit_byte_offsets(cuda_device, shape):
    new = [60, 0, 33]
    c, t, old = make(shape, [70, 5, 33], new, 64, "bf16", False, cuda_device, False, 64, shape[2] - 64, False, seed=35)
    ctx = t.append()
    assert ctx.status() == 0
    rows = (9 << 28) // shape[2] // shape[1] // 64 * 64     # 4.5 GB
    off = rows - c.k.shape[0]
    big = torch.ones(rows, c.k.shape[1], dtype=torch.bfloat16, device=cuda_device)
    big[off:] = old[0]
    big_v = None if c.v is None else torch.ones(rows, c.v.shape[1], dtype=torch.bfloat16, device=cuda_device)
    if big_v is not None:
        big_v[off:] = old[1]
    table = torch.where(c.page_table >= 0, c.page_table + off // 64, c.page_table)
    ctx.kv_append(t.k, t.v, big, big_v, table, t.before, t.after, tok_start=t.tok_start, cos_sin=t.cos_sin)
    assert ctx.status() == 0
    for pool, want in ((big, c.k), (big_v, c.v)):
        if pool is not None:
            assert torch.equal(pool[off:], want) and bool((pool[:off] == 1).all())


# ---- attention
def test_latent_rows_past_32_bit_byte_offsets(cuda_device):
    small = pu.Cache([150, 90], (16, 1, 576, 512), 64, "bf16", False, cuda_device, seed=36)
    rows = (9 << 28) // 576 // 64 * 64
    off = rows - small.k.shape[0]
    k = torch.zeros(rows, 576, dtype=torch.bfloat16, device=cuda_device)
    k[off:] = small.k
    ctx = binding.Context(None, 0, 0, 2, device=cuda_device, kv=small.params())
    out, lse = torch.empty(2, 16, 512, dtype=torch.bfloat16, device=cuda_device), torch.empty(2, 16, device=cuda_device)
    table = torch.where(small.page_table >= 0, small.page_table + off // 64, small.page_table)
    ctx.paged_attn(small.q, k, None, table, small.ctx_len, out, lse)
    assert ctx.status() == 0
    pu.check_attend(small, out, lse)


# 9 to 16 query heads per KV head are two groups of eight columns: full, and with absent heads in the second; with 1, 2, 4 and 8 KV heads in a
# block, alone and with others
PAIRED = [(128, 8, 128, 128), (64, 4, 128, 128), (32, 2, 64, 64), (96, 6, 64, 64), (16, 1, 64, 64), (36, 3, 128, 128), (72, 8, 128, 128),
          (30, 2, 64, 64), (60, 4, 128, 128), (11, 1, 64, 64)]


@pytest.mark.parametrize("dtype,e4m3", FORMS)
@pytest.mark.parametrize("shape", PAIRED)
def test_nine_to_sixteen_heads_per_kv_head(cuda_device, shape, dtype, e4m3):
    page = [16, 32, 64, 128, 256][sum(shape) % 5]
    c = pu.Cache(RAGGED, shape, page, dtype, e4m3, cuda_device, seed=sum(shape), poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


@pytest.mark.parametrize("dtype,e4m3", [("bf16", False), ("fp16", True)])
@pytest.mark.parametrize("shape", [(128, 8, 128, 128), (36, 3, 128, 128), (72, 8, 128, 128), (30, 2, 64, 64), (96, 6, 64, 64)])
@pytest.mark.parametrize("lengths", [[400] * 3, [700] * 9, [2500, 6000]])
def test_parts_of_nine_to_sixteen_heads_per_kv_head(cuda_device, shape, dtype, e4m3, lengths):
    c = pu.Cache(lengths, shape, 16, dtype, e4m3, cuda_device, seed=sum(lengths) + shape[0], poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
    again = pu.attend(c, ctx)[1:]
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("shape,dtype,e4m3", [((32, 8, 128, 128), "bf16", False), ((32, 8, 128, 128), "fp16", False), ((16, 1, 128, 128), "bf16", False),
                                              ((8, 2, 64, 64), "fp16", False), ((16, 8, 64, 64), "bf16", True), ((32, 2, 128, 128), "fp16", True),
                                              ((64, 1, 576, 512), "fp16", False), ((64, 1, 576, 512), "bf16", False)])
@pytest.mark.parametrize("page", [64, 128, 16])
@pytest.mark.parametrize("sink,window", [(0, 16), (4, 100), (65, 33), (130, 257)])
def test_sink_and_window_of_other_tiles(cuda_device, shape, dtype, e4m3, page, sink, window):
    """Strips of 16 tokens (128 dims) and of 32, one to eight KV heads in a block, both 16-bit types."""
    if shape[2] == 576 and page == 16:
        page = 256
    c = pu.Cache(RAGGED, shape, page, dtype, e4m3, cuda_device, seed=page + sink + window)
    c.poison(sink, window)
    ctx, out, lse = pu.attend(c, sink=sink, window=window)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse, sink, window)


@pytest.mark.parametrize("shape", [(16, 16, 64, 64), (12, 6, 64, 64), (24, 24, 128, 128)])
@pytest.mark.parametrize("dtype,e4m3", [("bf16", False), ("bf16", True)])
@pytest.mark.parametrize("batch", [40, 70])
def test_many_sequences_of_several_blocks_of_heads(cuda_device, shape, dtype, e4m3, batch):
    rng = np.random.default_rng(batch)
    lengths = [int(x) for x in rng.integers(0, 400, batch)]
    c = pu.Cache(lengths, shape, 16, dtype, e4m3, cuda_device, seed=37, poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
