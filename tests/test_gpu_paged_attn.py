"""lsa_paged_attn against the oracle (needs a B200): kinds of cache, lengths, masks, garbage where nobody looks, streams, graphs."""
import numpy as np
import pytest
import torch

import paged_util as pu
from paper_2608_01662_b200 import binding

pytestmark = pytest.mark.gpu

RAGGED = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300, 511, 0, 777, 1000]
# (query heads, KV heads, d_qk, d_v)
GROUPED = [(32, 8, 128, 128), (16, 1, 128, 128), (4, 4, 64, 64), (10, 2, 64, 64), (7, 1, 128, 128), (18, 6, 64, 64), (48, 3, 128, 128), (1, 1, 64, 64),
           (16, 16, 128, 128)]


@pytest.mark.parametrize("dtype,e4m3", [("bf16", False), ("fp16", False), ("bf16", True), ("fp16", True)])
@pytest.mark.parametrize("shape", GROUPED)
def test_grouped_heads(cuda_device, shape, dtype, e4m3):
    page = [16, 32, 64, 128, 256][sum(shape) % 5]
    c = pu.Cache(RAGGED, shape, page, dtype, e4m3, cuda_device, seed=sum(shape), poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("sink,window", [(0, 1), (0, 16), (4, 100), (20, 64), (65, 33), (130, 257), (0, 5000), (7, 1)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_sink_and_window(cuda_device, page, sink, window, e4m3):
    c = pu.Cache(RAGGED, (8, 2, 64, 64), page, "bf16", e4m3, cuda_device, seed=page + sink + window)
    c.poison(sink, window)
    ctx, out, lse = pu.attend(c, sink=sink, window=window)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse, sink, window)


def test_hidden_pages_need_not_be_mapped(cuda_device):
    """Pages between the sink and the window, and behind the last token, may be gone from the table."""
    sink, window = 20, 100
    c = pu.Cache([1000, 640, 90, 2000], (8, 2, 64, 64), 16, "bf16", False, cuda_device, seed=3)
    for b, n in enumerate(c.lengths):
        seen = {int(s) // 16 for s in pu.orc.seen_tokens(n, sink, window)}
        for i in range(c.table.shape[1]):
            if i not in seen:
                c.page_table[b, i] = -1
    ctx, out, lse = pu.attend(c, sink=sink, window=window)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse, sink, window)


@pytest.mark.parametrize("lengths", [[40000], [70001, 3], [1, 1, 30000, 1, 2], [9000] * 5, [0, 0, 0], [0], [1]])
@pytest.mark.parametrize("shape,dtype,e4m3", [((16, 1, 128, 128), "bf16", False), ((32, 8, 128, 128), "bf16", True), ((6, 6, 64, 64), "fp16", False)])
def test_long_sequences_are_split_and_joined(cuda_device, lengths, shape, dtype, e4m3):
    c = pu.Cache(lengths, shape, 64, dtype, e4m3, cuda_device, seed=len(lengths))
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
    again = pu.attend(c, ctx)[1:]
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])   # the same call gives the same bits


@pytest.mark.parametrize("shape", [(32, 8, 128, 128), (16, 1, 128, 128), (12, 4, 64, 64), (9, 3, 64, 64)])
@pytest.mark.parametrize("lengths", [[130], [300] * 3, [500, 500], [700] * 9, [1500, 40, 1500], [2500, 6000]])
def test_joins_of_few_some_and_many_parts(cuda_device, shape, lengths):
    """Sequences in 2 to 100 parts, alone and several of them."""
    c = pu.Cache(lengths, shape, 16, "bf16", False, cuda_device, seed=sum(lengths) + shape[0], poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
    out2 = torch.empty_like(out)
    ctx.paged_attn(c.q, c.k, c.v, c.page_table, c.ctx_len, out2)
    torch.cuda.synchronize()
    assert torch.equal(out, out2)


def test_large_batches(cuda_device):
    rng = np.random.default_rng(5)
    lengths = [int(x) for x in rng.integers(0, 90, 700)]
    c = pu.Cache(lengths, (4, 2, 64, 64), 16, "bf16", False, cuda_device, seed=6, poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


@pytest.mark.parametrize("dtype,e4m3", [("bf16", False), ("fp16", False), ("bf16", True)])
def test_scores_that_grow_along_the_sequence(cuda_device, dtype, e4m3):
    """Running maxima that move at nearly every strip, by more than the gap that triggers a rescaling."""
    c = pu.Cache([900, 3000], (8, 2, 128, 128), 64, dtype, e4m3, cuda_device, seed=8)
    c.q[:] = c.q[:, :, :1].abs().clamp(min=0.5, max=3)
    for b, n in enumerate(c.lengths):
        rows = torch.from_numpy(pu.orc.paged_rows(np.arange(n), c.table[b], c.page)).to(cuda_device)
        ramp = torch.linspace(-40, 40, n, device=cuda_device)[:, None]
        if e4m3:
            c.k[rows] = torch.full((n, 256), 8.0, device=cuda_device).to(torch.float8_e4m3fn).view(torch.uint8)
            c.k_scale[rows] = ramp / 60
        else:
            c.k[rows] = (ramp / 8).expand(n, 256).to(c.k.dtype)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


def test_value_scales_of_any_size(cuda_device):
    """e4m3 caches: value scales from 2^-60 to 2^60 in one sequence."""
    c = pu.Cache([500, 77], (8, 2, 128, 128), 64, "bf16", True, cuda_device, seed=9)
    e = torch.randint(-60, 61, c.v_scale.shape, device=cuda_device, generator=torch.Generator(cuda_device).manual_seed(1))
    c.v_scale.copy_(torch.exp2(e.float()))
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


def test_large_and_small_queries_of_e4m3_caches(cuda_device):
    c = pu.Cache([200], (4, 1, 128, 128), 64, "bf16", True, cuda_device, seed=10)
    c.q[0, 0] *= 2.0 ** 30
    c.q[0, 1] *= 2.0 ** -40
    c.q[0, 2] = 0
    c.k_scale *= 2.0 ** -30
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


def test_minus_infinite_scores(cuda_device):
    """A key whose score is -inf weighs nothing, also where all keys of a strip or a whole part are such; nothing else does so."""
    c = pu.Cache([64, 700], (2, 1, 64, 64), 16, "bf16", False, cuda_device, seed=11)
    c.q[:] = 0
    c.q[:, :, 0] = 1
    plain = c.k.clone()
    for b, n in enumerate(c.lengths):
        rows = torch.from_numpy(pu.orc.paged_rows(np.arange(n), c.table[b], c.page)).to(cuda_device)
        c.k[rows, 1:] = 0
        plain[rows, 1:] = 0
        gone = rows[: n - 3] if b else rows[::2]
        c.k[gone, 0] = -torch.inf
        plain[gone, 0] = -3e38
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    c.k = plain      # the same weights: exp of -4e36 is 0
    pu.check_attend(c, out, lse)


def test_nan_stays_with_its_head_and_sequence(cuda_device):
    c = pu.Cache([50, 60, 70], (4, 2, 64, 64), 16, "bf16", False, cuda_device, seed=12)
    row = int(pu.orc.paged_rows([31], c.table[1], 16)[0])
    c.k[row, 64 + 5] = torch.nan          # key head 1 of sequence 1: query heads 2 and 3
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    bad = torch.zeros(3, 4, dtype=torch.bool, device=cuda_device)
    bad[1, 2:] = True
    assert torch.equal(out.isnan().all(-1), bad) and torch.equal(out.isnan().any(-1), bad) and torch.equal(lse.isnan(), bad)
    pu.check_attend(c, out, lse, sequences=[0, 2])


@pytest.mark.parametrize("shape,dtype,e4m3", [((8, 2, 128, 128), "bf16", False), ((8, 2, 64, 64), "fp16", True)])
def test_pitches_and_absent_lse(cuda_device, shape, dtype, e4m3):
    """Pools, queries and outputs as parts of wider tensors, a table wider than the sequences need; nothing beside them is written."""
    c = pu.Cache(RAGGED, shape, 32, dtype, e4m3, cuda_device, seed=13, pad=48, width=100)
    B, H, d = len(RAGGED), shape[0], shape[2]
    wide_q = torch.zeros(B, H + 3, d, dtype=pu.DTYPES[dtype], device=cuda_device)
    wide_q[:, 2:2 + H] = c.q
    c.q = wide_q[:, 2:2 + H]
    wide = torch.full((B, H + 2, d), 5.0, dtype=pu.DTYPES[dtype], device=cuda_device)
    table = torch.full((B, 120), -1, dtype=torch.int32, device=cuda_device)
    table[:, :100] = c.page_table
    c.page_table = table[:, :100]
    ctx, out, lse = pu.attend(c, out=wide[:, 1:1 + H])
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
    assert bool((wide[:, 0] == 5).all()) and bool((wide[:, -1] == 5).all())
    ref = out.clone()
    out.zero_()
    ctx.paged_attn(c.q, c.k, c.v, c.page_table, c.ctx_len, out, None, k_scale=c.k_scale, v_scale=c.v_scale)
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


def test_bad_pages_and_lengths_are_reported_and_stay_with_their_sequence(cuda_device):
    c = pu.Cache([100, 200, 300, 40], (8, 2, 64, 64), 16, "bf16", False, cuda_device, seed=14)
    c.page_table[1, 3] = c.n_pages
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == -7 and ctx.status() == 0
    pu.check_attend(c, out, lse, sequences=[0, 2, 3])
    c.page_table[1, 3] = -5
    out, lse = pu.attend(c, ctx)[1:]
    assert ctx.status() == -7
    pu.check_attend(c, out, lse, sequences=[0, 2, 3])
    c.page_table.copy_(torch.from_numpy(c.table))
    c.ctx_len[3] = -1
    c.ctx_len[0] = 1 << 30
    c.ctx_len[0] = c.table.shape[1] * 16 + 1
    out, lse = pu.attend(c, ctx)[1:]
    assert ctx.status() == -7
    pu.check_attend(c, out, lse, sequences=[1, 2])
    assert bool((out[3] == 0).all()) and bool((lse[3] == -torch.inf).all())
    c.ctx_len.copy_(torch.tensor(c.lengths, dtype=torch.int32))
    out, lse = pu.attend(c, ctx)[1:]
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


def test_rows_past_32_bit_byte_offsets(cuda_device):
    """A pool of more than 4 GB whose last pages are used."""
    rows = 2_200_000 // 64 * 64
    k = torch.zeros(rows, 1024, dtype=torch.bfloat16, device=cuda_device)
    small = pu.Cache([150, 90], (16, 8, 128, 128), 64, "bf16", False, cuda_device, seed=15)
    v = torch.zeros(rows, 1024, dtype=torch.bfloat16, device=cuda_device)
    off = rows - small.k.shape[0]
    k[off:], v[off:] = small.k, small.v
    ctx = binding.Context(None, 0, 0, 2, device=cuda_device, kv=small.params())
    out, lse = torch.empty(2, 16, 128, dtype=torch.bfloat16, device=cuda_device), torch.empty(2, 16, device=cuda_device)
    table = torch.where(small.page_table >= 0, small.page_table + off // 64, small.page_table)
    ctx.paged_attn(small.q, k, v, table, small.ctx_len, out, lse)
    assert ctx.status() == 0
    pu.check_attend(small, out, lse)


def test_another_stream_and_a_captured_graph(cuda_device):
    """A context on a side stream; the call captured once and replayed for other lengths and queries."""
    st = torch.cuda.Stream(cuda_device)
    c = pu.Cache([300, 1, 3000, 0], (16, 2, 128, 128), 64, "bf16", False, cuda_device, seed=16, width=60)
    out, lse = torch.empty(4, 16, 128, dtype=torch.bfloat16, device=cuda_device), torch.empty(4, 16, device=cuda_device)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        ctx = binding.Context(None, 0, 0, 4, device=cuda_device, stream=st, kv=c.params())
        pu.attend(c, ctx, out, lse)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        pu.attend(c, ctx, out, lse)
    for lengths in ([300, 1, 3000, 0], [10, 1, 2999, 0], [0, 0, 17, 0], [299, 1, 1, 0]):
        c.lengths = lengths
        c.ctx_len.copy_(torch.tensor(lengths, dtype=torch.int32))
        c.q.mul_(0.9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.status() == 0
        pu.check_attend(c, out, lse)


def test_small_workspace_is_refused(cuda_device):
    c = pu.Cache([10], (8, 2, 64, 64), 16, "bf16", False, cuda_device, seed=17)
    small = binding.Context(None, 0, 0, 1, device=cuda_device, kv=binding.make_kv_params(1, 1, 64, 64, 16))
    large = binding.Context(None, 0, 0, 1, device=cuda_device, kv=c.params())
    large.h, small.h = small.h, large.h       # the parameters of one, the workspace of the other
    with pytest.raises(binding.LsaError) as e:
        pu.attend(c, large)
    assert e.value.code == -3


def test_no_sequences(cuda_device):
    kv = binding.make_kv_params(8, 2, 64, 64, 16)
    ctx = binding.Context(None, 0, 0, 1, device=cuda_device, kv=kv)
    e = torch.empty(0, 8, 64, dtype=torch.bfloat16, device=cuda_device)
    pool = torch.zeros(32, 128, dtype=torch.bfloat16, device=cuda_device)
    before = ctx.launch_count()
    ctx.paged_attn(e, pool, pool, torch.zeros(0, 3, dtype=torch.int32, device=cuda_device), torch.zeros(0, dtype=torch.int32, device=cuda_device), e)
    assert ctx.launch_count() == before and ctx.status() == 0


def test_many_small_weights(cuda_device):
    c = pu.many_small_weights((8, 8, 64, 64), 16, cuda_device)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse, sequences=[0, 7, 39])


@pytest.mark.parametrize("shape", [(2, 1, 128, 128), (6, 2, 64, 64), (6, 3, 64, 64), (12, 6, 128, 128), (12, 12, 64, 64), (32, 16, 128, 128)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_scales_of_e4m3_caches(cuda_device, shape, page):
    """Scales come in copies of one, two or four heads of a row, or of whole rows, out of boxes of a page."""
    c = pu.Cache([1, 15, 33, 255, 256, 257, 700], shape, page, "bf16", True, cuda_device, seed=22, poison=True)
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_bad_page_counts_as_zero_rows(cuda_device, e4m3):
    c = pu.Cache([200, 333], (4, 1, 64, 64), 16, "bf16", e4m3, cuda_device, seed=23)
    for page in (-1, c.n_pages, 2 ** 31 - 1):
        c.page_table[1, 3] = page
        ctx, out, lse = pu.attend(c)
        assert ctx.status() == -7
        zero = int(c.table[1, 3])
        keep = c.table.copy()
        rows = slice(zero * 16, zero * 16 + 16)
        old = [None if t is None else t[rows].clone() for t in (c.k, c.v)]
        c.k[rows] = 0
        c.v[rows] = 0
        pu.check_attend(c, out, lse)
        c.k[rows], c.v[rows] = old
        assert np.array_equal(keep, c.table)


def test_two_contexts_on_two_streams(cuda_device):
    """Calls that run at the same time, each with its own workspace."""
    cs = [pu.Cache([2000, 3, 700], (16, 2, 128, 128), 64, "bf16", False, cuda_device, seed=24), pu.Cache([300, 5000], (64, 1, 576, 512), 64, "bf16", False, cuda_device, seed=25)]
    streams = [torch.cuda.Stream(cuda_device) for _ in cs]
    calls = []
    torch.cuda.synchronize()
    for c, st in zip(cs, streams):
        with torch.cuda.stream(st):
            ctx = binding.Context(None, 0, 0, len(c.lengths), device=cuda_device, stream=st, kv=c.params())
            calls.append(pu.attend(c, ctx))
    torch.cuda.synchronize()
    first = [(out.clone(), lse.clone()) for _, out, lse in calls]
    for _ in range(20):
        for c, st, (ctx, out, lse) in zip(cs, streams, calls):
            with torch.cuda.stream(st):
                pu.attend(c, ctx, out, lse)
    torch.cuda.synchronize()
    for c, (ctx, out, lse), (out1, lse1) in zip(cs, calls, first):
        assert ctx.status() == 0 and torch.equal(out, out1) and torch.equal(lse, lse1)
        pu.check_attend(c, out, lse)


@pytest.mark.parametrize("shape", [(8, 1, 128, 128), (16, 1, 64, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_products_of_weights_and_scales_that_rise_and_fall(cuda_device, shape, dtype):
    """e4m3: value scales that grow and shrink by more than fp16's range along a sequence, with scores that grow against them: what comes
    to matter late must not be rounded by what mattered before."""
    c = pu.Cache([1500, 1500], shape, 64, dtype, True, cuda_device, seed=27)
    c.q[:] = 0
    c.q[..., 0] = 1
    c.k[:, 1:] = 0
    c.k[:, 0] = torch.tensor([1.0], device=cuda_device).to(torch.float8_e4m3fn).view(torch.uint8)
    for b, (score, scale) in enumerate([((0, 240), (60, -60)), ((0, 0), (-60, 14))]):   # in powers of two, first to last token
        rows = torch.from_numpy(pu.orc.paged_rows(np.arange(1500), c.table[b], 64)).to(cuda_device)
        c.k_scale[rows, 0] = torch.linspace(score[0], score[1], 1500, device=cuda_device) * (c.d ** 0.5 * 0.6931472)
        c.v_scale[rows, 0] = torch.exp2(torch.linspace(scale[0], scale[1], 1500, device=cuda_device))
    ctx, out, lse = pu.attend(c)
    assert ctx.status() == 0
    pu.check_attend(c, out, lse)
