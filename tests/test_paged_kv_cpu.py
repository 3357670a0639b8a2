"""lsa_kv_append and lsa_paged_attn without a GPU: the oracle's definitions against plain ones, and the calls' refusals."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import lsa_oracle as orc
from paper_2608_01662_b200 import binding

MLA = dict(n_heads=64, n_kv_heads=1, d_qk=576, d_v=512, kv_page=64, latent=True)
GQA = dict(n_heads=32, n_kv_heads=8, d_qk=128, d_v=128, kv_page=16)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product_and_depends_on_distance_only(interleaved):
    rng = np.random.default_rng(0)
    n, at, d = 8, 4, 24
    freq = 10.0 ** -np.arange(n)
    x, y = rng.standard_normal((2, d))

    def turned(v, pos):
        return orc.rotate_pairs(v, np.cos(pos * freq), np.sin(pos * freq), at, interleaved)

    def complex_of(v):
        part = v[at:at + 2 * n]
        return part[0::2] + 1j * part[1::2] if interleaved else part[:n] + 1j * part[n:]

    assert np.allclose(complex_of(turned(x, 5)), complex_of(x) * np.exp(1j * 5 * freq), atol=1e-14)
    keep = [i for i in range(d) if not at <= i < at + 2 * n]
    assert np.array_equal(turned(x, 5)[keep], x[keep])
    assert abs(turned(x, 17) @ turned(y, 9) - turned(x, 108) @ turned(y, 100)) < 1e-12


def test_seen_tokens_by_definition():
    for n in (0, 1, 2, 5, 9, 30):
        for sink in (0, 1, 4):
            for window in (0, 1, 3, 8, 40):
                want = [s for s in range(n) if window == 0 or s >= n - window or s < sink]
                assert list(orc.seen_tokens(n, sink, window)) == want


@pytest.mark.parametrize("H,G,sink,window", [(6, 2, 0, 0), (4, 4, 0, 0), (3, 1, 2, 5), (8, 2, 0, 7)])
def test_paged_attend_equals_the_library_on_gathered_heads(H, G, sink, window):
    rng = np.random.default_rng(1)
    d, dv, page, n = 16, 8, 4, 23
    table = rng.permutation(9).astype(np.int32)[:6]
    k, v = rng.standard_normal((36, G, d)), rng.standard_normal((36, G, dv))
    q = rng.standard_normal((H, d))
    out, lse = orc.paged_attend(q, k, v, table, n, page, G, sink=sink, window=window, sm_scale=0.3)
    rows = [int(table[s // page]) * page + s % page for s in range(n)]
    mask = torch.tensor([window == 0 or s >= n - window or s < sink for s in range(n)])
    kk = torch.from_numpy(k[rows]).transpose(0, 1).repeat_interleave(H // G, 0)
    vv = torch.from_numpy(v[rows]).transpose(0, 1).repeat_interleave(H // G, 0)
    ref = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q)[:, None], kk, vv, attn_mask=mask[None, None], scale=0.3)[:, 0]
    assert np.abs(out - ref.numpy()).max() < 1e-12
    z = (0.3 * torch.from_numpy(q)[:, None] @ kk.transpose(1, 2))[:, 0].masked_fill(~mask, -math.inf)
    assert np.abs(lse - torch.logsumexp(z, 1).numpy()).max() < 1e-12


def test_paged_attend_of_nothing():
    out, lse = orc.paged_attend(np.ones((2, 4)), np.ones((4, 1, 4)), np.ones((4, 1, 4)), np.zeros(1, np.int32), 0, 4, 1, sm_scale=1.0)
    assert np.all(out == 0) and np.all(np.isneginf(lse))


def test_parameters_struct():
    assert ctypes.sizeof(binding.LsaKvParams) == 60
    kv = binding.make_kv_params(**MLA)
    assert kv.struct_size == 60 and abs(kv.sm_scale * 24 - 1) <= 2.0 ** -24   # one rounding to fp32
    assert binding.kv_workspace_bytes(kv) >= 256 + 2 * 148 * 64 * 513 * 4
    assert binding.kv_workspace_bytes(binding.make_kv_params(**GQA)) % 256 == 0


@pytest.mark.parametrize("change,code", [
    (dict(n_heads=65), -2), (dict(n_heads=0), -1), (dict(d_qk=512), -2), (dict(d_v=576), -2), (dict(e4m3=True), -2),
    (dict(kv_page=32), -2), (dict(kv_page=512), -2), (dict(n_kv_heads=2), -2), (dict(d_rope=8), -2), (dict(d_rope=64, rope_at=520), -2),
    (dict(d_rope=64, rope_at=528), -2), (dict(d_rope=-16), -1), (dict(sm_scale=0.0), -1), (dict(sm_scale=-1.0), -1), (dict(sm_scale=math.nan), -1),
    (dict(sm_scale=math.inf), -1), (dict(sm_scale=2.5e38), -1), (dict(sink=-1), -1), (dict(window=-5), -1)])
def test_latent_parameters_refused(change, code):
    with pytest.raises(binding.LsaError) as e:
        binding.kv_workspace_bytes(binding.make_kv_params(**{**MLA, **change}))
    assert e.value.code == code


@pytest.mark.parametrize("change,code", [
    (dict(n_kv_heads=3), -1), (dict(n_kv_heads=1), -2), (dict(n_heads=256), -2), (dict(d_qk=96, d_v=96), -2), (dict(d_v=64), -2),
    (dict(kv_page=8), -2), (dict(kv_page=24), -2), (dict(kv_page=512), -2), (dict(d_rope=144), -2), (dict(d_rope=64, rope_at=80), -2)])
def test_grouped_parameters_refused(change, code):
    with pytest.raises(binding.LsaError) as e:
        binding.kv_workspace_bytes(binding.make_kv_params(**{**GQA, **change}))
    assert e.value.code == code


def test_bad_struct_size_and_flags():
    for field, value in (("struct_size", 56), ("dtype", 2), ("cache_e4m3", 2), ("latent", -1), ("rope_interleaved", 3)):
        kv = binding.make_kv_params(**GQA)
        setattr(kv, field, value)
        with pytest.raises(binding.LsaError) as e:
            binding.kv_workspace_bytes(kv)
        assert e.value.code == -1
    assert binding.lib().lsa_kv_workspace_bytes(ctypes.byref(binding.make_kv_params(**GQA)), None) == -1


# Calls whose arguments are judged before anything needs a device: addresses that are never followed, no context.
A = 1 << 20


def _attn(kv, **kw):
    v = 0 if kv.latent else A
    a = dict(q=A, ld_q=kv.n_heads * kv.d_qk, k=A, ld_k=kv.n_kv_heads * kv.d_qk, v=v, ld_v=kv.n_kv_heads * kv.d_v, ks=0, vs=0, n_pages=10, pt=A,
             stride=5, ctx=A, batch=2, out=A, ld_out=kv.n_heads * kv.d_v, lse=0)
    a.update(kw)
    return binding.lib().lsa_paged_attn(None, ctypes.byref(kv), *a.values())


def _append(kv, **kw):
    v = 0 if kv.latent else A
    a = dict(kn=A, ld_kn=kv.n_kv_heads * kv.d_qk, vn=v, ld_vn=kv.n_kv_heads * kv.d_v, q=A, ld_q=kv.n_heads * kv.d_qk, qo=2 * A,
             ld_qo=kv.n_heads * kv.d_qk, n_tok=2, start=0, cs=A if kv.d_rope else 0, n_pos=100, k=A, ld_k=kv.n_kv_heads * kv.d_qk, v=v,
             ld_v=kv.n_kv_heads * kv.d_v, ks=0, vs=0, n_pages=10, pt=A, stride=5, ctx=A, batch=2, ctx_out=0)
    a.update(kw)
    return binding.lib().lsa_kv_append(None, ctypes.byref(kv), *a.values())


@pytest.mark.parametrize("which", [MLA, GQA])
@pytest.mark.parametrize("change,code", [
    (dict(), -1),                                     # everything in order but the context
    (dict(k=A + 8), -2), (dict(q=A + 2), -2), (dict(out=A + 4), -2), (dict(ld_q=100), -2), (dict(ld_out=8), -2), (dict(ld_k=64), -2),
    (dict(n_pages=1 << 31), -2), (dict(stride=1 << 31), -2), (dict(stride=0), -1), (dict(n_pages=-1), -1), (dict(batch=-1), -1),
    (dict(k=0), -1), (dict(pt=0), -1), (dict(ctx=0), -1), (dict(q=0), -1), (dict(out=0), -1), (dict(ks=A, vs=A), -1)])
def test_attention_arguments_refused(which, change, code):
    assert _attn(binding.make_kv_params(**which), **change) == code


@pytest.mark.parametrize("which", [MLA, GQA])
@pytest.mark.parametrize("change,code", [
    (dict(), -1), (dict(kn=A + 8), -2), (dict(ld_kn=40), -2), (dict(q=A + 4), -2), (dict(qo=A + 4), -2), (dict(qo=0), -1), (dict(q=0), -1),
    (dict(cs=0), -1), (dict(cs=A + 4), -2), (dict(n_tok=3), -1), (dict(n_tok=-1, start=A), -1), (dict(n_pos=-1), -1), (dict(kn=0), -1),
    (dict(ld_k=24), -2), (dict(qo=A, ld_qo=8192 * 8), -1), (dict(n_pages=1 << 31), -2)])
def test_append_arguments_refused(which, change, code):
    assert _append(binding.make_kv_params(**which, d_rope=64), **change) == code


def test_kinds_of_cache_and_their_pointers():
    mla, gqa, e4m3 = binding.make_kv_params(**MLA), binding.make_kv_params(**GQA), binding.make_kv_params(**GQA, e4m3=True)
    assert _attn(mla, v=A) == -1 and _attn(gqa, v=0) == -1             # values of a latent cache are its keys
    assert _attn(e4m3) == -1 and _attn(e4m3, ks=A) == -1               # codes come with both scales
    assert _attn(e4m3, ks=A, vs=A, ld_k=1024 + 8) == -2                # 16 codes are 16 bytes
    assert _attn(e4m3, ks=A, vs=A, v=A + 8) == -2
    for scales in (dict(ks=A + 4, vs=A), dict(ks=A, vs=A + 8)):        # those of four heads are fetched at once
        assert _attn(e4m3, **scales) == -2 and _append(e4m3, **scales) == -2
    assert _append(mla, vn=A) == -1 and _append(gqa, vn=0) == -1 and _append(gqa, cs=A) == -1
    assert _append(gqa, ld_vn=1000) == -2 and _append(gqa, v=A + 8) == -2 and _append(gqa, vn=A + 8) == -2


def test_binding_refuses_tensors_of_another_form():
    """The binding's own checks, which need no library call."""
    x = torch.zeros(6, 8, 128, dtype=torch.bfloat16)
    assert binding._kv_rows(x, 8, 128, torch.bfloat16, "x", 6)[1] == 1024
    assert binding._kv_rows(x.view(6, 1024), 8, 128, torch.bfloat16, "x", 6)[1] == 1024
    wide = torch.zeros(6, 20, 128, dtype=torch.bfloat16)
    assert binding._kv_rows(wide[:, 4:12], 8, 128, torch.bfloat16, "x", 6)[1] == 2560
    for bad in (x.float(), x[:5], x[:, :4], x[:, ::2], x[..., ::2], x.transpose(0, 1), x.transpose(0, 1).contiguous(), x.transpose(1, 2).contiguous(), x.flatten(), x.view(3, 2, 8, 128)):
        with pytest.raises(binding.LsaError) as e:
            binding._kv_rows(bad, 8, 128, torch.bfloat16, "x", 6)
        assert e.value.code == -1
    with pytest.raises(binding.LsaError):
        binding._kv_flat(torch.zeros(4, dtype=torch.int64), torch.int32, 4, "n")
    with pytest.raises(binding.LsaError):
        binding._kv_flat(torch.zeros(4, dtype=torch.int32), torch.int32, 5, "n")
    for call in (lambda: binding._kv_rows(x, 8, 128, torch.bfloat16, "x", 6, 0), lambda: binding._kv_flat(torch.zeros(4), torch.float32, 4, "x", 0),
                 lambda: binding._kv_table(torch.zeros(2, 3, dtype=torch.int32), "x", 0)):
        with pytest.raises(binding.LsaError) as e:      # host memory where the device's is wanted
            call()
        assert e.value.code == -1


def test_binding_looks_at_page_tables():
    """The kernels may follow a row of the table up to its pitch."""
    big = torch.zeros(4, 10, dtype=torch.int32)
    assert binding._kv_table(big, "t")[:2] == (4, 10)
    assert binding._kv_table(big[:, :6], "t")[:2] == (4, 10)        # the first columns: every row's pitch is there
    assert binding._kv_table(big[:3, 4:8], "t")[:2] == (3, 10)      # (another row follows)
    assert binding._kv_table(big[1:2, 4:8], "t")[:2] == (1, 4)
    assert binding._kv_table(big[:0], "t")[0] == 0
    for bad in (big[:, 4:], big.t(), big[:, ::2], big[:1, ::2], big[0], big.long(), big[:1].expand(4, 10)):
        with pytest.raises(binding.LsaError) as e:
            binding._kv_table(bad, "t")
        assert e.value.code == -1


@pytest.mark.parametrize("which,u,t", [(MLA, 1, 64), (GQA, 8, 16), (dict(GQA, n_heads=128, n_kv_heads=128), 8, 16), (dict(GQA, n_heads=4096, n_kv_heads=4096), 8, 16),
                                       (dict(GQA, n_heads=6, n_kv_heads=6), 2, 64), (dict(GQA, n_heads=3, n_kv_heads=3), 1, 128)])
@pytest.mark.parametrize("pages", [1, 100, 65536, (1 << 31) // 256 - 8])
def test_tiles_are_numbered_in_32_bits(which, u, t, pages):
    """Both sides of the most sequences that a call takes, by the widths of their tables (no context: what is accepted ends with -1)."""
    kv = binding.make_kv_params(**which)
    kv.kv_page = 256
    most = (2 ** 31 - 161) // ((pages * 256 // t + 2) * (kv.n_kv_heads // u))
    assert _attn(kv, stride=pages, batch=min(most, 2 ** 31 - 1)) == -1
    if most < 2 ** 31 - 1:
        assert _attn(kv, stride=pages, batch=most + 1) == -2 and _attn(kv, stride=pages, batch=2 ** 31 - 1) == -2


def test_sparse_calls_of_a_context_without_their_parameters_are_refused():
    ctx = binding.Context.__new__(binding.Context)
    ctx.h, ctx.params, ctx.kv = None, None, binding.make_kv_params(**MLA)
    t = torch.zeros(4, 4)
    calls = [lambda: ctx.block_means(t, t, 4, t), lambda: ctx.index(t, t, t, t, t, 0, 4, 4, t, t), lambda: ctx.select(t, t, 0, 4, True, t, t),
             lambda: ctx.convert(t, t, 0, 4, t, t), lambda: ctx.sparse_attn(t, t, t, t, t, 0, 4, 4, t), lambda: ctx.append(t, t, t, t, t, t),
             lambda: ctx.merge([t], [t], 4, t), lambda: ctx.layer_group(t, t, t, t, t, 0, 4, 4, [t], [t], [t], [t], [t], t, t),
             lambda: ctx.layer_group_host(t, t, t, t, t, 0, 4, 4, [t], [t], [t], [t], 4, [t])]
    for call in calls:
        with pytest.raises(binding.LsaError) as e:
            call()
        assert e.value.code == -1
    with pytest.raises(binding.LsaError) as e:
        binding.Context(None, 0, 0)
    assert e.value.code == -1


def test_a_device_without_a_number_is_the_current_one(monkeypatch):
    """The context, its workspace and the tensors that its calls take are on one device, also where that is not the first."""
    from types import SimpleNamespace

    made, real = [], binding.lib()
    empty = torch.empty
    fake = SimpleNamespace(lsa_kv_workspace_bytes=real.lsa_kv_workspace_bytes, lsa_kv_append=None, lsa_paged_attn=None, lsa_destroy=lambda h: 0,
                           lsa_create=lambda h, device, *rest: made.append(device) or 0)
    monkeypatch.setattr(binding, "lib", lambda: fake)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: SimpleNamespace(cuda_stream=0))
    monkeypatch.setattr(torch, "empty", lambda n, dtype, device: made.append(torch.device(device)) or empty(8, dtype=dtype))
    for device, index in (("cuda", 3), (torch.device("cuda"), 3), ("cuda:1", 1), (None, 0)):
        made.clear()
        ctx = binding.Context(None, 0, 0, device=device, kv=binding.make_kv_params(**GQA))
        assert made == [torch.device("cuda", index), index] and ctx._kv_dev == index
