"""What the paged-cache entry points refuse on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

import paper_2512_14481_b200 as P

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BF16 = 1


@pytest.fixture(scope="module")
def addr():
    buf = (ctypes.c_char * 512)()
    yield (ctypes.addressof(buf) + 63) & ~63          # never dereferenced: every call must fail, or have nothing to do


def cache(a, **kw):
    d = dict(k=a, v=a, k_scale=None, v_scale=None, page_stride=16 * 4 * 64, token_stride=4 * 64, head_stride=64, num_pages=8,
             page_size=16, num_kv_heads=4, head_dim=64, kind=P.SASQ_KV_16BIT)
    d.update(kw)
    return P.KVCacheStruct(**d)


def batch(a, **kw):
    d = dict(page_table=a, seq_lens=a, q_starts=a, page_table_stride=8, batch=2, max_pages=8, total_q=4, max_q_len=2,
             max_seq_len=100, reserved=0)
    d.update(kw)
    return P.KVBatchStruct(**d)


def append(c, b, a, **kw):
    d = dict(q=a, k=a, v=a, q_out=a, qs=512, ks=256, vs=256, qos=512, heads=8, cs=a, positions=100, rot=64, inter=0, dt=BF16)
    d.update(kw)
    return P.load_library().sasq_rope_kv_append(
        ctypes.byref(c), ctypes.byref(b), d["q"], d["k"], d["v"], d["q_out"], d["qs"], d["ks"], d["vs"], d["qos"], d["heads"],
        d["cs"], d["positions"], d["rot"], d["inter"], d["dt"], None)


def attend(c, b, a, **kw):
    d = dict(q=a, out=a + 128, lse=None, qs=512, os=512, heads=8, scale=0.1, causal=1, dt=BF16, ws=a, nbytes=1 << 40)
    d.update(kw)
    return P.load_library().sasq_paged_attention(
        ctypes.byref(c), ctypes.byref(b), d["q"], d["out"], d["lse"], d["qs"], d["os"], d["heads"], d["scale"], d["causal"],
        d["dt"], d["ws"], d["nbytes"], None)


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("change,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(num_kv_heads=0), INVALID), (dict(head_dim=0), INVALID),
    (dict(num_pages=-1), INVALID), (dict(kind=2), INVALID), (dict(token_stride=4 * 64 + 4), INVALID),
    (dict(head_stride=-64), INVALID), (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED),
    (dict(page_size=512), UNSUPPORTED), (dict(num_pages=1 << 33), UNSUPPORTED)])
def test_caches(addr, call, change, status):
    assert call(cache(addr, **change), batch(addr), addr) == status


@pytest.mark.parametrize("call", [append, attend])
def test_factors_go_with_int8(addr, call):
    assert call(cache(addr, k_scale=addr, v_scale=addr), batch(addr), addr) == INVALID
    assert call(cache(addr, kind=P.SASQ_KV_INT8, k_scale=addr), batch(addr), addr) == INVALID
    assert call(cache(addr, kind=P.SASQ_KV_INT8, head_stride=64 + 8, k_scale=addr, v_scale=addr), batch(addr), addr) == INVALID
    assert call(cache(addr + 2), batch(addr), addr) in (OK, INVALID)
    assert call(cache(addr, k=addr + 2), batch(addr), addr) == INVALID


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("change,status", [
    (dict(page_table=None), INVALID), (dict(seq_lens=None), INVALID), (dict(q_starts=None), INVALID), (dict(batch=-1), INVALID),
    (dict(total_q=-1), INVALID), (dict(max_pages=9), INVALID), (dict(reserved=1), INVALID), (dict(max_q_len=-1), INVALID),
    (dict(max_seq_len=-2), INVALID), (dict(max_pages=1 << 28, page_table_stride=1 << 28), UNSUPPORTED), (dict(total_q=0), OK),
    (dict(batch=0), OK)])
def test_batches(addr, call, change, status):
    assert call(cache(addr), batch(addr, **change), addr) == status


def test_null_structs(addr):
    L = P.load_library()
    c, b = cache(addr), batch(addr)
    assert L.sasq_paged_attention(None, ctypes.byref(b), addr, addr, None, 512, 512, 8, 0.1, 1, BF16, addr, 1 << 30, None) == INVALID
    assert L.sasq_paged_attention(ctypes.byref(c), None, addr, addr, None, 512, 512, 8, 0.1, 1, BF16, addr, 1 << 30, None) == INVALID
    assert L.sasq_paged_attention_workspace(None, ctypes.byref(b), 8) == 0
    assert L.sasq_paged_attention_workspace(ctypes.byref(c), ctypes.byref(b), 7) == 0
    assert L.sasq_paged_attention_workspace(ctypes.byref(c), ctypes.byref(b), 8) > 0


@pytest.mark.parametrize("change,status", [
    (dict(dt=2), INVALID), (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(cs=None), INVALID), (dict(cs=1), INVALID), (dict(heads=-1), INVALID), (dict(heads=0), INVALID), (dict(qs=511), INVALID),
    (dict(qs=504), INVALID), (dict(ks=248), INVALID), (dict(vs=260), INVALID), (dict(qos=64), INVALID), (dict(rot=-16), INVALID),
    (dict(positions=-1), INVALID), (dict(rot=24), UNSUPPORTED), (dict(rot=80), UNSUPPORTED)])
def test_append_arguments(addr, change, status):
    assert append(cache(addr), batch(addr), addr, **change) == status


@pytest.mark.parametrize("dim", [8, 72, 272])
def test_append_head_dims(addr, dim):
    c = cache(addr, head_dim=dim, head_stride=dim, token_stride=4 * dim, page_stride=64 * dim)
    assert append(c, batch(addr), addr, qs=8 * dim, ks=4 * dim, vs=4 * dim, qos=8 * dim, rot=0) == UNSUPPORTED


@pytest.mark.parametrize("change,status", [
    (dict(dt=7), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(heads=0), INVALID), (dict(heads=6), INVALID),
    (dict(qs=504), INVALID), (dict(os=516), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(ws=None), WORKSPACE), (dict(nbytes=64), WORKSPACE)])
def test_attention_arguments(addr, change, status):
    assert attend(cache(addr), batch(addr), addr, **change) == status


def test_aliased_and_misaligned_attention(addr):
    assert attend(cache(addr), batch(addr), addr, out=addr) == INVALID
    assert attend(cache(addr), batch(addr), addr, out=addr + 8) == INVALID
    assert attend(cache(addr), batch(addr), addr, ws=addr + 8) == WORKSPACE
    for dim in (16, 80, 96, 256):
        c = cache(addr, head_dim=dim, head_stride=dim, token_stride=4 * dim, page_stride=64 * dim)
        assert attend(c, batch(addr), addr, qs=8 * dim, os=8 * dim) == UNSUPPORTED


def test_binding_refuses_cpu_tensors():
    import torch
    x = torch.zeros((2, 16, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        P.KVCache(x, x)
    i = torch.zeros((1, 1), dtype=torch.int32)
    with pytest.raises(TypeError):
        P.PagedBatch(i, i[0], i[0], 1)
