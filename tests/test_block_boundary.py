"""Refusals of block-scaled caches, rotated appends, truncation and adjusted logits: an
error before anything is launched or changed (no GPU needed)."""
import ctypes

import pytest

from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")
FAKE = 1 << 30


def block_desc(**kw):
    d = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, max_tokens=300, block_tokens=64, fp16_window=16,
             type_k="i8", type_v="e4m3", page_tokens=0, num_pages=0)
    d.update(kw)
    return kvq.make_block_desc(**d)


def handle(**kw):
    d = block_desc(**kw)
    return kvq.kvq_block_cache_init(d, FAKE, kvq.kvq_block_cache_bytes(d))


def align(x, a=256):
    return (x + a - 1) // a * a


@pytest.mark.parametrize("batch,hkv,tokens,block,R", [(1, 8, 4096, 64, 0), (3, 2, 1000, 32, 100), (2, 1, 50, 128, 60)])
def test_bytes(batch, hkv, tokens, block, R):
    cq, W = max(0, tokens - R) // block * block, R + block
    head = 2 * align(cq * 128) + align(cq // block * 8) + 2 * align(W * 256) + 256
    d = block_desc(batch=batch, num_q_heads=4 * hkv, num_kv_heads=hkv, max_tokens=tokens, block_tokens=block, fp16_window=R)
    assert kvq.kvq_block_cache_bytes(d) == 256 + batch * hkv * head


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), kvq.ERR_ARG), (dict(num_kv_heads=0), kvq.ERR_ARG), (dict(num_q_heads=7), kvq.ERR_ARG),
    (dict(num_q_heads=6), kvq.ERR_UNSUPPORTED), (dict(head_dim=64), kvq.ERR_UNSUPPORTED), (dict(max_tokens=0), kvq.ERR_ARG),
    (dict(block_tokens=16), kvq.ERR_ARG), (dict(block_tokens=256), kvq.ERR_ARG), (dict(fp16_window=-1), kvq.ERR_ARG),
    (dict(page_tokens=32), kvq.ERR_ARG), (dict(page_tokens=96), kvq.ERR_ARG), (dict(num_pages=3), kvq.ERR_ARG),
])
def test_bad_descriptors(kw, status):
    d = block_desc(**kw)
    assert kvq.kvq_block_cache_bytes(d) == 0
    with pytest.raises(kvq.KvqError) as e:
        kvq.kvq_block_cache_init(d, FAKE, 1 << 40)
    assert e.value.status == status


def test_bad_types_and_arenas():
    with pytest.raises(ValueError):
        block_desc(type_k="int4")
    d = block_desc()
    n = kvq.kvq_block_cache_bytes(d)
    for arena, size, status in ((FAKE, n - 1, kvq.ERR_CAPACITY), (FAKE + 16, n, kvq.ERR_ARG), (None, n, kvq.ERR_ARG)):
        with pytest.raises(kvq.KvqError) as e:
            kvq.kvq_block_cache_init(d, arena, size)
        assert e.value.status == status
    d.type_v = 2
    with pytest.raises(kvq.KvqError) as e:
        kvq.kvq_block_cache_init(d, FAKE, n)
    assert e.value.status == kvq.ERR_ARG
    assert kvq.lib().kvq_block_cache_init(None, ctypes.byref(block_desc()), FAKE, n) == kvq.ERR_ARG


def rotary(**kw):
    d = dict(q=FAKE, k=FAKE, v=FAKE, q_stride=1024, k_stride=256, v_stride=256, cos_table=FAKE, sin_table=FAKE,
             positions=None, table_rows=300, type=0, rotary_dim=128, adjacent_pairs=0, pad=0)
    d.update(kw)
    return kvq.Rotary(**d)


BAD_ROTARY = [
    dict(type=2), dict(type=-1), dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=144), dict(adjacent_pairs=2),
    dict(table_rows=0), dict(table_rows=2), dict(q_stride=1023), dict(k_stride=255), dict(v_stride=0), dict(k=None), dict(v=None),
    dict(cos_table=None), dict(sin_table=None), dict(k=FAKE + 1), dict(cos_table=FAKE + 2), dict(positions=FAKE + 2),
    dict(q=None), dict(v_stride=1 << 41),
]


@pytest.mark.parametrize("bad", BAD_ROTARY)
def test_rotary_refusals_change_nothing(bad):
    h = handle()
    try:
        r = rotary(**bad)
        n = (ctypes.c_int32 * 2)(3, 1)
        assert kvq.lib().kvq_append_rotary(h, ctypes.byref(r), 3, n, FAKE, None) == kvq.ERR_ARG
        assert kvq.kvq_last_error() and kvq.kvq_seq_len(h, 0) == kvq.kvq_seq_len(h, 1) == 0
    finally:
        kvq.kvq_cache_destroy(h)


def test_rotary_counts_and_capacity():
    h = handle()
    L = kvq.lib()
    try:
        r = ctypes.byref(rotary(table_rows=1000))
        for n, n_max, status in (((4, 0), 3, kvq.ERR_ARG), ((-1, 0), 3, kvq.ERR_ARG), ((301, 0), 400, kvq.ERR_CAPACITY),
                                 ((0, 0), -1, kvq.ERR_ARG)):
            assert L.kvq_append_rotary(h, r, n_max, (ctypes.c_int32 * 2)(*n), FAKE, None) == status
        assert L.kvq_append_rotary(None, r, 1, (ctypes.c_int32 * 2)(1, 1), FAKE, None) == kvq.ERR_ARG
        assert L.kvq_append_rotary(h, None, 1, (ctypes.c_int32 * 2)(1, 1), FAKE, None) == kvq.ERR_ARG
        assert L.kvq_append_rotary(h, r, 1, None, FAKE, None) == kvq.ERR_ARG
        # nothing to append: nothing is launched, whatever the pointers
        assert L.kvq_append_rotary(h, ctypes.byref(rotary(k=None, v=None, cos_table=None)), 0, (ctypes.c_int32 * 2)(0, 0), FAKE, None) == 0
    finally:
        kvq.kvq_cache_destroy(h)


def test_truncate_refusals():
    h = handle()
    try:
        kvq.kvq_truncate(h, [0, 0])
        for lens in ([1, 0], [0, 5]):
            with pytest.raises(kvq.KvqError) as e:
                kvq.kvq_truncate(h, lens)
            assert e.value.status == kvq.ERR_ARG
        with pytest.raises(ValueError):
            kvq.kvq_truncate(h, [0, 1 << 32])
        assert kvq.lib().kvq_truncate(h, None) == kvq.lib().kvq_truncate(None, (ctypes.c_int32 * 1)(0)) == kvq.ERR_ARG
    finally:
        kvq.kvq_cache_destroy(h)


def test_calls_on_a_block_cache():
    h = handle()
    try:
        with pytest.raises(kvq.KvqError) as e:
            kvq.kvq_decode_partials(h, FAKE, FAKE, 1 << 30)
        assert e.value.status == kvq.ERR_UNSUPPORTED
        with pytest.raises(kvq.KvqError) as e:
            kvq.kvq_decode_merge(h, FAKE, FAKE)
        assert e.value.status == kvq.ERR_UNSUPPORTED
        with pytest.raises(kvq.KvqError) as e:
            kvq.kvq_chunk_attention(h, FAKE, 5, FAKE, FAKE, 1 << 30)
        assert e.value.status == kvq.ERR_ARG  # (empty sequences)
        assert kvq.kvq_workspace_bytes(h) > 0 and kvq.kvq_chunk_workspace_bytes(h, 1025) == 0
        assert kvq.kvq_window_workspace_bytes(h, 3, 10, 2) > 0 and kvq.kvq_window_workspace_bytes(h, 3, 0, 2) == 0
        with pytest.raises(kvq.KvqError):
            kvq.kvq_set_split_tokens(h, 63)
    finally:
        kvq.kvq_cache_destroy(h)


def test_rows_of_the_binding():
    h = handle()
    try:
        k = torch.zeros((2, 3, 2, 128), dtype=torch.float16)
        q, cos = torch.zeros((2, 3, 8, 128), dtype=torch.float16), torch.zeros((300, 64))
        ok = dict(q=q, K=k, V=k, cos=cos, sin=cos, n_new=[1, 1], q_out=torch.zeros_like(q))
        bad = [dict(K=k.float()), dict(V=k.bfloat16()), dict(K=k[:, :, :1]), dict(q=q[..., :64]), dict(cos=cos.double()),
               dict(sin=cos[:10]), dict(n_new=[1]), dict(n_new=[1, 1 << 40]), dict(q_out=None), dict(q_out=q.float()),
               dict(V=k.transpose(2, 3).contiguous().transpose(2, 3)), dict(positions=torch.zeros((2, 2), dtype=torch.int32)),
               dict(positions=torch.zeros((2, 3), dtype=torch.int64)), dict(K=torch.zeros((2, 9, 2, 128), dtype=torch.float16)[:, ::3][:, :3].flip(1)[:, :, :, ::2])]
        for b in bad:
            with pytest.raises((ValueError, TypeError)):
                kvq.kvq_append_rotary(h, **{**ok, **b}, batch=2, num_q_heads=8, num_kv_heads=2)
        with pytest.raises(ValueError):  # (right in form, but not on a GPU)
            kvq.kvq_append_rotary(h, **ok, batch=2, num_q_heads=8, num_kv_heads=2)
        assert kvq.kvq_seq_len(h, 0) == 0
    finally:
        kvq.kvq_cache_destroy(h)


def adjustment(**kw):
    d = dict(logits=FAKE, row_stride=1000, type=0, batch=4, vocab=1000, history=0, tokens=None, length=None, prompt=None,
             repetition=None, presence=None, frequency=None, bias_token=None, bias=None, mask=None, mask_row=None,
             mask_stride=0, biases=0, mask_rows=0)
    d.update(kw)
    return kvq.DgapAdjustment(**d)


@pytest.mark.parametrize("bad,status", [
    (dict(logits=None), kvq.ERR_ARG), (dict(type=3), kvq.ERR_ARG), (dict(batch=0), kvq.ERR_ARG), (dict(vocab=0), kvq.ERR_ARG),
    (dict(vocab=(1 << 24) + 1, row_stride=1 << 25), kvq.ERR_UNSUPPORTED), (dict(row_stride=999), kvq.ERR_ARG),
    (dict(batch=1 << 22), kvq.ERR_UNSUPPORTED), (dict(logits=FAKE + 2), kvq.ERR_ARG), (dict(history=-1), kvq.ERR_ARG),
    (dict(history=(1 << 24) + 1, tokens=FAKE), kvq.ERR_ARG), (dict(history=3), kvq.ERR_ARG), (dict(biases=-1), kvq.ERR_ARG),
    (dict(biases=65536, bias_token=FAKE, bias=FAKE), kvq.ERR_ARG), (dict(biases=2, bias=FAKE), kvq.ERR_ARG),
    (dict(mask=FAKE, mask_rows=0, mask_stride=32), kvq.ERR_ARG), (dict(mask=FAKE, mask_rows=1, mask_stride=31), kvq.ERR_ARG),
    (dict(presence=FAKE + 1), kvq.ERR_ARG),
])
def test_adjust_refusals(bad, status):
    p = adjustment(**bad)
    assert kvq.lib().dgap_adjust(ctypes.byref(p), FAKE, 1 << 25, None) == status
    assert kvq.kvq_last_error()


def test_adjust_output_refusals():
    L, p = kvq.lib(), ctypes.byref(adjustment(row_stride=1008))
    assert L.dgap_adjust(None, FAKE, 1000, None) == kvq.ERR_ARG
    for out, stride in ((None, 1000), (FAKE, 999), (FAKE + 1, 1000), (FAKE, 1000)):  # (the last: in place, another stride)
        assert L.dgap_adjust(p, out, stride, None) == kvq.ERR_ARG


def test_adjust_binding():
    z = torch.zeros((3, 70))
    i = torch.zeros((3, 4), dtype=torch.int32)
    for bad in (dict(out=z.half()), dict(out=z[:2]), dict(tokens=i.long()), dict(tokens=i[0]), dict(length=i), dict(repetition=z[0]),
                dict(bias_token=i), dict(bias=z[:, :4]), dict(bias_token=i, bias=z[:, :3].contiguous()),
                dict(mask=i[:, :2]), dict(mask=i[:2, :3].contiguous()), dict(mask=i.float())):
        with pytest.raises(ValueError):
            kvq.dgap_adjust(z, **bad)
    with pytest.raises(TypeError):
        kvq.dgap_adjust(z.double())
    with pytest.raises(ValueError):  # (right in form, but not on a GPU)
        kvq.dgap_adjust(z)
