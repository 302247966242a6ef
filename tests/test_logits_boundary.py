"""Host-side tests of the calls on rows of logits and of windowed attention (no GPU
needed): each refusal is made before any device memory is touched, with a message,
and the bindings refuse what they can see of the tensors themselves.
"""
import ctypes
import math

import pytest

from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")

FAKE = 1 << 30  # an aligned address that is never dereferenced on these paths
ARG, UNSUPPORTED, CAPACITY = 1, 2, 3


def refused(status):
    assert status != 0
    assert len(kvq.kvq_last_error()) > 0
    return status


def sampling(**kw):
    p = dict(logits=FAKE, row_stride=1000, type=0, batch=3, vocab=1000, temperature=None, top_k=None, top_p=None, min_p=None,
             uniform=FAKE)
    p.update(kw)
    return kvq.DgapSampling(**p)


@pytest.mark.parametrize("kw", [dict(logits=None), dict(uniform=None), dict(type=3), dict(type=-1), dict(batch=0), dict(batch=-4),
                                dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(row_stride=999), dict(logits=FAKE + 2),
                                dict(batch=1 << 22), dict(batch=1 << 11, vocab=1 << 24, row_stride=1 << 24), dict(type=1, logits=FAKE + 1)], ids=str)
def test_sample_refuses(kw):
    p = sampling(**kw)
    refused(kvq.lib().dgap_sample(ctypes.byref(p), FAKE, None, FAKE, 1 << 40, None))


def test_sample_refuses_outputs_and_workspaces():
    p, need = sampling(), kvq.dgap_sample_workspace_bytes(3, 1000)
    f = kvq.lib().dgap_sample
    refused(f(None, FAKE, None, FAKE, need, None))
    refused(f(ctypes.byref(p), None, None, FAKE, need, None))
    refused(f(ctypes.byref(p), FAKE, None, None, need, None))
    refused(f(ctypes.byref(p), FAKE, None, FAKE, need - 1, None))
    refused(f(ctypes.byref(p), FAKE, None, FAKE + 8, need, None))
    assert kvq.dgap_sample_workspace_bytes(0, 10) == 0 and kvq.dgap_sample_workspace_bytes(1, 0) == 0
    assert kvq.dgap_sample_workspace_bytes(1, (1 << 24) + 1) == 0


def distillation(**kw):
    p = dict(logits=FAKE, row_stride=1000, type=0, rows=3, vocab=1000, k=16, teacher=FAKE, index=FAKE, temperature=2.0)
    p.update(kw)
    return kvq.DgapDistillation(**p)


BAD = [dict(rows=1 << 22), dict(rows=1 << 11, vocab=1 << 24, row_stride=1 << 24), dict(logits=None), dict(teacher=None), dict(index=None), dict(type=3), dict(rows=0), dict(rows=-1), dict(vocab=0),
       dict(vocab=(1 << 24) + 1), dict(k=0), dict(k=257), dict(row_stride=999), dict(temperature=0.0), dict(temperature=-1.0),
       dict(temperature=math.inf), dict(temperature=math.nan), dict(temperature=1e-45), dict(logits=FAKE + 2)]


@pytest.mark.parametrize("kw", BAD, ids=str)
def test_distill_refuses(kw):
    p = distillation(**kw)
    refused(kvq.lib().dgap_distill(ctypes.byref(p), FAKE, None, None, 0, None, FAKE, 1 << 40, None))
    refused(kvq.lib().dgap_distill_backward(ctypes.byref(p), FAKE, None, FAKE, 1000, None))


def test_distill_refuses_outputs_and_workspaces():
    p, need = distillation(), kvq.dgap_distill_workspace_bytes(3, 1000)
    f, b = kvq.lib().dgap_distill, kvq.lib().dgap_distill_backward
    refused(f(None, FAKE, None, None, 0, None, FAKE, need, None))
    refused(f(ctypes.byref(p), None, None, None, 0, None, FAKE, need, None))
    refused(f(ctypes.byref(p), FAKE, None, FAKE, 999, None, FAKE, need, None))
    refused(f(ctypes.byref(p), FAKE, None, FAKE + 2, 1000, None, FAKE, need, None))
    refused(f(ctypes.byref(p), FAKE, None, None, 0, None, None, need, None))
    refused(f(ctypes.byref(p), FAKE, None, None, 0, None, FAKE, need - 1, None))
    refused(f(ctypes.byref(p), FAKE, None, None, 0, None, FAKE + 4, need, None))
    refused(b(None, FAKE, None, FAKE, 1000, None))
    refused(b(ctypes.byref(p), None, None, FAKE, 1000, None))
    refused(b(ctypes.byref(p), FAKE, None, None, 1000, None))
    refused(b(ctypes.byref(p), FAKE, None, FAKE, 999, None))
    assert kvq.dgap_distill_workspace_bytes(0, 10) == 0 and kvq.dgap_distill_workspace_bytes(1, (1 << 24) + 1) == 0


def test_window_refuses():
    desc = kvq.make_desc(2, 8, 2, 128, 512, 32, 32, 0, [2, 4], [2, 8])
    h = kvq.kvq_cache_init(desc, FAKE, kvq.kvq_cache_bytes(desc))
    f = kvq.lib().kvq_window_attention
    for n_q, window, sinks, q, out in ((0, 8, 0, FAKE, FAKE), (1025, 8, 0, FAKE, FAKE), (1, 0, 0, FAKE, FAKE), (1, -3, 0, FAKE, FAKE),
                                       (1, 8, -1, FAKE, FAKE), (1, 8, 0, None, FAKE), (1, 8, 0, FAKE, None),
                                       (2, 8, 0, FAKE, FAKE)):  # (more queries than an empty cache holds)
        refused(f(h, q, n_q, window, sinks, out, FAKE, 1 << 40, None))
    refused(f(None, FAKE, 1, 8, 0, FAKE, FAKE, 1 << 40, None))
    bytes_of = lambda *a: kvq.kvq_window_workspace_bytes(h, *a)  # noqa: E731
    assert bytes_of(0, 8, 0) == bytes_of(1, 0, 0) == bytes_of(1, 8, -1) == bytes_of(1025, 8, 0) == 0
    # enough for any lengths, and no more than a window of everything needs
    assert 0 < bytes_of(1, 1, 0) <= bytes_of(1, 64, 0) <= bytes_of(1, 64, 40) <= bytes_of(1, 1 << 30, 0) == bytes_of(1, 1 << 30, 1 << 30)
    kvq.kvq_cache_destroy(h)


def test_window_binding_refuses_tensors():
    c = object.__new__(kvq.KVCache)  # (the checks come before anything of a cache but its shape)
    c.batch, c.num_q_heads, c.head_dim, c.handle = 2, 8, 128, None
    q = torch.zeros((2, 1, 8, 128), dtype=torch.half)
    for bad in (q.float(), q[:1], q[:, :, :4], q[..., :64], q.transpose(2, 3).contiguous().transpose(2, 3), torch.zeros((2, 8, 128)).half()):
        with pytest.raises((ValueError, IndexError)):
            c.window(bad, 8)
    for bad in (q, q.float()[:, :, :4], q.float()[:1]):
        with pytest.raises(ValueError):
            c.window(q, 8, out=bad)


def test_bindings_refuse_tensors():
    z, one, i32 = torch.zeros((2, 50)), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for bad in (z.double(), z.int()):
        with pytest.raises(TypeError):
            kvq.dgap_sample(bad, one, i32, ws)
    for bad in (z[0], z.t(), z[:, ::2], z[None]):
        with pytest.raises(ValueError):
            kvq.dgap_sample(bad, one, i32, ws)
    for kw in (dict(temperature=one.double()), dict(top_k=one), dict(top_p=torch.zeros(3)), dict(min_p=torch.zeros(4)[::2]),
               dict(logprobs=i32)):
        with pytest.raises(ValueError):
            kvq.dgap_sample(z, one, i32, ws, **kw)
    with pytest.raises(ValueError):  # not on a GPU
        kvq.dgap_sample(z, one, i32, ws)
    t, i = torch.zeros((2, 4)), torch.zeros((2, 4), dtype=torch.int32)
    for args, kw in (((z, t.half(), i, 2.0, one, ws), {}), ((z, t, i.long(), 2.0, one, ws), {}), ((z, t, i[:1], 2.0, one, ws), {}),
                     ((z, t, i, 2.0, one.double(), ws), {}), ((z, t, i, 2.0, one, ws), dict(grad=z.half())),
                     ((z, t, i, 2.0, one, ws), dict(grad=z[:, :40])), ((z, t, i, 2.0, one, ws), dict(lse=torch.zeros(3))),
                     ((z, t, i, 2.0, one, ws), {})):
        with pytest.raises(ValueError):
            kvq.dgap_distill(*args, **kw)
    with pytest.raises(ValueError):
        kvq.dgap_distill_backward(z, t, i, 2.0, one, z.clone())
