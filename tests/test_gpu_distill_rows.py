"""Rows of the teacher loss that hold no finite number, on each of its paths: rows in
registers (vocabularies to 32768), one launch per step, the loss alone, the gradient
from a kept log-sum-exp.
"""
import math

import numpy as np
import pytest

from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_distill import TYPES, check_row, inputs, run  # noqa: E402

VOCABS = [5, 20000, 40001]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("v", VOCABS)
def test_teacher_logits_without_a_softmax(v, kind):
    # q is the softmax of the row's entries: NaN with a NaN or +inf among them
    n, k = 7, 5
    z, t, i = inputs(n, v, k, seed=31, kind=kind)
    t[1, 2] = math.nan
    t[2] = math.nan
    t[3, 0] = math.inf
    t[4] = -math.inf
    t[4, 3] = math.nan
    t[5, 1] = math.nan                       # not an entry: its index is none
    i[5, 1] = -1
    bad = [1, 2, 3, 4]
    for backward in (False, True):
        loss, lse, grad = run(z, t, i, 2.0, backward=backward)
        for r in range(n):
            if r in bad:
                assert math.isnan(loss[r]) and np.isfinite(lse[r]), r
                listed = [x for x, y in zip(i[r], t[r]) if y != -math.inf]
                assert np.isnan(grad[r][listed]).all() and np.isfinite(np.delete(grad[r], listed)).all(), r
            else:
                check_row(z[r], t[r], i[r], 2.0, kind, 1.0, loss[r], lse[r], torch.from_numpy(grad[r]), backward)
    assert np.isnan(run(z, t, i, 2.0, want_grad=False)[0]).nonzero()[0].tolist() == bad


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("v", VOCABS)
def test_masked_rows_without_entries(v, kind):
    # loss and gradient 0, whatever the mask has left of the logits: padding must not reach the weights
    n, k = 6, 3
    z, t, i = inputs(n, v, k, seed=32, kind=kind)
    low = torch.finfo(TYPES[kind]).min
    z[1] = -math.inf
    z[2] = low
    z[3, :] = -math.inf
    z[3, v // 2] = low
    z[4] = torch.finfo(TYPES[kind]).max
    i[1:5] = -1
    t[2] = -math.inf
    for T in (0.5, 2.0, 1e30):
        for backward in (False, True):
            scale = [1.0, 1.0, -2.0, 3.0, math.inf, 0.5]
            loss, lse, grad = run(z, t, i, T, grad_loss=scale, backward=backward)
            assert (loss[1:5] == 0).all() and (grad[1:5] == 0).all(), (T, backward)
            assert lse[1] == -math.inf
            for r in (0, 5) if T < 1e9 else ():
                check_row(z[r], t[r], i[r], T, kind, scale[r], loss[r], lse[r], torch.from_numpy(grad[r]), backward)
        loss, lse, _ = run(z, t, i, T, want_grad=False)
        assert (loss[1:5] == 0).all() and lse[1] == -math.inf


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("v", [1, 7, 8, 13, 8193, 20000, 40001])
def test_gradient_alone_in_the_logits_place(v, kind):
    n, k = 3, min(v, 20)
    z, t, i = inputs(n, v, k, seed=33, kind=kind)
    loss, lse, want = run(z, t, i, 2.0, backward=True)
    base = torch.full((n, v + 9), 3.0, dtype=TYPES[kind], device="cuda")
    for off in (0, 1, 9):
        x = base[:, off:off + v]
        x.copy_(z)
        kvq.dgap_distill_backward(x, torch.from_numpy(t).cuda(), torch.from_numpy(i).cuda(), 2.0, torch.from_numpy(lse).cuda(), x)
        torch.cuda.synchronize()
        assert (x.double().cpu().numpy() == want).all()
        assert bool((base[:, :off] == 3.0).all()) and bool((base[:, off + v:] == 3.0).all())
        base.fill_(3.0)
