"""DGAP's correction inside a generation step (test_gpu_generation.py runs the steps and
compares the other operators): the corrected candidates' logits against the 64-bit
oracle on the logits that the step got, the others bit by bit, and the token drawn from
what the correction left.  Tolerances are those of test_dgap_gpu.py: a decision counts
where the oracle's risk is more than 1e-4 from the threshold, a corrected logit is
within 1e-4.
"""
import numpy as np
import pytest

from dgap_inputs import gen_weights
from oracle import dgap as odgap
from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_generation import K, VOCAB, Head, Step  # noqa: E402
from test_gpu_sample import check as check_tokens  # noqa: E402
from test_gpu_window import Setup  # noqa: E402


def weigh(s, w):
    """The step with the weights w."""
    t = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (w.w1, w.b1, w.w2, w.c1, w.cb1, w.c2)]
    s.weights = (w, t)
    s.params = kvq.dgap_params(VOCAB, K, odgap.TAU, t[0], t[1], t[2], w.b2, t[3], t[4], t[5], w.cb2)


@pytest.mark.parametrize("bias", [20.0, 0.0, -20.0])
def test_corrected_candidates(bias):
    c = Setup((200, 77, 131), (2, 4, 1), (2, 4, 8), R=32, cap=256, seed=41)
    s = Step(c.cache, Head(c.hq * 128), 3, c.hq)
    weigh(s, gen_weights(2, det_bias=bias, scale=1.0 if bias else 3.0))
    rng = np.random.default_rng(17)
    corrected = 0
    for step in range(8):
        u = rng.random(3).astype(np.float32)
        s.q.copy_(torch.from_numpy(c.queries(1)))
        s.u.copy_(torch.from_numpy(u))
        s.run()
        torch.cuda.synchronize()
        for r in range(3):
            z, got = s.plain[r].cpu().numpy(), s.logits[r].cpu().numpy()
            ref = odgap.restore(z, K, s.weights[0], odgap.TAU)
            decided = bool((got[ref.idx] != z[ref.idx]).any())
            if abs(ref.risk - odgap.TAU) > 1e-4:
                assert decided == ref.corrected, (step, r, ref.risk)
            want = z.astype(np.float64)
            if decided:
                want[ref.idx] += odgap.corrector(odgap.candidate_features(z, K), ref.phi, s.weights[0])
            assert np.abs(got[ref.idx] - want[ref.idx]).max() <= 1e-4, (step, r)
            others = np.ones(VOCAB, dtype=bool)
            others[ref.idx] = False
            assert np.array_equal(got[others].view(np.uint32), z[others].view(np.uint32))
            corrected += decided
        check_tokens(s.logits, list(u), list(s.T.cpu().numpy()), s.k.tolist(), list(s.p.cpu().numpy()))
    assert corrected == 24 if bias > 0 else corrected == 0 if bias < 0 else True
    print(f"[generation] detector bias {bias}: {corrected} of 24 rows corrected", flush=True)
