"""An H2O cache (adore_init_cache in H2O mode) that starts from the scores of its prompt's own attention: prompt_attention, prompt_scores, and
the tensor as it comes into init_cache.  The job then follows its oracle, and the slots hold what the definition keeps."""
import numpy as np
import pytest

from gen import Workload

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(B=2, H=3, d=64, D=128, K=24, R=4, S=90, T=8, dtype="f32", dprime=16),
                                dict(B=2, H=4, d=128, D=256, K=40, R=5, S=140, T=8, dtype="bf16", dprime=32)])
def test_scores_of_a_prompt_start_the_cache_that_decodes_behind_it(kw):
    import torch
    from paper_2407_02328_amd import prompt_attention, prompt_scores
    from gen.gpu_job import to_dev
    from tests import gpu_harness as h
    from tests.test_gpu_prompt import draw, reference
    w = Workload("h2o_from_prompt", L=1, h2o=True, **kw)
    job = h.GpuJob(w)
    k, v = (to_dev(x, job.st)[0] for x in job.prompt_np)
    q = draw(torch, (w.B, w.H, w.S, w.d), job.st, 7)
    out, lse = prompt_attention(q, k, v)
    scores = prompt_scores(q, k, lse)
    for b in range(w.B):
        want = reference(torch, *(x[b].transpose(0, 1) for x in (q, k, v, q)), w.d ** -0.5)
        # (the bound of test_gpu_prompt.py: exponents are sums of d products)
        t = 2.0 ** -24 * (w.d * want["size"] + 8)
        assert bool(((scores[b].double() - want["scores"]).abs() <= (2 * t + 2.0 ** -20) * want["scores"]).all())
    job.adore.init_cache(k[None], v[None], job.hidden, job.hidden[0][:, :w.S].contiguous(), scores, w.S)
    snap = job.snapshot()
    assert np.array_equal(snap["scores"][:, :, :w.S], scores.cpu().numpy())
    job.adore.close()
    # the same job next to its oracle, from the same scores: slots after the start and at every step
    worst, job, orc, differ = h.h2o_lockstep(w, w.T, score_init=scores.cpu().numpy(), check_cache_every=4)
    first = job.adore
    job.init(scores.cpu().numpy())
    assert np.array_equal(job.snapshot()["slot_pos"], snap["slot_pos"])
    first.close()
