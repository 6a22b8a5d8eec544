"""Distillation: what a teacher's values may hold, and a student that agrees
with its teacher."""
import numpy as np
import pytest

from gpu_util import say, torch_dev
from test_gpu_distill import MODES, teacher
from test_gpu_scores import KINDS, make

pytestmark = pytest.mark.gpu
INF = np.inf


@pytest.mark.parametrize("T,V", [(9, 700), (9, 40000), (300, 700), (150, 140000)])
def test_nan_among_the_values_is_seen(T, V):
    """Also where the student gives their tokens nothing, and where nothing but
    the given tokens counts."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    nan, K = float("nan"), 9
    for rest, beta, hard in MODES + [(True, 0.0, 1.0), (True, 1.0, 1.0), (False, 0.0, 1.0)]:
        say(f"[nan values] {T} {V} {rest} {beta} {hard}")
        x, label, _ = make(T, V, "float32", 11)
        ids, values = teacher(x, K, 3, rest, 1.0)
        lab = label if hard else None
        args = dict(labels=lab, rest=rest, beta=beta, hard=hard)
        good = S.distill_loss(x, ids, values, **args)
        on = torch.zeros(T, V, device=dev, dtype=torch.bool).scatter_(1, ids.long(), True)
        lost = ids[:, 2].long()
        x[0, lost[0]] = -INF                                 # a token that cannot come
        x[1, lost[1]] = -300.0                               # one of a probability below fp32's
        x[2, ~on[2]], x[2, lost[2]] = -INF, -INF             # nothing beside the list
        x[3, on[3]], values[3] = -INF, nan                   # nothing on it
        values[:3, 2] = nan
        for where in ("new", None, "inplace"):
            r = S.distill_loss(x.clone(), ids, values, dlogits=where, **args)
            torch.cuda.synchronize()
            assert bool(torch.isnan(r["div"][:4]).all()), r["div"][:4]
            assert bool(torch.isnan(r["stats"][:2]).all()), r["stats"]
            assert torch.equal(r["div"][4:], good["div"][4:])
            if where:
                bad = torch.isnan(r["dlogits"])
                assert bool(bad[[0, 1, 3]].all()), bad.sum(1)[:4]
                assert bool(bad[2, on[2]].all())
                assert torch.equal(r["dlogits"][4:], good["dlogits"][4:])


@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("kind", KINDS)
def test_a_student_that_agrees_has_no_divergence(T, kind):
    """The list is all there is, and the student's logits are its values: every
    difference of logarithms is 0 but for fp64's rounding, 2^-52 of at most 60
    for each of three sums over at most 256 tokens."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for V, K in ((300, 2), (5000, 64), (40001, 256)):
        say(f"[agree] {T} {V} {K} {kind}")
        x, _, gen = make(T, V, kind, K)
        ids = torch.rand(T, V, device=dev, generator=gen).topk(K, 1)[1]
        values = x.gather(1, ids).contiguous()
        x.fill_(-INF)
        x.scatter_(1, ids, values)
        r = S.distill_loss(x, ids.int(), values, rest=False)
        assert float(r["div"].abs().max()) <= 3 * 256 * 60 * 2.0**-52, r["div"]
        assert bool((r["div"] == r["div"]).all())
