"""Token scores where a row is sure of its token, and their gradient where its
factors leave fp32's range; the largest scales that a call allows."""
import numpy as np
import pytest

import scores_ref as R
from gpu_util import say, to_np, torch_dev
from test_gpu_scores import KINDS, check_scores, make, wide

pytestmark = pytest.mark.gpu
INF = np.inf


@pytest.mark.parametrize("T,V", [(4001, 1), (4001, 40), (1501, 3001), (40, 70001), (3, 300001)])
@pytest.mark.parametrize("kind", KINDS)
def test_sure_rows_stay_in_range(T, V, kind):
    """No entropy below 0, no log probability above."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    at = torch.arange(T, device=dev) * 7919 % V
    high = torch.linspace(-30, 30, T, device=dev)[:, None]
    hot = torch.zeros(T, V, device=dev, dtype=torch.bool).scatter_(1, at[:, None], True)
    rest = make(T, V, "float32", V)[0]
    for name, other in (("one token", torch.full_like(rest, -INF)), ("lowest", torch.full_like(rest, torch.finfo(getattr(torch, kind)).min)),
                        ("far", high - 200 + rest), ("near", high - 17 + 0.3 * rest)):
        for scale in (1.0, 0.7):
            say(f"[sure] {T} {V} {kind} {name} {scale}")
            x = torch.where(hot, high, other).to(getattr(torch, kind))
            n = min(V, 3)
            got = S.token_scores(x, at.int(), n, scale)
            torch.cuda.synchronize()
            assert bool((got["entropy"] >= 0).all()), float(got["entropy"].min())
            assert bool((got["logp"] <= 0).all()), float(got["logp"].max())
            assert bool((got["top_logp"] <= 0).all()), float(got["top_logp"].max())
            assert bool((got["norm"][:, 1] >= 0).all())
            if T * V < 1 << 22:
                check_scores(got, wide(x), to_np(at.int()), scale, n, name)


@pytest.mark.parametrize("T,V", [(5, 40), (300, 700), (5, 40000), (1100, 3000)])
@pytest.mark.parametrize("kind", KINDS)
def test_factors_beyond_fp32_leave_no_nan(T, V, kind):
    """A token of -Inf has no gradient, however large the row's derivatives."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for low in (-INF, torch.finfo(getattr(torch, kind)).min):
        x, label, _ = make(T, V, kind, 3)
        x[:, V // 2:] = low
        x[:, 0] = 1.0
        label.fill_(0)
        s = S.token_scores(x, label, 3, 2.0)
        big = torch.full((T,), 3e38, device=dev)
        top = dict(top_id=s["top_id"], d_top=torch.full((T, 3), -2e38, device=dev))
        none = torch.zeros(T, device=dev)
        for more in (dict(d_logp=big), dict(d_lse=big), dict(d_lse=big, **top), dict(d_lse=-big, entropy=s["entropy"], d_entropy=none),
                     dict(entropy=s["entropy"], d_entropy=big), dict(entropy=s["entropy"], d_entropy=-big, d_lse=-big, **top)):
            for where in ("new", "inplace"):
                say(f"[beyond] {T} {V} {kind} {low} {list(more)} {where}")
                d = S.token_scores_grad(x.clone(), s["norm"], labels=label, scale=2.0, dlogits=where, **more)
                torch.cuda.synchronize()
                assert not bool(torch.isnan(d).any()), torch.isnan(d).sum()
                assert not bool(d[:, V // 2:].any())
                assert bool(d[:, 0].any())


@pytest.mark.parametrize("T,V", [(5, 40), (300, 700), (5, 40000), (1100, 3000)])
@pytest.mark.parametrize("kind", KINDS)
def test_the_largest_scales(T, V, kind):
    """Any finite scale: a row is sure of its largest logits."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    x, label, _ = make(T, V, kind, 4)
    x.clamp_(max=8.0)
    x[:, 3] = x[:, V - 2] = 11.0
    label.fill_(3)
    for scale in (2e38, 3.4e38):
        say(f"[scale] {T} {V} {kind} {scale}")
        s = S.token_scores(x, label, 3, scale)
        two = float(np.log(2.0))
        for got, want in ((s["entropy"], two), (s["logp"], -two), (s["norm"][:, 1], two), (s["top_logp"][:, :2], -two)):
            assert float((got - want).abs().max()) <= R.z_bound(V), (scale, want)
        assert bool((s["top_id"][:, 0] == 3).all()) and bool((s["top_id"][:, 1] == V - 2).all())
        logp, _ = S.token_logprob(x, label, scale)
        assert float((logp + two).abs().max()) <= R.z_bound(V)
        one = torch.full((T,), 1e-37, device=dev)
        d = S.token_scores_grad(x, s["norm"], labels=label, d_logp=one, scale=scale)
        want = torch.zeros(T, V, device=dev, dtype=torch.float64)
        want[:, 3], want[:, V - 2] = scale * 1e-37 / 2, -scale * 1e-37 / 2
        lim = want.abs() * (4 * R.z_bound(V) + R.STEP[kind]) + R.LEAST[kind]
        assert bool(((d.double() - want).abs() <= lim).all())
        ids = torch.tensor([[3, V - 2]] * T, dtype=torch.int32, device=dev)
        values = torch.log(torch.tensor([[0.75, 0.25]] * T, device=dev))
        for where in ("new", "inplace"):
            r = S.distill_loss(x.clone(), ids, values, rest=False, scale=scale, grad_scale=1e-37, dlogits=where)
            want[:, 3], want[:, V - 2] = -0.25 * scale * 1e-37, 0.25 * scale * 1e-37
            assert bool(((r["dlogits"].double() - want).abs() <= 4 * lim).all())
