"""Token scores where a row is sure of its token, and their gradient where its
factors leave fp32's range."""
import numpy as np
import pytest

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
