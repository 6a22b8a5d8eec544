"""Token scores where a row is sure of its token."""
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
