"""Forms of the losses beside the ordinary ones: rows so far apart that their
offsets pass 32 bits, in every kernel that reads or writes them; the preference
loss without a gradient; many pairs of few long rows.  Against 64 bits, with
the bounds of test_gpu_loss."""
import numpy as np
import pytest

import train_ref as R
from gpu_util import say, to_np, torch_dev
from test_gpu_loss import U, check_gradient, lp_bound, make, policy_inputs

pytestmark = pytest.mark.gpu


def check_preference(r, h, l, bounds, ref, kind, beta=0.1, smoothing=0.0):
    """r: the loss' outputs; h, l: logits and labels, before the call."""
    V, pairs = h.shape[1], len(bounds) // 2
    stats, lp, d, coef = R.preference(h, l, bounds, ref, beta, smoothing)
    has = (l >= 0) & (l < V)
    clean = np.where(has[:, None], h, 0.0)
    err = np.where(has, lp_bound(clean, l, 1.0, V), 0)
    assert np.all(np.abs(to_np(r["logp"]) - lp) <= err)
    worst = max(np.sum(err[bounds[2 * b]:bounds[2 * b + 2]]) for b in range(pairs)) * beta
    got = to_np(r["stats"])
    lim = worst + 2 * U * np.abs(stats) + 1e-7
    assert np.all(np.abs(got - stats)[[0, 2, 3]] <= lim[[0, 2, 3]]) and abs(got[1] - stats[1]) < 1e-6
    if r["dlogits"] is not None:
        rel = worst if not smoothing else worst * beta / pairs / 4 / np.maximum(np.abs(coef), 1e-30)
        check_gradient(r["dlogits"].double().cpu().numpy(), d, np.abs(coef), clean, 1.0, V, kind,
                       np.where(coef != 0, rel, 0) + 8 * U)


def check_policy(r, h, l, a, kind):
    n = {k: None if v is None else to_np(v) for k, v in a.items()}
    stats, lp, d, coef = R.policy(h, l, **n, kl=0.05)
    used = (n["weight"] != 0) & (l >= 0)
    clean = np.where(used[:, None], h, 0.0)
    err = lp_bound(clean, l, 1.0, h.shape[1])
    assert np.all(np.abs(to_np(r["logp"]) - lp)[used] <= err[used])
    size = n["weight"] * (np.abs(np.exp(lp - n["old"]) * n["adv"]) + 0.05 * (np.exp(n["ref"] - lp) + 1)) * used
    rel = np.where(coef != 0, size / np.maximum(np.abs(coef), 1e-30), 0) * (err + 16 * U)
    total = np.sum(size * (err + 16 * U)) + 4 * U * np.abs(stats).max() + 1e-7
    assert np.all(np.abs(to_np(r["stats"])[:3] - stats[:3]) <= 2 * total)
    if r["dlogits"] is not None:
        check_gradient(r["dlogits"].double().cpu().numpy(), d, np.abs(coef), clean, 1.0, h.shape[1], kind, rel)


def test_rows_far_apart():
    """Offsets of up to 5.7e9 elements, the gradient in the logits' place:
    V = 700 takes the kernels of a workgroup a row, V = 33000 those of slices;
    130 rows the policy loss' single pass, 100 its two."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    ld = 44_000_001
    room = torch.empty(130 * ld, device=dev, dtype=torch.bfloat16)
    for T, V in ((130, 700), (130, 33000), (100, 700), (100, 33000)):
        y, label, gen = make(T, V, "bfloat16", T + V)
        label[T // 3] = -1
        a = policy_inputs(y, label, gen, 1.0, True, T)
        x = room.view(130, ld)[:T, 1:V + 1]
        h, l = y.double().cpu().numpy(), label.cpu().numpy()
        bounds = [0, T // 5, T // 2, T // 2, T]
        for name in ("logprob", "policy", "preference"):
            say(f"[far] {T} {V} {name}")
            x.copy_(y)
            if name == "logprob":
                lp, _ = S.token_logprob(x, label)
                has = l >= 0
                assert np.all(np.abs(to_np(lp) - R.rows(h, l, 1.0)[0])[has] <= lp_bound(h, l, 1.0, V)[has])
            elif name == "policy":
                check_policy(S.policy_loss(x, label, **a, kl=0.05, dlogits="inplace"), h, l, a, "bfloat16")
            else:
                check_preference(S.preference_loss(x, label, bounds, ref=a["ref"], dlogits="inplace"), h, l, bounds,
                                 to_np(a["ref"]), "bfloat16")


@pytest.mark.parametrize("T,V,pairs,kind", [(64, 900, 3, "bfloat16"), (700, 300, 7, "float16"), (40, 20000, 2, "float32"),
                                            (80, 20000, 37, "float32"), (90, 33000, 40, "bfloat16"),
                                            (700, 33000, 300, "float16")])
def test_preference_forms(T, V, pairs, kind):
    """Without a gradient, and with more pairs than a launch's arguments hold
    over rows that are cut into slices (empty sequences among them)."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    x, label, gen = make(T, V, kind, T + V, pad=5)
    label[torch.rand(T, device=dev, generator=gen) < 0.3] = -1
    x[label < 0] = float("nan")
    rng = np.random.default_rng(T)
    bounds = [0] + sorted(rng.integers(0, T + 1, 2 * pairs - 1).tolist()) + [T]
    h, l = x.double().cpu().numpy(), label.cpu().numpy()
    ref = (R.rows(h, l, 1.0)[0] + rng.standard_normal(T) * 0.5).astype(np.float32)
    for smoothing in (0.0, 0.2):
        call = dict(ref=torch.from_numpy(ref).to(dev), smoothing=smoothing)
        only = S.preference_loss(x, label, bounds, dlogits=None, **call)
        full = S.preference_loss(x, label, bounds, **call)
        check_preference(only, h, l, bounds, ref, kind, smoothing=smoothing)
        check_preference(full, h, l, bounds, ref, kind, smoothing=smoothing)
        assert only["dlogits"] is None
        for k in ("stats", "logp"):
            np.testing.assert_array_equal(to_np(only[k]), to_np(full[k]), err_msg=k)
