"""Scores and distillation without a GPU: refusals on the host, workspaces, and
the tests' own plain forms against differences."""
import ctypes
import itertools

import numpy as np
import pytest

import scores_ref as R
from paper_1802_08021_amd import sparcml as S
from test_train_abi import BAD_LOGITS, BIG, FAKE, logits, ws_size

FAR = 0x100000


def test_workspace_sizes():
    for op, least in ((S.OP_SCORES, 0), (S.OP_DISTILL, 1)):
        for a in ((least, 1, 1), (256, 2**31 - 1, 1000), (20, 5, 2**31 - 1)):
            rc, n = ws_size(op, *a)
            assert rc == S.OK and n > 0
        for a in ((least - 1, 5, 5), (257, 5, 5), (8, 0, 5), (8, 5, 0), (8, 2**31, 5), (8, 5, 2**31)):
            assert ws_size(op, *a)[0] == S.EINVAL, (op, a)


def test_a_workspace_serves_smaller_calls():
    rows = sorted(set(range(1, 40)) | {127, 341, 342, 511, 1023, 1024, 1025, 4096, 2**20})
    vocabs = [1, 7, 2048, 16384, 32000, 50001, 131072, 2**20, 2**31 - 1]
    tops = [1, 2, 20, 63, 64, 255, 256]
    for op in (S.OP_SCORES, S.OP_DISTILL):
        size = {(k, r, v): ws_size(op, k, r, v)[1] for k, r, v in itertools.product(tops, rows, vocabs)}
        for k, r, v in size:
            for smaller in ((tops[max(0, tops.index(k) - 1)], r, v), (k, rows[max(0, rows.index(r) - 1)], v),
                            (k, r, vocabs[max(0, vocabs.index(v) - 1)])):
                assert size[smaller] <= size[k, r, v]


def scores(x=None, top=3, ws=FAKE, ws_bytes=BIG, **over):
    x = logits() if x is None else x
    o = S.Scores(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, top)
    for k, v in over.items():
        setattr(o, k, v)
    return S.lib().sparcml_token_scores(ctypes.byref(x), ctypes.byref(o), ws, ws_bytes, None)


def test_scores_refusals():
    for over in BAD_LOGITS:
        if over != dict(label=None):
            assert scores(logits(**over)) == S.EINVAL, over
    assert scores(logits(label=None)) == S.EINVAL  # logp without labels
    for kw in (dict(top=11), dict(top=257, x=logits(vocab=1000, ld=1000)), dict(top_id=None), dict(top_logp=None)):
        assert scores(**kw) == S.EINVAL, kw
    assert S.lib().sparcml_token_scores(ctypes.byref(logits()), None, FAKE, BIG, None) == S.EINVAL
    assert scores(ws=None) == S.EWORKSPACE
    assert scores(ws_bytes=3) == S.EWORKSPACE


def grad(x=None, d=FAR, ldd=10, top=3, **over):
    x = logits() if x is None else x
    a = S.ScoresGrad(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, top)
    for k, v in over.items():
        setattr(a, k, v)
    return S.lib().sparcml_token_scores_grad(ctypes.byref(x), ctypes.byref(a), d, ldd, None)


def test_gradient_refusals():
    for over in BAD_LOGITS:
        assert grad(logits(**over)) == S.EINVAL, over  # (label None: d_logp without labels)
    for kw in (dict(d=None), dict(ldd=9), dict(ldd=2**31), dict(d=FAKE, ldd=12), dict(d=FAKE + 4), dict(d=FAKE - 156),
               dict(norm=None), dict(entropy=None), dict(top_id=None), dict(top=0), dict(top=11),
               dict(top=257, x=logits(vocab=1000, ld=1000), ldd=1000)):
        assert grad(**kw) == S.EINVAL, kw
    assert S.lib().sparcml_token_scores_grad(ctypes.byref(logits()), None, FAR, 10, None) == S.EINVAL


def distill(x=None, d=FAR, ldd=10, div=FAKE, stats=FAKE, ws=FAKE, ws_bytes=BIG, **over):
    x = logits() if x is None else x
    a = S.DistillArgs(FAKE, FAKE, FAKE, 4, 4, S.F32, 1, 1.0, 0.0, 0.0, 1.0)
    for k, v in over.items():
        setattr(a, k, v)
    return S.lib().sparcml_distill_loss(ctypes.byref(x), ctypes.byref(a), div, stats, d, ldd, ws, ws_bytes, None)


def test_distill_refusals():
    nan, inf = float("nan"), float("inf")
    for over in BAD_LOGITS:
        assert distill(logits(**over), hard=0.5) == S.EINVAL, over  # (label None: hard without labels)
    for kw in (dict(id=None), dict(value=None), dict(count=0), dict(count=5), dict(count=257, ld=300), dict(ld=3),
               dict(ld=2**31), dict(type=3), dict(rest=2), dict(beta=-0.1), dict(beta=1.1), dict(beta=nan), dict(hard=-0.1),
               dict(hard=1.1), dict(hard=nan), dict(rest=0, beta=0.5), dict(rest=0, teacher_scale=0.0),
               dict(rest=0, teacher_scale=-1.0), dict(rest=0, teacher_scale=nan), dict(rest=0, teacher_scale=inf),
               dict(grad_scale=inf), dict(grad_scale=nan), dict(div=None), dict(stats=None), dict(ldd=9), dict(d=FAKE + 8)):
        assert distill(**kw) == S.EINVAL, kw
    assert S.lib().sparcml_distill_loss(ctypes.byref(logits()), None, FAKE, FAKE, FAR, 10, FAKE, BIG, None) == S.EINVAL
    assert distill(ws=None) == S.EWORKSPACE
    assert distill(ws_bytes=8) == S.EWORKSPACE


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    x, y, i = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: S.token_scores(x, y), lambda: S.token_scores(x, top=257), lambda: S.token_scores(x, top=-1),
                 lambda: S.token_scores_grad(x, torch.zeros(4, 2)), lambda: S.distill_loss(x, i, torch.zeros(4, 2)),
                 lambda: S.distill_loss(x, i[:, :0], torch.zeros(4, 0)), lambda: S.distill_loss(x, y, y)):
        with pytest.raises(ValueError):
            call()


def test_plain_forms_agree_with_differences():
    rng = np.random.default_rng(0)
    T, V, K = 6, 13, 4
    x = rng.standard_normal((T, V)) * 2
    x[2, 5:] = -np.inf
    label = rng.integers(0, 5, T)
    label[3] = -1
    fixed = np.where(np.isfinite(x), 1.0, 0.0)
    ids = np.stack([rng.permutation(V)[:K] for _ in range(T)])
    ids[1, 2], ids[4, 3] = -1, ids[4, 0]
    values = np.log(rng.dirichlet(np.ones(K + 1), T)[:, :K])
    w = rng.random(T)
    w[5] = 0.0
    for rest, beta, hard in ((1, 0.0, 0.0), (1, 1.0, 0.25), (1, 0.3, 0.0), (0, 0.0, 0.5)):
        ok = np.ones(T, bool)
        if beta == 0:
            ok[2] = np.isfinite(x[2, ids[2]]).all()  # (else the loss is infinite)
        f = lambda y: R.distill(y, label, ids, values, w * ok, rest, beta, hard, 1.5, 0.7)  # noqa: E731,B023
        g = f(x)["grad"]
        for _ in range(10):
            v = rng.standard_normal((T, V)) * fixed
            diff = (f(x + 1e-5 * v)["stats"][0] - f(x - 1e-5 * v)["stats"][0]) / 2e-5
            assert abs(diff - np.sum(g * v)) < 1e-7 * (1 + np.abs(g * v).sum()), (rest, beta)
    a, l, b, c = (rng.standard_normal(T) for _ in range(4))
    d = rng.standard_normal((T, K))

    def total(y):
        s = R.scores(y, label, 1.5, 0)
        lp = 1.5 * y - s["lse"][:, None]
        has = label >= 0
        on = (ids >= 0) & np.isfinite(np.take_along_axis(x, ids, 1)) & has[:, None]
        return (np.sum((a * s["logp"] + l * s["lse"] + b * s["entropy"])[has])
                + np.sum(np.where(on, d * np.where(on, np.take_along_axis(lp, ids, 1), 0), 0)))

    s = R.scores(x, label, 1.5, 0)
    g, _ = R.scores_grad(x, label, s["norm"], 1.5, a, l, s["entropy"], b, ids, d)
    for _ in range(10):
        v = rng.standard_normal((T, V)) * fixed
        diff = (total(x + 1e-5 * v) - total(x - 1e-5 * v)) / 2e-5
        assert abs(diff - np.sum(g * v)) < 1e-6 * (1 + np.abs(g * v).sum())
