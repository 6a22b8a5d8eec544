"""Distillation from a teacher's lists against 64 bits (scores_ref: formulas
and how far fp32 sums may put the kernels off), and against differences."""
import numpy as np
import pytest

import scores_ref as R
from gpu_util import say, to_np, torch_dev
from test_gpu_scores import KINDS, make, wide

pytestmark = pytest.mark.gpu
U, INF = R.U, np.inf


def teacher(x, K, seed, rest, scale, ragged=False, kind="float32"):
    """Lists of a teacher that mostly agrees."""
    torch, dev = torch_dev()
    gen = torch.Generator(device=dev).manual_seed(seed)
    y = torch.nan_to_num(x.float(), nan=0.0, neginf=-30.0) * (0.8 * scale)
    y = y + 0.7 * torch.randn(x.shape, device=dev, generator=gen)
    v, ids = (torch.log_softmax(y, 1) if rest else y).topk(K, 1)
    ids = ids.int()
    if ragged:
        length = torch.randint(0, K + 1, (x.shape[0], 1), device=dev, generator=gen)
        ids.masked_fill_(torch.arange(K, device=dev) >= length, -1)
    return ids.contiguous(), v.to(getattr(torch, kind)).contiguous()


def check(r, x, label, ids, values, weight, kind, **args):
    n = lambda t: None if t is None else to_np(t)  # noqa: E731
    want = R.distill(np.nan_to_num(x, nan=0.0, neginf=-INF), n(label), n(ids), to_np(values.float()), n(weight), **args)
    has = R.used_rows(x, n(label)) & (np.ones(len(x), bool) if weight is None else n(weight) != 0)
    div = to_np(r["div"]).astype(np.float64)
    fin = np.isfinite(want["div"])
    np.testing.assert_array_equal(div[~fin], want["div"][~fin])
    lim = want["div_lim"] + U * np.abs(np.where(fin, want["div"], 0))
    off = np.abs(div[fin] - want["div"][fin])
    assert np.all(off <= lim[fin]), (float((off - lim[fin]).max()), np.argwhere(off > lim[fin])[:4])
    assert np.all(div[~has] == 0)
    w = np.where(has, 1.0 if weight is None else n(weight).astype(np.float64), 0.0)
    z = R.z_bound(x.shape[1])
    got, s = to_np(r["stats"]).astype(np.float64), want["stats"]
    each = np.sum(w * lim * fin) + z * np.sum(w) + 2 * U * np.sum(w * (np.abs(np.where(np.isfinite(want["nll"]), want["nll"], 0)) + 1))
    for a, b in zip(got, s):
        assert (a == b) if not np.isfinite(b) else abs(a - b) <= each + U * abs(b) + 1e-12, (got, s)
    if r["dlogits"] is not None:
        d = wide(r["dlogits"])
        lim = want["lim"] + np.abs(want["grad"]) * R.STEP[kind] + R.LEAST[kind]
        off = np.abs(d - want["grad"])
        assert np.all(off <= lim), (float((off - lim).max()), np.argwhere(~(off <= lim))[:5])
        assert not d[~has].any()


SHAPES = [(1, 1, 1), (1, 7, 3), (3, 2, 2), (5, 2048, 20), (2, 2049, 256), (4, 4097, 64), (37, 1000, 5), (1, 70001, 256),
          (300, 513, 100), (1100, 130, 130), (3, 131072, 20), (140, 9001, 33)]
MODES = [(True, 0.0, 0.0), (True, 1.0, 0.0), (True, 0.3, 0.25), (False, 0.0, 0.4)]


@pytest.mark.parametrize("T,V,K", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
def test_distill(T, V, K, kind):
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for m, (rest, beta, hard) in enumerate(MODES):
        scale, pad, shift, where = ((1.0, 0, 0, "new"), (0.7, 5, 1, "inplace"))[m % 2]
        say(f"[distill] {T} {V} {K} {kind} {rest} {beta} {hard} {where}")
        x, label, gen = make(T, V, kind, T * V + m, pad, shift)
        ids, values = teacher(x, K, m, rest, scale, ragged=m == 1, kind=("float32", "float32", "bfloat16", "float16")[m])
        weight = torch.rand(T, device=dev, generator=gen) if m else None
        lab = label if hard or m == 1 else None
        if T > 4:
            if weight is not None:
                weight[1] = 0.0
                x[1] = float("nan")
            if lab is not None:
                lab[2], lab[3] = -1, V
                x[2] = float("nan")
            if K > 3:
                ids[0, 2] = ids[0, 0]          # the same token twice
                ids[4, 1], ids[4, 2] = -7, V   # none
                values[4, 3] = -INF
        h = wide(x)
        args = dict(rest=rest, beta=beta, hard=hard, scale=scale, teacher_scale=0.9, grad_scale=2.0)
        r = S.distill_loss(x, ids, values, weight=weight, labels=lab, dlogits=where, **args)
        torch.cuda.synchronize()
        check(r, h, lab, ids, values, weight, kind, **args)
        if where == "inplace":
            assert r["dlogits"].data_ptr() == x.data_ptr()


@pytest.mark.parametrize("T,V", [(8, 700), (8, 40000), (300, 700), (150, 40000)])
@pytest.mark.parametrize("kind", KINDS)
def test_masked_and_lost_places(T, V, kind):
    """Listed, given and all other tokens of -Inf, rows of nothing, of the
    lowest value, students that are sure, teachers that leave nothing, lists
    without entries."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    K = 9
    for rest, beta, hard in MODES + [(True, 0.5, 1.0), (True, 0.0, 0.5)]:
        say(f"[masked distill] {T} {V} {kind} {rest} {beta} {hard}")
        x, label, _ = make(T, V, kind, 7, pad=3)
        ids, values = teacher(x, K, 3, rest, 1.0)
        x[0] = -INF                                   # nothing
        x[1, ids[1, 0].long()] = -INF                 # the teacher's first
        x[2, label[2].long()] = -INF                  # the given token
        keep = torch.zeros(V, device=dev, dtype=torch.bool)
        keep[ids[3].long()] = True
        x[3, ~keep] = -INF                            # nothing beside the list
        label[3] = ids[3, 2]
        x[4] = torch.finfo(x.dtype).min               # the lowest value everywhere
        x[5, ~(torch.arange(V, device=dev) == ids[5, 0])] = torch.finfo(x.dtype).min  # a student that is sure
        label[5] = ids[5, 0]
        ids[6] = -1                                   # no list
        if rest:
            values[7] = -INF
            values[7, 0] = 0.0                        # a teacher that is sure
        h = wide(x)
        args = dict(rest=rest, beta=beta, hard=hard, scale=1.0)
        lab = label if hard else None
        for where in ("new", None, "inplace"):
            r = S.distill_loss(x, ids, values, labels=lab, dlogits=where, **args)
            torch.cuda.synchronize()
            if where:
                assert bool(torch.isfinite(r["dlogits"].float()).all())
                assert not wide(r["dlogits"])[h == -INF].any()
            check(r, h, lab, ids, values, None, kind, **args)


@pytest.mark.parametrize("T,V", [(9, 700), (9, 40000), (300, 700), (150, 140000)])
def test_nan_stays_in_its_row_and_is_seen(T, V):
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    nan, K = float("nan"), 9
    for rest, beta, hard in MODES:
        say(f"[nan distill] {T} {V} {rest} {beta} {hard}")
        x, label, _ = make(T, V, "float32", 11)
        ids, values = teacher(x, K, 3, rest, 1.0)
        lab = label if hard else None
        good = S.distill_loss(x, ids, values, labels=lab, rest=rest, beta=beta, hard=hard)
        off = torch.ones(T, V, device=dev, dtype=torch.bool).scatter_(1, ids.long(), False)
        first = off.float().argmax(1)                  # an unlisted token of each row
        x[0, first[0]] = nan
        x[1, ids[1, 0].long()] = nan
        x[2] = nan
        x[3, first[3]] = INF
        x[4, ids[4, 1].long()] = INF
        x[5, off[5]], x[5, ids[5].long()] = -INF, nan  # nothing but NaN on the list
        values[6, 2] = nan
        for where in ("new", None, "inplace"):
            r = S.distill_loss(x.clone(), ids, values, labels=lab, rest=rest, beta=beta, hard=hard, dlogits=where)
            torch.cuda.synchronize()
            assert bool(torch.isnan(r["div"][:7]).all()), r["div"][:7]
            assert torch.equal(r["div"][7:], good["div"][7:]) and bool(torch.isnan(r["stats"][:2]).all())
            if where:
                bad = torch.isnan(r["dlogits"])
                assert bool(bad[[0, 1, 2, 3, 4, 6]].all()), bad.all(1)[:7]
                assert bool(bad[5, ids[5].long()].all())
                assert torch.equal(r["dlogits"][7:], good["dlogits"][7:])


def test_a_rest_of_little_is_not_lost():
    """Unlisted tokens that together have a ten millionth of the student's
    probability: their own gradient is as exact as any."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for T in (2, 200):
        x, _, gen = make(T, 5000, "float32", 1, spread=0.5)
        ids, values = teacher(x, 8, 2, True, 1.0)
        x.scatter_(1, ids.long(), 25.0 + torch.rand(T, 8, device=dev, generator=gen))
        args = dict(rest=True, beta=0.0, hard=0.0, scale=1.0)
        r = S.distill_loss(x, ids, values, **args)
        assert float((1 - r["stats"][3] / T).abs()) < 1e-6
        check(r, wide(x), None, ids, values, None, "float32", **args)


def test_views_of_longer_lists():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for T, V in ((5, 30000), (300, 900)):
        x, _, _ = make(T, V, "bfloat16", 4)
        ids, values = teacher(x, 40, 1, True, 1.0)
        a = S.distill_loss(x, ids[:, 3:20], values[:, 3:20], beta=0.4)
        b = S.distill_loss(x, ids[:, 3:20].contiguous(), values[:, 3:20].contiguous(), beta=0.4)
        for k in a:
            assert torch.equal(a[k], b[k]), k


def test_from_a_teachers_scores():
    """A teacher's pass and a student's step as they are used together: a
    student that is its teacher has no divergence and no gradient."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for T, V, kind in ((3, 60000, "float32"), (400, 1000, "float16")):
        x, label, gen = make(T, V, kind, 8)
        s = S.token_scores(x, label, 50)
        for beta in (0.0, 0.5, 1.0):
            r = S.distill_loss(x, s["top_id"], s["top_logp"], beta=beta)
            # lists are rounded to fp32: log probabilities by 2^-24 of at most 32
            assert float(r["div"].abs().max()) < 1e-5
            assert float(r["dlogits"].float().abs().max()) < 1e-5
        y = (x.float() + torch.randn(T, V, device=dev, generator=gen)).to(x.dtype)
        args = dict(rest=True, beta=0.2, hard=0.1, scale=1.0)
        r = S.distill_loss(y, s["top_id"], s["top_logp"], labels=label, **args)
        check(r, wide(y), label, s["top_id"], s["top_logp"], None, kind, **args)


def test_gradient_against_differences():
    """Central differences in 64 bits along random directions (third-order term
    below 1e-5 at a step of 1e-3)."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    rng = np.random.default_rng(3)
    T, V, K = 8, 53, 6
    x, label, gen = make(T, V, "float32", 6, spread=1.0)
    weight = torch.rand(T, device=dev, generator=gen)
    for rest, beta, hard in MODES:
        ids, values = teacher(x, K, 5, rest, 1.1)
        args = dict(rest=rest, beta=beta, hard=hard, scale=1.1, teacher_scale=0.8, grad_scale=1.0)
        d = wide(S.distill_loss(x, ids, values, weight=weight, labels=label, **args)["dlogits"])
        f = lambda y: R.distill(y, to_np(label), to_np(ids), to_np(values), to_np(weight), **args)["stats"][0]  # noqa: E731,B023
        h = wide(x)
        for _ in range(10):
            v = rng.standard_normal((T, V))
            diff = (f(h + 1e-3 * v) - f(h - 1e-3 * v)) / 2e-3
            assert abs(diff - np.sum(d * v)) <= 1e-4 * np.abs(d * v).sum() + 1e-6


@pytest.mark.parametrize("T,V,K,kind,pad,shift", [(140, 131073, 64, "float32", 2, 1), (133, 90001, 256, "bfloat16", 0, 0),
                                                  (129, 170000, 30, "float16", 5, 3), (2, 400003, 256, "float32", 0, 0),
                                                  ((1 << 21) + 70, 3, 2, "bfloat16", 0, 0)])
def test_long_rows_and_many(T, V, K, kind, pad, shift):
    """On the GPU's own fp64 what the others check in numpy: rows beyond a
    workgroup's registers and marks, more rows than a launch."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    say(f"[long distill] {T} {V} {K} {kind}")
    x, label, gen = make(T, V, kind, T + V, pad, shift)
    ids, values = teacher(x, K, 1, True, 1.0)
    weight = torch.rand(T, device=dev, generator=gen)
    weight[T // 2] = 0.0
    r = S.distill_loss(x, ids, values, weight=weight)
    z, zb = x.double(), R.z_bound(V)
    lse = torch.logsumexp(z, 1, keepdim=True)
    on = torch.zeros(T, V, device=dev, dtype=torch.bool).scatter_(1, ids.long(), True)
    lr = torch.logsumexp(z.masked_fill(on, -INF), 1, keepdim=True)
    v = values.double()
    rest = (1 - v.exp().sum(1, keepdim=True)).clamp(min=2.0**-24)
    some = torch.isfinite(lr)
    lp = z.gather(1, ids.long()) - lse
    div = (v.exp() * (v - lp)).sum(1, keepdim=True) + torch.where(some, rest * (rest.log() - lr + lse), 0.0)
    div = torch.where(weight[:, None] != 0, div, 0.0)[:, 0]
    assert float((r["div"].double() - div).abs().max()) <= 5 * zb + U * float(div.abs().max())
    F = v.exp().sum(1, keepdim=True) + torch.where(some, rest, 0.0)
    p = (z - lse).exp()
    share = torch.where(on, 0.0, (z - lr).exp()) * torch.where(some, rest, 0.0)
    q = torch.zeros_like(z).scatter_(1, ids.long(), v.exp())
    g = weight.double()[:, None] * (p * F - share - q)
    lim = weight.double()[:, None] * (p * F + share + q) * (3 * zb + 4 * U * 60 + 16 * U)
    lim += g.abs() * R.STEP[kind] + R.LEAST[kind]
    off = (r["dlogits"].double() - g).abs()
    assert bool((off <= lim).all()), float((off - lim).max())


def test_beyond_32_bits():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    T, V, last, K = 34000, 131072, 3, 12
    x = torch.empty(T, V, device=dev, dtype=torch.bfloat16)
    block = torch.randn(500, V, device=dev, dtype=torch.bfloat16)
    for i in range(0, T, 500):
        x[i:i + 500] = block
    x[-last:] = torch.randn(last, V, device=dev) * 2
    h = wide(x[-last:])
    ids = torch.zeros(T, K, dtype=torch.int32, device=dev)
    values = torch.zeros(T, K, device=dev)
    ids[-last:], values[-last:] = teacher(x[-last:], K, 1, True, 1.0)
    weight = torch.zeros(T, device=dev)
    weight[-last:] = 1.0
    args = dict(rest=True, beta=0.5, hard=0.0, scale=1.0)
    r = S.distill_loss(x, ids, values, weight=weight, dlogits="inplace", **args)
    part = {"stats": r["stats"], "div": r["div"][-last:], "dlogits": r["dlogits"][-last:]}
    check(part, h, None, ids[-last:], values[-last:], None, "bfloat16", **args)
    assert not bool(r["dlogits"][:500].any()) and not bool(r["dlogits"][T // 2:-last].any())


def test_graphs_streams_and_forward_only():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for T, V, kind in ((3, 50000, "float32"), (700, 3000, "bfloat16")):
        x, label, gen = make(T, V, kind, 9)
        ids, values = teacher(x, 30, 1, True, 1.0)
        calls = [S.DistillLossCall(x, ids, values, labels=label, hard=0.2, beta=0.5),
                 S.DistillLossCall(x, ids, values, labels=label, hard=0.2, beta=0.5, dlogits=None),
                 S.DistillLossCall(x, ids, values, rest=False)]
        outs = lambda: [to_np(t.float()).copy() for c in calls for t in (c.stats, c.div, c.dlogits) if t is not None]  # noqa: E731,B023
        for c in calls:
            c.run()
        torch.cuda.synchronize()
        eager = outs()
        np.testing.assert_array_equal(eager[0], eager[3])
        np.testing.assert_array_equal(eager[1], eager[4])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for c in calls:
                c.run()
        for _ in range(3):
            for c in calls:
                c.div.fill_(7.0)
                c.stats.fill_(7.0)
                if c.dlogits is not None:
                    c.dlogits.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            for e, g in zip(eager, outs()):
                np.testing.assert_array_equal(e, g)
        streams = [torch.cuda.Stream() for _ in calls]
        for _ in range(5):
            for c, st in zip(calls, streams):
                st.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(st):
                    c.run()
            torch.cuda.synchronize()
            for e, g in zip(eager, outs()):
                np.testing.assert_array_equal(e, g)


def test_refusals():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    x = torch.zeros(4, 10, device=dev)
    y = torch.zeros(4, dtype=torch.int32, device=dev)
    i, v, w = torch.zeros(4, 3, dtype=torch.int32, device=dev), torch.zeros(4, 3, device=dev), torch.ones(4, device=dev)
    for call in (lambda: S.distill_loss(x, i.long(), v), lambda: S.distill_loss(x, i, v.double()), lambda: S.distill_loss(x, i, v[:, :2]),
                 lambda: S.distill_loss(x, i[:3], v[:3]), lambda: S.distill_loss(x, i, v.cpu()), lambda: S.distill_loss(x, i.t(), v.t()),
                 lambda: S.distill_loss(x, i, v, weight=w[:3]), lambda: S.distill_loss(x, i, v, weight=w.half()),
                 lambda: S.distill_loss(x, i, v, labels=y.long()), lambda: S.distill_loss(x, i, v, dlogits="there"),
                 lambda: S.distill_loss(x, i, torch.zeros(4, 9, device=dev)[:, :3])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: S.distill_loss(x, i, v, beta=1.5), lambda: S.distill_loss(x, i, v, hard=0.5),
                 lambda: S.distill_loss(x, i, v, rest=False, beta=0.5), lambda: S.distill_loss(x, i, v, scale=-1.0),
                 lambda: S.distill_loss(x, i, v, grad_scale=float("nan")),
                 lambda: S.distill_loss(x, i[:1].expand(4, 3), v[:1].expand(4, 3))):
        with pytest.raises(S.SparcmlError) as e:
            call()
        assert e.value.status == S.EINVAL
