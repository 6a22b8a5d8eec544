"""Token scores and their gradient against 64 bits: lists equal in every place
(ties to the lowest index), numbers within what fp32 sums may put them off
(scores_ref), the gradient against the formula's and against differences."""
import numpy as np
import pytest

import scores_ref as R
from gpu_util import say, to_np, torch_dev

pytestmark = pytest.mark.gpu
U, INF = R.U, np.inf
KINDS = ("float32", "bfloat16", "float16")


def make(T, V, kind, seed, pad=0, shift=0, spread=3.0):
    """Rows at any place and stride, NaN between them."""
    torch, dev = torch_dev()
    gen = torch.Generator(device=dev).manual_seed(seed)
    ld = V + pad
    flat = torch.full((T * ld + shift,), float("nan"), device=dev, dtype=getattr(torch, kind))
    x = flat[shift:].view(T, ld)[:, :V]
    x.copy_(torch.randn(T, V, device=dev, generator=gen) * spread)
    label = torch.randint(0, V, (T,), device=dev, generator=gen).int()
    near = torch.rand(T, device=dev, generator=gen) < 0.5
    x[near, label[near].long()] = 9.0
    return x, label, gen


def wide(x):
    return x.double().cpu().numpy()


def check_scores(got, x, label, scale, n, what=""):
    """x: float64."""
    T, V = x.shape
    scale = float(np.float32(scale))
    want = R.scores(x, label, scale, n)
    got = {k: None if v is None else to_np(v).astype(np.float64) for k, v in got.items()}
    np.testing.assert_array_equal(got["top_id"], want["top_id"], err_msg=what)
    z = R.z_bound(V)
    top, ln = want["norm"][:, 0], want["norm"][:, 1]
    np.testing.assert_array_equal(got["norm"][:, 0], top, err_msg=what)

    def close(name, a, b, lim):
        same = a == b  # infinities
        off = np.where(same, 0.0, np.abs(np.where(same, 0.0, a) - np.where(same, 0.0, b)))
        assert np.all(off <= lim), (what, name, float(np.nanmax(off - lim)), np.argwhere(~(off <= lim))[:5])

    # (each is rounded once)
    close("ln", got["norm"][:, 1], ln, z + U * np.abs(np.where(np.isfinite(ln), ln, 0)))
    lse = want["lse"]
    close("lse", got["lse"], lse, z + U * np.abs(np.where(np.isfinite(lse), lse, 0)))
    fin = np.isfinite(ln)
    has = R.used_rows(x, label)
    if label is not None:
        lp = want["logp"]
        close("logp", got["logp"], lp, z + U * np.abs(np.where(np.isfinite(lp), lp, 0)))
    close("top_logp", got["top_logp"], want["top_logp"],
          z + U * np.abs(np.where(np.isfinite(want["top_logp"]), want["top_logp"], 0)))
    # entropy: log of the sum, and the mean difference: off by z of itself twice
    # (its sum and Z) and by the exponentials' arguments, 4 u of each difference
    lim = np.zeros(T)
    for t in np.nonzero(has & fin)[0]:
        d = scale * (top[t] - x[t])
        p = np.exp(-d - ln[t])
        lim[t] = z + 2 * z * np.sum(p[p > 0] * d[p > 0]) + 4 * U * np.sum(p[p > 0] * d[p > 0] ** 2)
    close("entropy", got["entropy"], want["entropy"], lim + U * want["entropy"])


SHAPES = [(1, 1, 1), (1, 7, 3), (3, 2, 2), (5, 2048, 20), (2, 2049, 256), (4, 4097, 64), (37, 1000, 5), (1, 70001, 256),
          (3, 16384, 0), (300, 513, 100), (1100, 130, 130), (3, 131072, 20), (1, 300001, 1), (1030, 5000, 9)]


@pytest.mark.parametrize("T,V,n", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
def test_scores(T, V, n, kind):
    from paper_1802_08021_amd import sparcml as S
    torch, _ = torch_dev()
    for scale, pad, shift, given in ((1.0, 0, 0, False), (0.7, 3, 1, True)):
        say(f"[scores] {T} {V} {n} {kind} {scale} {pad}")
        x, label, _ = make(T, V, kind, T + V, pad, shift)
        if T > 2 and given:
            label[1], label[2] = -1, V  # not in use
            x[1] = float("nan")
        got = S.token_scores(x, label if given else None, n, scale)
        torch.cuda.synchronize()
        assert (got["logp"] is None) == (not given)
        check_scores(got, wide(x), to_np(label) if given else None, scale, n)


def rows_of_note(V, kind, gen):
    """Rows that lists or sums stumble over, each with a name."""
    torch, dev = torch_dev()
    dtype = getattr(torch, kind)
    rnd = lambda: torch.randn(V, device=dev, generator=gen)  # noqa: E731
    low = torch.finfo(dtype).min
    step = torch.arange(V, device=dev)
    rows = {
        "all equal": torch.zeros(V, device=dev),
        "few values": (rnd() * 1.2).round(),
        "two zeros": torch.where(step % 3 == 0, -0.0, 0.0),
        "rising": step / V * 4,
        "falling": -step / V * 4,
        "negative": -rnd().abs() - 1,
        "nothing": torch.full((V,), -INF, device=dev),
        "one": torch.where(step == V - 1, 3.0, -INF),
        "lowest": torch.full((V,), low, device=dev),
        "one above lowest": torch.where(step == V // 2, 1.0, low),
        "half": torch.where(step < V // 2, rnd(), -INF),
        "every ninth": torch.where(step % 9 == 4, rnd(), -INF),
        "a block": torch.where((step > V // 3) & (step < V // 3 + 700), 5.0, -9.0) + rnd() * 0.1,
        "equal at the top": torch.where(step % 5 == 0, 2.5, -rnd().abs()),
        "large": rnd() * 3 + 3e4,
        "apart": torch.where(step % 2 == 0, 60000.0, -60000.0) + 0 * step,
    }
    return rows, dtype


@pytest.mark.parametrize("V,n", [(5, 5), (700, 256), (3001, 20), (40000, 64), (140001, 256)])
@pytest.mark.parametrize("kind", KINDS)
def test_rows_of_note(V, n, kind):
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    gen = torch.Generator(device=dev).manual_seed(V)
    rows, dtype = rows_of_note(V, kind, gen)
    x = torch.stack([r.float() for r in rows.values()]).to(dtype)
    label = torch.full((len(rows),), V - 1, dtype=torch.int32, device=dev)
    for many in (1, 70):  # by slices, and a workgroup a row
        say(f"[note] {V} {n} {kind} {many}")
        y, l = x.repeat(many, 1), label.repeat(many)
        got = S.token_scores(y, l, n)
        torch.cuda.synchronize()
        # (a row's place beside a line decides which lane sums what: rows of odd
        # lengths are the same only within their sums' bounds)
        for at in (0, many // 2, many - 1):
            part = {k: v[at * len(rows):(at + 1) * len(rows)] for k, v in got.items()}
            check_scores(part, wide(x), to_np(label), 1.0, n, str(list(rows)))


def test_rows_of_nan_end():
    """NaN or +Inf: numbers are NaN, the list is of the others."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for kind in KINDS:
        for T, V in ((3, 50000), (700, 999)):
            x, label, _ = make(T, V, kind, 3)
            x[0, 5], x[1, 7], x[2] = float("nan"), INF, float("nan")
            got = {k: to_np(v) for k, v in S.token_scores(x, label, 30).items()}
            for k in ("lse", "entropy", "logp"):
                assert np.isnan(got[k][:3]).all() and np.isfinite(got[k][3:]).all(), k
            h = wide(x)
            keep = np.where(np.isnan(h[0]), -INF, h[0])
            want = np.lexsort((np.arange(V), -keep))[:30]
            np.testing.assert_array_equal(got["top_id"][0], want)
            assert got["top_id"][1, 0] == 7 and np.all(got["top_id"][2] == -1)


def test_more_rows_than_a_launch_and_beyond_32_bits():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    T = (1 << 21) + 70
    x, label, _ = make(T, 3, "bfloat16", 1)
    r = S.token_scores(x, label, 2)
    last = {k: v[-50:] for k, v in r.items()}
    check_scores(last, wide(x[-50:]), to_np(label[-50:]), 1.0, 2)
    d = torch.ones(T, device=dev)
    g = S.token_scores_grad(x, r["norm"], labels=label, d_logp=d)
    want, lim = R.scores_grad(wide(x[-50:]), to_np(label[-50:]), to_np(r["norm"][-50:]), 1.0, np.ones(50))
    assert np.all(np.abs(wide(g[-50:]) - want) <= lim + np.abs(want) * R.STEP["bfloat16"] + R.LEAST["bfloat16"])
    del x, r, g
    T, V, last, n = 34000, 131072, 3, 17
    x = torch.empty(T, V, device=dev, dtype=torch.bfloat16)
    block = torch.randn(500, V, device=dev, dtype=torch.bfloat16)
    for i in range(0, T, 500):
        x[i:i + 500] = block
    x[-last:] = torch.randn(last, V, device=dev) * 2
    label = torch.full((T,), -1, dtype=torch.int32, device=dev)
    label[-last:] = 77
    h, l = wide(x[-last:]), to_np(label[-last:])
    r = S.token_scores(x, label, n)
    check_scores({k: v[-last:] for k, v in r.items()}, h, l, 1.0, n)
    assert not bool(r["lse"][:-last].any()) and bool((r["top_id"][:-last] == -1).all())
    d = torch.ones(T, device=dev)
    g = S.token_scores_grad(x, r["norm"], labels=label, d_logp=d, entropy=r["entropy"], d_entropy=d, dlogits="inplace")
    want, lim = R.scores_grad(h, l, to_np(r["norm"][-last:]), 1.0, np.ones(last), None, to_np(r["entropy"][-last:]), np.ones(last))
    assert np.all(np.abs(wide(g[-last:]) - want) <= lim + np.abs(want) * R.STEP["bfloat16"] + R.LEAST["bfloat16"])
    assert not bool(g[:500].any()) and not bool(g[T // 2:-last].any())


# ---------------------------------------------------------------- gradient

def check_grad(d, x, label, norm, kind, scale, **more):
    more = {k: None if v is None else to_np(v) for k, v in more.items()}
    want, lim = R.scores_grad(x, label, to_np(norm), float(np.float32(scale)), **more)
    off = np.abs(wide(d) - want)
    lim = lim + np.abs(want) * R.STEP[kind] + R.LEAST[kind]
    assert np.all(off <= lim), (float((off - lim).max()), np.argwhere(~(off <= lim))[:5])


@pytest.mark.parametrize("T,V,n", SHAPES[:-2] + [(130, 9001, 256)])
@pytest.mark.parametrize("kind", KINDS)
def test_gradient(T, V, n, kind):
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    cases = [(1.0, 0, 0, "new", "logp lse entropy top"), (0.7, 5, 1, "inplace", "logp entropy top"),
             (1.25, 0, 0, "inplace", "lse"), (1.0, 3, 0, "new", "entropy")]
    for scale, pad, shift, where, which in cases:
        say(f"[scores grad] {T} {V} {n} {kind} {where} {which}")
        x, label, gen = make(T, V, kind, T * V + n, pad, shift)
        given = "logp" in which
        if T > 4 and given:
            label[1], label[2] = -5, V
            x[1] = float("nan")
            x[3, label[3].long()] = -INF
            x[4, V // 2:] = -INF
        s = S.token_scores(x, label if given else None, n, scale)
        rnd = lambda *shape: torch.randn(*shape, device=dev, generator=gen)  # noqa: E731
        more = {"d_" + k: rnd(T) for k in ("logp", "lse", "entropy") if k in which}
        if "entropy" in which:
            more["entropy"] = s["entropy"]
        if "top" in which and n:
            more["top_id"], more["d_top"] = s["top_id"], rnd(T, n)
            if T > 4 and n > 2:
                more["top_id"][0, 1] = more["top_id"][0, 0]  # the same token twice
                more["top_id"][0, 2] = label[0]
                more["top_id"][4, 1] = V - 1                 # a token that cannot come
                more["top_id"][4, 0] = V
        h = wide(x)
        d = S.token_scores_grad(x, s["norm"], labels=label if given else None, scale=scale, dlogits=where, **more)
        torch.cuda.synchronize()
        check_grad(d, np.nan_to_num(h, nan=0.0, neginf=-INF), to_np(label) if given else None, s["norm"], kind, scale, **more)
        if where == "inplace":
            assert d.data_ptr() == x.data_ptr()


def test_rows_without_derivatives_are_not_read():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for T, V in ((6, 30000), (400, 700)):
        x, label, gen = make(T, V, "bfloat16", 5)
        s = S.token_scores(x, label, 4)
        x[2] = float("nan")
        x[3] = -INF
        s["norm"][3, 1] = -INF
        a, b, c, d = (torch.randn(T, *k, device=dev, generator=gen) for k in ((), (), (), (4,)))
        for y in (a, b, c, d):
            y[2] = 0
        for where in ("new", "inplace"):
            g = S.token_scores_grad(x.clone(), s["norm"], labels=label, d_logp=a, d_lse=b, entropy=s["entropy"],
                                    d_entropy=c, top_id=s["top_id"], d_top=d, dlogits=where)
            assert bool(torch.isfinite(g.float()).all()) and not bool(g[2:4].any()) and bool(g[4].any())


def test_gradient_of_nan_rows_is_nan():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for T, V in ((6, 30000), (400, 700), (1100, 40)):
        x, label, gen = make(T, V, "float32", 9)
        x[1, V // 2], x[2], x[3, V - 1] = float("nan"), float("nan"), INF
        s = S.token_scores(x, label, 4)
        rnd = lambda *shape: torch.randn(*shape, device=dev, generator=gen)  # noqa: E731
        for more in (dict(d_logp=rnd(T)), dict(d_lse=rnd(T)), dict(entropy=s["entropy"], d_entropy=rnd(T)),
                     dict(top_id=s["top_id"], d_top=rnd(T, 4))):
            for where in ("new", "inplace"):
                g = S.token_scores_grad(x.clone(), s["norm"], labels=label, dlogits=where, **more)
                bad = torch.isnan(g).all(1)
                # (no entry of row 2 is on its list, of which nothing is left)
                assert bool(bad[1]) and bool(bad[3]) and (bool(bad[2]) or "d_top" in more), list(more)
                assert bool(torch.isfinite(g[4:]).all()) and bool(torch.isfinite(g[0]).all())


def test_masked_and_lowest_rows_have_gradients():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for kind in KINDS:
        for V in (700, 40000):
            gen = torch.Generator(device=dev).manual_seed(V)
            rows, dtype = rows_of_note(V, kind, gen)
            x = torch.stack([r.float() for r in rows.values()]).to(dtype)
            T, n = len(rows), 20
            label = torch.full((T,), V - 1, dtype=torch.int32, device=dev)
            s = S.token_scores(x, label, n)
            rnd = lambda *shape: torch.randn(*shape, device=dev, generator=gen)  # noqa: E731
            more = dict(d_logp=rnd(T), d_lse=rnd(T), entropy=s["entropy"], d_entropy=rnd(T), top_id=s["top_id"],
                        d_top=rnd(T, n))
            d = S.token_scores_grad(x, s["norm"], labels=label, **more)
            assert bool(torch.isfinite(d.float()).all()) and not bool(d[x == -INF].any())
            check_grad(d, wide(x), to_np(label), s["norm"], kind, 1.0, **more)


def test_gradient_against_differences():
    """The loss a logp + b entropy + l lse + g top along random directions, by
    central differences in 64 bits (third-order term below 1e-5 at 1e-3)."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    rng = np.random.default_rng(1)
    T, V, n, scale = 9, 61, 7, 1.1
    x, label, gen = make(T, V, "float32", 2, spread=1.0)
    s = S.token_scores(x, label, n, scale)
    rnd = lambda *shape: torch.randn(*shape, device=dev, generator=gen)  # noqa: E731
    a, b, l, g = rnd(T), rnd(T), rnd(T), rnd(T, n)
    d = wide(S.token_scores_grad(x, s["norm"], labels=label, d_logp=a, d_lse=l, entropy=s["entropy"], d_entropy=b,
                                 top_id=s["top_id"], d_top=g, scale=scale))
    h, lab, ids, s32 = wide(x), to_np(label), to_np(s["top_id"]), float(np.float32(scale))
    a, b, l, g = (to_np(y).astype(np.float64) for y in (a, b, l, g))

    def total(y):
        r = R.scores(y, lab, s32, 0)
        lp = s32 * y - r["lse"][:, None]
        return np.sum(a * r["logp"] + b * r["entropy"] + l * r["lse"]) + np.sum(g * np.take_along_axis(lp, ids, 1))

    for _ in range(20):
        v = rng.standard_normal((T, V))
        diff = (total(h + 1e-3 * v) - total(h - 1e-3 * v)) / 2e-3
        assert abs(diff - np.sum(d * v)) <= 1e-4 * np.abs(d * v).sum() + 1e-6


def test_graphs_streams_and_two_calls_at_once():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for T, V, kind in ((3, 50000, "float32"), (700, 3000, "bfloat16")):
        x, label, gen = make(T, V, kind, 9)
        x2, label2, _ = make(T, V, kind, 10)
        a = torch.randn(T, device=dev, generator=gen)
        calls = [S.TokenScoresCall(x, label, 20), S.TokenScoresCall(x2, None, 256)]
        calls[0].run()
        grad = S.TokenScoresGradCall(x, calls[0].norm, labels=label, d_logp=a, entropy=calls[0].entropy, d_entropy=a,
                                     top_id=calls[0].top_id, d_top=torch.randn(T, 20, device=dev, generator=gen))
        calls.append(grad)
        outs = lambda: [to_np(t.float()).copy() for c in calls for t in (  # noqa: E731
            (c.dlogits,) if c is grad else (c.lse, c.entropy, c.norm, c.top_id, c.top_logp))]
        for c in calls:
            c.run()
        torch.cuda.synchronize()
        eager = outs()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for c in calls:
                c.run()
        for _ in range(3):
            for c in calls[:2]:
                c.lse.fill_(7.0)
                c.top_id.fill_(7)
            grad.dlogits.fill_(7.0)
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


def test_timers_have_records():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    x, label, _ = make(4, 30000, "float32", 1)
    S.timing_enable(True)
    try:
        s = S.token_scores(x, label, 3)
        S.token_scores_grad(x, s["norm"], labels=label, d_lse=s["lse"])
        torch.cuda.synchronize()
        assert S.timing_read(S.TIMER_SCORES) > 0 and S.timing_read(S.TIMER_SCORES_GRAD) > 0
    finally:
        S.timing_enable(False)


def test_refusals():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    x = torch.zeros(4, 10, device=dev)
    y = torch.zeros(4, dtype=torch.int32, device=dev)
    f, m, i = torch.zeros(4, device=dev), torch.zeros(4, 2, device=dev), torch.zeros(4, 3, dtype=torch.int32, device=dev)
    g = torch.zeros(4, 3, device=dev)
    for call in (lambda: S.token_scores(x.double()), lambda: S.token_scores(x.t()), lambda: S.token_scores(x[0]),
                 lambda: S.token_scores(x, y.long()), lambda: S.token_scores(x, y[:3]), lambda: S.token_scores(x, y.cpu()),
                 lambda: S.token_scores(x, top=257), lambda: S.token_scores_grad(x, f), lambda: S.token_scores_grad(x, m.half()),
                 lambda: S.token_scores_grad(x, m, d_entropy=f), lambda: S.token_scores_grad(x, m, d_top=g),
                 lambda: S.token_scores_grad(x, m, top_id=i, d_top=g[:, :2]), lambda: S.token_scores_grad(x, m, top_id=i.long(), d_top=g),
                 lambda: S.token_scores_grad(x, m, d_lse=f, dlogits=None), lambda: S.token_scores_grad(x, m, d_lse=f[:3])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: S.token_scores(x, top=11), lambda: S.token_scores(x, scale=0.0), lambda: S.token_scores_grad(x, m, d_logp=f),
                 lambda: S.token_scores(x[:1].expand(4, 10))):
        with pytest.raises(S.SparcmlError) as e:
            call()
        assert e.value.status == S.EINVAL
