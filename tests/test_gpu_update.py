"""AdamW over many tensors and the gradient norm.  The 32-bit form is
specified operation by operation, so its weights and moments are compared bit
for bit with that sequence in numpy's fp32, and with 64 bits under the bound
its roundings give; codes and scales of the 8-bit form likewise bit for bit
with the rounding by its draws."""
import numpy as np
import pytest

import train_ref as R
from gpu_util import say, to_np, torch_dev

pytestmark = pytest.mark.gpu
F = np.float32

LAYOUTS = {
    "one": [1],
    "block edges": [255, 256, 257, 3, 1],
    "empty ones": [0, 5, 0, 4096, 0],
    "piece edges": [4095, 4097, 8192, 1023, 1025],
    "ragged": [70001, 33, 12288, 5, 999],
}


def make(lens, gtype, bits, copy, seed, shift=0):
    """A model in flat buffers that begin ``shift`` elements in, so that the
    tensors lie at odd addresses."""
    torch, dev = torch_dev()
    gen = torch.Generator(device=dev).manual_seed(seed)
    total = sum(lens)
    flat = lambda dt: torch.zeros(total + shift, dtype=dt, device=dev)[shift:]  # noqa: E731
    rnd = lambda: torch.randn(total, device=dev, generator=gen)  # noqa: E731
    st = {"param": flat(torch.float32), "grad": flat(gtype)}
    st["param"].copy_(rnd() * 0.05)
    st["grad"].copy_(rnd() * torch.exp(rnd()) * 1e-2)
    blocks = [-(-n // 256) for n in lens]
    if bits == 32:
        st["m"], st["v"] = flat(torch.float32), flat(torch.float32)
        st["m"].copy_(rnd() * 1e-2)
        st["v"].copy_(rnd().square() * 1e-4)
    else:
        for k in ("m", "v"):
            st[k] = flat(torch.uint8)
            st[k].copy_(torch.randint(0, 127, (total,), device=dev, generator=gen))
            st[k + "_scale"] = torch.exp2(torch.randint(-16, -13, (sum(blocks),), device=dev, generator=gen).float())
        st["m"] += (128 * (torch.rand(total, device=dev, generator=gen) < 0.5)).to(torch.uint8)
    if copy is not None:
        st["copy"] = flat(copy)
    st["lens"], st["blocks"] = lens, blocks
    return st


def call_of(st, **more):
    from paper_1802_08021_amd import sparcml as S
    v = {k: list(st[k].split(st["blocks"] if k.endswith("scale") else st["lens"]))
         for k in st if k not in ("lens", "blocks")}
    kw = {k: v[k] for k in ("m_scale", "v_scale") if k in v}
    return S.AdamwCall(v["param"], v["grad"], v["m"], v["v"], copies=v.get("copy"), **kw, **more)


def arrays(st):
    return {k: to_np(st[k].float() if st[k].dtype.itemsize == 2 else st[k]).copy()
            for k in st if k not in ("lens", "blocks")}


def parts(a, lens):
    return np.split(a, np.cumsum(lens)[:-1])


def expected(before, st, bits, step, decay, lr_scale, factor, seed, wide, **hyper):
    """New arrays by tensors: in fp32 as specified, or (wide) in 64 bits."""
    out = {k: [] for k in ("param", "m", "v", "m_scale", "v_scale")}
    split = {k: parts(before[k], st["blocks"] if k.endswith("scale") else st["lens"]) for k in before if k != "copy"}
    for t, n in enumerate(st["lens"]):
        m, v = split["m"][t], split["v"][t]
        if bits == 8:
            m = R.decode(m, split["m_scale"][t])
            v = R.decode(v, split["v_scale"][t])
            v = v * v if wide else v.astype(F) * v.astype(F)
        p, m, v, root = R.adamw(split["param"][t], split["grad"][t], m, v, step=step, decay=decay[t],
                                lr_scale=lr_scale[t], factor=factor, bits=64 if wide else 32, **hyper)
        if bits == 8 and not wide:
            w = R.philox_words(n, t, step, seed)
            m, ms = R.encode(m, w & np.uint64(0xFFFF), False)
            v, vs = R.encode(root, w >> np.uint64(16), True)
            out["m_scale"].append(ms)
            out["v_scale"].append(vs)
        out["param"].append(p)
        out["m"].append(m)
        out["v"].append(v)
    return {k: np.concatenate(v) for k, v in out.items() if v}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("gname,cname,shift", [("float32", None, 0), ("bfloat16", "bfloat16", 1),
                                               ("float16", "float16", 3)])
def test_adamw_matches_the_specified_operations(bits, layout, gname, cname, shift):
    torch, _ = torch_dev()
    lens = LAYOUTS[layout]
    copy = getattr(torch, cname) if cname else None
    st = make(lens, getattr(torch, gname), bits, copy, seed=len(layout) + bits, shift=shift)
    decay = [0.1 * (t % 3) for t in range(len(lens))]
    lr_scale = [1.0 - 0.25 * (t % 2) for t in range(len(lens))]
    call = call_of(st, decay=decay, lr_scale=lr_scale)
    clip = torch.tensor([2.5, 0.4], device=st["param"].device)
    hyper = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8)
    factor = float(F(0.5) * F(0.4))
    for step in (1, 7):
        say(f"[adamw] {bits} {layout} {gname} step {step}")
        before = arrays(st)
        call.run(step=step, clip=clip, grad_scale=0.5, seed=99, **hyper)
        torch.cuda.synchronize()
        after = arrays(st)
        want = expected(before, st, bits, step, decay, lr_scale, factor, 99, False, **hyper)
        for k, w in want.items():
            np.testing.assert_array_equal(after[k], w, err_msg=k)
        if copy is not None:
            np.testing.assert_array_equal(
                after["copy"], torch.from_numpy(want["param"]).to(copy).float().numpy(), err_msg="copy")
        # 64 bits: each of about ten roundings of the update moves it by 2^-24 of
        # itself at most, the weight's three by 2^-24 of the weight
        wide = expected(before, st, bits, step, decay, lr_scale, factor, 99, True, **hyper)
        u = 2.0**-24
        moved = np.abs(wide["param"] - before["param"]) + 0.01 * np.abs(before["param"])
        # (cancellation of m: both of its terms' roundings, through the division)
        assert np.all(np.abs(after["param"] - wide["param"]) <= 3 * u * np.abs(before["param"]) + 16 * u * moved + 1e-9)
        if bits == 32:
            np.testing.assert_allclose(after["v"], wide["v"], rtol=6 * u, atol=1e-38)


def test_adamw_skips_when_the_factor_is_zero_and_runs_on_other_streams():
    torch, dev = torch_dev()
    for bits in (32, 8):
        st = make([5000, 77], torch.float32, bits, torch.bfloat16, seed=5)
        call = call_of(st)
        before = arrays(st)
        call.run(lr=1e-2, step=1, clip=torch.tensor([float("inf"), 0.0], device=dev))
        torch.cuda.synchronize()
        for k, a in arrays(st).items():
            np.testing.assert_array_equal(a, before[k], err_msg=k)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            call.run(lr=1e-2, step=1)
        other.synchronize()
        want = expected(before, st, bits, 1, [0.0] * 2, [1.0] * 2, 1.0, 0, False, lr=1e-2, beta1=0.9, beta2=0.999,
                        eps=1e-8)
        got = arrays(st)
        for k, w in want.items():
            np.testing.assert_array_equal(got[k], w, err_msg=k)


def test_adamw_from_zero_states_and_zero_gradients():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    for bits in (32, 8):
        p = [torch.randn(n, device=dev) for n in (300, 1)]
        g = [torch.zeros(300, device=dev), torch.full((1,), 2.0, device=dev)]
        state = S.adamw_state(p, bits)
        kw = {} if bits == 32 else {"m_scale": state[2], "v_scale": state[3]}
        start = [to_np(x).copy() for x in p]
        S.AdamwCall(p, g, state[0], state[1], **kw).run(lr=0.1, step=1)
        torch.cuda.synchronize()
        # no gradient so far: nothing moves; a first gradient moves by lr
        np.testing.assert_array_equal(to_np(p[0]), start[0])
        np.testing.assert_allclose(to_np(p[1]), start[1] - 0.1, rtol=1e-5)
        assert all(bool(torch.isfinite(x.float()).all()) for x in state[0] + state[1])


def test_eight_bit_moments_are_unbiased():
    """The mean of a moment over steps drawn with many seeds is its value: a
    rounding is a coin of known probability, so the mean of K of them lies
    within 6 standard deviations, unit/2 sqrt(1/K) at most."""
    torch, dev = torch_dev()
    n, K = 1024, 400
    st = make([n], torch.float32, 8, None, seed=3)
    call = call_of(st)
    start = {k: st[k].clone() for k in ("param", "m", "v", "m_scale", "v_scale")}
    before = arrays(st)
    total = {"m": np.zeros(n), "v": np.zeros(n)}
    for seed in range(K):
        for k, x in start.items():
            st[k].copy_(x)
        call.run(lr=0.0, step=3, seed=seed, beta2=0.99)
        a = arrays(st)
        for k in total:
            total[k] += R.decode(a[k], a[k + "_scale"])
    p, m, v, root = R.adamw(before["param"], before["grad"], R.decode(before["m"], before["m_scale"]),
                            R.decode(before["v"], before["v_scale"]) ** 2, lr=0.0, step=3, beta2=0.99)
    for k, x in (("m", m), ("v", root)):
        scale = np.repeat(a[k + "_scale"].astype(np.float64), 256)
        y = np.abs(x) / scale
        unit = scale * 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(y, 1e-30))), -6) - 3)
        want = np.where(y < 2.0**-9, scale * 2.0**-9, x) if k == "v" else x
        # 2^-17: the draws have 16 bits
        assert np.all(np.abs(total[k] / K - want) <= unit * (6 * 0.5 / np.sqrt(K) + 2.0**-16)), k


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("gname,shift", [("float32", 0), ("bfloat16", 1), ("float16", 3)])
def test_grad_norm(layout, gname, shift):
    from paper_1802_08021_amd import sparcml as S
    torch, _ = torch_dev()
    st = make(LAYOUTS[layout], getattr(torch, gname), 32, None, seed=11, shift=shift)
    grads = list(st["grad"].split(st["lens"]))
    g = arrays(st)["grad"].astype(np.float64)
    for scale, top in ((1.0, float("inf")), (0.25, 1e-3), (1.0, 1e9)):
        say(f"[norm] {layout} {gname} {scale} {top}")
        call = S.GradNormCall(grads)
        call.run(top, scale)
        first = to_np(call.out).copy()
        call.run(top, scale)
        norm = scale * np.sqrt(np.sum(g * g))
        # fp64 sums, one rounding of each output
        np.testing.assert_allclose(first[0], norm, rtol=2.0**-23)
        np.testing.assert_allclose(first[1], min(1.0, top / (norm + 1e-6)), rtol=2.0**-22)
        np.testing.assert_array_equal(to_np(call.out), first)


def test_grad_norm_of_large_entries_infinities_and_nothing():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    big = torch.full((70000,), 3e37, device=dev)
    np.testing.assert_array_equal(to_np(S.grad_norm([big, big[:5]], 1.0)), [np.inf, 0.0])  # beyond fp32
    np.testing.assert_allclose(to_np(S.grad_norm([big[:100]], 1.0)), [3e38, 1 / 3e38], rtol=1e-6)
    for bad in (float("inf"), float("nan")):
        x = torch.ones(5000, device=dev)
        x[4321] = bad
        out = to_np(S.grad_norm([torch.ones(3, device=dev), x], 1.0))
        assert not np.isfinite(out[0]) and out[1] == 0.0
    np.testing.assert_array_equal(to_np(S.grad_norm([big[:0]], 1.0)), [0.0, 1.0])


def test_norm_and_step_replay_in_a_graph():
    torch, dev = torch_dev()
    for bits in (32, 8):
        a = make([9001, 1200], torch.float32, bits, None, seed=8)
        b = {k: (x.clone() if hasattr(x, "clone") else x) for k, x in a.items()}
        ca, cb = call_of(a), call_of(b)

        def step(c):
            c.run(lr=1e-3, step=4, clip=c.grad_norm(0.1), seed=12)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(ca)
        for _ in range(4):
            a["grad"].mul_(0.9)
            b["grad"].mul_(0.9)
            graph.replay()
            step(cb)
            torch.cuda.synchronize()
            for k in ("param", "m", "v"):
                np.testing.assert_array_equal(to_np(a[k]), to_np(b[k]), err_msg=k)
            assert float(ca.out[0]) == float(cb.out[0])


def test_a_tensor_beyond_32_bits():
    """Elements past 2^32 of one tensor: the last blocks move as specified,
    with the draws of their own place."""
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    n, tail = 2**32 + 1234, 4000
    p = torch.zeros(n, device=dev)
    g = torch.zeros(n, device=dev, dtype=torch.bfloat16)
    gen = torch.Generator(device=dev).manual_seed(1)
    p[-tail:] = torch.randn(tail, device=dev, generator=gen)
    g[-tail:] = torch.randn(tail, device=dev, generator=gen).to(g.dtype)
    m, v, ms, vs = S.adamw_state([p], 8)
    before = [to_np(p[-tail:]).copy(), to_np(g[-tail:].float()).copy()]
    call = S.AdamwCall([p], [g], m, v, m_scale=ms, v_scale=vs)
    np.testing.assert_allclose(float(call.grad_norm()[0]), np.linalg.norm(before[1].astype(np.float64)), rtol=1e-6)
    call.run(lr=1e-2, step=2, seed=77)
    torch.cuda.synchronize()
    zero = np.zeros(tail, F)
    want, wm, wv, root = R.adamw(*before, zero, zero, lr=1e-2, step=2, bits=32)
    np.testing.assert_array_equal(to_np(p[-tail:]), want)
    first = -(-(n - tail) // 256) * 256  # the first whole block of the tail
    k = first - (n - tail)
    w = R.philox_words(n - first, 0, 2, 77, first)
    codes, scale = R.encode(wm[k:], w & np.uint64(0xFFFF), False)
    np.testing.assert_array_equal(to_np(m[0].view(torch.uint8)[first:]), codes)
    np.testing.assert_array_equal(to_np(ms[0][first // 256:]), scale)
    codes, scale = R.encode(root[k:], w >> np.uint64(16), True)
    np.testing.assert_array_equal(to_np(v[0].view(torch.uint8)[first:]), codes)
    np.testing.assert_array_equal(to_np(vs[0][first // 256:]), scale)
    assert not bool(p[:1 << 20].any())


def test_refusals_of_tensors():
    from paper_1802_08021_amd import sparcml as S
    torch, dev = torch_dev()
    p, g = [torch.zeros(8, device=dev)], [torch.zeros(8, device=dev)]
    m, v = S.adamw_state(p)
    with pytest.raises(ValueError):
        S.AdamwCall(p, [g[0].double()], m, v)
    with pytest.raises(ValueError):
        S.AdamwCall([p[0].half()], g, m, v)
    with pytest.raises(ValueError):
        S.AdamwCall(p, g, [m[0][:7]], v)
    with pytest.raises(ValueError):
        S.AdamwCall(p, g, m, v, copies=[torch.zeros(8, device=dev)])
    with pytest.raises(ValueError):
        S.AdamwCall(p, g, m, v, decay=[0.0, 0.0])
    with pytest.raises(ValueError):
        S.AdamwCall(p, g, m, v, m_scale=[torch.zeros(1, device=dev)])
    with pytest.raises(ValueError):
        S.AdamwCall(p, g, m + m, v)
    with pytest.raises(ValueError):
        S.GradNormCall([torch.zeros(8, 8, device=dev).t()[:, :3]])
    with pytest.raises(ValueError):
        S.grad_norm([])
    call = S.AdamwCall(p, g, m, v)
    for bad in (dict(lr=-1.0, step=1), dict(lr=float("nan"), step=1), dict(lr=0.1, step=1, beta1=1.0),
                dict(lr=0.1, step=1, beta2=-0.1), dict(lr=0.1, step=1, eps=0.0), dict(lr=0.1, step=1, eps=1e-60),
                dict(lr=0.1, step=1, grad_scale=float("inf"))):
        with pytest.raises(S.SparcmlError) as e:
            call.run(**bad)
        assert e.value.status == S.EINVAL
    with pytest.raises(ValueError):
        call.run(lr=0.1, step=0)
    with pytest.raises(S.SparcmlError):
        call.grad_norm(0.0)
    with pytest.raises(S.SparcmlError):
        call.grad_norm(1.0, grad_scale=-1.0)
