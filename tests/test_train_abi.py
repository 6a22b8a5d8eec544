"""C-ABI checks of the training operators that need no GPU: every argument
error is found on the host, before any device work."""
import ctypes

import numpy as np
import pytest

import train_ref as R
from paper_1802_08021_amd import sparcml as S

FAKE = 0x1000  # never dereferenced: every call below fails validation first
BIG = 1 << 40


def ws_size(op, P, N, max_nnz):
    n = ctypes.c_size_t(0)
    return S.lib().sparcml_workspace_size(op, P, N, max_nnz, 1.0, ctypes.byref(n)), n.value


def test_workspace_sizes():
    for op, good, bad in (
            (S.OP_TENSORS, [(1, 0, 0), (65535, 2**42, 0)], [(0, 1, 0), (65536, 1, 0), (1, 2**42 + 1, 0)]),
            (S.OP_LOGPROB, [(1, 1, 1), (1, 2**31 - 1, 1000)], [(1, 0, 1), (1, 1, 0), (1, 2**31, 1), (1, 1, 2**31)]),
            (S.OP_POLICY, [(1, 5, 2**31 - 1)], [(1, 0, 5), (0, 5, 5)]),
            (S.OP_PREFERENCE, [(65535, 5, 5)], [(0, 5, 5), (65536, 5, 5), (1, 5, 0)])):
        for a in good:
            rc, n = ws_size(op, *a)
            assert rc == S.OK and n > 0, (op, a)
        for a in bad:
            assert ws_size(op, *a)[0] == S.EINVAL, (op, a)
    assert ws_size(S.OP_TENSORS, 4, 2**30, 0)[1] > ws_size(S.OP_TENSORS, 4, 2**20, 0)[1]


def tensors(count=2, n=10, **over):
    arr = (S.Tensor * count)()
    for a in arr:
        for k in ("param", "grad", "m", "v", "m_scale", "v_scale"):
            setattr(a, k, FAKE)
        a.n, a.lr_scale = n, 1.0
        for k, x in over.items():
            setattr(a, k, x)
    return arr


def prepare(arr, count=2, gtype=S.F32, ctype=S.BF16, bits=32, plan=True, ws=FAKE, ws_bytes=BIG):
    p = S.Tensors()
    return S.lib().sparcml_tensors_prepare(count, arr, gtype, ctype, bits, ctypes.byref(p) if plan else None, ws,
                                           ws_bytes, None)


def test_prepare_refusals():
    assert prepare(tensors(), count=0) == S.EINVAL
    assert prepare(tensors(), count=65536) == S.EINVAL
    assert prepare(None) == S.EINVAL
    assert prepare(tensors(), plan=False) == S.EINVAL
    assert prepare(tensors(), gtype=3) == S.EINVAL
    assert prepare(tensors(), gtype=-1) == S.EINVAL
    assert prepare(tensors(), bits=16) == S.EINVAL
    for k in ("param", "grad", "m", "v"):
        assert prepare(tensors(**{k: None})) == S.EINVAL
    for k in ("m_scale", "v_scale"):
        assert prepare(tensors(**{k: None}), bits=8) == S.EINVAL
    assert prepare(tensors(copy=FAKE), ctype=S.F32) == S.EINVAL
    assert prepare(tensors(copy=FAKE), ctype=7) == S.EINVAL
    assert prepare(tensors(n=2**34 + 1)) == S.EINVAL
    assert prepare(tensors(decay=float("nan"))) == S.EINVAL
    assert prepare(tensors(lr_scale=float("inf"))) == S.EINVAL
    assert prepare(tensors(count=300, n=2**34), count=300) == S.EINVAL  # more than 2^42 together
    assert prepare(tensors(), ws=None) == S.EWORKSPACE
    assert prepare(tensors(), ws_bytes=16) == S.EWORKSPACE
    assert "workspace" in S.last_error()


def test_step_and_norm_refuse_without_a_plan():
    p, a = S.Tensors(), S.AdamwArgs(lr=0.1, beta1=0.9, beta2=0.9, eps=1e-8, grad_scale=1.0, step=1)
    L = S.lib()
    assert L.sparcml_adamw(None, ctypes.byref(a), None, None) == S.EINVAL
    assert L.sparcml_adamw(ctypes.byref(p), ctypes.byref(a), None, None) == S.EINVAL  # never prepared
    assert L.sparcml_grad_norm(ctypes.byref(p), 1.0, 1.0, FAKE, None) == S.EINVAL
    assert "plan" in S.last_error()


def logits(**over):
    a = S.Logits(FAKE, FAKE, 4, 10, 10, S.F32, 1.0)
    for k, x in over.items():
        setattr(a, k, x)
    return a


BAD_LOGITS = [dict(x=None), dict(label=None), dict(rows=0), dict(rows=2**31), dict(vocab=0), dict(ld=9),
              dict(vocab=2**31, ld=2**31), dict(ld=2**31), dict(type=3), dict(scale=0.0), dict(scale=-1.0),
              dict(scale=float("nan")), dict(scale=float("inf"))]


def test_token_logprob_refusals():
    f = S.lib().sparcml_token_logprob
    for over in BAD_LOGITS:
        assert f(ctypes.byref(logits(**over)), FAKE, FAKE, FAKE, BIG, None) == S.EINVAL, over
    assert f(None, FAKE, FAKE, FAKE, BIG, None) == S.EINVAL
    assert f(ctypes.byref(logits()), None, FAKE, FAKE, BIG, None) == S.EINVAL
    assert f(ctypes.byref(logits()), FAKE, FAKE, None, BIG, None) == S.EWORKSPACE
    assert f(ctypes.byref(logits()), FAKE, FAKE, FAKE, 3, None) == S.EWORKSPACE


def policy(lo=0.2, hi=0.2, kl=0.0, gs=1.0, ref=None, x=None, d=0x100000, ldd=10, logp=FAKE, stats=FAKE, ws=FAKE,
           ws_bytes=BIG, **null):
    a = S.PolicyArgs(FAKE, ref, FAKE, FAKE, lo, hi, kl, gs)
    for k in null:
        setattr(a, k, None)
    x = logits() if x is None else x
    return S.lib().sparcml_policy_loss(ctypes.byref(x), ctypes.byref(a), logp, stats, d, ldd, ws, ws_bytes, None)


def test_policy_refusals():
    for over in BAD_LOGITS:
        assert policy(x=logits(**over)) == S.EINVAL, over
    nan, inf = float("nan"), float("inf")
    for kw in (dict(lo=-0.1), dict(lo=1.1), dict(lo=nan), dict(hi=-0.1), dict(hi=nan), dict(kl=nan, ref=FAKE),
               dict(gs=inf), dict(logp=None), dict(stats=None), dict(old_logp=1), dict(adv=1), dict(weight=1),
               dict(ldd=9), dict(ldd=2**31), dict(d=FAKE, ldd=12), dict(d=FAKE + 4), dict(d=FAKE + 156),
               dict(d=FAKE - 156)):
        assert policy(**kw) == S.EINVAL, kw
    assert policy(ws=None) == S.EWORKSPACE
    assert policy(ws_bytes=8) == S.EWORKSPACE
    assert S.lib().sparcml_policy_loss(ctypes.byref(logits()), None, FAKE, FAKE, None, 0, FAKE, BIG, None) == S.EINVAL


def preference(bounds=(0, 2, 4), pairs=None, beta=0.1, eps=0.0, gs=1.0, x=None, d=0x100000, ldd=10, logp=FAKE,
               stats=FAKE, ws=FAKE, ws_bytes=BIG):
    b = (ctypes.c_uint64 * len(bounds))(*bounds) if bounds else None
    x = logits() if x is None else x
    return S.lib().sparcml_preference_loss(ctypes.byref(x), len(bounds or ()) // 2 if pairs is None else pairs, b, None,
                                           beta, eps, gs, logp, stats, d, ldd, ws, ws_bytes, None)


def test_preference_refusals():
    for over in BAD_LOGITS:
        assert preference(x=logits(**over)) == S.EINVAL, over
    nan = float("nan")
    for kw in (dict(bounds=None, pairs=1), dict(pairs=0), dict(pairs=65536), dict(bounds=(1, 2, 4)),
               dict(bounds=(0, 3, 2)), dict(bounds=(0, 2, 3)), dict(bounds=(0, 2, 5)), dict(bounds=(0, 5, 4)),
               dict(bounds=(0, 3, 2, 3, 4)), dict(beta=nan), dict(gs=nan), dict(eps=-0.1), dict(eps=1.1),
               dict(eps=nan), dict(logp=None), dict(stats=None), dict(ldd=9), dict(d=FAKE + 8)):
        assert preference(**kw) == S.EINVAL, kw
    assert preference(ws=None) == S.EWORKSPACE
    assert preference(ws_bytes=8) == S.EWORKSPACE


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    x, y, f = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for call in (lambda: S.token_logprob(x, y), lambda: S.policy_loss(x, y, f, f, f),
                 lambda: S.preference_loss(x, y, [0, 2, 4]), lambda: S.grad_norm([f]),
                 lambda: S.AdamwCall([f], [f], [f], [f])):
        with pytest.raises(ValueError):
            call()


def test_plain_forms_agree_with_differences():
    """The tests' own formulas: the losses' derivatives by central differences,
    the codes' nearest neighbours, the draws' known answer."""
    rng = np.random.default_rng(0)
    T, V = 8, 11
    x = rng.standard_normal((T, V))
    label = rng.integers(0, V, T)
    label[3] = -1
    f32 = lambda a: a.astype(np.float32)  # noqa: E731
    old, adv, w = f32(rng.standard_normal(T) - 2.4), f32(rng.standard_normal(T)), f32(rng.random(T))
    ref = f32(rng.standard_normal(T) - 2.4)
    for f in (lambda y: R.policy(y, label, old, adv, w, ref, kl=0.1, scale=1.5),
              lambda y: R.preference(y, label, [0, 2, 4, 4, 8], ref, 0.5, 0.1, 1.5)):
        g = f(x)[2]
        for _ in range(20):
            v = rng.standard_normal((T, V))
            diff = (f(x + 1e-5 * v)[0][0] - f(x - 1e-5 * v)[0][0]) / 2e-5
            assert abs(diff - np.sum(g * v)) < 1e-7 * (1 + np.abs(g * v).sum())
    # Random123's known answer for the zero counter and key
    assert [hex(w) for w in R.philox_words(4, 0, 0, 0)] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    v = f32(rng.standard_normal(700))
    for draw in (0, 32768, 65535):
        c, s = R.encode(v, np.full(700, draw), False)
        assert np.all(np.abs(R.decode(c, s) - v) <= np.abs(v) / 8 + np.repeat(s, 256)[:700] * 2.0**-9)
