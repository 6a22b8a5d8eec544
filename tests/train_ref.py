"""Plain numpy forms of the training operators for their tests: the update in
64 bits and, operation by operation, in the 32 bits it is specified in; the
losses in 64 bits."""
import numpy as np

F = np.float32
BLOCK = 256


def philox_words(n, tensor, step, seed, first=0):
    """Word j & 3 of the Philox4x32-10 block at counter (j >> 2, tensor,
    step, 0), first <= j < first + n (plain ten rounds; first a multiple of 4)."""
    cnt = -(-n // 4)
    c = [np.arange(first // 4, first // 4 + cnt, dtype=np.uint64), np.full(cnt, tensor, np.uint64), np.full(cnt, step, np.uint64),
         np.zeros(cnt, np.uint64)]
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
    mask, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    for i in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> s32) ^ c[1] ^ k[0], p1 & mask, (p0 >> s32) ^ c[3] ^ k[1], p0 & mask]
        k = [(k[0] + np.uint64(0x9E3779B9)) & mask, (k[1] + np.uint64(0xBB67AE85)) & mask]
    return np.stack(c, 1).reshape(-1)[:n]


def e4m3_values():
    """Value of each of the 256 codes (OCP E4M3: bias 7, no infinities)."""
    v = np.zeros(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        x = f * 2.0**-9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        v[c] = np.nan if (c & 127) == 127 else (-x if c & 128 else x)
    return v


VALUES = e4m3_values()


def decode(codes, scale):
    """Moments of codes and scales, exact in fp32 and in 64 bits."""
    return VALUES[codes] * np.repeat(scale.astype(np.float64), BLOCK)[: codes.size]


def encode(x, draws, root):
    """Codes (uint8) and scales of x (fp32), rounded by 16-bit draws."""
    n, nb = x.size, -(-x.size // BLOCK)
    a = np.zeros(nb * BLOCK)
    a[:n] = np.abs(x.astype(np.float64))
    top = a.reshape(nb, BLOCK).max(1)
    power = np.full(nb, -100)
    for b in np.nonzero(top)[0]:
        k = -100
        while top[b] > 448 * 2.0**k:
            k += 1
        power[b] = k
    y = a[:n] / np.repeat(2.0**power, BLOCK)[:n]
    if root:
        y = np.maximum(y, 2.0**-9)
    unit = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(y, 2.0**-30))), -6) - 3)
    q = np.floor(y / unit + draws.astype(np.float64) / 65536) * unit
    pos = VALUES[:127]
    codes = np.searchsorted(pos, q).astype(np.uint8)
    assert np.array_equal(pos[codes], q)
    return np.where(np.signbit(x), codes | 128, codes).astype(np.uint8), (2.0**power).astype(F)


def adamw(p, g, m, v, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0, lr_scale=1.0, factor=1.0, bits=64):
    """New (p, m, v, root) from flat arrays, every operation in ``bits``."""
    T = np.float64 if bits == 64 else F
    p, g, m, v = (a.astype(T) for a in (p, g, m, v))
    decay, lr_scale = float(F(decay)), float(F(lr_scale))
    g = g * T(factor)
    m = T(beta1) * m + T(1 - beta1) * g
    v = T(beta2) * v + T(1 - beta2) * (g * g)
    root = np.sqrt(v)
    ibc2 = 1 / np.sqrt(1 - beta2**step)
    p = p * T(1 - lr * lr_scale * decay) - T(lr / (1 - beta1**step) * lr_scale) * (m / (root * T(ibc2) + T(eps)))
    return p, m, v, root


def rows(logits, labels, scale):
    """(lp, lse, softmax, has) of each row in 64 bits."""
    x = logits.astype(np.float64) * scale
    T, V = x.shape
    has = (labels >= 0) & (labels < V)
    lp, lse, soft = np.zeros(T), np.zeros(T), np.zeros((T, V))
    for t in np.nonzero(has)[0]:
        top = x[t].max()
        if top == -np.inf:
            lp[t] = lse[t] = -np.inf
            continue
        e = np.exp(x[t] - top)
        lse[t] = top + np.log(e.sum())
        lp[t] = x[t, labels[t]] - lse[t]
        soft[t] = e / e.sum()
    return lp, lse, soft, has


def dlogits(soft, labels, coef, scale):
    d = np.zeros_like(soft)
    for t in np.nonzero(coef)[0]:
        if soft[t].any():
            d[t] = -coef[t] * scale * soft[t]
            d[t, labels[t]] += coef[t] * scale
    return d


def policy(logits, labels, old, adv, weight, ref=None, clip_lo=0.2, clip_hi=0.2, kl=0.0, scale=1.0, grad_scale=1.0):
    clean = np.where((weight != 0)[:, None], logits, 0)
    lp, lse, soft, has = rows(clean, np.where(weight != 0, labels, -1), scale)
    out = np.zeros(4)
    coef = np.zeros(lp.size)
    for t in np.nonzero(has)[0]:
        w, A, rho = float(weight[t]), float(adv[t]), np.exp(lp[t] - float(old[t]))
        lo, hi = float(F(1 - float(F(clip_lo)))), float(F(1 + float(F(clip_hi))))
        u, held = rho * A, min(max(rho, lo), hi) * A
        k = dk = 0.0
        if ref is not None:
            far = float(ref[t]) - lp[t]
            k, dk = np.expm1(far) - far, -np.expm1(far)
        out += w * np.array([float(F(kl)) * k - min(u, held), -min(u, held), k, float(u > held)])
        coef[t] = w * (float(F(kl)) * dk - (u if u <= held else 0.0))
    return out, lp, grad_scale * dlogits(soft, labels, coef, scale), coef


def preference(logits, labels, bounds, ref=None, beta=0.1, smoothing=0.0, scale=1.0, grad_scale=1.0):
    lp, lse, soft, has = rows(logits, labels, scale)
    beta, smoothing = float(F(beta)), float(F(smoothing))
    ratio = np.where(has, lp - (0 if ref is None else ref.astype(np.float64)), 0.0)
    pairs = len(bounds) // 2
    out, coef = np.zeros(4), np.zeros(lp.size)
    for b in range(pairs):
        lo, mid, end = bounds[2 * b: 2 * b + 3]
        good, bad = beta * ratio[lo:mid].sum(), beta * ratio[mid:end].sum()
        h = good - bad
        sig = lambda z: 1 / (1 + np.exp(-z))  # noqa: E731
        loss = (1 - smoothing) * np.logaddexp(0, -h) + smoothing * np.logaddexp(0, h)
        q = beta * (smoothing * sig(h) - (1 - smoothing) * sig(-h)) / pairs
        coef[lo:mid], coef[mid:end] = q, -q
        out += np.array([loss, h > 0, good, bad]) / pairs
    coef = np.where(has, coef, 0.0)
    return out, lp, grad_scale * dlogits(soft, labels, coef, scale), coef
