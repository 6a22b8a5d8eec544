"""Plain numpy forms, in 64 bits, of scores, their gradient and distillation,
for their tests; and how far fp32 sums may put the kernels off."""
import numpy as np

U = 2.0**-24
STEP = {"float32": U, "bfloat16": 2.0**-8, "float16": 2.0**-11}
LEAST = {"float32": 1e-37, "bfloat16": 1e-37, "float16": 2.0**-25}
INF = np.inf


def z_bound(V):
    """A row's sum adds at most V / 256 + 33 terms in a row in a lane and joins
    lanes in a tree (12 steps); a term is off by its exponential's own error (2 u) and by
    its argument's (4 u |d|, weighted by the term: 2^-d d is at most 0.54, and
    68 u covers a thousand terms' share of it)."""
    return (V / 256 + 113) * U


def used_rows(x, label):
    T, V = x.shape
    return np.ones(T, bool) if label is None else (label >= 0) & (label < V)


def scores(x, label, scale, n):
    """x: float64 (unused rows may hold anything)."""
    T, V = x.shape
    has = used_rows(x, label)
    out = {"logp": np.zeros(T), "lse": np.zeros(T), "entropy": np.zeros(T), "norm": np.zeros((T, 2)),
           "top_id": np.full((T, n), -1), "top_logp": np.full((T, n), -INF)}
    for t in np.nonzero(has)[0]:
        top = x[t].max()
        if top == -INF:
            out["lse"][t] = out["norm"][t, 1] = -INF
            if label is not None:
                out["logp"][t] = -INF
            continue
        d = scale * (x[t] - top)
        ln = np.log(np.exp(d).sum())
        p = np.exp(d - ln)
        out["norm"][t] = top, ln
        out["lse"][t] = scale * top + ln
        out["entropy"][t] = -np.sum(p[p > 0] * (d - ln)[p > 0])
        if label is not None:
            out["logp"][t] = d[label[t]] - ln
        order = np.lexsort((np.arange(V), -x[t]))[:n]
        order = order[x[t, order] > -INF]
        out["top_id"][t, :order.size] = order
        out["top_logp"][t, :order.size] = (d - ln)[order]
    return out


def scores_grad(x, label, norm, scale, d_logp=None, d_lse=None, entropy=None, d_entropy=None, top_id=None, d_top=None):
    """The gradient, and the size of what it adds up in units of fp32's error."""
    T, V = x.shape
    has = used_rows(x, label) & (norm[:, 1] > -INF)
    g, lim = np.zeros((T, V)), np.zeros((T, V))
    norm = norm.astype(np.float64)
    for t in np.nonzero(has)[0]:
        to, size = np.zeros(V), np.zeros(V)
        if d_logp is not None and x[t, label[t]] > -INF:
            to[label[t]] += d_logp[t]
            size[label[t]] += abs(d_logp[t])
        if d_top is not None:
            for i, v in enumerate(top_id[t]):
                if 0 <= v < V and x[t, v] > -INF:
                    to[v] += d_top[t, i]
                    size[v] += abs(d_top[t, i])
        l = 0.0 if d_lse is None else float(d_lse[t])
        b = 0.0 if d_entropy is None else float(d_entropy[t])
        H = 0.0 if d_entropy is None else float(entropy[t])
        if l == 0 and b == 0 and not size.any():
            continue
        d = scale * (x[t] - norm[t, 0])
        lp = d - norm[t, 1]
        p = np.exp(lp)
        lp = np.where(p > 0, lp, 0.0)
        d = np.where(p > 0, d, 0.0)
        g[t] = scale * (to + p * (l - to.sum() - b * (lp + H)))
        # the exponent: 3 u of the difference, 2 u of the sum's log, u of both;
        # the factors: 8 u of each of their terms
        arg = U * (3 * np.abs(d) + 2 * abs(norm[t, 1]) + np.abs(lp))
        whole = abs(l) + size.sum() + abs(b) * abs(H)
        lim[t] = scale * (p * ((whole + abs(b) * np.abs(lp)) * (arg + 10 * U) + abs(b) * arg) + 4 * U * size)
    return g, lim


def first_entries(ids, values, V):
    """Which entries of a row's list are there."""
    there, seen = np.zeros(ids.size, bool), set()
    for i, v in enumerate(ids):
        if 0 <= v < V and values[i] != -INF and v not in seen:
            there[i] = True
            seen.add(v)
    return there


def distill(x, label, ids, values, weight, rest, beta, hard, scale, teacher_scale=1.0, grad_scale=1.0):
    """dict(div, nll, covered, stats, grad, lim, div_lim): lim as in scores_grad."""
    T, V = x.shape
    f32 = lambda y: float(np.float32(y))  # noqa: E731
    beta, hard, scale, teacher_scale, grad_scale = map(f32, (beta, hard, scale, teacher_scale, grad_scale))
    w = np.ones(T) if weight is None else weight.astype(np.float64)
    has = used_rows(x, label) & (w != 0)
    out = {k: np.zeros(T) for k in ("div", "nll", "covered", "div_lim")}
    grad, lim = np.zeros((T, V)), np.zeros((T, V))
    z = z_bound(V)
    with np.errstate(all="ignore"):
        for t in np.nonzero(has)[0]:
            if x[t].max() == -INF:
                continue
            y = scale * (x[t] - x[t].max())  # (the difference first: beside the lowest value a sum's log is nothing)
            lse = np.log(np.exp(y).sum())
            lp_all = y - lse
            p_all = np.exp(lp_all)
            there = first_entries(ids[t], values[t], V)
            on = ids[t][there]
            v = values[t][there].astype(np.float64)
            off = np.ones(V, bool)
            off[on] = False
            left = y[off] if off.any() else np.array([-INF])
            lse_off = -INF if left.max() == -INF else left.max() + np.log(np.exp(left - left.max()).sum())
            lp = list(lp_all[on])
            if rest:
                lq = list(v)
                r = max(1 - np.exp(v).sum(), 2.0**-24)
                if lse_off > -INF:
                    lq.append(np.log(r))
                    lp.append(lse_off - lse)
            else:
                s = teacher_scale * v
                lq = list(s - (s.max() + np.log(np.exp(s - s.max()).sum()))) if s.size else []
            lq, lp = np.array(lq), np.array(lp)
            q, p = np.exp(lq), np.exp(lp)
            zero = lambda a, b: np.where(a == 0, 0.0, a * b)  # noqa: E731
            if beta == 0:
                terms, f = zero(q, lq - lp), -q
            elif beta == 1:
                terms = f = zero(p, lp - lq)
            else:
                m = np.log(beta * q + (1 - beta) * p)
                f = (1 - beta) * zero(p, lp - m)
                terms = beta * zero(q, lq - m) + f
            f = np.where(lp == -INF, 0.0, f)
            # lp is off by z (of the rest by 2 z), and p, f and the terms with it
            apart = np.where(np.isfinite(lp), np.abs(lp - lq), 0.0)
            e_f = 2 * z * p * (1 + apart) * (beta != 0) + 1e-15
            out["div"][t] = terms.sum()
            out["div_lim"][t] = np.sum(2 * z * (p + q) * (1 + apart * (beta != 0))) + 1e-12
            out["covered"][t] = p_all[on].sum()
            h = 0.0
            if label is not None:
                out["nll"][t] = -lp_all[label[t]]
                h = hard if lp_all[label[t]] > -INF else 0.0
            k = w[t] * grad_scale * scale
            F = f.sum()
            g = p_all * (h - (1 - hard) * F)
            size = p_all * (h + (1 - hard) * np.abs(f).sum())
            more = p_all * e_f.sum()
            g[on] += (1 - hard) * f[:on.size]
            size[on] += (1 - hard) * np.abs(f[:on.size])
            more[on] += e_f[:on.size]
            if rest and lse_off > -INF:
                share = np.where(off, np.exp(y - left.max()), 0.0)
                share /= share.sum()
                g += (1 - hard) * f[-1] * share
                size += (1 - hard) * abs(f[-1]) * share
                more += e_f[-1] * share
            if label is not None:
                g[label[t]] -= h
                size[label[t]] += h
            d = np.where(p_all > 0, y.max() - y, 0.0)
            grad[t] = k * g
            lim[t] = abs(k) * (size * (3 * z + 4 * U * d + 16 * U) + more)
        loss = np.where(hard == 1, 0.0, (1 - hard) * out["div"]) + np.where(hard == 0, 0.0, hard * out["nll"])
        out["stats"] = np.array([np.sum(np.where(has, w * a, 0.0))
                                 for a in (loss, out["div"], out["nll"], out["covered"])])
    out["grad"], out["lim"] = grad, lim
    return out
