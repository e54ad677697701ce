"""The learner's operators written out in 64 bits (numpy), each with a bound on how far a 32-bit
evaluation in any order of association may be off.

The bounds count roundings.  U = 2^-24 is half a step of a 32-bit number, HALF[t] that of a stored
type.  A recurrence's error obeys the recurrence itself: E_t = |a_t| E_{t-1} + c U M_t with M the
recurrence of magnitudes and c the roundings of one step; products of gates over a span of n steps
carry n roundings, which is one more per step.
"""
import numpy as np

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
# half the distance of the smallest numbers
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def sigmoid(g):
    return 1.0 / (1.0 + np.exp(-g))


def stored(v, err, dtype):
    """Bound of a value with error `err` after it is rounded to its type."""
    return err + HALF[dtype] * (np.abs(v) + err) + TINY[dtype]


def scan(x, gate, h0=None, cut=None, form="linear", reverse=False, dy=None, dlast=None,
         dtype="f32"):
    """x [T][B][D]; gate like it or [D]; returns {name: (value, bound)}."""
    T, B, D = x.shape
    gated, col = form == "gated", gate.ndim == 1
    # roundings of one step.  linear: the fused multiply-add, the product of gates and the
    # composition of spans.  gated: also those of e^-|g| (its argument is off by |g| log2(e) U,
    # the exponential by 2), the reciprocal (2), their product and 1 + e.
    c = 4.0 if not gated else 14.0 + 2.0 * np.max(np.abs(gate), initial=0.0)
    full = np.broadcast_to(gate, x.shape)
    a = sigmoid(full) if gated else full
    rest = sigmoid(-full) if gated else np.ones_like(full)
    keep = np.ones((T, B, 1)) if cut is None else (cut == 0).astype(float)[:, :, None]
    order = range(T - 1, -1, -1) if reverse else range(T)
    s = np.zeros((B, D)) if h0 is None else h0.astype(float)
    M, E = np.abs(s), np.zeros((B, D))
    y, came = np.zeros_like(x), np.zeros_like(x)
    Ey, Ecame = np.zeros_like(x), np.zeros_like(x)
    for t in order:
        came[t] = np.where(keep[t] != 0, s, 0.0)
        Ecame[t] = np.where(keep[t] != 0, E, 0.0)
        M = np.where(keep[t] != 0, np.abs(a[t]) * M, 0.0) + np.abs(rest[t] * x[t])
        s = a[t] * came[t] + rest[t] * x[t]
        E = np.abs(a[t]) * Ecame[t] + c * U * M
        y[t], Ey[t] = s, E
    out = {"y": (y, stored(y, Ey, dtype)), "last": (s, E + U * np.abs(s))}
    if dy is None:
        return out
    back = np.zeros((B, D)) if dlast is None else dlast.astype(float)
    M, E = np.abs(back), np.zeros((B, D))
    lam, El = np.zeros_like(x), np.zeros_like(x)
    for t in reversed(list(order)):
        lam[t] = dy[t] + back
        Mt = np.abs(dy[t]) + M
        El[t] = E + c * U * Mt
        back = keep[t] * a[t] * lam[t]
        M = keep[t] * np.abs(a[t]) * Mt
        E = keep[t] * np.abs(a[t]) * El[t] + c * U * M
    out["dh0"] = (back, E + U * np.abs(back))
    # the states come back from y, rounded to its type; h0 does not
    Eh = Ecame + HALF[dtype] * (np.abs(came) + Ecame) + TINY[dtype]
    if gated:
        dx, Edx = lam * rest, El * rest + c * U * np.abs(lam * rest)
        slope = a * rest
        d = lam * (came - x) * slope
        Ed = (El * np.abs(came - x) + np.abs(lam) * (Eh + U * np.abs(came - x))) * slope + \
            (2 * c + 4) * U * np.abs(d)
    else:
        dx, Edx = lam, El
        d = lam * came
        Ed = El * np.abs(came) + np.abs(lam) * Eh + El * Eh + 2 * U * np.abs(d)
    out["dx"] = (dx, stored(dx, Edx, dtype))
    if col:
        # a sum of T x B terms in any order: at most one rounding per term of what is summed so far
        n = T * B
        total = np.sum(np.abs(d), axis=(0, 1))
        d, Ed = d.sum((0, 1)), Ed.sum((0, 1)) + n * U * total
    out["dgate"] = (d, stored(d, Ed, dtype))
    return out


def tokens(logits, ids=None, dlogp=None, dentropy=None, top=0, dtype="f32"):
    """logits [N][A] in 64 bits; returns {name: (value, bound)}, alternatives without a bound for
    their ids (they have to be equal)."""
    l = logits.astype(float)
    N, A = l.shape
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):     # of rows that are NaN
        m = np.max(np.where(np.isnan(l), -np.inf, l), 1, keepdims=True)
        bad = np.isnan(l).any(1) | (m[:, 0] == np.inf)
        empty = (m[:, 0] == -np.inf) & ~bad
        origin = np.where(np.isfinite(m), m, 0.0)
        live = l > -np.inf
        t = np.where(live, l - origin, 0.0)
        e = np.where(live, np.exp(t), 0.0)
        S = e.sum(1, keepdims=True)
        lse = np.where(empty[:, None], 0.0, np.log(np.where(S > 0, S, 1.0)))
        p = np.where(S > 0, e / np.where(S > 0, S, 1.0), 0.0)
        logp = np.where(live, t - lse, -np.inf)
        H = np.where(empty, 0.0, lse[:, 0] - (p * t).sum(1))
        mean, square = (p * np.abs(t)).sum(1), (p * t * t).sum(1)
    # terms that one thread adds one after another, and the joining of threads and waves
    depth = min(A, A / 64.0 + 64.0)
    El = U * (depth + 8.0 + 4.0 * mean + 2.0 * np.abs(lse[:, 0]))          # of log S
    EH = U * ((depth + 12.0) * (1.0 + mean) + 6.0 * square + 2.0 * np.abs(lse[:, 0])) + U * H
    H = np.where(bad, np.nan, H)
    out = {"entropy": (H, EH), "bad": bad}

    def of_logp(v, tv):
        return np.where(np.isfinite(v), El.reshape(-1, *([1] * (v.ndim - 1))) + 3.0 * U *
                        (np.abs(tv) + np.abs(np.where(np.isfinite(v), v, 0.0))), 0.0)
    rows = np.arange(N)
    if ids is not None:
        inside = (ids >= 0) & (ids < A)
        at = np.where(inside, ids, 0)
        v = np.where(inside, logp[rows, at], 0.0)
        v = np.where(bad & inside, np.nan, v)
        out["logp"] = (v, of_logp(v, t[rows, at]))
    if top:
        order = np.argsort(np.where(live, -l, np.inf), axis=1, kind="stable")[:, :top]
        if order.shape[1] < top:
            order = np.pad(order, ((0, 0), (0, top - order.shape[1])), constant_values=-1)
        ok = (order >= 0) & np.take_along_axis(live, np.maximum(order, 0), 1)
        out["top_ids"] = np.where(ok & ~bad[:, None], order, -1)
        v = np.where(ok, np.take_along_axis(logp, np.maximum(order, 0), 1), -np.inf)
        v = np.where(bad[:, None], np.nan, v)
        out["top_logp"] = (v, of_logp(v, np.take_along_axis(t, np.maximum(order, 0), 1)))
    if dlogp is not None or dentropy is not None:
        g = np.zeros(N) if dlogp is None else np.where(inside, dlogp, 0.0)
        gh = np.zeros(N) if dentropy is None else dentropy
        lp = np.where(live & ~bad[:, None], np.where(bad[:, None], 0.0, t) - lse, 0.0)
        Hs = np.where(bad, 0.0, H)
        inner = -g[:, None] - gh[:, None] * (lp + Hs[:, None])
        size = np.abs(g)[:, None] + np.abs(gh)[:, None] * (np.abs(lp) + Hs[:, None])
        d = np.where(bad[:, None], 0.0, p) * inner
        # a probability below the smallest normal number, 2^-126, counts as 0: its term is off by
        # itself, p |inner| < 2^-126 |inner|
        Ed = 2.0 ** -126 * np.abs(inner) + p * (np.abs(inner) * ((2.0 * np.abs(t) + 8.0) * U + 2.0 * El[:, None]) +
                  6.0 * U * size + np.abs(gh)[:, None] * (EH + El)[:, None])
        if dlogp is not None:
            hit = inside & live[rows, at]
            d[rows[hit], at[hit]] += g[hit]
            Ed[rows[hit], at[hit]] += 2 * U * np.abs(g[hit])
        d = np.where(bad[:, None], np.nan, d)
        out["dlogits"] = (d, stored(np.where(np.isnan(d), 0.0, d), Ed, dtype))
    return out


def draw(logits, u):
    """(action, log-probability) of each row; logits [N][A], u [N]."""
    l = logits.astype(float)
    actions, logps = [], []
    for row, x in zip(l, u.astype(float)):
        if np.isnan(row).any() or (row == np.inf).any():
            actions.append(0), logps.append(np.nan)
        elif not (row > -np.inf).any():
            actions.append(0), logps.append(-np.inf)
        else:
            e = np.exp(row - row.max())
            live = np.flatnonzero(row > -np.inf)
            total = np.cumsum(e)
            over = live[total[live] > x * total[-1]]
            i = int(over[0]) if len(over) else int(live[-1])
            actions.append(i), logps.append(row[i] - row.max() - np.log(total[-1]))
    return np.array(actions), np.array(logps)


def check(got, want, name, dtype="f32"):
    """got within the bound of want = (value, bound); NaN and infinities in the same places.

    The largest f16 number is 65504 = 2^16 - 2^5; the next step would be 2^16, and what is at or
    above the middle of the two, 65520, is rounded to infinity.  A value whose whole bound lies there
    has to be infinite, one whose bound holds 65520 may be."""
    v, bound = want
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == v.shape, f"{name}: shape {got.shape}, not {v.shape}"
    if dtype == "f16":
        bound = np.broadcast_to(bound, v.shape)
        past = np.abs(v) - bound >= 65520.0
        maybe = ~past & (np.abs(v) + bound >= 65520.0) & np.isinf(got) & (np.sign(got) == np.sign(v))
        v = np.where(past | maybe, np.copysign(np.inf, v), v)
    fine = np.isfinite(v)
    assert np.array_equal(np.isnan(got), np.isnan(v)), f"{name}: NaN in other places"
    assert np.array_equal(got[~fine & ~np.isnan(v)], v[~fine & ~np.isnan(v)]), f"{name}: infinities"
    over = np.abs(got - np.where(fine, v, 0.0)) > np.broadcast_to(bound, v.shape)
    over &= fine
    if over.any():
        at = tuple(np.argwhere(over)[0])
        raise AssertionError(f"{name}: {int(over.sum())} of {v.size} off, the first at {at}: "
                             f"{got[at]!r}, not {v[at]!r} +- "
                             f"{np.broadcast_to(bound, v.shape)[at]:.3g}")
