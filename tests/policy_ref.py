"""Plain 64-bit numpy forms of the placement policy operators, one row at a
time, with the error bounds that the GPU tests hold the kernels to.

EPS is half a step of float32: every float32 operation is off by at most EPS
relative to its result, the exponential and the logarithm by a few of them."""
import numpy as np
import torch

EPS = 2.0**-24
#: half a step of the type that a gradient is rounded to
HALF_STEP = {"float32": 2.0**-24, "bfloat16": 2.0**-8, "float16": 2.0**-11}
#: below this a float16 is spaced evenly: half its step there
HALF_TINY = {"float32": 0.0, "bfloat16": 0.0, "float16": 2.0**-25}
NO_PLACE = 65535
#: The smallest float32 that is held to EPS of itself is 2^-126.  A weight
#: exp z below it may become 0, which moves it by less than 2^-126 and, as the
#: weights' sum is 1 - 2^-8 at least, its probability by less than 2^-125.
TINY = 2.0**-125


def policy_of(s, block, scen0, n_pol):
    return ((scen0 + s) // block) % n_pol


def settings_of(n_pol, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """float64 [n_pol, 4], each value as float32 holds it."""
    cols = [np.broadcast_to(np.asarray(x, np.float32), (n_pol,)) for x in (temperature, top_k, top_p, min_p)]
    return np.stack(cols, 1).astype(np.float64)


def kept_sums(x, T, k, p, m):
    """(C, last) of one row: the sums of the kept weights and the last resource
    of positive weight; None where it has no valid distribution."""
    if np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
        return None
    if not (0 <= T < np.inf and k >= 0 and 0 <= p <= 1 and 0 <= m <= 1):
        return None
    order = np.lexsort((np.arange(x.size), -x))
    order = order[x[order] > -np.inf]
    if T == 0 or p == 0:
        k = 1
    w = np.exp((x - x.max()) / (T if T else 1.0))
    order = order[:int(k)] if k >= 1 else order
    ws = w[order]
    if 0 < p < 1:
        before = np.concatenate([[0.0], np.cumsum(ws)[:-1]])
        order = order[(before < p * ws.sum()) | (np.arange(order.size) == 0)]
        ws = w[order]
    order = order[(ws >= m) | (np.arange(order.size) == 0)]
    kept = np.zeros(x.size)
    kept[order] = w[order]
    return np.cumsum(kept), np.flatnonzero(kept)[-1]


def draw(C, last, u):
    place = np.searchsorted(C, np.maximum(u, 0.0) * C[-1], side="right")
    return np.where(np.isnan(u), NO_PLACE, np.minimum(place, last))


def sample(logits, u, settings, block=1, scen0=0):
    P, N, R = logits.shape
    S = u.shape[1]
    pol = policy_of(np.arange(S), block, scen0, P)
    place = np.full((N, S), NO_PLACE, np.int64)
    for p in np.unique(pol):
        at = np.flatnonzero(pol == p)
        for v in range(N):
            sums = kept_sums(logits[p, v], *settings[p])
            if sums is not None:
                place[v, at] = draw(*sums, u[v, at])
    return place


def log_pi(x, T):
    """(log-probabilities, z) of one row; NaN where it is invalid, -inf where empty."""
    if np.isnan(x).any() or (x == np.inf).any() or not 0 < T < np.inf:
        return np.full(x.size, np.nan), np.zeros(x.size)
    if (x == -np.inf).all():
        return np.full(x.size, -np.inf), np.zeros(x.size)
    z = (x - x.max()) / T
    return z - np.log(np.exp(z).sum()), np.where(np.isfinite(z), z, 0.0)


def logp(logits, place, settings, block=1, scen0=0):
    """(logp [S], bound [S]).  A term's z = (l - max) / T carries three
    roundings, its logarithm of the sum those of at most 1024 exponentials added
    by lane and then across lanes: EPS (4 |z| + 40).  At most 32 terms are added
    in 32 bits (EPS * 32 of their magnitudes), the rest in 64, and the total is
    rounded once."""
    P, N, R = logits.shape
    S = place.shape[1]
    pol = policy_of(np.arange(S), block, scen0, P)
    total, size, off = np.zeros(S), np.zeros(S), np.zeros(S)
    for p in np.unique(pol):
        at = np.flatnonzero(pol == p)
        for v in range(N):
            lp, z = log_pi(logits[p, v], settings[p, 0])
            a = place[v, at]
            ok = a < R
            t = np.where(ok, lp[np.minimum(a, R - 1)], np.nan if np.isnan(lp).any() else -np.inf)
            total[at] += t
            size[at] += np.where(np.isfinite(t), np.abs(t), 0)
            off[at] += 4 * np.abs(z[np.minimum(a, R - 1)]) + 40
    return total, EPS * (33 * size + off)


def grad(logits, place, weight, settings, block=1, scen0=0, dtype="float32"):
    """(grad [P, N, R], bound).  A resource's sum h of n weights is off by at
    most EPS n sum |w|; W adds at most 30 roundings of sum |h|; pi as in logp."""
    P, N, R = logits.shape
    S = place.shape[1]
    pol = policy_of(np.arange(S), block, scen0, P)
    g, tol = np.zeros((P, N, R)), np.zeros((P, N, R))
    for p in range(P):
        at = np.flatnonzero(pol == p)
        T = settings[p, 0]
        for v in range(N):
            lp, z = log_pi(logits[p, v], T)
            if np.isnan(lp).any():
                g[p, v] = np.nan
                continue
            allowed = logits[p, v] > -np.inf
            a, w = place[v, at], weight[at]
            ok = a < R
            h = np.bincount(a[ok], w[ok], R)[:R] * allowed
            n = np.bincount(a[ok], minlength=R)[:R] * allowed
            A = np.bincount(a[ok], np.abs(w[ok]), R)[:R] * allowed
            W = h.sum()
            pi = np.exp(lp)
            g[p, v] = np.where(allowed, (h - W * pi) / T, 0)
            d_w = EPS * ((n * A).sum() + 30 * np.abs(h).sum())
            d = EPS * n * A + pi * d_w + np.abs(W) * pi * EPS * (4 * np.abs(z) + 44)
            d = (d + EPS * 2 * (np.abs(h) + np.abs(W) * pi) + np.abs(W) * TINY) / T + 4 * EPS * np.abs(g[p, v])
            tol[p, v] = d + HALF_STEP[dtype] * (np.abs(g[p, v]) + d) + HALF_TINY[dtype]
    return g, tol


def distill(logits, ids, top, settings, weight=None, dtype="float32"):
    """(loss [P, N], its bound, grad, its bound)."""
    P, N, R = logits.shape
    K = ids.shape[2]
    loss, ltol = np.zeros((P, N)), np.zeros((P, N))
    g, gtol = np.zeros((P, N, R)), np.zeros((P, N, R))
    for p in range(P):
        T = settings[p, 0]
        for v in range(N):
            lp, z = log_pi(logits[p, v], T)
            allowed = logits[p, v] > -np.inf
            use = (ids[p, v] < R) & (top[p, v] != -np.inf)
            y = top[p, v][use]
            if np.isnan(lp).any() or np.isnan(y).any() or (y == np.inf).any():
                loss[p, v] = np.nan
                g[p, v] = np.nan
                continue
            if not use.any():
                continue
            y = (y - y.max()) / T
            t = np.exp(y) / np.exp(y).sum()
            i = ids[p, v][use]
            q = np.bincount(i, t, R)[:R]
            # an entry's weight: the roundings of y, of the exponential, of a sum of K and of the quotient
            dq = np.bincount(i, t * EPS * (4 * np.abs(y) + K + 40) + TINY, R)[:R]
            pi = np.exp(lp)
            dpi = pi * EPS * (4 * np.abs(z) + 44) + TINY
            pos = q > 0
            if (pos & ~allowed).any():
                loss[p, v] = np.inf
            else:
                term = np.zeros(R)
                term[pos] = q[pos] * (np.log(q[pos]) - lp[pos])
                loss[p, v] = term.sum()
                dterm = np.zeros(R)
                lq = np.log(q[pos])
                dterm[pos] = dq[pos] * (1 + np.abs(lq - lp[pos])) + q[pos] * EPS * (4 * np.abs(z[pos]) + 44 + 4 * np.abs(lq) + 4 * np.abs(lp[pos]))
                ltol[p, v] = dterm.sum() + 24 * EPS * np.abs(term).sum() + EPS * abs(loss[p, v])
            w = 1.0 if weight is None else weight[p, v]
            g[p, v] = np.where(allowed, w * (pi - q) / T, 0)
            d = abs(w) / T * (dpi + dq) + 4 * EPS * np.abs(g[p, v])
            gtol[p, v] = d + HALF_STEP[dtype] * (np.abs(g[p, v]) + d) + HALF_TINY[dtype]
    return loss, ltol, g, gtol


def near(got, want, tol, what):
    """Every value within its bound; infinities and NaN in the same places."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN elsewhere"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), f"{what}: infinities differ"
    fine = np.isfinite(want)
    off = np.abs(got[fine] - want[fine]) - np.broadcast_to(tol, want.shape)[fine]
    assert not (off > 0).any() and np.isfinite(got[fine]).all(), f"{what}: {off.max():.3g} over the bound"


def grid_of(weight, n_scen):
    """The largest step that a weight may be rounded to where scenarios share a
    row: sums of up to min(n_scen rounded up to 512, 2^22) weights below 2^(e + 1) are exact
    in float64 on multiples of 2^(e + L - 52), for L the bits of that count; e is
    of the largest finite weight of the policy."""
    w = np.abs(weight[np.isfinite(weight)])
    if not w.size or not w.max():
        return 0.0
    n = min(-(-n_scen // 512) * 512, 2**22)
    return 2.0 ** (np.floor(np.log2(w.max())) + n.bit_length() - 52)


def grad_shared(logits, place, weight, settings, block=1, scen0=0, dtype="float32"):
    """(grad, bound) where weights are rounded to the grid and their sums exact:
    a resource's sum of n weights is off by n half steps and one rounding to
    float32, W by 30 roundings more, pi as in logp."""
    P, N, R = logits.shape
    S = place.shape[1]
    pol = policy_of(np.arange(S), block, scen0, P)
    g, tol = np.zeros((P, N, R)), np.zeros((P, N, R))
    for p in range(P):
        at = np.flatnonzero(pol == p)
        T, w = settings[p, 0], weight[at].astype(np.float64)
        half = grid_of(w, S) / 2
        for v in range(N):
            lp, z = log_pi(logits[p, v], T)
            allowed = logits[p, v] > -np.inf
            a = place[v, at]
            ok = a < R
            h = np.bincount(a[ok], w[ok], R)[:R] * allowed
            d_h = (np.bincount(a[ok], minlength=R)[:R] * half + EPS * np.abs(h)) * allowed
            W, pi = h.sum(), np.exp(lp)
            g[p, v] = np.where(allowed, (h - W * pi) / T, 0)
            d = d_h + pi * (d_h.sum() + 30 * EPS * np.abs(h).sum()) + np.abs(W) * pi * EPS * (4 * np.abs(z) + 44)
            d = (d + EPS * 2 * (np.abs(h) + np.abs(W) * pi) + np.abs(W) * TINY) / T + 4 * EPS * np.abs(g[p, v])
            tol[p, v] = (d + HALF_STEP[dtype] * (np.abs(g[p, v]) + d) + HALF_TINY[dtype]) * allowed
    return g, tol


# One scenario a policy, all rows at once (torch, 64 bits, on the logits' device).


def sample_each(x, u, settings):
    """int64 [n_ops, n_pol] from float64 x [n_pol, n_ops, n_res], u [n_ops, n_pol]."""
    T, k, p, m = (settings[:, i, None, None] for i in range(4))
    bad = (x.isnan() | (x == float("inf"))).any(-1) | (x == -float("inf")).all(-1)
    bad |= ~((T >= 0) & (T < float("inf")) & (k >= 0) & (p >= 0) & (p <= 1) & (m >= 0) & (m <= 1))[..., 0]
    one = (T == 0) | (p == 0)
    k = k.floor().masked_fill(k < 1, x.shape[-1]).masked_fill(one, 1)
    p = p.masked_fill(one, 1)
    T = T.masked_fill(T == 0, 1)
    x = x + 0.0  # -0 and 0 are the same logit
    s, order = x.sort(dim=-1, descending=True, stable=True)
    w = ((s - s[..., :1]) / T).exp()
    at = torch.arange(x.shape[-1], device=x.device)
    keep = (s > -float("inf")) & (at < k)
    c = (w * keep).cumsum(-1)
    before = torch.cat([torch.zeros_like(c[..., :1]), c[..., :-1]], -1)
    keep &= (before < p * c[..., -1:]) | (p >= 1) | (at == 0)
    keep &= (w >= m) | (at == 0)
    kept = torch.zeros_like(w).scatter_(-1, order, w * keep)
    c = kept.cumsum(-1)
    u = u.T[..., None]
    place = (c <= u.clamp(min=0) * c[..., -1:]).sum(-1)
    place = torch.minimum(place, torch.where(kept > 0, at, 0).amax(-1))
    return place.masked_fill(bad | u[..., 0].isnan(), NO_PLACE).T


def learn_each(x, place, weight, T, dtype):
    """(logp [n_pol], bound, grad, bound) from float64 x, int64 place [n_ops,
    n_pol], float64 weight [n_pol] and T [n_pol]; bounds as logp's and grad's."""
    z = (x - x.amax(-1, keepdim=True)) / T[:, None, None]
    allowed = x > -float("inf")
    lse = z.exp().sum(-1, keepdim=True).log()
    lp = z - lse
    at = place.T[..., None]
    there = at < x.shape[-1]
    at = at.clamp(max=x.shape[-1] - 1)
    t = torch.where(there, lp.gather(-1, at), -float("inf"))[..., 0]
    za = torch.where(allowed, z.abs(), 0)
    off = EPS * (33 * t.abs() + 4 * za.gather(-1, at)[..., 0] + 40)
    w = weight[:, None, None]
    h = torch.zeros_like(x).scatter_(-1, at, w * there) * allowed
    W, pi, T = h.sum(-1, keepdim=True), lp.exp(), T[:, None, None]
    g = torch.where(allowed, (h - W * pi) / T, 0)
    d = EPS * (h.abs() + 31 * pi * W.abs() + W.abs() * pi * (4 * za + 44) + 2 * (h.abs() + W.abs() * pi)) + W.abs() * TINY
    d = d / T + 4 * EPS * g.abs()
    return t.sum(-1), off.sum(-1), g, d + HALF_STEP[dtype] * (g.abs() + d) + HALF_TINY[dtype]
