"""Plain 64-bit forms of the operators over given arrays (gated scan, token log probabilities, distillation), one step and one row at a
time, each with the bound that fp32 arithmetic and one final rounding leave a kernel.

Bounds, elementwise, u = 2^-24 (half a step of fp32).  Sums and products may be taken in any order:
  * a coefficient is wrong by at most KC u of its parts: the exponential by 2 + 1.2 |g| units in the last place (2 u each; |g| <= 8 in
    the tests: 24 u), tanh by 24 u where it is formed from an exponential, a few roundings;
  * a term of the scan, product of coefficients, by KC u for each factor: with S_t = |a_t| S_{t-1} + |b_t|, the sum of the terms' sizes,
    the error obeys E_t = |a_t| E_{t-1} + KC u S_t, and adding the terms in a tree of at most 32 levels adds 32 u S_t;
  * a result of 16-bit type is rounded once: eps / 2 of it, or half the smallest step."""
import numpy as np
import torch

U = 2.0 ** -24
KC = 64.0
CLASSIC, IMPLICIT, GIVEN = 0, 1, 2


def rounding(ref, dtype):
    fi = torch.finfo(dtype)
    return np.abs(ref) * fi.eps / 2 + fi.smallest_normal * fi.eps / 2


def to64(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy()


def _cell(g, c, cell, dt):
    if cell == GIVEN:
        return g, c, None, None, None
    z, n = 1 / (1 + np.exp(-g)), np.tanh(c)
    r = 1 / (1 + dt * z) if cell == IMPLICIT else np.ones_like(z)
    a = r if cell == IMPLICIT else 1 - dt * z
    return a, dt * z * n * r, z, n, r


def scan_forward(gate, cand, h0, cell, dt, lengths=None, reset=None):
    """-> (h, hT, bound of h before rounding, bound of hT)"""
    T, B, H = gate.shape
    a, b, _, _, _ = _cell(gate, cand, cell, dt)
    h = np.zeros((B, H)) if h0 is None else h0.copy()
    S, E = np.abs(h), np.zeros((B, H))
    out, bound = np.zeros((T, B, H)), np.zeros((T, B, H))
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(T):
            live = np.ones(B, bool) if lengths is None else t < lengths
            fresh = np.zeros(B, bool) if reset is None else reset[t].astype(bool)
            hn = np.where(fresh[:, None], b[t], a[t] * h + b[t])
            Sn = np.where(fresh[:, None], 0, np.abs(a[t]) * S) + np.abs(b[t])
            En = np.where(fresh[:, None], 0, np.abs(a[t]) * E) + KC * U * Sn
            h, S, E = (np.where(live[:, None], x, y) for x, y in ((hn, h), (Sn, S), (En, E)))
            out[t] = np.where(live[:, None], h, 0)
            bound[t] = np.where(live[:, None], E + 32 * U * S, 0)
    return out, h, bound, E + 32 * U * S


def scan_backward(gate, cand, h, h0, seed, dhT, cell, dt, lengths=None, reset=None):
    """-> (dgate, dcand, dh0) and their bounds before rounding"""
    T, B, H = gate.shape
    a, b, z, n, r = _cell(gate, cand, cell, dt)
    mu = np.zeros((B, H)) if dhT is None else dhT.copy()
    S, E = np.abs(mu), np.zeros((B, H))
    dg, dc, bg, bc = (np.zeros((T, B, H)) for _ in range(4))
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(T - 1, -1, -1):
            live = (np.ones(B, bool) if lengths is None else t < lengths)[:, None]
            fresh = (np.zeros(B, bool) if reset is None else reset[t].astype(bool))[:, None]
            sd = 0.0 if seed is None else seed[t]
            lam = mu + sd
            Sl = S + np.abs(sd)
            El = E + 34 * U * Sl
            hp = (np.zeros((B, H)) if h0 is None else h0) if t == 0 else h[t - 1]
            hp = np.where(fresh, 0, hp)
            if cell == GIVEN:
                g_, c_ = lam * hp, lam
                eg, ec = El * np.abs(hp) + 2 * U * Sl * np.abs(hp), El
            else:
                k = dt * r[t] ** 2
                g_, c_ = lam * k * (n[t] - hp) * z[t] * (1 - z[t]), lam * dt * z[t] * r[t] * (1 - n[t] ** 2)
                eg = k * z[t] * (El * np.abs(n[t] - hp) * (1 - z[t]) + KC * U * Sl * (np.abs(n[t]) + np.abs(hp)))
                ec = dt * z[t] * r[t] * (El * (1 - n[t] ** 2) + KC * U * Sl)
            dg[t], dc[t], bg[t], bc[t] = (np.where(live, x, 0) for x in (g_, c_, eg, ec))
            mn, Sn = np.where(fresh, 0, a[t] * lam), np.where(fresh, 0, np.abs(a[t]) * Sl)
            En = np.where(fresh, 0, np.abs(a[t]) * El) + KC * U * Sn
            mu, S, E = (np.where(live, x, y) for x, y in ((mn, mu), (Sn, S), (En, E)))
    return (dg, dc, mu), (bg, bc, E + 32 * U * S)


def _softmax(x):
    """-> (probabilities, log probabilities, log of the sum, |distance of each to the largest|); rows of -inf: 0, -inf, -inf"""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = x.max(1, keepdims=True)
        m0 = np.where(np.isneginf(m), 0, m)
        d = x - m0
        e = np.exp(d)
        s = e.sum(1, keepdims=True)
        lse = m0 + np.log(s)
        p = np.where(s == 0, 0, e / s)
        logp = np.where(np.isneginf(x), -np.inf, d - np.log(s))      # (not x - lse: rows at the type's lowest value would lose log s, in 64 bits too)
        bad = np.isnan(x).any(1, keepdims=True) | np.isposinf(x).any(1, keepdims=True)
        p, logp, lse = (np.where(bad, np.nan, v) for v in (p, logp, lse))
    return p, logp, lse[:, 0], np.where(np.isfinite(d), np.abs(d), 0)


def _rel_sum(p, d, V):
    """Relative error of a row's sum of exponentials: of each term 2 (2 + 1.2 |d|) u and 2 u |d| from its argument, of adding V terms at
    most (V / 256 + 32) u (a thread's own terms one after the other, then a tree)."""
    return U * (2 * (2 + 2.2 * (np.nan_to_num(p) * d).sum(1)) + V / 256 + 32)


def logprobs(x, tokens, top):
    """-> dict of logprob, entropy, lse, top_logprob, top_id and the bounds of the first four"""
    N, V = x.shape
    p, logp, lse, d = _softmax(x)
    with np.errstate(invalid="ignore"):
        ent = np.where(np.isneginf(lse), 0, -np.where(p == 0, 0, p * logp).sum(1))
        has = (tokens >= 0) & (tokens < V)
        t = np.where(has, tokens, 0)
        lp = np.where(has, logp[np.arange(N), t], 0)
        rel = _rel_sum(p, d, V)
        size = np.nan_to_num(np.abs(x).max(1, initial=0, where=np.isfinite(x)))
        blse = rel + U * (2 * np.abs(np.nan_to_num(lse, neginf=0)) + 2 * size)
        wd = (np.nan_to_num(p) * d).sum(1)
        bent = rel * (2 + 2 * wd) + 8 * U * (wd + 1 + np.log(V))
    # falling values, equal ones in rising order of their index; NaN behind -inf
    rank = np.where(np.isnan(x), -np.inf, x)
    order = np.lexsort((np.broadcast_to(np.arange(V), x.shape), np.isnan(x), -rank), axis=1)[:, :top]
    tl = np.take_along_axis(logp, order, 1)
    far = np.nan_to_num(np.abs(lp), posinf=0, neginf=0)
    return dict(logprob=lp, entropy=ent, lse=lse, top_logprob=tl, top_id=order, b_lse=blse, b_entropy=bent,
                b_logprob=np.where(has, blse + 2 * U * far, 0), b_top=blse[:, None] + 2 * U * np.nan_to_num(np.abs(tl), posinf=0, neginf=0))


def logprobs_backward(x, tokens, lse, entropy, dlogprob, dentropy):
    N, V = x.shape
    with np.errstate(invalid="ignore"):
        l = lse[:, None]
        dead = np.isneginf(l)
        logp = np.where(dead, -np.inf, x - l)
        p = np.where(dead, 0, np.exp(logp))
        lp = np.where(p == 0, 0, logp)
        gl = np.zeros(N) if dlogprob is None else np.where((tokens >= 0) & (tokens < V), dlogprob, 0)
        ge, ent = (np.zeros(N), np.zeros(N)) if dentropy is None else (dentropy, entropy)
        inner = gl[:, None] + ge[:, None] * (lp + ent[:, None])
        g = np.where(p == 0, 0, -p * inner)
        if dlogprob is not None:
            for r in range(N):
                if 0 <= tokens[r] < V and not dead[r]:
                    g[r, tokens[r]] += gl[r]
        # the exponential of a rounded difference, then four roundings of the parts
        parts = p * (np.abs(gl)[:, None] + np.abs(ge)[:, None] * (np.abs(lp) + np.abs(ent)[:, None]))
        far = np.abs(np.where(p == 0, 0, x)) + np.abs(np.where(dead, 0, l))
        bound = parts * U * (2 * (2 + 1.2 * np.abs(lp)) + 2 * np.abs(lp) + far + 12) + np.abs(gl)[:, None] * 2 * U * (np.arange(V)[None] == np.asarray(tokens if tokens is not None else np.full(N, -1))[:, None])
    return g, np.nan_to_num(bound)


def distill(x, ids, y, w, tau):
    """-> (loss, row_loss, dlogits) and their bounds before rounding"""
    N, V = x.shape
    K = ids.shape[1]
    with np.errstate(invalid="ignore", divide="ignore"):
        q, logq, _, d = _softmax(x / tau)
        valid = (ids >= 0) & (ids < V)
        yy = np.where(valid, y, -np.inf) / tau
        p, logp, _, dy = _softmax(yy)
        present = (~np.isneginf(yy)).any(1)
        t = np.where(valid, ids, 0)
        lq = np.where(valid, np.take_along_axis(logq, t, 1), 0)
        terms = np.where(p == 0, 0, p * (logp - lq))
        row = np.where(present, tau * tau * terms.sum(1), 0)
        ww = np.full(N, 1.0 / N) if w is None else w
        loss = np.where(ww == 0, 0, ww * row).sum()
        g, pk = q.copy(), np.zeros_like(q)
        for r in range(N):
            np.add.at(pk[r], t[r][valid[r]], p[r][valid[r]])
        g = (ww * tau)[:, None] * (g - pk)
        g[~present | (ww == 0)] = 0
        # x / tau is rounded (u |x / tau|, as 1 / tau and as a product), so is its distance to the largest
        rq = _rel_sum(q, d, V)[:, None] + U * (2 * (2 + 2.2 * d) + 4 * np.abs(np.where(np.isfinite(x), x, 0)).max(1, keepdims=True, initial=0) / tau + 8)
        rp = U * (2 * (2 + 2.2 * dy) + (2 * (2 + 2.2 * (np.nan_to_num(p) * dy).sum(1)) + K / 8 + 32)[:, None] + 4 * np.abs(np.where(np.isfinite(yy), yy, 0)).max(1, keepdims=True, initial=0) + 8)
        bp = np.zeros_like(q)
        for r in range(N):
            np.add.at(bp[r], t[r][valid[r]], np.nan_to_num(p * rp)[r][valid[r]])
        bound_g = np.abs(ww * tau)[:, None] * (np.nan_to_num(q * rq) + bp + 4 * U * (np.nan_to_num(q) + np.nan_to_num(pk)))
        mq = rq.max(1, keepdims=True)
        brow = tau * tau * np.nan_to_num(p * (rp * (np.abs(logp - lq) + 1) + mq + (K / 8 + 16) * U * (np.abs(logp) + np.abs(lq))), posinf=0, neginf=0).sum(1)
        bloss = (np.abs(ww) * (brow + (N / 1024 + 16) * U * np.abs(np.nan_to_num(row, posinf=0)))).sum()
    return (loss, row, g), (bloss, brow, bound_g)


def check(got, ref, bound, name=""):
    """got within the bound of ref, elementwise; NaN and infinities in the same places."""
    got = to64(got) if torch.is_tensor(got) else np.asarray(got, dtype=np.float64)
    ref, bound = np.asarray(ref, dtype=np.float64), np.broadcast_to(bound, np.shape(ref))
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{name}: NaN in other places"
    assert np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)]), f"{name}: infinities in other places"
    err = np.abs(got[fine] - ref[fine])
    over = err - bound[fine]
    assert err.size == 0 or over.max() <= 0, f"{name}: off by {err[over.argmax()]:.3g} where {bound[fine][over.argmax()]:.3g} is allowed ({(over > 0).sum()} of {err.size})"
