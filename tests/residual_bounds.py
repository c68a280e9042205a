"""The residual step and its gradient in 64 bits with what each element's error is counted against, built from the terms that
enter that element: one degree at a time, apart from tests/residual_ref.py, and with terms that can be left out, so that
a test of the bounds can show that they notice it.

u = 2^-24.  S = 2^-15 = 512 u is what a sum may be off by, of the sum of its terms' magnitudes: a lane adds at most some 300 of
them in sequence (400 of a weight's gradient), a tree of at most 20 steps and a few roundings of each term follow.  A
sum of a channel's K coefficients may be one sequence: S + K u.  First order throughout; S^2 and the like is below the
tenth that 1.1 adds.

Gradient, r, a and the statistics being given:
  xh2, xh1, g2, P = scale w1: 2 u of themselves;  sigmoid: 8 u of itself (an exponential, a sum, a quotient);
  D = dr + r2 (g2 - xh2 along - mean): eD = S MD,  MD = |dr| + r2 (|g2| + |xh2| mean|g2 xh2| + mean|g2|), the means' own
      errors among it;
  g1 = D sig P: 1.1 S Mu,  Mu = MD sig |P|  (|D| <= MD);
  its means: 2.2 S mean(Mu |xh1|) and 2.2 S mean(Mu): the terms' errors and the sum's;
  da = r1 (g1 - xh1 along1 - mean1): 2.3 S r1 (Mu + |xh1| mean(Mu |xh1|) + mean(Mu));
  dgate = sig' sum_k D s t: (2.2 S + K u) sig' sum_k MD |s| Mt,  Mt = |xh1 w1| + |b1|;
  sums over the rows: 2.2 S of the sums of MD sig |xh1| and MD sig;  of |dh xh2| and |dh|: 1.1 S.
Step, from x, a and the gate:
  mean1: S mean|a|;  size: 1.1 S of itself (the squares' sum S / 2, the mean's error squared);
  t: et = 1.2 S (|w1| (r1 mean|a| [l = 0] + |xh1|) + |b1| / 16),  r: er = |s| sig et + 32 u (|x| + |s| sig Mt);
  mean2: em = mean(er) + S mean|r|;  1 / size: rel = 1.1 (r2^2 mean(|r - mean| (er + em)) + S);
  h: |w2| (r2 (er + em [l = 0]) + |xh2| rel) + 8 u |b2|, times 1.1.
"""
import torch

U, S = 2.0 ** -24, 2.0 ** -15
TERMS = ("along2", "mean2", "along1", "mean1", "shift", "scale", "w1", "w2", "sig", "slope", "r2", "r1", "dr")


def degrees(L):
    return [slice(l * l, (l + 1) ** 2) for l in range(L + 1)]


def _filled(L, C, like, scale, w1, b1, w2, b2):
    ones, zeros = torch.ones(L + 1, C, dtype=like.dtype, device=like.device), torch.zeros(C, dtype=like.dtype, device=like.device)
    return [o if t is None else t for t, o in ((scale, ones), (w1, ones), (b1, zeros), (w2, ones), (b2, zeros))]


def _mean(t):
    return t.mean((1, 2), keepdim=True)


def backward(r, a, L, stats, dh, dr, gate, scale, w1, b1, w2, b2, post, without=()):
    """(gradients, bounds) on float64 tensors.  without: terms that are left out, of TERMS."""
    N, C, K = r.shape
    scale, w1, b1, w2, _ = _filled(L, C, r, scale, w1, b1, w2, b2)
    has = lambda n: 0.0 if n in without else 1.0  # noqa: E731
    keep = lambda n, t: torch.ones_like(t) if n in without else t  # noqa: E731
    s, w1g, w2g = keep("scale", scale), keep("w1", w1), keep("w2", w2)
    sig = torch.ones(N, C, dtype=r.dtype, device=r.device) if gate is None else torch.special.expit(gate)
    slope = keep("slope", sig * (1.0 - sig))
    sig = keep("sig", sig)[..., None]
    dr = torch.zeros_like(r) if dr is None else dr * has("dr")
    mean1, rstd1, mean2, rstd2 = stats
    g = {n: torch.zeros_like(r) for n in ("dx", "da")}
    e = {n: torch.zeros_like(r) for n in ("dx", "da")}
    for n in ("dscale", "dw_post", "dw_pre"):
        g[n], e[n] = torch.zeros_like(scale), torch.zeros_like(scale)
    sum_t, sum_e = torch.zeros_like(r[..., 0]), torch.zeros_like(r[..., 0])
    for l, k in enumerate(degrees(L)):
        zero = 1.0 if l == 0 else 0.0
        row = lambda t: t[:, l][:, None, None]  # noqa: E731
        r2 = row(keep("r2", rstd2))
        xh2 = (r[..., k] - zero * mean2[:, None, None]) * row(rstd2)
        d = dh[..., k]
        g2 = d * w2g[l][None, :, None]
        D = dr[..., k] + r2 * (g2 - has("along2") * xh2 * _mean(g2 * xh2) - has("mean2") * zero * _mean(g2))
        MD = dr[..., k].abs() + r2 * (g2.abs() + xh2.abs() * _mean((g2 * xh2).abs()) + zero * _mean(g2.abs()))
        g["dx"][..., k], e["dx"][..., k] = D, S * MD
        g["dw_pre"][l], e["dw_pre"][l] = (d * xh2).sum((0, 2)), 1.1 * S * (d * xh2).abs().sum((0, 2))
        xh1 = (a[..., k] - zero * mean1[:, None, None]) * row(rstd1) if post else a[..., k]
        w, b = (w1g[l][None, :, None], zero * b1[None, :, None]) if post else (1.0, 0.0)
        t, Mt = xh1 * w + has("shift") * b, (xh1 * w).abs() + (b.abs() if post else 0.0)
        sl = s[l][None, :, None]
        sum_t += (D * sl * t).sum(2)
        sum_e += (MD * sl.abs() * Mt).sum(2)
        g1, Mu = D * sig * sl * w, MD * sig * (sl * w).abs()
        if post:
            r1 = row(keep("r1", rstd1))
            g["da"][..., k] = r1 * (g1 - has("along1") * xh1 * _mean(g1 * xh1) - has("mean1") * zero * _mean(g1))
            e["da"][..., k] = 2.3 * S * r1 * (Mu + xh1.abs() * _mean(Mu * xh1.abs()) + zero * _mean(Mu))
        else:
            g["da"][..., k], e["da"][..., k] = g1, 1.1 * S * Mu
        g["dscale"][l] = (D * sig * t).sum((0, 2))
        e["dscale"][l] = 2.2 * S * (MD * sig * Mt).sum((0, 2))
        if post:
            g["dw_post"][l] = (D * sig * sl * xh1).sum((0, 2))
            e["dw_post"][l] = 2.2 * S * (MD * sig * sl.abs() * xh1.abs()).sum((0, 2))
        if l == 0:
            g["db_post"], e["db_post"] = (D * sig * sl).sum((0, 2)), 2.2 * S * (MD * sig * sl.abs()).sum((0, 2))
            g["db_pre"], e["db_pre"] = d.sum((0, 2)), 1.1 * S * d.abs().sum((0, 2))
    g["dgate"], e["dgate"] = slope * sum_t, slope * (2.2 * S + K * U) * sum_e
    return g, e


def forward(x, a, L, gate, scale, w1, b1, w2, b2, post, eps=1e-5):
    """(results, bounds): r, h and the statistics by name."""
    N, C, K = x.shape
    scale, w1, b1, w2, b2 = _filled(L, C, x, scale, w1, b1, w2, b2)
    sig = (torch.ones(N, C, dtype=x.dtype, device=x.device) if gate is None else torch.special.expit(gate))[..., None]
    v = {"r": torch.zeros_like(x), "h": torch.zeros_like(x)}
    e = {"r": torch.zeros_like(x), "h": torch.zeros_like(x)}
    for n in ("post", "pre") if post else ("pre",):
        for d in (v, e):
            d["rstd_" + n] = torch.zeros(N, L + 1, dtype=x.dtype, device=x.device)
    for l, k in enumerate(degrees(L)):
        zero = 1.0 if l == 0 else 0.0
        t = a[..., k]
        if post:
            m = zero * _mean(t)
            r1 = 1.0 / torch.sqrt(_mean((t - m).square()) + eps)
            xh1, M = (t - m) * r1, zero * _mean(t.abs())
            if l == 0:
                v["mean_post"], e["mean_post"] = m[:, 0, 0], S * M[:, 0, 0]
            v["rstd_post"][:, l], e["rstd_post"][:, l] = r1[:, 0, 0], 1.1 * S * r1[:, 0, 0]
            w, b = w1[l][None, :, None], zero * b1[None, :, None]
            t, Mt = xh1 * w + b, (xh1 * w).abs() + b.abs()
            et = 1.2 * S * (w.abs() * (r1 * M + xh1.abs()) + b.abs() / 16)
        else:
            Mt, et = t.abs(), torch.zeros_like(t)
        so = scale[l][None, :, None] * sig
        r = x[..., k] + so * t
        er = so.abs() * et + 32 * U * (x[..., k].abs() + so.abs() * Mt)
        v["r"][..., k], e["r"][..., k] = r, er
        m, em = zero * _mean(r), zero * (_mean(er) + S * _mean(r.abs()))
        r2 = 1.0 / torch.sqrt(_mean((r - m).square()) + eps)
        xh2 = (r - m) * r2
        rel = 1.1 * (r2.square() * _mean((r - m).abs() * (er + em)) + S)
        if l == 0:
            v["mean_pre"], e["mean_pre"] = m[:, 0, 0], em[:, 0, 0]
        v["rstd_pre"][:, l], e["rstd_pre"][:, l] = r2[:, 0, 0], (r2 * rel)[:, 0, 0]
        w, b = w2[l][None, :, None], zero * b2[None, :, None]
        v["h"][..., k] = xh2 * w + b
        e["h"][..., k] = 1.1 * (w.abs() * (r2 * (er + em) + xh2.abs() * rel) + 8 * U * b.abs())
    return v, e
