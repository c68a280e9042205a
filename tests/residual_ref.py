"""Plain 64-bit forms of the residual step (x + scale sigmoid(gate) t with the norms around it) and of its gradient, for
their tests: degree by degree, on float64 tensors."""
import torch

from layers_ref import degree_slices


def forward(x, a, L, gate, scale, w_post, b_post, w_pre, b_pre, post, eps=1e-5):
    """r, h, (mean_post, rstd_post, mean_pre, rstd_pre)."""
    r, h = torch.empty_like(x), torch.empty_like(x)
    stats = [[], [], [], []]
    open_ = 1.0 if gate is None else (1.0 / (1.0 + torch.exp(-gate)))[..., None]

    def norm(v, l, w, b, at):
        if l == 0:
            m = v.mean((1, 2))
            stats[at].append(m)
            v = v - m[:, None, None]
        rs = 1.0 / torch.sqrt(v.square().mean((1, 2)) + eps)
        stats[at + 1].append(rs)
        v = v * rs[:, None, None]
        if w is not None:
            v = v * w[l][None, :, None]
        return v + b[None, :, None] if l == 0 and b is not None else v

    for l, k in enumerate(degree_slices(L)):
        t = norm(a[..., k], l, w_post, b_post, 0) if post else a[..., k]
        if scale is not None:
            t = t * scale[l][None, :, None]
        sum_ = x[..., k] + open_ * t
        r[..., k], h[..., k] = sum_, norm(sum_, l, w_pre, b_pre, 2)
    m1, r1, m2, r2 = stats
    return r, h, (m1[0] if post else None, torch.stack(r1, 1) if post else None, m2[0], torch.stack(r2, 1))


def backward(r, a, L, stats, dh, dr, gate, scale, w_post, b_post, w_pre, b_pre, post):
    """The gradients, and for each of them the magnitudes that its errors are counted against: "row" sizes (one number
    a row) of dx, da, dgate; sums of the terms' magnitudes of the weights' gradients, and of the rows' sizes."""
    N, C, K = r.shape
    mean1, rstd1, mean2, rstd2 = stats
    ones = torch.ones(L + 1, C, dtype=r.dtype, device=r.device)
    zeros = torch.zeros(C, dtype=r.dtype, device=r.device)
    s, w1, w2 = (ones if t is None else t for t in (scale, w_post, w_pre))
    b1 = zeros if b_post is None else b_post
    g = torch.ones(N, C, dtype=r.dtype, device=r.device) if gate is None else 1.0 / (1.0 + torch.exp(-gate))
    out = {n: torch.zeros(N, C, K, dtype=r.dtype, device=r.device) for n in ("dx", "da")}
    for n in ("dscale", "dw_post", "dw_pre"):
        out[n] = torch.zeros_like(ones)
    out["dgate"] = torch.zeros(N, C, dtype=r.dtype, device=r.device)
    size = {n: torch.zeros_like(ones) for n in ("dscale", "dw_post", "dw_pre")}

    def big(t):
        return t.abs().amax((1, 2))

    X2 = (big(r) + mean2.abs()) * rstd2.amax(1)
    G2 = big(dh) * w2.abs().max()
    MD = (0.0 if dr is None else big(dr)) + rstd2.amax(1) * G2 * (2 + X2 ** 2)
    X1 = (big(a) + mean1.abs()) * rstd1.amax(1) if post else big(a)
    T = w1.abs().max() * X1 + b1.abs().max() if post else X1
    sm = s.abs().max()
    rows = {"dx": MD, "dgate": K * MD * sm * T, "sum": (MD * T).sum(), "u": MD.sum(),
            "da": MD * sm * (rstd1.amax(1) * w1.abs().max() * (2 + X1 ** 2) if post else 1.0)}

    def back(gg, xh, rs, l):
        d = gg - xh * (gg * xh).mean((1, 2), keepdim=True)
        if l == 0:
            d = d - gg.mean((1, 2), keepdim=True)
        return d * rs[:, l][:, None, None]

    for l, k in enumerate(degree_slices(L)):
        xh2 = (r[..., k] - (mean2[:, None, None] if l == 0 else 0.0)) * rstd2[:, l][:, None, None]
        d = dh[..., k]
        out["dw_pre"][l], size["dw_pre"][l] = (d * xh2).sum((0, 2)), (d * xh2).abs().sum((0, 2))
        D = (0.0 if dr is None else dr[..., k]) + back(d * w2[l][None, :, None], xh2, rstd2, l)
        out["dx"][..., k] = D
        xh1 = a[..., k]
        t = xh1
        if post:
            xh1 = (xh1 - (mean1[:, None, None] if l == 0 else 0.0)) * rstd1[:, l][:, None, None]
            t = xh1 * w1[l][None, :, None] + (b1[None, :, None] if l == 0 else 0.0)
        u = D * g[..., None]
        out["dgate"] += g * (1.0 - g) * (D * s[l][None, :, None] * t).sum(2)
        out["dscale"][l] = (u * t).sum((0, 2))
        size["dscale"][l] = (u * xh1 * w1[l][None, :, None]).abs().sum((0, 2))
        if l == 0:
            size["dscale"][l] += (u * b1[None, :, None]).abs().sum((0, 2))
        us = u * s[l][None, :, None]
        out["dw_post"][l], size["dw_post"][l] = (us * xh1).sum((0, 2)), (us * xh1).abs().sum((0, 2))
        if l == 0:
            out["db_post"], size["db_post"] = us.sum((0, 2)), us.abs().sum((0, 2))
            out["db_pre"], size["db_pre"] = d.sum((0, 2)), d.abs().sum((0, 2))
        out["da"][..., k] = back(us * w1[l][None, :, None], xh1, rstd1, l) if post else us
    return out, rows, size
