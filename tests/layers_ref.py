"""Plain 64-bit forms of the layers around the product (normalisation, dropout,
attention) for their tests: elementary operations on float64 tensors, segment
by segment and head by head, and the generator of the draws in Python integers
/ numpy."""
import math

import numpy as np
import torch


def philox(index, seed, offset):
    """Philox4x32-10: index (array of nonnegative ints), four uint32 arrays."""
    M = np.uint64(0xFFFFFFFF)
    index = np.asarray(index, dtype=np.uint64)
    c = [index & M, index >> np.uint64(32), np.full_like(index, offset & 0xFFFFFFFF),
         np.full_like(index, (offset >> 32) & 0xFFFFFFFF)]
    k = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)  # below 2^64
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & M, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & M]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def draws(call, half, seed, offset):
    """The 16-bit draw `half` of call `call` (arrays of one shape)."""
    w = philox(call, seed, offset)
    half = np.asarray(half)
    word = np.choose(half // 2, w).astype(np.uint64)
    return np.where(half % 2 == 0, word & np.uint64(0xFFFF), word >> np.uint64(16)).astype(np.int64)


def threshold(p):
    return min(65535, int(math.floor(p * 65536 + 0.5)))


def keep_groups(groups, p, seed, offset, first=0):
    g = np.arange(first, first + groups, dtype=np.int64)
    return draws(g // 8, g % 8, seed, offset) >= threshold(p)


def keep_attention(b, hk, nq, nk, max_q, max_k, G, Hk, p, seed, offset):
    """[nq * G, nk] of one segment and key head."""
    R, j = np.arange(nq * G)[:, None], np.arange(nk)[None, :]
    nr, nc = (max_q * G + 3) // 4, (max_k + 3) // 4
    call = 2 * (((b * Hk + hk) * nr + R // 4) * nc + j // 4) + (R // 2) % 2
    return draws(call, (R % 2) * 4 + j % 4, seed, offset) >= threshold(p)


def degree_slices(L):
    return [slice(l * l, (l + 1) ** 2) for l in range(L + 1)]


def norm(x, L, w, b, eps):
    """x, w, b float64 -> y, mean, rstd."""
    y, rstd, mean = torch.empty_like(x), [], x[..., 0].mean(1)
    for l, sl in enumerate(degree_slices(L)):
        a = x[..., sl] - (mean[:, None, None] if l == 0 else 0.0)
        r = 1.0 / torch.sqrt(a.square().mean((1, 2)) + eps)
        rstd.append(r)
        y[..., sl] = a * r[:, None, None] * (1.0 if w is None else w[l][None, :, None])
    if b is not None:
        y[..., 0] += b
    return y, mean, torch.stack(rstd, 1)


def norm_backward(x, dy, L, w, mean, rstd):
    """dx, dw, db and the sums of the magnitudes of dw's and db's terms."""
    C = x.shape[1]
    dx = torch.empty_like(x)
    dw = torch.zeros(L + 1, C, dtype=x.dtype, device=x.device)
    size = torch.zeros_like(dw)
    for l, sl in enumerate(degree_slices(L)):
        r = rstd[:, l][:, None, None]
        xh = (x[..., sl] - (mean[:, None, None] if l == 0 else 0.0)) * r
        d = dy[..., sl]
        g = d if w is None else d * w[l][None, :, None]
        t = g - xh * (g * xh).mean((1, 2), keepdim=True)
        if l == 0:
            t = t - g.mean((1, 2), keepdim=True)
        dx[..., sl] = t * r
        dw[l] = (d * xh).sum((0, 2))
        size[l] = (d * xh).abs().sum((0, 2))
    return dx, dw, dy[..., 0].sum(0), size, dy[..., 0].abs().sum(0)


def segments(off, B, most, total):
    if off is None:
        return [(b * most, (b + 1) * most) for b in range(B)]
    off = [int(i) for i in off]
    return [(off[b], off[b + 1]) for b in range(B)]


def attention(q, k, v, scale, qseg, kseg, mask, p, rng, max_q, max_k, grad=None):
    """q [Tq, H, d], k, v [Tk, Hk, d] float64.  Without grad: o, lse and the bound's sums m P |v|.  grad = (do, o, lse):
    dq, dk, dv and for each two sums of magnitudes: what a rounding of P or dS, and what an fp32 error in P or dP,
    is counted against."""
    H, Hk, d = q.shape[1], k.shape[1], q.shape[2]
    G = H // Hk
    dev = q.device
    o, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=q.dtype, device=dev)
    size = torch.zeros_like(q)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    sizes = [torch.zeros_like(t) for t in (q, k, v) for _ in range(2)]
    for b, ((q0, q1), (k0, k1)) in enumerate(zip(qseg, kseg)):
        keys = torch.arange(k0, k1, device=dev)
        there = torch.ones(k1 - k0, dtype=torch.bool, device=dev) if mask is None else mask[k0:k1].bool()
        keys = keys[there]
        if q1 == q0 or len(keys) == 0:
            continue
        for h in range(H):
            kk, vv, qq = k[keys, h // G], v[keys, h // G], q[q0:q1, h]
            s = qq @ kk.T * scale
            m = torch.ones_like(s)
            if p:
                t = threshold(p)
                full = keep_attention(b, h // G, q1 - q0, k1 - k0, max_q, max_k, G, Hk, p, *rng)[h % G::G]
                m = torch.from_numpy(full).to(dev)[:, there].double() * (65536.0 / (65536 - t))
            if grad is None:
                pr = torch.softmax(s, 1) * m
                o[q0:q1, h] = pr @ vv
                size[q0:q1, h] = pr @ vv.abs()
                lse[q0:q1, h] = torch.logsumexp(s, 1)
                continue
            do, og, lg = (t[q0:q1, h] for t in grad)
            pr = torch.exp(s - lg[:, None])
            delta = (do * og).sum(1, keepdim=True)
            ds = pr * ((do @ vv.T) * m - delta) * scale
            # what an fp32 error in P or dP is counted against
            e32 = pr * ((do.abs() @ vv.abs().T) * m + (do * og).abs().sum(1, keepdim=True)) * abs(scale)
            dq[q0:q1, h] = ds @ kk
            sizes[0][q0:q1, h] = ds.abs() @ kk.abs()
            sizes[1][q0:q1, h] = e32 @ kk.abs()
            dk[keys, h // G] += ds.T @ qq
            sizes[2][keys, h // G] += ds.abs().T @ qq.abs()
            sizes[3][keys, h // G] += e32.T @ qq.abs()
            dv[keys, h // G] += (pr * m).T @ do
            sizes[4][keys, h // G] += (pr * m).T @ do.abs()
            sizes[5][keys, h // G] += (pr * m).T @ do.abs()
    if grad is None:
        return o, lse, size
    return (dq, sizes[0], sizes[1]), (dk, sizes[2], sizes[3]), (dv, sizes[4], sizes[5])
