"""Plain 64-bit form of the attention with a bias by distance and of its gradient, for its tests: segment by segment and
head by head; buckets from their edges, found in Python / numpy numbers."""
import math
import struct

import numpy as np
import torch

from layers_ref import keep_attention, threshold


def number(x):
    """Place of a positive fp32 number among them all."""
    return struct.unpack("<I", struct.pack("<f", x))[0]


def value(n):
    return struct.unpack("<f", struct.pack("<I", n))[0]


def edges(buckets, r0sq, per_octave):
    """First squared distances of buckets 1 .. buckets - 1."""
    first = number(r0sq)
    return [value(first + i * (1 << 23) // per_octave) for i in range(buckets - 1)]


def squared_distances(a, b):
    """[len(a), len(b)] of numpy fp32 positions: fp32 differences, one rounding to fp32 for dx^2 and for each sum."""
    with np.errstate(over="ignore", invalid="ignore"):
        d = (a[:, None, :] - b[None, :, :]).astype(np.float32).astype(np.float64)
        s = (d[..., 0] * d[..., 0]).astype(np.float32).astype(np.float64)
        s = (d[..., 1] * d[..., 1] + s).astype(np.float32).astype(np.float64)
        return (d[..., 2] * d[..., 2] + s).astype(np.float32)


def bucket_of(a, b, buckets, r0sq, per_octave):
    d2 = squared_distances(a, b)
    e = np.array(edges(buckets, r0sq, per_octave), dtype=np.float32)
    return np.where(np.isnan(d2), buckets - 1, np.searchsorted(e, np.nan_to_num(d2, nan=0.0, posinf=np.inf), side="right"))


def attention(q, k, v, bias, q_pos, k_pos, r0sq, per_octave, scale, qseg, kseg, mask, p, rng, max_q, max_k, grad=None):
    """q [Tq, H, d], k, v [Tk, Hk, d], bias [H, buckets] float64, positions fp32.  Without grad: o, lse and the sums
    P |v|.  grad = (do, o, lse): for dq, dk, dv, dbias each (value, what a rounding of P or dS is counted against, what an
    fp32 error of P or dP is counted against)."""
    H, Hk, nb = q.shape[1], k.shape[1], bias.shape[1]
    G, dev = H // Hk, q.device
    o, lse, size = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=q.dtype, device=dev), torch.zeros_like(q)
    out = {n: [torch.zeros_like(t) for _ in range(3)] for n, t in (("dq", q), ("dk", k), ("dv", v), ("dbias", bias))}
    qp, kp = q_pos.cpu().numpy(), k_pos.cpu().numpy()
    for b, ((q0, q1), (k0, k1)) in enumerate(zip(qseg, kseg)):
        there = torch.ones(k1 - k0, dtype=torch.bool, device=dev) if mask is None else mask[k0:k1].bool()
        keys = torch.arange(k0, k1, device=dev)[there]
        if q1 == q0 or len(keys) == 0:
            continue
        bucket = torch.from_numpy(bucket_of(qp[q0:q1], kp[keys.cpu().numpy()], nb, r0sq, per_octave)).to(dev)
        for h in range(H):
            kk, vv, qq = k[keys, h // G], v[keys, h // G], q[q0:q1, h]
            s = qq @ kk.T * scale + bias[h][bucket]
            m = torch.ones_like(s)
            if p:
                full = keep_attention(b, h // G, q1 - q0, k1 - k0, max_q, max_k, G, Hk, p, *rng)[h % G::G]
                m = torch.from_numpy(full).to(dev)[:, there].double() * (65536.0 / (65536 - threshold(p)))
            if grad is None:
                pr = torch.nan_to_num(torch.softmax(s, 1), nan=0.0) * m
                o[q0:q1, h], size[q0:q1, h], lse[q0:q1, h] = pr @ vv, pr @ vv.abs(), torch.logsumexp(s, 1)
                continue
            do, og, lg = (t[q0:q1, h] for t in grad)
            pr = torch.where((lg == -math.inf)[:, None], 0.0, torch.exp(s - lg[:, None]))
            ds = pr * ((do @ vv.T) * m - (do * og).sum(1, keepdim=True))
            e32 = pr * ((do.abs() @ vv.abs().T) * m + (do * og).abs().sum(1, keepdim=True))
            for i, t in enumerate((ds, ds.abs(), e32)):
                a = (lambda x: x) if i == 0 else torch.abs
                c = scale if i == 0 else abs(scale)
                out["dq"][i][q0:q1, h] = t @ a(kk) * c
                out["dk"][i][keys, h // G] += t.T @ a(qq) * c
                out["dv"][i][keys, h // G] += (pr * m).T @ a(do)
                out["dbias"][i][h] += torch.bincount(bucket.reshape(-1), t.reshape(-1), nb)
    return (o, lse, size) if grad is None else out
