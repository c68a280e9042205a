"""The layers around the product on the CPU: sizes that one launch cannot hold are refused before it, layouts of outputs
that do not overlap are not, and the plain 64-bit forms of the GPU tests against autograd."""
import ctypes
import itertools
import math
import random

import pytest

torch = pytest.importorskip("torch")

import layers_ref as R  # noqa: E402
from test_layers_host import INVALID, OK, UNSUPPORTED, at, attn_desc, drop  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402


def test_dropout_refuses_more_than_a_launch_holds():
    far = dict(res=None, rng=at(1 << 20), y=at(2000), dtype=1)
    assert drop(groups=1 << 37, K=1, **far) == UNSUPPORTED
    assert drop(groups=(1 << 37) // 49 + 1, K=49, **far) == UNSUPPORTED
    assert drop(groups=1, K=1 << 31, **far) == UNSUPPORTED


# ------------------------------------------------------------------ outputs' layouts

def backward_into(grads, T, H, d):
    """The attention gradient's checks of (pointer, row, head) outputs, B = 0 segments: nothing is launched."""
    desc = attn_desc(B=0, H=H, Hk=H, d=d, Tq=T, Tk=T, max_q=T, max_k=T, q_off=at(20), k_off=at(21))
    ins = [gtp._Rows(at(i), H * d, d) for i in range(5)]
    outs = [gtp._Rows(*g) for g in grads]
    status = gtp.lib().gtp_attention_backward(ctypes.byref(desc), *map(ctypes.byref, ins), at(5), *map(ctypes.byref, outs),
                                              at(6), 1 << 40, None)
    return status, gtp.lib().gtp_last_error().decode()


@pytest.mark.parametrize("T,H,d", [(100, 4, 64), (1, 4, 64), (100, 1, 64), (1, 1, 9), (33, 12, 7)])
def test_gradients_into_any_slice_of_a_packed_tensor(T, H, d):
    n = T * H * d
    for name, strides, step in (("[T, 3, H, d]", (3 * H * d, d), H * d), ("[T, H, 3, d]", (3 * H * d, 3 * d), d),
                                ("[H, T, 3, d]", (3 * d, 3 * T * d), d), ("[H, 3, T, d]", (d, 3 * T * d), T * d),
                                ("[3, T, H, d]", (H * d, d), n), ("[3, H, T, d]", (d, T * d), n)):
        grads = [(at(40) + 4 * i * step, *strides) for i in range(3)]
        assert backward_into(grads, T, H, d)[0] == OK, name
        grads[2] = (grads[1][0] + 4 * (d - 1), *strides)
        assert backward_into(grads, T, H, d) == (INVALID, "two outputs overlap"), name


def test_overlaps_are_found_by_their_elements():
    """Random layouts of one pair of strides, each output's own rows apart: refused where an element is shared, and
    only there."""
    r, seen = random.Random(5), [0, 0]
    for _ in range(3000):
        T, H, d = r.randint(1, 5), r.randint(1, 4), r.randint(1, 5)
        inner = d + r.randint(0, 7)
        if r.random() < 0.5:
            head, row = inner, inner * (H - 1) + d + r.randint(0, 30)
        else:
            row, head = inner, inner * (T - 1) + d + r.randint(0, 30)
        move = r.randint(-40, 40)
        own = {t * row + h * head + i for t in range(T) for h in range(H) for i in range(d)}
        shared = bool(own & {e + move for e in own})
        grads = [(at(30), row, head), (at(40), row, head), (at(40) + 4 * move, row, head)]
        status, msg = backward_into(grads, T, H, d)
        assert (status, shared) in ((OK, False), (INVALID, True)), (T, H, d, row, head, move)
        seen[shared] += 1
    assert min(seen) > 300


def test_an_output_is_told_from_any_input():
    """o against keys of another length, whose rows may meet each other (expanded, windows)."""
    r, seen = random.Random(6), [0, 0]
    for _ in range(3000):
        Tq, Tk, H, d = r.choice([1, 1, 3]), r.randint(1, 6), r.randint(1, 3), r.randint(1, 5)
        head = d + r.randint(0, 6)
        row = head * (H - 1) + d + r.randint(0, 9)
        krow = row if Tq > 1 else r.choice([0, 1, d - 1, row, 2 * row])
        move = r.randint(-60, 60)
        o = {t * row + h * head + i for t in range(Tq) for h in range(H) for i in range(d)}
        k = {move + t * krow + h * head + i for t in range(Tk) for h in range(H) for i in range(d)}
        desc = attn_desc(B=0, H=H, Hk=H, d=d, Tq=Tq, Tk=Tk, max_q=Tq, max_k=Tk)
        rows = [gtp._Rows(*t) for t in ((at(0), H * d, d), (at(40) + 4 * move, krow, head), (at(2), H * d, d), (at(40), row, head))]
        status = gtp.lib().gtp_attention(ctypes.byref(desc), *map(ctypes.byref, rows), at(5), at(6), 1 << 40, None)
        shared = bool(o & k)
        assert (status, shared) in ((OK, False), (INVALID, True)), (Tq, Tk, H, d, row, head, krow, move)
        seen[shared] += 1
    assert min(seen) > 300


# ------------------------------------------------------------------ descriptions at the edge of what fits

def test_attention_refuses_a_scale_that_overflows_in_units_of_log_2():
    for scale in (3e38, -2.4e38):
        desc = attn_desc(scale=scale)
        assert gtp.lib().gtp_attention_work(ctypes.byref(desc), 0) == -1
    assert gtp.lib().gtp_attention_work(ctypes.byref(attn_desc(scale=2.3e38)), 0) >= 0


def test_attention_work_size_fits():
    """Expanded keys (a row stride of 0) of any number: the size is right or refused, never wrapped."""
    for shift in range(30, 62):
        desc = attn_desc(B=1, H=1, Hk=1, d=4, Tq=1 << 20, Tk=1 << shift, max_q=1 << 20, max_k=64)
        n = gtp.lib().gtp_attention_work(ctypes.byref(desc), 1)
        assert n == -1 or n >= 4 << 20, shift
        desc = attn_desc(B=1, H=1, Hk=1, d=4, Tq=1 << 20, Tk=1 << shift, max_q=1 << 20, max_k=1)
        few = gtp.lib().gtp_attention_work(ctypes.byref(desc), 1)
        assert (few == -1) == (n == -1) and (few == -1 or few >= (4 << 20) + (32 << shift)), shift


# ------------------------------------------------------------------ the binding

@pytest.mark.parametrize("Tq,Tk,max_q,max_k,B", [
    (0, 12, 0, 12, 1), (0, 12, 0, 4, 3), (0, 12, 0, None, 1), (0, 12, 5, 12, 1), (12, 0, 4, 0, 3), (12, 0, None, 0, 1),
    (0, 0, 0, 0, 1), (0, 0, None, None, 1), (6, 9, 2, None, 3), (6, 9, None, 3, 3), (6, 9, None, None, 1)])
def test_equal_segments_of_no_rows_on_one_side(Tq, Tk, max_q, max_k, B):
    """Without offsets the number of segments comes from the side that has rows."""
    q, k = torch.zeros(Tq, 2, 8), torch.zeros(Tk, 2, 8)
    desc, _ = gtp._attn(q, k, k, None, None, None, max_q, max_k, None, 0.0, None)
    assert desc[4] == B and desc[4] * desc[7] == Tq and desc[4] * desc[8] == Tk
    a = gtp._Attn(*desc)
    assert gtp.lib().gtp_attention_work(ctypes.byref(a), 0) == 0


def test_current_stream_without_the_short_way(monkeypatch):
    """The current stream's handle where torch lacks the function that gives it without an object."""
    class Fake:
        cuda_stream = 77
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Fake())
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.delattr(torch._C, "_cuda_getDevice", raising=False)
    assert gtp._stream().value == 77 and gtp._stream(Fake()).value == 77


# ------------------------------------------------------------------ the plain 64-bit forms against autograd

def randn64(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float64)


@pytest.mark.parametrize("N,C,L", [(1, 1, 0), (5, 7, 0), (4, 1, 1), (3, 6, 2), (2, 3, 5)])
@pytest.mark.parametrize("weights", [True, False])
def test_plain_norm_against_autograd(N, C, L, weights):
    """The forward against one written coefficient by coefficient, the gradient against its derivative."""
    g = torch.Generator().manual_seed(N + C + L)
    x, dy = randn64(g, N, C, (L + 1) ** 2), randn64(g, N, C, (L + 1) ** 2)
    x[..., 0] += 0.5
    w, b = (randn64(g, L + 1, C), randn64(g, C)) if weights else (None, None)
    leaves = [t.requires_grad_() for t in (x, w, b) if t is not None]
    rows = []
    for n in range(N):
        mu = sum(x[n, c, 0] for c in range(C)) / C
        out = []
        for l in range(L + 1):
            a = [[x[n, c, k] - (mu if k == 0 else 0.0) for k in range(l * l, (l + 1) ** 2)] for c in range(C)]
            v = sum(e * e for r in a for e in r) / (C * (2 * l + 1))
            out.append(torch.stack([torch.stack(r) / (v + 1e-5).sqrt() * (1.0 if w is None else w[l, c]) +
                                    (b[c] if b is not None and l == 0 else 0.0) for c, r in enumerate(a)]))
        rows.append(torch.cat(out, 1))
    want = torch.stack(rows)
    y, mean, rstd = R.norm(x.detach(), L, *(None if t is None else t.detach() for t in (w, b)), 1e-5)
    assert torch.allclose(y, want, rtol=1e-12, atol=1e-12)
    grads = torch.autograd.grad((want * dy).sum(), leaves)
    dx, dw, db, sw, sb = R.norm_backward(x.detach(), dy, L, None if w is None else w.detach(), mean, rstd)
    # one channel at degree 0 is its own mean: a gradient of zero, out of terms of rstd = 1 / sqrt(eps)
    size = float(rstd.max())
    assert torch.allclose(dx, grads[0], rtol=1e-10, atol=1e-10 * size)
    if weights:
        assert torch.allclose(dw, grads[1], rtol=1e-10, atol=1e-10) and torch.allclose(db, grads[2], rtol=1e-10, atol=1e-10)
    assert bool((sw >= dw.abs() - 1e-12).all()) and bool((sb >= db.abs() - 1e-12).all())


@pytest.mark.parametrize("H,Hk,masked,p", [(1, 1, 0, 0.0), (4, 2, 0, 0.0), (6, 2, 0.4, 0.0), (4, 4, 0, 0.3), (4, 1, 0.3, 0.2)])
def test_plain_attention_against_autograd(H, Hk, masked, p):
    """One query row at a time, every key of every segment with a factor of 0 or 1 for belonging to it, against the form
    by segments; the gradient against its derivative."""
    g = torch.Generator().manual_seed(H + 10 * Hk)
    ql, kl, d, G = [3, 0, 5, 2], [4, 6, 7, 0], 6, H // Hk
    qo, ko = ([0, *itertools.accumulate(n)] for n in (ql, kl))
    q, k, v = (randn64(g, sum(n), h, d).requires_grad_() for n, h in ((ql, H), (kl, Hk), (kl, Hk)))
    do = randn64(g, sum(ql), H, d)
    mask = (torch.rand(sum(kl), generator=g) >= masked).to(torch.uint8) if masked else None
    rng, scale = (12345, 3), 0.7
    outs, lses = [], []
    for b in range(len(ql)):
        for i in range(ql[b]):
            for h in range(H):
                there = torch.zeros(sum(kl), dtype=torch.bool)
                there[ko[b]:ko[b + 1]] = True
                if mask is not None:
                    there &= mask.bool()
                if not bool(there.any()):
                    outs.append(torch.zeros(d, dtype=torch.float64))
                    lses.append(torch.tensor(-math.inf, dtype=torch.float64))
                    continue
                e = torch.exp((k[:, h // G] * q[qo[b] + i, h]).sum(1) * scale) * there
                keep = torch.ones(sum(kl), dtype=torch.float64)
                if p:
                    full = R.keep_attention(b, h // G, ql[b], kl[b], max(ql), max(kl), G, Hk, p, *rng)
                    keep[ko[b]:ko[b + 1]] = torch.from_numpy(full[i * G + h % G]).double() * 65536 / (65536 - R.threshold(p))
                outs.append((e * keep / e.sum()) @ v[:, h // G])
                lses.append(e.sum().log())
    want, wl = torch.stack(outs).view(sum(ql), H, d), torch.stack(lses).view(sum(ql), H)
    grads = torch.autograd.grad((want * do).sum(), (q, k, v))
    args = (scale, list(zip(qo, qo[1:])), list(zip(ko, ko[1:])), mask, p, rng, max(ql), max(kl))
    t = [x.detach() for x in (q, k, v)]
    o, lse, size = R.attention(*t, *args)
    assert torch.allclose(o, want, rtol=1e-11, atol=1e-12) and torch.equal(torch.isinf(lse), torch.isinf(wl))
    ok = ~torch.isinf(wl)
    assert torch.allclose(lse[ok], wl[ok], rtol=1e-11, atol=1e-12) and bool((size >= o.abs() - 1e-12).all())
    for (got, a, c), e in zip(R.attention(*t, *args, (do, o, lse)), grads):
        assert torch.allclose(got, e, rtol=1e-10, atol=1e-11)
        assert bool((a >= got.abs() - 1e-12).all()) and bool((c >= got.abs() - 1e-12).all())
