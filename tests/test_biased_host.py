"""The attention with a bias by distance on the CPU: refusals of the C entries (made-up pointers) and of the binding, the
buckets' edges, work sizes, and the plain 64-bit form of the GPU tests against autograd."""
import ctypes
import math
import struct

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import biased_ref as R  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402
from test_layers_host import BAD_DESC, at, attn_desc, rows  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
OK, INVALID, UNSUPPORTED = gtp.GTP_OK, gtp.GTP_ERR_INVALID_ARG, gtp.GTP_ERR_UNSUPPORTED


def bias_desc(bias=at(40), q_pos=at(41), k_pos=at(42), r0sq=1.0, buckets=32, per_octave=4):
    return struct.pack("<3Qf2i4x", bias or 0, q_pos or 0, k_pos or 0, r0sq, buckets, per_octave)


def split(more):
    b = {n: more.pop(n) for n in list(more) if n in ("bias", "q_pos", "k_pos", "r0sq", "buckets", "per_octave")}
    return bias_desc(**b), attn_desc(**more)


def fwd(o=None, lse=at(5), work=at(6), nbytes=1 << 40, **more):
    b, a = split(more)
    r = [rows(0, 4), rows(1, 2), rows(2, 2), o or rows(3, 4)]
    return gtp.lib().gtp_attention_biased(ctypes.byref(a), b, *map(ctypes.byref, r), lse, work, nbytes, None)


def bwd(dbias=at(43), lse=at(5), work=at(6), nbytes=1 << 40, dq="", dk="", dv="", **more):
    b, a = split(more)
    ins = [rows(0, 4), rows(1, 2), rows(2, 2), rows(3, 4), rows(4, 4)]
    outs = [g if g != "" else r for g, r in ((dq, rows(7, 4)), (dk, rows(8, 2)), (dv, rows(9, 2)))]
    return gtp.lib().gtp_attention_biased_backward(
        ctypes.byref(a), b, *map(ctypes.byref, ins), lse, *(None if r is None else ctypes.byref(r) for r in outs), dbias,
        work, nbytes, None)


BAD_BIAS = [dict(bias=None), dict(q_pos=None), dict(k_pos=None), dict(r0sq=0.0), dict(r0sq=-1.0), dict(r0sq=math.nan),
            dict(r0sq=math.inf), dict(r0sq=2.0 ** -101), dict(buckets=0), dict(buckets=65), dict(buckets=-1),
            dict(per_octave=0), dict(per_octave=3), dict(per_octave=32), dict(per_octave=-4), dict(bias=at(40) + 2),
            dict(q_pos=at(41) + 1), dict(k_pos=at(42) + 2), dict(r0sq=2.0 ** 125, per_octave=1, buckets=6)]


@pytest.mark.parametrize("bad", BAD_BIAS + BAD_DESC)
def test_bad_descriptions(bad):
    assert fwd(**bad) == INVALID and bwd(**bad) == INVALID
    assert gtp.lib().gtp_last_error()
    b, a = split(dict(bad))
    assert gtp.lib().gtp_attention_biased_work(ctypes.byref(a), b, 0) == -1
    assert gtp.lib().gtp_attention_biased_work(ctypes.byref(a), b, 1) == -1


def test_refusals():
    for bad in (dict(o=rows(0, 4)), dict(o=rows(40, 4)), dict(o=rows(41, 4)), dict(o=rows(42, 4)), dict(lse=at(40)),
                dict(lse=at(42)), dict(lse=None), dict(work=None, Tk=20000, max_k=20000)):
        assert fwd(**bad) == INVALID, bad
    for bad in (dict(work=None), dict(nbytes=16), dict(work=at(40)), dict(work=at(43)), dict(dbias=at(0)), dict(dbias=at(5)),
                dict(dbias=at(7)), dict(dbias=at(40)), dict(dbias=at(41)), dict(dbias=at(43) + 2), dict(dbias=at(6)),
                dict(dk=None), dict(dv=None), dict(dq=rows(41, 4)), dict(dq=rows(42, 4))):
        assert bwd(**bad) == INVALID, bad
    assert bwd(dq=None, dk=None, dv=None, dbias=None) == OK
    lib, a, b = gtp.lib(), attn_desc(), bias_desc()
    assert lib.gtp_attention_biased_work(ctypes.byref(a), None, 0) == -1
    assert lib.gtp_attention_biased(ctypes.byref(a), None, None, None, None, None, None, None, 0, None) == INVALID
    assert lib.gtp_attention_biased_work(None, b, 0) == -1
    # the query heads of a key head have 65 x 64 biases
    assert fwd(H=130, Hk=2, buckets=64) == UNSUPPORTED
    assert fwd(H=514, Hk=2, buckets=1) == UNSUPPORTED
    assert fwd(d=257) == UNSUPPORTED
    assert fwd(B=0, Tq=0, Tk=0, max_q=0, max_k=0, q_pos=None, k_pos=None) == OK


def test_work_holds_what_every_workgroup_leaves():
    """The gradient's work is larger than without a bias by a table for each tile of query rows at least; where the
    buckets are made ahead, both directions' by a byte a pair."""
    lib = gtp.lib()
    for H, Hk, B, n in ((4, 2, 2, 60), (8, 8, 64, 49), (16, 4, 2, 4300), (8, 2, 1, 1)):
        a = attn_desc(H=H, Hk=Hk, B=B, Tq=B * n, Tk=B * n, max_q=n, max_k=n)
        plain = lib.gtp_attention_work(ctypes.byref(a), 1)
        extra = lib.gtp_attention_biased_work(ctypes.byref(a), bias_desc(), 1) - plain
        assert extra >= B * -(-(n * H // Hk) // 128) * H * 32 * 4
        pairs = B * n * n if H >= 4 and n > 256 else 0
        assert extra >= pairs
        more = lib.gtp_attention_biased_work(ctypes.byref(a), bias_desc(), 0) - lib.gtp_attention_work(ctypes.byref(a), 0)
        assert pairs <= more <= 1.1 * pairs


@pytest.mark.parametrize("buckets,r0,per", [(1, 1.0, 4), (2, 1.0, 1), (3, 0.7, 16), (32, 1.3, 4), (64, 2.0 ** -50, 1), (64, 3.7, 8)])
def test_edges(buckets, r0, per):
    got = gtp.gtp_attention_bias_edges(buckets, r0, per)
    assert got == R.edges(buckets, r0 * r0, per)
    assert got == sorted(set(got)) and len(got) == buckets - 1
    for i, e in enumerate(got[:-per]):  # an octave on, twice the distance, where the spacing does not change between
        assert abs(got[i + per] / e - 2.0) <= 1.0 / per + 1e-6
    if buckets > 1:
        assert got[0] == np.float32(r0 * r0)
    for bad in ((0, 1.0, 4), (65, 1.0, 4), (4, 0.0, 4), (4, 1.0, 5), (4, math.nan, 4)):
        with pytest.raises(gtp.GTPError):
            gtp.gtp_attention_bias_edges(*bad)


def test_reference_buckets():
    """By edges and by numbers; on an edge, just below it, at the ends, NaN."""
    r0sq, per, nb = 1.69, 4, 20
    e = R.edges(nb, r0sq, per)
    g = np.random.default_rng(0)
    a, b = (g.standard_normal((40, 3)) * 3).astype(np.float32), (g.standard_normal((50, 3)) * 3).astype(np.float32)
    d2 = R.squared_distances(a, b)
    got = R.bucket_of(a, b, nb, r0sq, per)
    want = np.clip((d2.view(np.int32).astype(np.int64) - R.number(r0sq) >> 23 - 2) + 1, 0, nb - 1)
    assert np.array_equal(got, want) and got.min() == 0 and got.max() == nb - 1
    x = np.zeros((3, 3), dtype=np.float32)
    x[1] = math.nan
    x[2] = math.inf
    assert R.bucket_of(x, np.zeros((1, 3), np.float32), nb, r0sq, per)[:, 0].tolist() == [0, nb - 1, nb - 1]
    assert all(e[i] < e[i + 1] for i in range(nb - 2))


def test_binding_refusals():
    z = lambda *s, dtype=F32: torch.zeros(s, dtype=dtype)  # noqa: E731
    q, k, pos, kpos, bias = z(6, 4, 8), z(5, 2, 8), z(6, 3), z(5, 3), z(4, 16)
    f, b = gtp.gtp_attention_biased, gtp.gtp_attention_biased_backward
    lse = z(6, 4)
    for call, error in (
            (lambda: f(q, k, k, z(3, 16), pos, kpos), ValueError), (lambda: f(q, k, k, z(4), pos, kpos), ValueError),
            (lambda: f(q, k, k, None, pos, kpos), ValueError), (lambda: f(q, k, k, bias.double(), pos, kpos), TypeError),
            (lambda: f(q, k, k, bias, z(5, 3), kpos), ValueError), (lambda: f(q, k, k, bias, pos, z(6, 3)), ValueError),
            (lambda: f(q, k, k, bias, pos), TypeError),  # k_pos left out, as many keys as queries only
            (lambda: f(q, k, k, bias, pos.bfloat16(), kpos), TypeError), (lambda: f(q, k, k, bias, z(6, 4), kpos), ValueError),
            (lambda: f(q, k, k, z(16, 4).T, pos, kpos), ValueError), (lambda: f(q, k, k, bias, pos, kpos), ValueError),
            (lambda: b(q, k, k, bias, pos, kpos, 1.0, 4, q, q, lse, need=("dpos",)), ValueError),
            (lambda: b(q, k, k, bias, pos, kpos, 1.0, 4, q, q, z(6, 3)), ValueError),
            (lambda: b(q, k, k, bias, pos, kpos, 1.0, 4, q, z(6, 4, 7), lse), ValueError),
            (lambda: f(q, k, k, bias, pos, kpos, 1e30), ValueError), (lambda: f(q, k, k, bias, pos, kpos, 1.0, 2.5), ValueError),
            (lambda: b(q, k, k, bias, pos, kpos, 1.0, 4, q, q, lse), ValueError)):  # not device tensors
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("p", [0.0, 0.3])
def test_plain_form_against_autograd(p):
    g = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    q, k, v, bias = n(9, 4, 5), n(11, 2, 5), n(11, 2, 5), n(4, 6)
    bias[:, 5] = -math.inf
    qp, kp = n(9, 3).float() * 2, n(11, 3).float() * 2
    mask = torch.tensor([1, 1, 0, 1, 1, 1, 0, 1, 1, 1, 1])
    more = (1.0, 2, 0.4, [(0, 4), (4, 9)], [(0, 6), (6, 11)], mask, p, (5, 7), 5, 6)
    for t in (q, k, v, bias):
        t.requires_grad_()
    o, lse, _ = R.attention(q.clone(), k, v, bias, qp, kp, *more)
    do = n(9, 4, 5)
    (o * do).sum().backward()
    with torch.no_grad():
        got = R.attention(q, k, v, bias, qp, kp, *more, grad=(do, o, lse))
    for name, t in (("dq", q), ("dk", k), ("dv", v), ("dbias", bias)):
        assert torch.allclose(got[name][0], torch.nan_to_num(t.grad), rtol=1e-8, atol=1e-10), name
