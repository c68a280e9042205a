"""The layers around the product on the CPU: refusals of the C entries (made-up
pointers: every argument is checked before the first HIP call) and of the
Python binding, the sizes of their work memory, and the reference generator
against the published known answers of Philox4x32-10."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layers_ref as R  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
OK, INVALID, UNSUPPORTED = gtp.GTP_OK, gtp.GTP_ERR_INVALID_ARG, gtp.GTP_ERR_UNSUPPORTED
GB = 1 << 30


def at(i):
    """A made-up device address: the i-th GiB."""
    return (100 + i) * GB


def test_philox_known_answers():
    """The Random123 distribution's answers for zeros, ones and digits of pi."""
    for ctr, key, want in (
            ((0, 0, 0, 0), (0, 0), "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
            ((0xffffffff,) * 4, (0xffffffff,) * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
             "d16cfe09 94fdcceb 5001e420 24126ea1")):
        index = ctr[0] | ctr[1] << 32
        got = R.philox(np.array([index], dtype=np.uint64), key[0] | key[1] << 32, ctr[2] | ctr[3] << 32)
        assert [int(w[0]) for w in got] == [int(h, 16) for h in want.split()]


# ------------------------------------------------------------------ normalisation and dropout

def norm(L=2, x=at(0), dtype=0, w=at(1), b=at(2), eps=1e-5, N=10, C=8, y=at(3), mean=at(4), rstd=at(5)):
    return gtp.lib().gtp_layer_norm(L, x, dtype, w, b, eps, N, C, y, mean, rstd, None)


def norm_back(L=2, x=at(0), dtype=0, w=at(1), mean=at(2), rstd=at(3), dy=at(4), N=10, C=8, dx=at(5), dw=at(6), db=at(7),
              work=at(8), nbytes=1 << 26):
    return gtp.lib().gtp_layer_norm_backward(L, x, dtype, w, mean, rstd, dy, N, C, dx, dw, db, work, nbytes, None)


def test_norm_refusals():
    for bad in (dict(L=-1), dict(L=65), dict(dtype=2), dict(N=-1), dict(C=-1), dict(x=None), dict(y=None), dict(eps=0.0),
                dict(eps=math.nan), dict(eps=-1.0), dict(eps=math.inf), dict(N=1 << 62), dict(x=at(0) + 2), dict(y=at(3) + 1),
                dict(w=at(1) + 2), dict(y=at(0) + 16), dict(mean=at(0)), dict(rstd=at(3)), dict(mean=at(5)), dict(y=at(1))):
        assert norm(**bad) == INVALID, bad
        assert gtp.lib().gtp_last_error()
    assert norm(N=1 << 31, C=1, L=0, x=at(0), y=at(100)) == UNSUPPORTED
    assert norm(N=1, C=1 << 31, L=0, x=at(0), y=at(100), w=None, b=None) == UNSUPPORTED
    assert norm(N=0, x=None, y=None) == OK and norm(C=0, x=None, y=None) == OK


def test_norm_backward_refusals():
    for bad in (dict(L=65), dict(dtype=7), dict(x=None), dict(dy=None), dict(mean=None), dict(rstd=None), dict(work=None),
                dict(nbytes=15), dict(work=at(8) + 4), dict(dx=at(0)), dict(dw=at(1)), dict(db=at(6)), dict(work=at(0)),
                dict(dw=at(6) + 2), dict(dx=at(4) + 4)):
        assert norm_back(**bad) == INVALID, bad
    assert norm_back(dx=None, dw=None, db=None) == OK
    assert norm_back(C=0) == OK
    w = gtp.lib().gtp_layer_norm_backward_work
    assert w(2, 0, -1, 8) == -1 and w(65, 0, 1, 1) == -1 and w(2, 5, 1, 1) == -1 and w(2, 0, 0, 8) == 0
    assert w(2, 0, 10, 8) >= 4 * 4 * 8


def drop(x=at(0), res=at(1), dtype=0, p=0.1, rng=at(2), groups=100, K=9, y=at(3)):
    return gtp.lib().gtp_dropout(x, res, dtype, p, rng, groups, K, y, None)


def test_dropout_refusals():
    for bad in (dict(p=-0.1), dict(p=1.0), dict(p=math.nan), dict(dtype=3), dict(x=None), dict(y=None), dict(rng=None),
                dict(groups=-1), dict(K=-1), dict(groups=1 << 62, K=4), dict(x=at(0) + 1), dict(rng=at(2) + 4),
                dict(y=at(0) + 4), dict(y=at(1) + 400), dict(y=at(2))):
        assert drop(**bad) == INVALID, bad
    assert drop(groups=0, x=None, y=None) == OK


# ------------------------------------------------------------------ attention

def attn_desc(**more):
    d = dict(dtype=0, H=4, Hk=2, d=64, B=2, Tq=100, Tk=200, max_q=60, max_k=120, q_off=at(20), k_off=at(21),
             key_mask=None, scale=0.125, p=0.0, rng=None)
    d.update(more)
    return gtp._Attn(*(d[n] for n, _ in gtp._Attn._fields_))


def rows(i, heads, d=64, **more):
    r = dict(data=at(i), row=heads * d, head=d)
    r.update(more)
    return gtp._Rows(r["data"], r["row"], r["head"])


def fwd(desc=None, q=None, k=None, v=None, o=None, lse=at(5), work=at(6), nbytes=1 << 40, **more):
    desc = desc or attn_desc(**more)
    q, k, v, o = q or rows(0, 4), k or rows(1, 2), v or rows(2, 2), o or rows(3, 4)
    return gtp.lib().gtp_attention(ctypes.byref(desc), ctypes.byref(q), ctypes.byref(k), ctypes.byref(v),
                                   ctypes.byref(o), lse, work, nbytes, None)


def bwd(desc=None, lse=at(5), work=at(6), nbytes=1 << 40, dq="", dk="", dv="", **more):
    desc = desc or attn_desc(**more)
    ins = [rows(0, 4), rows(1, 2), rows(2, 2), rows(3, 4), rows(4, 4)]
    outs = [g if g != "" else r for g, r in ((dq, rows(7, 4)), (dk, rows(8, 2)), (dv, rows(9, 2)))]
    return gtp.lib().gtp_attention_backward(ctypes.byref(desc), *map(ctypes.byref, ins), lse,
                                            *(None if r is None else ctypes.byref(r) for r in outs), work, nbytes, None)


BAD_DESC = [dict(dtype=2), dict(H=0), dict(Hk=0), dict(H=3), dict(d=0), dict(B=-1), dict(Tq=-1), dict(max_q=101),
            dict(max_k=201), dict(scale=math.nan), dict(scale=math.inf), dict(p=1.0), dict(p=-1e-3), dict(p=math.nan),
            dict(p=0.5), dict(p=0.5, rng=at(30) + 4), dict(q_off=None), dict(k_off=None), dict(q_off=at(20) + 4),
            dict(Tq=1 << 60)]


@pytest.mark.parametrize("bad", BAD_DESC)
def test_attention_refuses_descriptions(bad):
    assert fwd(**bad) == INVALID and bwd(**bad) == INVALID
    assert gtp.lib().gtp_attention_work(ctypes.byref(attn_desc(**bad)), 0) == -1
    assert gtp.lib().gtp_attention_work(ctypes.byref(attn_desc(**bad)), 1) == -1


def test_attention_refusals():
    assert fwd(d=257) == UNSUPPORTED and bwd(d=257) == UNSUPPORTED
    assert fwd(B=1 << 30, Tq=1 << 30, max_q=1 << 28) == UNSUPPORTED
    assert gtp.lib().gtp_attention(None, None, None, None, None, None, None, 0, None) == INVALID
    assert fwd(lse=None) == INVALID and fwd(lse=at(5) + 2) == INVALID and fwd(lse=at(0)) == INVALID
    assert fwd(lse=at(3)) == INVALID and fwd(lse=at(20)) == INVALID
    for bad in (dict(q=rows(0, 4, data=None)), dict(q=rows(0, 4, data=at(0) + 2)), dict(k=rows(1, 2, row=-64)),
                dict(v=rows(2, 2, head=1 << 61, row=1 << 61)), dict(o=rows(3, 4, row=0)), dict(o=rows(3, 4, head=32)),
                dict(o=rows(0, 4)), dict(o=rows(1, 4)), dict(o=rows(3, 4, data=at(20) - 1024))):
        assert fwd(**bad) == INVALID, bad
    assert bwd(lse=None) == INVALID and bwd(work=None) == INVALID and bwd(nbytes=0) == INVALID
    assert bwd(work=at(6) + 8) == INVALID and bwd(work=at(0)) == INVALID and bwd(work=at(7)) == INVALID
    assert bwd(dk=None) == INVALID and bwd(dv=None) == INVALID
    assert bwd(dq=rows(0, 4)) == INVALID and bwd(dk=rows(9, 2)) == INVALID and bwd(dv=rows(4, 2)) == INVALID
    assert bwd(dq=None, dk=None, dv=None) == OK
    # nothing to do: no launch
    assert fwd(B=0, Tq=0, Tk=0, max_q=0, max_k=0) == OK


def test_attention_slices_of_a_packed_tensor_do_not_overlap():
    """q, k, v of one [T, 3, 4, 64] tensor and the gradients of another are told from real overlaps."""
    T, n = 100, 3 * 4 * 64
    desc = dict(H=4, Hk=4, Tq=T, Tk=T, max_q=60, max_k=60)
    q, k, v = (rows(0, 4, data=at(0) + 4 * i * 256, row=n, head=64) for i in range(3))
    assert fwd(q=q, k=k, v=v, o=rows(0, 4, data=at(0) + 4 * 255, row=n, head=64), **desc) == INVALID
    dq, dk = (rows(0, 4, data=at(40) + 4 * i * 256, row=n, head=64) for i in range(2))
    assert bwd(dq=dq, dk=dk, dv=rows(0, 4, data=at(40) + 4 * 300, row=n, head=64), **desc) == INVALID
    msg = gtp.lib().gtp_last_error().decode()
    assert "two outputs overlap" in msg


def test_attention_work_grows_with_rows():
    w = gtp.lib().gtp_attention_work
    assert w(ctypes.byref(attn_desc()), 1) >= 100 * 4 * 4
    assert w(ctypes.byref(attn_desc()), 0) >= 0


# ------------------------------------------------------------------ the binding

def z(*shape, dtype=F32):
    return torch.zeros(shape, dtype=dtype)


def test_binding_norm():
    x = z(4, 8, 9)
    with pytest.raises(ValueError, match="x must be"):
        gtp.gtp_layer_norm(z(4, 8, 8), 2)
    with pytest.raises(ValueError, match="w has shape"):
        gtp.gtp_layer_norm(x, 2, z(2, 8))
    with pytest.raises(ValueError, match="b has shape"):
        gtp.gtp_layer_norm(x, 2, None, z(9))
    with pytest.raises(TypeError):
        gtp.gtp_layer_norm(x.double(), 2)
    with pytest.raises(TypeError, match="y has dtype"):
        gtp.gtp_layer_norm(x, 2, y=z(4, 8, 9, dtype=BF16))
    with pytest.raises(ValueError, match="contiguous"):
        gtp.gtp_layer_norm(z(8, 4, 9).transpose(0, 1), 2)
    with pytest.raises(ValueError, match="device tensor"):
        gtp.gtp_layer_norm(x, 2)
    with pytest.raises(TypeError, match="dy has dtype"):
        gtp.gtp_layer_norm_backward(x, z(4, 8, 9, dtype=BF16), 2, z(4), z(4, 3))
    with pytest.raises(ValueError, match="rstd has shape"):
        gtp.gtp_layer_norm_backward(x, x, 2, z(4), z(4, 2))
    with pytest.raises(ValueError, match="unknown gradients"):
        gtp.gtp_layer_norm_backward(x, x, 2, z(4), z(4, 3), need=("dy",))
    with pytest.raises(ValueError, match="device tensor"):
        gtp.gtp_layer_norm_backward(x, x, 2, z(4), z(4, 3))


def test_binding_dropout():
    x, rng = z(4, 8, 9), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError, match="rng has shape"):
        gtp.gtp_dropout(x, 0.1, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(TypeError, match="rng has dtype"):
        gtp.gtp_dropout(x, 0.1, z(2))
    with pytest.raises(ValueError, match="res has shape"):
        gtp.gtp_dropout(x, 0.1, rng, res=z(4, 8, 8))
    with pytest.raises(TypeError, match="res has dtype"):
        gtp.gtp_dropout(x, 0.1, rng, res=z(4, 8, 9, dtype=BF16))
    with pytest.raises(ValueError, match="device tensor"):
        gtp.gtp_dropout(x, 0.1, rng)


def test_binding_attention():
    q, k = z(6, 4, 16), z(9, 2, 16)
    off = torch.tensor([0, 3, 6])
    with pytest.raises(ValueError, match="multiple"):
        gtp.gtp_attention(z(6, 3, 16), k, k)
    with pytest.raises(ValueError, match="k has shape"):
        gtp.gtp_attention(q, z(9, 2, 8), z(9, 2, 8))
    with pytest.raises(ValueError, match="v has shape"):
        gtp.gtp_attention(q, k, z(8, 2, 16))
    with pytest.raises(TypeError, match="k has dtype"):
        gtp.gtp_attention(q, k.bfloat16(), k)
    with pytest.raises(TypeError):
        gtp.gtp_attention(q.half(), k.half(), k.half())
    with pytest.raises(ValueError, match="one length"):
        gtp.gtp_attention(q, k, k, q_off=off, k_off=torch.tensor([0, 9]))
    with pytest.raises(TypeError, match="q_off has dtype"):
        gtp.gtp_attention(q, k, k, q_off=off.int(), k_off=off)
    with pytest.raises(ValueError, match="key_mask has shape"):
        gtp.gtp_attention(q, k, k, key_mask=torch.zeros(6, dtype=torch.uint8))
    with pytest.raises(ValueError, match="last dimension"):
        gtp.gtp_attention(z(6, 4, 32)[..., ::2], k, k)
    with pytest.raises(ValueError, match="o has shape"):
        gtp.gtp_attention(q, k, k, o=z(6, 4, 8))
    with pytest.raises(ValueError, match="device tensor"):
        gtp.gtp_attention(q, k, k)
    with pytest.raises(ValueError, match="lse has shape"):
        gtp.gtp_attention_backward(q, k, k, q, q, z(4, 6))
    with pytest.raises(ValueError, match="do has shape"):
        gtp.gtp_attention_backward(q, k, k, q, z(6, 2, 16), z(6, 4))
    with pytest.raises(ValueError, match="unknown gradients"):
        gtp.gtp_attention_backward(q, k, k, q, q, z(6, 4), need=("dx",))
    with pytest.raises(ValueError, match="device tensor"):
        gtp.gtp_attention_backward(q, k, k, q, q, z(6, 4))
