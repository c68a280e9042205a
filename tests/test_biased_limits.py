"""Limits of the attention with a bias by distance: the work of large segments and arguments out of range (on the CPU);
segments whose buckets are no longer made ahead (-m gpu)."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

import biased_ref as B  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402
from test_biased_host import bias_desc  # noqa: E402
from test_layers_host import at, attn_desc, rows  # noqa: E402


def test_work_stays_bounded_for_large_segments():
    """The buckets made ahead take a byte a pair up to 1 GiB; beyond, the work grows with the rows as without a bias."""
    lib, GiB = gtp.lib(), 1 << 30
    for n, B, H, Hk in ((16384, 1, 8, 8), (32768, 1, 8, 8), (32768, 1, 8, 2), (8192, 16, 4, 4), (32769, 1, 8, 8), (65536, 1, 8, 8),
                        (131000, 1, 16, 4), (8192, 17, 4, 4), (1 << 20, 1, 4, 1)):
        a = attn_desc(H=H, Hk=Hk, B=B, Tq=B * n, Tk=B * n, max_q=n, max_k=n)
        pairs = B * (-(-n // 64) * 64) ** 2
        ahead = pairs if pairs <= GiB else 0
        more = lib.gtp_attention_biased_work(ctypes.byref(a), bias_desc(), 0) - lib.gtp_attention_work(ctypes.byref(a), 0)
        assert more == ahead
        # the gradient: the workgroups' tables besides, of 64 rows of a key head at least for each of 128 parts of the keys at
        # most, and those of their sums
        most = 128 * B * -(-n * (H // Hk) // 64) * H * 32 * 4
        more = lib.gtp_attention_biased_work(ctypes.byref(a), bias_desc(), 1) - lib.gtp_attention_work(ctypes.byref(a), 1)
        assert ahead <= more <= ahead + 2 * most


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [32760, 32769])  # the buckets made ahead just below 1 GiB, and at each score
def test_rows_on_both_sides_of_the_limit(n, dtype):
    """Some rows' results and gradients against the 64-bit form of these rows.  A lane adds up to n / 2 terms in sequence:
    (n / 2 + 256) u of their magnitudes, and a score's error moves P by as much; bf16: 2^-8 of P and dS besides."""
    g = torch.Generator(device="cuda").manual_seed(n)
    H, d, nb = 4, 16, 24
    q, k, v, do = (torch.randn((n, H, d), generator=g, device="cuda").to(dtype) for _ in range(4))
    pos = torch.rand((n, 3), generator=g, device="cuda") * 60.0
    bias = torch.randn((H, nb), generator=g, device="cuda")
    print(f"biased n={n} {dtype}", flush=True)
    o, lse = gtp.gtp_attention_biased(q, k, v, bias, pos, r0=2.0)
    grads = gtp.gtp_attention_biased_backward(q, k, v, bias, pos, None, 2.0, 4, o, do, lse)
    at = torch.cat([torch.arange(24, device="cuda"), torch.randint(n, (24,), generator=g, device="cuda"),
                    torch.arange(n - 24, n, device="cuda")])
    m = len(at)
    args = (q[at].double(), k.double(), v.double(), bias.double(), pos[at], pos, 4.0, 4, 1.0 / math.sqrt(d), [(0, m)], [(0, n)],
            None, 0.0, None, m, n)
    largest = 1 + float(q.double().norm(dim=-1).amax() * k.double().norm(dim=-1).amax()) / math.sqrt(d) + float(bias.abs().max())
    c, half = (n / 2 + 256) * 2.0 ** -24 * largest, 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23
    want, wl, size = B.attention(*args)
    assert bool(((o[at].double() - want).abs() <= half * want.abs() + (half + c) * size).all())
    assert bool(((lse[at].double() - wl).abs() <= c).all())
    dq, s, e32 = B.attention(*args, grad=(do[at].double(), o[at].double(), lse[at].double()))["dq"]
    assert bool(((grads["dq"][at].double() - dq).abs() <= half * dq.abs() + half * s + c * e32).all())
    # the gradients of keys and bias: sums over all rows, the same on both sides of the limit but for rounding; here
    # against their sum rules: dS sums to zero over a row's keys, so dbias does over the buckets; P to one: dv to do
    total = lambda t: t.double().sum((0, 2))  # noqa: E731
    size = do.double().abs().sum((0, 2))
    assert bool(((total(grads["dv"]) - total(do)).abs() <= (c + 2 * half) * size).all())
    rows = (do.double().abs().sum(-1) * v.double().abs().amax((0, 2))).sum(0) * 2  # of |dS| by head
    assert bool((grads["dbias"].double().sum(1).abs() <= c * rows + half * (do.double() * o.double()).abs().sum((0, 2))).all())


def test_outputs_that_are_not_asked_for():
    """Refused before anything else happens: they would stay as they were."""
    z = torch.zeros
    q, k, lse, pos = z(6, 4, 8), z(6, 2, 8), z(6, 4), z(6, 3)

    def call(need, **out):
        gtp.gtp_attention_biased_backward(q, k, k, z(4, 16), pos, None, 1.0, 4, q, q, lse, need=need, **out)

    for need, name in ((("dk", "dv"), "dq"), (("dbias",), "dq"), (("dq",), "dk"), (("dq", "dbias"), "dv"), ((), "dq")):
        with pytest.raises(ValueError, match="not among need"):
            call(need, **{name: torch.zeros_like(q if name == "dq" else k)})
    # dk and dv are made together: either may be given where one is asked for
    for need, name in ((("dq",), "dq"), (("dk",), "dv"), (("dv",), "dk")):
        with pytest.raises(ValueError, match="device tensor"):
            call(need, **{name: torch.zeros_like(q if name == "dq" else k)})


def test_negative_r0():
    """Its square would do for the library."""
    z = torch.zeros
    q, k, lse, pos, bias = z(6, 4, 8), z(6, 2, 8), z(6, 4), z(6, 3), z(4, 16)
    for r0 in (-1.0, -1e-3, -1e30, -math.inf):
        with pytest.raises(ValueError, match="r0"):
            gtp.gtp_attention_biased(q, k, k, bias, pos, r0=r0)
        with pytest.raises(ValueError, match="r0"):
            gtp.gtp_attention_biased_backward(q, k, k, bias, pos, None, r0, 4, q, q, lse)
        with pytest.raises(ValueError, match="r0"):
            gtp.gtp_attention_bias_edges(16, r0)


def test_edges_of_numbers_out_of_range():
    """Neither cut to 32 bits nor answered with a list of that many."""
    for buckets, per in ((2 ** 32 + 4, 4), (4, 2 ** 32 + 4), (-(2 ** 32) + 4, 4), (2 ** 70, 4), (4, 4.0), (4.0, 4), (10 ** 9, 4), (65, 4),
                         (-1, 4), (0, 4)):
        with pytest.raises((ValueError, gtp.GTPError)):
            gtp.gtp_attention_bias_edges(buckets, 1.0, per)
    with pytest.raises((ValueError, gtp.GTPError)):
        gtp.gtp_attention_bias_edges(4, 1e200)
    assert gtp.gtp_attention_bias_edges(4, 1.0, 1) == [1.0, 2.0, 4.0] and gtp.gtp_attention_bias_edges(1, 1.0) == []
    assert len(gtp.gtp_attention_bias_edges(64, 1.0)) == 63


def test_too_little_work_names_its_size_function():
    lib, a = gtp.lib(), attn_desc(Tk=20000, max_k=20000)
    r = [ctypes.byref(rows(i, h)) for i, h in ((0, 4), (1, 2), (2, 2), (3, 4))]
    back = [ctypes.byref(rows(i, h)) for i, h in ((4, 4), (7, 4), (8, 2), (9, 2))]
    for name, biased in (("gtp_attention", ()), ("gtp_attention_biased", (bias_desc(),))):
        assert getattr(lib, name)(ctypes.byref(a), *biased, *r, at(5), at(6), 16, None) == gtp.GTP_ERR_INVALID_ARG
        assert name + "_work" in lib.gtp_last_error().decode()
        more = (at(43),) if biased else ()
        assert getattr(lib, name + "_backward")(ctypes.byref(a), *biased, *r, back[0], at(5), *back[1:], *more, at(6), 16,
                                                None) == gtp.GTP_ERR_INVALID_ARG
        assert name + "_work" in lib.gtp_last_error().decode()
