"""The attention with a bias by distance and its gradient on the GPU against the plain 64-bit form of
tests/biased_ref.py: types, lengths from none to long, shared heads, every head length's kernel, positions on bucket edges,
NaN and infinite, cutoffs that leave rows empty, absent keys, strides, streams, graphs, run-to-run equality, the
poisoned-LDS build.

Tolerances as in tests/test_layers.py: rounding to bf16 moves a value by 2^-8 of itself at most; sums are off by 2^-16 of
their terms' magnitudes at most; with bf16 inputs P and dS enter the matrix products with another 2^-8.  A score's
error moves P by as much, and a score has the bias beside the product: 1 + |q| |k| scale + |bias| takes its place.  dbias
sums dS before its rounding to bf16.
"""
import math
import os

import pytest

torch = pytest.importorskip("torch")

import biased_ref as B  # noqa: E402
import layers_ref as R  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402
from test_layers import C32, RNG, Case, close, difference, gen, off_by_one, offsets, out_tol, randn  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
POISON_LIB = os.path.join(os.path.dirname(gtp.__file__), "libgtp_poison.so")


def _say(msg):
    print(msg, flush=True)


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gtp.lib()


class Biased(Case):
    def __init__(self, dtype, ql, kl, H, Hk, d, masked=0.0, p=0.0, buckets=24, per=4, r0=1.0, box=3.0, cutoff=False, **more):
        super().__init__(dtype, ql, kl, H, Hk, d, masked, p, **more)
        g = gen(31 + sum(ql) + sum(kl) + buckets)
        self.k_pos = torch.rand((sum(kl), 3), generator=g, device="cuda") * box
        self.q_pos = self.k_pos.clone() if ql == kl else torch.rand((sum(ql), 3), generator=g, device="cuda") * box
        self.bias = randn(g, H, buckets)
        if cutoff:
            self.bias[:, -1] = -math.inf
        self.r0, self.per = r0, per

    def ref(self, grad=None):
        qs, ks = (R.segments(offsets(n).tolist(), len(n), 0, 0) for n in (self.ql, self.kl))
        t = [x.double() for x in (self.q, self.k, self.v)]
        if self.mask is not None:
            t[1], t[2] = (torch.where(self.mask.bool()[:, None, None], x, 0.0) for x in t[1:])
        return B.attention(*t, self.bias.double(), self.q_pos, self.k_pos, self.r0 * self.r0, self.per, self.scale, qs, ks,
                           self.mask, self.p, RNG, max(self.ql), max(self.kl), grad)

    def forward(self, **more):
        return gtp.gtp_attention_biased(self.q, self.k, self.v, self.bias, self.q_pos, self.k_pos, self.r0, self.per,
                                        **{**self.args, **more})

    def backward(self, o, lse, **more):
        return gtp.gtp_attention_biased_backward(self.q, self.k, self.v, self.bias, self.q_pos, self.k_pos, self.r0,
                                                 self.per, o, self.do, lse, **{**self.args, **more})

    def largest(self):
        b = self.bias[torch.isfinite(self.bias)].abs()
        return 1 + (self.q.double().norm(dim=-1).amax() * self.k_norm() * abs(self.scale)) + (b.max() if b.numel() else 0)

    def check_forward(self, o, lse):
        ro, rl, size = self.ref()
        half = 2.0 ** -8 if self.dtype == BF16 else 0.0
        close(o, ro, out_tol(ro, self.dtype) + (half + C32 * self.largest()) * size + 1e-30, "o")
        none = torch.isinf(rl)
        assert torch.equal(torch.isinf(lse), none) and bool((lse[none] < 0).all()) and bool((o[none] == 0).all())
        close(lse[~none], rl[~none], C32 * self.largest() * torch.ones_like(rl[~none]), "lse")

    def check_backward(self, o, lse, grads, names=("dq", "dk", "dv", "dbias")):
        ref = self.ref((self.do.double(), o.double(), lse.double()))
        half = 2.0 ** -8 if self.dtype == BF16 else 0.0
        for n in names:
            want, size, e32 = ref[n]
            own = 0.0 if n == "dbias" else out_tol(want, self.dtype) + half * size
            close(grads[n], want, own + C32 * self.largest() * e32 + 1e-30, n)


# (query lengths, key lengths, H, Hk, d, share of absent keys, p, more)
CASES = [
    ([1], [1], 1, 1, 1, 0, 0, {}), ([1], [1], 2, 1, 9, 0, 0.3, dict(buckets=1)), ([1, 1, 1], [5, 1, 33], 3, 3, 16, 0, 0, dict(buckets=2)),
    ([27] * 4, [27] * 4, 8, 8, 32, 0, 0, {}), ([5, 49, 32, 33, 1, 31], [5, 49, 32, 33, 1, 31], 2, 2, 72, 0, 0.1, dict(per=8)),
    ([0, 3, 0, 64], [4, 0, 0, 65], 2, 2, 64, 0, 0, {}), ([40, 7], [40, 90], 6, 2, 75, 0.3, 0, dict(buckets=64, per=16)),
    ([129, 128, 127], [63, 64, 65], 2, 1, 100, 0, 0.2, dict(per=1)), ([300], [257], 1, 1, 128, 0, 0, dict(buckets=33)),
    ([1], [3001], 4, 1, 64, 0.1, 0, {}), ([2, 2], [1000, 1999], 8, 2, 128, 0, 0.1, dict(buckets=64)), ([33], [1], 5, 1, 3, 0, 0, {}),
    ([200], [131], 2, 2, 144, 0, 0, {}), ([70], [70], 2, 1, 200, 0.2, 0.1, dict(buckets=64)), ([65, 20], [65, 20], 1, 1, 256, 0, 0, dict(buckets=64)),
    ([150], [150], 2, 1, 256, 0.1, 0.1, dict(buckets=64)), ([150], [140], 2, 2, 190, 0, 0, dict(buckets=64)),
    ([511], [513], 1, 1, 48, 0.5, 0, dict(r0=0.5)), ([1025], [1023], 2, 2, 40, 0, 0, dict(box=9.0)), ([31], [700], 12, 4, 24, 0.9, 0.5, {}),
    ([2000], [3], 3, 1, 64, 0, 0, {}), ([1500], [40], 4, 2, 96, 0.2, 0.1, dict(buckets=7)), ([3], [4], 1, 1, 217, 0, 0, {}),
    ([90, 60], [90, 60], 4, 4, 36, 0, 0, dict(cutoff=True, buckets=8, per=2, box=6.0)),
    # buckets made ahead: long segments, four heads and more
    ([600, 433], [600, 433], 4, 4, 64, 0, 0, dict(buckets=64, per=8, box=9.0)), ([300, 511], [520, 400], 8, 4, 72, 0.2, 0.1, {}),
    ([289], [1000], 4, 1, 120, 0, 0, dict(cutoff=True)), ([700], [545], 4, 4, 32, 0.5, 0, {}), ([513], [257], 6, 2, 190, 0, 0.1, {}),
    ([300], [300], 4, 4, 250, 0.1, 0, dict(buckets=64)), ([401, 0, 399], [0, 300, 390], 4, 4, 96, 0, 0, {}),
    # workgroups of eight waves, for two on a SIMD beside the sums
    ([520, 37, 260], [300, 290, 5], 4, 4, 128, 0.2, 0.1, dict(buckets=64)), ([300, 150], [270, 80], 8, 2, 100, 0, 0.1, dict(buckets=64)),
    ([1100], [70], 2, 1, 128, 0, 0, dict(buckets=64)), ([70, 33], [60, 20], 16, 1, 96, 0.1, 0, dict(buckets=64)),
    ([513], [700], 4, 2, 60, 0, 0, dict(buckets=64, cutoff=True)),
    ([3], [40], 63, 1, 190, 0, 0, dict(buckets=64)), ([5], [33], 256, 1, 9, 0, 0, dict(buckets=16)),
    ([20], [500], 64, 1, 16, 0, 0, dict(buckets=64)), ([9], [40], 37, 1, 20, 0, 0.2, dict(buckets=5)),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ql,kl,H,Hk,d,masked,p,more", CASES)
def test_attention_and_gradient(ql, kl, H, Hk, d, masked, p, more, dtype):
    _say(f"biased q={ql} k={kl} H={H}/{Hk} d={d} masked={masked} p={p} {more} {dtype}")
    c = Biased(dtype, ql, kl, H, Hk, d, masked, p, **more)
    o, lse = c.forward()
    torch.cuda.synchronize()
    c.check_forward(o, lse)
    g = c.backward(o, lse)
    torch.cuda.synchronize()
    c.check_backward(o, lse, g)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_bias_is_the_attention_without(dtype):
    """A bias of zeros: the same but for one rounding of each score."""
    c = Biased(dtype, [60, 33], [60, 33], 4, 2, 64, 0.1, 0.1)
    c.bias.zero_()
    o, lse = c.forward()
    c.check_forward(o, lse)
    o2, lse2 = Case.forward(c)
    _, _, size = c.ref()
    assert float((lse - lse2).abs().max()) < 1e-5
    close(o, o2.double(), 2 * out_tol(o2.double(), dtype) + (2.0 ** -7 if dtype == BF16 else 0) * size + C32 * c.largest() * size, "o")


def test_positions_on_the_edges():
    """Pairs exactly on an edge, one unit in the last place below it, of distance zero, infinite and NaN: P of one-hot
    values names each pair's bucket."""
    nb, per, r0sq = 16, 4, 1.5 * 1.5
    e = B.edges(nb, r0sq, per)
    x = []
    for v in e:
        for n in (B.number(math.sqrt(v)) + i for i in range(-3, 4)):
            x.append(B.value(n))
    x += [0.0, 1e30, math.inf, math.nan, -math.nan]
    k_pos = torch.zeros((len(x), 3))
    k_pos[:, 0] = torch.tensor(x)
    q_pos = torch.zeros((1, 3))
    bias = torch.linspace(-1, 1, nb)[None].contiguous()
    n = len(x)
    q, k = torch.zeros((1, 1, n)), torch.zeros((n, 1, n))
    v = torch.eye(n)[:, None].contiguous()
    o, lse = gtp.gtp_attention_biased(q.cuda(), k.cuda(), v.cuda(), bias.cuda(), q_pos.cuda(), k_pos.cuda(), 1.5, per)
    got = (o[0, 0].log() + lse[0, 0]).cpu()  # the bias of each key
    bucket = B.bucket_of(q_pos.numpy(), k_pos.numpy(), nb, r0sq, per)[0]
    assert len(set(bucket.tolist())) == nb and bucket[-5:].tolist() == [0] + [nb - 1] * 4
    assert float((got - bias[0][torch.from_numpy(bucket)]).abs().max()) < 0.03  # buckets are 2 / 15 apart


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_cutoff_leaves_rows_empty(dtype):
    """Atoms beyond the cutoff of every key: o = 0, lse = -inf, no gradients from them, whatever v holds."""
    c = Biased(dtype, [40, 30], [50, 60], 4, 2, 64, buckets=12, per=2, cutoff=True)
    c.q_pos[5] += 1e4
    c.q_pos[60:] -= 1e4
    o, lse = c.forward()
    empty = [5] + list(range(60, 70))
    assert bool((lse[empty] == -math.inf).all()) and bool((o[empty] == 0).all()) and bool(torch.isfinite(lse[:5]).all())
    c.check_forward(o, lse)
    g = c.backward(o, lse)
    c.check_backward(o, lse, g)
    assert bool((g["dq"][empty] == 0).all()) and bool((g["dbias"][:, -1] == 0).all())
    c.v[0] = math.inf
    g2 = c.backward(o, lse)
    assert bool((g2["dq"][empty] == 0).all()) and bool(torch.isfinite(g2["dq"][60:]).all())
    c.bias.fill_(-math.inf)
    o, lse = c.forward()
    g = c.backward(o, lse)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all()) and not any(bool(t.any()) for t in g.values())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_absent_keys_hold_anything(dtype, p):
    c = Biased(dtype, [40, 50, 20], [130, 60, 70], 4, 2, 64, masked=0.4, p=p)
    c.mask[130:190] = 0
    o, lse = c.forward()
    assert bool((o[40:90] == 0).all()) and bool((lse[40:90] == -math.inf).all())
    g = c.backward(o, lse)
    c.check_forward(o, lse)
    c.check_backward(o, lse, g)
    assert bool((g["dk"][~c.mask.bool()] == 0).all())
    for junk in (math.nan, math.inf, -math.inf, torch.finfo(dtype).min, torch.finfo(dtype).max):
        for t in (c.k, c.v, c.k_pos):
            t[~c.mask.bool()] = junk
        o2, lse2 = c.forward()
        g2 = c.backward(o, lse)
        assert torch.equal(o, o2) and torch.equal(lse, lse2) and all(torch.equal(g[n], g2[n]) for n in g), junk


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_biases_and_scales(dtype):
    for scale in (8.0, -1.5, 0.0):
        c = Biased(dtype, [100], [300], 4, 2, 64, scale=scale)
        c.bias *= 50.0
        o, lse = c.forward()
        c.check_forward(o, lse)
        c.check_backward(o, lse, c.backward(o, lse))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 75])
def test_slices_expanded_inputs_and_alignment(dtype, d):
    c = Biased(dtype, [33, 64, 90], [33, 64, 90], 4, 4, d)
    o, lse = c.forward()
    g = c.backward(o, lse)
    T = sum(c.ql)
    for shift in (0, 1):
        buf = torch.zeros(T * 3 * 4 * d + shift, dtype=dtype, device="cuda")[shift:].view(T, 3, 4, d)
        buf[:, 0], buf[:, 1], buf[:, 2] = c.q, c.k, c.v
        out = torch.full_like(buf, 7.0)
        q, k, v = buf.unbind(1)
        pos, bias = off_by_one(c.q_pos), off_by_one(c.bias)
        o2, lse2 = gtp.gtp_attention_biased(q, k, v, bias, pos, None, c.r0, c.per, **c.args)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        g2 = gtp.gtp_attention_biased_backward(q, k, v, bias, pos, None, c.r0, c.per, o, c.do, lse, **c.args,
                                               dq=out[:, 0], dk=out[:, 1], dv=out[:, 2])
        assert all(torch.equal(out[:, i], g[n]) for i, n in enumerate(("dq", "dk", "dv")))
        assert torch.equal(g2["dbias"], g["dbias"])
    o2, lse2 = c.forward(q_off=None, k_off=None, max_q=None, max_k=None)  # one segment of everything
    assert o2.shape == o.shape and not torch.equal(o2, o)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_parts_of_the_gradient(dtype):
    for ql, kl in (([80, 33], [80, 33]), ([4], [5000])):
        c = Biased(dtype, ql, kl, 4, 2, 40, masked=0.1, p=0.1)
        o, lse = c.forward()
        g = c.backward(o, lse)
        for need in (("dq",), ("dbias",), ("dk", "dv"), ("dv",), ("dq", "dbias"), ("dbias", "dk"), ()):
            part = c.backward(o, lse, need=need)
            assert set(part) == set(need) and all(torch.equal(part[n], g[n]) for n in need), need


def test_rows_of_no_segment_and_nothing_at_all():
    c = Biased(F32, [20, 30], [20, 30], 2, 2, 32)
    o, lse = c.forward()
    g = c.backward(o, lse)
    off = torch.tensor([0, 20], dtype=torch.int64, device="cuda")
    o2, lse2 = torch.full_like(o, 5.0), torch.full_like(lse, 5.0)
    c.forward(q_off=off, k_off=off, max_q=20, max_k=20, o=o2, lse=lse2)
    assert torch.equal(o2[:20], o[:20]) and bool((o2[20:] == 5).all()) and bool((lse2[20:] == 5).all())
    off = torch.tensor([-5, 20, 1 << 40], dtype=torch.int64, device="cuda")  # cut to the tensor
    o2, lse2 = c.forward(q_off=off, k_off=off)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    # a segment of more rows than max_q says is cut there; what is left out adds nothing to dbias
    g1 = c.backward(o, lse, max_q=20)
    assert bool(torch.isfinite(g1["dbias"]).all()) and not torch.equal(g1["dbias"], g["dbias"])
    for nq, nk in ((0, 7), (7, 0), (0, 0)):
        e = Biased(F32, [nq], [nk], 2, 1, 16)
        o, lse = e.forward()
        assert not bool(o.any()) and bool((lse == -math.inf).all())
        assert not any(bool(t.any()) for t in e.backward(o, lse).values())


@pytest.mark.parametrize("masked,p", [(0.0, 0.0), (0.2, 0.25)])
def test_gradient_against_differences(masked, p):
    c = Biased(F32, [30, 9], [30, 21], 4, 2, 24, masked=masked, p=p, buckets=9, per=2)
    o, lse = c.forward()
    g = c.backward(o, lse)
    pos = (c.q_pos, c.k_pos, c.r0, c.per)
    f = lambda q, k, v, b: float((gtp.gtp_attention_biased(q, k, v, b, *pos, **c.args)[0].double() * c.do.double()).sum())  # noqa: E731
    gg = gen(7)
    base = {"dq": c.q, "dk": c.k, "dv": c.v, "dbias": c.bias}
    for i, (name, t) in enumerate(base.items()):
        u = randn(gg, *t.shape)
        got, step = difference(lambda z: f(*(z if j == i else x for j, x in enumerate(base.values()))), t, u, 1e-2)
        want = float((g[name].double() * step).sum())
        # a cubic term of relative size h^2, and outputs' errors of 2^-20 |do| each
        noise = 2.0 ** -20 * float(c.do.double().abs().sum()) + 1e-3 * float((g[name].double() * step).abs().sum())
        _say(f"  {name}: difference {got:.6f} gradient {want:.6f}")
        assert abs(got - want) <= noise


def test_turning_the_atoms_changes_nothing():
    """Quarter turns and reflections, exact in fp32: the same distances from other coordinates, but for the order of the
    three squares, which the buckets do not notice on coordinates of few bits."""
    c = Biased(F32, [50], [50], 4, 4, 36)
    c.k_pos = (c.k_pos * 64).round() / 64
    c.q_pos = c.k_pos.clone()
    o, lse = c.forward()
    for t in (lambda x: x[:, [1, 2, 0]], lambda x: x * torch.tensor([1.0, -1.0, -1.0], device="cuda"), lambda x: x + 16.0):
        c2 = t(c.k_pos).contiguous()
        o2, lse2 = gtp.gtp_attention_biased(c.q, c.k, c.v, c.bias, c2, c2, c.r0, c.per, **c.args)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_far_into_a_long_cache(dtype):
    d, n = 128, 17_000_000
    k, v, pos = torch.zeros((n, 1, d), dtype=dtype, device="cuda"), torch.zeros((n, 1, d), dtype=dtype, device="cuda"), torch.zeros((n, 3), device="cuda")
    c = Biased(dtype, [70], [300], 2, 1, d)
    k[-300:], v[-300:], pos[-300:] = c.k, c.v, c.k_pos
    args = {**c.args, "k_off": torch.tensor([n - 300, n], dtype=torch.int64, device="cuda")}
    geometry = (c.bias, c.q_pos, pos, c.r0, c.per)
    o, lse = gtp.gtp_attention_biased(c.q, k, v, *geometry, **args)
    want, wl = c.forward()
    assert torch.equal(o, want) and torch.equal(lse, wl)
    g2 = gtp.gtp_attention_biased_backward(c.q, k, v, *geometry, o, c.do, lse, **args, need=("dq", "dbias"))
    g = c.backward(o, lse)
    assert torch.equal(g2["dq"], g["dq"]) and torch.equal(g2["dbias"], g["dbias"])


def test_every_pair_counts_once_in_dbias():
    """P = 1 / keys and dP that is a constant of the key: a bucket's sum counts its pairs."""
    n, nb = 2500, 12
    c = Biased(F32, [n], [n], 1, 1, 4, buckets=nb, per=2, box=8.0)
    c.q.zero_()
    c.bias.zero_()
    c.v.zero_()
    c.v[:, 0, 0] = torch.arange(n, device="cuda") % 2 * 2.0 - 1.0  # mean 0: o = 0 and delta = 0
    c.do.zero_()
    c.do[:, 0, 0] = 1.0
    o, lse = c.forward()
    g = c.backward(torch.zeros_like(o), lse, need=("dbias",))["dbias"][0].double().cpu() * n
    import numpy as np
    bucket = B.bucket_of(c.q_pos.cpu().numpy(), c.k_pos.cpu().numpy(), nb, 1.0, 2)
    sign = c.v[:, 0, 0].cpu().numpy()
    want = np.array([(bucket == b).astype(float).dot(sign).sum() for b in range(nb)])
    count = np.array([(bucket == b).sum() for b in range(nb)])
    # each term is 1 / n to 2^-20: lost or doubled pairs are whole numbers
    assert np.all(np.abs(g.numpy() - want) < 0.3 + 2.0 ** -20 * count), (g.numpy() - want)


def everything(dtype):
    out = []
    for ql, kl, H, Hk, d, p, more in (([30, 49], [30, 49], 4, 4, 72, 0.1, {}), ([300], [300], 4, 2, 64, 0.0, dict(buckets=64)),
                                      ([2], [4000], 4, 2, 64, 0.0, {}), ([3000], [9], 2, 1, 128, 0.1, {}),
                                      ([90], [80], 2, 2, 160, 0.0, dict(buckets=64)), ([200], [200], 2, 1, 250, 0.0, dict(buckets=64)),
                                      ([700], [700], 8, 2, 32, 0.0, dict(buckets=3)),
                                      ([400, 301], [400, 301], 4, 4, 72, 0.1, dict(buckets=64))):
        c = Biased(dtype, ql, kl, H, Hk, d, 0.1, p, **more)
        o, lse = c.forward()
        out += [o, lse, *c.backward(o, lse).values()]
    return out


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_same_bits_again_and_poisoned_lds(dtype):
    a, b = everything(dtype), everything(dtype)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    with gtp.use_library(POISON_LIB):
        c = everything(dtype)
        torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, c))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_on_another_stream_and_in_two_graphs(dtype):
    c = Biased(dtype, [3], [9000], 4, 2, 64, 0.1, 0.1)
    e = Biased(dtype, [60, 41], [60, 41], 4, 4, 36)
    o, lse = c.forward()
    g = c.backward(o, lse)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        o2, l2 = c.forward(stream=s)
        g2 = c.backward(o2, l2, stream=s)
        junk = torch.full((1 << 20,), 3.0, device="cuda")
        del junk
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, l2) and all(torch.equal(g[n], g2[n]) for n in g)

    def both(x):
        a, b = x.forward()
        return [a, b, *x.backward(a, b).values()]

    graphs = []
    for x in (c, e):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both(x)
        graphs.append((graph, x, out))
    for turn in range(3):
        for graph, x, out in graphs:
            x.bias.copy_(randn(gen(60 + turn), *x.bias.shape))
            x.q_pos.add_(0.25)
            graph.replay()
        torch.cuda.synchronize()
        for graph, x, out in graphs:
            want = both(x)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), turn
