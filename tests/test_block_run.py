"""The layers of a block in a row, as a model runs them, on the GPU: norm -> attention biased by the atoms' distances -> the
residual step with its norms, gate and scale (the next part's input), twice over, and the gradients back through all of
it; against differences, under rotations, in a graph with changed inputs, and two at once on two streams."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2401_10216_amd import gtp  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gtp.lib()


class Block:
    """Features [T, C, 4] of degree 1; per layer a linear map of q (channels, within a degree), the rest learned by the layers."""

    def __init__(self, C=16, H=4, layers=2, buckets=12, p=0.0, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.C, self.H, self.p = C, H, p
        self.first = {"w": 1 + 0.1 * n(2, C), "b": 0.1 * n(C)}
        self.layers = [{"wq": n(2, C, C) / C ** 0.5, "bias": n(H, buckets), "gate": n(C, C) / C ** 0.5,
                        "scale": 0.5 + 0.1 * n(2, C), "w_post": 1 + 0.1 * n(2, C), "b_post": 0.1 * n(C),
                        "w_pre": 1 + 0.1 * n(2, C), "b_pre": 0.1 * n(C)} for _ in range(layers)]

    def linear(self, w, x):
        return torch.cat([w[0] @ x[:, :, :1], w[1] @ x[:, :, 1:]], 2).contiguous()

    def heads(self, x):
        return x.view(x.shape[0], self.H, -1)

    def forward(self, x, pos, off, longest, rng=None):
        args = dict(q_off=off, k_off=off, max_q=longest, max_k=longest, p=self.p, rng=rng if self.p else None)
        h, mean, rstd = gtp.gtp_layer_norm(x, 1, self.first["w"], self.first["b"])
        saved = [(x, mean, rstd)]
        for P in self.layers:
            q = self.heads(self.linear(P["wq"], h))
            k = self.heads(h)
            o, lse = gtp.gtp_attention_biased(q, k, k, P["bias"], pos, pos, 1.0, 2, **args)
            gate = (h[:, :, 0] @ P["gate"].T).contiguous()
            w = {n: P[n] for n in ("scale", "w_post", "b_post", "w_pre", "b_pre")}
            r, h2, stats = gtp.gtp_residual_norm(x, o.view_as(x), 1, gate=gate, **w)
            saved.append((h, q, o, lse, gate, r, stats, args, pos))
            x, h = r, h2
        return x, h, saved

    def backward(self, saved, dx, dh):
        """Gradients for dx of the stream and dh of its last norm."""
        grads = []
        for P, (h, q, o, lse, gate, r, stats, args, pos) in zip(reversed(self.layers), reversed(saved[1:])):
            w = {n: P[n] for n in ("scale", "w_post", "b_post", "w_pre", "b_pre")}
            g = gtp.gtp_residual_norm_backward(r, o.view_as(r), 1, stats, dh, dr=dx, gate=gate, **w)
            k = self.heads(h)
            at = gtp.gtp_attention_biased_backward(q, k, k, P["bias"], pos, pos, 1.0, 2, o, self.heads(g["da"]), lse, **args)
            dq, dgate = at["dq"].view_as(r), g["dgate"]
            dh = (at["dk"] + at["dv"]).view_as(r) + self.linear(P["wq"].transpose(1, 2).contiguous(), dq)
            dh[:, :, 0] += dgate @ P["gate"]
            dx = g["dx"]
            own = {n: g["d" + n] for n in w}
            own["bias"], own["gate"] = at["dbias"], dgate.T @ h[:, :, 0]
            own["wq"] = torch.stack([torch.matmul(dq[:, :, s].transpose(0, 1).reshape(self.C, -1),
                                                  h[:, :, s].transpose(0, 1).reshape(self.C, -1).T)
                                     for s in (slice(0, 1), slice(1, 4))])
            grads.append(own)
        x, mean, rstd = saved[0]
        nb = gtp.gtp_layer_norm_backward(x, dh.contiguous(), 1, mean, rstd, self.first["w"])
        return dx + nb["dx"], grads[::-1], {"w": nb["dw"], "b": nb["db"]}


def molecules(sizes, C, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(sizes)
    x = torch.randn((T, C, 4), generator=g, device="cuda")
    pos = torch.rand((T, 3), generator=g, device="cuda") * 4
    off = torch.tensor([0] + list(sizes)).cumsum(0).cuda()
    return x, pos, off, max(sizes)


@pytest.mark.parametrize("p", [0.0, 0.2])
def test_gradients_against_differences(p):
    """Central differences of a scalar in fp32 calls summed in 64 bits: a cubic term of relative size h^2 = 1e-4 of the
    terms, and outputs' errors of some 2^-20 of the cotangents' sizes through two layers."""
    b = Block(p=p)
    x, pos, off, longest = molecules((9, 1, 14), 16)
    rng = torch.tensor([7, 3], dtype=torch.int64, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    c1, c2 = (torch.randn(x.shape, generator=g, device="cuda") for _ in range(2))

    def f(x):
        r, h, _ = b.forward(x, pos, off, longest, rng)
        return float((r.double() * c1.double()).sum() + (h.double() * c2.double()).sum())

    r, h, saved = b.forward(x, pos, off, longest, rng)
    dx, grads, first = b.backward(saved, c1, c2)
    noise = 2.0 ** -18 * float((c1.double().abs() + c2.double().abs()).sum())

    def check(name, tensor, grad):
        u = torch.randn(tensor.shape, generator=g, device="cuda")
        keep, step = tensor.clone(), 3e-3
        tensor.copy_(keep + step * u)
        up, hi = f(x), tensor.double().clone()
        tensor.copy_(keep - step * u)
        dn, lo = f(x), tensor.double().clone()
        tensor.copy_(keep)
        want = float((grad.double() * (hi - lo)).sum())
        bound = noise + 5e-3 * float((grad.double() * (hi - lo)).abs().sum())
        print(f"  {name}: difference {up - dn:.6f} gradient {want:.6f} bound {bound:.6f}", flush=True)
        assert abs((up - dn) - want) <= bound, name

    check("x", x, dx)
    for name in ("w", "b"):
        check("first " + name, b.first[name], first[name])
    for i, P in enumerate(b.layers):
        for name in P:
            check(f"layer {i} {name}", P[name], grads[i][name])


def test_turning_features_and_atoms_turns_the_result():
    b = Block(seed=3)
    x, pos, off, longest = molecules((12, 7), 16, seed=4)
    pos = (pos * 16).round() / 16  # quarter turns and few bits: the same distances to the last bit
    D = torch.tensor([[0.0, 1, 0], [0, 0, -1], [1, 0, 0]], device="cuda")
    turn = lambda t: torch.cat([t[..., :1], t[..., 1:] @ D.T], -1).contiguous()  # noqa: E731
    r, h, _ = b.forward(x, pos, off, longest)
    r2, h2, _ = b.forward(turn(x), (pos @ D.T).contiguous(), off, longest)
    # sums of the three components in another order: some units in the last place of values up to about 8
    assert float((r2 - turn(r)).abs().max()) < 1e-4 and float((h2 - turn(h)).abs().max()) < 1e-4


def test_in_a_graph_and_on_two_streams():
    b = Block(seed=6, p=0.1)
    x, pos, off, longest = molecules((20, 33, 5), 16, seed=7)
    rng = torch.tensor([9, 0], dtype=torch.int64, device="cuda")
    c = torch.randn_like(x)

    def run():
        r, h, saved = b.forward(x, pos, off, longest, rng)
        dx, grads, first = b.backward(saved, c, c)
        return [r, h, dx, *first.values(), *(t for g in grads for t in g.values())]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for i in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda"))
        pos.add_(0.125 * (i + 1))
        pos.mul_(1.0 + 0.1 * i)
        rng[1] = i
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = run()
        torch.cuda.synchronize()
        # torch's own products choose their kernels anew in a graph: sums in another order
        for a, e in zip(got, want):
            assert float((a - e).abs().max()) <= 1e-4 * (1 + float(e.abs().max())), i
    streams = [torch.cuda.Stream() for _ in range(2)]
    want = [t.clone() for t in run()]
    results = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            results.append(run())
    torch.cuda.synchronize()
    for got in results:
        for a, e in zip(got, want):
            assert float((a - e).abs().max()) <= 1e-4 * (1 + float(e.abs().max()))
    assert not any(math.isnan(float(t.sum())) for t in want)
