"""A training step of one equivariant block on a batch of molecules: normalisation, attention over the atoms of each
molecule with dropped probabilities, dropout of whole channels into the residual, and a Gaunt tensor product of the
result with itself (a feature interaction with learnable per-degree weights), with every gradient.

    python examples/molecule_block.py [--molecules 64] [--atoms 27] [--channels 64] [--L 2] [--steps 20]

Features are SH coefficients [atoms, C, (L+1)^2]; linear maps mix channels within a degree.  Every part commutes with
rotations of the features, the draws included (a channel is dropped whole, a probability is invariant), so the block
does.  Molecules have different numbers of atoms, packed one after the other.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2401_10216_amd import gtp  # noqa: E402


class Block:
    """y = x + drop(Wo attention(Wq h, Wk h, Wv h)), h = norm(x);  out = y + GTP(y, y) with weights per degree."""

    def __init__(self, C, L, heads, p, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.C, self.L, self.H, self.p = C, L, heads, p
        self.plan = gtp.Plan(L, L, L)
        self.params = {"norm_w": torch.ones(L + 1, C, device=device), "norm_b": torch.zeros(C, device=device),
                       "wp": torch.full((1, L + 1), 0.1, device=device)}
        for n in ("wq", "wk", "wv", "wo"):
            self.params[n] = torch.randn((L + 1, C, C), generator=g, device=device) / C ** 0.5

    def _degrees(self):
        return [slice(l * l, (l + 1) ** 2) for l in range(self.L + 1)]

    def _linear(self, w, x):
        return torch.cat([w[l] @ x[:, :, s] for l, s in enumerate(self._degrees())], 2)

    def _linear_backward(self, w, x, dy):
        dx = torch.cat([w[l].T @ dy[:, :, s] for l, s in enumerate(self._degrees())], 2)
        dw = torch.stack([torch.einsum("nim,njm->ij", dy[:, :, s], x[:, :, s]) for s in self._degrees()])
        return dx, dw

    def _heads(self, x):
        return x.reshape(x.shape[0], self.H, -1)

    def forward(self, x, offsets, longest, rng):
        """rng: int64[2, 2] on the device, a generator state for the probabilities and one for the channels."""
        P = self.params
        s = {"x": x, "args": dict(q_off=offsets, k_off=offsets, max_q=longest, max_k=longest, p=self.p, rng=rng[0]),
             "rng": rng}
        s["h"], s["mean"], s["rstd"] = gtp.gtp_layer_norm(x, self.L, P["norm_w"], P["norm_b"])
        s["q"], s["k"], s["v"] = (self._heads(self._linear(P[n], s["h"])) for n in ("wq", "wk", "wv"))
        s["o"], s["lse"] = gtp.gtp_attention(s["q"], s["k"], s["v"], **s["args"])
        a = self._linear(P["wo"], s["o"].view_as(x))
        s["y"] = gtp.gtp_dropout(a, self.p, rng[1], res=x)
        return s["y"] + gtp.gtp_full_weighted(self.plan, s["y"], s["y"], wout=P["wp"]), s

    def backward(self, s, dout):
        P, x = self.params, s["x"]
        pr = gtp.gtp_full_weighted_backward(self.plan, s["y"], s["y"], dout, wout=P["wp"], need=("dx1", "dx2", "dwout"))
        g = {"wp": pr["dwout"]}
        dy = dout + pr["dx1"] + pr["dx2"]
        da = gtp.gtp_dropout(dy, self.p, s["rng"][1])
        do, g["wo"] = self._linear_backward(P["wo"], s["o"].view_as(x), da)
        at = gtp.gtp_attention_backward(s["q"], s["k"], s["v"], s["o"], self._heads(do), s["lse"], **s["args"])
        dh = torch.zeros_like(x)
        for n, d in (("wq", "dq"), ("wk", "dk"), ("wv", "dv")):
            part, g[n] = self._linear_backward(P[n], s["h"], at[d].view_as(x))
            dh += part
        nb = gtp.gtp_layer_norm_backward(x, dh, self.L, s["mean"], s["rstd"], P["norm_w"])
        g["norm_w"], g["norm_b"] = nb["dw"], nb["db"]
        return dy + nb["dx"], g


def molecules(count, atoms, device="cuda", seed=0):
    """Offsets of molecules of about `atoms` atoms, and the longest."""
    n = torch.randint(max(1, atoms // 2), atoms + atoms // 2 + 1, (count,),
                      generator=torch.Generator().manual_seed(seed))
    return torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(device), int(n.max())


def train(count=64, atoms=27, C=64, L=2, heads=8, p=0.1, steps=20, lr=0.1, say=print):
    """The losses (half the squared distance to a fixed target, a channel) of `steps` steps of gradient descent."""
    offsets, longest = molecules(count, atoms)
    T = int(offsets[-1])
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((T, C, (L + 1) ** 2), generator=g, device="cuda")
    target = x + 0.3 * torch.randn(x.shape, generator=g, device="cuda")
    block = Block(C, L, heads, p)
    rng = torch.tensor([[7, 0], [7, 1 << 32]], dtype=torch.int64, device="cuda")
    losses = []
    for step in range(steps):
        out, s = block.forward(x, offsets, longest, rng)
        diff = out - target
        losses.append(float(diff.square().sum()) / (2 * T * C))
        _, grads = block.backward(s, diff / (T * C))
        for n, d in grads.items():
            block.params[n] -= lr * d
        rng[:, 1] += 1  # other draws next step
        say(f"step {step}: loss {losses[-1]:.4f}")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("molecules", 64), ("atoms", 27), ("channels", 64), ("L", 2), ("steps", 20)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args()
    train(a.molecules, a.atoms, a.channels, a.L, steps=a.steps)
