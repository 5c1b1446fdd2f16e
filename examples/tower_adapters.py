"""Trains low-rank adapters of several collections over one shared query tower, and serves them together.

The tower (a table of token vectors, a norm, a projection in 8 bits) is frozen and shared.  Every collection has its own base vectors and its
own pair of small matrices beside the projection, trained with dropout of their input and of the tower's vectors; a batch mixes rows of all
collections, each with the id of its adapter, some with none.  The gradient reaches the token vectors past the projection and through the
adapters.  Afterwards one batch of single tokens, of whatever collections, is projected in one call, and the vectors search each collection's codes.

    python examples/tower_adapters.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paper_1812_09162_amd import binding as qb  # noqa: E402
from query_tower import encode  # noqa: E402

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


class SharedTower:
    """table [tokens, width] and norm (trained), projection [d, width] in 8 bits (frozen); adapters a [collections, rank, width], b [collections, rank, d]."""

    def __init__(self, tokens, width, d, collections, rank, seed, device, p=0.1):
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device=device)  # noqa: E731
        self.p = {"table": rand(tokens, width) * width ** -0.5, "norm": torch.ones(width, device=device),
                  "a": rand(collections, rank, width) * width ** -0.5, "b": torch.zeros(collections, rank, d, device=device)}
        w = rand(d, width) * width ** -0.5
        self.w, self.wt = qb.vec_quantize_blocks(w), qb.vec_quantize_blocks(w, transposed=True)
        self.scale, self.rate = width ** 0.5, p
        self.scales = torch.full((collections,), 2.0, device=device)  # of each adapter
        self.state = torch.tensor([seed, 0], device=device)           # dropout's seed and step
        self.m = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.v = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.step = 0

    def forward(self, ids, which, train=False):
        """Vectors [n, d] float32 of tokens `ids`, each with adapter `which` (-1: none), and what the backward pass reads."""
        bf16, rate = torch.bfloat16, self.rate if train else 0.0
        x = qb.vec_lookup(self.p["table"], ids, scale=self.scale, dtype=bf16)
        h = qb.vec_dropout(x, rate, self.state, layer=0) if train else x
        y, _, q, s = qb.vec_norm(h, self.p["norm"], quant=E4M3)
        z = qb.vec_matmul_blocks(q, s, *self.w, dtype=torch.float32)
        a, b = self.p["a"].to(bf16), self.p["b"].to(bf16)
        z, t = qb.vec_adapter(y, a, b, which, scales=self.scales, base=z, p=rate, state=self.state, layer=1, want_t=train, out=None if train else (z, None))
        return z, (ids, which, h, y, t, a, b)

    def backward(self, dz, kept):
        """Gradients of the table, the norm and the adapters from that of the vectors."""
        ids, which, h, y, t, a, b = kept
        dz = dz.to(torch.bfloat16)
        dy = qb.vec_matmul_blocks(*qb.vec_quantize_blocks(dz, dtype=E5M2), *self.wt)  # past the adapters
        dy, da, db = qb.vec_adapter_grad(dz, y, t, a, b, which, scales=self.scales, dx_base=dy, p=self.rate, state=self.state, layer=1)
        dh, dnorm = qb.vec_norm_grad(dy, h, self.p["norm"])
        dx = qb.vec_dropout(dh, self.rate, self.state, layer=0)
        dtable = qb.vec_lookup_grad(dx, ids, self.p["table"].shape[0], scale=self.scale, dtype=torch.float32)
        return {"table": dtable, "norm": dnorm, "a": da, "b": db}

    def update(self, grads, lr):
        self.step += 1
        self.state[1] += 1  # other masks from now on
        for k, g in grads.items():
            self.m[k].lerp_(g, 0.1)
            self.v[k].lerp_(g * g, 0.01)
            self.p[k] -= lr * (self.m[k] / (1 - 0.9 ** self.step)) / ((self.v[k] / (1 - 0.99 ** self.step)).sqrt() + 1e-8)


def main(steps=400, tokens=300, n=4000, collections=4, width=256, d=96, rank=16, batch=1024, seed=0):
    """(first loss, last loss, shares of tokens whose vector is among the 100 results of each collection)"""
    device = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=device).manual_seed(seed)
    base = torch.randn((collections, n, d), generator=g, device=device)
    base /= base.norm(dim=2, keepdim=True)
    target = torch.randint(0, n, (collections, tokens), generator=g, device=device)
    tower, losses = SharedTower(tokens, width, d, collections, rank, seed, device), []
    for _ in range(steps):
        ids = torch.randint(0, tokens, (batch,), generator=g, device=device)
        which = torch.randint(-1, collections, (batch,), generator=g, device=device)
        z, kept = tower.forward(ids, which, train=True)
        off = torch.where((which >= 0)[:, None], z - base[which.clamp(min=0), target[which.clamp(min=0), ids]], 0.0)  # rows without an adapter: no target
        losses.append(off.square().sum() / (which >= 0).sum())
        tower.update(tower.backward(off * (2.0 / batch), kept), lr=0.003)
    # all tokens of all collections in one call
    every = torch.arange(tokens, device=device).repeat(collections)
    which = torch.arange(collections, device=device).repeat_interleave(tokens)
    z = tower.forward(every, which)[0].view(collections, tokens, d)
    found = []
    for c in range(collections):
        index, codes = encode(base[c].contiguous())
        ids, _, _ = qb.pq_search_topk(index, z[c].contiguous(), codes, 400, 100)
        found.append(float((ids == target[c][:, None]).any(1).float().mean()))
        index.close()
    return float(losses[0]), float(losses[-1]), found


if __name__ == "__main__":
    first, last, found = main(int(sys.argv[1]) if len(sys.argv) > 1 else 400)
    print(f"mean squared distance to the base vectors: {first:.3f} at first, {last:.4f} at last")
    print("among 100 results, by collection: " + ", ".join(f"{f:.3f}" for f in found))
