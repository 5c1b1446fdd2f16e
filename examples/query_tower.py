"""Trains a query tower with 8-bit products and searches a product-quantized index with the vectors it makes.

Every token stands for one vector of a base set.  The tower looks a token's row up, passes it through a residual layer
(root-mean-square norm, 8-bit product) and projects it (norm, 8-bit product) to a query vector, which should come to lie
near the token's base vector; its gradients are 8-bit products too, along the other sides of the same matrices.  The base set is
encoded with a product quantizer; before and after training, the tower's query vectors search the codes, and the
results are ranked again with the base vectors looked up by id.

    python examples/query_tower.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1812_09162_amd import binding as qb  # noqa: E402

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


class Tower:
    """table [tokens, width], two norms and two weight matrices (float32 masters), with Adam."""

    def __init__(self, tokens, width, d, seed, device):
        g = torch.Generator(device=device).manual_seed(seed)
        self.p = {
            "table": torch.randn((tokens, width), generator=g, device=device) * width ** -0.5,
            "norm1": torch.ones(width, device=device), "norm2": torch.ones(width, device=device),
            "w1": torch.randn((width, width), generator=g, device=device) * width ** -0.5,
            "w2": torch.randn((d, width), generator=g, device=device) * width ** -0.5,
        }
        self.m = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.v = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.scale, self.step = width ** 0.5, 0

    def forward(self, ids):
        """Query vectors [n, d] float32, and what the backward pass reads."""
        p = self.p
        x = qb.vec_lookup(p["table"], ids, scale=self.scale, dtype=torch.bfloat16)
        y1, _, q1, s1 = qb.vec_norm(x, p["norm1"], quant=E4M3)
        u = qb.vec_matmul_blocks(q1, s1, *qb.vec_quantize_blocks(p["w1"]))
        y2, h, q2, s2 = qb.vec_norm(u, p["norm2"], residual=x, quant=E4M3)
        z = qb.vec_matmul_blocks(q2, s2, *qb.vec_quantize_blocks(p["w2"]), dtype=torch.float32)
        return z, (ids, x, y1, y2, h)

    def backward(self, dz, kept):
        """Gradients of all parameters from that of the query vectors."""
        p, (ids, x, y1, y2, h) = self.p, kept

        def product(dy, y, w):
            """dy w and dy^T y: gradients of the input and the weights of y w^T."""
            dx = qb.vec_matmul_blocks(*qb.vec_quantize_blocks(dy, dtype=E5M2), *qb.vec_quantize_blocks(w, transposed=True))
            dw = qb.vec_matmul_blocks(*qb.vec_quantize_blocks(dy, dtype=E5M2, transposed=True), *qb.vec_quantize_blocks(y, transposed=True),
                                      dtype=torch.float32)
            return dx, dw

        dy2, dw2 = product(dz.to(torch.bfloat16), y2, p["w2"])
        dh, dnorm2 = qb.vec_norm_grad(dy2, h, p["norm2"])
        dy1, dw1 = product(dh, y1, p["w1"])
        dx, dnorm1 = qb.vec_norm_grad(dy1, x, p["norm1"], dh=dh)
        dtable = qb.vec_lookup_grad(dx, ids, p["table"].shape[0], scale=self.scale, dtype=torch.float32)
        return {"table": dtable, "norm1": dnorm1, "norm2": dnorm2, "w1": dw1, "w2": dw2}

    def update(self, grads, lr):
        self.step += 1
        for k, g in grads.items():
            self.m[k].lerp_(g, 0.1)
            self.v[k].lerp_(g * g, 0.01)
            m, v = self.m[k] / (1 - 0.9 ** self.step), self.v[k] / (1 - 0.99 ** self.step)
            self.p[k] -= lr * m / (v.sqrt() + 1e-8)


def encode(base, m=16, bits=4, rounds=5):
    """A product quantizer for the base vectors (k-means per sub-space) and their codes."""
    n, d = base.shape
    width, k = d // m, 1 << bits
    x = base.view(n, m, width).transpose(0, 1).contiguous()
    c = x[:, torch.randperm(n, device=base.device, generator=torch.Generator(device=base.device).manual_seed(0))[:k]].contiguous()
    for _ in range(rounds):
        near = torch.cdist(x, c).argmin(2)
        for j in range(m):
            c[j] = torch.stack([x[j][near[j] == i].mean(0) if bool((near[j] == i).any()) else c[j, i] for i in range(k)])
    index = qb.PqIndex(d, [bits] * m, [width] * m, c.reshape(-1).contiguous(), 8)
    return index, qb.pq_encode(index, base)


def recall(tower, index, codes, base, target, R=100):
    """Shares of tokens whose base vector is among the R results, and the first of them after ranking again."""
    z, _ = tower.forward(torch.arange(target.numel(), device=base.device))
    ids, _, _ = qb.pq_search_topk(index, z, codes, 400, R)
    found = (ids == target[:, None]).any(1).float().mean()
    rows = qb.vec_lookup(base, ids)  # (padding, id -1, would come back as zeros)
    best = ids.gather(1, (rows - z[:, None]).square().sum(2).argmin(1, keepdim=True))[:, 0]
    return float(found), float((best == target).float().mean())


def main(steps=400, tokens=2000, n=20_000, width=256, d=96, batch=1024, seed=0):
    """(first loss, last loss, recalls before, recalls after)"""
    device = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=device).manual_seed(seed)
    base = torch.randn((n, d), generator=g, device=device)
    base /= base.norm(dim=1, keepdim=True)
    target = torch.randint(0, n, (tokens,), generator=g, device=device)
    index, codes = encode(base)
    tower = Tower(tokens, width, d, seed, device)
    before, losses = recall(tower, index, codes, base, target), []
    for i in range(steps):
        ids = torch.randint(0, tokens, (batch,), generator=g, device=device)
        z, kept = tower.forward(ids)
        off = z - base[target[ids]]
        losses.append(off.square().sum(1).mean())
        tower.update(tower.backward(off * (2.0 / batch), kept), lr=0.003)
    after = recall(tower, index, codes, base, target)
    index.close()
    return float(losses[0]), float(losses[-1]), before, after


if __name__ == "__main__":
    first, last, before, after = main(int(sys.argv[1]) if len(sys.argv) > 1 else 400)
    print(f"mean squared distance to the base vectors: {first:.3f} at first, {last:.4f} at last")
    print(f"among 100 results {before[0]:.3f} -> {after[0]:.3f}, first after ranking again {before[1]:.3f} -> {after[1]:.3f}")
