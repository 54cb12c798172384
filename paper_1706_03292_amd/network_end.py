"""Training the end of a network on one node that stands for P workers: what
makes the payloads, and their synchronisation.

Each worker's features go through dropout, a residual sum and a layer norm (one
pass), then the classifier with its softmax cross entropy.  The backward pass
leaves its results where the synchronisation reads them: the normalisation's
gradients in the workers' dense shards, the classifier's -- by Alg. 1's choice
for its size -- either as this worker's rows of the sufficient factors or as its
dense shard.  One ``SyncIteration`` then updates gamma, beta and the classifier.

``python -m paper_1706_03292_amd.network_end`` trains it on drawn data and
prints the loss of every tenth step.
"""
from __future__ import annotations

import torch

from . import api


class NetworkEnd:
    """Dropout, residual, layer norm and classifier over ``features`` features
    and ``classes`` classes, trained by P workers of B rows each.  Parameters
    are fp32; with ``dtype`` bfloat16 the activations are bf16 and each step
    works on a bf16 copy of the classifier."""

    def __init__(self, classes: int, features: int, B: int, P: int, lr: float, momentum: float = 0.9, p: float = 0.1,
                 dtype: torch.dtype = torch.float32, seed: int = 0, device=None):
        dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.B, self.P, self.p, self.dtype = B, P, p, dtype
        self.W = torch.randn(classes, features, generator=gen, device=dev) * features ** -0.5
        self.gamma, self.beta = torch.ones(features, device=dev), torch.zeros(features, device=dev)
        # a worker's generator: its own seed, the offset counts steps
        self.rng = torch.tensor([[1000003 * seed + w, 0] for w in range(P)], dtype=torch.int64, device=dev)
        self.scheme = api.hybcomm_choose(classes, features, B, P)
        empty = lambda *shape: torch.empty(shape, device=dev)  # noqa: E731
        zeros_like = torch.zeros_like
        self.dgamma, self.dbeta = empty(P, features), empty(P, features)
        fc = {"fc": True, "W": self.W, "buf": zeros_like(self.W)}
        if self.scheme == api.SFB:
            self.U, self.V = empty(P * B, classes), empty(P * B, features)
            fc.update(U=self.U, V=self.V)
        else:
            self.dW = empty(P, classes, features)
            fc.update(shards=self.dW)
        self.pool = api.StreamPool(2, device=dev)
        self.sync = api.SyncIteration(
            self.pool, [{"fc": False, "W": self.gamma, "shards": self.dgamma, "buf": zeros_like(self.gamma)},
                        {"fc": False, "W": self.beta, "shards": self.dbeta, "buf": zeros_like(self.beta)}, fc],
            B, P, lr, momentum)

    def worker_step(self, w: int, x: torch.Tensor, residual: torch.Tensor, target: torch.Tensor,
                    dloss: torch.Tensor, W: torch.Tensor):
        """Worker w's forward and backward pass on its B rows; its payloads are
        written.  Returns (loss of each row, dx, dresidual)."""
        rows = slice(w * self.B, (w + 1) * self.B)
        y, h, mean, rstd = api.norm_forward(x, self.gamma, self.beta, residual=residual, p=self.p, rng=self.rng[w])
        if self.scheme == api.SFB:
            loss, _, dy = api.xent_factor(y, W, target, dloss, U=self.U[rows])
            self.V[rows].copy_(y)
        else:
            loss, lse = api.xent_forward(y, W, target)
            dy, _ = api.xent_backward(y, W, target, lse, dloss, dW=self.dW[w])
        dx, dresidual, _, _ = api.norm_backward(dy, h, self.gamma, mean, rstd, p=self.p, rng=self.rng[w],
                                                dgamma=self.dgamma[w], dbeta=self.dbeta[w])
        return loss, dx, dresidual

    def step(self, x: torch.Tensor, residual: torch.Tensor, target: torch.Tensor):
        """One iteration: every worker's rows (P*B of them, worker after
        worker), then the synchronisation.  Rows without a target (outside the
        classes) count for nothing, whatever they hold.  Returns (mean loss, dx,
        dresidual)."""
        valid = (target >= 0) & (target < self.W.shape[0])
        # Their gradients are 0, but the normalisation's sums and the rebuild from
        # factors multiply those with the rows' values.
        x, residual = (torch.where(valid[:, None], v, torch.zeros_like(v)) for v in (x, residual))
        dloss = valid.float() / valid.sum().clamp(min=1)
        W = self.W if self.dtype == torch.float32 else self.W.to(self.dtype)
        out = []
        for w in range(self.P):
            r = slice(w * self.B, (w + 1) * self.B)
            out.append(self.worker_step(w, x[r], residual[r], target[r], dloss[r], W))
        self.sync()
        self.rng[:, 1] += 1
        loss, dx, dresidual = (torch.cat(t) for t in zip(*out))
        return (loss * dloss).sum(), dx, dresidual

    def close(self) -> None:
        self.pool.close()


def main() -> None:
    classes, features, B, P = 1000, 512, 32, 4
    end = NetworkEnd(classes, features, B, P, lr=0.5, dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(1)
    centre = torch.randn(classes, features, generator=gen, device="cuda")
    for i in range(101):
        target = torch.randint(0, classes, (P * B,), generator=gen, device="cuda")
        x = (centre[target] + torch.randn(P * B, features, generator=gen, device="cuda")).to(end.dtype)
        loss, _, _ = end.step(x, torch.zeros_like(x), target)
        if i % 10 == 0:
            print(f"step {i}: loss {float(loss):.4f} ({'factors' if end.scheme == api.SFB else 'shards'})", flush=True)
    end.close()


if __name__ == "__main__":
    main()
