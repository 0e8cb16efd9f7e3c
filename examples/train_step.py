"""A data-parallel training step around the library's collectives, on one GPU.

P virtual ranks hold the same small residual model (layer norm, linear layer,
over and over) and different data.  One step:

  forward and backward   spccl_layer_norm, spccl_layer_norm_backward (and torch's
                         matrix products); every gradient is written into the
                         rank's flat bucket, the norms' by the backward pass itself
  pruning                spccl_prune: what reaches the threshold is sent, the rest
                         is carried to later steps in the rank's residual
  reduction              spccl_vr_all_reduce over the ranks' buckets
  update                 spccl_adamw_step over all tensors, from the reduced bucket
                         or, with --message, from its Pici message

    python examples/train_step.py [--steps 40] [--state 8|32] [--sparsity 0.9] [--message]

prints the loss of every tenth step.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_04676_amd as S  # noqa: E402

ALIGN = 64          # a tensor of a message starts at a multiple of 64 elements


class Bucket:
    """Named tensors as views of one flat array, as a gradient bucket holds them."""

    def __init__(self, shapes: dict, ranks: int):
        self.shapes, self.starts, at = shapes, {}, 0
        for name, shape in shapes.items():
            self.starts[name] = at
            at += -(-shape.numel() // ALIGN) * ALIGN
        self.total = -(-at // (ranks * ALIGN)) * ranks * ALIGN       # the ring's chunks are equal

    def new(self, dtype=torch.float32) -> torch.Tensor:
        return torch.zeros(self.total, dtype=dtype, device="cuda")

    def view(self, flat: torch.Tensor, name: str) -> torch.Tensor:
        at = self.starts[name]
        return flat[at:at + self.shapes[name].numel()].view(self.shapes[name])


class Model:
    """x <- x + norm(x) W, layer by layer, then norm(x) W_out; its forward and
    backward pass for one rank."""

    def __init__(self, width: int, layers: int, outputs: int, ranks: int, seed: int = 0):
        self.width, self.layers, self.outputs = width, layers, outputs
        size, shapes = torch.Size, {}
        for k in range(layers + 1):
            last = k == layers
            shapes[f"weight{k}"], shapes[f"bias{k}"] = size([width]), size([width])
            shapes[f"linear{k}"] = size([width, outputs if last else width])
        self.bucket = Bucket(shapes, ranks)
        self.params = self.bucket.new()
        g = torch.Generator(device="cuda").manual_seed(seed)
        for name, shape in shapes.items():
            p = self.param(name)
            if name.startswith("linear"):
                p.copy_(torch.randn(shape, generator=g, device="cuda") * width ** -0.5)
            else:
                p.fill_(1.0 if name.startswith("weight") else 0.0)

    def param(self, name):
        return self.bucket.view(self.params, name)

    def forward(self, x):
        """The prediction, and what the backward pass needs."""
        kept = []
        for k in range(self.layers + 1):
            h = torch.empty_like(x)
            mean, rstd = torch.empty(len(x), device="cuda"), torch.empty(len(x), device="cuda")
            S.spccl_layer_norm(x, self.param(f"weight{k}"), self.param(f"bias{k}"), h, mean, rstd)
            kept.append((x, h, mean, rstd))
            out = h @ self.param(f"linear{k}")
            x = out if k == self.layers else x + out
        return x, kept

    def backward(self, kept, grad, flat):
        """Writes every parameter's gradient into the bucket `flat`."""
        x = kept[0][0]
        scratch = torch.empty(max(16, S.spccl_layer_norm_scratch_bytes(*x.shape)), dtype=torch.uint8, device="cuda")
        for k in range(self.layers, -1, -1):
            x, h, mean, rstd = kept[k]
            torch.mm(h.t(), grad, out=self.bucket.view(flat, f"linear{k}"))
            dh = grad @ self.param(f"linear{k}").t()
            dx = torch.empty_like(x)
            S.spccl_layer_norm_backward(dh, x, self.param(f"weight{k}"), mean, rstd, dx,
                                        self.bucket.view(flat, f"weight{k}"), self.bucket.view(flat, f"bias{k}"), scratch)
            grad = dx if k == self.layers else grad + dx
        return grad


class Trainer:
    def __init__(self, model: Model, ranks: int, state: int = 8, sparsity: float = 0.9, message: bool = False,
                 lr: float = 3e-3):
        self.model, self.ranks, self.sparsity, self.message, self.lr, self.t = model, ranks, sparsity, message, lr, 0
        b = model.bucket
        self.grads = [b.new() for _ in range(ranks)]
        self.residuals = [b.new() for _ in range(ranks)]
        self.reduced = [b.new() for _ in range(ranks)]
        self.scratch = torch.empty(S.spccl_vr_scratch_bytes(ranks, b.total // ranks, S.SPCCL_F32), dtype=torch.uint8,
                                   device="cuda")
        self.ws = S.alloc_workspace(b.total, S.SPCCL_F32)
        self.scale = torch.tensor([1.0 / ranks], device="cuda")      # the mean over the ranks
        self.msg = S.alloc_stream(b.total, S.SPCCL_F32) if message else None
        kind = S.SPCCL_STATE_F8 if state == 8 else S.SPCCL_STATE_F32
        self.states, tensors = {}, []
        for name, shape in b.shapes.items():
            self.states[name] = S.alloc_adamw_state(shape.numel(), kind)
            grad = dict(grad=b.view(self.reduced[0], name))
            if message:
                grad = dict(grad=S.operand(self.msg, S.SPCCL_STREAM, S.SPCCL_FMT_PICI), grad_dtype=S.SPCCL_F32,
                            grad_offset=b.starts[name], grad_n=b.total)
            decay = 0.01 if name.startswith("linear") else 0.0
            tensors.append(S.adamw_tensor(model.param(name), weight_decay=decay, **grad, **self.states[name]))
        self.table = torch.empty(S.spccl_adamw_plan_bytes(tensors), dtype=torch.uint8, device="cuda")
        self.plan = S.spccl_adamw_plan(tensors, self.table)

    def threshold(self, rank: int) -> torch.Tensor:
        """The magnitude that the wanted share of a sample of the gradient lies below."""
        sample = (self.grads[rank][::7] + self.residuals[rank][::7]).abs()
        return torch.quantile(sample, self.sparsity).reshape(1)

    def step(self, data) -> float:
        """One step over the ranks' (input, target) pairs; the mean loss before it."""
        loss = torch.zeros((), device="cuda")
        for r, (x, y) in enumerate(data):
            pred, kept = self.model.forward(x)
            err = pred - y
            loss += err.square().mean() / self.ranks
            self.model.backward(kept, err * (2.0 / err.numel()), self.grads[r])
            if self.sparsity > 0:
                S.spccl_prune(self.grads[r], self.residuals[r], self.threshold(r), 1.0, self.grads[r])
        S.spccl_vr_all_reduce(self.grads, self.reduced, self.scratch)
        if self.message:
            S.spccl_compress(self.reduced[0], self.msg, self.ws)
        self.t += 1
        S.spccl_adamw_step(self.plan, self.ws, self.lr, step=self.t, seed=self.t, grad_scale=self.scale)
        return float(loss)


def batches(model: Model, ranks: int, rows: int, seed: int = 1):
    """Inputs and a fixed random teacher's outputs, other ones for each rank."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    teacher = torch.randn(model.width, model.outputs, generator=g, device="cuda") * model.width ** -0.5
    out = []
    for _ in range(ranks):
        x = torch.randn(rows, model.width, generator=g, device="cuda")
        out.append((x, torch.tanh(x @ teacher)))
    return out


def train(steps: int = 40, ranks: int = 4, width: int = 256, layers: int = 2, rows: int = 512, state: int = 8,
          sparsity: float = 0.9, message: bool = False, say=None):
    """The losses of `steps` steps and the trainer."""
    model = Model(width, layers, 32, ranks)
    trainer = Trainer(model, ranks, state, sparsity, message)
    data = batches(model, ranks, rows)
    losses = []
    for t in range(steps):
        losses.append(trainer.step(data))
        if say and (t % 10 == 0 or t == steps - 1):
            say(f"step {t:4d}  loss {losses[-1]:.5f}")
    if S.spccl_read_status(trainer.ws):
        raise RuntimeError("the library reports a device error")
    return losses, trainer


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--ranks", type=int, default=4)
    ap.add_argument("--state", type=int, choices=(8, 32), default=8)
    ap.add_argument("--sparsity", type=float, default=0.9)
    ap.add_argument("--message", action="store_true", help="give the step the reduced gradient as a Pici message")
    a = ap.parse_args()
    train(a.steps, a.ranks, state=a.state, sparsity=a.sparsity, message=a.message, say=print)


if __name__ == "__main__":
    main()
