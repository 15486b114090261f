"""One pipeline-stage boundary in 8 bits: forward and backward, on one GPU.

    python -m paper_2211_05322_amd.stage_boundary [--batch 8 --seq 1024 --hidden 4096 --out 4096]

The sending stage holds an activation [batch, seq, hidden] with batch and
hidden sharded over a (2, 4) mesh; the receiving stage wants it with batch and
sequence sharded, hidden whole, on its own (2, 4) mesh.  Each sender takes its
shard to 8 bits (128 divides the hidden shards, so blocks do not cross
devices), two plans move codes and scales -- half the bytes of the 16-bit
reshard, meant for links between GPUs (within one, the 16-bit move is several
times faster) -- and every receiver reads them back, normalises its rows and
multiplies them by the stage's first weights in 8 bits.  On the way back the
receivers take the gradients of the product and of the norm, weight gradients
adding up over the devices as over micro-batches, and the activation's gradient
returns through the reverse plans, in 8 bits too.
"""

from __future__ import annotations

import argparse
import time

import torch

from paper_2211_05322_amd import binding as B

MESH = (2, 4)
SENDER, RECEIVER = "S^0 R S^1", "S^0 S^1 R"


class Boundary:
    """The plans of one boundary and the receiving stage's first weights."""

    def __init__(self, batch, seq, hidden, weight, gamma, beta):
        if hidden % (128 * MESH[1]):
            raise ValueError(f"hidden must be a multiple of {128 * MESH[1]}, so that blocks of 128 do not cross devices")
        self.shape = (batch, seq, hidden)
        blocks = (batch, seq, hidden // 128)
        self.plans = {}
        for way, src, dst in (("forward", SENDER, RECEIVER), ("backward", RECEIVER, SENDER)):
            self.plans[way] = (B.reshard_plan(self.shape, "float8_e4m3fn", MESH, src, MESH, dst),
                               B.reshard_plan(blocks, "float8_e8m0fnu", MESH, src, MESH, dst))
            for plan in self.plans[way]:
                B.reshard_plan_upload(plan)
        self.gamma, self.beta = gamma, beta
        # weights once, in tiles, for both products that read them
        self.weight, self.weight_t = B.reshard_quantize(weight, 128, transposed="both")
        self.dweight = torch.zeros(weight.shape, dtype=torch.float32, device=weight.device)
        self.dgamma, self.dbeta = (torch.zeros(hidden, dtype=torch.float32, device=weight.device) for _ in range(2))

    def move(self, way, shards):
        """16-bit shards across the boundary in 8 bits."""
        sent = [B.reshard_quantize(x, dense=True) for x in shards]
        codes, scales = self.plans[way]
        arrived = [B.empty_shards(codes, 1), B.empty_shards(scales, 1)]
        B.reshard_execute(codes, [b.data for b in sent], arrived[0])
        B.reshard_execute(scales, [b.scales for b in sent], arrived[1])
        return [B.reshard_dequantize(B.Blocked(q, s), shards[0].dtype) for q, s in zip(*arrived)]

    def forward(self, shards):
        """The senders' shards to the receivers' outputs of the first product, and what the backward pass needs."""
        outs, kept = [], []
        for x in self.move("forward", shards):
            y, mean, rstd = B.reshard_layer_norm(x, self.gamma, self.beta)
            rows, columns = B.reshard_quantize(y, transposed="both")
            outs.append(B.reshard_matmul(rows, self.weight, x.dtype))
            kept.append((x, mean, rstd, columns))
        return outs, kept

    def backward(self, grads, kept):
        """The outputs' gradients to the senders' shards' gradients; the weights' gradients are added up."""
        back = []
        for dz, (x, mean, rstd, columns) in zip(grads, kept):
            rows, along_tokens = B.reshard_quantize(dz, transposed="both")
            dy = B.reshard_matmul(rows, self.weight_t, dz.dtype)
            B.reshard_matmul(along_tokens, columns, out=self.dweight, accumulate=True)
            dx, _, _ = B.reshard_layer_norm_backward(dy, x, self.gamma, mean, rstd, self.dgamma, self.dbeta,
                                                     accumulate=True)
            back.append(dx)
        return self.move("backward", back)


def scatter(x, spec):
    """Each device's dense shard of a whole tensor."""
    rep = " ".join("R" * x.dim())
    plan = B.reshard_plan(x.shape, str(x.dtype).replace("torch.", ""), (1,), rep, MESH, spec)
    shards = B.empty_shards(plan, 1)
    B.reshard_execute(plan, [x], shards)
    return shards


def gather(shards, shape, spec):
    """The whole tensor from its shards."""
    rep = " ".join("R" * len(shape))
    plan = B.reshard_plan(shape, str(shards[0].dtype).replace("torch.", ""), MESH, spec, (1,), rep)
    out = B.empty_shards(plan, 1)
    B.reshard_execute(plan, shards, out)
    return out[0]


def example(batch, seq, hidden, out, seed=0, dtype=torch.bfloat16):
    """(boundary, activation, the output's gradient) on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return std * torch.randn(shape, generator=g, device="cuda")
    edge = Boundary(batch, seq, hidden, normal(out, hidden, std=0.02).to(dtype), 1 + normal(hidden, std=0.1),
                    normal(hidden, std=0.1))
    return edge, normal(batch, seq, hidden).to(dtype), normal(batch, seq, out, std=1e-2).to(dtype)


def _ms(f, reps=10):
    f()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(reps):
        f()
    torch.cuda.synchronize()
    return (time.perf_counter() - t) / reps * 1e3


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("batch", 8), ("seq", 1024), ("hidden", 4096), ("out", 4096)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args()
    edge, x, dz = example(a.batch, a.seq, a.hidden, a.out)
    shards, grads = scatter(x, SENDER), scatter(dz, RECEIVER)
    outs, kept = edge.forward(shards)
    back = edge.backward(grads, kept)
    z, dx = gather(outs, dz.shape, RECEIVER), gather(back, x.shape, SENDER)

    # the same in float32, no 8 bits anywhere
    xf = x.float().requires_grad_()
    w = B.reshard_dequantize(edge.weight, torch.float32).requires_grad_()
    y = torch.nn.functional.layer_norm(xf, (a.hidden,), edge.gamma, edge.beta)
    ref = (y.reshape(-1, a.hidden) @ w.t()).view(dz.shape)
    ref.backward(dz.float())
    for name, got, want in (("output", z, ref), ("activation's gradient", dx, xf.grad), ("weights' gradient", edge.dweight, w.grad)):
        rel = ((got.float() - want).norm() / want.norm()).item()
        print(f"{name:24s} off by {100 * rel:.2f} % of its norm from float32 without 8 bits")
    print(f"forward  {_ms(lambda: edge.forward(shards)):.3f} ms")
    print(f"backward {_ms(lambda: edge.backward(grads, kept)):.3f} ms")


if __name__ == "__main__":
    main()
