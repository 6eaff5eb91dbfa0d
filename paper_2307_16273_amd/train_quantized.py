"""Trains a small residual network in 8-bit integers on the GPU, answers with it row by row, and proves the forward products of its last step.

    python -m paper_2307_16273_amd.train_quantized [--layers 8] [--width 1024] [--batch 64] [--steps 5] [--lr X]

Layer l normalises the residual stream, in 8 bits with a scale for each row, and multiplies it by its weights, in 8 bits with a scale for
each column; its output is added to the stream by the next layer's norm.  Gradients go back through the same integers.  The target is the
output of a network of other weights; the loss is half the mean square of the difference.  After the last step
  - the forward pass runs once more for single rows, as a serving program would, and has to give the batch's rows bit for bit;
  - sumcheck_matmul proves the products of all layers on the stacks of 8-bit activations and weights, and its claim on their result is
    compared with the multilinear extension of the int32 accumulators that matmul_i8 returns.  (The integers of the gradients stay inside
    matmul_i8_backward and are not proved.)
One line of JSON for each step and for what follows.  Layers, width and batch are powers of two, as the proof wants them.
"""
import argparse
import json
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def forward(zk, ctx, x, net):
    """Returns the network's output and what the backward pass needs of each layer."""
    kept, stream, y = [], x, None
    for wq, sw, gain in zip(net["q"], net["s"], net["gain"]):
        n = zk.rmsnorm_i8(ctx, stream if y is None else y, gain, residual=None if y is None else stream)
        if y is not None:
            stream = n["total"]
        y = zk.matmul_i8(ctx, n["q"], wq, n["scale"], sw, dtype=x.dtype)
        kept.append((n, stream))
    return stream.float() + y.float(), kept


def quantise_weights(zk, ctx, net):
    got = zk.quantize_i8(ctx, net["w"], axis=-2)
    net["stack"], net["q"], net["s"] = got["q"], list(got["q"]), list(got["scale"])


def network(torch, zk, ctx, layers, width, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    net = dict(w=torch.randn(layers, width, width, generator=g, device="cuda") * (1.0 / width) ** 0.5,
               gain=[torch.ones(width, device="cuda") for _ in range(layers)])
    quantise_weights(zk, ctx, net)
    return net


def step(zk, ctx, x, target, net, lr):
    """One step of gradient descent; returns the loss in front of it (a tensor) and the step's kept activations."""
    out, kept = forward(zk, ctx, x, net)
    diff = out - target
    loss = 0.5 * diff.square().mean()
    d = (diff / x.shape[0]).to(x.dtype)         # the mean over the rows; over the columns it is the learning rate's
    used = net["stack"]
    for l in reversed(range(len(kept))):
        n, stream = kept[l]
        back = zk.matmul_i8_backward(ctx, d, n["q"], n["scale"], net["q"][l], net["s"][l])
        norm = zk.rmsnorm_i8_backward(ctx, back["da"], stream, net["gain"][l], n["rstd"], dtotal=d)
        net["w"][l].sub_(back["dw"], alpha=lr)
        net["gain"][l].sub_(norm["dweight"], alpha=lr)
        d = norm["dx"]
    quantise_weights(zk, ctx, net)
    return loss, kept, used


def prove(torch, zk, ctx, kept, weights):
    """Proof of all layers' products; returns its dict and whether its claim is the accumulators' multilinear extension."""
    acts = torch.stack([n["q"] for n, _ in kept])
    acc = zk.matmul_i8(ctx, acts, weights)
    a = zk.tensor_wrap_int(ctx, acts.to(torch.int32))
    w = zk.tensor_wrap_int(ctx, weights.to(torch.int32))
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    res = zk.sumcheck_matmul(ctx, a, w, zk.Transcript(7))
    ms = 1e3 * (time.perf_counter() - t0)
    layers, rows, cols = acc.shape
    point = res["points"][:layers.bit_length() + rows.bit_length() + cols.bit_length() - 3]
    at = zk.mle_partial_eval(ctx, zk.tensor_wrap_int(ctx, acc), 0, 3, point)
    return res, ms, int.from_bytes(at.download(), "little") == res["claims"][0]


def check(layers, width, batch, steps):
    for name, n in (("layers", layers), ("width", width), ("batch", batch)):
        if n < 1 or n & (n - 1):
            raise ValueError(f"{name}: a power of two is needed for the proof, not {n}")
    if steps < 1:
        raise ValueError(f"steps: at least one is needed, whose products are proved, not {steps}")


def run(layers=8, width=1024, batch=64, steps=5, lr=None, say=print):
    check(layers, width, batch, steps)
    import torch
    if lr is None:
        # Steps below 2 / (largest curvature) shrink the loss.  A layer's is about the largest eigenvalue of n^T n / batch, for random
        # rows (1 + sqrt(width / batch))^2, and the layers add up along the stream.
        lr = 0.5 / (layers * (1 + (width / batch) ** 0.5) ** 2)
    import paper_2307_16273_amd as zk
    ctx = zk.Context(0)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(batch, width, generator=g, device="cuda").to(torch.bfloat16)
    target, _ = forward(zk, ctx, x, network(torch, zk, ctx, layers, width, 2))
    net = network(torch, zk, ctx, layers, width, 3)
    losses, kept, used = [], None, None
    for k in range(steps):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        loss, kept, used = step(zk, ctx, x, target, net, lr)
        losses.append(float(loss))
        say(json.dumps({"step": k, "loss": losses[-1], "step_ms": 1e3 * (time.perf_counter() - t0)}))
    whole, _ = forward(zk, ctx, x, net)
    rows_equal = all(torch.equal(forward(zk, ctx, x[i:i + 1], net)[0], whole[i:i + 1]) for i in range(min(batch, 4)))
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(20):
        forward(zk, ctx, x[:1], net)
    torch.cuda.synchronize()
    say(json.dumps({"rows_equal": rows_equal, "single_row_us": 1e6 / 20 * (time.perf_counter() - t0)}))
    res, ms, holds = prove(torch, zk, ctx, kept, used)
    say(json.dumps({"proof_ms": ms, "proof_bytes": len(res["proof"]), "claim_is_the_accumulators": holds}))
    ctx.close()
    return losses, rows_equal, holds


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--lr", type=float, default=None)
    args = ap.parse_args()
    try:
        check(args.layers, args.width, args.batch, args.steps)
    except ValueError as e:
        ap.error(str(e))
    run(args.layers, args.width, args.batch, args.steps, args.lr, lambda s: print(s, flush=True))


if __name__ == "__main__":
    main()
