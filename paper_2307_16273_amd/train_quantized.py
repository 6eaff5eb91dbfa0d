"""Trains a small residual network in 8-bit integers on the GPU, answers with it row by row, and proves the forward products of its last step.

    python -m paper_2307_16273_amd.train_quantized [--layers 8] [--width 1024] [--batch 64] [--steps 5] [--lr X]
        [--loss squares|policy|preference] [--optimizer sgd|adamw] [--state-bits 32|8] [--limit X]

Layer l normalises the residual stream, in 8 bits with a scale for each row, and multiplies it by its weights, in 8 bits with a scale for
each column; its output is added to the stream by the next layer's norm.  Gradients go back through the same integers.  A network of other
weights is the teacher.  By --loss the network learns
  squares     the teacher's output: half the mean square of the difference;
  policy      to choose: its output is the logits of a choice of one entry for each row, choices are drawn from it at every other step, and an
              entry's reward is its log-probability under the teacher's output; policy_loss, with the network of before as the reference;
  preference  the teacher's preferences: rows 2 i and 2 i + 1 ask the same, each answered by an entry drawn from the network of before, and
              the answer that the teacher finds likelier is preferred; preference_loss, with the network of before as the reference.
adamw updates all tensors with one call, its states in 32 or 8 bits; --limit scales gradients whose norm is above it, and leaves a step out whose
norm is not finite.  After the last step
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


def squares(zk, ctx, target):
    """An objective: from the network's output its loss (a tensor) and the gradient of the output."""
    def of(out):
        diff = out - target
        return 0.5 * diff.square().mean(), diff / out.shape[0]       # the mean over the rows; over the columns it is the learning rate's
    return of


def draw(torch, logits, seed):
    return torch.multinomial(torch.softmax(logits, 1), 1, generator=torch.Generator(device="cuda").manual_seed(seed))[:, 0]


def policy(torch, zk, ctx, teacher, before):
    """teacher, before: outputs for the batch of the teacher and of the network before the first step."""
    held, steps = {}, 0

    def of(out):
        nonlocal steps
        if steps % 2 == 0:
            tokens = draw(torch, out, 100 + steps)
            reward = zk.token_logprobs(ctx, teacher, tokens)["logp"]
            held.update(tokens=tokens, old=zk.token_logprobs(ctx, out, tokens)["logp"], ref=zk.token_logprobs(ctx, before, tokens)["logp"],
                        advantage=(reward - reward.mean()) / (reward.std(correction=0) + 1e-6))
        steps += 1
        got = zk.policy_loss(ctx, out, held["tokens"], held["old"], held["advantage"], ref_logp=held["ref"], kl=0.01)
        return got["loss"], got["dlogits"]
    return of


def preference(torch, zk, ctx, teacher, before):
    tokens = draw(torch, before, 100)
    likely = zk.token_logprobs(ctx, teacher, tokens)["logp"].view(-1, 2)
    tokens = torch.where((likely[:, :1] >= likely[:, 1:]), tokens.view(-1, 2), tokens.view(-1, 2).flip(1)).reshape(-1)
    ref = zk.token_logprobs(ctx, before, tokens)["logp"]
    offsets = torch.arange(before.shape[0] + 1, device="cuda")      # sequences of one row each

    def of(out):
        got = zk.preference_loss(ctx, out, tokens, offsets, ref_logp=ref, beta=0.5)
        return got["loss"], got["dlogits"]
    return of


def sgd(torch, zk, ctx, net, lr, limit):
    def update(dw, dgain):
        if limit:       # a norm that is not finite leaves the step out: its factor would turn every weight to NaN
            factor = zk.gradient_norm(ctx, dw + dgain, limit)["factor"]
            whole, none = torch.isfinite(factor), torch.zeros((), device="cuda")
            dw, dgain = ([torch.where(whole, d * factor, none) for d in l] for l in (dw, dgain))
        for l in range(len(dw)):
            net["w"][l].sub_(dw[l], alpha=lr)
            net["gain"][l].sub_(dgain[l], alpha=lr)
    return update


def adamw(zk, ctx, net, lr, limit, bits):
    params = list(net["w"]) + net["gain"]
    state, steps = zk.adamw_state(params, bits), 0

    def update(dw, dgain):
        nonlocal steps
        steps += 1
        factor = zk.gradient_norm(ctx, dw + dgain, limit)["factor"] if limit else None
        zk.adamw_step(ctx, params, dw + dgain, state, steps, lr, factor=factor)
    return update


def step(zk, ctx, x, objective, net, update):
    """One step; returns the loss in front of it (a tensor) and the step's kept activations."""
    out, kept = forward(zk, ctx, x, net)
    loss, d = objective(out)
    d = d.to(x.dtype)
    used = net["stack"]
    dw, dgain = [], []
    for l in reversed(range(len(kept))):
        n, stream = kept[l]
        back = zk.matmul_i8_backward(ctx, d, n["q"], n["scale"], net["q"][l], net["s"][l])
        norm = zk.rmsnorm_i8_backward(ctx, back["da"], stream, net["gain"][l], n["rstd"], dtotal=d)
        dw.insert(0, back["dw"])
        dgain.insert(0, norm["dweight"])
        d = norm["dx"]
    update(dw, dgain)
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


LOSSES, OPTIMIZERS, BITS = ("squares", "policy", "preference"), ("sgd", "adamw"), (32, 8)


def check(layers, width, batch, steps, loss="squares", optimizer="sgd", state_bits=32, limit=None):
    for name, x, known in (("loss", loss, LOSSES), ("optimizer", optimizer, OPTIMIZERS), ("state_bits", state_bits, BITS)):
        if x not in known:
            raise ValueError(f"{name}: one of {', '.join(map(str, known))}, not {x}")
    if loss == "preference" and batch == 1:
        raise ValueError("batch: two rows at least are needed, answers come in pairs")
    if limit is not None and not limit > 0:
        raise ValueError(f"limit: a positive norm, not {limit}")
    for name, n in (("layers", layers), ("width", width), ("batch", batch)):
        if n < 1 or n & (n - 1):
            raise ValueError(f"{name}: a power of two is needed for the proof, not {n}")
    if steps < 1:
        raise ValueError(f"steps: at least one is needed, whose products are proved, not {steps}")


def run(layers=8, width=1024, batch=64, steps=5, lr=None, say=print, loss="squares", optimizer="sgd", state_bits=32, limit=None):
    check(layers, width, batch, steps, loss, optimizer, state_bits, limit)
    import torch
    if lr is None and optimizer == "adamw":
        # The first steps move every weight by about lr, all in the direction that counts: a row of normalised activations answers by lr times
        # the sum of their magnitudes, up to `width`, in each layer.  All layers together move an output by about a quarter.
        lr = 0.25 / (layers * width)
    if lr is None:
        # Steps below 2 / (largest curvature) shrink the loss.  A layer's is about the largest eigenvalue of n^T n / batch, for random
        # rows (1 + sqrt(width / batch))^2, and the layers add up along the stream.
        lr = 0.5 / (layers * (1 + (width / batch) ** 0.5) ** 2)
    import paper_2307_16273_amd as zk
    ctx = zk.Context(0)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(batch, width, generator=g, device="cuda").to(torch.bfloat16)
    if loss == "preference":
        x = x[::2].repeat_interleave(2, 0)
    target, _ = forward(zk, ctx, x, network(torch, zk, ctx, layers, width, 2))
    net = network(torch, zk, ctx, layers, width, 3)
    if loss == "squares":
        objective = squares(zk, ctx, target)
    else:
        objective = (policy if loss == "policy" else preference)(torch, zk, ctx, target, forward(zk, ctx, x, net)[0])
    update = sgd(torch, zk, ctx, net, lr, limit) if optimizer == "sgd" else adamw(zk, ctx, net, lr, limit, state_bits)
    losses, kept, used = [], None, None
    for k in range(steps):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        value, kept, used = step(zk, ctx, x, objective, net, update)
        losses.append(float(value))
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
    ap.add_argument("--loss", default="squares")
    ap.add_argument("--optimizer", default="sgd")
    ap.add_argument("--state-bits", type=int, default=32)
    ap.add_argument("--limit", type=float, default=None)
    args = ap.parse_args()
    how = dict(loss=args.loss, optimizer=args.optimizer, state_bits=args.state_bits, limit=args.limit)
    try:
        check(args.layers, args.width, args.batch, args.steps, **how)
    except ValueError as e:
        ap.error(str(e))
    run(args.layers, args.width, args.batch, args.steps, args.lr, lambda s: print(s, flush=True), **how)


if __name__ == "__main__":
    main()
