#!/usr/bin/env python
"""A scale-only training step of a mixture-of-experts layer, from its router to the loss.

One layer of E frozen FP4 experts (gate, up and down projections, SwiGLU) with a residual
connection under a frozen vocabulary projection; the block scales of the experts train. Every
step runs

    sq_route, sq_sort_tokens, sq_dispatch       tokens to the rows of their experts
    sq_grouped_project_scales, sq_grouped_fwd   the experts with their current scales
    sq_combine                                  rows back to their tokens, weighted
    sq_head_loss_grad                           loss and the gradient that the backward pass starts from
    sq_combine_grad                             ... to the experts' rows and the routing weights
    sq_grouped_bwd_dx, sq_grouped_scale_grad    ... through the experts to rows and scales
    sq_dispatch_grad, sq_route_grad             ... to the tokens and the router's logits

    python examples/moe_step.py [--tokens 512] [--steps 10] ...
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2609_04526_gb300 as sq  # noqa: E402
from paper_2609_04526_gb300 import synth  # noqa: E402

LINEARS = ("gate", "up", "down")


class Layer:
    """E experts of width hidden -> inter -> hidden, top_k per token, and a vocabulary projection.
    `latent` holds the trained scales of each linear, fp32 [E, N, K / block]."""

    def __init__(self, fmt, E, top_k, hidden, inter, vocab, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.fmt, self.E, self.top_k = fmt, E, top_k
        self.weights, self.latent = {}, {}
        for name in LINEARS:
            n, k = (hidden, inter) if name == "down" else (inter, hidden)
            parts = [synth.quantize_rtn(torch.randn(n, k, generator=g, device=device) * k ** -0.5, fmt) for _ in range(E)]
            codes, scales = (torch.stack([getattr(p, a) for p in parts]).contiguous() for a in ("codes", "scales"))
            w = sq.GroupedWeight(fmt, E, n, k, codes, scales, [p.ws2 for p in parts])
            self.weights[name] = w
            self.latent[name] = _effective(w)
        self.router = torch.randn(E, hidden, generator=g, device=device) * hidden ** -0.5
        self.head = (torch.randn(vocab, hidden, generator=g, device=device) * 2 * hidden ** -0.5).bfloat16()


def _effective(w):
    """fp32 scale of each block: its byte on the E4M3 or E8M0 grid, times the tensor scale."""
    if w.fmt == sq.MXFP4:
        return torch.ldexp(torch.ones((), device=w.scales.device), w.scales.int() - 127)
    return w.scales.view(torch.float8_e4m3fn).float() * torch.tensor(w.ws2, device=w.scales.device)[:, None, None]


def step(h, layer, X, labels, valid=None):
    """Loss (fp32 [T]) of hidden rows X (bf16 [T, hidden]) for their labels and, of the mean loss over
    the labelled tokens, the gradients of the latent scales, of X (without the residual path's) and of
    the router's logits."""
    fmt, k = layer.fmt, layer.top_k
    bytes_, masks, now = {}, {}, {}
    for name, w in layer.weights.items():  # the trained scales on their grid, as they would be merged
        bytes_[name], masks[name] = h.sq_grouped_project_scales(w, layer.latent[name])
        now[name] = sq.GroupedWeight(fmt, w.E, w.N, w.K, w.codes, bytes_[name], w.ws2)

    logits = X.float() @ layer.router.t()
    experts, weights = h.sq_route(logits, k, valid=valid)
    offsets, row_of, slot_of = h.sq_sort_tokens(experts, layer.E)
    rows = offsets.tolist()  # the grouped calls take them from the host
    Xs = h.sq_dispatch(X, row_of, slot_of)
    gate, up = (torch.zeros(Xs.shape[0], now[n].N, dtype=Xs.dtype, device=Xs.device) for n in ("gate", "up"))
    h.sq_grouped_fwd(now["gate"], rows, Xs, Y=gate)
    h.sq_grouped_fwd(now["up"], rows, Xs, Y=up)
    act = torch.nn.functional.silu(gate) * up
    Ys = torch.zeros_like(Xs)
    h.sq_grouped_fwd(now["down"], rows, act, Y=Ys)
    out = X + h.sq_combine(Ys, row_of, weights)

    targets = (labels >= 0) & (labels < layer.head.shape[0])
    dloss = targets.float() / targets.sum().clamp(min=1)
    loss, _, dout = h.sq_head_loss_grad(out, layer.head, labels, dloss)

    dYs, dweights = h.sq_combine_grad(dout, Ys, row_of, slot_of, weights)
    grads = {"down": h.sq_grouped_scale_grad(layer.weights["down"], rows, act, dYs, mask=masks["down"])}
    dact = torch.zeros_like(act)
    h.sq_grouped_bwd_dx(now["down"], rows, dYs, dX=dact)
    sig = torch.sigmoid(gate)
    dgate, dup = dact * up * sig * (1 + gate * (1 - sig)), dact * gate * sig
    dXs = torch.zeros_like(Xs)
    part = torch.zeros_like(Xs)
    for name, d in (("gate", dgate), ("up", dup)):
        grads[name] = h.sq_grouped_scale_grad(layer.weights[name], rows, Xs, d, mask=masks[name])
        h.sq_grouped_bwd_dx(now[name], rows, d, dX=part)
        dXs += part
    dX = h.sq_dispatch_grad(dXs, row_of)
    dlogits = h.sq_route_grad(logits, experts, dweights)
    return {"loss": loss, "scale_grads": grads, "dX": dX, "dlogits": dlogits, "rows": rows, "out": out}


def batch(layer, tokens, seed=1, device="cuda"):
    """Hidden rows and labels that the layer can learn: the label depends on the row."""
    g = torch.Generator(device=device).manual_seed(seed)
    X = torch.randn(tokens, layer.head.shape[1], generator=g, device=device).bfloat16()
    labels = (X.float() @ torch.randn(layer.head.shape[1], layer.head.shape[0], generator=g, device=device)).argmax(1)
    labels[torch.rand(tokens, generator=g, device=device) < 0.25] = -100  # prompt tokens are no targets
    return X, labels


def train(h, layer, X, labels, steps, lr):
    """Signed-gradient steps on the latent scales, relative to each scale. Returns the mean losses."""
    losses = []
    for _ in range(steps):
        out = step(h, layer, X, labels)
        losses.append(out["loss"].sum() / (labels >= 0).sum())
        for name, g in out["scale_grads"].items():
            layer.latent[name] -= lr * layer.latent[name].abs() * g.sign()
    h.sq_sync()
    return torch.stack(losses).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--top-k", type=int, default=4)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--inter", type=int, default=768)
    ap.add_argument("--vocab", type=int, default=4000)
    ap.add_argument("--format", choices=("nvfp4", "mxfp4"), default="nvfp4")
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--lr", type=float, default=None,
                    help="relative step of a scale: 0.05, or 0.2 for MXFP4, whose scales are powers of two")
    args = ap.parse_args()
    h = sq.Handle()
    fmt = sq.NVFP4 if args.format == "nvfp4" else sq.MXFP4
    layer = Layer(fmt, args.experts, args.top_k, args.hidden, args.inter, args.vocab)
    X, labels = batch(layer, args.tokens)
    lr = args.lr if args.lr is not None else 0.2 if fmt == sq.MXFP4 else 0.05
    for i, loss in enumerate(train(h, layer, X, labels, args.steps, lr)):
        print(f"step {i}: loss {loss:.4f}")


if __name__ == "__main__":
    main()
