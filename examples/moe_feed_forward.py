"""A chain of DiT feed-forward layers that are mixtures of experts between two norms.

    a = Pre(h) (1 + c) + s                       fb_op_sandwich_norm without a block output
    per layer: router, experts up, experts down,
               h = rs h + g Post(sum_j p_j e_j), a = Pre(h) (1 + c') + s'   fb_moe_forward

Every layer is one call; the norm behind a layer's experts also forms the next layer's input.
The first layer is checked against plain torch in float64 on the router's own choice.

    python examples/moe_feed_forward.py [--tokens 1560] [--layers 4] [--experts 8] [--top-k 2]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_04461_gb300 import flashbon as fb, synth  # noqa: E402

D, HIDDEN, EPS, RESID_SCALE = 1536, 2048, 1e-6, 0.875


class Layer:
    def __init__(self, g, experts, top_k):
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.router = torch.zeros(-(-experts // 128) * 128, D, dtype=torch.bfloat16, device="cuda")
        self.router[:experts] = (2 * D ** -0.5 * randn(experts, D)).to(torch.bfloat16)
        self.w1 = (D ** -0.5 * randn(experts, 2 * HIDDEN, D)).to(torch.bfloat16)
        self.w2 = (HIDDEN ** -0.5 * randn(experts, D, HIDDEN)).to(torch.bfloat16)
        self.post_w = 1 + 0.1 * randn(D)
        self.gate, self.shift, self.scale = 0.5 * randn(1, D), 0.1 * randn(1, D), 0.1 * randn(1, D)
        self.moe = fb.make_moe(self.router, self.w1, self.w2, top_k, act="swiglu", renorm=True)


def run(model, layers, h, a, valid=None):
    """All layers in place: h the fp32 residual stream, a the normed input (its buffer is
    reused)."""
    first = fb.make_sandwich(h, pre="layer", pre_eps=EPS, mul=layers[0].scale, add=layers[0].shift, a=a)
    model.op_sandwich_norm(first)
    for i, layer in enumerate(layers):
        after = layers[(i + 1) % len(layers)]  # whose input norm comes next
        s = fb.make_sandwich(h, h_out=h, post="rms", post_eps=EPS, post_w=layer.post_w,
                             gate=layer.gate, resid_scale=RESID_SCALE, pre="layer", pre_eps=EPS,
                             mul=after.scale, add=after.shift, a=a)
        model.moe_forward(layer.moe, a, s, valid=valid)


def first_layer64(layer, h, experts, top_k):
    """The first layer's h in float64."""
    x = h.double()
    a = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + EPS).sqrt()
    a = a * (1 + layer.scale.double()) + layer.shift.double()
    logits = a.to(torch.bfloat16).double() @ layer.router[:experts].double().T
    top, idx = logits.topk(top_k, 1)
    p = torch.softmax(top, 1)
    y = torch.zeros_like(x)
    for e in range(experts):
        t, j = (idx == e).nonzero(as_tuple=True)
        u = a[t] @ layer.w1[e].double().T
        u = u[:, :HIDDEN] * torch.sigmoid(u[:, :HIDDEN]) * u[:, HIDDEN:]
        y[t] += p[t, j, None] * (u @ layer.w2[e].double().T)
    u = y / ((y * y).mean(1, keepdim=True) + EPS).sqrt() * layer.post_w.double()
    return RESID_SCALE * x + layer.gate.double() * u


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=1560)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--top-k", type=int, default=2)
    args = ap.parse_args(argv)
    g = torch.Generator("cuda").manual_seed(0)
    layers = [Layer(g, args.experts, args.top_k) for _ in range(args.layers)]
    h0 = torch.randn(args.tokens, D, generator=g, device="cuda")
    a = torch.empty(args.tokens, D, dtype=torch.bfloat16, device="cuda")
    with fb.Model(synth.TINY, synth.make_weights(synth.TINY)) as model:
        h = h0.clone()
        run(model, layers[:1], h, a)
        want = first_layer64(layers[0], h0, args.experts, args.top_k)
        step = want - RESID_SCALE * h0.double()
        err = ((h.double() - want).norm() / step.norm()).item()
        h = h0.clone()
        run(model, layers, h, a)
        t = time.perf_counter()
        run(model, layers, h, a)
        ms = (time.perf_counter() - t) * 1e3
    print(f"{args.tokens} tokens, {args.layers} layers of {args.experts} experts (top {args.top_k}): "
          f"{ms:.3f} ms; first layer off by {err:.2e} of what it adds")
    return err


if __name__ == "__main__":
    main()
