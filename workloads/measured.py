"""Layer times of a profile measured on this GPU, with the library's operators.

A profile's ``layer_ns`` are forward + backward times of a layer for one
micro-batch. Here a layer is its projections and its feed-forward block (dense,
or top-k experts) on one rank of a tensor-parallel group; the attention between the
projections is left out, its output being the values:

    q = x Wq^T;  [k | v] = x Wkv^T;  h = x + v Wo^T;  y = h + block(h)

(q and k are formed, and their gradients taken, though they are zero then.) All experts are on
this rank. A training runtime's layers take other times; these are a layer's without attention.
:class:`Layer` runs it with ``heddle_linear`` and ``heddle_gated_ffn`` and their
backward passes, :func:`train` a step of several layers that ends with
``heddle_clip_grad_norm`` and an update, and :func:`measure` puts times into the
first GPU type of a workload's profile, so that plans are priced with them:

    python -m workloads.measured c2_7b_dense --templates 1000
"""
from __future__ import annotations

import argparse
import copy

import numpy as np
import torch

from paper_2609_34244_amd import heddle as H

TOKENS = 2048                  # of a micro-batch: boundary_bytes = tokens * hidden * 2


class Layer:
    """One rank's part of a layer: bf16 weights and what its backward pass needs."""

    def __init__(self, hidden, width, units, experts=0, top_k=1, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape):
            return torch.randn(shape, generator=g, device=device).mul_(shape[-1] ** -0.5).bfloat16()

        lead = (experts,) if experts else ()
        self.width, self.experts, self.top_k = width, experts, top_k
        self.w = {"q": weight(width, hidden), "kv": weight(2 * width, hidden), "out": weight(hidden, width),
                  "in": weight(*lead, 2 * units, hidden), "down": weight(*lead, hidden, units)}

    def forward(self, x, picked=None):
        """picked: [tokens, top_k] expert of each token, for expert layers"""
        self.x = x
        self.q, kv = H.heddle_linear(x, self.w["q"]), H.heddle_linear(x, self.w["kv"])
        self.v = kv[:, self.width:]
        h = H.heddle_linear(self.v, self.w["out"], residual=x)
        rows, self.offsets = h, None
        if self.experts:
            flat = picked.flatten()
            self.order = torch.argsort(flat, stable=True)
            self.back = torch.argsort(self.order, stable=True)
            ends = torch.searchsorted(flat[self.order], torch.arange(self.experts + 1, device=flat.device))
            self.offsets = ends.to(torch.int32)
            rows = h[self.order // self.top_k]
        self.rows, self.p = rows, rows.new_empty(rows.shape[0], self.w["in"].shape[-2])
        y = H.heddle_gated_ffn(rows, self.w["in"], self.w["down"], residual=None if self.experts else h, preact=self.p,
                               offsets=self.offsets)
        return h + y[self.back].view(-1, self.top_k, y.shape[1]).mean(1) if self.experts else y

    def backward(self, dy):
        """(gradient of x, gradients of the weights by name)"""
        dr = (dy / self.top_k)[self.order // self.top_k] if self.experts else dy
        g = H.heddle_gated_ffn_backward(dr, self.rows, self.w["in"], self.w["down"], self.p, offsets=self.offsets)
        dh = g["dx"]
        if self.experts:
            dh = dh[self.back].view(-1, self.top_k, dh.shape[1]).sum(1)
        dh = dh + dy
        dkv = dh.new_zeros(dh.shape[0], 2 * self.width)
        o = H.heddle_linear_backward(dh, self.v, self.w["out"], dx=dkv[:, self.width:])
        q = H.heddle_linear_backward(torch.zeros_like(self.q), self.x, self.w["q"])
        kv = H.heddle_linear_backward(dkv, self.x, self.w["kv"])
        return q["dx"] + kv["dx"] + dh, {"q": q["dw"], "kv": kv["dw"], "out": o["dw"], "in": g["dw_in"], "down": g["dw_out"]}


def train(layers, x, target, picked=None, rate=0.1, max_norm=1.0):
    """One step on 1/2 mean (y - target)^2 per value; returns (loss, gradient norm) as tensors."""
    y = x
    for layer in layers:
        y = layer.forward(y, picked)
    off = y.float() - target.float()
    dy, grads = (off / off.numel()).to(x.dtype), []
    for layer in reversed(layers):
        dy, g = layer.backward(dy)
        grads += [(layer, k, v) for k, v in g.items()]
    norm = H.heddle_clip_grad_norm([v for _, _, v in grads], max_norm)
    for layer, k, v in grads:
        layer.w[k].sub_(v, alpha=rate)
    return 0.5 * off.square().mean(), norm


def sizes(cfg):
    """(hidden, units, experts, units of an expert, top_k) of a configuration: a layer's
    parameters are 4 hidden^2 of projections and 3 hidden units of its block"""
    hidden = cfg["boundary_bytes"] // (2 * TOKENS)
    units = max(32, (cfg["dense_params_per_layer"] - 4 * hidden * hidden) // (3 * hidden) // 32 * 32)
    moe = cfg.get("moe")
    if not moe:
        return hidden, units, 0, 0, 1
    return hidden, units, moe["n_experts"], max(32, (moe["expert_params"] // (3 * hidden) + 31) // 32 * 32), moe["top_k"]


def layer_time(hidden, width, units, experts, top_k, repeat=5):
    """ns of a forward and a backward pass of one micro-batch: the least of `repeat`"""
    layer = Layer(hidden, width, units, experts, top_k)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(TOKENS, hidden, generator=g, device="cuda").bfloat16() for _ in range(2))
    picked = torch.rand(TOKENS, experts, generator=g, device="cuda").topk(top_k, 1).indices if experts else None
    best = None
    for i in range(repeat + 1):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        layer.forward(x, picked)
        layer.backward(dy)
        end.record()
        end.synchronize()
        ns = int(start.elapsed_time(end) * 1e6)
        best = ns if i == 1 else best if i == 0 else min(best, ns)       # the first pass warms up
    return best


def measure(cfg, profile, repeat=5):
    """A copy of the profile whose first GPU type has measured layer times at
    every TP degree that it has times for."""
    hidden, units, experts, expert_units, top_k = sizes(cfg)
    p = copy.deepcopy(profile)
    times = {}
    for k, tp in enumerate(int(t) for t in p.tp_degrees):
        if not p.profiled[0, k]:
            continue
        width = max(32, hidden // tp)
        dense = layer_time(hidden, width, max(32, units // tp), 0, 1, repeat)
        moe = layer_time(hidden, width, max(32, expert_units // tp), experts, top_k, repeat) if experts else dense
        times[tp] = (dense, moe)
        p.layer_ns[0, k] = np.where(p.is_moe == 1, moe, dense)
        if p.xlayer_ns is not None:
            # the experts' share of the measured time stays what it was of the time before
            old = profile.layer_ns[0, k].astype(np.float64)
            p.xlayer_ns[0, k] = np.rint(p.layer_ns[0, k] * (profile.xlayer_ns[0, k] / old)).astype(np.int64)
    return p.check(), times


def main():
    from workloads.gen import CONFIG_NAMES, load_config, make_workload
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("config", nargs="?", default="c2_7b_dense", choices=CONFIG_NAMES)
    a.add_argument("--templates", type=int, default=1000)
    a = a.parse_args()
    w = make_workload(a.config, n=a.templates)
    profile, times = measure(load_config(a.config), w.profile)
    for tp, (dense, moe) in times.items():
        print(f"TP {tp}, without attention: dense layer {dense / 1e3:.1f} us" + (f", expert layer {moe / 1e3:.1f} us" if w.profile.is_moe.any() else ""))
    n_stages, stages = H.to_device(w.n_stages, w.stages)
    for what, p in (("synthetic", w.profile), ("measured", profile)):
        best = H.heddle_best_plan(H.heddle_load_profile(p), n_stages, stages, [int(x) for x in w.m], 0)
        print(f"{what} times: best plan " + ("none" if best is None else f"{best[0]}, iteration {best[2] / 1e6:.3f} ms"))


if __name__ == "__main__":
    main()
