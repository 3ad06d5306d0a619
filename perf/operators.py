"""The feed-forward and gradient operators' work, as measurable cases.

* ``linear``  Y = act(X W^T + b) + R, alone or with its backward pass
  (``heddle_linear``, ``heddle_linear_backward``);
* ``ffn``     the gated feed-forward block, dense or over expert groups, alone
  or with its backward pass (``heddle_gated_ffn``,
  ``heddle_gated_ffn_backward``);
* ``clip``    the global norm of many gradient tensors and clipping by it
  (``heddle_clip_grad_norm``).

Sizes follow the named configurations: hidden sizes 4096 and 8192 at 2048
tokens a sequence, feed-forward widths from their parameters per layer (10816
and 24032), 64 experts of width 1632, top 2, and their TP shards.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _linear(m, k, n, act="none", bias=False, residual=False, train=False, dtype="bf16"):
    return {"kind": "linear", "m": m, "k": k, "n": n, "act": act, "bias": bias, "residual": residual, "train": train,
            "dtype": dtype}


def _ffn(tokens, d, f, experts=1, act="silu", residual=False, train=False, dtype="bf16"):
    return {"kind": "ffn", "tokens": tokens, "d": d, "f": f, "experts": experts, "act": act, "residual": residual,
            "train": train, "dtype": dtype}


def _clip(tensors, elements, types):
    return {"kind": "clip", "tensors": tensors, "elements": elements, "types": types}


def listed():
    return [
        # an output projection while one sequence is answered token by token
        dict(_linear(1, 4096, 4096, residual=True), name="linear_token"),
        # a projection over a prompt of the 8192-wide model, everything in the epilogue
        dict(_linear(2048, 8192, 8192, act="gelu", bias=True, residual=True), name="linear_prompt"),
        # an ungated layer's training step on two sequences
        dict(_linear(4096, 4096, 10816, act="gelu_tanh", bias=True, train=True), name="linear_train"),
        # sizes that no tile or vector divides, fp16
        dict(_linear(1001, 1027, 513, act="relu", bias=True, residual=True, train=True, dtype="fp16"), name="linear_odd"),
        # the block for a single token
        dict(_ffn(1, 4096, 10816, residual=True), name="ffn_token"),
        # 16 tokens' top-2 experts: most experts without rows, the others with one or two
        dict(_ffn(32, 4096, 1632, experts=64), name="ffn_experts_decode"),
        # the block's training step on two sequences
        dict(_ffn(4096, 4096, 10816, residual=True, train=True), name="ffn_train"),
        # one sequence's top-2 rows over 64 experts, training
        dict(_ffn(4096, 4096, 1632, experts=64, train=True), name="ffn_experts_train"),
        # four sequences through the widest block, training
        dict(_ffn(8192, 8192, 24032, train=True), name="ffn_train_wide"),
        # gradients of a small module: a few matrices and vectors
        dict(_clip(9, 1000003, "fp32"), name="clip_small"),
        # one layer's gradients of the 4096-wide model
        dict(_clip(10, 200000000, "bf16"), name="clip_layer"),
        # a pipeline stage's gradients: many tensors, matrices in bf16, vectors in fp32
        dict(_clip(320, 1600000000, "mixed"), name="clip_stage"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """half of them whole vectors, half of them any number"""
    v = _log_uniform(rng, lo, hi)
    return max(8, v // 8 * 8) if rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["linear", "linear", "ffn", "ffn", "ffn", "clip"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    train = rng.random() < 0.5
    if kind == "linear":
        return _linear(_log_uniform(rng, 1, 8192), _size(rng, 128, 8192), _size(rng, 128, 24032),
                       rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), rng.random() < 0.5,
                       rng.random() < 0.5, train, dtype)
    if kind == "ffn":
        tokens, residual = _log_uniform(rng, 1, 8192), rng.random() < 0.5
        act = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"])
        if rng.random() < 0.5:
            # EP and expert-TP shards of the 64 experts
            return _ffn(tokens, rng.choice([2048, 4096]), 1632 // rng.choice([1, 2, 4, 8]), rng.choice([8, 16, 32, 64]),
                        act, residual, train, dtype)
        return _ffn(tokens, _size(rng, 512, 8192), _size(rng, 512, 10816), 1, act, residual, train, dtype)
    elements = _log_uniform(rng, 1000, 1000000000)
    return _clip(min(elements, _log_uniform(rng, 1, 400)), elements, rng.choice(["fp32", "bf16", "fp16", "mixed"]))


def _tensor_sizes(case):
    """The sizes of a module's tensors, from the case alone: every third one a
    vector, the others matrices whose sizes differ by up to a factor of four."""
    rng = random.Random("%(tensors)d %(elements)d %(types)s" % case)
    weights = [rng.uniform(1, 4) if i % 3 else rng.uniform(1, 4) / 4096 for i in range(case["tensors"])]
    if case["tensors"] == 1:
        return [case["elements"]]
    total = sum(weights)
    sizes = [max(1, int(case["elements"] * w / total)) for w in weights]
    sizes[-1] = max(1, sizes[-1] + case["elements"] - sum(sizes))
    return sizes


def _tensor_type(case, i):
    return _TYPES["bf16" if i % 3 else "fp32"] if case["types"] == "mixed" else _TYPES[case["types"]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=None):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype or _TYPES[case["dtype"]]).mul_(scale)

    s = {"case": case}
    if case["kind"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        s["x"], s["w"] = normal(m, k), normal(n, k, scale=k ** -0.5)
        s["bias"] = normal(n, scale=0.1) if case["bias"] else None
        s["residual"] = normal(m, n) if case["residual"] else None
        s["dy"] = normal(m, n, scale=0.1) if case["train"] else None
    elif case["kind"] == "ffn":
        t, d, f, e = case["tokens"], case["d"], case["f"], case["experts"]
        lead = (e,) if e > 1 else ()
        s["x"] = normal(t, d)
        s["w_in"], s["w_out"] = normal(*lead, 2 * f, d, scale=d ** -0.5), normal(*lead, d, f, scale=f ** -0.5)
        s["residual"] = normal(t, d) if case["residual"] else None
        s["dy"] = normal(t, d, scale=0.1) if case["train"] else None
        s["offsets"], s["rows"] = None, [t]
        if e > 1:
            # a router's load: uneven, and some experts without rows
            share = torch.softmax(torch.randn(e, generator=g, device="cuda"), 0)
            picked = torch.multinomial(share, t, replacement=True, generator=g)
            counts = (picked[:, None] == torch.arange(e, device="cuda")[None]).sum(0)
            s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
            s["rows"] = counts.tolist()
    else:
        sizes = _tensor_sizes(case)
        s["grads"] = [normal(n, scale=0.01, dtype=_tensor_type(case, i)) for i, n in enumerate(sizes)]
        # the clipped gradients go to one flat buffer per type, as a bucket for the optimiser
        types = sorted({str(t.dtype) for t in s["grads"]})
        s["flat"] = {t: torch.empty(sum(x.numel() for x in s["grads"] if str(x.dtype) == t), device="cuda",
                                    dtype=next(x.dtype for x in s["grads"] if str(x.dtype) == t)) for t in types}
        views = {t: iter(s["flat"][t].split([x.numel() for x in s["grads"] if str(x.dtype) == t])) for t in types}
        s["out"] = [next(views[str(x.dtype)]) for x in s["grads"]]
        s["max_norm"] = 1.0
    return s


def _act(z, name):
    if name == "relu":
        return z * (z > 0)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if name == "gelu_tanh":
        t = torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * (2 / math.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _linear_plain(s):
    c, dt = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(dt)}
    if c["train"]:
        dz = s["dy"].float() * _act_grad(z, c["act"])
        out["dx"], out["dw"] = (dz @ w).to(dt), (dz.t() @ x).to(dt)
        if s["bias"] is not None:
            out["db"] = dz.sum(0).to(dt)
    return out


def _block_plain(act, x, w_in, w_out, dy):
    """one expert's rows, in 32 bits: y, and with dy the gradients of x and the weights"""
    x, w_in, w_out = x.float(), w_in.float(), w_out.float()
    f = w_out.shape[1]
    p = x @ w_in.t()
    h = _act(p[:, :f], act) * p[:, f:]
    y = h @ w_out.t()
    if dy is None:
        return y, None, None, None
    dy = dy.float()
    dh = dy @ w_out
    dp = torch.cat([dh * p[:, f:] * _act_grad(p[:, :f], act), dh * _act(p[:, :f], act)], 1)
    return y, dp @ w_in, dp.t() @ x, dy.t() @ h


def _ffn_plain(s):
    c, dt = s["case"], s["x"].dtype
    if c["experts"] == 1:
        y, dx, dw_in, dw_out = _block_plain(c["act"], s["x"], s["w_in"], s["w_out"], s["dy"])
        dw_in, dw_out = (None, None) if dx is None else (dw_in.to(dt), dw_out.to(dt))
    else:
        xs = s["x"].split(s["rows"])
        dys = s["dy"].split(s["rows"]) if c["train"] else [None] * len(xs)
        parts = [(_block_plain(c["act"], x, wi, wo, dy)) for x, wi, wo, dy in zip(xs, s["w_in"], s["w_out"], dys)]
        y = torch.cat([p[0] for p in parts])
        dx = dw_in = dw_out = None
        if c["train"]:
            dx = torch.cat([p[1] for p in parts])
            dw_in, dw_out = torch.stack([p[2].to(dt) for p in parts]), torch.stack([p[3].to(dt) for p in parts])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(dt)}
    if c["train"]:
        out.update(dx=dx.to(dt), dw_in=dw_in, dw_out=dw_out)
    return out


def _clip_plain(s):
    norm = torch.sqrt(torch.stack([(g.float() * g.float()).sum() for g in s["grads"]]).sum())
    factor = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0)
    clipped = [(g.float() * factor).to(g.dtype) for g in s["grads"]]
    out = {t: torch.cat([x for x in clipped if str(x.dtype) == t]) for t in s["flat"]}
    return dict(out, norm=norm.reshape(1))


def _linear_own(s):
    from paper_2609_34244_amd import heddle as H
    c = s["case"]
    act = H.ACTIVATIONS[c["act"]]
    z = torch.empty_like(s["dy"]) if c["train"] and c["act"] != "none" else None
    out = {"y": H.heddle_linear(s["x"], s["w"], bias=s["bias"], act=act, residual=s["residual"], preact=z)}
    if c["train"]:
        out.update(H.heddle_linear_backward(s["dy"], s["x"], s["w"], act=act, preact=z,
                                            want_db=s["bias"] is not None))
    return out


def _ffn_own(s):
    from paper_2609_34244_amd import heddle as H
    c = s["case"]
    act = H.ACTIVATIONS[c["act"]]
    p = s["x"].new_empty(c["tokens"], 2 * c["f"]) if c["train"] else None
    out = {"y": H.heddle_gated_ffn(s["x"], s["w_in"], s["w_out"], act=act, residual=s["residual"], preact=p,
                                   offsets=s["offsets"])}
    if c["train"]:
        out.update(H.heddle_gated_ffn_backward(s["dy"], s["x"], s["w_in"], s["w_out"], p, act=act,
                                               offsets=s["offsets"]))
    return out


def _clip_own(s):
    from paper_2609_34244_amd import heddle as H
    norm = H.heddle_clip_grad_norm(s["grads"], s["max_norm"], out=s["out"])
    return dict(s["flat"], norm=norm)


def run(state):
    kind = state["case"]["kind"]
    if kind == "linear":
        return _linear_own(state) if own else _linear_plain(state)
    if kind == "ffn":
        return _ffn_own(state) if own else _ffn_plain(state)
    return _clip_own(state) if own else _clip_plain(state)


def work(case):
    """Inputs once, outputs once. Of the experts only those with rows count:
    at most one per row. A training step's gradients of the weights are
    outputs for every expert."""
    train = 1 if case.get("train") else 0
    if case["kind"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        values = m * k + n * k + m * n * (1 + case["residual"]) + n * case["bias"]
        values += train * (m * n + m * k + n * k + n * case["bias"])
        return {"bytes": 2 * values, "flops": 2 * m * k * n * (1 + 2 * train)}
    if case["kind"] == "ffn":
        t, d, f = case["tokens"], case["d"], case["f"]
        used = min(case["experts"], t)
        values = 2 * t * d + used * 3 * d * f + t * d * case["residual"]
        values += train * (2 * t * d + case["experts"] * 3 * d * f)
        return {"bytes": 2 * values, "flops": 6 * t * d * f * (1 + 2 * train)}
    total = sum(n * _tensor_type(case, i).itemsize for i, n in enumerate(_tensor_sizes(case)))
    return {"bytes": 2 * total, "flops": 3 * case["elements"]}


def _act64(z, name):
    nn = torch.nn.functional
    return {"none": lambda: z, "relu": lambda: nn.relu(z), "silu": lambda: nn.silu(z), "gelu": lambda: nn.gelu(z),
            "gelu_tanh": lambda: nn.gelu(z, approximate="tanh")}[name]()


def exact(case, seed):
    """The definitions in 64 bits; gradients by automatic differentiation."""
    s = prepare(case, seed)
    wide = lambda t: None if t is None else t.double().requires_grad_(bool(case["train"]))  # noqa: E731
    if case["kind"] == "linear":
        x, w, b = wide(s["x"]), wide(s["w"]), wide(s["bias"])
        z = torch.mm(x, w.t())
        y = _act64(z if b is None else z + b, case["act"])
        y = y if s["residual"] is None else y + s["residual"].double()
        out = {"y": y.detach()}
        if case["train"]:
            y.backward(s["dy"].double())
            out.update(dx=x.grad, dw=w.grad)
            if b is not None:
                out["db"] = b.grad
        return out
    if case["kind"] == "ffn":
        many = case["experts"] > 1
        out = {"y": [], "dx": [], "dw_in": [], "dw_out": []}
        w_in, w_out = (s["w_in"], s["w_out"]) if many else (s["w_in"][None], s["w_out"][None])
        row = 0
        for e, count in enumerate(s["rows"]):
            x, wi, wo = wide(s["x"][row:row + count]), wide(w_in[e]), wide(w_out[e])
            gate, up = torch.mm(x, wi.t()).chunk(2, 1)
            y = torch.mm(_act64(gate, case["act"]) * up, wo.t())
            out["y"].append(y.detach())
            if case["train"]:
                y.backward(s["dy"][row:row + count].double())
                out["dx"].append(x.grad)
                out["dw_in"].append(wi.grad)
                out["dw_out"].append(wo.grad)
            row += count
        y = torch.cat(out["y"])
        got = {"y": y if s["residual"] is None else y + s["residual"].double()}
        if case["train"]:
            got["dx"] = torch.cat(out["dx"])
            got["dw_in"] = torch.stack(out["dw_in"]) if many else out["dw_in"][0]
            got["dw_out"] = torch.stack(out["dw_out"]) if many else out["dw_out"][0]
        return got
    norm = math.sqrt(math.fsum(float(g.double().square().sum()) for g in s["grads"]))
    factor = min(1.0, s["max_norm"] / (norm + 1e-6))
    out = {t: torch.cat([g.double() * factor for g in s["grads"] if str(g.dtype) == t]) for t in s["flat"]}
    return dict(out, norm=torch.tensor([norm], dtype=torch.float64, device="cuda"))
