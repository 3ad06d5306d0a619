"""What a layer does between its products, as measurable cases.

* ``attention``  softmax(mask(cap tanh(scale q k / cap) - slope |distance|)) v over
  shared key heads, packed documents, prefixes and caches, alone or with its
  backward pass (``heddle_attention``, ``heddle_attention_backward``);
* ``norm``       layer normalisation, alone or with its backward pass
  (``heddle_layer_norm``, ``heddle_layer_norm_backward``);
* ``balance``    a router's counts and balance loss, alone or with its gradient
  (``heddle_expert_balance``, ``heddle_expert_balance_backward``).

Sizes follow the named configurations: hidden sizes 4096 and 8192 in heads of
128 at 2048 tokens a sequence, 64 experts, top 2.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _attention(sequences, queries, keys, heads, kv_heads, dim=128, causal=True, cap=0.0, slopes=False, prefix=False,
               packed=False, train=False, dtype="bf16"):
    """packed: `sequences` documents of uneven lengths, sequences * queries rows in all.
    Not packed and fewer queries than keys: a cache of `keys` rows a sequence, filled to uneven lengths."""
    return {"kind": "attention", "sequences": sequences, "queries": queries, "keys": keys, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "causal": causal, "cap": cap, "slopes": slopes, "prefix": prefix,
            "packed": packed, "train": train, "dtype": dtype}


def _norm(rows, columns, residual=False, train=False, dtype="bf16", weights="same"):
    return {"kind": "norm", "rows": rows, "columns": columns, "residual": residual, "train": train, "dtype": dtype,
            "weights": weights}


def _balance(tokens, experts, picks, residual=False, train=False, dtype="fp32"):
    return {"kind": "balance", "tokens": tokens, "experts": experts, "picks": picks, "residual": residual, "train": train,
            "dtype": dtype}


def listed():
    return [
        # one sequence's next token over its cache, 32 heads, distance bias
        dict(_attention(1, 1, 2048, 32, 32, slopes=True), name="attention_token"),
        # the next tokens of 32 sequences over long caches, 64 heads on 8 key heads, capped scores
        dict(_attention(32, 1, 8192, 64, 8, cap=50.0), name="attention_decode"),
        # a long prompt whose first part sees itself whole
        dict(_attention(1, 8192, 8192, 32, 8, prefix=True, slopes=True), name="attention_prompt"),
        # the 4096-wide model's training step on two sequences' tokens packed of 11 documents
        dict(_attention(11, 372, 372, 32, 32, packed=True, train=True), name="attention_train_documents"),
        # the 8192-wide model's training step on four sequences, capped scores
        dict(_attention(4, 2048, 2048, 64, 8, cap=30.0, train=True), name="attention_train_wide"),
        # a narrow head that no tile divides, odd lengths, heads in threes, fp16
        dict(_attention(3, 333, 333, 12, 4, dim=80, causal=False, slopes=True, train=True, dtype="fp16"), name="attention_odd"),
        # one token
        dict(_norm(1, 4096), name="norm_token"),
        # two sequences of the 4096-wide model, training, with the gradient that went past the layer
        dict(_norm(4096, 4096, residual=True, train=True), name="norm_train"),
        # rows that no vector divides, fp16 with weights kept in fp32
        dict(_norm(1001, 1027, train=True, dtype="fp16", weights="fp32"), name="norm_odd"),
        # a router's step for 32 sequences' next tokens
        dict(_balance(32, 64, 2), name="balance_decode"),
        # a router's training step on two sequences
        dict(_balance(4096, 64, 2, train=True), name="balance_train"),
        # 64 sequences, with the gradient that reaches the scores through the experts' weights
        dict(_balance(131072, 64, 2, residual=True, train=True, dtype="bf16"), name="balance_train_large"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "norm", "norm", "balance"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    train = rng.random() < 0.5
    if kind == "norm":
        rows = _log_uniform(rng, 1, 32768)
        columns = _log_uniform(rng, 64, 16384)
        while rows * columns > 1 << 26:
            rows = rows // 2 + 1
        if rng.random() < 0.5:
            columns = max(8, columns // 8 * 8)
        return _norm(rows, columns, rng.random() < 0.5, train, rng.choice([dtype, dtype, "fp32"]), rng.choice(["same", "fp32"]))
    if kind == "balance":
        experts = _log_uniform(rng, 4, 512)
        tokens = _log_uniform(rng, 1, 131072)
        while tokens * experts > 131072 * 64:
            tokens = tokens // 2 + 1
        return _balance(tokens, experts, rng.randint(1, min(8, experts)), rng.random() < 0.5, train,
                        rng.choice(["fp32", "fp32", dtype]))
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 6, 8) if g * kv_heads <= 64])
    dim = rng.choice([128, 128, 64, 8 * rng.randint(4, 16)])
    mask = dict(causal=rng.random() < 0.75, cap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.4,
                prefix=rng.random() < 0.3, dtype=dtype)
    shape = rng.choice(["decode", "batch", "documents"])
    sequences = _log_uniform(rng, 1, 32)
    if shape == "decode":
        queries = rng.choice([1, 1, 1, rng.randint(2, 8)])
        keys = _log_uniform(rng, 16, 16384)
        while sequences * keys * kv_heads * dim > 32 * 8192 * 8 * 128:
            sequences = sequences // 2
        return _attention(max(1, sequences), queries, keys, heads, kv_heads, dim, **mask)
    length = _log_uniform(rng, 1, 4096)
    while sequences > 1 and sequences * length * length * heads * dim > 4 * 2048 * 2048 * 64 * 128:
        sequences //= 2
    while length * length * heads * dim > 4 * 2048 * 2048 * 64 * 128:
        length //= 2
    if shape == "documents":
        # the documents' lengths are uneven: together no longer than the longest case allows for one
        while (sequences * length) ** 2 * heads * dim > 4 * 2048 * 2048 * 64 * 128 and length > 1:
            length //= 2
    return _attention(sequences, length, length, heads, kv_heads, dim, packed=shape == "documents", train=train, **mask)


def _lengths(case):
    """(queries of each sequence, keys of each, prefix of each), from the case alone"""
    rng = random.Random(" ".join(str(case[k]) for k in sorted(case) if k != "name"))
    n = case["sequences"]
    if case["packed"]:
        total = n * case["queries"]
        cuts = sorted(rng.randint(0, total) for _ in range(n - 1))
        keys = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        queries = keys
    elif case["queries"] < case["keys"]:
        queries = [case["queries"]] * n
        keys = [case["keys"] if i == 0 else rng.randint(case["queries"], case["keys"]) for i in range(n)]
    else:
        queries, keys = [case["queries"]] * n, [case["keys"]] * n
    return queries, keys, [rng.randint(0, k) for k in keys] if case["prefix"] else None


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=None):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype or _TYPES[case["dtype"]]).mul_(scale)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    s = {"case": case}
    if case["kind"] == "norm":
        m, n = case["rows"], case["columns"]
        wt = _TYPES["fp32"] if case["weights"] == "fp32" else _TYPES[case["dtype"]]
        # a residual stream's values: columns of their own size and offset
        s["x"] = (normal(m, n) * normal(n).abs() + normal(n, scale=0.5)).contiguous()
        s["w"], s["bias"] = (normal(n, scale=0.1, dtype=torch.float32) + 1).to(wt), normal(n, scale=0.1, dtype=wt)
        s["dy"] = normal(m, n, scale=0.1) if case["train"] else None
        s["residual"] = normal(m, n, scale=0.1) if case["train"] and case["residual"] else None
    elif case["kind"] == "balance":
        t, e, k = case["tokens"], case["experts"], case["picks"]
        # scores of a router that favours some experts
        s["logits"] = (normal(t, e) + normal(e)).contiguous()
        noise = torch.rand(t, e, generator=g, device="cuda")
        s["picked"] = (s["logits"].float() + noise).topk(k, 1).indices
        s["scale"] = 0.01
        s["residual"] = normal(t, e, scale=1e-3) if case["train"] and case["residual"] else None
    else:
        n, lq, lk, hq, hk, d = (case[k] for k in ("sequences", "queries", "keys", "heads", "kv_heads", "dim"))
        queries, keys, prefix = _lengths(case)
        s["queries"], s["keys"], s["prefix_of"] = queries, keys, prefix
        s["q_offsets"] = s["k_lengths"] = None
        if lq == lk:
            # q, k and v as one projection left them
            rows = normal(n * lq, hq + 2 * hk, d)
            rows = rows if case["packed"] else rows.view(n, lq, hq + 2 * hk, d)
            s["q"], s["k"], s["v"] = rows[..., :hq, :], rows[..., hq:hq + hk, :], rows[..., hq + hk:, :]
            if case["packed"]:
                s["q_offsets"] = ints([0] + torch.tensor(keys).cumsum(0).tolist())
        else:
            s["q"], s["k"], s["v"] = normal(n, lq, hq, d), normal(n, lk, hk, d), normal(n, lk, hk, d)
            s["k_lengths"] = ints(keys)
        s["prefix"] = ints(prefix) if prefix else None
        s["slopes"] = torch.tensor([2.0 ** (-8 * (h + 1) / hq) for h in range(hq)], device="cuda") if case["slopes"] else None
        s["dy"] = normal(*s["q"].shape) if case["train"] else None
    return s


def _sequences(s):
    """(index, rows of q, rows of k) of every sequence with queries; rows as an index into the tensors"""
    row = 0
    for i, (lq, lk) in enumerate(zip(s["queries"], s["keys"])):
        if s["case"]["packed"]:
            if lq:
                yield i, slice(row, row + lq), slice(row, row + lk)
            row += lq
        else:
            yield i, (i, slice(0, lq)), (i, slice(0, lk))


def _scores_plain(s, i, q, k, head):
    """scores after the cap and the bias, masked ones -inf, and tanh of the capped scores; q: [h, lq, d], k: [h, lk, d]"""
    c = s["case"]
    lq, lk = q.shape[1], k.shape[1]
    z = torch.matmul(q, k.transpose(1, 2)) * c["dim"] ** -0.5
    t = None
    if c["cap"]:
        t = torch.tanh(z / c["cap"])
        z = c["cap"] * t
    at = torch.arange(lq, device=q.device)[:, None] + (lk - lq)
    j = torch.arange(lk, device=q.device)[None]
    if s["slopes"] is not None:
        z = z - s["slopes"][head:head + q.shape[0], None, None] * (at - j).abs()
    if c["causal"]:
        seen = j <= at
        if s["prefix_of"]:
            seen = seen | (j < s["prefix_of"][i])
        z = torch.where(seen, z, torch.full_like(z[:1, :1, :1], -math.inf))
    return z, t


def _attention_plain(s):
    c, dt = s["case"], s["q"].dtype
    group = c["heads"] // c["kv_heads"]
    out = {"y": torch.empty(s["q"].shape, dtype=dt, device="cuda")}
    if c["train"]:
        out.update({n: torch.empty(t.shape, dtype=dt, device="cuda") for n, t in (("dq", s["q"]), ("dk", s["k"]), ("dv", s["v"]))})
    for i, rq, rk in _sequences(s):
        lq, lk = s["queries"][i], s["keys"][i]
        step = max(1, min(c["kv_heads"], (1 << 28) // (group * lq * lk)))        # key heads at a time
        for h in range(0, c["kv_heads"], step):
            hs = slice(h * group, min(h + step, c["kv_heads"]) * group)
            ks = slice(h, h + step)
            q = s["q"][rq][:, hs].float().transpose(0, 1).contiguous()
            k = s["k"][rk][:, ks].float().transpose(0, 1).repeat_interleave(group, 0)
            v = s["v"][rk][:, ks].float().transpose(0, 1).repeat_interleave(group, 0)
            z, t = _scores_plain(s, i, q, k, hs.start)
            top = z.amax(2, keepdim=True)
            e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
            total = e.sum(2, keepdim=True)
            p = e / torch.where(total == 0, torch.ones_like(total), total)
            y = torch.matmul(p, v)
            out["y"][rq][:, hs] = y.transpose(0, 1).to(dt)
            if c["train"]:
                dy = s["dy"][rq][:, hs].float().transpose(0, 1).contiguous()
                dz = p * (torch.matmul(dy, v.transpose(1, 2)) - (dy * y).sum(2, keepdim=True))
                if t is not None:
                    dz = dz * (1 - t * t)
                dz = dz * c["dim"] ** -0.5
                shared = lambda x: x.view(-1, group, lk, c["dim"]).sum(1).transpose(0, 1).to(dt)  # noqa: E731
                out["dq"][rq][:, hs] = torch.matmul(dz, k).transpose(0, 1).to(dt)
                out["dk"][rk][:, ks] = shared(torch.matmul(dz.transpose(1, 2), q))
                out["dv"][rk][:, ks] = shared(torch.matmul(p.transpose(1, 2), dy))
    return out


def _norm_plain(s):
    dt, wt = s["x"].dtype, s["w"].dtype
    x, w = s["x"].float(), s["w"].float()
    mean = x.mean(1, keepdim=True)
    off = x - mean
    rstd = torch.rsqrt((off * off).mean(1, keepdim=True) + 1e-5)
    xh = off * rstd
    out = {"y": (xh * w + s["bias"].float()).to(dt)}
    if s["dy"] is not None:
        dy = s["dy"].float()
        g = dy * w
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        out.update(dx=dx.to(dt), dw=(dy * xh).sum(0).to(wt), db=dy.sum(0).to(wt))
    return out


def _balance_plain(s):
    c, e = s["case"], s["case"]["experts"]
    z = s["logits"].float()
    p = torch.exp(z - z.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    counts = (s["picked"].flatten()[:, None] == torch.arange(e, device="cuda")[None]).sum(0)
    mean = p.mean(0)
    factor = s["scale"] * e / (c["tokens"] * c["picks"])
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    out = {"loss": (factor * (counts * mean).sum()).reshape(1), "mean": mean, "counts": counts.to(torch.int32),
           "offsets": offsets.to(torch.int32)}
    if c["train"]:
        dz = factor / c["tokens"] * p * (counts - (p * counts).sum(1, keepdim=True))
        if s["residual"] is not None:
            dz = dz + s["residual"].float()
        out["dlogits"] = dz.to(s["logits"].dtype)
    return out


def _attention_own(s):
    from paper_2609_34244_amd import heddle as H
    c = s["case"]
    how = dict(causal=c["causal"], cap=c["cap"], slopes=s["slopes"], prefix=s["prefix"], q_offsets=s["q_offsets"],
               k_offsets=s["q_offsets"], k_lengths=s["k_lengths"])
    lse = torch.empty(s["q"].shape[:-1], dtype=torch.float32, device="cuda") if c["train"] else None
    out = {"y": H.heddle_attention(s["q"], s["k"], s["v"], lse=lse, **how)}
    if c["train"]:
        out.update(H.heddle_attention_backward(s["dy"], s["q"], s["k"], s["v"], out["y"], lse, **how))
    return out


def _norm_own(s):
    from paper_2609_34244_amd import heddle as H
    stats = None if s["dy"] is None else torch.empty(s["x"].shape[0], 2, dtype=torch.float32, device="cuda")
    out = {"y": H.heddle_layer_norm(s["x"], s["w"], s["bias"], eps=1e-5, stats=stats)}
    if s["dy"] is not None:
        out.update(H.heddle_layer_norm_backward(s["dy"], s["x"], s["w"], stats, residual=s["residual"], want_db=True))
    return out


def _balance_own(s):
    from paper_2609_34244_amd import heddle as H
    got = H.heddle_expert_balance(s["logits"], s["picked"], scale=s["scale"])
    out = {k: got[k] for k in ("loss", "mean", "counts", "offsets")}
    if s["case"]["train"]:
        out["dlogits"] = H.heddle_expert_balance_backward(s["logits"], s["picked"], got["counts"], got["rows"],
                                                          scale=s["scale"], residual=s["residual"])
    return out


def run(state):
    kind = state["case"]["kind"]
    if kind == "attention":
        return _attention_own(state) if own else _attention_plain(state)
    if kind == "norm":
        return _norm_own(state) if own else _norm_plain(state)
    return _balance_own(state) if own else _balance_plain(state)


def work(case):
    """Inputs once, outputs once. A pair of a query and a key that it sees costs
    two products of the head's width, and five in the backward pass, which
    forms the scores again."""
    train = 1 if case["train"] else 0
    size = 2 if case["dtype"] != "fp32" else 4
    if case["kind"] == "norm":
        m, n = case["rows"], case["columns"]
        wsize = 4 if case["weights"] == "fp32" else size
        values = 2 * m * n + train * (2 * m * n + m * n * case["residual"])
        return {"bytes": size * values + wsize * n * (2 + 2 * train), "flops": m * n * (8 + 12 * train)}
    if case["kind"] == "balance":
        t, e = case["tokens"], case["experts"]
        return {"bytes": size * t * e * (1 + train * (1 + case["residual"])) + 8 * t * case["picks"] + 12 * e,
                "flops": t * e * (5 + 5 * train)}
    queries, keys, prefix = _lengths(case)
    pairs = 0
    for i, (lq, lk) in enumerate(zip(queries, keys)):
        if not case["causal"]:
            pairs += lq * lk
        else:
            pairs += sum(min(lk, max(lk - lq + a + 1, prefix[i] if prefix else 0)) for a in range(lq))
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    q, k = sum(queries) * hq * d, 2 * sum(keys) * hk * d
    return {"bytes": 2 * (2 * q + k + train * (2 * q + k)), "flops": pairs * hq * d * (4 + 10 * train)}


def exact(case, seed):
    """The definitions in 64 bits; gradients by automatic differentiation."""
    s = prepare(case, seed)
    wide = lambda t: None if t is None else t.double().requires_grad_(bool(case["train"]))  # noqa: E731
    if case["kind"] == "norm":
        x, w, b = wide(s["x"]), wide(s["w"]), wide(s["bias"])
        y = torch.nn.functional.layer_norm(x, (case["columns"],), w, b, 1e-5)
        out = {"y": y.detach()}
        if case["train"]:
            y.backward(s["dy"].double())
            out.update(dx=x.grad if s["residual"] is None else x.grad + s["residual"].double(), dw=w.grad, db=b.grad)
        return out
    if case["kind"] == "balance":
        z = wide(s["logits"])
        p = torch.softmax(z, 1)
        counts = torch.bincount(s["picked"].flatten(), minlength=case["experts"])
        share = counts.double() / (case["tokens"] * case["picks"])
        loss = s["scale"] * case["experts"] * torch.dot(share, p.mean(0))
        out = {"loss": loss.detach().reshape(1), "mean": p.mean(0).detach(), "counts": counts.to(torch.int32),
               "offsets": torch.nn.functional.pad(counts.cumsum(0), (1, 0)).to(torch.int32)}
        if case["train"]:
            loss.backward()
            out["dlogits"] = z.grad if s["residual"] is None else z.grad + s["residual"].double()
        return out
    group, d = case["heads"] // case["kv_heads"], case["dim"]
    out = {"y": torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")}
    if case["train"]:
        out.update({n: torch.zeros(t.shape, dtype=torch.float64, device="cuda") for n, t in (("dq", s["q"]), ("dk", s["k"]), ("dv", s["v"]))})
    for i, rq, rk in _sequences(s):
        lq, lk = s["queries"][i], s["keys"][i]
        step = max(1, (1 << 30) // max(1, lk * group * lq) if lq * lk * group < 1 << 27 else 1)
        for h in range(0, case["kv_heads"], step):
            n = min(step, case["kv_heads"] - h)
            q = wide(s["q"][rq][:, h * group:(h + n) * group].transpose(0, 1))
            k, v = (wide(s[t][rk][:, h:h + n].transpose(0, 1)) for t in ("k", "v"))
            z = torch.matmul(q.view(n, group, lq, d).reshape(n, group * lq, d), k.transpose(1, 2)).view(n * group, lq, lk) / math.sqrt(d)
            if case["cap"]:
                z = torch.tanh(z / case["cap"]) * case["cap"]
            place = torch.arange(lk - lq, lk, device="cuda", dtype=torch.float64).view(-1, 1)
            key = torch.arange(lk, device="cuda", dtype=torch.float64).view(1, -1)
            if case["slopes"]:
                z = z - s["slopes"].double()[h * group:(h + n) * group].view(-1, 1, 1) * (place - key).abs()
            if case["causal"]:
                hidden = key > place
                if s["prefix_of"]:
                    hidden &= key >= s["prefix_of"][i]
                z = z.masked_fill(hidden, -math.inf)
            y = torch.matmul(torch.softmax(z, 2).view(n, group * lq, lk), v).view(n * group, lq, d)
            out["y"][rq][:, h * group:(h + n) * group] = y.detach().transpose(0, 1)
            if case["train"]:
                y.backward(s["dy"][rq][:, h * group:(h + n) * group].double().transpose(0, 1))
                out["dq"][rq][:, h * group:(h + n) * group] = q.grad.transpose(0, 1)
                out["dk"][rk][:, h:h + n], out["dv"][rk][:, h:h + n] = k.grad.transpose(0, 1), v.grad.transpose(0, 1)
    return out
