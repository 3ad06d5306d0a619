"""Calls of attention that between them reach every kernel, chosen by the library's own
rules: attention_plan.h, which test_attention_plan.py compiles and asks."""
import itertools
import random

_MODES = [dict(), dict(cap=9.0), dict(slopes=True), dict(cap=9.0, slopes=True)]
_r = random.Random(17)

# documents of uneven lengths, none and one row among them; odd and even numbers of tiles of 128, and tiles of one key
FEW = [700, 0, 513, 640, 1, 1200, 900]
SHORT = [300, 0, 129, 257, 1, 256, 128, 33, 290]
MANY = [_r.choice([0, 1, 513, 640, 700, 770, 1000]) for _ in range(67)] + [900, 1000, 1024]
MANY_SHORT = [_r.choice([0, 1, 7, 130, 200, 257, 300]) for _ in range(70)]


def case(queries, keys, heads, kv_heads, dim, dtype, **how):
    return dict(queries=queries, keys=keys, hq=heads, hk=kv_heads, dim=dim, dtype=dtype, **how)


def cases():
    out = {}
    # (queries, keys, heads, key heads): one sequence length for all but the last, which is shorter
    large = [([600, 600], [600, 600], 104, 52), ([700, 650], [513, 513], 54, 54), ([513, 513], [700, 3], 104, 52), ([640, 520], [640, 640], 54, 54)]
    middle = [([300] * 3 + [40], [290] * 4, 44, 22), ([129] * 4, [257] * 4, 33, 33), ([257] * 4, [129] * 4, 44, 44), ([200, 130, 1, 0], [700, 700, 33, 640], 44, 44)]
    small = [([140], [140], 2, 1), ([90], [150], 3, 3), ([150], [90], 4, 2), ([77, 33], [77, 77], 2, 2)]
    for (i, how), dim in itertools.product(enumerate(_MODES), (64, 128)):
        narrow = {64: (64, 40, 56, 64), 128: (128, 80, 128, 104)}[dim][i]
        name = f"{dim} {'+'.join(how) or 'plain'}"
        types = ("bf16", "fp16") if (i + dim // 64) % 2 else ("fp16", "bf16")
        at = i if dim == 64 else 3 - i
        prefix = [[100, 333], None, [300, 0], [1, 520]][at]
        out[f"large {name}"] = case(*large[at], narrow, types[0], causal=at != 3, prefix=prefix, **how)
        prefix = [[20, 140, 290, 0], None, [60, 3, 0, 500], None][at]
        out[f"middle {name}"] = case(*middle[at], narrow, types[1], causal=at != 1, prefix=prefix, **how)
        out[f"small {name}"] = case(*small[at], narrow, types[0], causal=at != 2, **how)
        # 7 documents, found in the order of their work; 70, found by search
        out[f"documents {name}"] = case(FEW, FEW, 32, 16, narrow, types[0], causal=True, packed=True, prefix=[9, 0, 200, 0, 1, 600, 0] if at == 1 else None, **how)
        out[f"short documents {name}"] = case(SHORT, SHORT[1:] + SHORT[:1] if at == 2 else SHORT, 16, 16, narrow, types[1], causal=at != 3, packed=True, lead=30, **how)
        if at in (0, 2):
            out[f"many documents {name}"] = case(MANY, MANY, 4 if at else 3, 2 if at else 3, narrow, types[0], causal=True, packed=True, **how)
            out[f"many short documents {name}"] = case(MANY_SHORT, MANY_SHORT, 2, 2, narrow, types[1], causal=True, packed=True, room=(70, 9), **how)
        # few queries: keys in parts, in one, and of documents
        out[f"parts {name}"] = case([1, 1], [3000, 700], 16, 2, narrow, types[0], causal=at != 1, train=False, **how)
        out[f"parts of two tiles {name}"] = case([6], [2500], 24, 3, narrow, types[1], causal=True, prefix=[2497], train=False, **how)
        out[f"whole caches {name}"] = case([1] * 40, [3000 - 70 * j for j in range(39)] + [3000], 8, 8, narrow, types[1], causal=True, train=False, **how)
        out[f"parts of documents {name}"] = case([2, 0, 1, 1], [4000, 9, 0, 3000], 8, 2, narrow, types[0], causal=True, packed=True, train=False, room=(3, 1), **how)
        if at == 3:
            out[f"parts of many documents {name}"] = case([1] * 70, [2000 + (j * 37) % 500 for j in range(70)], 2, 1, narrow, types[1], causal=True, packed=True,
                                                          train=False, **how)
    return out


def sizes(c):
    """(sequences, rows of q, rows of k, heads, key heads) as the library's rules see them"""
    n, room, lead = len(c["queries"]), c.get("room", (0, 0)), c.get("lead", 0)
    if c.get("packed"):
        rows = [lead + sum(c[k]) + r for k, r in zip(("queries", "keys"), room)]
    else:
        rows = [n * (max(c[k]) + r) for k, r in zip(("queries", "keys"), room)]
    return n, *rows, c["hq"], c["hk"]


def mode(c):
    return ("cap" if c.get("cap") else "") + ("slopes" if c.get("slopes") else "")
