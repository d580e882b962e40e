"""Sorted tokens and products with an epilogue from their definitions, in 64 bits or with Python's own numbers, on the CPU.  Shares
no code with the package."""
import math

import torch


def picks(row, n):
    """Of one token's logits (Python numbers): the experts, largest first, and None where fewer are left."""
    order = sorted((e for e in range(len(row)) if row[e] != -math.inf), key=lambda e: (-math.inf if math.isnan(row[e]) else -row[e], not math.isnan(row[e]), e))
    return (order + [None] * n)[:n]


def shares(row, chosen, renormalise):
    over = [row[e] for e in chosen if e is not None] if renormalise else [v for v in row if v != -math.inf]
    if not over:
        return [0.0] * len(chosen)
    if any(math.isnan(v) or v == math.inf for v in over):
        return [0.0 if e is None else math.nan for e in chosen]
    top = max(over)
    total = math.fsum(math.exp(v - top) for v in over)
    return [0.0 if e is None else math.exp(row[e] - top) / total for e in chosen]


def sort(ids, experts):
    """places, tokens, offsets (lists) of ids [T][P]."""
    T, P = len(ids), len(ids[0]) if ids else 0
    key = [e if 0 <= e < experts else experts for row in ids for e in row]
    order = sorted(range(T * P), key=lambda i: key[i])  # Python's sort keeps the order of equals
    places = [0] * (T * P)
    for row, pair in enumerate(order):
        places[pair] = row
    offsets = [sum(k < e for k in key) for e in range(experts + 1)]
    return places, [pair // P for pair in order], offsets


def activation(name, z):
    """fp64."""
    if name == "relu":
        return z.clamp(min=0)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return z * torch.special.erfc(-z / math.sqrt(2)) / 2
    if name == "gelu_tanh":
        # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)), which keeps its digits where tanh u is next to -1
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


# The steepest that each is (silu 1.0999 at 2.40, gelu 1.1290 at 1.41, gelu_tanh 1.1295 at 1.41)
SLOPE = {None: 1.0, "relu": 1.0, "silu": 1.1, "gelu": 1.13, "gelu_tanh": 1.13}
