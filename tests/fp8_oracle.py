"""The operators for dense layers in 8 bits from their definitions, in 64 bits, element by element or row by row, with torch on
the CPU.  Shares no code with the package."""
import math

import torch

F8 = torch.float8_e4m3fn
BLOCK = 128
LEAST = 2.0 ** -126


def dense(Q, S, block_rows):
    """The values that an 8-bit matrix stands for."""
    Q, S = Q.cpu(), S.cpu()
    rows, cols = Q.shape
    r = torch.arange(rows) // block_rows
    c = torch.arange(cols) // BLOCK
    return Q.view(torch.uint8).clone().view(F8).double() * S.double()[r][:, c]


def scales(y, block_rows):
    """Of fp64 values: max(amax / 448, 2^-126) of each block."""
    out = [[max(float(part.abs().max()) / 448.0, LEAST) for part in rows.split(BLOCK, 1)] for rows in y.split(block_rows, 0)]
    return torch.tensor(out, dtype=torch.float64)


def half_step(v):
    """Half the distance of the e4m3 values around v (|v| <= 448)."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    return torch.exp2(e - 4)


def check_quantised(y, Q, S, block_rows, rel):
    """Q and S are y in 8 bits; y itself is known to a relative error of `rel`."""
    Q, S = Q.cpu(), S.cpu().double()
    want = scales(y, block_rows)
    assert S.shape == want.shape and Q.shape == y.shape
    # amax to rel, its division by 448 rounded once
    assert ((S - want).abs() <= (rel + 2.0 ** -23) * want).all(), ((S - want).abs() / want).max()
    r = torch.arange(y.shape[0]) // block_rows
    c = torch.arange(y.shape[1]) // BLOCK
    v = y / S[r][:, c]
    q = Q.view(torch.uint8).clone().view(F8).double()
    # the nearest value, or with v this close to the middle of two either of them; y * (1 / S) is rounded twice more
    assert ((q - v).abs() <= half_step(v) * (1 + 1e-12) + (rel + 2.0 ** -22) * v.abs()).all()


def rmsnorm(x, r, w, eps):
    t = x.double() + (0 if r is None else r.double())
    y = torch.empty_like(t)
    for i in range(t.shape[0]):
        y[i] = t[i] / math.sqrt(float((t[i] ** 2).sum()) / t.shape[1] + eps) * w.double()
    return t, y


def silu_mul(x):
    n = x.shape[1] // 2
    g, u = x[:, :n].double(), x[:, n:].double()
    return g / (1 + torch.exp(-g)) * u


def picks(logits, n):
    """Of one token: the largest logits, the lowest index of equals."""
    return sorted(range(len(logits)), key=lambda e: (-logits[e], e))[:n]


def moe(x, router, w13, w2, n_picks, renormalise):
    """w13 [E, 2 I, H], w2 [E, H, I]: fp64.  Returns y, and the same sum over magnitudes."""
    x, router = x.double(), router.double()
    I = w2.shape[2]
    y, mag = torch.zeros_like(x), torch.zeros_like(x)
    for t in range(x.shape[0]):
        logits = [float(v) for v in (router * x[t]).sum(1)]
        chosen = picks(logits, n_picks)
        top = max(logits)
        share = {e: math.exp(logits[e] - top) for e in range(len(logits))}
        norm = sum(share[e] for e in chosen) if renormalise else sum(share.values())
        for e in chosen:
            up = w13[e] @ x[t]
            h = up[:I] / (1 + torch.exp(-up[:I])) * up[I:]
            y[t] += share[e] / norm * (w2[e] @ h)
            mag[t] += share[e] / norm * (w2[e].abs() @ h.abs())
    return y, mag
