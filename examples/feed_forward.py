"""Two feed-forward parts of a decoder on one GPU: a gated layer whose first matrix is encrypted and whose second is dense in
8 bits, and a layer of experts in 8 bits.

    t = x + r                       add_rmsnorm_fp8: the sum, its RMS norm in 8 bits, and in 16 bits where spmm wants it
    u = norm(t) W13^T               few tokens: spmm on the encrypted W13
                                    many: matmul_fp8 on the copy that decode and quant_fp8 have made of it
    d = (silu(gate) * up) W2^T      silu_mul_fp8, matmul_fp8
    s = t + d                       add_rmsnorm_fp8
    y = s + experts(norm(s))        moe_fp8, 64 tokens a call

    python examples/feed_forward.py [--config large_q1] [--tokens 1,8,64,1024] [--experts 8] [--picks 2]

prints the time of a pass and how far its parts are from 64-bit arithmetic.  Inputs and weights are synthetic.
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

import paper_1905_10138_amd as xe
from synth_inputs import CONFIGS, make_workload

# Tokens up to which the encrypted matrix itself is multiplied: it has a seventh of the decoded copy's bytes, and takes as long for
# 64 tokens and longer for more (16384 x 4096, one plane: 15.7 us and the copy 14.4 at 64 tokens, 39 and 31 at 256).
MOST_ENCRYPTED = 64


def encrypt(workload):
    """The workload's matrix, encrypted on the GPU."""
    cfg = workload.cfg
    mask = torch.from_numpy(xe.pack_bits(workload.keep[:, :workload.n], cfg.n_out).view(np.int64)).cuda()
    planes = np.stack([xe.pack_bits(p[:, :workload.n], cfg.n_out) for p in workload.planes])
    rows = (workload.M.astype(np.uint64) << np.arange(cfg.n_in, dtype=np.uint64)).sum(axis=1).astype(np.uint32)
    return xe.encode(workload.m, workload.n, cfg.n_in, cfg.q, rows, mask, torch.from_numpy(planes.view(np.int64)).cuda(),
                     torch.from_numpy(workload.alpha).cuda(), n_out=cfg.n_out)


class GatedLayer:
    """norm, W13 (encrypted; gates before ups), silu(gate) * up, W2 (outputs, inputs), which is given in 16 or 32 bits."""

    def __init__(self, encrypted, W2, norm):
        self.encrypted, self.norm = encrypted, norm
        self.W13 = xe.quant_fp8(xe.decode(encrypted, xe.OUT_BF16), block_rows=xe.FP8_BLOCK)
        self.W2 = xe.quant_fp8(W2, block_rows=xe.FP8_BLOCK)

    def up(self, x, r):
        """x + r and the gates and ups of its norm."""
        tokens, features = x.shape
        if tokens > MOST_ENCRYPTED:
            Q, S, t, _ = xe.add_rmsnorm_fp8(x, self.norm, r)
            return t, xe.matmul_fp8(Q, S, *self.W13)
        columns = torch.empty((features, tokens), dtype=x.dtype, device=x.device)  # spmm's order: a column a token
        _, _, t, _ = xe.add_rmsnorm_fp8(x, self.norm, r, normed=columns.t())
        return t, xe.spmm(self.encrypted, columns).t().contiguous()

    def down(self, u):
        return xe.matmul_fp8(*xe.silu_mul_fp8(u), *self.W2)

    def __call__(self, x, r):
        t, u = self.up(x, r)
        return t, self.down(u)


class ExpertLayer:
    """norm, router and experts: W13 (experts, 2 inner, hidden), W2 (experts, hidden, inner), given in 16 or 32 bits."""

    def __init__(self, router, W13, W2, norm, picks):
        self.router, self.norm, self.picks = router, norm, picks
        self.W13 = xe.quant_fp8(W13, block_rows=xe.FP8_BLOCK)
        self.W2 = xe.quant_fp8(W2, block_rows=xe.FP8_BLOCK)

    def experts(self, n):
        out = torch.empty_like(n)
        for i in range(0, n.shape[0], xe.MOE_MAX_TOKENS):
            part = slice(i, i + xe.MOE_MAX_TOKENS)
            xe.moe_fp8(n[part], self.router, *self.W13, *self.W2, self.picks, Y=out[part])
        return out

    def __call__(self, x, r):
        _, _, t, n = xe.add_rmsnorm_fp8(x, self.norm, r, normed=True)
        return t, self.experts(n)


def build(workload, experts, picks, inner, seed=0):
    """Both layers: W13 of the first is the workload's matrix, the experts have `inner` inner features."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def draw(*shape, scale=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)

    H, I = workload.n, workload.m // 2
    gated = GatedLayer(encrypt(workload), draw(H, I, scale=I ** -0.5), 1 + draw(H, scale=0.1, dtype=torch.float32))
    moe = ExpertLayer(draw(experts, H, scale=H ** -0.5), draw(experts, 2 * inner, H, scale=H ** -0.5),
                      draw(experts, H, inner, scale=inner ** -0.5), 1 + draw(H, scale=0.1, dtype=torch.float32), picks)
    return gated, moe, draw


def forward(gated, moe, x, r):
    t, d = gated(x, r)
    s, y = moe(d, t)
    return s + y


def off_by(got, want):
    return float((got.double() - want).norm() / want.norm())


def compare(gated, moe, x, r):
    """How far each part is from 64-bit arithmetic on its own inputs (2-norm)."""
    def norm(t, w):
        return t * (t.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w.double()

    def dense(Q, S):
        return Q.double() * S.double().repeat_interleave(128, 0)[:Q.shape[0]].repeat_interleave(128, 1)[:, :Q.shape[1]]

    _, u = gated.up(x, r)
    want = norm(x.double() + r.double(), gated.norm) @ xe.decode(gated.encrypted, xe.OUT_F32).double().t()
    d = gated.down(u)
    gate, up = u.double().chunk(2, 1)
    return off_by(u, want), off_by(d, (gate * torch.sigmoid(gate) * up) @ dense(*gated.W2).t())


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--config", default="large_q1", choices=sorted(CONFIGS))
    p.add_argument("--tokens", default="1,8,64,1024")
    p.add_argument("--experts", type=int, default=8)
    p.add_argument("--picks", type=int, default=2)
    p.add_argument("--inner", type=int, default=2048)
    args = p.parse_args()
    gated, moe, draw = build(make_workload(CONFIGS[args.config]), args.experts, args.picks, args.inner)
    for tokens in map(int, args.tokens.split(",")):
        x, r = draw(tokens, gated.encrypted.n), draw(tokens, gated.encrypted.n)
        for _ in range(3):
            forward(gated, moe, x, r)
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(20):
            forward(gated, moe, x, r)
        torch.cuda.synchronize()
        us = (time.perf_counter() - began) / 20 * 1e6
        up, down = compare(gated, moe, x, r)
        print(f"{tokens:5d} tokens: {us:8.1f} us a pass, off 64 bits by {up:.2e} (norm, W13) and {down:.2e} (gate, W2)", flush=True)


if __name__ == "__main__":
    main()
