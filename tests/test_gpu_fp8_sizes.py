"""Dense layers in 8 bits on the GPU: larger sizes, every side of what the sizes decide (the tile, how a reduction is split, how
many tokens of an expert go together), and operands that reach beyond 32 bits.  Tolerances: those of test_gpu_fp8.py."""
import pytest
import torch

import paper_1905_10138_amd as xe
import fp8_oracle as ref
from test_gpu_fp8 import DEV, F8, U, check_moe, gen, normal, random_8bit

pytestmark = pytest.mark.gpu

# from one row of tiles to many, short and long reductions, rows of results on and off 16-byte boundaries
PRODUCTS = [(1, 8326, 129), (1, 13312, 273), (1, 15400, 181), (3, 1021, 9000), (18, 4380, 134), (34, 3035, 290), (40, 4096, 4096),
            (65, 16384, 700), (70, 300, 5000), (74, 8202, 424), (100, 4096, 4100), (130, 5000, 1300), (261, 14207, 65), (300, 6001, 900),
            (520, 4096, 2048), (1000, 8200, 777), (1061, 12379, 66), (1237, 5152, 136), (2100, 4200, 1000), (4000, 4096, 129)]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(M, N, K, out):
    g = gen(M * 7 + N * 3 + K)
    A, SA = random_8bit(g, M, K, 1)
    W, SW = random_8bit(g, N, K, 128)
    Y = xe.matmul_fp8(A, SA, W, SW, out_dtype=out)
    a, w = ref.dense(A, SA, 1).to(DEV), ref.dense(W, SW, 128).to(DEV)
    want, mag = a @ w.t(), a.abs() @ w.abs().t()
    err = (Y.double() - want).abs()
    if out is torch.float32:
        assert (err <= (K / 128 + 128) * 2 * U * mag).all(), (err / mag).max()
        assert err.norm() <= 4e-6 * want.norm()
    else:  # 128 times the largest magnitudes of both rows in a block are no less than 128 times the largest product
        pad = -K % 128
        tops = [torch.nn.functional.pad(v.abs(), (0, pad)).reshape(v.shape[0], -1, 128).amax(2) for v in (a, w)]
        largest = 128 * (tops[0] @ tops[1].t())
        assert (err <= 2.0 ** -8 * want.abs() * 1.01 + 2.0 ** -13 * largest).all()
        assert err.norm() <= (2.0 ** -8 + 1e-4) * want.norm()
    again = torch.full((M, N + 1), 9.0, dtype=out, device=DEV)   # rows off 16-byte boundaries: the same values
    xe.matmul_fp8(A, SA, W, SW, Y=again[:, :N])
    assert torch.equal(again[:, :N], Y) and (again[:, N] == 9.0).all()


def spread(t, ld):
    """The rows of t in memory, ld elements apart."""
    rows, cols = t.shape
    out = torch.empty((rows - 1) * ld + cols + 16, dtype=t.dtype, device=DEV).as_strided((rows, cols), (ld, 1))
    raw = torch.uint8 if t.dtype is F8 else t.dtype
    out.view(raw).copy_(t.view(raw))
    return out


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M", [3, 40, 150, 1100])
def test_product_of_operands_beyond_32_bits(M, out):
    g = gen(M)
    N, K, ld = 1100, 300, 1 << 22
    A, SA = random_8bit(g, M, K, 1)
    W, SW = random_8bit(g, N, K, 128)
    plain = xe.matmul_fp8(A, SA, W, SW, out_dtype=out)
    Y = torch.empty((M - 1) * ld + N + 16, dtype=out, device=DEV).as_strided((M, N), (ld, 1))
    xe.matmul_fp8(spread(A, ld), SA, spread(W, ld), SW, Y=Y)
    assert torch.equal(Y, plain)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_beyond_32_bits(dtype):
    g = gen(3)
    ld = (1 << 30) + 8
    x, r = normal(g, 4, 600, dtype=dtype).to(DEV), normal(g, 4, 600, dtype=dtype).to(DEV)
    w = normal(g, 600).to(DEV)
    far = spread(x, ld)
    for got, want in [(xe.quant_fp8(far), xe.quant_fp8(x)), (xe.quant_fp8(far, block_rows=128), xe.quant_fp8(x, block_rows=128)),
                      (xe.silu_mul_fp8(far), xe.silu_mul_fp8(x))]:
        assert torch.equal(got[0].float(), want[0].float()) and torch.equal(got[1], want[1])
    total = torch.empty(3 * ld + 616, dtype=dtype, device=DEV).as_strided((4, 600), (ld, 1))
    got, want = xe.add_rmsnorm_fp8(far, w, r, total=total, normed=True), xe.add_rmsnorm_fp8(x, w, r, normed=True)
    assert all(torch.equal(a.float(), b.float()) for a, b in zip(got, want))
    y = xe.add_rmsnorm_fp8(x, w, r, normed=total)[3]
    assert torch.equal(y, want[3])


def test_stacks_beyond_32_bits():
    g = gen(5)
    mat = (1 << 31) + 64
    x = normal(g, 3, 130, 200, dtype=torch.bfloat16).to(DEV)
    far = torch.empty(2 * mat + 130 * 200, dtype=torch.bfloat16, device=DEV).as_strided((3, 130, 200), (mat, 200, 1))
    far.copy_(x)
    got, want = xe.quant_fp8(far, block_rows=128), xe.quant_fp8(x, block_rows=128)
    assert torch.equal(got[0].float(), want[0].float()) and torch.equal(got[1], want[1])
    T, H, I, E = 5, 200, 96, 3
    tokens, router = normal(g, T, H, dtype=torch.bfloat16).to(DEV), normal(g, E, H, dtype=torch.bfloat16).to(DEV)
    W13, S13 = random_8bit(g, 2 * I, H, 128, lead=(E,))
    W2, S2 = random_8bit(g, H, I, 128, lead=(E,))
    plain = xe.moe_fp8(tokens, router, W13, S13, W2, S2, 3)

    def apart(W):
        out = torch.empty(2 * mat + W.shape[1] * W.stride(1), dtype=F8, device=DEV).as_strided(W.shape, (mat, W.stride(1), 1))
        out.view(torch.uint8).copy_(W.view(torch.uint8))
        return out
    assert torch.equal(xe.moe_fp8(tokens, router, apart(W13), S13, apart(W2), S2, 3), plain)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", [(648, 9046, 68), (1080, 11586, 129), (1052, 7849, 302), (334, 10347, 931), (3000, 3000, 1000), (1934, 1568, 69),
                                   (17, 4576, 513), (74, 8202, 424), (1, 8219, 398), (1, 14874, 136), (700, 4096, 1111), (2048, 5000, 300)])
def test_product_of_middling_sizes(M, N, K, out):
    test_product(M, N, K, out)


# tokens per expert beyond one pass, one expert for all, one workgroup to 32 for a sum, few and many rows of inner features
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,I,E,n", [(64, 144, 72, 2, 2), (64, 130, 40, 1, 1), (63, 96, 56, 3, 3), (33, 128, 264, 2, 1), (1, 128, 4200, 3, 2),
                                       (6, 200, 3000, 2, 1), (64, 100, 16, 256, 8), (1, 300, 24, 256, 16), (4, 128, 2048, 16, 4),
                                       (16, 64, 2048, 16, 4), (40, 64, 2048, 16, 3), (4, 4500, 130, 4, 2)])
def test_experts(T, H, I, E, n, dtype):
    check_moe(T, H, I, E, n, dtype)


def test_experts_of_many_hidden_features():
    check_moe(2, 33000, 20, 2, 1, torch.bfloat16)


@pytest.mark.parametrize("T", [1, 5])
@pytest.mark.parametrize("renormalise", [True, False])
def test_experts_of_what_is_not_finite(T, renormalise):
    g = gen(T)
    H, I, E = 136, 40, 6
    x, router = normal(g, T, H, dtype=torch.bfloat16).to(DEV), normal(g, E, H, dtype=torch.bfloat16).to(DEV)
    W13, S13 = random_8bit(g, 2 * I, H, 128, lead=(E,))
    W2, S2 = random_8bit(g, H, I, 128, lead=(E,))
    clean = xe.moe_fp8(x, router, W13, S13, W2, S2, 2, renormalise=renormalise)
    for v in (float("nan"), -float("nan"), float("inf"), -float("inf")):   # in a token: its row, no other
        bad = x.clone()
        bad[T // 2, 7] = v
        Y = xe.moe_fp8(bad, router, W13, S13, W2, S2, 2, renormalise=renormalise)
        keep = torch.arange(T, device=DEV) != T // 2
        assert torch.equal(Y[keep], clean[keep]) and not torch.isfinite(Y[~keep]).any()
    for bits in (0x7FC0, -0x40):                                           # in a row of the router, of either sign: all tokens
        bad = router.clone()
        bad.view(torch.int16)[3, 9] = bits
        assert torch.isnan(xe.moe_fp8(x, bad, W13, S13, W2, S2, 2, renormalise=renormalise)).all()


# few steps of the second product and many, few workgroups of the first and many, an expert for all tokens
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,I,E,n", [(1, 520, 2600, 9, 4), (1, 70, 2500, 12, 5), (2, 300, 1000, 6, 3), (2, 64, 1500, 8, 2), (3, 1000, 700, 8, 2),
                                       (4, 130, 129, 1, 1), (4, 2050, 300, 16, 4), (4, 96, 2000, 40, 10), (3, 200, 16, 256, 16)])
def test_experts_of_up_to_four_tokens(T, H, I, E, n, dtype):
    check_moe(T, H, I, E, n, dtype)
    check_moe(T, H, I, E, n, dtype, renormalise=False)


def test_what_is_not_finite_stays_with_its_token():
    g = gen(3)
    T, H, I, E = 3, 136, 40, 6
    x, router = normal(g, T, H, dtype=torch.bfloat16).to(DEV), normal(g, E, H, dtype=torch.bfloat16).to(DEV)
    W13, S13 = random_8bit(g, 2 * I, H, 128, lead=(E,))
    W2, S2 = random_8bit(g, H, I, 128, lead=(E,))
    clean = xe.moe_fp8(x, router, W13, S13, W2, S2, 3)
    for t in range(T):
        bad = x.clone()
        bad[t, 5] = float("nan")
        Y = xe.moe_fp8(bad, router, W13, S13, W2, S2, 3)
        keep = torch.arange(T, device=DEV) != t
        assert torch.equal(Y[keep], clean[keep]) and torch.isnan(Y[~keep]).all()


# 96 MB of weights and more are read another way: the same values as those of each token
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,I,E,n", [(1, 4096, 4100, 2, 2), (4, 4000, 2100, 5, 2), (9, 4096, 2048, 4, 2), (40, 2048, 2050, 9, 3)])
def test_experts_of_many_bytes(T, H, I, E, n, dtype):
    g = torch.Generator(device=DEV).manual_seed(T)

    def weights(*shape):
        q = (torch.randn(shape, generator=g, device=DEV) * 60).clamp(-448, 448).to(F8)
        ld = -(-shape[-1] // 16) * 16
        out = torch.full((*shape[:-1], ld), 0x7F, dtype=torch.uint8, device=DEV)
        out[..., :shape[-1]] = q.view(torch.uint8)
        blocks = (shape[0], -(-shape[1] // 128), -(-shape[2] // 128))
        return out.view(F8)[..., :shape[-1]], torch.exp2(torch.randn(blocks, generator=g, device=DEV)) / 60 / shape[-1] ** 0.5

    def dense(q, s):
        return q.double() * s.double().repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]
    x = torch.randn((T, H), generator=g, device=DEV).to(dtype)
    router = (torch.randn((E, H), generator=g, device=DEV) * 2 / H ** 0.5).to(dtype)
    (W13, S13), (W2, S2) = weights(E, 2 * I, H), weights(E, H, I)
    Y = xe.moe_fp8(x, router, W13, S13, W2, S2, n)
    shares, chosen = torch.softmax(x.double() @ router.double().t(), 1).topk(n, 1)
    shares = shares / shares.sum(1, keepdim=True)
    want, mag = torch.zeros((2, T, H), dtype=torch.float64, device=DEV)
    for e in range(E):
        w13, w2 = dense(W13[e], S13[e]), dense(W2[e], S2[e])
        gate, up = (x.double() @ w13.t()).chunk(2, 1)
        h = gate * torch.sigmoid(gate) * up
        f = (shares * (chosen == e)).sum(1, keepdim=True)
        want += f * (h @ w2.t())
        mag += f * (h.abs() @ w2.abs().t())
    err = (Y.double() - want).abs()
    if dtype is torch.bfloat16:
        assert (err <= 2.0 ** -8 * 1.01 * want.abs() + 2.0 ** -15 * mag).all()
        assert err.norm() <= (2.0 ** -8 + 2.0 ** -14) * want.norm()
    else:
        assert (err <= 2.0 ** -18 * mag).all() and err.norm() <= 4e-6 * want.norm()
