"""Tokens sorted by expert on the GPU: picks, the sort, rows there and back, the gradient of the way back, against their definitions in 64
bits (experts_oracle.py).

U is half a step of fp32.  Shares: logits are multiples of 1/4, so that their differences are exact; an exponential is off by at most 2 steps
(4 U), sums of E <= 256 terms on 16 lanes by (16 + 4) U, a division by U, and both exponentials and the sum enter: 4 + 4 + 20 + 1 < 32 U.
Sums over p <= 16 products: one rounding a term and one for the residual, of what the magnitudes add up to.  A row's inner product: 8 terms
in a row, 4 times for each 8192 columns of a workgroup, a tree of 6 and one of 4: less than cols / 256 + 32 roundings of the magnitudes' sum.
A result in bf16 is rounded by 2^-8 of it at most, after that."""
import math

import pytest
import torch

import paper_1905_10138_amd as xe
import experts_oracle as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.bfloat16, torch.float32]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g).to(dtype)


def draw_ids(g, T, P, E, without=0.0):
    """P different experts a token; -1 for a share of `without` of the pairs."""
    ids = torch.rand((T, E), generator=g).argsort(1)[:, :P].to(torch.int32).contiguous() if P <= E else torch.randint(0, E, (T, P), generator=g, dtype=torch.int32)
    ids[torch.rand((T, P), generator=g) < without] = -1
    return ids


def sorted_pairs(g, T, P, E, without=0.0):
    ids = draw_ids(g, T, P, E, without)
    places, tokens, offsets = xe.sort_tokens(ids.to(DEV), E)
    return ids, places, tokens, offsets


# ---------------------------------------------------------------------------------------------- picks

def check_picks(logits, n, renormalise, on_gpu=None):
    T = logits.shape[0]
    ids, shares = xe.pick_experts(logits.to(DEV) if on_gpu is None else on_gpu, n, renormalise=renormalise)
    assert ids.shape == shares.shape == (T, n) and ids.dtype == torch.int32 and shares.dtype == torch.float32
    got, got_shares = ids.tolist(), shares.tolist()
    for t, row in enumerate(logits.double().tolist()):
        chosen = ref.picks(row, n)
        assert got[t] == [-1 if e is None else e for e in chosen], t
        for a, b in zip(got_shares[t], ref.shares(row, chosen, renormalise)):
            assert math.isnan(a) if math.isnan(b) else abs(a - b) <= 32 * U * b + 2.0 ** -126, (t, a, b)


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,E,n", [(1, 1, 1), (1, 2, 2), (1, 256, 16), (17, 16, 16), (16, 17, 3), (33, 32, 5), (64, 64, 6), (5, 33, 8), (130, 128, 8), (100, 65, 1),
                                   (257, 100, 5), (300, 256, 16), (9, 255, 1), (15, 129, 4)])
def test_picks(T, E, n, dtype, renormalise):
    logits = (normal(gen(T + E), T, E) * 8).round() / 4  # (many equal ones)
    check_picks(logits.to(dtype), n, renormalise)


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("E", [3, 16, 40, 130])
def test_picks_of_masked_and_strange_logits(E, renormalise):
    g = gen(E)
    x = (normal(g, 40, E) * 8).round() / 4
    inf, nan = math.inf, math.nan
    x[0] = -inf                                        # nothing to pick
    x[1] = -inf
    x[1, E - 1] = -3.0                                 # one
    x[2, torch.randperm(E, generator=g)[:E - 2]] = -inf
    x[3] = torch.finfo(torch.float32).min              # not masked: equal, and very low
    x[4] = torch.finfo(torch.float32).min
    x[4, 2] = 0.0
    x[5] = 0.0
    x[5, ::2] = -0.0                                   # equal to 0
    x[6, 1] = nan
    x[7, 2], x[7, 0] = inf, -inf
    x[8] = -inf
    x[8, 1], x[8, 2] = nan, inf
    x[9] = inf
    x[10, torch.rand(E, generator=g) < 0.5] = -inf
    x[11:][torch.rand((29, E), generator=g) < 0.3] = -inf
    check_picks(x, min(3, E), renormalise)
    negative_nan = x.clone()
    negative_nan.view(torch.int32)[12, 0] = -0x400000  # a NaN with its sign set
    check_picks(negative_nan, min(3, E), renormalise)
    low = x.to(torch.bfloat16)                         # (fp32's lowest value becomes -inf in bf16: its own instead)
    low[3] = torch.finfo(torch.bfloat16).min
    low[4] = torch.finfo(torch.bfloat16).min
    low[4, 2] = 0.0
    check_picks(low, min(3, E), renormalise)


@pytest.mark.parametrize("dtype", DTYPES)
def test_picks_strided(dtype):
    x = ((normal(gen(1), 70, 45) * 8).round() / 4).to(dtype)
    wide = torch.full((70, 101), 99.0, dtype=dtype, device=DEV)
    wide[:, 3:48] = x.to(DEV)
    check_picks(x, 4, True, on_gpu=wide[:, 3:48])


# ---------------------------------------------------------------------------------------------- sort

def check_sort(ids, E, dtype=torch.int32):
    T, P = ids.shape
    places, tokens, offsets = xe.sort_tokens(ids.to(dtype).to(DEV), E)
    assert places.shape == (T, P) and tokens.shape == (T * P,) and offsets.shape == (E + 1,)
    assert places.dtype == tokens.dtype == offsets.dtype == torch.int32
    want = ref.sort(ids.tolist(), E)
    assert offsets.tolist() == want[2] and tokens.tolist() == want[1] and places.reshape(-1).tolist() == want[0]


@pytest.mark.parametrize("T,P,E", [(0, 2, 8), (1, 1, 1), (1, 6, 64), (1, 16, 256), (7, 3, 5), (64, 6, 64), (683, 3, 10), (2048, 1, 3), (2049, 1, 256), (341, 16, 100),
                                   (5462, 3, 16), (5461, 3, 16), (1024, 16, 255), (1025, 16, 256), (9000, 8, 33), (16384, 8, 128)])
def test_sort(T, P, E):
    check_sort(draw_ids(gen(T + P + E), T, P, E, 0.1), E)


@pytest.mark.parametrize("T,P,E", [(32768, 8, 128), (87381, 3, 256), (200000, 5, 9), (600000, 2, 200), (262145, 2, 64)])
def test_sort_of_many_pairs(T, P, E):
    # (as test_sort; Python's lists would take seconds)
    ids = torch.randint(-1, E + 1, (T, P), generator=gen(T), dtype=torch.int32)
    places, tokens, offsets = xe.sort_tokens(ids.to(DEV), E)
    key = torch.where(ids < 0, E, ids).reshape(-1).long()
    order = torch.sort(key, stable=True).indices
    assert torch.equal(tokens.cpu().long(), order // P) and torch.equal(places.cpu().reshape(-1)[order].long(), torch.arange(T * P))
    assert offsets.tolist() == [0] + torch.bincount(key, minlength=E + 1)[:E].cumsum(0).tolist()


@pytest.mark.parametrize("T,P,E", [(300, 2, 8), (12000, 2, 8), (140000, 2, 8), (270000, 2, 8)])
@pytest.mark.parametrize("what", ["all to one", "none", "one only", "descending", "the same twice"])
def test_sort_of_uneven_shares(T, P, E, what):
    ids = torch.full((T, P), {"all to one": 5, "none": -1, "one only": -1, "descending": 0, "the same twice": 3}[what], dtype=torch.int32)
    if what == "one only":
        ids[T // 2, 1] = 7
    if what == "descending":
        ids[:] = (E - 1 - torch.arange(T * P).reshape(T, P) * E // (T * P)).to(torch.int32)
    if what == "the same twice":
        ids[::3] = 1
    check_sort(ids, E)


@pytest.mark.parametrize("T", [50, 9000])
def test_sort_of_wide_ids_and_ids_out_of_range(T):
    g = gen(T)
    ids = torch.randint(-3, 12, (T, 3), generator=g)
    ids[0] = torch.tensor([1 << 40, -(1 << 40), (1 << 32) + 2])  # (their low halves would be experts)
    check_sort(ids, 9, torch.int64)
    ids[0] = torch.tensor([1 << 30, -(1 << 31), 9])
    check_sort(ids, 9, torch.int32)


# ---------------------------------------------------------------------------------------------- rows

def plan(ids, places, offsets):
    """(share of the pairs that have an expert, their rows) on the CPU."""
    return places.cpu().long(), places.cpu() < offsets.cpu()[-1]


def want_gather(x, places, have, shares, dtype):
    T, P = places.shape
    s = torch.ones(T, P, dtype=torch.float64) if shares is None else shares.double()
    y = torch.where(have[:, :, None], x.double()[:, None] * s[:, :, None], 0.0)
    out = torch.empty(T * P, x.shape[1], dtype=torch.float64)
    out[places.reshape(-1)] = y.reshape(T * P, -1)
    return out


# a row of one element, ends of pieces, a part of a workgroup, several workgroups a token; one pick to sixteen
ROWS = [(1, 1, 1, 1), (1, 6, 64, 2048), (3, 2, 4, 7), (5, 3, 3, 8), (7, 5, 9, 33), (64, 2, 8, 129), (33, 16, 40, 511), (40, 4, 16, 514), (130, 8, 64, 1000),
        (9, 9, 20, 2050), (300, 2, 8, 2047), (20, 7, 11, 4097), (4, 16, 256, 9216), (1000, 1, 2, 96)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,P,E,H", ROWS)
def test_rows_there_and_back(T, P, E, H, dtype):
    g = gen(T + P + H)
    ids, places, tokens, offsets = sorted_pairs(g, T, P, E, 0.2)
    at, have = plan(ids, places, offsets)
    x, rows = normal(g, T, H, dtype=dtype), normal(g, T * P, H, dtype=dtype)
    residual, dy, shares = normal(g, T, H, dtype=dtype), normal(g, T, H, dtype=dtype), torch.rand((T, P), generator=g)
    mag_r = rows.double().abs()[at] * have[:, :, None]
    for s in (None, shares):
        s_gpu, s64 = (None, torch.ones(T, P, dtype=torch.float64)) if s is None else (s.to(DEV), s.double())
        # there: exact without shares, else one product rounded in fp32 and once more to 16 bits
        R = xe.gather_tokens(x.to(DEV), places, offsets, s_gpu)
        want = want_gather(x, at, have, s, dtype)
        assert R.dtype == dtype and R.shape == (T * P, H)
        assert (R.cpu().double() - want).abs().le((0 if s is None else HALF[dtype] * (1 + U) + U) * want.abs() + (0 if s is None else 2.0 ** -133)).all()
        # back
        for r in (None, residual):
            Y = xe.combine_tokens(rows.to(DEV), places, offsets, s_gpu, None if r is None else r.to(DEV))
            want = torch.where(have[:, :, None], rows.double()[at], 0.0).mul(s64[:, :, None]).sum(1)
            mag = mag_r.mul(s64[:, :, None]).sum(1) + (0 if r is None else r.double().abs())
            want = want + (0 if r is None else r.double())
            assert Y.dtype == dtype and Y.shape == (T, H)
            assert (Y.cpu().double() - want).abs().le((P + 1) * U * mag * 1.01 + (HALF[dtype] * want.abs() * 1.01 if dtype is torch.bfloat16 else 0)).all()
    # the gradient
    dR, dshares = xe.combine_tokens_grad(dy.to(DEV), rows.to(DEV), places, offsets, shares.to(DEV))
    want = want_gather(dy, at, have, shares, dtype)
    assert dR.dtype == dtype and (dR.cpu().double() - want).abs().le((HALF[dtype] * (1 + U) + U) * want.abs() + 2.0 ** -133).all()
    terms = torch.where(have[:, :, None], rows.double()[at], 0.0) * dy.double()[:, None]
    assert dshares.dtype == torch.float32 and dshares.shape == (T, P)
    assert (dshares.cpu().double() - terms.sum(2)).abs().le((H / 256 + 32) * U * terms.abs().sum(2)).all()
    assert (dshares.cpu()[~have] == 0).all()
    # and it is gather's in turn
    assert torch.equal(xe.gather_tokens(dy.to(DEV), places, offsets, shares.to(DEV)), dR)


def test_gradient_against_differences():
    # Small multiples of 1/8: every sum is exact in fp32, and combine_tokens is linear in each argument, so that a difference is the gradient
    g = gen(2)
    T, P, E, H = 3, 2, 4, 5
    ids, places, tokens, offsets = sorted_pairs(g, T, P, E, 0.3)
    rows = torch.randint(-16, 17, (T * P, H), generator=g).float().to(DEV)
    dy = torch.randint(-16, 17, (T, H), generator=g).float().to(DEV)
    shares = (torch.randint(1, 9, (T, P), generator=g).float() / 8).to(DEV)
    dR, dshares = xe.combine_tokens_grad(dy, rows, places, offsets, shares)

    def loss(r, s):
        return float((xe.combine_tokens(r, places, offsets, s).double() * dy.double()).sum())
    for i in range(T * P):
        for c in range(H):
            step = torch.zeros_like(rows)
            step[i, c] = 1.0
            assert (loss(rows + step, shares) - loss(rows - step, shares)) / 2 == float(dR[i, c])
    for t in range(T):
        for p in range(P):
            step = torch.zeros_like(shares)
            step[t, p] = 0.125
            assert (loss(rows, shares + step) - loss(rows, shares - step)) / 0.25 == float(dshares[t, p])
    # gather's: of X combine_tokens, of the shares the second result for X and R's gradient
    x = torch.randint(-16, 17, (T, H), generator=g).float().to(DEV)
    d = torch.randint(-16, 17, (T * P, H), generator=g).float().to(DEV)
    d_rows = xe.combine_tokens(d, places, offsets, shares)
    d_shares = xe.combine_tokens_grad(x, d, places, offsets, shares)[1]

    def loss_of_gather(v, s):
        return float((xe.gather_tokens(v, places, offsets, s).double() * d.double()).sum())
    for t in range(T):
        for c in range(H):
            step = torch.zeros_like(x)
            step[t, c] = 1.0
            assert (loss_of_gather(x + step, shares) - loss_of_gather(x - step, shares)) / 2 == float(d_rows[t, c])
        for p in range(P):
            step = torch.zeros_like(shares)
            step[t, p] = 0.125
            assert (loss_of_gather(x, shares + step) - loss_of_gather(x, shares - step)) / 0.25 == float(d_shares[t, p])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H", [7, 96, 515, 2049])
def test_rows_strided_and_in_place(H, dtype):
    g = gen(H)
    T, P, E = 21, 3, 6
    ids, places, tokens, offsets = sorted_pairs(g, T, P, E, 0.2)
    shares = torch.rand((T, P), generator=g).to(DEV)

    def apart(t):  # the same values with rows of another leading dimension, off 16-byte boundaries, and something around them
        wide = torch.full((t.shape[0] + 2, H + 13), 77.0, dtype=dtype, device=DEV)
        wide[1:-1, 5:5 + H] = t
        return wide, wide[1:-1, 5:5 + H]

    def untouched(wide):
        return (wide[0] == 77).all() and (wide[-1] == 77).all() and (wide[:, :5] == 77).all() and (wide[:, 5 + H:] == 77).all()
    x, r, rows = (normal(g, n, H, dtype=dtype).to(DEV) for n in (T, T, T * P))
    R = xe.gather_tokens(x, places, offsets, shares)
    around, out = apart(torch.zeros_like(R))
    assert xe.gather_tokens(apart(x)[1], places, offsets, shares, R=out) is out
    assert torch.equal(out, R) and untouched(around)
    Y = xe.combine_tokens(rows, places, offsets, shares, r)
    around, out = apart(r)
    assert xe.combine_tokens(apart(rows)[1], places, offsets, shares, out, Y=out) is out
    assert torch.equal(out, Y) and untouched(around)
    dR, ds = xe.combine_tokens_grad(x, rows, places, offsets, shares)
    around, out = apart(rows)
    got = xe.combine_tokens_grad(apart(x)[1], out, places, offsets, shares, dR=out)
    assert torch.equal(out, dR) and torch.equal(got[0], dR) and torch.equal(got[1], ds) and untouched(around)


def test_rows_that_are_not_finite_stay_where_they_are():
    g = gen(4)
    T, P, E, H = 12, 3, 5, 300
    ids, places, tokens, offsets = sorted_pairs(g, T, P, E, 0.3)
    at, have = plan(ids, places, offsets)
    used = int(offsets[-1])
    assert 0 < used < T * P
    rows, shares = normal(g, T * P, H).to(DEV), torch.rand((T, P), generator=g).to(DEV)
    clean = xe.combine_tokens(rows, places, offsets, shares)
    bad = rows.clone()
    bad[used:] = math.nan                       # rows without an expert are not read
    assert torch.equal(xe.combine_tokens(bad, places, offsets, shares), clean)
    dR, ds = xe.combine_tokens_grad(clean, bad, places, offsets, shares)
    assert torch.isfinite(dR).all() and torch.isfinite(ds).all() and (dR[used:] == 0).all()
    for v in (math.nan, math.inf, -math.inf):   # in a row: in its token, no other
        bad = rows.clone()
        bad[0, 5] = v
        Y = xe.combine_tokens(bad, places, offsets, shares)
        owner = int(tokens[0])
        keep = torch.arange(T, device=DEV) != owner
        assert torch.equal(Y[keep], clean[keep]) and not torch.isfinite(Y[owner, 5]) and torch.equal(Y[owner, 6:], clean[owner, 6:])


def test_places_out_of_range_are_pairs_without_an_expert():
    g = gen(8)
    T, P, E, H = 6, 2, 4, 40
    ids, places, tokens, offsets = sorted_pairs(g, T, P, E)
    bad = places.clone()
    bad[2, 1], bad[4, 0] = T * P, -5
    rows, shares = normal(g, T * P, H).to(DEV), torch.rand((T, P), generator=g).to(DEV)
    kept = shares.clone()
    kept[2, 1] = kept[4, 0] = 0
    assert torch.equal(xe.combine_tokens(rows, bad, offsets, shares), xe.combine_tokens(rows, places, offsets, kept))
    marked = torch.full_like(rows, 5.0)
    xe.gather_tokens(rows[:T], bad, offsets, R=marked)
    assert (marked[places[2, 1]] == 5).all() and (marked[places[4, 0]] == 5).all()
    none = offsets.clone()
    none[-1] = -3                               # as if no pair had an expert
    assert (xe.combine_tokens(rows, places, none, shares) == 0).all()
    dR, ds = xe.combine_tokens_grad(rows[:T], rows, bad, offsets, shares, dR=marked)
    assert (marked[places[2, 1]] == 5).all() and ds[2, 1] == 0 and ds[4, 0] == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_beyond_32_bits(dtype):
    g = gen(3)
    T, P, E, H = 3, 2, 2, 200
    ids, places, tokens, offsets = sorted_pairs(g, T, P, E)
    shares = torch.rand((T, P), generator=g).to(DEV)
    x, rows = normal(g, T, H, dtype=dtype).to(DEV), normal(g, T * P, H, dtype=dtype).to(DEV)
    ld = (1 << 30) + 24
    far = torch.empty(5 * ld + H, dtype=dtype, device=DEV).as_strided((T * P, H), (ld, 1))
    xe.gather_tokens(x, places, offsets, shares, R=far)
    assert torch.equal(far, xe.gather_tokens(x, places, offsets, shares))
    far.copy_(rows)
    assert torch.equal(xe.combine_tokens(far, places, offsets, shares), xe.combine_tokens(rows, places, offsets, shares))
    dR, ds = xe.combine_tokens_grad(x, rows, places, offsets, shares)
    got = xe.combine_tokens_grad(x, far, places, offsets, shares, dR=far)
    assert torch.equal(got[0], dR) and torch.equal(got[1], ds)
    xe.combine_tokens(rows, places, offsets, shares, Y=far[:T])
    assert torch.equal(far[:T], xe.combine_tokens(rows, places, offsets, shares))


def test_many_pairs_there_and_back():
    g = gen(12)
    T, P, E, H = 1 << 20, 8, 64, 9
    ids = torch.randint(-1, E, (T, P), generator=g, dtype=torch.int32).to(DEV)
    places, tokens, offsets = xe.sort_tokens(ids, E)
    x = torch.randint(-8, 9, (T, H), generator=g).float().to(DEV)
    R = xe.gather_tokens(x, places, offsets)
    used = int(offsets[-1])
    assert torch.equal(R[:used], x[tokens[:used].long()]) and (R[used:] == 0).all()
    have = (places < used).sum(1, keepdim=True)
    assert torch.equal(xe.combine_tokens(R, places, offsets), x * have)  # (sums of small whole numbers are exact)
    shares = torch.ones(T, P, device=DEV)
    dR, ds = xe.combine_tokens_grad(x, R, places, offsets, shares)
    assert torch.equal(dR, R) and torch.equal(ds, torch.where(places < used, x.square().sum(1, keepdim=True), 0.0))


def test_no_tokens():
    ids, shares = xe.pick_experts(torch.empty(0, 8, device=DEV), 2)
    assert ids.shape == shares.shape == (0, 2)
    places, tokens, offsets = xe.sort_tokens(ids, 8)
    assert offsets.tolist() == [0] * 9 and tokens.numel() == 0
    x = torch.empty(0, 16, device=DEV)
    assert xe.gather_tokens(x, places, offsets, shares).shape == (0, 16)
    assert xe.combine_tokens(x, places, offsets, shares, x).shape == (0, 16)
    assert [t.shape for t in xe.combine_tokens_grad(x, x, places, offsets, shares)] == [(0, 16), (0, 2)]


def test_refusals():
    g = gen(1)
    ids, places, tokens, offsets = sorted_pairs(g, 6, 2, 4)
    x, rows, shares = normal(g, 6, 16).to(DEV), normal(g, 12, 16).to(DEV), torch.rand((6, 2), generator=g).to(DEV)
    short = torch.zeros(1, dtype=torch.int32, device=DEV)
    for call in (lambda: xe.pick_experts(x.half(), 2), lambda: xe.pick_experts(x.cpu(), 2), lambda: xe.pick_experts(x.t(), 2), lambda: xe.pick_experts(x[0], 2),
                 lambda: xe.sort_tokens(places.float(), 4), lambda: xe.sort_tokens(places.cpu(), 4), lambda: xe.sort_tokens(places.t(), 4),
                 lambda: xe.sort_tokens(places[0], 4),
                 lambda: xe.gather_tokens(x[:5], places, offsets), lambda: xe.gather_tokens(x, places.long(), offsets),
                 lambda: xe.gather_tokens(x, places, offsets.long()), lambda: xe.gather_tokens(x, places, short), lambda: xe.gather_tokens(x, places, offsets, shares.t()),
                 lambda: xe.gather_tokens(x, places, offsets, shares.bfloat16()), lambda: xe.gather_tokens(x, places, offsets, shares[:5]),
                 lambda: xe.gather_tokens(x, places, offsets, R=rows[:5]), lambda: xe.gather_tokens(x, places, offsets, R=rows.bfloat16()),
                 lambda: xe.combine_tokens(rows[:11], places, offsets), lambda: xe.combine_tokens(rows, places, offsets, residual=x[:5]),
                 lambda: xe.combine_tokens(rows, places, offsets, residual=x.bfloat16()), lambda: xe.combine_tokens(rows, places, offsets, Y=x[:, :15]),
                 lambda: xe.combine_tokens(rows, places.cpu(), offsets), lambda: xe.combine_tokens_grad(x, rows, places, offsets, None),
                 lambda: xe.combine_tokens_grad(x.bfloat16(), rows, places, offsets, shares), lambda: xe.combine_tokens_grad(x[:5], rows, places, offsets, shares),
                 lambda: xe.combine_tokens_grad(x, rows, places, offsets, shares, dR=rows[:3])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: xe.pick_experts(x, 17), lambda: xe.pick_experts(x, 0), lambda: xe.pick_experts(x, -1), lambda: xe.sort_tokens(places, 0),
                 lambda: xe.sort_tokens(places, 257), lambda: xe.pick_experts(torch.zeros(2, 300, device=DEV), 2)):
        with pytest.raises(xe.XorencError):
            call()
    for call in (lambda: xe.pick_experts(None, 2), lambda: xe.pick_experts(x, "2"), lambda: xe.sort_tokens([1], 2), lambda: xe.gather_tokens(x, None, offsets)):
        with pytest.raises(TypeError):
            call()


def test_on_another_stream_and_in_graphs():
    g = gen(6)
    T, P, E, H = 2600, 8, 40, 264   # (a sort with a workspace)
    x, residual = normal(g, T, H, dtype=torch.bfloat16).to(DEV), normal(g, T, H, dtype=torch.bfloat16).to(DEV)
    logits = normal(g, T, E).to(DEV)

    def whole():
        ids, shares = xe.pick_experts(logits, P)
        places, tokens, offsets = xe.sort_tokens(ids, E)
        R = xe.gather_tokens(x, places, offsets)
        Y = xe.combine_tokens(R, places, offsets, shares, residual)
        return (ids, shares, places, tokens, offsets, R, Y, *xe.combine_tokens_grad(Y, R, places, offsets, shares))
    want = whole()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = whole()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = whole()
        graphs.append((graph, out))
    for k in range(3):
        logits.copy_(normal(g, T, E))
        x.copy_(normal(g, T, H, dtype=torch.bfloat16))
        want = whole()
        for graph, out in graphs:
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), k
