"""The tokens' rows there and back where they pass the caches by: 16-bit calls that read or write more than 2^26 values, whose kernels have loads and stores of
their own.  Each is compared with its definition in 64 bits, and bit by bit with the same call on a third of the columns at a time, which goes through the
caches (columns have nothing to do with each other, but for the gradient's inner products).  Tolerances as in test_gpu_tokens.py.  And the sort of
so many pairs that its segments are long, with ids of 64 bits."""
import pytest
import torch

import paper_1905_10138_amd as xe

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
MOST = 1 << 26          # values that a call may move through the caches

# (picks, columns): two, four, eight and more picks at a time; a workgroup of 64 and of 256 threads a token in the gradient; widths that end inside a piece of
# eight, in the last of several passes of a workgroup, before the first piece is full, and on a piece's end
SIZES = [(1, 4099), (2, 1357), (3, 2050), (4, 515), (6, 331), (8, 1024), (9, 4101), (16, 263), (2, 5)]


class Rows:
    """Inputs of a call that moves more than MOST values: x (tokens, columns) and r (pairs, columns), a fifth of the pairs without an expert."""

    def __init__(self, P, H, E=16):
        self.P, self.H, self.T = P, H, MOST // ((P + 1) * H) + 5
        self.g = torch.Generator(device=DEV).manual_seed(P + H)
        T, g = self.T, self.g
        assert T * P < 1 << 24 and T * (P + 1) * H > MOST and T * (2 * P + 1) * -(-H // 3) <= MOST
        ids = torch.randint(0, E, (T, P), generator=g, device=DEV, dtype=torch.int32)
        ids[torch.rand((T, P), generator=g, device=DEV) < 0.2] = -1
        self.places, self.tokens, self.offsets = xe.sort_tokens(ids, E)
        self.used = int(self.offsets[-1])
        assert 0 < self.used < T * P
        self.at, self.have = self.places.long(), self.places < self.used
        self.shares = torch.rand((T, P), generator=g, device=DEV)

    def normal(self, rows):
        return torch.randn((rows, self.H), generator=self.g, device=DEV).to(torch.bfloat16)

    def thirds(self):
        step = -(-self.H // 3)
        return [slice(c, min(c + step, self.H)) for c in range(0, self.H, step)]

    def apart(self, t):
        """The same values in rows of another leading dimension, off 16-byte boundaries; and what is around them."""
        wide = torch.full((t.shape[0] + 2, self.H + 13), 77.0, dtype=t.dtype, device=DEV)
        wide[1:-1, 5:5 + self.H] = t
        return wide, wide[1:-1, 5:5 + self.H]


def untouched(wide, H):
    return bool((wide[0] == 77).all() and (wide[-1] == 77).all() and (wide[:, :5] == 77).all() and (wide[:, 5 + H:] == 77).all())


def close(got, want, off):
    """|got - want| <= off, off and want in 64 bits."""
    return bool(((got.double() - want).abs() <= off).all())


@pytest.mark.parametrize("P,H", SIZES)
def test_there(P, H):
    s = Rows(P, H)
    x = s.normal(s.T)
    # without shares a copy; with them one product of fp32, rounded to 16 bits
    copy = torch.zeros((s.T * P, H), dtype=x.dtype, device=DEV)
    copy[s.at[s.have]] = x.unsqueeze(1).expand(-1, P, -1)[s.have]
    assert torch.equal(xe.gather_tokens(x, s.places, s.offsets), copy)
    R = xe.gather_tokens(x, s.places, s.offsets, s.shares)
    copy[s.at[s.have]] = (x.float().unsqueeze(1) * s.shares.unsqueeze(2))[s.have].to(x.dtype)
    assert torch.equal(R, copy)
    del copy
    for c in s.thirds():
        assert torch.equal(R[:, c], xe.gather_tokens(x[:, c], s.places, s.offsets, s.shares))
    around, out = s.apart(torch.full_like(R, 3.0))
    assert xe.gather_tokens(s.apart(x)[1], s.places, s.offsets, s.shares, R=out) is out
    assert torch.equal(out, R) and untouched(around, H)


@pytest.mark.parametrize("P,H", SIZES)
def test_back(P, H):
    s = Rows(P, H)
    rows, residual = s.normal(s.T * P), s.normal(s.T)
    for shares in (None, s.shares):
        want, mag = torch.zeros((s.T, H), dtype=torch.float64, device=DEV), torch.zeros((s.T, H), dtype=torch.float64, device=DEV)
        for p in range(P):
            term = torch.where(s.have[:, p:p + 1], rows[s.at[:, p]].double(), 0.0) * (1.0 if shares is None else shares[:, p:p + 1].double())
            want += term
            mag += term.abs_()
        for r in (None, residual):
            if r is not None:
                want += r.double()
                mag += r.double().abs()
            Y = xe.combine_tokens(rows, s.places, s.offsets, shares, r)
            assert close(Y, want, 1.01 * ((P + 1) * U * mag + 2.0 ** -8 * want.abs()))
    for c in s.thirds():
        assert torch.equal(Y[:, c], xe.combine_tokens(rows[:, c], s.places, s.offsets, s.shares, residual[:, c]))
    around, out = s.apart(residual)     # onto the residual itself
    assert xe.combine_tokens(s.apart(rows)[1], s.places, s.offsets, s.shares, out, Y=out) is out
    assert torch.equal(out, Y) and untouched(around, H)


@pytest.mark.parametrize("P,H", SIZES)
def test_the_gradient(P, H):
    s = Rows(P, H)
    dy, rows = s.normal(s.T), s.normal(s.T * P)
    rows[s.used:] = float("nan")        # (not read)
    dR, dshares = xe.combine_tokens_grad(dy, rows, s.places, s.offsets, s.shares)
    assert torch.equal(dR, xe.gather_tokens(dy, s.places, s.offsets, s.shares))
    for c in s.thirds():
        assert torch.equal(dR[:, c], xe.combine_tokens_grad(dy[:, c], rows[:, c], s.places, s.offsets, s.shares)[0])
    for p in range(P):
        terms = torch.where(s.have[:, p:p + 1], rows[s.at[:, p]].double(), 0.0) * dy.double()
        assert close(dshares[:, p], terms.sum(1), (H / 256 + 32) * U * terms.abs().sum(1))
    assert (dshares[~s.have] == 0).all()
    around, out = s.apart(rows)         # dR in the place of R
    got = xe.combine_tokens_grad(s.apart(dy)[1], out, s.places, s.offsets, s.shares, dR=out)
    assert torch.equal(out, dR) and torch.equal(got[1], dshares) and untouched(around, H)


def test_in_a_graph():
    s = Rows(2, 1357)
    x, residual = s.normal(s.T), s.normal(s.T)

    def whole():
        R = xe.gather_tokens(x, s.places, s.offsets)
        Y = xe.combine_tokens(R, s.places, s.offsets, s.shares, residual)
        return (R, Y, *xe.combine_tokens_grad(Y, R, s.places, s.offsets, s.shares))
    whole()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = whole()
    for k in range(3):
        x.copy_(s.normal(s.T))
        s.shares.copy_(torch.rand(s.shares.shape, generator=s.g, device=DEV))
        want = whole()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k


@pytest.mark.parametrize("T,P,E", [(262144, 2, 9), (600000, 2, 200), (65536, 8, 256), (174763, 3, 64)])
def test_sort_of_many_wide_ids(T, P, E):
    g = torch.Generator().manual_seed(T)
    assert T * P >= 1 << 19
    ids = torch.randint(-1, E + 1, (T, P), generator=g)
    far = torch.rand((T, P), generator=g) < 0.05        # their low halves would be experts
    ids = torch.where(far, ids + (torch.randint(1, 4, (T, P), generator=g) << 32), ids)
    places, tokens, offsets = xe.sort_tokens(ids.to(DEV), E)
    key = torch.where((ids < 0) | (ids >= E), E, ids).reshape(-1)
    order = torch.sort(key, stable=True).indices
    assert torch.equal(tokens.cpu().long(), order // P) and torch.equal(places.cpu().reshape(-1)[order].long(), torch.arange(T * P))
    assert offsets.tolist() == [0] + torch.bincount(key, minlength=E + 1)[:E].cumsum(0).tolist()
    narrow = xe.sort_tokens(key.view(T, P).to(torch.int32).to(DEV), E)
    assert all(torch.equal(a, b) for a, b in zip((places, tokens, offsets), narrow))
