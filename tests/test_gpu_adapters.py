"""lp_linear_adapters and lp_qkv_projection_adapters against the definition in 64 bits.

Tolerance.  Sums of bf16 products are formed in binary32, at most d_in / 32 + 2 rank / 32 of them one after the other with a few
roundings around (bias, wavefronts' parts): c = (d_in / 32 + rank / 16 + 24) 2^-24 of the sum of magnitudes.  t = s D x carries the same error, and
2^-17 of itself as two bf16.  So a projection is off by
    c (|W| |x| + |b| + s |U| |D| |x|) + 2^-17 |U| |t|,
formed element by element below, and by 2^-8 of the result when it is rounded.  A head that is normalised multiplies this by gain / rms, once for the
element and once, through the rms, for all of them (at most the largest of them times |v|); a rotation adds what both elements of a pair are off by,
and angles of p radians in binary32 turns are off by (p + 1) 2^-21 with the hardware's sine and cosine (2^-18) behind them.
"""
import ctypes as C

import numpy as np
import pytest

from paper_2512_07350_amd import binding as lp
from tests import routes

pytestmark = pytest.mark.gpu

EPS = 1e-6


def way(lengths, ranks, d_in, d_out, head_dim=0, cus=None):
    """What a call runs: routes.GemmWay, and the tile of the down products ((0, 0): one launch for all)."""
    fn = lp._lib().lp_internal_adapted_way
    fn.argtypes = [C.POINTER(C.c_int64), C.POINTER(C.c_int32), C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int64)]
    starts = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    out = (C.c_int64 * 8)()
    assert fn((C.c_int64 * len(starts))(*starts), (C.c_int32 * len(ranks))(*ranks), len(ranks), d_in, d_out, head_dim, routes._cus(cus), out) == 0
    return routes.GemmWay((out[0], out[1]), (out[2], out[3]) if out[2] else None, out[4], out[5]), (out[6], out[7])


class Case:
    def __init__(self, lengths, ranks, d_in, d_out, sections=1, bias=True, seed=1, up=0.2, own=True, x_scale=1.0):
        import torch
        self.lengths, self.ranks, self.d_in, self.d_out, self.sections = list(lengths), list(ranks), d_in, d_out, sections
        self.starts = np.concatenate([[0], np.cumsum(lengths)]).tolist()
        self.n = self.starts[-1]
        gen = torch.Generator(device="cuda").manual_seed(9000 + 7 * seed + self.n)
        f = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
        bf = lambda t: t.to(torch.bfloat16)
        self.x = bf(x_scale * f(self.n, d_in))
        self.w = bf(f(d_out, d_in) * d_in ** -0.5)
        self.bias = 0.5 * f(d_out) if bias else None
        self.adapters = [(bf(f(sections * r, d_in) * d_in ** -0.5), bf(up * f(d_out, r)), 0.75 + 0.25 * i) if r else None
                         for i, r in enumerate(self.ranks)]

    def workspace(self, extra=0):
        import torch
        size = lp.lp_adapter_workspace_size(self.n, max(self.ranks), self.sections)
        # NaN everywhere: what no one wrote in this call shows
        return torch.full((size // 2 + 64 + extra,), float("nan"), dtype=torch.bfloat16, device="cuda"), size

    def want(self, rows=slice(None)):
        """(projection in 64 bits, what binary32 may be off by) of the rows."""
        import torch
        c = (self.d_in / 32 + max(self.ranks) / 16 + 24) * 2.0 ** -24
        index = torch.arange(self.n, device="cuda")[rows]
        x, w = self.x[index].double(), self.w.double()
        y = x @ w.t()
        off = c * (x.abs() @ w.abs().t())
        if self.bias is not None:
            y += self.bias.double()
            off += c * self.bias.double().abs()
        part = self.d_out // self.sections
        for r, ad in enumerate(self.adapters):
            here = (index >= self.starts[r]) & (index < self.starts[r + 1])
            if ad is None or not bool(here.any()):
                continue
            down, up, scale = ad[0].double(), ad[1].double(), float(np.float32(ad[2]))
            rank = up.shape[1]
            t, ta = scale * (x[here] @ down.t()), scale * (x[here].abs() @ down.abs().t())
            for s in range(self.sections):
                cols, k = slice(s * part, (s + 1) * part), slice(s * rank, (s + 1) * rank)
                y[here, cols] += t[:, k] @ up[cols].t()
                off[here, cols] += (c * ta[:, k] + 2.0 ** -17 * t[:, k].abs()) @ up[cols].abs().t() + c * (ta[:, k] @ up[cols].abs().t())
        return y, off

    def linear(self, extra=3):
        import torch
        y = torch.full((self.n + extra, self.d_out), 77.0, dtype=torch.bfloat16, device="cuda")
        ws, size = self.workspace()
        lp.lp_linear_adapters(self.x, self.w, self.bias, y, lp.make_requests(self.starts), self.d_in, self.d_out, lp.make_adapters(self.adapters), ws, size,
                              torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.isnan(ws[size // 2:].float()).all()
        assert (y[self.n:] == 77.0).all()
        return y[:self.n]


def inside(got, want, off, what=""):
    import torch
    assert got.shape == want.shape and torch.isfinite(got.float()).all(), what
    excess = (got.double() - want).abs() - (off + 2.0 ** -8 * (want.abs() + off))
    assert float(excess.max()) <= 0, (what, float(excess.max()), divmod(int(excess.argmax()), want.shape[-1]))


# one token to several tiles, requests that share tiles, without rows, without adapters, ranks of part of a k-tile, one and several, k of
# fewer k-tiles than stages
@pytest.mark.parametrize("lengths,ranks,d_in,d_out", [
    ([1], [8], 64, 128), ([1, 1, 1], [8, 0, 40], 64, 384), ([5, 0, 12, 3], [16, 24, 0, 64], 128, 256), ([33, 31], [32, 256], 192, 128),
    ([64, 64, 64], [8, 16, 32], 320, 640), ([130, 1, 127, 300], [72, 8, 136, 0], 448, 1152), ([1] * 64, [8 * (1 + i % 5) for i in range(64)], 512, 512),
    ([257, 255, 1], [128, 0, 96], 1536, 1536), ([520], [64], 5120, 640), ([700, 800], [48, 200], 2112, 1408),
])
def test_linear_adapters(lengths, ranks, d_in, d_out):
    for bias in (True, False):
        c = Case(lengths, ranks, d_in, d_out, bias=bias)
        inside(c.linear(), *c.want(), (lengths, ranks))


TILINGS = [
    # wavefronts that share k (3 and 9 k-tiles, fewer and more than its 8 stages, 17 and 30), 64 x 64, four wavefronts to 256 features
    (40, 192, 640, "64x32"), (77, 576, 896, "64x32"), (33, 1088, 384, "64x32"), (95, 1920, 256, "64x32"), (150, 64, 1152, "64x64"), (300, 320, 2048, "64x64"),
    (4033, 2112, 1536, "256x128"), (2560, 4096, 6144, "256x256"), (4097, 2112, 4224, "256x256+128x128"), (4353, 2112, 4096, "256x256+128x64"),
    (6145, 2176, 3584, "256x256+256x128"),
    (66, 64, 8448, "128x64"), (1438, 1024, 1152, "128x64"), (1345, 576, 1536, "128x128"), (75077, 64, 128, "128x128+128x64"),
    (12001, 1024, 384, "256x128"), (3783, 128, 3840, "256x256"), (3600, 128, 4608, "256x256+128x64"), (4097, 1024, 4608, "256x256+128x128"),
    (3601, 512, 6144, "256x256+256x128"),
]


@pytest.mark.parametrize("n,d_in,d_out,tiles", TILINGS)
def test_linear_adapters_of_every_tiling(n, d_in, d_out, tiles):
    """Four requests whose edges lie inside tiles, one in the middle without adapter."""
    lengths = [n // 3 + 5, n // 4, n // 5, 0]
    lengths[3] = n - sum(lengths)
    ranks = [72, 0, 16, 32]                              # 72: two launches
    assert str(way(lengths, ranks, d_in, d_out)[0]) == tiles and way(lengths, ranks, d_in, d_out)[1] != (0, 0)
    c = Case(lengths, ranks, d_in, d_out)
    y = c.linear()
    edges = [s + i for s in c.starts for i in (-2, -1, 0, 1) if 0 <= s + i < n]
    import torch
    rows = torch.tensor(sorted(set(edges + list(range(0, n, max(1, n // 400))) + list(range(min(n, 40))))), device="cuda")
    inside(y[rows], *c.want(rows), tiles)
    assert torch.isfinite(y.float()).all()


@pytest.mark.parametrize("d_in", [64, 192, 1088, 2112])
@pytest.mark.parametrize("lengths,ranks,tile", [
    ([40, 1, 33], [8, 72, 256], (64, 32)),
    ([9000, 77, 3], [16, 72, 64], (64, 128)), ([3000, 0, 6000, 130], [64, 8, 40, 0], (64, 128)),
    ([3000, 2501], [128, 96], (128, 64)), ([65, 4000, 63], [200, 136, 8], (128, 64)),
])
def test_down_products_of_every_tile(lengths, ranks, tile, d_in):
    """t itself: W and the bias are zero, so that nothing but the adapters is in y."""
    import torch
    assert way(lengths, ranks, d_in, 128)[1] == tile
    c = Case(lengths, ranks, d_in, 128, bias=False)
    c.w.zero_()
    y = c.linear()
    rows = torch.tensor(sorted(set(list(range(0, c.n, max(1, c.n // 700))) + [s + i for s in c.starts for i in range(-3, 3) if 0 <= s + i < c.n])), device="cuda")
    inside(y[rows], *c.want(rows))
    assert torch.isfinite(y.float()).all()


# one token to eight token tiles, ranks of one group of 8 rows to all eight, runs that share a tile, have none of its rows or no rows at all, fewer
# and more k-tiles than stages
@pytest.mark.parametrize("lengths,ranks", [
    ([1], [8]), ([1], [64]), ([1, 1, 1, 1, 1, 1, 1, 1], [8] * 8), ([3, 0, 1, 40, 2], [16, 8, 0, 24, 8]), ([31, 1, 33], [40, 0, 24]),
    ([200, 56], [32, 32]), ([70, 60, 50], [8, 48, 0]),
    # more ranks in all than a tile takes, up to it in one; a tile's last run the next one's first
    ([32, 32, 32, 64], [64, 64, 56, 8]), ([40, 24, 20, 13, 31, 32], [40, 24, 40, 16, 8, 64]), ([8] * 32, [16] * 32), ([33, 63, 33, 63], [32, 32, 32, 32]),
])
@pytest.mark.parametrize("d_in,d_out", [(64, 128), (192, 640), (576, 384), (1088, 256), (2112, 1536)])
def test_few_rows_in_one_launch(lengths, ranks, d_in, d_out):
    assert way(lengths, ranks, d_in, d_out)[1] == (0, 0)
    c = Case(lengths, ranks, d_in, d_out, bias=d_in != 192, seed=21)
    inside(c.linear(), *c.want(), (lengths, ranks))
    c = Case(lengths, ranks, d_in, d_out, bias=False, seed=22, up=10.0)
    c.w.zero_()
    inside(c.linear(), *c.want(), (lengths, ranks))


@pytest.mark.parametrize("heads,grids,ranks", [
    (4, [(2, 3, 5), (1, 1, 2), (4, 2, 8), (1, 5, 3), (2, 7, 7)], [48, 16, 64, 0, 64]),
    (2, [(1, 1, 1)], [8]), (4, [(5, 8, 5), (1, 1, 1), (3, 5, 7)], [8, 0, 16]), (8, [(2, 3, 5), (0, 1, 1), (1, 7, 3)], [24, 8, 32]), (20, [(1, 2, 9)], [64]),
])
def test_qkv_of_few_rows_in_one_launch(heads, grids, ranks):
    c = Qkv(grids, ranks, heads, 64, seed=23)
    assert way(c.lengths, ranks, c.d_in, c.d_out, 64)[1] == (0, 0)
    c.check()


@pytest.mark.parametrize("where", ["x", "down", "up"])
def test_few_rows_with_a_request_of_nan(where):
    import torch
    c = Case([7, 9, 20], [16, 24, 16], 320, 384)
    assert way(c.lengths, c.ranks, 320, 384)[1] == (0, 0)
    if where == "x":
        c.x[8, 3], c.x[15, 319] = float("nan"), float("inf")
    else:
        c.adapters[1][0 if where == "down" else 1].view(-1)[-1] = float("inf")
    y = c.linear()
    for rows in (slice(0, 7), slice(16, 36)):
        inside(y[rows], *c.want(rows))
    if where == "up":
        assert torch.isnan(y[7:16, -1].float()).all()


def test_more_elements_than_32_bits_count():
    """x of 2.2e9 elements; rows at its ends, at the border of the requests and behind element 2^31."""
    import torch
    c = Case([200000, 160001], [16, 32], 6144, 128)
    y = c.linear()
    rows = torch.tensor([0, 1, 199999, 200000, 349524, 349525, 349526, 349530, 359999, 360000], device="cuda")
    inside(y[rows], *c.want(rows))


def test_large_adapters_beside_small_weights():
    """The adapter's part a hundred times the projection's: t keeps 17 bits."""
    c = Case([300, 50], [64, 16], 512, 256, up=20.0)
    inside(c.linear(), *c.want())


def test_neighbours_with_one_adapter_are_one_run():
    import torch
    c = Case([200, 0, 311, 77], [32, 16, 32, 0], 256, 384)
    c.adapters[2] = c.adapters[0]
    a = c.linear()
    inside(a, *c.want())
    joined = Case([511, 77], [32, 0], 256, 384)
    joined.x, joined.w, joined.bias, joined.adapters = c.x, c.w, c.bias, [c.adapters[0], None]
    assert torch.equal(a, joined.linear())


def test_requests_without_adapters_are_the_plain_projection():
    import torch
    c = Case([300, 220], [0, 0], 1536, 1536)
    y = c.linear()
    plain = torch.empty_like(y)
    lp.lp_linear(c.x, c.w, c.bias, plain, c.n, c.d_in, c.d_out, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(y, plain)


def test_a_request_of_nan_leaves_the_others_alone():
    """NaN and infinities in one request's rows and in its adapter."""
    import torch
    c = Case([70, 30, 60], [32, 40, 16], 256, 256)
    c.x[75, 3] = float("nan")
    c.x[80] = float("inf")
    c.adapters[1][1][5, 7] = float("inf")
    y = c.linear()
    for rows in (slice(0, 70), slice(100, 160)):
        inside(y[rows], *c.want(rows))
    assert torch.isnan(y[70:100].float()).all()            # what is said of an adapter that is not finite: not taken for zeros


@pytest.mark.parametrize("at", [0, 1, 1000, 81919, 2 ** 19 + 4, 5120 * 256 - 1])
def test_every_part_of_an_adapter_is_looked_over(at):
    import torch
    c = Case([20, 20, 9], [8, 256, 256], 64, 5120)
    c.adapters[1][1].view(-1)[at] = float("-inf")
    y = c.linear()
    inside(y[:20], *c.want(slice(0, 20)))
    inside(y[40:], *c.want(slice(40, 49)))
    assert torch.isnan(y[20:40].float()).all()


# ---- q | k | v

class Qkv(Case):
    def __init__(self, grids, ranks, heads, hd, bias=True, offsets=None, split=None, base=10000.0, seed=2):
        import torch
        lengths = [a * b * c for a, b, c in grids]
        super().__init__(lengths, ranks, heads * hd, 3 * heads * hd, 3, bias, seed)
        self.grids, self.heads, self.hd, self.base = grids, heads, hd, base
        hw = 2 * (hd // 6)
        self.split = split or (hd - 2 * hw, hw, hw)
        self.offsets = offsets or [(i, 3 * i, 2) for i in range(len(grids))]
        gen = torch.Generator(device="cuda").manual_seed(77 + seed)
        self.gains = [1.0 + 0.2 * torch.randn(heads, hd, generator=gen, device="cuda") for _ in range(2)]

    def run(self):
        import torch
        out = [torch.full((self.n + 2, self.heads, self.hd), 77.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        ropes = [lp.make_rope(g if g[0] * g[1] * g[2] else (1, 1, 1), o, self.split, self.base, self.hd) for g, o in zip(self.grids, self.offsets)]
        ws, size = self.workspace() if max(self.ranks) else (None, 0)
        lp.lp_qkv_projection_adapters(self.x, self.w, self.bias, self.gains[0], self.gains[1], EPS, ropes, *out, lp.make_requests(self.starts),
                                      self.heads, self.hd, lp.make_adapters(self.adapters), ws, size, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all((t[self.n:] == 77.0).all() for t in out)
        return [t[:self.n] for t in out]

    def angles(self):
        import torch
        out = []
        for g, o in zip(self.grids, self.offsets):
            i = torch.arange(g[0] * g[1] * g[2], device="cuda")
            where = (i // (g[1] * g[2]) + o[0], i // g[2] % g[1] + o[1], i % g[2] + o[2]) if len(i) else (i, i, i)
            out.append(torch.stack([where[ax].double() * self.base ** (-2.0 * j / p) for ax, p in enumerate(self.split) for j in range(p // 2)], 1))
        return torch.cat(out)

    def check(self, rows=slice(None)):
        import torch
        got = self.run()
        y, off = self.want(rows)
        m, dm = y.shape[0], self.heads * self.hd
        inside(got[2][rows].reshape(m, dm), y[:, 2 * dm:], off[:, 2 * dm:], "v")
        angle = self.angles()[rows][:, None]
        cos, sin = angle.cos(), angle.sin()
        turn = (angle.abs() + 1.0) * 2.0 ** -21 + 2.0 ** -18
        for p, name in enumerate("qk"):
            z = y[:, p * dm:(p + 1) * dm].reshape(m, self.heads, self.hd)
            o = off[:, p * dm:(p + 1) * dm].reshape(m, self.heads, self.hd)
            inv = 1.0 / torch.sqrt((z * z).mean(-1, keepdim=True) + EPS)
            gain = self.gains[p].double()
            v = z * inv * gain
            ov = inv * gain.abs() * (o + (z * inv).abs() * o.max(-1, keepdim=True).values) + 2.0 ** -20 * v.abs()
            a, b, oa, ob = v[..., 0::2], v[..., 1::2], ov[..., 0::2], ov[..., 1::2]
            size = oa + ob + turn * (a.abs() + b.abs())
            want = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).reshape(m, dm)
            inside(got[p][rows].reshape(m, dm), want, torch.stack((size, size), -1).reshape(m, dm), name)
        assert all(torch.isfinite(t.float()).all() for t in got)


@pytest.mark.parametrize("grids,ranks,heads,hd", [
    ([(1, 1, 1)], [8], 2, 64), ([(1, 1, 1)] * 3 + [(2, 1, 1)], [8, 0, 16, 8], 1, 128),
    ([(2, 5, 7), (1, 1, 1), (3, 3, 4)], [16, 0, 40], 2, 64), ([(3, 4, 30), (5, 2, 9)], [32, 256], 1, 128),
    ([(3, 10, 13), (3, 10, 13), (0, 1, 1), (7, 3, 11)], [64, 64, 8, 16], 12, 128),
    ([(1, 1, 3)] * 64, [8 * (i % 3) for i in range(64)], 4, 64), ([(5, 7, 3), (2, 2, 2)], [0, 0], 4, 64),
])
def test_qkv_adapters(grids, ranks, heads, hd):
    Qkv(grids, ranks, heads, hd).check()
    Qkv(grids, ranks, heads, hd, bias=False, split=(hd, 0, 0), base=100.0).check()


@pytest.mark.parametrize("heads,hd,grid,tiles", [
    (8, 64, (3, 5, 9), "64x32"), (20, 64, (3, 3, 11), "64x32"), (2, 64, (3, 6, 6), "64x64"), (4, 64, (9, 11, 13), "64x64"),
    (2, 64, (3, 23, 39), "128x64"), (8, 128, (3, 5, 9), "128x64"), (1, 128, (1, 5, 5), "128x64"), (16, 64, (3, 13, 17), "128x128"),
    (8, 128, (3, 20, 20), "128x128"), (36, 128, (6, 10, 10), "128x128+128x64"), (8, 64, (23, 13, 9), "256x128"), (4, 128, (9, 23, 13), "256x128"),
    (8, 64, (11, 33, 15), "256x256"), (10, 128, (7, 23, 23), "256x256"), (6, 64, (22, 18, 33), "256x256+128x64"),
    (12, 128, (9, 20, 20), "256x256+128x64"), (10, 64, (18, 27, 19), "256x256+128x128"), (6, 128, (19, 12, 36), "256x256+128x128"),
    (10, 64, (18, 19, 30), "256x256+256x128"), (3, 128, (16, 34, 33), "256x256+256x128"),
])
def test_qkv_adapters_of_every_tiling(heads, hd, grid, tiles):
    """The grid in three requests along its first axis, as far as it has them."""
    import torch
    t = grid[0]
    grids = [(a,) + grid[1:] for a in (t - t // 2 - t // 3, t // 3, t // 2)]
    c = Qkv(grids, [72, 0, 40], heads, hd)
    assert str(way(c.lengths, c.ranks, c.d_in, c.d_out, hd)[0]) == tiles
    edges = [s + i for s in c.starts for i in (-2, -1, 0, 1) if 0 <= s + i < c.n]
    c.check(torch.tensor(sorted(set(edges + list(range(0, c.n, max(1, c.n // 150))))), device="cuda"))


def test_qkv_without_adapters_is_the_plain_projection_of_each_request():
    import torch
    c = Qkv([(3, 5, 7), (2, 9, 4)], [0, 0], 4, 128)
    got = c.run()
    for r, (g, o) in enumerate(zip(c.grids, c.offsets)):
        rows = slice(c.starts[r], c.starts[r + 1])
        plain = [torch.empty(c.lengths[r], c.heads, c.hd, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        lp.lp_qkv_projection(c.x[rows], c.w, c.bias, c.gains[0], c.gains[1], EPS, lp.make_rope(g, o, head_dim=c.hd), *plain, c.lengths[r], c.heads, c.hd,
                             torch.cuda.current_stream().cuda_stream)
        for a, b in zip(got, plain):
            # another tiling may add up in another order; the rounding is the same but where a sum lies next to a border
            assert (a[rows].float() - b.float()).abs().max() <= 2.0 ** -7 * b.float().abs().max()


# ---- as they are used

def test_two_calls_on_two_streams_with_a_workspace_each():
    import torch
    a, b = Case([900, 600], [64, 16], 1536, 1536, seed=3), Case([700, 800], [32, 32], 1536, 1536, seed=4)
    want = [c.linear().clone() for c in (a, b)]
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for c in (a, b):
        outs.append((torch.empty(c.n, c.d_out, dtype=torch.bfloat16, device="cuda"), c.workspace()))
    torch.cuda.synchronize()
    for _ in range(5):
        for c, st, (y, (ws, size)) in zip((a, b), streams, outs):
            lp.lp_linear_adapters(c.x, c.w, c.bias, y, lp.make_requests(c.starts), c.d_in, c.d_out, lp.make_adapters(c.adapters), ws, size, st.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for (y, _), w in zip(outs, want))


def test_two_graphs_with_a_workspace_each():
    """Calls of two launches, captured, and replayed in turn on two streams with eager calls between."""
    import torch
    cases, graphs, outs, tables = [Case([900, 0, 600, 40], [64, 8, 16, 0], 1536, 1536, seed=31), Case([300, 5000], [96, 24], 640, 384, seed=32)], [], [], []
    for c in cases:
        assert way(c.lengths, c.ranks, c.d_in, c.d_out)[1] != (0, 0)
        y, (ws, size) = torch.empty(c.n, c.d_out, dtype=torch.bfloat16, device="cuda"), c.workspace()
        call = lambda c=c, y=y, ws=ws, size=size: lp.lp_linear_adapters(c.x, c.w, c.bias, y, lp.make_requests(c.starts), c.d_in, c.d_out,
                                                                       lp.make_adapters(c.adapters), ws, size, torch.cuda.current_stream().cuda_stream)
        call()
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        graphs.append((graph, side))
        outs.append(y)
        tables.append(ws)
    for turn in range(4):
        for c, y, ws in zip(cases, outs, tables):
            c.x.mul_(0.5)
            y.fill_(float("nan"))
            ws.fill_(float("nan"))                         # contents are irrelevant on entry
        torch.cuda.synchronize()
        for graph, side in graphs:
            with torch.cuda.stream(side):
                graph.replay()
        torch.cuda.synchronize()
        for c, y in zip(cases, outs):
            assert torch.equal(y, c.linear())              # eager, with a workspace of its own
    for c, y in zip(cases, outs):
        inside(y, *c.want())


def test_the_blocks_of_two_requests_from_a_graph():
    """The self-attention half of a block over a packed batch: modulated norm, projection with adapters, attention per request, output projection with
    adapters, gated residual and the next norm.  Replayed with other inputs, and every link against its definition on what it was given."""
    import torch
    from tests import gpu_util as g
    heads, hd, grids, ranks = 4, 64, [(3, 8, 9), (2, 11, 10)], [16, 32]
    dm = heads * hd
    q = Qkv(grids, ranks, heads, hd, seed=11)
    o = Case(q.lengths, ranks[::-1], dm, dm, seed=12)
    n, starts = q.n, q.starts
    gen = torch.Generator(device="cuda").manual_seed(5)
    f = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    h, mod = f(n, dm), 0.3 * f(2, 6, dm)
    h_out, normed, y, last = torch.empty_like(h), torch.empty(n, dm, dtype=torch.bfloat16, device="cuda"), *(
        torch.empty(n, dm, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    qkv = [torch.empty(n, heads, hd, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    att = torch.empty_like(qkv[0])
    req, norm = lp.make_requests(starts), lp.make_norm(lp.LP_NORM_LAYER, EPS)
    m1, m2 = lp.make_modulation(scale=mod[:, 0], shift=mod[:, 1]), lp.make_modulation(gate=mod[:, 2], scale=mod[:, 3], shift=mod[:, 4])
    ropes = [lp.make_rope(gr, off, q.split, q.base, hd) for gr, off in zip(grids, q.offsets)]
    tq, to = lp.make_adapters(q.adapters), lp.make_adapters(o.adapters)
    (ws, size), (aws, asize) = q.workspace(), g.workspace(hd)

    def half():
        st = torch.cuda.current_stream().cuda_stream
        lp.lp_norm_modulate(h, lp.LP_F32, normed, req, dm, norm, m1, stream=st)
        lp.lp_qkv_projection_adapters(normed, q.w, q.bias, q.gains[0], q.gains[1], EPS, ropes, *qkv, req, heads, hd, tq, ws, size, st)
        for a, b in zip(starts, starts[1:]):
            lp.lp_attention(*(t[a:b] for t in qkv), att[a:b], b - a, heads, hd, dm, hd, 0.0, aws, asize, st)
        lp.lp_linear_adapters(att, o.w, o.bias, y, req, dm, dm, to, ws, size, st)
        lp.lp_gated_residual_norm(h, lp.LP_F32, y, h_out, last, req, dm, None, norm, m2, stream=st)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        half()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        half()
    results = (normed, *qkv, att, y, h_out, last)
    for scale in (1.0, 0.3, 4.0):
        h.mul_(scale)
        for t in results:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in results]
        half()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, results))
    # every link on its own inputs: rounding to bf16 and 2^-12 of the terms, which the finer tests above hold it to
    spread = lambda v: torch.repeat_interleave(v.double(), torch.tensor(q.lengths, device="cuda"), 0)
    layer = lambda t: (t - t.mean(-1, keepdim=True)) / torch.sqrt(t.var(-1, unbiased=False, keepdim=True) + EPS)
    close = lambda a, want, slack: inside(a, want, torch.full_like(want, slack))
    close(normed, layer(h.double()) * (1 + spread(mod[:, 0])) + spread(mod[:, 1]), 2.0 ** -12)
    q.x = normed
    yq, off = q.want()
    inside(qkv[2].reshape(n, dm), yq[:, 2 * dm:], off[:, 2 * dm:])
    for a, b in zip(starts, starts[1:]):
        qq, kk, vv = (t[a:b].float().permute(1, 0, 2).double() for t in qkv)
        p = torch.softmax(torch.matmul(qq, kk.transpose(1, 2).contiguous()) / hd ** 0.5, -1)
        err = (att[a:b].double() - torch.matmul(p, vv.contiguous()).permute(1, 0, 2)).abs()
        assert float(err.max()) <= 2e-2 * float(vv.abs().max()) and float(err.mean()) <= 2e-3 * float(vv.abs().max())
    o.x = att.reshape(n, dm)
    inside(y, *o.want())
    hw = h.double() + spread(mod[:, 2]) * y.double()
    close(h_out, hw, 2.0 ** -12 * float(hw.abs().max()))
    close(last, layer(hw) * (1 + spread(mod[:, 3])) + spread(mod[:, 4]), 2.0 ** -12)


def test_a_workspace_is_not_looked_at_without_adapters():
    """Neither where it lies nor how large it is."""
    import torch
    c = Qkv([(3, 5, 7), (2, 9, 4)], [0, 0], 4, 64)
    want = c.run()
    out = [torch.empty_like(t) for t in want]
    ropes = [lp.make_rope(g, o, c.split, c.base, c.hd) for g, o in zip(c.grids, c.offsets)]
    st = torch.cuda.current_stream().cuda_stream
    for ws in (c.x, c.w, out[0], out[2], c.x.data_ptr() + 2):
        lp.lp_qkv_projection_adapters(c.x, c.w, c.bias, c.gains[0], c.gains[1], EPS, ropes, *out, lp.make_requests(c.starts), c.heads, c.hd,
                                      lp.make_adapters(c.adapters), ws, 3, st)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        lin = Case(c.lengths, [0, 0], 256, 256)
        y = torch.empty(lin.n, 256, dtype=torch.bfloat16, device="cuda")
        lp.lp_linear_adapters(lin.x, lin.w, lin.bias, y, lp.make_requests(lin.starts), 256, 256, lp.make_adapters(lin.adapters), y, 3, st)
        assert torch.equal(y, lin.linear())


@pytest.mark.parametrize("same,one_launch", [(True, True), (False, False)])
def test_the_internal_say_on_a_call_is_what_it_runs(same, one_launch):
    """A call of one launch leaves its workspace as it was; the first launch of two writes its beginning.  Two requests of 64 ranks in one tile: one
    launch if they have one adapter."""
    import torch
    c = Case([10, 10], [64, 64], 512, 512, seed=41)
    if same:
        c.adapters[1] = c.adapters[0]
    req, table = lp.make_requests(c.starts), lp.make_adapters(c.adapters)
    assert (routes.adapted(req, table, 512, 512)[1] == (0, 0)) == one_launch
    y, (ws, size) = torch.empty(c.n, 512, dtype=torch.bfloat16, device="cuda"), c.workspace()
    lp.lp_linear_adapters(c.x, c.w, c.bias, y, req, 512, 512, table, ws, size, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert bool(torch.isnan(ws.float()).all()) == one_launch
    inside(y, *c.want())


# ---- calls of two launches

def test_merged_runs_of_two_launches():
    """Neighbours with one adapter, a request without rows between them, are one run in the down products and the k-tiles too."""
    import torch
    c = Case([2000, 0, 3110, 77], [72, 16, 72, 0], 576, 896, seed=51)
    c.adapters[2] = c.adapters[0]
    ways = routes.adapted(lp.make_requests(c.starts), lp.make_adapters(c.adapters), c.d_in, c.d_out)
    assert ways[1] != (0, 0)
    y = c.linear()
    rows = torch.tensor(sorted(set(range(0, c.n, 17)) | {1999, 2000, 2001, 5109, 5110, 5186}), device="cuda")
    inside(y[rows], *c.want(rows))
    joined = Case([5110, 77], [72, 0], 576, 896)
    joined.x, joined.w, joined.bias, joined.adapters = c.x, c.w, c.bias, [c.adapters[0], None]
    assert routes.adapted(lp.make_requests(joined.starts), lp.make_adapters(joined.adapters), c.d_in, c.d_out) == ways
    assert torch.equal(y, joined.linear())


def test_one_workspace_for_the_calls_of_a_stream():
    """q | k | v, then a projection with other adapters of other requests, in one workspace, again and again with nothing between them: eager, and
    from a graph that replays with eager calls in the same workspace between."""
    import torch
    q = Qkv([(3, 20, 20), (5, 9, 11), (1, 1, 1)], [72, 0, 40], 4, 64, seed=52)
    o = Case([900, 0, 595, 200, 1], [16, 8, 128, 32, 0], 256, 256, seed=53)
    p = Case([q.n], [96], 256, 256, seed=54)
    tables = [lp.make_adapters(c.adapters) for c in (q, o, p)]
    requests = [lp.make_requests(c.starts) for c in (q, o, p)]
    for c, r, t, hd in zip((q, o, p), requests, tables, (64, 0, 0)):
        assert routes.adapted(r, t, c.d_in, c.d_out, hd)[1] != (0, 0)
    want = [*q.run(), o.linear(), p.linear()]             # a workspace each
    size = max(lp.lp_adapter_workspace_size(q.n, 72, 3), lp.lp_adapter_workspace_size(o.n, 128, 1), lp.lp_adapter_workspace_size(p.n, 96, 1))
    ws = torch.full((size // 2 + 64,), float("nan"), dtype=torch.bfloat16, device="cuda")
    out = [torch.empty_like(t) for t in want]
    ropes = [lp.make_rope(g, off, q.split, q.base, q.hd) for g, off in zip(q.grids, q.offsets)]

    def calls():
        st = torch.cuda.current_stream().cuda_stream
        lp.lp_qkv_projection_adapters(q.x, q.w, q.bias, q.gains[0], q.gains[1], EPS, ropes, *out[:3], requests[0], q.heads, q.hd, tables[0], ws, size, st)
        lp.lp_linear_adapters(o.x, o.w, o.bias, out[3], requests[1], o.d_in, o.d_out, tables[1], ws, size, st)
        lp.lp_linear_adapters(p.x, p.w, p.bias, out[4], requests[2], p.d_in, p.d_out, tables[2], ws, size, st)

    def check():
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.isnan(ws[size // 2:].float()).all()
        for t in out:
            t.fill_(77.0)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            calls()
    side.synchronize()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
        calls()
    for _ in range(4):
        graph.replay()
        check()
        calls()
        check()


@pytest.mark.parametrize("value", ["inf", "nan"])
@pytest.mark.parametrize("n,d_in,d_out,tiles", [
    (1438, 1024, 1152, "128x64"), (1345, 576, 1536, "128x128"), (12001, 1024, 384, "256x128"), (3783, 128, 3840, "256x256"), (3600, 128, 4608, "256x256+128x64"),
    (4033, 2112, 1536, "256x128"), (2560, 4096, 6144, "256x256"), (4097, 2112, 4224, "256x256+128x128"), (6145, 2176, 3584, "256x256+256x128"),
])
def test_an_adapter_that_is_not_finite_on_large_tiles(n, d_in, d_out, tiles, value):
    """U of the second of four requests, whose edges lie inside tiles: its rows are NaN throughout, the others as ever."""
    import torch
    lengths = [n // 3 + 5, n // 4, n // 5, 0]
    lengths[3] = n - sum(lengths)
    c = Case(lengths, [72, 40, 16, 32], d_in, d_out, seed=55)
    ways = way(c.lengths, c.ranks, d_in, d_out)
    assert str(ways[0]) == tiles and ways[1] != (0, 0) and ways[0].threads == (256 if d_in >= 2112 else 512)
    c.adapters[1][1].view(-1)[-1 if value == "inf" else d_out * 20 + 3] = float(value)
    y = c.linear()
    a, b = c.starts[1], c.starts[2]
    assert torch.isnan(y[a:b].float()).all()
    edges = [s + i for s in c.starts for i in (-2, -1, 0, 1)]
    rows = torch.tensor([r for r in sorted(set(edges) | set(range(0, n, max(1, n // 300)))) if 0 <= r < n and not a <= r < b], device="cuda")
    inside(y[rows], *c.want(rows))
    assert torch.isfinite(y[:a].float()).all() and torch.isfinite(y[b:].float()).all()


@pytest.mark.parametrize("heads,hd,grid,tiles", [(8, 128, (3, 20, 20), "128x128"), (4, 128, (9, 23, 13), "256x128"), (8, 64, (11, 33, 15), "256x256"),
                                                 (12, 128, (9, 20, 20), "256x256+128x64")])
def test_a_qkv_adapter_that_is_not_finite_on_large_tiles(heads, hd, grid, tiles):
    import torch
    t = grid[0]
    c = Qkv([(a,) + grid[1:] for a in (t - t // 2 - t // 3, t // 3, t // 2)], [72, 24, 40], heads, hd, seed=56)
    ways = way(c.lengths, c.ranks, c.d_in, c.d_out, hd)
    assert str(ways[0]) == tiles and ways[1] != (0, 0)
    c.adapters[1][1][2 * c.d_in + 5, 7] = float("inf")     # of v
    want = [x.clone() for x in c.run()]
    a, b = c.starts[1], c.starts[2]
    assert torch.isnan(want[2][a:b].float()).all()
    clean = Qkv(c.grids, [72, 24, 40], heads, hd, seed=56)
    clean.check()
    for got, fine in zip(want, clean.run()):
        assert torch.equal(got[:a], fine[:a]) and torch.equal(got[b:], fine[b:])
