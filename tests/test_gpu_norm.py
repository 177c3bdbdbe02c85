"""lp_norm_modulate and lp_gated_residual_norm against the definition in 64 bits.

Tolerance.  Sums run over at most 24 elements of a thread one after the other, six exchanges between lanes and 16 wavefronts:
fewer than 64 roundings of 2^-24 with the scaling behind them, so that a sum is off by less than 2^-18 of the sum of magnitudes.  With
a = mean |x| / sqrt(var + eps), a normalised element v is off by 2^-18 (1 + a + |v|); the weights multiply that, and what is added
behind them rounds a few times (2^-22 of the terms).  The store rounds by 2^-8 of the value (bf16) or 2^-24 (binary32).  What
the residual's sum is off by passes through the normalisation behind it as (delta + mean delta) / sqrt(var + eps), and as much
again times |v| through the variance.
"""
import numpy as np
import pytest

from paper_2512_07350_amd import binding as lp
from paper_2512_07350_amd import synth

pytestmark = pytest.mark.gpu

KINDS = {"layer": lp.LP_NORM_LAYER, "rms": lp.LP_NORM_RMS}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _norm64(x, kind, eps, w, b):
    """(normalised x times weight plus bias, what binary32 may be off by, 1 / sqrt(var + eps), |v|)"""
    c = x - x.mean(-1, keepdims=True) if kind == "layer" else x
    inv = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    v = c * inv
    off = 2.0 ** -18 * (1.0 + np.abs(x).mean(-1, keepdims=True) * inv + np.abs(v))
    w = 1.0 if w is None else w.astype(np.float64)
    b = 0.0 if b is None else b.astype(np.float64)
    return v * w + b, off * np.abs(w) + 2.0 ** -22 * np.abs(b), inv * np.abs(w), np.abs(v)


def _inside(got, want, off, half, what):
    assert got.shape == want.shape and np.all(np.isfinite(got)), what
    excess = np.abs(got - want) - (off + half * (np.abs(want) + off))
    assert excess.max() <= 0, (what, float(excess.max()), np.unravel_index(excess.argmax(), excess.shape))


class Case:
    """Inputs on the host, and what a call on them gives."""

    def __init__(self, lengths, d, x="bf16", norm="layer", post=None, affine=True, modulated=True, eps=1e-6, seed=1, offset=0.5, spread=1.0):
        self.lengths, self.d, self.x, self.norm, self.post, self.eps = lengths, d, x, norm, post, eps
        self.starts = np.concatenate([[0], np.cumsum(lengths)]).tolist()
        n = self.n = self.starts[-1]
        f = lambda i, *shape: synth.normal_f32(7000 + 31 * d + seed, shape, substream=i)
        self.round = (lambda v: synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(v))) if x == "bf16" else (lambda v: v)
        self.h = self.round(np.float32(spread) * f(1, n, d) + np.float32(offset))
        self.u = synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(f(2, n, d)))
        self.vec = {k: 0.3 * f(3 + i, len(lengths), d) if modulated else None for i, k in enumerate(("gate", "scale", "shift"))}
        self.w, self.b, self.pw, self.pb = (np.float32(m) + np.float32(0.2) * f(6 + i, d) if affine else None for i, m in enumerate((1, 0, 1, 0)))

    def per_row(self, name, otherwise):
        v = self.vec[name]
        return otherwise if v is None else np.repeat(v.astype(np.float64), self.lengths, axis=0)

    def modulate(self, h, h_off):
        y, off, inv, v = _norm64(h, self.norm, self.eps, self.w, self.b)
        passed = h_off + np.mean(h_off, axis=-1, keepdims=True)
        off = off + inv * passed * (1.0 + v)
        scale, shift = self.per_row("scale", 0.0), self.per_row("shift", 0.0)
        return y * (1.0 + scale) + shift, off * np.abs(1.0 + scale) + 2.0 ** -22 * (np.abs(y) * (1.0 + np.abs(scale)) + np.abs(shift))

    def residual(self):
        """(h_out, off) of the 64-bit definition."""
        u, gate, h = self.u.astype(np.float64), self.per_row("gate", 1.0), self.h.astype(np.float64)
        off = np.zeros_like(u)
        if self.post:
            u, off, _, _ = _norm64(u, self.post, self.eps, self.pw, self.pb)
        return h + gate * u, np.abs(gate) * off + 2.0 ** -22 * (np.abs(h) + np.abs(gate * u))

    # ---- on the device
    def dev(self, a, kind, pad=0, extra=0, fill=77.0):
        """Rows of `a` in a buffer of row stride d + pad with `extra` rows behind; returns (tensor, stride)."""
        import torch
        t = torch.full((self.n + extra, self.d + pad), fill, dtype=torch.bfloat16 if kind == "bf16" else torch.float32, device="cuda")
        if a is not None:
            t[:self.n, :self.d] = torch.from_numpy(np.ascontiguousarray(a)).cuda().to(t.dtype)
        return t, self.d + pad

    def host_structs(self):
        import torch
        on = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.keep = [on(a) for a in (self.w, self.b, self.pw, self.pb)] + [on(self.vec[k]) for k in ("gate", "scale", "shift")]
        w, b, pw, pb, gate, scale, shift = self.keep
        return (lp.make_requests(self.starts), lp.make_norm(KINDS[self.norm], self.eps, w, b) if self.norm else None,
                lp.make_norm(KINDS[self.post], self.eps, pw, pb) if self.post else None,
                lp.make_modulation(gate, scale, shift) if gate is not None else None)

    def type(self):
        return lp.LP_BF16 if self.x == "bf16" else lp.LP_F32

    def check_norm(self, pad=(0, 0), extra=0):
        import torch
        req, norm, _, mod = self.host_structs()
        x, sx = self.dev(self.h, self.x, pad[0])
        y, sy = self.dev(None, "bf16", pad[1], extra)
        lp.lp_norm_modulate(x, self.type(), y, req, self.d, norm, mod, sx, sy, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        got = y.float().cpu().numpy()
        want, off = self.modulate(self.h.astype(np.float64), 0.0 * self.h)
        _inside(got[:self.n, :self.d], want, off, HALF["bf16"], "y")
        assert np.all(got[:, self.d:] == 77.0) and np.all(got[self.n:] == 77.0)

    def check_residual(self, pad=(0, 0, 0, 0), extra=0):
        import torch
        req, norm, post, mod = self.host_structs()
        (h, sh), (u, su) = self.dev(self.h, self.x, pad[0]), self.dev(self.u, "bf16", pad[1])
        (o, so), (y, sy) = self.dev(None, self.x, pad[2], extra), self.dev(None, "bf16", pad[3], extra)
        lp.lp_gated_residual_norm(h, self.type(), u, o, y if self.norm else None, req, self.d, post, norm, mod, sh, su, so, sy,
                                  torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        want, off = self.residual()
        got = o.float().cpu().numpy().astype(np.float64)
        _inside(got[:self.n, :self.d], want, off, HALF[self.x], "h_out")
        gy = y.float().cpu().numpy()
        if self.norm:
            _inside(gy[:self.n, :self.d], *self.modulate(want, off), HALF["bf16"], "y")
            assert np.all(gy[:, self.d:] == 77.0) and np.all(gy[self.n:] == 77.0)
        else:
            assert np.all(gy == 77.0)
        assert np.all(got[:, self.d:] == 77.0) and np.all(got[self.n:] == 77.0)


# every number of threads to a row and elements to a thread, in whole pieces and one by one; both sides of where they change
WIDTHS = [1, 7, 8, 65, 504, 512, 520, 1016, 1024, 1025, 1032, 1153, 1536, 1544, 2048, 2056, 4096, 4097, 4104, 5120, 6144, 6152, 8192, 16383, 16384]


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_of_every_width(d, x):
    Case([3, 0, 2], d, x, "layer" if d % 16 else "rms").check_norm()
    Case([3, 0, 2], d, x, "rms" if d % 16 else "layer", affine=False).check_norm()


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_residual_of_every_width(d, x):
    Case([1, 4], d, x, "rms" if d % 16 else "layer", post="layer" if d % 16 else "rms").check_residual()
    Case([1, 4], d, x, None, post=None, affine=False).check_residual()


@pytest.mark.parametrize("norm", ["layer", "rms", None])
@pytest.mark.parametrize("post", ["layer", "rms", None])
@pytest.mark.parametrize("affine,modulated", [(True, True), (False, True), (True, False)])
def test_residual_forms(norm, post, affine, modulated):
    for x in ("bf16", "f32"):
        Case([5, 9], 264, x, norm, post, affine, modulated).check_residual()


@pytest.mark.parametrize("lengths", [[1], [0, 0, 1, 0], [1] * 64, [0, 3, 0, 0, 5, 1, 0], [2500, 1, 2499], [700] * 7])
def test_rows_find_their_request(lengths):
    for d in (128, 136, 1600):
        Case(lengths, d).check_norm()
        Case(lengths, d, "f32", "rms", "rms").check_residual()


def test_many_rows_to_a_group():
    """More rows than the chip takes at once, so that every group of threads walks over several, across requests."""
    Case([9000, 3, 0, 11000], 72).check_norm()
    Case([5000, 7001], 776, "f32", "layer", "rms").check_residual()


@pytest.mark.parametrize("d,pad", [(320, 8), (320, 3), (321, 5), (6400, 24)])
def test_padded_rows_and_what_lies_behind(d, pad):
    Case([4, 3], d).check_norm((pad, 2 * pad), extra=3)
    Case([4, 3], d, "f32", "layer", "layer").check_residual((pad, 8, 2 * pad, pad), extra=2)


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_rows_far_from_zero(norm):
    """Means a thousand times the spread, rows that are constant, and rows of zeros."""
    Case([6], 1536, "f32", norm, offset=1000.0).check_norm()
    Case([6], 5120, "f32", norm, offset=-300.0, spread=0.0).check_norm()
    Case([6], 520, "bf16", norm, offset=0.0, spread=0.0).check_norm()
    Case([6], 1536, "f32", norm, offset=3e8, spread=1e7).check_norm()


def test_one_vector_for_all_requests():
    import torch
    c = Case([3, 4, 2], 256)
    for k in c.vec:
        c.vec[k] = np.repeat(c.vec[k][:1], 3, axis=0)
    req, norm, _, _ = c.host_structs()
    scale, shift = (torch.from_numpy(c.vec[k][0]).cuda() for k in ("scale", "shift"))
    x, s = c.dev(c.h, "bf16")
    y, _ = c.dev(None, "bf16")
    lp.lp_norm_modulate(x, lp.LP_BF16, y, req, c.d, norm, lp.make_modulation(scale=scale, shift=shift), stream=torch.cuda.current_stream().cuda_stream)
    want, off = c.modulate(c.h.astype(np.float64), 0.0 * c.h)
    _inside(y.float().cpu().numpy(), want, off, HALF["bf16"], "y")


@pytest.mark.parametrize("d", [256, 259, 5120])
def test_in_place(d):
    import torch
    st = torch.cuda.current_stream().cuda_stream
    c = Case([40, 33], d, "bf16", "layer", "rms")
    req, norm, post, mod = c.host_structs()
    x, _ = c.dev(c.h, "bf16")
    y, _ = c.dev(None, "bf16")
    lp.lp_norm_modulate(x, lp.LP_BF16, y, req, d, norm, mod, stream=st)
    z = x.clone()
    lp.lp_norm_modulate(z, lp.LP_BF16, z, req, d, norm, mod, stream=st)
    assert torch.equal(z, y)
    u, _ = c.dev(c.u, "bf16")
    o, y2 = torch.empty_like(x), torch.empty_like(x)
    lp.lp_gated_residual_norm(x, lp.LP_BF16, u, o, y, req, d, post, norm, mod, stream=st)
    lp.lp_gated_residual_norm(x, lp.LP_BF16, u, x, y2, req, d, post, norm, mod, stream=st)
    assert torch.equal(x, o) and torch.equal(y, y2)


def test_a_row_of_nan_stays_alone():
    import torch
    c = Case([5, 6], 1536, "f32", "layer", "layer")
    req, norm, post, mod = c.host_structs()
    h, _ = c.dev(c.h, "f32")
    u, _ = c.dev(c.u, "bf16")
    h[4, 17] = float("nan")
    h[9, 1000] = float("inf")
    o, y = torch.empty_like(h), torch.empty_like(u)
    lp.lp_gated_residual_norm(h, lp.LP_F32, u, o, y, req, c.d, post, norm, mod, stream=torch.cuda.current_stream().cuda_stream)
    fine = [r for r in range(11) if r not in (4, 9)]
    want, off = c.residual()
    _inside(o.cpu().numpy().astype(np.float64)[fine], want[fine], off[fine], HALF["f32"], "h_out")
    wy, oy = c.modulate(want, off)
    _inside(y.float().cpu().numpy()[fine], wy[fine], oy[fine], HALF["bf16"], "y")


def test_rows_further_apart_than_32_bits():
    import torch
    stride, d, n = 3 << 28, 64, 4                          # the last row starts past 2^31 elements
    c = Case([1, 3], d, "bf16", "rms")
    req, norm, _, mod = c.host_structs()
    x = torch.empty(stride * (n - 1) + d, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    for i in range(n):
        x[i * stride:i * stride + d] = torch.from_numpy(c.h[i]).cuda().to(torch.bfloat16)
    lp.lp_norm_modulate(x, lp.LP_BF16, y, req, d, norm, mod, stride, stride, torch.cuda.current_stream().cuda_stream)
    got = np.stack([y[i * stride:i * stride + d].float().cpu().numpy() for i in range(n)])
    want, off = c.modulate(c.h.astype(np.float64), 0.0 * c.h)
    _inside(got, want, off, HALF["bf16"], "y")


def test_on_another_stream_and_replayed_from_a_graph():
    import torch
    c = Case([300, 200], 1536, "f32", "rms", "rms")
    req, norm, post, mod = c.host_structs()
    (h, _), (u, _) = c.dev(c.h, "f32"), c.dev(c.u, "bf16")
    o, y = torch.empty_like(h), torch.empty_like(u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = lambda st: (lp.lp_gated_residual_norm(h, lp.LP_F32, u, o, y, req, c.d, post, norm, mod, stream=st),
                       lp.lp_norm_modulate(o, lp.LP_F32, u, req, c.d, norm, mod, stream=st))
    with torch.cuda.stream(side):
        call(side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    keep_u = c.dev(c.u, "bf16")[0]
    with torch.cuda.graph(graph, stream=side):
        call(torch.cuda.current_stream().cuda_stream)
    for scale in (1.0, 0.5, 2.0):
        h.mul_(scale)
        u.copy_(keep_u)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (o, y, u)]
        u.copy_(keep_u)
        call(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (o, y, u)))


def test_a_row_is_the_same_in_every_batch():
    import torch
    st = torch.cuda.current_stream().cuda_stream
    for d in (776, 1153, 5120):
        c = Case([900, 1500, 600], d, "f32", "layer", "rms")
        req, norm, post, mod = c.host_structs()
        (h, _), (u, _) = c.dev(c.h, "f32"), c.dev(c.u, "bf16")
        o, y = torch.empty_like(h), torch.empty_like(u)
        lp.lp_gated_residual_norm(h, lp.LP_F32, u, o, y, req, d, post, norm, mod, stream=st)
        alone = slice(1700, 1703)
        o1, y1 = torch.empty_like(h[alone]), torch.empty_like(u[alone])
        gate, scale, shift = (torch.from_numpy(c.vec[k][1:2].copy()).cuda() for k in ("gate", "scale", "shift"))
        lp.lp_gated_residual_norm(h[alone], lp.LP_F32, u[alone], o1, y1, lp.make_requests([0, 3]), d, post, norm, lp.make_modulation(gate, scale, shift),
                                  stream=st)
        assert torch.equal(o[alone], o1) and torch.equal(y[alone], y1)


@pytest.mark.parametrize("d", [264, 1153])
@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("post", [None, "layer", "rms"])
def test_infinite_vectors_where_no_bias_stands(d, norm, post):
    """The definition has no bias there for an infinity to meet: the element is an infinity of the product's sign, and all others are as ever."""
    import torch
    st = torch.cuda.current_stream().cuda_stream
    c = Case([2, 3, 2], d, "f32", norm, post)
    c.b = c.pb = None
    inf, rows, at = float("inf"), slice(2, 5), (0, 5, d - 1)
    plus, minus = c.vec["scale"].copy(), c.vec["gate"].copy()
    plus[1, at], minus[1, at] = (inf, -inf, inf), (-inf, inf, -inf)

    def split(got, want, off, half, factor, what):
        """Infinities in their places; the rest against `want`."""
        ends = np.zeros(got.shape, bool)
        ends[rows, at] = True
        assert np.array_equal(got[rows][:, at], factor[rows][:, at] * np.array(what)), (got[rows][:, at], factor[rows][:, at])
        _inside(np.where(ends, 0.0, got), np.where(ends, 0.0, want), np.where(ends, 0.0, off), half, "the rest")

    # the scale
    want, off = c.modulate(c.h.astype(np.float64), 0.0 * c.h)
    v = _norm64(c.h.astype(np.float64), norm, c.eps, c.w, None)[0]
    assert np.abs(v[rows][:, at]).min() > 1e-6
    fine, c.vec["scale"] = c.vec["scale"], plus
    req, pre, behind, mod = c.host_structs()
    x, _ = c.dev(c.h, "f32")
    y, _ = c.dev(None, "bf16")
    lp.lp_norm_modulate(x, lp.LP_F32, y, req, d, pre, mod, stream=st)
    split(y.float().cpu().numpy().astype(np.float64), want, off, HALF["bf16"], v, (inf, -inf, inf))
    # the gate
    c.vec["scale"] = fine
    want, off = c.residual()
    u = c.u.astype(np.float64)
    u = _norm64(u, post, c.eps, c.pw, None)[0] if post else u
    assert np.abs(u[rows][:, at]).min() > 1e-6
    c.vec["gate"] = minus
    req, pre, behind, mod = c.host_structs()
    on_u, _ = c.dev(c.u, "bf16")
    o = torch.empty_like(x)
    lp.lp_gated_residual_norm(x, lp.LP_F32, on_u, o, y, req, d, behind, pre, mod, stream=st)
    split(o.cpu().numpy().astype(np.float64), want, off, HALF["f32"], u, (-inf, inf, -inf))
    others = [0, 1, 5, 6]
    wy, oy = c.modulate(want, off)
    _inside(y.float().cpu().numpy()[others], wy[others], oy[others], HALF["bf16"], "y")


# 1024 threads to a row whose last pieces lie partly or wholly past its end, in whole pieces and in single elements
@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8200, 8201, 9001, 12288, 12296, 16376])
def test_widths_between_8192_and_16384(d, x):
    Case([3, 0, 2], d, x, "layer").check_norm((8, 16), extra=1)
    Case([1, 4], d, x, "rms", post="layer").check_residual((8, 0, 16, 8), extra=1)


@pytest.mark.parametrize("d", [7001, 8192, 9001, 12296])
def test_several_wide_rows_to_a_workgroup(d):
    """512 and 1024 threads to a row: every workgroup takes two or three, which belong to one request or to several; four sums to a row."""
    import torch
    lengths = [600, 1, 0, 1, 1, 400, 300]
    assert sum(lengths) > 4 * torch.cuda.get_device_properties(0).multi_processor_count
    Case(lengths, d, "bf16", "layer").check_norm()
    Case(lengths, d, "f32", "layer", "layer").check_residual()
