"""Refusals of the calls over several requests -- no GPU needed: arguments are checked before anything touches a device."""
import ctypes as C

import pytest

from paper_2512_07350_amd import binding as lp

INF, NAN = float("inf"), float("nan")


def _norm(req=None, x=1 << 20, y=1 << 21, x_type=lp.LP_BF16, d=64, sx=64, sy=64, norm="rms", mod=None):
    req = lp.make_requests([0, 3]) if req is None else req
    norm = lp.make_norm(lp.LP_NORM_RMS, 1e-6) if norm == "rms" else norm
    return lp._lib().lp_norm_modulate(x, x_type, y, lp._ref(req) if req != "null" else None, d, sx, sy, lp._ref(norm), lp._ref(mod), None)


def _residual(h=1 << 20, u=1 << 21, o=1 << 22, y=1 << 23, h_type=lp.LP_F32, d=64, sh=64, su=64, so=64, sy=64, post=None, norm="rms", mod=None,
              starts=(0, 3)):
    norm = lp.make_norm(lp.LP_NORM_RMS, 1e-6) if norm == "rms" else norm
    return lp._lib().lp_gated_residual_norm(h, h_type, u, o, y, lp._ref(lp.make_requests(starts)), d, sh, su, so, sy, lp._ref(post),
                                            lp._ref(norm), lp._ref(mod), None)


def test_requests_are_checked():
    bad, inv = lp.make_requests, lp.LP_ERR_INVALID_ARG
    assert _norm("null") == inv
    assert _norm(bad([1, 3])) == inv and _norm(bad([0, 3, 2])) == inv and _norm(bad([0, -1])) == inv
    assert _norm(lp.lp_requests(-1, None)) == inv and _norm(lp.lp_requests(2, None)) == inv
    assert _norm(bad(range(66))) == lp.LP_ERR_LIMIT
    assert _norm(bad([0, 2 ** 31 - 1])) == lp.LP_ERR_UNSUPPORTED
    # nothing to do: no pointer is looked at
    for r in (lp.make_requests([]), lp.make_requests([0]), lp.make_requests([0, 0, 0]), lp.lp_requests(0, None)):
        assert _norm(r, None, None) == lp.LP_OK
    assert _residual(None, None, None, None, starts=(0, 0)) == lp.LP_OK


def test_norm_refusals():
    inv = lp.LP_ERR_INVALID_ARG
    assert _norm(x=None) == inv and _norm(y=None) == inv and _norm(norm=None) == inv
    assert _norm(x_type=2) == inv and _norm(d=0) == inv and _norm(sx=63) == inv and _norm(sy=0) == inv
    assert _norm(d=16385, sx=16385, sy=16385) == lp.LP_ERR_UNSUPPORTED
    assert _norm(x=(1 << 20) + 1) == inv and _norm(x=(1 << 20) + 2, x_type=lp.LP_F32) == inv and _norm(y=(1 << 20) + 1) == inv
    assert _norm(y=1 << 20, x_type=lp.LP_F32) == inv and _norm(y=1 << 20, sy=72) == inv        # in place: one type, one stride
    for kind, eps in ((2, 1e-6), (-1, 1e-6), (0, -1e-6), (0, NAN), (1, INF)):
        assert _norm(norm=lp.make_norm(kind, eps)) == inv
    assert _norm(norm=lp.make_norm(0, 0.0, weight=2)) == inv
    assert _norm(mod=lp.make_modulation(scale=64, stride=63)) == inv and _norm(mod=lp.make_modulation(shift=66, stride=64)) == inv


def test_residual_refusals():
    inv = lp.LP_ERR_INVALID_ARG
    for name in ("h", "u", "o", "y"):
        assert _residual(**{name: None}) == inv
    assert _residual(norm=None) == inv                                                          # y without a norm
    assert _residual(o=1 << 21) == inv and _residual(y=1 << 20) == inv and _residual(y=1 << 21) == inv and _residual(y=1 << 22) == inv
    assert _residual(o=1 << 20, so=128) == inv                                                  # in place: one stride
    for name in ("sh", "su", "so", "sy"):
        assert _residual(**{name: 63}) == inv
    assert _residual(h=(1 << 20) + 2) == inv and _residual(u=(1 << 21) + 1) == inv
    assert _residual(post=lp.make_norm(5, 1e-6)) == inv
    assert _residual(mod=lp.make_modulation(gate=64, stride=1)) == inv


def test_modulation_of_tensors_takes_their_stride():
    import torch
    t = torch.zeros(3, 6, 32)
    m = lp.make_modulation(gate=t[:, 2], scale=t[:, 0], shift=t[:, 1])
    assert m.stride == 192 and m.scale == t.data_ptr() and m.gate == t.data_ptr() + 4 * 64
    assert lp.make_modulation(scale=t[0, 0]).stride == 0 and lp.make_modulation().stride == 0
    with pytest.raises(ValueError):
        lp.make_modulation(scale=t[:, 0], shift=t[0, 1])
    with pytest.raises(ValueError):
        lp.make_modulation(scale=t[:, 0].t())


def _adapters(*specs):
    """(down, up, rank, scale) as given, addresses unchecked."""
    return (lp.lp_adapter * max(len(specs), 1))(*[lp.lp_adapter(*s) for s in specs])


GOOD = (1 << 24, 1 << 25, 16, 1.0)


def _linear(x=1 << 20, w=1 << 21, bias=None, y=1 << 22, starts=(0, 3), d_in=128, d_out=256, adapters=None, ws=1 << 26, size=1 << 20):
    adapters = _adapters(GOOD) if adapters is None else adapters
    return lp._lib().lp_linear_adapters(x, w, bias, y, lp._ref(lp.make_requests(starts)), d_in, d_out, None if adapters == "null" else adapters, ws, size, None)


def test_linear_adapters_refusals():
    inv, uns = lp.LP_ERR_INVALID_ARG, lp.LP_ERR_UNSUPPORTED
    for name in ("x", "w", "y"):
        assert _linear(**{name: None}) == inv and _linear(**{name: (1 << 22) + 8}) == inv
    assert _linear(bias=4) == inv and _linear(y=1 << 20) == inv and _linear(y=1 << 21) == inv
    assert _linear(d_in=100) == uns and _linear(d_out=192) == uns and _linear(d_in=0) == inv
    assert _linear(adapters="null") == inv and _linear(starts=(0, 3, 2)) == inv and _linear(starts=range(66)) == lp.LP_ERR_LIMIT
    for bad, status in (((1 << 24, 1 << 25, -8, 1.0), inv), ((1 << 24, 1 << 25, 4, 1.0), uns), ((1 << 24, 1 << 25, 264, 1.0), uns),
                        ((None, 1 << 25, 8, 1.0), inv), ((1 << 24, None, 8, 1.0), inv), (((1 << 24) + 8, 1 << 25, 8, 1.0), inv),
                        ((1 << 24, (1 << 25) + 2, 8, 1.0), inv), ((1 << 24, 1 << 25, 8, NAN), inv), ((1 << 24, 1 << 25, 8, INF), inv)):
        assert _linear(adapters=_adapters(bad)) == status
        assert _linear(starts=(0, 3, 3), adapters=_adapters(GOOD, bad)) == status               # of a request without rows too
    assert _linear(ws=None) == inv and _linear(ws=(1 << 26) + 8) == inv and _linear(size=3200 + 3 * 128 - 1) == inv
    assert _linear(ws=1 << 20) == inv and _linear(ws=1 << 21) == inv and _linear(ws=1 << 22) == inv
    # nothing to do
    assert _linear(None, None, None, None, (0, 0), ws=None, size=0) == lp.LP_OK and _linear(starts=(), adapters="null") == lp.LP_OK


def test_workspace_size():
    size = lp._lib().lp_adapter_workspace_size
    assert size(10, 8, 1) == size(10, 32, 1) == 3200 + 10 * 128 and size(10, 33, 1) == 3200 + 10 * 256
    assert size(10, 256, 3) == 3200 + 10 * 3 * 8 * 128
    assert size(0, 8, 1) == 0 and size(10, 0, 3) == 0
    assert size(-1, 8, 1) == size(1, -8, 1) == size(1, 8, 2) == lp.LP_ERR_INVALID_ARG
    assert size(1, 264, 1) == size(2 ** 31 - 1, 8, 1) == lp.LP_ERR_UNSUPPORTED
    with pytest.raises(lp.LPError):
        lp.lp_adapter_workspace_size(1, 8, 2)


def _qkv(x=1 << 20, w=1 << 21, gq=1 << 22, gk=1 << 23, q=1 << 27, k=1 << 28, v=1 << 29, eps=1e-6, starts=(0, 4, 4, 10), heads=2, hd=64, ropes=None,
         adapters=None, ws=1 << 26, size=1 << 20):
    if ropes is None:
        ropes = [lp.make_rope((1, 2, 2), head_dim=64), lp.make_rope((9, 9, 9), split=(0, 0, 64), base=5.0, head_dim=64), lp.make_rope((1, 1, 6), head_dim=64)]
    ropes = (lp.lp_rope * 3)(*ropes) if ropes != "null" else None
    return lp._lib().lp_qkv_projection_adapters(x, w, None, gq, gk, eps, ropes, q, k, v, lp._ref(lp.make_requests(starts)), heads, hd,
                                                _adapters(GOOD, GOOD, GOOD) if adapters is None else adapters, ws, size, None)


def test_qkv_adapters_refusals():
    inv, uns = lp.LP_ERR_INVALID_ARG, lp.LP_ERR_UNSUPPORTED
    for name in ("x", "w", "gq", "gk", "q", "k", "v"):
        assert _qkv(**{name: None}) == inv and _qkv(**{name: (1 << 22) + 8}) == inv
    assert _qkv(ropes="null") == inv and _qkv(heads=0) == inv and _qkv(hd=96) == uns and _qkv(heads=3) == uns and _qkv(eps=-1.0) == inv
    rope = lambda *a, **kw: lp.make_rope(*a, head_dim=64, **kw)
    fine = [rope((1, 2, 2)), rope((9, 9, 9)), rope((1, 1, 6))]
    for i, bad in ((0, rope((1, 2, 3))), (2, rope((6, 1, 1), base=5.0)), (2, rope((6, 1, 1), split=(20, 24, 20))), (2, rope((6, 1, 1), split=(23, 21, 20))),
                   (0, rope((-2, -2, 1))), (0, rope((1, 2, 2), base=-1.0))):
        assert _qkv(ropes=fine[:i] + [bad] + fine[i + 1:]) == inv
    assert _qkv(q=1 << 28) == inv and _qkv(v=1 << 20) == inv
    assert _qkv(ws=None) == inv and _qkv(size=3200 + 10 * 3 * 128 - 1) == inv and _qkv(ws=1 << 27) == inv
    assert _qkv(starts=(0, 0, 0, 0)) == lp.LP_OK


def test_tables_shorter_than_the_requests_are_refused():
    req = lp.make_requests([0, 2, 4, 6])
    with pytest.raises(ValueError):
        lp.lp_linear_adapters(1 << 20, 1 << 21, None, 1 << 22, req, 64, 128, lp.make_adapters([None]))
    with pytest.raises(ValueError):
        lp.lp_qkv_projection_adapters(1, 2, None, 3, 4, 1e-6, [lp.make_rope((1, 1, 2))], 5, 6, 7, req, 1, 128, lp.make_adapters([None] * 3))


@pytest.mark.parametrize("grid,split", [((1, 1, 4), (2 ** 31 - 2, 2 ** 31 - 2, 68)),                 # 2^32 + 64 features
                                        ((968973220, 49477, 384773), (64, 0, 0))])                   # 2^64 + 4 cells
def test_rotations_that_fit_only_modulo_a_power_of_two(grid, split):
    rope = lp.make_rope(grid, split=split, head_dim=64)
    fine = lp.make_rope((1, 1, 6), split=split, head_dim=64)
    assert _qkv(ropes=[rope, rope, fine]) == lp.LP_ERR_INVALID_ARG
    assert lp._lib().lp_qkv_projection(1 << 20, 1 << 21, None, 1 << 22, 1 << 23, 1e-6, C.byref(rope), 1 << 27, 1 << 28, 1 << 29, 4, 2, 64,
                                       None) == lp.LP_ERR_INVALID_ARG
    assert lp._lib().lp_qk_norm_rope(1 << 20, 1 << 21, 1e-6, C.byref(rope), 4, 2, 64, 128, 64, None) == lp.LP_ERR_INVALID_ARG


def _taken(call, *args, **kw):
    """The binding hands the call on: it is the library that refuses its missing x."""
    with pytest.raises(lp.LPError) as e:
        call(*args, **kw)
    assert e.value.status == lp.LP_ERR_INVALID_ARG


def _refused(call, *args, **kw):
    with pytest.raises(ValueError):
        call(*args, **kw)


def test_adapters_of_another_projection_are_refused():
    import torch
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    req, two = lp.make_requests([0, 2]), lp.make_requests([0, 2, 4])
    linear = lambda table, r=req: lp.lp_linear_adapters(None, 1 << 21, None, 1 << 22, r, 128, 256, table, 1 << 26, 1 << 20)
    ropes = [lp.make_rope((1, 1, 2), head_dim=64)] * 2
    qkv = lambda table, r=req: lp.lp_qkv_projection_adapters(None, 2 << 20, None, 3 << 20, 4 << 20, 1e-6, ropes, 5 << 20, 6 << 20, 7 << 20, r, 2, 64, table,
                                                             1 << 26, 1 << 20)
    for_linear, for_qkv = (z(16, 128), z(256, 16), 1.0), (z(48, 128), z(384, 16), 1.0)
    none = (z(0, 128), z(256, 0), 1.0)                     # of rank 0
    _taken(linear, lp.make_adapters([for_linear]))
    _taken(linear, lp.make_adapters([none, for_linear]), two)
    _taken(linear, lp.make_adapters([for_linear, for_qkv]))                                         # the second belongs to no request
    _taken(linear, lp.make_adapters([(z(16, 128, dtype=torch.int16), z(256, 16, dtype=torch.int16), 1.0)]))
    _taken(qkv, lp.make_adapters([None, for_qkv]), two)
    _refused(qkv, lp.make_adapters([for_linear]))
    _refused(qkv, lp.make_adapters([for_qkv, for_linear]), two)
    for down, up in (((48, 128), (256, 16)), ((16, 64), (256, 16)), ((16, 192), (256, 16)), ((16, 128), (128, 16)), ((16, 128), (384, 16))):
        _refused(linear, lp.make_adapters([(z(*down), z(*up), 1.0)]))
    # the table's entry is another by now: nothing is known of its sizes
    table = lp.make_adapters([for_qkv])
    table[0] = lp.lp_adapter(1 << 24, 1 << 25, 16, 1.0)
    _taken(linear, table)
    for bad in ((z(16, 128, dtype=torch.float32), z(256, 16)), (z(16, 128), z(256, 16, dtype=torch.float16)), (z(16, 128), z(256, 0)), (z(20, 128), z(256, 16))):
        _refused(lp.make_adapters, [(*bad, 1.0)])
    _refused(linear, lp.make_adapters([]))
    _refused(lp.lp_qkv_projection_adapters, None, 2, None, 3, 4, 1e-6, [], 5, 6, 7, req, 2, 64, lp.make_adapters([None]))


def test_vectors_that_do_not_hold_the_requests_are_refused():
    import torch
    z = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)
    req, pre = lp.make_requests([0, 2, 3, 3]), lp.make_norm(lp.LP_NORM_RMS, 1e-6)
    norm = lambda mod, n=pre: lp.lp_norm_modulate(None, lp.LP_BF16, 1 << 20, req, 32, n, mod)
    residual = lambda mod, n=pre, post=None: lp.lp_gated_residual_norm(None, lp.LP_F32, 1 << 20, 1 << 21, None if n is None else 1 << 22, req, 32, post, n, mod)
    m = lp.make_modulation
    all_of = z(3, 6, 32)
    for call in (norm, residual):
        _taken(call, m(scale=all_of[:, 1], shift=all_of[:, 5]))
        _taken(call, m(scale=z(32)))                        # one for all
        _taken(call, m(scale=z(1, 32).expand(2, 32)))
        _taken(call, m(scale=z(96), stride=32))             # the caller's own stride
        _taken(call, m(scale=z(3, 4, 8)))
        _taken(call, m(scale=all_of.data_ptr(), stride=32))
        _taken(call, m())
        for bad in (m(scale=all_of[:2, 1]), m(shift=z(1, 32)), m(shift=z(3, 31)), m(scale=z(31)), m(scale=z(95), stride=32), m(shift=z(3, 32), stride=64)):
            _refused(call, bad)
        _refused(call, None, lp.make_norm(lp.LP_NORM_RMS, 1e-6, weight=z(31)))
        _refused(call, None, lp.make_norm(lp.LP_NORM_LAYER, 1e-6, bias=z(8)))
        _taken(call, None, lp.make_norm(lp.LP_NORM_LAYER, 1e-6, z(32), z(40)))
    _refused(residual, None, pre, lp.make_norm(lp.LP_NORM_RMS, 1e-6, weight=z(31)))
    # vectors that a call does not use
    _taken(norm, m(gate=z(1, 32)))
    _refused(residual, m(gate=z(1, 32)))
    some = z(3, 64)
    _taken(residual, m(gate=some[:, :32], scale=some[:2, :32]), None)
    _refused(residual, m(gate=all_of[:2, 0]), None)
    _refused(m, scale=z(3, 32, dtype=torch.bfloat16))
    _refused(m, gate=1 << 20)
    _refused(lp.make_norm, lp.LP_NORM_RMS, 1e-6, z(32, dtype=torch.float64))
    _refused(lp.make_norm, lp.LP_NORM_RMS, 1e-6, z(64)[::2])


def test_a_width_past_32_bits_is_the_librarys_to_refuse():
    _taken(lp.lp_norm_modulate, None, lp.LP_BF16, 1 << 20, lp.make_requests([0, 2]), 1 << 32, lp.make_norm(lp.LP_NORM_RMS, 1e-6), lp.make_modulation())


def test_vectors_that_a_call_does_not_use_are_not_looked_at():
    none = dict(req=lp.make_requests([0, 0]), x=None, y=None)                       # accepted: no rows, nothing is launched
    m = lp.make_modulation
    for vectors in (m(gate=64, stride=1), m(gate=66, stride=64), m(gate=66, scale=64, stride=64)):
        assert _norm(mod=vectors, **none) == lp.LP_OK
    last = dict(h=None, u=None, o=None, y=None, norm=None, starts=(0, 0))
    for vectors in (m(scale=64, stride=1), m(scale=66, shift=65, stride=64), m(gate=64, scale=66, stride=64)):
        assert _residual(mod=vectors, **last) == lp.LP_OK
    # those that it uses are
    assert _norm(mod=m(shift=66, stride=64), **none) == lp.LP_ERR_INVALID_ARG and _norm(mod=m(scale=64, stride=1), **none) == lp.LP_ERR_INVALID_ARG
    assert _residual(mod=m(gate=66, stride=64), **last) == lp.LP_ERR_INVALID_ARG and _residual(mod=m(gate=64, stride=1), **last) == lp.LP_ERR_INVALID_ARG
    assert _residual(mod=m(scale=66, stride=64), **dict(last, norm="rms")) == lp.LP_ERR_INVALID_ARG


def test_a_norm_takes_anything_that_has_an_address():
    class Buffer:
        def data_ptr(self):
            return 1 << 20
    norm = lp.make_norm(lp.LP_NORM_LAYER, 1e-6, Buffer(), 1 << 21)
    assert (norm.weight, norm.bias) == (1 << 20, 1 << 21)
    _taken(lp.lp_norm_modulate, None, lp.LP_BF16, 1 << 20, lp.make_requests([0, 2]), 64, norm)
