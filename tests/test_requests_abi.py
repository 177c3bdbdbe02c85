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
