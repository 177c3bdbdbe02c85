"""Wait states and M0 around the statements of test_wait_states, in the kernels of the calls over several requests too, and that every family of them is
among the kernels looked at."""
import collections
import os

import pytest

from paper_2512_07350_amd import build
from tests import test_wait_states as ws

# kernels of each family in the library: the tilings of lp_linear and lp_qkv_projection (at head_dim 64 and 128), as they are, with adapters, and in one launch;
# the tiles of the down products; attention's forms
FAMILIES = {"linear": 15, "qkv": 18, "linear, adapters": 15, "qkv, adapters": 18, "linear, one launch": 1, "qkv, one launch": 1, "down": 3, "attention": 8}


def family(name):
    if "adapter_down_kernel" in name:
        return "down"
    if "attention_kernel" in name:
        return "attention"
    return ("qkv" if "gemm_kernelILb1" in name else "linear") + (", one launch" if "FewArgs" in name else ", adapters" if "AdaptedArgs" in name else "")


def test_every_family_of_kernels_keeps_its_wait_states(tmp_path, monkeypatch):
    if not os.path.exists(ws.OBJDUMP):
        pytest.skip("no llvm-objdump beside hipcc")
    monkeypatch.setattr(ws, "KERNELS", ("attention_kernel", "gemm_kernel", "adapter_down_kernel"))
    seen = collections.Counter()
    for name, code, before in ws.kernels(build.LIB, tmp_path):
        assert any(x.product for x in code), name
        seen[family(name)] += 1
        bad = ws.too_close(code, before)
        assert not bad, (name, [(code[j].op, code[i].op, passed) for i, j, passed in bad[:4]])
        assert not ws.m0_lost(code, before), name
    assert seen == FAMILIES
