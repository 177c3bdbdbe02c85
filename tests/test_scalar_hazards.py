"""Scalar registers that a vector instruction writes (v_readlane, v_readfirstlane, a compare) and a memory instruction reads: five wait states stand between
them.  The compiler sees to that for its own instructions; the global -> LDS loads are assembly statements of which it knows nothing.  Read off the built
library, along every path of the kernels that have such statements."""
import os
import re

import pytest

from paper_2512_07350_amd import build
from tests import test_wait_states as ws

KERNELS = ("attention", "gemm_kernel", "adapter_down_kernel")


def scalars(text):
    out = set()
    for lo, hi, one in re.findall(r"\bs(?:\[(\d+):(\d+)\]|(\d+))(?!\w)", text):
        out |= set(range(int(lo), int(hi) + 1)) if lo else {int(one)}
    return out | ({"vcc"} if "vcc" in text else set())


class Instruction(ws.Instruction):
    def __init__(self, text):
        super().__init__(text)
        op, _, rest = text.partition(" ")
        vector = op.startswith(("v_readlane", "v_readfirstlane", "v_cmp"))
        self.writes_s = scalars(re.split(r",(?![^\[]*\])", rest)[0]) if vector else set()
        self.reads_s = scalars(rest) if op.startswith(("buffer_", "global_", "scratch_")) else set()


def too_close(code, before):
    bad = []
    for i, x in enumerate(code):
        paths, seen = [(j, 0) for j in before[i]] if x.reads_s else [], set()
        while paths:
            j, passed = paths.pop()
            if passed >= 5 or (j, passed) in seen:
                continue
            seen.add((j, passed))
            if code[j].writes_s & x.reads_s:
                bad.append((i, j, passed))
            paths += [(k, passed + code[j].states) for k in before[j]]
    return bad


def test_scalars_reach_memory_instructions(tmp_path, monkeypatch):
    if not os.path.exists(ws.OBJDUMP):
        pytest.skip("no llvm-objdump beside hipcc")
    monkeypatch.setattr(ws, "Instruction", Instruction)
    monkeypatch.setattr(ws, "KERNELS", KERNELS)
    count = 0
    for name, code, before in ws.kernels(build.LIB, tmp_path):
        count += 1
        assert not too_close(code, before), name
    assert count >= 60


def test_the_check_sees_what_stands_too_close():
    line = lambda *texts: ([Instruction(t) for t in texts], [[j] if j >= 0 else [] for j in range(-1, len(texts) - 1)])
    load = "buffer_load_dwordx4 v0, s[4:7], s8 offen lds"
    assert too_close(*line("v_readlane_b32 s5, v1, s2", "s_nop 3", load)) == [(2, 0, 4)]
    assert not too_close(*line("v_readlane_b32 s5, v1, s2", "s_nop 4", load))
    assert too_close(*line("v_readfirstlane_b32 s8, v1", load)) == [(1, 0, 0)]
    assert not too_close(*line("v_readlane_b32 s9, v1, s2", load))
