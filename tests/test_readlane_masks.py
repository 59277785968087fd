"""v_readlane takes a value from a lane whether that lane is active or not, but what a register holds there is only what the lane
computed while it was: the compiler may load, copy or reload a value under a mask that has left the lane out.  So the lanes of a
wavefront that read each other's registers do it while all of them are active.  In the code the compiler makes of gemm_f32.hip
today (no GPU: read from the library's own assembly), along every path: no v_readlane where the execution mask may be narrower
than at the kernel's start."""
import os
import re
import subprocess

import pytest

from paper_2006_16668_amd import build
from test_attention_wait_states import _kernels


def _scalars(operand):
    m = re.fullmatch(r"s(?:(\d+)|\[(\d+):(\d+)\])", operand)
    return frozenset() if not m else frozenset(range(int(m.group(1) or m.group(2)), int(m.group(1) or m.group(3)) + 1))


def _step(ins, whole, saved):
    """State behind an instruction: whether all lanes are active, and the scalar registers that hold a mask of all lanes."""
    ops = re.split(r",\s*", ins.text.partition(" ")[2])
    known = lambda o: o == "-1" or o in saved or (o == "exec" and whole)
    was, dest = whole, ops[0]
    gone = _scalars(dest)
    kept = frozenset(s for s in saved if not _scalars(s) & gone)
    if ins.name in ("s_and_saveexec_b64", "s_or_saveexec_b64"):
        whole = was and known(ops[1]) if ins.name.startswith("s_and") else was or known(ops[1])
        return whole, kept | {dest} if was else kept
    if dest == "exec":
        if ins.name == "s_mov_b64":
            return known(ops[1]), kept
        return ins.name == "s_or_b64" and any(known(o) for o in ops[1:]), kept
    if ins.name == "s_mov_b64" and known(ops[1]):
        return whole, kept | {dest}
    return whole and not ins.name.startswith("v_cmpx"), kept


def narrowed(code):
    """(v_readlane instructions, those that a narrower mask may reach)"""
    state, todo = {0: (True, frozenset())}, [0]
    while todo:
        i = todo.pop()
        whole, saved = _step(code[i], *state[i])
        for n in code[i].next:
            met = (whole, saved) if n not in state else (whole and state[n][0], saved & state[n][1])
            if state.get(n) != met:
                state[n] = met
                todo.append(n)
    # (scalar values that the compiler keeps in lanes of a register: v_writelane reaches a lane that is not active, too)
    kept = {re.split(r",\s*", c.text.partition(" ")[2])[0] for c in code if c.name.startswith("v_writelane")}
    reads = [i for i in state if code[i].name.startswith("v_readlane") and re.split(r",\s*", code[i].text)[1] not in kept]
    return len(reads), [code[i].text for i in reads if not state[i][0]]


SAMPLE = """_Zk:
	v_readlane_b32 s8, v1, 4
	s_and_saveexec_b64 s[0:1], vcc
	s_cbranch_execz .LBB0_2
	{inside}
	{lost}
.LBB0_2:
	s_or_b64 exec, exec, s[0:1]
	v_readlane_b32 s9, v1, 5
	s_endpgm
.Lfunc_end0:
"""


@pytest.mark.parametrize("inside,lost,faults", [
    ("s_nop 0", "s_nop 0", 0), ("v_readlane_b32 s9, v1, 5", "s_nop 0", 1), ("s_nop 0", "s_mov_b32 s1, 0", 1), ("s_nop 0", "s_mov_b32 s2, 0", 0),
    ("s_and_saveexec_b64 s[4:5], vcc", "s_or_b64 exec, exec, s[4:5]", 0), ("s_and_saveexec_b64 s[0:1], vcc", "s_nop 0", 1)])
def test_the_check_finds_what_it_looks_for(inside, lost, faults):
    code, = _kernels(SAMPLE.format(inside=inside, lost=lost)).values()
    reads, wrong = narrowed(code)
    assert reads == 2 + inside.startswith("v_readlane") and len(wrong) == faults, wrong


def test_registers_of_other_lanes_are_read_by_whole_wavefronts(tmp_path):
    out, src = str(tmp_path / "gemm_f32.s"), "gemm_f32.hip"
    subprocess.run([build._hipcc(), *build.FLAGS, *build.EXTRA_FLAGS.get(src, []), "-S", "--cuda-device-only",
                    os.path.join(build.CSRC, src), "-o", out], check=True, capture_output=True)
    found = {k: narrowed(code) for k, code in _kernels(open(out).read()).items() if code}
    reading = {k: v for k, v in found.items() if v[0]}
    assert len(reading) == 10                            # a vocabulary's logits, their statistics and gradient, in every form
    for name, (reads, wrong) in reading.items():
        assert not wrong, (name, reads, len(wrong), wrong[:3])
