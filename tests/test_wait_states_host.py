"""Wait states around inline asm, in the assembly of the kernels (no GPU needed).

gfx950 needs two wait states between a vector instruction that writes a scalar register (a
comparison's lanes) and a vector instruction that reads it.  The compiler keeps them for its own
instructions and does not look into inline asm, whose reads must bring their own."""
import os
import re
import subprocess

import pytest

from tests.test_build_flags import _builder

NEEDED = 2


def scalars(operand):
    """Scalar registers that an operand names."""
    m = re.match(r"s\[(\d+):(\d+)\]$", operand)
    if m:
        return range(int(m.group(1)), int(m.group(2)) + 1)
    m = re.match(r"s(\d+)$", operand)
    return [int(m.group(1))] if m else ["vcc"] if operand.startswith("vcc") else []


def short_waits(text):
    """(line, write, read, states between) of every vector read of a scalar register that a
    vector instruction wrote fewer than NEEDED states before, in the order of the text."""
    found, written, at = [], {}, 0
    for number, line in enumerate(text.splitlines(), 1):
        line = line.split(";")[0].strip()
        if re.match(r"[\w$.]+:$", line) and not line.startswith(".L"):
            written = {}
        if not line or line[0] in ".#" or line.endswith(":"):
            continue
        op, _, rest = line.partition(" ") if " " in line else line.partition("\t")
        args = [a.strip() for a in rest.replace("\t", " ").split(",")] if rest else []
        if op.startswith("v_"):
            late = [written[r] for a in args[1:] for r in scalars(a) if r in written and at - written[r][0] < NEEDED]
            if late:
                found.append((number, late[0][1], line, at - late[0][0]))
        for r in scalars(args[0]) if args else []:
            written.pop(r, None)
            if op.startswith("v_"):
                written[r] = (at + 1, line)
        m = re.match(r"s_nop\s+(\d+)", line)
        at += int(m.group(1)) + 1 if m else 1
    return found


def test_the_search_finds_short_waits():
    text = """kernel:
\tv_cmp_eq_u32_e64 s[4:5], 0, v1
\t;;#ASMSTART
\tv_cndmask_b32_e64 v2, v3, v2, s[4:5]
\t;;#ASMEND
\tv_cmp_eq_u32_e64 s[6:7], 0, v1
\tv_mov_b32_e32 v9, v8
\tv_cndmask_b32_e64 v2, v3, v2, s[6:7]
\tv_cmp_eq_u32_e64 s[6:7], 0, v1
\ts_nop 1
\tv_cndmask_b32_e64 v2, v3, v2, s[6:7]
\tv_cmp_eq_u32_e32 vcc, 0, v1
\ts_mov_b64 vcc, 0
\tv_cndmask_b32_e32 v2, v3, v2, vcc
"""
    assert [(n, d) for n, _, _, d in short_waits(text)] == [(4, 0), (8, 1)]


@pytest.mark.parametrize("src", ["attn_fwd.hip", "window_fwd.hip", "window_bwd.hip", "rope.hip", "sparsify.hip"])
def test_scalar_registers_are_read_late_enough(tmp_path, src):
    b = _builder()
    try:
        cc = b.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    out = str(tmp_path / "k.s")
    subprocess.check_call([cc] + b.common_flags() + b.EXTRA_FLAGS.get(src, []) +
                          ["--offload-device-only", "-S", os.path.join(b.CSRC, src), "-o", out],
                          stderr=subprocess.DEVNULL)
    text = open(out).read()
    assert re.search(r"\tv_cndmask_b32|\tv_cmp", text)
    found = short_waits(text)
    assert not found, "%d places, the first: %s" % (len(found), (found[0],))
