"""The score chains of the absorbed attention's kernel, in the assembly that the compiler makes of it (CPU: needs hipcc, no GPU).

Its matrix instructions are written out with their registers tied from step to step, and a result may be read twelve wait states after the last
step at the earliest, which that step's statement waits for.  The compiler does not know of those waits: a copy that it makes of the registers between two steps
would read them too early.  So it must make none."""
import os
import re
import subprocess

import pytest

from paper_2505_13254_amd import build as B


def _registers(text):
    found = set()
    for lo, hi in re.findall(r"\bv\[(\d+):(\d+)\]", text):
        found |= set(range(int(lo), int(hi) + 1))
    return found | {int(x) for x in re.findall(r"\bv(\d+)\b", text)}


def _broken_chains(assembly):
    """(number of chains, lines that touch a chain's registers between its steps)."""
    lines, chains, bad, mine = assembly.split("\n"), 0, [], None
    for n, line in enumerate(lines):
        code = line.split(";")[0]
        step = re.match(r"\s+v_mfma_f32_32x32x16_bf16 v\[(\d+):(\d+)\], (\S+), (\S+), (\S+)", code)
        if step:
            to = set(range(int(step.group(1)), int(step.group(2)) + 1))
            if step.group(5) == "0":
                mine, chains = to, chains + 1
            if to != mine or _registers(step.group(3) + step.group(4)) & to:
                bad.append((n, line))
            if "s_nop 11" in lines[n + 1]:
                mine = None
        elif mine is not None and _registers(code) & mine:
            bad.append((n, line))
    return chains, bad


def test_the_check_sees_a_copy():
    step = "\tv_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], %s\n"
    fine = step % "0" + step % "v[0:15]" + "\tv_add_f32 v30, v31, v32\n" + step % "v[0:15]" + "\ts_nop 11\n\tv_mov_b32 v40, v3\n"
    assert _broken_chains(fine) == (1, [])
    assert _broken_chains(fine.replace("v_add_f32 v30, v31, v32", "v_mov_b64 v[30:31], v[2:3]"))[1]
    assert _broken_chains(step % "0" + step.replace("v[0:15]", "v[50:65]") % "v[50:65]" + "\ts_nop 11\n")[1]


def test_no_copy_between_the_steps_of_a_chain(tmp_path):
    try:
        exe = B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = str(tmp_path / "a.s")
    subprocess.check_call([exe] + B.FLAGS + ["--cuda-device-only", "-S", os.path.join(B.CSRC, "latent_attn_tree.hip"), "-o", out], stderr=subprocess.DEVNULL)
    chains, bad = _broken_chains(open(out).read())
    assert chains >= 6 and not bad, bad[:3]
