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


def _in_loops(assembly, kernel, wanted):
    """Lines with `wanted` that lie on a cycle of the kernel's control flow: they are reached again from themselves."""
    lines = assembly.split("\n")
    start = next(n for n, line in enumerate(lines) if re.match(r"^\S*%s\S*:" % kernel, line))
    end = next(n for n in range(start, len(lines)) if ".Lfunc_end" in lines[n])
    code = [line.split(";")[0].strip() for line in lines[start:end]]
    label = {c[:-1]: n for n, c in enumerate(code) if c.endswith(":")}

    def after(n):
        jump = re.match(r"(s_c?branch\w*)\s+(\S+)", code[n])
        to = [label[jump.group(2)]] if jump else []
        return to + ([n + 1] if n + 1 < len(code) and not code[n].startswith(("s_endpgm", "s_branch")) else [])

    bad = []
    for n in [n for n, c in enumerate(code) if wanted in c]:
        seen, todo = set(), after(n)
        while todo:
            x = todo.pop()
            if x not in seen:
                seen.add(x)
                todo += after(x)
        if n in seen:
            bad.append(code[n])
    return bad


def test_the_check_sees_a_loop():
    text = "k_x:\n\tscratch_load_dword v1, off, off\n.LBB0_1:\n\tv_mov_b32 v0, v1\n\ts_cbranch_scc1 .LBB0_1\n\ts_endpgm\n.Lfunc_end0:\n"
    assert not _in_loops(text, "k_x", "scratch_")
    assert _in_loops(text.replace("v_mov_b32 v0, v1", "scratch_store_dword off, v1, off"), "k_x", "scratch_")


def test_no_register_is_kept_in_memory_inside_a_loop(tmp_path):
    """A load from there would wait for every tile on its way."""
    try:
        exe = B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = str(tmp_path / "a.s")
    subprocess.check_call([exe] + B.FLAGS + ["--cuda-device-only", "-S", os.path.join(B.CSRC, "latent_attn_tree.hip"), "-o", out], stderr=subprocess.DEVNULL)
    text = open(out).read()
    for most in (1, 2, 4):
        assert not _in_loops(text, "k_lat_treeILi%dE" % most, "scratch_"), most
