"""The flags of odd values in the expanded attention's kernel, in the assembly that the compiler makes of it (CPU: needs hipcc, no GPU).

Some threads clear the flags at the kernel's start, others set them when they look at the first masked tile: on every way from the one to the other the waves have
to meet.  A flag that is cleared after it was set is lost, and a value that was no number has then become zero."""
import os
import re
import subprocess

import pytest

from paper_2505_13254_amd import build as B


def _reaches(assembly, kernel, wanted, barrier="s_barrier"):
    """Lines with `wanted` that the kernel's start reaches without passing a barrier."""
    lines = assembly.split("\n")
    start = next(n for n, line in enumerate(lines) if re.match(r"^\S*%s\S*:" % kernel, line))
    end = next(n for n in range(start, len(lines)) if ".Lfunc_end" in lines[n])
    code = [line.split(";")[0].strip() for line in lines]
    label = {code[n][:-1]: n for n in range(start, end) if code[n].endswith(":")}
    seen, todo, found = set(), [start + 1], []
    while todo:
        n = todo.pop()
        while n < end and n not in seen:
            seen.add(n)
            if wanted in code[n]:
                found.append((n, lines[n]))
            if code[n].startswith((barrier, "s_endpgm")):
                break
            jump = re.match(r"(s_c?branch\w*)\s+(\S+)", code[n])
            if jump:
                todo.append(label[jump.group(2)])
                if jump.group(1) == "s_branch":
                    break
            assert not code[n].startswith(("s_setpc", "s_swappc")), lines[n]
            n += 1
    return found


def test_the_check_sees_a_way_around():
    text = "k_x:\n\ts_cbranch_scc1 .LBB0_2\n\ts_barrier\n\ts_branch .LBB0_2\n.LBB0_2:\n\tds_or_b32 v0, v1\n\ts_endpgm\n.Lfunc_end0:\n"
    assert _reaches(text, "k_x", "ds_or_b32")
    assert not _reaches(text.replace("\tds_or", "\ts_barrier\n\tds_or"), "k_x", "ds_or_b32")


def test_the_waves_meet_between_clearing_and_setting(tmp_path):
    try:
        exe = B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = str(tmp_path / "a.s")
    subprocess.check_call([exe] + B.FLAGS + ["--cuda-device-only", "-S", os.path.join(B.CSRC, "latent_attn_prompt.hip"), "-o", out], stderr=subprocess.DEVNULL)
    text = open(out).read()
    assert "ds_or_b32" in text
    found = _reaches(text, "k_lat_promptE", "ds_or_b32")
    assert not found, found[:3]
