"""Host logic of hs_tree_attention_mx, on the CPU, from the planner's own source: random batches under AddressSanitizer and
UndefinedBehaviorSanitizer, checked for what the kernels rely on (every row block and page in one item, at most 64 splits, none of
them without keys, records within the workspace for both formats, divisions that the device makes by a float product), and the
kinds of work items that the GPU tests' batches are cut into."""
import os
import shutil
import subprocess

import pytest

import test_gpu_attention_mx as gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    csrc, out = os.path.join(ROOT, "paper_2505_13254_amd", "csrc"), tmp_path_factory.mktemp("plan_mx")
    common = [hipcc, "-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-x", "hip", "-Xclang", "-target-feature", "-Xclang",
              "-packed-fp32-ops", "-I" + os.path.join(ROOT, "include"), "-I" + csrc, "-Wno-unused-variable",
              "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
    procs = []
    for src in (os.path.join(ROOT, "tests", "host", "plan_mx.cpp"), os.path.join(csrc, "kv_cache_mx.hip"), os.path.join(csrc, "api.cpp")):
        obj = str(out / (os.path.basename(src) + ".o"))
        procs.append((obj, subprocess.Popen(common + ["-c", src, "-o", obj], stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    for _, p in procs:
        text, _ = p.communicate(timeout=600)
        assert p.returncode == 0, text.decode()[-2000:]
    exe = str(out / "plan_mx")
    link = subprocess.run([hipcc, "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", "-o", exe] + [o for o, _ in procs],
                          stdout=subprocess.PIPE, stderr=subprocess.STDOUT, timeout=300)
    assert link.returncode == 0, link.stdout.decode()[-2000:]

    def run(*args, text=""):
        r = subprocess.run([exe] + [str(a) for a in args], input=text, capture_output=True, text=True, timeout=300,
                           env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0", LD_PRELOAD=""))
        assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
        return r.stdout

    return run


def forms(planner, batches):
    """For each (fmt, Hq, Hkv, D, rows, lens): the set of (kind, row blocks, row groups, splits, pages) of its sequences."""
    text = "".join("%d %d %d %d %d %s %s\n" % (f, Hq, Hkv, D, len(r), " ".join(map(str, r)), " ".join(map(str, l))) for f, Hq, Hkv, D, r, l in batches)
    return [{tuple(map(int, x.split())) for x in line.split(";")[:-1]} for line in planner("form", text=text).splitlines()]


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_random_batches(planner, seed):
    assert planner("fuzz", 3000, seed).startswith("ok")


@pytest.mark.parametrize("seed", [1, 2])
def test_launches_hold_what_they_attend_to(planner, seed):
    """The arguments of a call's launches name every sequence of the host arrays once, with its rows and length, and neither of the
    device arrays of offsets and lengths: a captured launch that read them would, once they have changed, work on other items than it was
    planned for and write records behind its workspace."""
    assert planner("args", 400, seed).startswith("ok")


def test_the_kinds_of_the_gpu_tests(planner):
    """Batches that are there to reach one kind of work item reach it, uncut, in both formats."""
    batches = [(f, 32, 8, 128, rows, [L] * len(rows)) for f in (0, 1) for L in (100, 230) for _, rows in gpu.KINDS]
    for (kind, rows), got in zip(gpu.KINDS * 4, forms(planner, batches)):
        assert {x[0] for x in got} == {kind} and {x[2:4] for x in got} == {(1, 1)}, (kind, rows[:1], got)


def test_the_kinds_of_calls_that_fill_the_chip(planner):
    """Among the full-chip batches of the GPU tests all four kinds occur, at each head size and in each format."""
    for f in (0, 1):
        for D in (128, 64):
            got = forms(planner, [(f, Hq, Hkv, D, rows, lens) for rows, lens, Hq, Hkv, _ in gpu.FULL])
            assert {x[0] for g in got for x in g} == {0, 1, 2, 3}


def test_the_kinds_that_are_cut(planner):
    for f in (0, 1):
        got = forms(planner, [(f, 32, 8, 128, *gpu.CUT)])[0]
        assert {2, 3} <= {x[0] for x in got if x[3] > 1}
