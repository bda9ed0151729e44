"""What the context's calls for beams answer, on the CPU, where the operators' kernels are not built in and where no launch
holds the work: each says which of the two it is, and nothing has changed."""
import os
import subprocess

import pytest

from paper_2609_26100_amd import tss as abi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/llvm/bin/clang++"


@pytest.fixture(scope="module")
def answers(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("ROCm clang++ not installed")
    at = tmp_path_factory.mktemp("reorder")

    def build(name, *flags):
        exe = str(at / name)
        cmd = [CLANG, "-std=c++17", "-O1", "-x", "c++", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
               "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2609_26100_amd", "csrc"),
               "-Wno-everything", *flags, os.path.join(ROOT, "tests", "host_reorder", "reorder.cpp"),
               os.path.join(ROOT, "tests", "host_asan", "stub_launchers.cpp"), "-L/opt/rocm/lib", "-lamdhip64",
               "-Wl,-rpath,/opt/rocm/lib", "-o", exe]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]

        def run(*args):
            r = subprocess.run([exe, *args], capture_output=True, text=True, timeout=60)
            assert r.returncode == 0, r.stderr
            reorder, lengths, beams = r.stdout.splitlines()
            return reorder.split(" ", 1), [int(x) for x in lengths.split()], beams.split(" ", 1)
        return run

    return build("without"), build("with", "-DWITH_KERNELS")


def test_without_the_kernels(answers):
    for status, text in answers[0]()[::2]:
        assert int(status) == abi.TSS_EINVAL and text == "built without the operators' kernels"
    assert answers[0]()[1] == [40, 50, 60]


def test_work_that_no_launch_holds(answers):
    reorder, lengths, beams = answers[1]("refuse")
    assert int(reorder[0]) == abi.TSS_EINVAL and reorder[1] == "too many pages for one launch"
    assert lengths == [40, 50, 60]
    assert int(beams[0]) == abi.TSS_EINVAL and beams[1] == "vocabulary too large"


def test_work_that_one_does(answers):
    reorder, lengths, _ = answers[1]("fit")
    assert int(reorder[0]) == 0 and lengths == [50, 50, 40]
