"""The learner's calls driven by a plain C program (needs an MI355X)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
PACKAGE = os.path.join(os.path.dirname(HERE), "paper_2602_01665_amd")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    binary = str(tmp_path_factory.mktemp("c") / "abi_c_learner")
    subprocess.run(["gcc", "-std=c11", "-O1", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__",
                    "-I", os.path.join(os.path.dirname(HERE), "include"), "-isystem", os.path.join(ROCM, "include"),
                    os.path.join(HERE, "abi_c_learner.c"), "-o", binary, "-L", PACKAGE, "-ltabx",
                    "-L", os.path.join(ROCM, "lib"), "-lamdhip64", "-lm", "-Wl,-rpath," + PACKAGE,
                    "-Wl,-rpath," + os.path.join(ROCM, "lib")], check=True)
    return binary


def test_it_compiles_and_links(program):
    assert os.path.exists(program)


@pytest.mark.gpu
def test_it_agrees_with_the_formulas(program):
    print("[gpu]", program, flush=True)
    r = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "abi_c_learner: PASS" in r.stdout, r.stdout + r.stderr
