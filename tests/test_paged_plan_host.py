"""How the keys of a paged cache are shared out, on a machine without a GPU: the plain C++ that the kernels and their launches use."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name,ok", [("paged_long_check", "long keys ok"), ("paged_launch_check", "launches ok")])
def test_host_checks(tmp_path, name, ok):
    exe = str(tmp_path / name)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-I",
                    os.path.join(ROOT, "paper_2412_20501_amd", "csrc"), os.path.join(ROOT, "tests", "c_abi", name + ".cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and ok in res.stdout, res.stdout + res.stderr


def test_the_plan_is_rounded_as_written(tmp_path):
    """The kernels of a call make the plan each for themselves and have to agree on it: no operations are fused, with the compiler and the default that the kernels are built with."""
    clang = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++")
    source, out = tmp_path / "plan.cpp", tmp_path / "plan.s"
    source.write_text('#include "paged_plan.h"\n'
                      "int part(int64_t work, int64_t tiles, int longest, const tr::Share& share) { return tr::part_keys(work, tiles, longest, share); }\n"
                      "float other(float a, float b, float c) { return a * b + c; }\n")
    subprocess.run([clang, "-O3", "-std=c++17", "-mfma", "-ffp-contract=fast-honor-pragmas", "-I", os.path.join(ROOT, "paper_2412_20501_amd", "csrc"), "-S", str(source), "-o", str(out)], check=True)
    text = out.read_text()
    assert text.count("vfmadd") == 1, "one in the function that may"
