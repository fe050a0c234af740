"""How the keys of a paged cache are shared out, on a machine without a GPU: the plain C++ that the kernels and their launches use."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name,ok", [("paged_long_check", "long keys ok")])
def test_host_checks(tmp_path, name, ok):
    exe = str(tmp_path / name)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-I",
                    os.path.join(ROOT, "paper_2412_20501_amd", "csrc"), os.path.join(ROOT, "tests", "c_abi", name + ".cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and ok in res.stdout, res.stdout + res.stderr
