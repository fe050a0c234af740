"""tr_cache_weigh on a machine without a GPU: how much work a call may ask for, and which kernels it takes."""
import os
import subprocess

import pytest

from test_evict_host import ROOT, SHAPE, Call, tr  # noqa: F401  (tr: a fixture)


@pytest.mark.parametrize("n_seqs,Hkv,stretches", [
    (14322, 3, 49981),      # 2^31 - 2 stretches of 64 keys: rounded up to eighths, their number would pass 2^31 - 1
    (1 << 16, 8, 1 << 12),  # 2^31
])
def test_more_keys_than_can_be_shared_out(tr, n_seqs, Hkv, stretches):  # noqa: F811
    assert n_seqs * Hkv * stretches >= 2 ** 31 - 8
    c = Call(tr, page=64)
    wide = lambda name, D: c.like(name, H=Hkv, stride_b=Hkv * 64 * D)   # noqa: E731
    q = c.like("q", H=Hkv, stride_b=Hkv * 7 * 128)
    st, msg = c("weigh", q=q, lse=c.like("lse", H=Hkv, stride_b=Hkv * 7), kp=wide("kp", 128), ks=wide("ks", 1), w=wide("w", 1),
                seqs=c.like("seqs", n_seqs=n_seqs, max_pages=stretches, table_stride=stretches))
    assert st == SHAPE and "too many keys" in msg, (st, msg)


def test_forms(tmp_path):
    exe = str(tmp_path / "weigh_form_check")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-I",
                    os.path.join(ROOT, "paper_2412_20501_amd", "csrc"), os.path.join(ROOT, "tests", "c_abi", "weigh_form_check.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "weigh forms ok" in res.stdout, res.stdout + res.stderr
