"""Trees of drafted tokens and evictions on a machine without a GPU: what the calls refuse before anything is launched, and which bits of a tree the kernels read."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, DTYPE, SHAPE, STRIDE, ALIAS, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5, 6, 7


@pytest.fixture(scope="module")
def tr():
    from paper_2412_20501_amd.build import ensure_built
    ensure_built()
    import paper_2412_20501_amd as m
    m.raw_lib()
    return m


def _t(tr, dtype, B, H, S, D, at, strides=None):
    return tr.TrTensor(0x7F0000000000 + (at << 36), dtype, B, H, S, D, *(strides or (H * S * D, S * D, D)))


class Call:
    """A valid call on addresses that nothing is behind, to be spoilt one argument at a time."""

    def __init__(self, tr, f8=True, D=128, page=32, seqs=3, tokens=7):
        self.tr, self.lib = tr, tr.raw_lib()
        P = tr.TR_F8E4M3 if f8 else tr.TR_BF16
        self.a = {
            "q": _t(tr, tr.TR_BF16, 1, 8, tokens, D, 1), "out": _t(tr, tr.TR_BF16, 1, 8, tokens, D, 2), "lse": _t(tr, tr.TR_F32, 1, 8, tokens, 1, 3),
            "kp": _t(tr, P, 10, 2, page, D, 8), "vp": _t(tr, P, 10, 2, page, D, 9),
            "ks": _t(tr, tr.TR_F8E8M0, 10, 2, page, 1, 10) if f8 else None, "vs": _t(tr, tr.TR_F8E8M0, 10, 2, page, 1, 11) if f8 else None,
            "w": _t(tr, tr.TR_F32, 10, 2, page, 1, 12),
            "seqs": tr.TrSequences(0x7FF000000000, 0x7FF100000000, 0x7FF200000000, None, seqs, 4, 4),
            "tree": tr.TrTree(0x7FF300000000, tokens, 2, 2), "kept": tr.TrKept(0x7FF400000000, 0x7FF500000000, 2, 50, 100, 50), "start": 0x7FF600000000,
            "causal": 1, "scale": 0.1, "fresh": 1, "first": 4, "last": 10, "ws": 0, "bytes": 0,
        }

    def __call__(self, name, **other):
        a = dict(self.a, **other)
        ref = lambda x: None if a[x] is None else ctypes.byref(a[x])   # noqa: E731
        if name == "tree":
            st = self.lib.tr_paged_attn_tree(*map(ref, ("q", "kp", "vp", "ks", "vs", "seqs", "tree")), a["scale"], ref("out"), ref("lse"), a["ws"], a["bytes"], None)
        elif name == "weigh":
            st = self.lib.tr_cache_weigh(*map(ref, ("q", "lse", "kp", "ks", "seqs")), a["causal"], a["scale"], a["fresh"], ref("w"), None)
        elif name == "select":
            st = self.lib.tr_cache_select(ref("w"), ref("seqs"), a["first"], a["last"], ref("kept"), None)
        else:
            st = self.lib.tr_cache_keep(*map(ref, ("kp", "vp", "ks", "vs", "w", "seqs", "kept")), a["start"], None)
        return st, self.lib.tr_last_error().decode()

    def like(self, name, **fields):
        t = type(self.a[name]).from_buffer_copy(self.a[name])
        for f, x in fields.items():
            setattr(t, f, x)
        return t


def test_struct_layout_matches_header(tr):
    assert ctypes.sizeof(tr.TrTree) == 32 and ctypes.sizeof(tr.TrKept) == 48


def test_pages_and_sequences_that_are_none(tr):
    c, b = Call(tr), Call(tr, f8=False)
    for name in ("tree", "weigh", "keep"):
        assert c(name, kp=None)[0] == NULL and c(name, kp=c.like("kp", ptr=None))[0] == NULL
        assert c(name, kp=c.like("kp", dtype=tr.TR_F32))[0] == DTYPE
        assert c(name, ks=None)[0] == NULL and b(name, ks=c.a["ks"])[0] == DTYPE
        assert c(name, kp=c.like("kp", ptr=0x7F8000000008))[0] == STRIDE
        assert Call(tr, D=96)(name)[0] == SHAPE and Call(tr, page=24)(name)[0] == SHAPE
    for name in ("tree", "weigh", "select", "keep"):
        assert c(name, seqs=None)[0] == NULL and c(name, seqs=c.like("seqs", kv_len=None))[0] == NULL and c(name, seqs=c.like("seqs", page_table=None))[0] == NULL
        assert c(name, seqs=c.like("seqs", n_seqs=-1))[0] == SHAPE and c(name, seqs=c.like("seqs", max_pages=(1 << 25) + 1, table_stride=1 << 26))[0] == SHAPE
        assert c(name, seqs=c.like("seqs", table_stride=3))[0] == STRIDE and c(name, seqs=c.like("seqs", kv_len=0x7FF100000002))[0] == STRIDE
    for name in ("tree", "weigh"):
        assert c(name, seqs=c.like("seqs", q_start=None))[0] == NULL and c(name, seqs=c.like("seqs", q_pos=0x7FF300000001))[0] == STRIDE
        assert c(name, seqs=c.like("seqs", n_seqs=(1 << 16) + 1))[0] == SHAPE


def test_tree_rejects(tr):
    c = Call(tr)
    assert c("tree", tree=None)[0] == NULL and "tree" in c("tree", tree=None)[1]
    assert c("tree", tree=c.like("tree", bits=None))[0] == NULL
    for f in (dict(tokens=6), dict(words=0), dict(words=-1), dict(words=(1 << 15) + 1, stride=1 << 16)):
        assert c("tree", tree=c.like("tree", **f))[0] == SHAPE
    for f in (dict(stride=1), dict(stride=-2), dict(bits=0x7FF300000002)):
        assert c("tree", tree=c.like("tree", **f))[0] == STRIDE
    assert c("tree", q=None)[0] == NULL and c("tree", q=c.like("q", dtype=tr.TR_F32))[0] == DTYPE
    assert c("tree", q=c.like("q", H=7, stride_b=7 * 7 * 128))[0] == SHAPE
    assert c("tree", out=c.like("out", S=6))[0] == SHAPE and c("tree", lse=c.like("lse", D=2, stride_s=2, stride_h=14))[0] == SHAPE
    assert c("tree", scale=0.0)[0] == UNSUPPORTED and c("tree", scale=float("nan"))[0] == UNSUPPORTED
    assert c("tree", tree=c.like("tree", bits=c.a["out"].ptr))[0] == ALIAS and c("tree", tree=c.like("tree", bits=c.a["lse"].ptr + 4))[0] == ALIAS
    need = tr.raw_lib().tr_paged_attn_tree_workspace_bytes(ctypes.byref(c.like("q")), ctypes.byref(c.like("kp")), 3, 40)
    assert need > 0
    long = dict(seqs=c.like("seqs", max_pages=40, table_stride=40))
    assert c("tree", ws=0x7FE000000000, bytes=need - 1, **long)[0] == WORKSPACE and c("tree", ws=0x7FE000000008, bytes=need, **long)[0] == WORKSPACE
    assert c("tree", ws=c.a["tree"].bits, bytes=need, **long)[0] == ALIAS


def test_weigh_rejects(tr):
    c = Call(tr)
    assert c("weigh", q=None)[0] == NULL and c("weigh", lse=None)[0] == NULL and c("weigh", w=None)[0] == NULL
    assert c("weigh", q=c.like("q", dtype=tr.TR_F32))[0] == DTYPE and c("weigh", lse=c.like("lse", dtype=tr.TR_BF16))[0] == DTYPE
    assert c("weigh", w=c.like("w", dtype=tr.TR_BF16))[0] == DTYPE
    assert c("weigh", q=c.like("q", B=2), lse=c.like("lse", B=2))[0] == SHAPE
    assert c("weigh", q=c.like("q", H=7, stride_b=7 * 7 * 128), lse=c.like("lse", H=7))[0] == SHAPE
    assert c("weigh", q=c.like("q", H=0), lse=c.like("lse", H=0))[0] == SHAPE
    assert c("weigh", lse=c.like("lse", S=6))[0] == SHAPE and c("weigh", lse=c.like("lse", D=2, stride_s=2, stride_h=14))[0] == SHAPE
    for f in (dict(B=9), dict(H=1), dict(S=16), dict(D=4)):
        assert c("weigh", w=c.like("w", **f))[0] in (SHAPE, STRIDE)
    assert c("weigh", w=c.like("w", stride_s=2, stride_h=64, stride_b=128))[0] == STRIDE
    assert c("weigh", w=c.like("w", stride_h=34, stride_b=68))[0] == STRIDE and c("weigh", w=c.like("w", ptr=c.a["w"].ptr + 4))[0] == STRIDE
    assert c("weigh", w=c.like("w", stride_b=0))[0] == STRIDE and c("weigh", w=c.like("w", stride_h=16))[0] == STRIDE      # written: must not overlap itself
    for s in (0.0, -1.0, float("inf"), float("nan")):
        assert c("weigh", scale=s)[0] == UNSUPPORTED
    for other in ("q", "lse", "kp", "ks"):
        assert c("weigh", w=c.like("w", ptr=c.a[other].ptr))[0] == ALIAS
    for at in ("page_table", "kv_len", "q_start"):
        assert c("weigh", w=c.like("w", ptr=getattr(c.a["seqs"], at)))[0] == ALIAS
    big = dict(S=1 << 28, stride_h=128 << 28)
    assert c("weigh", q=c.like("q", **big), lse=c.like("lse", S=1 << 28, stride_h=1 << 28))[0] == SHAPE                     # 2^31 rows
    st, msg = c("weigh", seqs=c.like("seqs", n_seqs=1 << 16, max_pages=1 << 15, table_stride=1 << 15))
    assert st == SHAPE and "too many keys" in msg


def test_select_rejects(tr):
    c = Call(tr)
    assert c("select", w=None)[0] == NULL and c("select", w=c.like("w", dtype=tr.TR_BF16))[0] == DTYPE and c("select", w=c.like("w", D=2, stride_s=2))[0] == SHAPE
    assert c("select", kept=None)[0] == NULL and c("select", kept=c.like("kept", keys=None))[0] == NULL and c("select", kept=c.like("kept", count=None))[0] == NULL
    for f in (dict(heads=1), dict(heads=3), dict(max_keys=-1), dict(max_keys=(1 << 30) + 1)):
        assert c("select", kept=c.like("kept", **f))[0] == SHAPE
    for f in (dict(stride_b=-1), dict(stride_h=49), dict(stride_b=99), dict(keys=0x7FF400000002), dict(count=0x7FF500000001)):
        assert c("select", kept=c.like("kept", **f))[0] == STRIDE
    for first, last in ((-1, 0), (0, -1), (51, 0), (0, 51), (25, 26), (1 << 62, 1 << 62)):
        assert c("select", first=first, last=last)[0] == SHAPE
    assert c("select", kept=c.like("kept", keys=c.a["w"].ptr))[0] == ALIAS and c("select", kept=c.like("kept", count=c.a["seqs"].kv_len))[0] == ALIAS
    assert c("select", kept=c.like("kept", count=c.a["kept"].keys + 40))[0] == ALIAS


def test_keep_rejects(tr):
    c = Call(tr)
    assert c("keep", vp=None)[0] == NULL and c("keep", vs=None)[0] == NULL and c("keep", kept=None)[0] == NULL
    assert c("keep", vp=c.like("vp", B=9))[0] == SHAPE and c("keep", vp=c.like("vp", stride_b=2 * 32 * 128 * 2))[0] == STRIDE
    assert c("keep", kept=c.like("kept", heads=3))[0] == SHAPE and c("keep", kept=c.like("kept", max_keys=-1))[0] == SHAPE
    assert c("keep", start=0x7FF600000002)[0] == STRIDE
    assert c("keep", w=c.like("w", S=16))[0] in (SHAPE, STRIDE) and c("keep", w=c.like("w", dtype=tr.TR_BF16))[0] == DTYPE
    assert c("keep", **{f: c.like(f, stride_b=0) for f in ("kp", "vp")})[0] == STRIDE
    for f in ("kp", "vp", "ks", "vs"):
        assert c("keep", w=c.like("w", ptr=c.a[f].ptr))[0] == ALIAS
        assert c("keep", kept=c.like("kept", keys=c.a[f].ptr))[0] == ALIAS
        assert c("keep", start=c.a[f].ptr)[0] == ALIAS
    assert c("keep", vp=c.like("vp", ptr=c.a["kp"].ptr + 128))[0] == ALIAS
    assert c("keep", kept=c.like("kept", count=c.a["w"].ptr))[0] == ALIAS


def test_calls_without_work(tr):
    """Nothing is launched (there is no GPU here), nothing is wrong."""
    c = Call(tr)
    none = dict(seqs=c.like("seqs", n_seqs=0))
    for name in ("tree", "weigh", "select", "keep"):
        assert c(name, **none)[0] == 0
    empty = dict(q=c.like("q", S=0), lse=c.like("lse", S=0))
    assert c("weigh", **empty)[0] == 0
    assert c("tree", out=c.like("out", S=0), tree=c.like("tree", tokens=0, bits=None), **empty)[0] == 0
    assert c("keep", kept=c.like("kept", max_keys=0, keys=None))[0] == 0
    assert c("weigh", seqs=c.like("seqs", max_pages=0))[0] == 0 and c("keep", seqs=c.like("seqs", max_pages=0))[0] == 0


def test_tensors_that_are_not_on_the_gpu(tr):
    i = lambda *s: torch.zeros(s, dtype=torch.int32)   # noqa: E731
    w = torch.zeros(4, 2, 16)
    with pytest.raises(ValueError, match="current GPU"):
        tr.tr_cache_select(w, i(1, 4), i(1), 0, 0, i(1, 2, 8), i(1))
    with pytest.raises(TypeError):
        tr.tr_cache_select(None, i(1, 4), i(1), 0, 0, i(1, 2, 8), i(1))
    with pytest.raises(ValueError, match="dimension"):
        tr.tr_paged_attn_tree_workspace_bytes(torch.zeros(1, 8, 3, 128, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16), i(4))


@pytest.mark.parametrize("name,ok", [("tree_bits_check", "tree bits ok"), ("tree_launch_check", "tree launches ok")])
def test_host_checks(tmp_path, name, ok):
    exe = str(tmp_path / name)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-I",
                    os.path.join(ROOT, "paper_2412_20501_amd", "csrc"), os.path.join(ROOT, "tests", "c_abi", name + ".cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and ok in res.stdout, res.stdout + res.stderr
