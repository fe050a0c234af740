"""The operators on a paged cache on a machine without a GPU: what they refuse before anything is launched, and the bounds that their kernels keep."""
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
            "k": _t(tr, tr.TR_BF16, 1, 2, tokens, D, 4), "v": _t(tr, tr.TR_BF16, 1, 2, tokens, D, 5),
            "k_out": _t(tr, tr.TR_BF16, seqs, 2, 50, D, 6), "v_out": _t(tr, tr.TR_BF16, seqs, 2, 50, D, 7),
            "kp": _t(tr, P, 10, 2, page, D, 8), "vp": _t(tr, P, 10, 2, page, D, 9),
            "ks": _t(tr, tr.TR_F8E8M0, 10, 2, page, 1, 10) if f8 else None, "vs": _t(tr, tr.TR_F8E8M0, 10, 2, page, 1, 11) if f8 else None,
            "seqs": tr.TrSequences(0x7FF000000000, 0x7FF100000000, 0x7FF200000000, None, seqs, 4, 4),
            "first": 0, "causal": 1, "scale": 0.1, "ws": 0, "bytes": 0,
        }

    def __call__(self, name, **other):
        a = dict(self.a, **other)
        ref = lambda x: None if a[x] is None else ctypes.byref(a[x])   # noqa: E731
        if name == "write":
            st = self.lib.tr_cache_write(*map(ref, ("k", "v", "kp", "vp", "ks", "vs", "seqs")), None)
        elif name == "read":
            st = self.lib.tr_cache_read(*map(ref, ("kp", "vp", "ks", "vs", "seqs")), a["first"], ref("k_out"), ref("v_out"), None)
        else:
            st = self.lib.tr_paged_attn(*map(ref, ("q", "kp", "vp", "ks", "vs", "seqs")), a["causal"], a["scale"], ref("out"), ref("lse"), a["ws"], a["bytes"], None)
        return st, self.lib.tr_last_error().decode()

    def like(self, name, **fields):
        t = type(self.a[name]).from_buffer_copy(self.a[name])
        for f, x in fields.items():
            setattr(t, f, x)
        return t


ALL = ("write", "read", "attn")


def test_a_cache_that_is_none(tr):
    c, b = Call(tr), Call(tr, f8=False)
    for name in ALL:
        assert c(name, kp=None)[0] == NULL and c(name, vp=None)[0] == NULL and c(name, kp=c.like("kp", ptr=None))[0] == NULL
        assert c(name, kp=c.like("kp", dtype=tr.TR_F32))[0] == DTYPE and c(name, kp=c.like("kp", dtype=tr.TR_F8E8M0))[0] == DTYPE
        assert c(name, kp=c.like("kp", dtype=4))[0] == DTYPE
        assert c(name, kp=c.like("kp", dtype=tr.TR_BF16))[0] == DTYPE                    # K and V of one type
        assert c(name, ks=None)[0] == NULL and c(name, vs=None)[0] == NULL               # e4m3 has scales
        assert b(name, ks=c.a["ks"])[0] == DTYPE                                         # bf16 has none
        assert c(name, ks=c.like("ks", dtype=tr.TR_F32))[0] == DTYPE
        assert c(name, vp=c.like("vp", B=9))[0] == SHAPE and c(name, vp=c.like("vp", S=16))[0] == SHAPE
        assert c(name, ks=c.like("ks", S=16))[0] == SHAPE and c(name, vs=c.like("vs", B=9))[0] == SHAPE
        assert c(name, vp=c.like("vp", stride_b=2 * 32 * 128 * 2))[0] == STRIDE
        assert c(name, vs=c.like("vs", stride_b=128))[0] == STRIDE
        assert c(name, kp=c.like("kp", ptr=0x7F8000000008))[0] == STRIDE
        for f in ("ks", "vs"):
            assert c(name, **{f: c.like(f, ptr=c.a[f].ptr + 8)})[0] == STRIDE
        both = {f: c.like(f, stride_b=72) for f in ("ks", "vs")}
        assert c(name, **both)[0] == STRIDE
        both = {f: c.like(f, stride_s=2, stride_h=64, stride_b=128) for f in ("ks", "vs")}
        assert c(name, **both)[0] == STRIDE
        both = {f: c.like(f, stride_s=(1 << 24) + 16, stride_h=1 << 30, stride_b=1 << 31) for f in ("kp", "vp")}
        st, msg = c(name, **both)
        assert st == STRIDE and "2^24" in msg
    for page in (0, 8, 24, 40):
        st, msg = Call(tr, page=page)("attn")
        assert st == SHAPE and "page size" in msg
    st, msg = Call(tr, D=96)("attn")
    assert st == SHAPE and "head dim" in msg
    st, msg = Call(tr, D=32)("write")
    assert st == SHAPE and "head dim" in msg


def test_sequences_that_are_none(tr):
    c = Call(tr)
    for name in ALL:
        assert c(name, seqs=None)[0] == NULL
        assert c(name, seqs=c.like("seqs", kv_len=None))[0] == NULL and c(name, seqs=c.like("seqs", page_table=None))[0] == NULL
        assert c(name, seqs=c.like("seqs", n_seqs=-1))[0] == SHAPE and c(name, seqs=c.like("seqs", max_pages=-1))[0] == SHAPE
        assert c(name, seqs=c.like("seqs", max_pages=(1 << 25) + 1, table_stride=1 << 26))[0] == SHAPE      # 32 keys a page: more than 2^30 keys
        assert c(name, seqs=c.like("seqs", table_stride=3))[0] == STRIDE
        assert c(name, seqs=c.like("seqs", kv_len=0x7FF100000002))[0] == STRIDE
    for name in ("write", "attn"):
        assert c(name, seqs=c.like("seqs", q_start=None))[0] == NULL
        assert c(name, seqs=c.like("seqs", q_pos=0x7FF300000001))[0] == STRIDE


def test_write_rejects(tr):
    c = Call(tr)
    assert c("write", k=None)[0] == NULL and c("write", k=c.like("k", dtype=tr.TR_F32))[0] == DTYPE
    assert c("write", k=c.like("k", B=2), v=c.like("v", B=2))[0] == SHAPE
    assert c("write", k=c.like("k", H=1))[0] == SHAPE and c("write", v=c.like("v", S=6))[0] == SHAPE
    assert c("write", v=c.like("v", stride_h=8 * 128))[0] == STRIDE
    assert c("write", k=c.like("k", stride_s=132, stride_h=7 * 132), v=c.like("v", stride_s=132, stride_h=7 * 132))[0] == STRIDE
    big = dict(S=1 << 30, stride_h=128 << 30)
    assert c("write", k=c.like("k", **big), v=c.like("v", **big))[0] == SHAPE
    # what is written must not overlap itself, K and V, pages and scales, what is read
    assert c("write", **{f: c.like(f, stride_b=0) for f in ("kp", "vp")})[0] == STRIDE
    assert c("write", vp=c.a["kp"])[0] == ALIAS and c("write", vp=c.like("vp", ptr=c.a["kp"].ptr + 64))[0] == ALIAS
    assert c("write", vs=c.a["ks"])[0] == ALIAS and c("write", ks=c.like("ks", ptr=c.a["kp"].ptr), vs=c.like("vs", ptr=c.a["kp"].ptr + (1 << 30)))[0] == ALIAS
    assert c("write", k=c.like("k", ptr=c.a["kp"].ptr))[0] == ALIAS
    assert c("write", seqs=c.like("seqs", kv_len=c.a["vp"].ptr))[0] == ALIAS


def test_k_and_v_in_one_array(tr):
    """K and V side by side in a page or in a row are apart; shifted by less or by more than their step they are not.  (A write without tokens, so that nothing is launched.)"""
    c = Call(tr, tokens=0)
    base = c.a["kp"].ptr

    def write(off, sb, sh, ss, size=(10, 2, 32, 128)):
        f = dict(zip(("B", "H", "S", "D"), size), stride_b=sb, stride_h=sh, stride_s=ss)
        return c("write", kp=c.like("kp", **f), vp=c.like("vp", ptr=base + off, **f))[0]
    half = 2 * 32 * 128
    assert write(half, 2 * half, 32 * 128, 128) == 0                     # [pages, 2, heads, keys, D]
    assert write(128, 2 * half, 256, 2 * 256) == 0                       # [pages, keys, heads, 2, D]
    assert write(2 * 128, 2 * half, 128, 4 * 128) == 0                   # [pages, keys, 2, heads, D]
    assert write(half + 128, 2 * half, 32 * 128, 128) == ALIAS
    assert write(half - 16, 2 * half, 32 * 128, 128) == ALIAS
    assert write(3 * half, 2 * half, 32 * 128, 128) == 0                 # the half of the page after: apart too
    assert write(64, 2 * half, 256, 2 * 256) == ALIAS
    assert write(128, 2 * half + 128, 256, 2 * 256) == ALIAS             # steps of the pages that are no multiple of the rows'


def test_more_than_a_launch_holds(tr):
    c = Call(tr)
    def call(name, fields, S, H=2):   # noqa: E306
        return c(name, **{f: c.like(f, H=H, S=S, stride_h=128 * S, stride_b=128 * S * H) for f in fields})
    st, msg = call("write", ("k", "v"), 1 << 28)
    assert st == SHAPE and "2^24" in msg
    st, msg = call("read", ("k_out", "v_out"), 1 << 30)
    assert st == SHAPE and "2^24" in msg


def test_layout_of_the_sequences(tr):
    assert ctypes.sizeof(tr.TrSequences) == 4 * 8 + 3 * 8 and tr.TrSequences.n_seqs.offset == 32


def test_read_rejects(tr):
    c = Call(tr)
    assert c("read", first=-1)[0] == SHAPE
    assert c("read", k_out=c.like("k_out", dtype=tr.TR_F32))[0] == DTYPE and c("read", k_out=c.like("k_out", B=2))[0] == SHAPE
    assert c("read", k_out=c.like("k_out", H=1))[0] == SHAPE and c("read", v_out=c.like("v_out", S=49))[0] == SHAPE
    assert c("read", **{f: c.like(f, B=2) for f in ("k_out", "v_out")})[0] == SHAPE       # three sequences
    assert c("read", v_out=c.like("v_out", stride_h=51 * 128))[0] == STRIDE
    assert c("read", **{f: c.like(f, stride_h=0) for f in ("k_out", "v_out")})[0] == STRIDE
    assert c("read", v_out=c.a["k_out"])[0] == ALIAS and c("read", k_out=c.like("k_out", ptr=c.a["ks"].ptr))[0] == ALIAS
    assert c("read", v_out=c.like("v_out", ptr=c.a["seqs"].page_table))[0] == ALIAS


def test_attn_rejects(tr):
    c = Call(tr)
    assert c("attn", q=None)[0] == NULL and c("attn", lse=None)[0] == NULL
    assert c("attn", q=c.like("q", dtype=tr.TR_F8E4M3))[0] == DTYPE and c("attn", out=c.like("out", dtype=tr.TR_F8E4M3))[0] == DTYPE
    assert c("attn", lse=c.like("lse", dtype=tr.TR_BF16))[0] == DTYPE
    assert c("attn", **{f: c.like(f, B=2) for f in ("q", "out", "lse")})[0] == SHAPE
    assert c("attn", q=c.like("q", D=64))[0] == SHAPE and c("attn", out=c.like("out", S=6))[0] == SHAPE and c("attn", lse=c.like("lse", H=4))[0] == SHAPE
    assert c("attn", **{f: c.like(f, H=7) for f in ("q", "out", "lse")})[0] == SHAPE      # 7 heads on 2
    assert c("attn", scale=0.0)[0] == UNSUPPORTED and c("attn", scale=float("nan"))[0] == UNSUPPORTED and c("attn", scale=float("inf"))[0] == UNSUPPORTED
    assert c("attn", out=c.like("out", stride_h=0))[0] == STRIDE and c("attn", q=c.like("q", ptr=c.a["q"].ptr + 8))[0] == STRIDE
    for f in ("q", "kp", "vs"):
        assert c("attn", out=c.like("out", ptr=c.a[f].ptr))[0] == ALIAS
    assert c("attn", lse=c.like("lse", ptr=c.a["out"].ptr))[0] == ALIAS and c("attn", lse=c.like("lse", ptr=c.a["seqs"].q_start))[0] == ALIAS
    need = c.lib.tr_paged_attn_workspace_bytes(ctypes.byref(c.a["q"]), ctypes.byref(c.a["kp"]), 3, 64)
    assert need > 0
    wide = c.like("seqs", max_pages=64, table_stride=64)
    assert c("attn", seqs=wide, ws=0x7FE000000000, bytes=need - 1)[0] == WORKSPACE
    assert c("attn", seqs=wide, ws=0x7FE000000080, bytes=need)[0] == WORKSPACE
    assert c("attn", seqs=wide, ws=c.a["vp"].ptr, bytes=need)[0] == ALIAS
    big = dict(S=1 << 28, stride_h=128 << 28)
    assert c("attn", q=c.like("q", **big), out=c.like("out", **big), lse=c.like("lse", S=1 << 28, stride_h=1 << 28))[0] == SHAPE


def test_calls_with_nothing_to_do(tr):
    """No tokens, no sequences, no rows: nothing is launched (there is no GPU here)."""
    for f8 in (False, True):
        c = Call(tr, f8=f8, tokens=0)
        assert c("write")[0] == 0 and c("attn")[0] == 0
        none = Call(tr, f8=f8, seqs=0)
        assert none("write")[0] == 0 and none("attn")[0] == 0 and none("read")[0] == 0
        assert c("read", **{f: c.like(f, S=0) for f in ("k_out", "v_out")})[0] == 0
        w = c.lib.tr_paged_attn_workspace_bytes
        assert w(ctypes.byref(c.a["q"]), ctypes.byref(c.a["kp"]), 3, 64) == 0 and w(None, None, 3, 64) == 0


def test_python_operands(tr):
    """Tensors must be on the current GPU; index arrays int32 of the right sizes are looked at first where no GPU is."""
    q = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    pages = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    table, n = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    lse = torch.zeros(1, 4, 2)
    call = lambda **o: tr.tr_paged_attn(*(o.get(x, y) for x, y in (("q", q), ("kp", pages), ("vp", pages), ("table", table), ("n", n))),   # noqa: E731
                                        torch.zeros(2, dtype=torch.int32), True, 0.1, q, lse)
    with pytest.raises(ValueError, match="current GPU"):
        call()
    with pytest.raises(TypeError, match="a tensor is expected"):
        call(q=None)
    with pytest.raises(ValueError, match="strided"):
        call(q=q.float().to_sparse())
    with pytest.raises(ValueError, match="current GPU"):
        tr.tr_cache_write(q, q, pages, pages, table, n, n)
    with pytest.raises(ValueError, match="current GPU"):
        tr.tr_cache_read(pages, pages, table, n, q, q)
    # 8192 keys: keys are shared out; what the workspace holds for that grows with the head dim only
    many = torch.zeros(1, 512, dtype=torch.int32)
    with pytest.raises(ValueError, match=r"\[B,H,S,D\]"):
        tr.tr_paged_attn_workspace_bytes(q[0], pages, many)
    with pytest.raises(ValueError, match="page_table"):
        tr.tr_paged_attn_workspace_bytes(q, pages, many[0])
    assert tr.tr_paged_attn_workspace_bytes(q, pages, many) > 0 and tr.tr_paged_attn_workspace_bytes(q[:, :, :0], pages, many) == 0


def test_bounds_of_the_kernels(tmp_path):
    """csrc/paged_plan.h, by which the kernels address tables, pages and scratch, compiled for the host with its reads checked."""
    exe = str(tmp_path / "paged_plan_check")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-I",
                    os.path.join(ROOT, "paper_2412_20501_amd", "csrc"), os.path.join(ROOT, "tests", "c_abi", "paged_plan_check.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "paged plan ok" in res.stdout, res.stdout + res.stderr
