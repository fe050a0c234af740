"""Sizes that the operators on a paged cache refuse, on a machine without a GPU: addresses that nothing is behind, refused before anything is launched."""
import ctypes

import pytest

SHAPE = 3
BASE = 1 << 44


@pytest.fixture(scope="module")
def tr():
    from paper_2412_20501_amd.build import ensure_built
    ensure_built()
    import paper_2412_20501_amd as m
    m.raw_lib()
    return m


def _t(tr, dtype, B, H, S, D, at):
    return tr.TrTensor(BASE + (at << 40), dtype, B, H, S, D, H * S * D, S * D, D)


def _seqs(tr, n, max_pages=4):
    return tr.TrSequences(BASE + (20 << 40), BASE + (21 << 40), BASE + (22 << 40), None, n, max_pages, max_pages)


def _refs(*x):
    return [None if y is None else ctypes.byref(y) for y in x]


def test_more_rows_of_heads_than_a_read_counts(tr):
    """2^24 sequences of 64 heads, K and V: their number passes 2^31, in which the kernel counts."""
    lib, n = tr.raw_lib(), 1 << 24

    def read(n, H, S=1):   # (S = 0: nothing to read)
        pages = [_t(tr, tr.TR_BF16, 10, H, 16, 64, i) for i in (1, 2)]
        out = [_t(tr, tr.TR_BF16, n, H, S, 64, i) for i in (3, 4)]
        s = _seqs(tr, n)
        st = lib.tr_cache_read(*_refs(*pages, None, None, s), 0, *_refs(*out), None)
        return st, lib.tr_last_error().decode()
    for n, H in ((1 << 24, 64), (1 << 24, 100), (1 << 20, 1024)):
        st, msg = read(n, H)
        assert st == SHAPE and "2^31" in msg, (n, H, st, msg)
    assert read((1 << 24) - 1, 64, 0)[0] == 0


def test_more_sequences_than_an_attention_call_takes(tr):
    """Every workgroup of the attention goes through the sequences: beyond 2^16 of them a call would hold the GPU for seconds to hours."""
    lib = tr.raw_lib()
    pages = [_t(tr, tr.TR_BF16, 10, 2, 16, 64, i) for i in (1, 2)]

    def attend(n, S):
        q, out, lse = _t(tr, tr.TR_BF16, 1, 4, S, 64, 3), _t(tr, tr.TR_BF16, 1, 4, S, 64, 4), _t(tr, tr.TR_F32, 1, 4, S, 1, 5)
        s = _seqs(tr, n, 64)
        st = lib.tr_paged_attn(*_refs(q, *pages, None, None, s), 1, 0.1, *_refs(out, lse), None, 0, None)
        return st, lib.tr_last_error().decode(), lib.tr_paged_attn_workspace_bytes(*_refs(q, pages[0]), n, 64)
    for n in ((1 << 16) + 1, 1 << 24):
        st, msg, need = attend(n, 100)
        assert st == SHAPE and "2^16" in msg and need == 0
    st, msg, need = attend(1 << 16, 0)
    assert st == 0 and need == 0
    q = _t(tr, tr.TR_BF16, 1, 4, 100, 64, 3)
    assert lib.tr_paged_attn_workspace_bytes(*_refs(q, pages[0]), 1 << 16, 64) > 0


def test_workspace_bytes_of_calls_that_are_none(tr):
    """0 for types and shapes that tr_paged_attn refuses."""
    lib = tr.raw_lib()

    def need(q=None, pages=None, n=3, max_pages=64):
        a = dict(dtype=tr.TR_BF16, B=1, H=4, S=100, D=64)
        b = dict(dtype=tr.TR_F8E4M3, B=10, H=2, S=16, D=64)
        a.update(q or {})
        b.update(pages or {})
        return lib.tr_paged_attn_workspace_bytes(*_refs(*(_t(tr, x["dtype"], x["B"], x["H"], x["S"], x["D"], i) for i, x in enumerate((a, b)))), n, max_pages)
    assert need() > 0 and need(pages=dict(dtype=tr.TR_BF16)) > 0
    for q in (dict(dtype=tr.TR_F32), dict(dtype=tr.TR_F8E4M3), dict(B=2), dict(B=0), dict(D=96), dict(D=128), dict(H=3)):
        assert need(q=q) == 0, q
    for pages in (dict(dtype=tr.TR_F32), dict(dtype=tr.TR_F8E8M0), dict(dtype=7), dict(D=128), dict(S=24), dict(S=8), dict(B=-1), dict(H=0)):
        assert need(pages=pages) == 0, pages
    assert need(n=-1) == 0 and need(max_pages=-1) == 0
