"""tr_paged_attn against a 64-bit implementation, within bounds that follow from its roundings (paged_util)."""
import pytest
import torch

from paged_util import Cache, attention, check

pytestmark = pytest.mark.gpu


def _run(lib, c, Hq, causal=True, pos=None, out_dtype=torch.bfloat16, workspace=True, seed=1, scale=None, behind=0, q=None):
    """(results of the call, found by the oracle); tokens `behind` the last sequence stay as they were."""
    g = torch.Generator().manual_seed(seed)
    if q is None:
        q = torch.randn(1, c.tokens + behind, Hq, c.D, generator=g).bfloat16().cuda().transpose(1, 2)
    out = torch.full((1, c.tokens + behind, Hq, c.D), 3.5, dtype=out_dtype, device="cuda").transpose(1, 2)
    lse = torch.full((1, Hq, c.tokens + behind), 4.5, device="cuda")
    scale = c.D ** -0.5 if scale is None else scale
    ws = torch.full((lib.tr_paged_attn_workspace_bytes(q, c.pages["k"], c.table),), 255, dtype=torch.uint8, device="cuda") if workspace else None
    p = None if pos is None else torch.tensor(pos, dtype=torch.int32, device="cuda")
    lib.tr_paged_attn(q, *c.args(), c.q_start, causal, scale, out, lse, *c.scale_args(), q_pos=p, workspace=ws)
    if behind:
        assert (out[:, :, c.tokens:] == 3.5).all() and (lse[:, :, c.tokens:] == 4.5).all()
    return q, out, lse, attention(c, q, scale, causal, pos)


SHAPES = [
    # keys, new tokens, Hkv, query heads a K/V head, page
    ([1], [1], 1, 1, 16),
    ([5], [1], 2, 4, 16),
    ([31, 32, 33], [1, 1, 1], 2, 4, 16),
    ([127, 128, 129, 130], [1, 2, 3, 4], 1, 5, 32),
    ([300, 0, 17, 1], [1, 0, 1, 1], 2, 7, 48),
    ([1000, 3], [3, 3], 2, 8, 64),
    ([4500], [1], 1, 8, 16),
    ([2000, 10, 1999], [1, 1, 1], 2, 16, 128),
    ([5000, 33], [5, 33], 1, 4, 32),
    ([90], [90], 2, 2, 16),
    ([700, 650], [130, 257], 2, 3, 48),
    ([1500, 40, 900], [513, 1, 64], 1, 4, 16),
    ([600], [600], 2, 1, 32),
]


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", SHAPES)
def test_lengths(lib, shape, D, f8):
    kv, q, Hkv, gq, page = shape
    c = Cache(kv, q, Hkv, D, page, f8, "head" if len(kv) % 2 else "token", seed=D + len(kv))
    for workspace in (True, False):
        _, out, lse, found = _run(lib, c, Hkv * gq, workspace=workspace, behind=2)
        print(check(found, out, lse))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_fp32_results_and_no_mask(lib, D, causal, f8):
    c = Cache([200, 4000, 77], [9, 2, 77], 2, D, 32, f8, "head", seed=5)
    _, out, lse, found = _run(lib, c, 8, causal, out_dtype=torch.float32)
    check(found, out, lse)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n", [3, 70])
def test_positions(lib, n, f8):
    """New tokens in front of all keys (rows that see none), between them, and behind them."""
    c = Cache([150, 2500, 64, 40], [n] * 4, 2, 128, 16, f8, "head", seed=6)
    pos = [-2, 1000 - n, 64, -1000]
    _, out, lse, found = _run(lib, c, 8, True, pos)
    check(found, out, lse)
    assert (out[:, :, c.starts[3]:] == 0).all() and torch.isneginf(lse[:, :, c.starts[3]:]).all()
    assert (out[:, :, 0] == 0).all() and torch.isneginf(lse[:, :, 0]).all()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n", [1, 70])
def test_entries_that_are_no_pages(lib, n, f8):
    c = Cache([500, 3000], [n, n], 2, 128, 16, f8, "token", seed=7)
    c.table[0, 3], c.table[0, 30], c.table[1, 0], c.table[1, 100] = -1, c.n_pages, 2 ** 31 - 1, -2 ** 31
    _, out, lse, found = _run(lib, c, 8)
    check(found, out, lse)
    c.table.fill_(-1)
    _, out, lse, found = _run(lib, c, 8)
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("n", [4, 70])
def test_bad_values_reach_the_rows_that_see_them(lib, n, bad, f8):
    """An infinity or NaN in V of a new token: later rows have it, earlier ones nothing of it.  (e4m3 has no infinities: NaN.)"""
    c = Cache([333, 2000], [n, n], 2, 128, 16, f8, "head", seed=8)
    for b in range(2):
        key = c.kv[b] - n // 2
        page, slot = int(c.table[b, key // 16]), key % 16
        if f8:
            c.pages["v"].view(torch.uint8)[page, 1, slot, 5] = 127
        else:
            c.pages["v"][page, 1, slot, 5] = bad
    _, out, lse, found = _run(lib, c, 8)
    check(found, out, lse)
    assert out[0, 4:, c.starts[1] - 1, 5].isfinite().sum() == 0 and out[0, :4].isfinite().all()


def test_bad_scores(lib):
    """A NaN in K of a key that all rows see: out = NaN, lse = -inf, as of a block step; other heads have nothing of it."""
    for n, kv in ((1, 200), (1, 5000), (70, 500)):
        c = Cache([kv], [n], 2, 128, 16, False, "head", seed=9)
        c.pages["k"][int(c.table[0, 2]), 1, 3, 5] = float("nan")
        _, out, lse, _ = _run(lib, c, 8)
        assert out[:, 4:].isnan().all() and torch.isneginf(lse[:, 4:]).all()
        assert out[:, :4].isfinite().all() and lse[:, :4].isfinite().all()


@pytest.mark.parametrize("n", [1, 70])
def test_scores_far_apart(lib, n):
    """Scores that grow by hundreds along the keys, so that references are replaced again and again, and the other way round."""
    for sign in (1.0, -1.0):
        c = Cache([900], [n], 1, 64, 16, False, "head", seed=10, std=0.1)
        for i in range(900):
            c.pages["k"][int(c.table[0, i // 16]), 0, i % 16, 0] = sign * (i // 8)
        q = torch.zeros(1, 4, n, 64, dtype=torch.bfloat16, device="cuda")
        q[..., 0] = 8.0
        _, out, lse, found = _run(lib, c, 4, scale=1.0, q=q)
        check(found, out, lse)


def test_sequences_that_share_pages(lib):
    """Two sequences with the same first pages, and one page twice in a table."""
    c = Cache([160, 160, 64], [1, 20, 5], 2, 128, 16, False, "head", seed=12)
    c.table[1, :6] = c.table[0, :6]
    c.table[2, 1] = c.table[2, 0]
    _, out, lse, found = _run(lib, c, 8)
    check(found, out, lse)


def test_many_sequences(lib):
    """More sequences than a wave has lanes, most without new tokens or keys."""
    kv = [(37 * i) % 700 if i % 3 else 0 for i in range(200)]
    q = [[1, 0, 2, 30][i % 4] if i % 5 else 0 for i in range(200)]
    kv = [max(a, b) for a, b in zip(kv, q)]
    kv[150] = 6000
    c = Cache(kv, q, 2, 64, 32, True, "head", seed=13)
    _, out, lse, found = _run(lib, c, 8, behind=3)
    check(found, out, lse)


@pytest.mark.parametrize("f8", [False, True])
def test_a_prompt_among_many_tokens(lib, f8):
    """A chunk of a prompt and drafts in a call whose sequences have few rows on average."""
    q = [1] * 70
    q[33], q[50], q[60] = 330, 6, 9
    c = Cache([n + 13 * (i % 7) for i, n in enumerate(q)], q, 1, 128, 16, f8, "head", seed=18)
    _, out, lse, found = _run(lib, c, 4, behind=1)
    check(found, out, lse)


def test_arrays_with_wrong_entries(lib):
    """Lengths and starts out of range are taken as the nearest that is: nothing else is touched."""
    c = Cache([48, 48, 48], [2, 2, 2], 1, 128, 16, False, "head", seed=14, poison=False)
    q = torch.randn(1, 4, 6, 128, device="cuda").bfloat16()
    out, lse = torch.full((1, 4, 6, 128), 3.5, device="cuda"), torch.full((1, 4, 6), 4.5, device="cuda")
    lens = torch.tensor([-5, 1 << 30, 48], dtype=torch.int32, device="cuda")
    starts = torch.tensor([-3, 2, 4, 1 << 30], dtype=torch.int32, device="cuda")
    lib.tr_paged_attn(q, *c.args()[:3], lens, starts, True, 0.1, out, lse)
    assert (out[:, :, :2] == 0).all() and torch.isneginf(lse[:, :, :2]).all() and out.isfinite().all()
    lib.tr_cache_write(q[:, :1], q[:, 1:2], *c.args()[:3], lens, starts)
    backwards = torch.tensor([6, 4, 2, 0], dtype=torch.int32, device="cuda")
    out.fill_(3.5)
    lib.tr_paged_attn(q, *c.args(), backwards, True, 0.1, out, lse)
    assert (out == 3.5).all()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", [([12001], [300], 1, 4, 64), ([9000, 20, 300], [700, 1, 31], 2, 2, 16), ([40000, 1], [1, 1], 1, 8, 16), ([6000] * 5, [7] * 5, 1, 4, 32)])
def test_long_caches(lib, shape, D, f8):
    """Keys that are shared out among workgroups, and the same without a workspace."""
    kv, q, Hkv, gq, page = shape
    c = Cache(kv, q, Hkv, D, page, f8, "head", seed=15)
    for workspace in (True, False):
        _, out, lse, found = _run(lib, c, Hkv * gq, workspace=workspace, behind=1)
        print(check(found, out, lse))


@pytest.mark.parametrize("form", ["pages", "rows", "heads"])
def test_k_and_v_in_one_array(lib, form):
    """K and V as the two halves of each page, of each row and of each token's heads; results and queries head by head."""
    H, page, D = 2, 32, 64
    c = Cache([500, 77, 300], [3, 40, 100], H, D, page, False, "head", seed=16)
    P = c.n_pages
    if form == "pages":
        both = torch.empty(P, 2, H, page, D, dtype=torch.bfloat16, device="cuda")
        k, v = both[:, 0], both[:, 1]
    elif form == "rows":
        both = torch.empty(P, page, H, 2 * D, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        k, v = both[..., :D], both[..., D:]
    else:
        both = torch.empty(P, page, 2 * H, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        k, v = both[:, :H], both[:, H:]
    k.copy_(c.pages["k"])
    v.copy_(c.pages["v"])
    c.pages = {"k": k, "v": v}
    q = torch.randn(1, 8, c.tokens, D, device="cuda").bfloat16()
    out = torch.zeros(1, 8, c.tokens, D + 24, dtype=torch.bfloat16, device="cuda")[..., :D]
    lse = torch.zeros(c.tokens, 8, device="cuda").t().unsqueeze(0)
    lib.tr_paged_attn(q, *c.args(), c.q_start, True, 0.1, out, lse)
    check(attention(c, q, 0.1, True), out, lse)
    new = torch.randn(1, c.tokens, H, D, device="cuda").bfloat16().transpose(1, 2)
    lib.tr_cache_write(new, new + 1, *c.args(), c.q_start)
    assert torch.equal(c.rows("k", 1)[0][37:].transpose(0, 1), new[0, :, 3:43].double())
    assert torch.equal(c.rows("v", 2)[0][200:].transpose(0, 1), (new + 1)[0, :, 43:].double())
    back = [torch.empty(3, H, 500, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lib.tr_cache_read(*c.args(), *back)
    assert torch.equal(back[0][0].double(), c.rows("k", 0)[0].transpose(0, 1)) and torch.equal(back[1][1, :, :77].double(), c.rows("v", 1)[0].transpose(0, 1))


def test_what_the_gpu_refuses(lib):
    """Operands on the CPU, index arrays of other types and sizes."""
    c = Cache([20], [2], 1, 64, 16, False, "head", seed=17)
    q, out, lse = (torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)), None, torch.zeros(1, 2, 2, device="cuda")
    q, out = q
    call = lambda **o: lib.tr_paged_attn(o.get("q", q), *c.args()[:2], o.get("table", c.table), o.get("n", c.kv_len), o.get("start", c.q_start), True, 0.1,   # noqa: E731
                                         o.get("out", out), lse, q_pos=o.get("pos"), workspace=o.get("ws"))
    call()
    with pytest.raises(ValueError, match="different devices"):
        call(out=out.cpu())
    with pytest.raises(ValueError, match="different devices"):
        call(start=c.q_start.cpu())
    with pytest.raises(TypeError, match="page_table must be int32"):
        call(table=c.table.long())
    with pytest.raises(TypeError, match="unsupported dtype"):
        call(q=q.half())
    with pytest.raises(ValueError, match="kv_len must have 1 elements"):
        call(n=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="q_start must have 2 elements"):
        call(start=c.kv_len)
    with pytest.raises(ValueError, match="dimension"):
        call(table=c.table[0])
    with pytest.raises(ValueError, match="contiguous"):
        call(ws=torch.zeros(64, 64, dtype=torch.uint8, device="cuda").t()[:, :3])
    with pytest.raises(lib.TokenRingError, match="TR_ERR_ALIAS"):
        call(out=q)
    long = torch.full((1, 64), -1, dtype=torch.int32, device="cuda")
    with pytest.raises(lib.TokenRingError, match="too small"):
        call(table=long, ws=torch.zeros(256, dtype=torch.uint8, device="cuda"))


def test_a_cache_without_pages(lib):
    """No page at all: nothing is seen, written or read."""
    for f8 in (False, True):
        t = torch.float8_e4m3fn if f8 else torch.bfloat16
        pages = torch.empty(0, 2, 16, 64, dtype=t, device="cuda")
        s = torch.empty(0, 2, 16, dtype=torch.float8_e8m0fnu, device="cuda") if f8 else None
        ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
        table, kv, start = ints(*range(64)).view(1, 64), ints(1000), ints(0, 300)
        q = torch.randn(1, 2, 300, 64, device="cuda").bfloat16()
        out, lse = torch.full_like(q, 7), torch.zeros(1, 2, 300, device="cuda")
        lib.tr_paged_attn(q, pages, pages, table, kv, start, True, 0.1, out, lse, s, s)
        assert (out == 0).all() and torch.isneginf(lse).all()
        k = torch.full((1, 2, 1000, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        v = k.clone()
        lib.tr_cache_read(pages, pages, table, kv, k, v, 0, s, s)
        lib.tr_cache_write(q, q, pages, pages, table, kv, start, s, s)
        torch.cuda.synchronize()
        assert (k == 7).all() and (v == 7).all()
