"""tr_cache_weigh against a 64-bit implementation, within bounds that follow from its roundings (evict_util)."""
import math

import pytest
import torch

from evict_util import causal_mask, lse_of, weigh
from paged_util import Cache

pytestmark = pytest.mark.gpu


def _run(lib, c, Hq, causal=True, fresh=True, pos=None, seed=1, layout="dense", behind=0, q=None, lse=None, change=None):
    g = torch.Generator().manual_seed(seed)
    if q is None:
        q = torch.randn(1, c.tokens + behind, Hq, c.D, generator=g).bfloat16().cuda().transpose(1, 2)
    seen_of = (lambda b: causal_mask(c, b, pos)) if causal else (lambda b: torch.ones(c.q[b], c.kv[b], dtype=torch.bool))
    scale = c.D ** -0.5
    if lse is None:
        lse = lse_of(c, q, scale, seen_of)
    if change is not None:
        change(q, lse)
    w = torch.rand(c.n_pages, c.Hkv, c.page, generator=g).cuda() * 0.3
    if layout != "dense":                     # heads apart, as within a larger array
        big = torch.full((c.n_pages, c.Hkv + 1, c.page + 16), 9.0, device="cuda")
        big[:, 1:, :c.page] = w
        w = big[:, 1:, :c.page]
    before = w.clone()
    p = None if pos is None else torch.tensor(pos, dtype=torch.int32, device="cuda")
    lib.tr_cache_weigh(q, lse, c.pages["k"], c.table, c.kv_len, c.q_start, causal, scale, w, fresh, c.scales["k"], p)
    ref, err = weigh(c, q, lse, scale, before, fresh, seen_of, pos)
    same = err == 0
    assert torch.equal(w[same], before[same]), "weights of slots that hold no key in question"
    share = ((w.double() - ref).abs() / err)[~same]
    print("share of the bound", float(share.max()) if share.numel() else 0.0)
    assert not share.numel() or float(share.max()) <= 1
    if layout != "dense":
        assert (big[:, 0] == 9).all() and (big[:, :, c.page:] == 9).all()
    return w


SHAPES = [
    # keys, new tokens, Hkv, query heads a K/V head, page
    ([1], [1], 1, 1, 16),
    ([5], [1], 2, 4, 16),
    ([63, 64, 65], [1, 1, 1], 2, 4, 16),
    ([255, 256, 257, 258], [1, 2, 3, 4], 1, 5, 32),
    ([300, 0, 17, 1], [1, 0, 1, 1], 2, 7, 48),
    ([1000, 3], [3, 3], 2, 8, 64),
    ([4500], [1], 1, 8, 16),
    ([2000, 10, 1999], [1, 1, 1], 2, 16, 128),
    ([5000, 33], [5, 33], 1, 4, 32),
    ([90], [90], 2, 2, 16),
    ([700, 650], [130, 257], 2, 3, 48),
    ([1500, 40, 900], [513, 1, 64], 1, 4, 16),
    ([600], [600], 2, 1, 32),
    ([400, 300, 200, 100, 50, 25, 12, 6], [40, 1, 1, 1, 1, 1, 1, 1], 1, 4, 16),
]


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", SHAPES)
def test_lengths(lib, shape, D, f8):
    kv, q, Hkv, gq, page = shape
    c = Cache(kv, q, Hkv, D, page, f8, "head" if len(kv) % 2 else "token", seed=D + len(kv))
    _run(lib, c, Hkv * gq, behind=2)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gq", [1, 5, 8])
@pytest.mark.parametrize("mixed", [False, True])
def test_many_items(lib, mixed, gq, D, f8):
    """More stretches of keys than compute units, of sequences with many rows alone and among single tokens."""
    kv = [600 + 17 * (i % 13) for i in range(40)]
    q = [70 + i % 5 if not mixed or i % 3 == 0 else i % 2 for i in range(40)]
    c = Cache(kv, q, 4 if not mixed else 8, D, 32, f8, "token" if gq == 5 else "head", seed=gq)
    _run(lib, c, c.Hkv * gq)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("kv,q,Hkv,gq", [
    ([300, 75, 1, 90, 0, 64, 65, 257, 30], [100, 1, 1, 3, 0, 1, 2, 1, 1], 2, 4),      # short keys: a mixture for few rows on average
    ([27] * 8 + [26], [1] * 8 + [23], 4, 7),
    ([900, 40, 800, 1000, 700, 650, 300, 5, 33], [500, 1, 1, 130, 1, 1, 9, 1, 17], 3, 5),   # 64 keys a workgroup for many rows
    ([3000] + [100] * 11, [200] + [1] * 11, 12, 1),                                   # 256
    ([6, 5, 4, 3, 2, 1, 1, 300], [6, 5, 4, 3, 2, 1, 1, 300], 1, 1),                   # nothing but new tokens
])
def test_a_prompt_among_few(lib, kv, q, Hkv, gq, causal, D, f8):
    c = Cache(kv, q, Hkv, D, 16, f8, "token" if gq == 4 else "head", seed=11)
    w = _run(lib, c, Hkv * gq, causal, causal, behind=3)
    assert torch.equal(w, _run(lib, c, Hkv * gq, causal, causal, behind=3))
    if causal and gq > 1:
        c.table[0, 1] = -1
        pos = [n // 2 if i % 2 else n + 3 for i, n in enumerate(kv)]
        _run(lib, c, Hkv * gq, True, True, pos, layout="apart")


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("n", [2, 77])
def test_masks_and_fresh_keys(lib, n, fresh, causal, f8):
    c = Cache([200, 1500, n], [n, n, n], 2, 128, 32, f8, "head", seed=5)
    _run(lib, c, 8, causal, fresh, layout="strided")


@pytest.mark.parametrize("n", [3, 70])
def test_positions(lib, n):
    """New tokens in front of all keys, partly, between them, behind them."""
    c = Cache([150, 2500, 64, 40, 333], [n] * 5, 2, 128, 16, False, "head", seed=6)
    for fresh in (False, True):
        _run(lib, c, 8, True, fresh, [-2, 1000 - n, 64, -1000, 330])


@pytest.mark.parametrize("n", [1, 70])
def test_entries_that_are_no_pages(lib, n):
    c = Cache([500, 3000], [n, n], 2, 128, 16, True, "token", seed=7)
    c.table[0, 3], c.table[0, 30], c.table[1, 0], c.table[1, 100], c.table[1, -1] = -1, c.n_pages, 2 ** 31 - 1, -2 ** 31, -1
    _run(lib, c, 8)


@pytest.mark.parametrize("n", [1, 5, 70])
def test_rows_that_add_nothing(lib, n):
    """Tokens whose lse is not finite, whatever their row of q holds."""
    c = Cache([500, 300], [n, n], 2, 64, 16, False, "head", seed=8)

    def change(q, lse):
        for i, x in enumerate((-math.inf, math.inf, math.nan)):
            lse[0, 2 * i, n // 2] = x
            q[0, 2 * i, n // 2] = math.nan if i % 2 else math.inf
    _run(lib, c, 8, change=change)


@pytest.mark.parametrize("n", [2, 40])
def test_masked_keys_may_hold_anything(lib, n):
    """A NaN in K of the last key, which only the last token sees and whose weights alone it reaches."""
    c = Cache([333], [n], 2, 128, 16, False, "head", seed=9)
    q = torch.randn(1, 8, n, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    seen_of = lambda b: causal_mask(c, b)   # noqa: E731
    lse = lse_of(c, q, 0.1, seen_of)
    w0 = torch.zeros(c.n_pages, 2, 16, device="cuda")
    w1 = w0.clone()
    args = (c.table, c.kv_len, c.q_start, True, 0.1)
    lib.tr_cache_weigh(q, lse, c.pages["k"], *args, w0)
    page, slot = int(c.table[0, 332 // 16]), 332 % 16
    c.pages["k"][page, :, slot] = math.nan
    lib.tr_cache_weigh(q, lse, c.pages["k"], *args, w1)
    assert w1[page, :, slot].isnan().all()
    w1[page, :, slot] = w0[page, :, slot]
    assert torch.equal(w0, w1)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [2, 40, 500])
def test_masked_keys_may_hold_anything_in_8_bits(lib, n, D):
    """A NaN among the values, and a scale that is none, of the two last keys: they reach the weights of those keys alone."""
    c = Cache([633], [n], 2, D, 16, True, "head", seed=9)
    q = torch.randn(1, 8, n, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    lse = lse_of(c, q, 0.1, lambda b: causal_mask(c, b))
    w0 = torch.zeros(c.n_pages, 2, 16, device="cuda")
    w1 = w0.clone()
    args = (c.table, c.kv_len, c.q_start, True, 0.1)
    lib.tr_cache_weigh(q, lse, c.pages["k"], *args, w0, True, c.scales["k"])
    at = [(int(c.table[0, key // 16]), key % 16) for key in (631, 632)]
    c.pages["k"].view(torch.uint8)[at[0][0], :, at[0][1], 3] = 0x7f
    c.scales["k"].view(torch.uint8)[at[1][0], :, at[1][1]] = 255
    lib.tr_cache_weigh(q, lse, c.pages["k"], *args, w1, True, c.scales["k"])
    for page, slot in at:
        assert w1[page, :, slot].isnan().all()
        w1[page, :, slot] = w0[page, :, slot]
    assert torch.equal(w0, w1)


def test_steps_add_up_to_what_a_chunk_adds(lib):
    """A prompt token by token, and at once: each key's weights over the causal softmax, whose sum over the keys is one a row."""
    n, Hq = 150, 8
    c = Cache([n], [n], 2, 128, 16, False, "head", seed=10)
    q = torch.randn(1, Hq, n, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    lse = lse_of(c, q, 0.1, lambda b: causal_mask(c, b))
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    at_once, steps = (torch.full((c.n_pages, 2, 16), 5.0, device="cuda") for _ in range(2))
    lib.tr_cache_weigh(q, lse, c.pages["k"], c.table, ints(n), ints(0, n), True, 0.1, at_once)
    for t in range(n):
        lib.tr_cache_weigh(q[:, :, t:t + 1], lse[:, :, t:t + 1], c.pages["k"], c.table, ints(t + 1), ints(0, 1), True, 0.1, steps)
    pages = c.table[0, :-(-n // 16)].long()
    a = at_once[pages].transpose(0, 1).reshape(2, -1)[:, :n].double()
    s = steps[pages].transpose(0, 1).reshape(2, -1)[:, :n].double()
    # both are sums of the same n * 4 terms, each to (128 + 16) half steps of a score that is below 64, and a few
    assert ((a - s).abs() <= 2 * 2.0 ** -24 * ((128 + 16) * 64 + 4 * n) * a).all()
    assert (a.sum(-1) - 4 * n).abs().max() <= 4 * n * 2.0 ** -24 * ((128 + 16) * 64 + 4 * n)


def test_reproducible_captured_and_on_another_stream(lib):
    c = Cache([3000, 500, 4096], [25, 1, 140], 2, 128, 16, True, "head", seed=11)
    a = _run(lib, c, 8)
    b = _run(lib, c, 8)
    assert torch.equal(a, b)
    q = torch.randn(1, 8, c.tokens, 128, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    lse = lse_of(c, q, 0.1, lambda b: causal_mask(c, b))
    w = torch.zeros(c.n_pages, 2, 16, device="cuda")
    args = (c.table, c.kv_len, c.q_start, True, 0.1)
    lib.tr_cache_weigh(q, lse, c.pages["k"], *args, w, False, c.scales["k"])
    once = w.clone()
    w.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lib.tr_cache_weigh(q, lse, c.pages["k"], *args, w, False, c.scales["k"], stream=side)
    side.synchronize()
    assert torch.equal(w, once)
    graph = torch.cuda.CUDAGraph()
    w.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lib.tr_cache_weigh(q, lse, c.pages["k"], *args, w, False, c.scales["k"])
    for _ in range(3):
        w.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, once)
