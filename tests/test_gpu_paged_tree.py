"""tr_paged_attn_tree against a 64-bit implementation, within bounds that follow from its roundings (paged_util)."""
import math
import random

import pytest
import torch

from evict_util import attention_on, packed, seen_in_tree, tree_of
from paged_util import Cache, check

pytestmark = pytest.mark.gpu


def _bits(c, seed, words, kind="tree"):
    """Bits of every sequence's tokens [n, n], and the tensor of all."""
    rng = random.Random(seed)
    sees = []
    for n in c.q:
        if kind == "tree":
            sees.append(tree_of([rng.randrange(-1, i) if i else -1 for i in range(n)]))
        else:                       # any bits at all, rows without one among them
            g = torch.Generator().manual_seed(rng.randrange(1 << 30))
            x = torch.rand(n, n, generator=g) < 0.4
            x[::3] = False
            sees.append(x)
    sees = [x[:, :32 * words] for x in sees]
    rows = [packed(x, words) for x in sees]
    return sees, torch.cat(rows).cuda() if rows else torch.zeros(0, words, dtype=torch.int32).cuda()


def _run(lib, c, Hq, words=None, pos=None, out_dtype=torch.bfloat16, workspace=True, seed=1, behind=0, kind="tree", q=None):
    g = torch.Generator().manual_seed(seed)
    if q is None:
        q = torch.randn(1, c.tokens + behind, Hq, c.D, generator=g).bfloat16().cuda().transpose(1, 2)
    words = max(1, (max(c.q) + 31) // 32) if words is None else words
    sees, tree = _bits(c, seed, words, kind)
    tree = torch.cat([tree, torch.full((behind, words), -1, dtype=torch.int32, device="cuda")])
    out = torch.full((1, c.tokens + behind, Hq, c.D), 3.5, dtype=out_dtype, device="cuda").transpose(1, 2)
    lse = torch.full((1, Hq, c.tokens + behind), 4.5, device="cuda")
    scale = c.D ** -0.5
    ws = torch.full((lib.tr_paged_attn_tree_workspace_bytes(q, c.pages["k"], c.table),), 255, dtype=torch.uint8, device="cuda") if workspace else None
    p = None if pos is None else torch.tensor(pos, dtype=torch.int32, device="cuda")
    lib.tr_paged_attn_tree(q, *c.args(), c.q_start, tree, scale, out, lse, *c.scale_args(), q_pos=p, workspace=ws)
    if behind:
        assert (out[:, :, c.tokens:] == 3.5).all() and (lse[:, :, c.tokens:] == 4.5).all()
    return q, out, lse, attention_on(c, q, scale, lambda b: seen_in_tree(c, b, sees[b], pos))


SHAPES = [
    # keys, drafts, Hkv, query heads a K/V head, page
    ([1], [1], 1, 1, 16),
    ([6], [5], 2, 4, 16),
    ([31, 33, 64], [8, 8, 8], 2, 4, 16),
    ([300, 0, 17, 9], [9, 0, 7, 1], 2, 7, 48),
    ([127, 130], [2, 30], 1, 5, 32),
    ([1000, 40], [25, 33], 2, 4, 64),
    ([4500], [8], 1, 4, 16),
    ([4500], [64], 1, 8, 16),
    ([90], [90], 2, 2, 16),
    ([2000, 700, 650], [31, 130, 257], 2, 3, 48),
    ([1500, 40, 900], [513, 1, 64], 1, 4, 16),
]


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", SHAPES)
def test_trees(lib, shape, D, f8):
    kv, q, Hkv, gq, page = shape
    c = Cache(kv, q, Hkv, D, page, f8, "head" if len(kv) % 2 else "token", seed=D + len(kv))
    for workspace in (True, False):
        _, out, lse, found = _run(lib, c, Hkv * gq, workspace=workspace, behind=2)
        print(check(found, out, lse))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n", [1, 7, 40, 100])
def test_any_bits(lib, n, f8):
    """Bits that are no tree: tokens that see later ones, and none of the drafts, not even themselves; a sequence that is nothing but drafts has rows that see no key."""
    c = Cache([n, 300 + n, 2500], [n, n, n], 2, 128, 16, f8, "head", seed=5)
    _, out, lse, found = _run(lib, c, 8, kind="any", out_dtype=torch.float32)
    check(found, out, lse)
    assert (out[:, :, 0] == 0).all() and torch.isneginf(lse[:, :, 0]).all()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kv,q,Hkv,gq", [
    ([9000], [25], 2, 4),                    # 100 rows, 36 parts
    ([9000, 40, 3000, 130], [5, 3, 20, 4], 1, 4),
    ([5000, 4999], [1, 2], 1, 1),            # a row or two
    ([6000, 700], [77, 131], 1, 5),          # two and three tiles, the last ones of few rows
    ([20000], [300], 1, 1),
])
def test_few_tiles_in_many_parts(lib, kv, q, Hkv, gq, D, f8):
    """Trees behind long texts, whose parts the waves of the fold share; also with parts that some rows, or all, see nothing of, and with an infinity in V."""
    c = Cache(kv, q, Hkv, D, 32, f8, "head", seed=len(kv) + D)
    _, out, lse, found = _run(lib, c, Hkv * gq, behind=2)
    check(found, out, lse)
    pos = [n // 3 if i % 2 == 0 else -2 for i, n in enumerate(kv)]
    _, out, lse, found = _run(lib, c, Hkv * gq, pos=pos, kind="any", out_dtype=torch.float32)
    check(found, out, lse)
    key = kv[0] - q[0]                       # the first draft
    page, slot = int(c.table[0, key // 32]), key % 32
    if f8:
        c.pages["v"].view(torch.uint8)[page, 0, slot, 7] = 127
    else:
        c.pages["v"][page, 0, slot, 7] = math.inf
    _, out, lse, found = _run(lib, c, Hkv * gq, kind="any")
    check(found, out, lse)


MANY = [
    # keys, drafts, Hkv, query heads a K/V head, page
    ([700, 30, 1500, 33, 400, 0, 64, 901] * 2, [25, 30, 25, 33, 25, 0, 64, 1] * 2, 8, 4, 32),          # 128 tiles of up to 256 rows
    ([1300, 64, 500] * 5, [64, 64, 64] * 5, 8, 4, 16),                                                # two tiles of 128 rows each
    ([200, 41, 333, 100, 40, 900] * 8, [40, 41, 33, 40, 40, 37] * 8, 12, 1, 48),                      # more tiles than units
    ([4000, 350, 80, 2222] * 10, [60, 70, 65, 75] * 10, 8, 4, 64),                                    # two and three tiles each
]


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", MANY)
def test_many_trees(lib, shape, D, f8):
    """Trees that fill the chip: one launch of smaller tiles, or of whole ones where keys are in 8 bits."""
    kv, q, Hkv, gq, page = shape
    c = Cache(kv, q, Hkv, D, page, f8, "head" if D == 64 else "token", seed=D + len(kv))
    for workspace in (True, False):
        _, out, lse, found = _run(lib, c, Hkv * gq, workspace=workspace, behind=2)
        check(found, out, lse)
    again = _run(lib, c, Hkv * gq, workspace=False, behind=2)
    assert torch.equal(out, again[1]) and torch.equal(lse, again[2])


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_many_trees_with_any_bits_positions_and_bad_values(lib, D, f8):
    kv, q, Hkv, gq, page = MANY[0]
    pos = [n // 2 if i % 3 == 0 else -5 if i % 3 == 1 else n for i, n in enumerate(kv)]
    c = Cache(kv, q, Hkv, D, page, f8, "head", seed=3)
    for at in (None, pos):
        _, out, lse, found = _run(lib, c, Hkv * gq, pos=at, kind="any", out_dtype=torch.float32)
        check(found, out, lse)
    for b in (0, 2, 4):
        key = kv[b] - q[b] + 1
        where, slot = int(c.table[b, key // page]), key % page
        if f8:
            c.pages["v"].view(torch.uint8)[where, 1, slot, 5] = 127
        else:
            c.pages["v"][where, 1, slot, 5] = math.inf
    c.table[0, 3] = -1
    c.table[10, 20] = c.n_pages + 7
    c.table[12, 0] = 1 << 30
    _, out, lse, found = _run(lib, c, Hkv * gq)
    check(found, out, lse)


def test_words_that_are_too_few_and_too_many(lib):
    """Drafts behind the last word are seen by none; words behind the last draft say nothing."""
    for n, words in ((70, 1), (70, 2), (70, 9), (20, 3)):
        c = Cache([500, 90], [n, n], 2, 64, 16, False, "head", seed=6)
        q, out, lse, found = _run(lib, c, 8, words=words, kind="any")
        check(found, out, lse)


def test_one_row_for_all_tokens(lib):
    """A tree of stride 0: every token has the same bits."""
    c = Cache([200, 90], [6, 6], 2, 128, 16, False, "head", seed=7)
    g = torch.Generator().manual_seed(3)
    q = torch.randn(1, 8, 12, 128, generator=g).bfloat16().cuda()
    tree = torch.tensor([[0b010110]], dtype=torch.int32, device="cuda").expand(12, 1)
    out, lse = torch.empty_like(q), torch.empty(1, 8, 12, device="cuda")
    lib.tr_paged_attn_tree(q, *c.args(), c.q_start, tree, 128 ** -0.5, out, lse)
    sees = torch.tensor([[0, 1, 1, 0, 1, 0]]).bool().expand(6, 6)
    check(attention_on(c, q, 128 ** -0.5, lambda b: seen_in_tree(c, b, sees)), out, lse)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n", [3, 70])
def test_positions(lib, n, f8):
    """Drafts in front of all keys, partly among them, between them (the keys behind them are nobody's), and behind them."""
    c = Cache([150, 2500, 64, 40, 333], [n] * 5, 2, 128, 16, f8, "head", seed=6)
    pos = [-2, 1000 - n, 64, -1000, 330]
    _, out, lse, found = _run(lib, c, 8, pos=pos)
    check(found, out, lse)
    assert (out[:, :, c.starts[3]:c.starts[4]] == 0).all() and torch.isneginf(lse[:, :, c.starts[3]:c.starts[4]]).all()


@pytest.mark.parametrize("n", [1, 33, 100])
def test_a_chain_is_causal(lib, n):
    """A tree without branches is what tr_paged_attn computes, to the bit where both share out the keys alike."""
    c = Cache([n, 700, 3000], [n] * 3, 2, 128, 32, False, "head", seed=8)
    words = (n + 31) // 32
    tree = torch.cat([packed(tree_of(list(range(-1, n - 1))), words)] * 3).cuda()
    q = torch.randn(1, 8, c.tokens, 128, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    o, l = torch.empty_like(q), torch.empty(1, 8, c.tokens, device="cuda")
    o2, l2 = torch.empty_like(q), torch.empty(1, 8, c.tokens, device="cuda")
    lib.tr_paged_attn_tree(q, *c.args(), c.q_start, tree, 0.1, o, l)
    lib.tr_paged_attn(q, *c.args(), c.q_start, True, 0.1, o2, l2)
    sees = tree_of(list(range(-1, n - 1)))
    found = attention_on(c, q, 0.1, lambda b: seen_in_tree(c, b, sees))
    check(found, o, l)
    check(found, o2, l2)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("n", [4, 70])
def test_bad_values_reach_the_branch_that_sees_them(lib, n, bad, f8):
    """An infinity or NaN in V of a draft: tokens below it have it, the other branches nothing of it; a NaN in K of a draft likewise."""
    c = Cache([333, 2000], [n, n], 2, 128, 16, f8, "head", seed=8)
    for b in range(2):
        key = c.kv[b] - n + 1
        page, slot = int(c.table[b, key // 16]), key % 16
        if f8:
            c.pages["v"].view(torch.uint8)[page, 1, slot, 5] = 127
        else:
            c.pages["v"][page, 1, slot, 5] = bad
    _, out, lse, found = _run(lib, c, 8)
    check(found, out, lse)
    parents_bad = out[0, 4:, :, 5].isfinite()
    assert not parents_bad.all() and parents_bad.any()


@pytest.mark.parametrize("n", [4, 70])
def test_masked_keys_may_hold_anything(lib, n):
    """K and V of drafts that a token does not see, NaN among them, reach nothing."""
    c = Cache([333], [n], 2, 128, 16, False, "head", seed=9)
    page, slot = int(c.table[0, 332 // 16]), 332 % 16      # the last draft, which only its own token sees
    c.pages["k"][page, :, slot] = float("nan")
    c.pages["v"][page, :, slot] = float("nan")
    _, out, lse, found = _run(lib, c, 8)
    assert out[:, :, :n - 1].isfinite().all() and lse[:, :, :n - 1].isfinite().all()
    assert out[:, :, n - 1].isnan().all()
    c2 = Cache([333], [n], 2, 128, 16, False, "head", seed=9)
    _, out2, lse2, found2 = _run(lib, c2, 8)
    for (rows, ref_o, ref_l, d_o, d_l) in found2:
        check([(slice(0, n - 1), ref_o[:, :, :-1], ref_l[:, :, :-1], d_o[:, :, :-1], d_l[:, :, :-1])], out, lse)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [4, 40, 70])
def test_masked_keys_may_hold_anything_in_8_bits(lib, n, D):
    """The same of 8-bit drafts whose scales are none."""
    c = Cache([333], [n], 2, D, 16, True, "head", seed=9)
    page, slot = int(c.table[0, 332 // 16]), 332 % 16
    for name in "kv":
        c.scales[name].view(torch.uint8)[page, :, slot] = 255
    _, out, lse, _ = _run(lib, c, 8)
    assert out[:, :, n - 1].isnan().all()
    _, _, _, found = _run(lib, Cache([333], [n], 2, D, 16, True, "head", seed=9), 8)
    for (rows, ref_o, ref_l, d_o, d_l) in found:
        check([(slice(0, n - 1), ref_o[:, :, :-1], ref_l[:, :, :-1], d_o[:, :, :-1], d_l[:, :, :-1])], out, lse)


@pytest.mark.parametrize("n", [3, 70])
def test_entries_that_are_no_pages(lib, n):
    c = Cache([500, 3000], [n, n], 2, 128, 16, False, "token", seed=7)
    c.table[0, 3], c.table[0, 30], c.table[1, 0], c.table[1, 100], c.table[1, -1] = -1, c.n_pages, 2 ** 31 - 1, -2 ** 31, -1
    _, out, lse, found = _run(lib, c, 8)
    check(found, out, lse)


def test_reproducible_and_captured(lib):
    c = Cache([3000, 500, 4096], [25, 1, 40], 2, 128, 16, True, "head", seed=11)
    first = _run(lib, c, 8)
    again = _run(lib, c, 8, q=first[0])
    assert torch.equal(first[1], again[1]) and torch.equal(first[2], again[2])
    q = first[0]
    sees, tree = _bits(c, 1, 2)
    out, lse = torch.zeros_like(first[1]), torch.zeros_like(first[2])
    ws = torch.empty(lib.tr_paged_attn_tree_workspace_bytes(q, c.pages["k"], c.table), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.tr_paged_attn_tree(q, *c.args(), c.q_start, tree, c.D ** -0.5, out, lse, *c.scale_args(), workspace=ws)
    for seed in (1, 2, 3):
        sees, other = _bits(c, seed, 2)
        tree.copy_(other)
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        check(attention_on(c, q, c.D ** -0.5, lambda b: seen_in_tree(c, b, sees[b])), out, lse)
        if seed == 1:
            assert torch.equal(out, first[1])
