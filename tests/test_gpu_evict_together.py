"""Trees of drafted tokens, weights of keys, selection and moving as a server uses them: one after the other, with the cache's other operators, captured, on streams, past 32 bits."""
import math
import random

import pytest
import torch

from evict_util import attention_on, causal_mask, keep, lse_of, packed, seen_in_tree, select, tree_of, weigh
from paged_util import F32_STEP, Cache, attention, check

pytestmark = pytest.mark.gpu


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _tokens(n, H, D, seed):
    return torch.randn(1, n, H, D, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda().transpose(1, 2)


def _tensors(c, w):
    t = {x: c.pages[x].view(torch.uint8) if c.f8 else c.pages[x].view(torch.int16) for x in "kv"}
    if c.f8:
        t.update({x + "s": c.scales[x].view(torch.uint8) for x in "kv"})
    return dict(t, w=w)


def _near(w, ref, err):
    assert ((w.double() - ref).abs() <= err).all()


class Server:
    """One layer's cache of a few sequences, its weights, and the oracle's idea of both."""

    def __init__(self, lib, room, Hkv, gq, D, f8, seed):
        self.lib, self.c = lib, Cache([room] * 3, [1] * 3, Hkv, D, 16, f8, "head", seed=seed)
        self.Hq, self.seed = Hkv * gq, seed
        self.c.kv = [0] * 3
        self.w = torch.full((self.c.n_pages, Hkv, 16), math.nan, device="cuda")     # what a page that was just given out may hold

    def lengths(self, kv, new):
        c = self.c
        c.kv, c.q = list(kv), list(new)
        c.kv_len.copy_(_ints(*kv))
        c.starts = [0]
        for n in new:
            c.starts.append(c.starts[-1] + n)
        c.tokens, c.q_start = c.starts[-1], _ints(*c.starts)

    def step(self, new):
        """New tokens: written, attended, weighed."""
        lib, c = self.lib, self.c
        self.lengths([a + b for a, b in zip(c.kv, new)], new)
        self.seed += 1
        q, k, v = _tokens(c.tokens, self.Hq, c.D, self.seed), _tokens(c.tokens, c.Hkv, c.D, self.seed + 100), _tokens(c.tokens, c.Hkv, c.D, self.seed + 200)
        out, lse = torch.zeros_like(q), torch.zeros(1, self.Hq, c.tokens, device="cuda")
        lib.tr_cache_write(k, v, *c.args(), c.q_start, *c.scale_args())
        lib.tr_paged_attn(q, *c.args(), c.q_start, True, c.D ** -0.5, out, lse, *c.scale_args())
        check(attention(c, q, c.D ** -0.5, True), out, lse)
        before = self.w.clone()
        lib.tr_cache_weigh(q, lse, c.pages["k"], c.table, c.kv_len, c.q_start, True, c.D ** -0.5, self.w, True, c.scales["k"])
        ref, err = weigh(c, q, lse, c.D ** -0.5, before.nan_to_num(0), True, lambda b: causal_mask(c, b))
        touched = ~torch.isnan(self.w)
        _near(self.w[touched], ref[touched], err[touched])
        return q, out, lse

    def live(self, b):
        """Weights of a sequence's keys [Hkv, keys]."""
        n = self.c.kv[b]
        return self.w[self.c.table[b, :-(-n // 16)].long()].transpose(0, 1).reshape(self.c.Hkv, -1)[:, :n] if n else self.w.new_zeros(self.c.Hkv, 0)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_a_server_that_evicts(lib, D, f8):
    s = Server(lib, 700, 2, 4, D, f8, 20)
    c = s.c
    seen = [0, 0, 0]
    for new in ([300, 500, 17], [1, 1, 1], [1, 0, 1], [3, 1, 40]):
        s.step(new)
        seen = [a + b for a, b in zip(seen, new)]
        for b in range(3):        # no NaN of a fresh page is left, and every token's weights add up to one a query head
            assert s.live(b).isfinite().all()
            assert (s.live(b).sum(-1) - 4 * seen[b]).abs().max() <= 4 * seen[b] * 2.0 ** -24 * ((D + 16) * 64 + 4 * 600)
    for _ in range(2):
        keys, count = torch.zeros(3, 2, 200, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
        w = s.w.nan_to_num(0)
        lib.tr_cache_select(w, c.table, c.kv_len, 4, 50, keys, count)
        lists = select(c, w.cpu(), 4, 50, 200)
        n = [min(x, 200) for x in c.kv]
        assert count.tolist() == n and all(keys[b, h, :n[b]].tolist() == lists[b][h] for b in range(3) for h in range(2))
        s.w.copy_(w)
        ref = keep(c, {k: t.cpu() for k, t in _tensors(c, s.w).items()}, lists, n, None)
        lib.tr_cache_keep(*c.args(), keys, count, None, *c.scale_args(), s.w)
        for k, t in _tensors(c, s.w).items():
            assert torch.equal(t.cpu(), ref[k]), k
        s.lengths(n, [0, 0, 0])
        for new in ([1, 1, 1], [20, 1, 1]):        # and on, on what is left
            s.step(new)


@pytest.mark.parametrize("f8", [False, True])
def test_drafts_verified_and_accepted(lib, f8):
    """Trees of drafts written behind the texts, attended at once; an accepted path is moved together and reads like tokens that came one by one."""
    D, H, gq, n = 128, 2, 4, 13
    rng = random.Random(3)
    c = Cache([413, 33, 1000], [n] * 3, H, D, 16, f8, "token", seed=30)
    parents = [[rng.randrange(-1, i) if i else -1 for i in range(n)] for _ in range(3)]
    sees = [tree_of(p) for p in parents]
    q, k, v = _tokens(3 * n, H * gq, D, 31), _tokens(3 * n, H, D, 32), _tokens(3 * n, H, D, 33)
    out, lse = torch.zeros_like(q), torch.zeros(1, H * gq, 3 * n, device="cuda")
    lib.tr_cache_write(k, v, *c.args(), c.q_start, *c.scale_args())
    lib.tr_paged_attn_tree(q, *c.args(), c.q_start, torch.cat([packed(x, 1) for x in sees]).cuda(), D ** -0.5, out, lse, *c.scale_args())
    check(attention_on(c, q, D ** -0.5, lambda b: seen_in_tree(c, b, sees[b])), out, lse)
    paths = []
    for b in range(3):
        leaf = max(range(n), key=lambda i: int(sees[b][i].sum()))
        paths.append([j for j in range(n) if sees[b][leaf, j]])
    start = [x - n for x in c.kv]
    w = torch.rand(c.n_pages, H, 16, device="cuda")
    most = max(map(len, paths))
    keys = _ints(*[x for b, p in enumerate(paths) for x in [start[b] + j for j in p] + [0] * (most - len(p))]).view(3, 1, most)
    ref = keep(c, {x: t.cpu() for x, t in _tensors(c, w).items()}, [[[start[b] + j for j in p]] for b, p in enumerate(paths)], [len(p) for p in paths], start)
    lib.tr_cache_keep(*c.args(), keys, _ints(*map(len, paths)), _ints(*start), *c.scale_args(), w)
    for x, t in _tensors(c, w).items():
        assert torch.equal(t.cpu(), ref[x]), x
    # the accepted tokens alone, causally: what the tree gave them
    rows = torch.tensor([b * n + j for b, p in enumerate(paths) for j in p], device="cuda")
    c.kv, c.q = [s + len(p) for s, p in zip(start, paths)], [len(p) for p in paths]
    c.starts = [0, len(paths[0]), len(paths[0]) + len(paths[1]), len(rows)]
    c.kv_len, c.q_start, c.tokens = _ints(*c.kv), _ints(*c.starts), len(rows)
    q2 = q[:, :, rows]
    out2, lse2 = torch.zeros_like(q2), torch.zeros(1, H * gq, len(rows), device="cuda")
    lib.tr_paged_attn(q2, *c.args(), c.q_start, True, D ** -0.5, out2, lse2, *c.scale_args())
    found = attention(c, q2, D ** -0.5, True)
    check(found, out2, lse2)
    check(found, out[:, :, rows], lse[:, :, rows])
    # and weighed, by the lse of either
    weights = torch.zeros(c.n_pages, H, 16, device="cuda")
    lib.tr_cache_weigh(q2, lse[:, :, rows].contiguous(), c.pages["k"], c.table, c.kv_len, c.q_start, True, D ** -0.5, weights, True, c.scales["k"])
    _near(weights, *weigh(c, q2, lse[:, :, rows], D ** -0.5, torch.zeros_like(weights), True, lambda b: causal_mask(c, b)))


def test_parts_of_a_cache_on_two_devices(lib):
    """Each device attends to the keys that it holds and weighs them by the merged lse: all weights together are one a row and head."""
    D, H, gq, n, kv = 128, 2, 4, 9, 900
    a, b = Cache([500], [n], H, D, 16, False, "head", seed=40), Cache([400], [n], H, D, 32, False, "token", seed=41)
    q = _tokens(n, H * gq, D, 42)
    pos = [kv - n, kv - n - 500]                     # of the first new token, in each device's keys: the new ones are the second's last
    acc_o, acc_l = torch.zeros(1, H * gq, n, D, device="cuda"), torch.full((1, H * gq, n), -math.inf, device="cuda")
    for c, p in zip((a, b), pos):
        o, l = torch.zeros(1, H * gq, n, D, device="cuda"), torch.zeros(1, H * gq, n, device="cuda")
        lib.tr_paged_attn(q, *c.args(), c.q_start, True, D ** -0.5, o, l, q_pos=_ints(p))
        lib.tr_merge(acc_o, acc_l, o, l)
    total = 0.0
    for c, p in zip((a, b), pos):
        w = torch.zeros(c.n_pages, H, c.page, device="cuda")
        lib.tr_cache_weigh(q, acc_l, c.pages["k"], c.table, c.kv_len, c.q_start, True, D ** -0.5, w, True, q_pos=_ints(p))
        _near(w, *weigh(c, q, acc_l, D ** -0.5, torch.zeros_like(w), True, lambda _: causal_mask(c, 0, [p]), [p]))
        total = total + w.double().sum((0, 2))
    assert (total - gq * n).abs().max() <= gq * n * F32_STEP * ((D + 16) * 64 + 4 * kv)


@pytest.mark.parametrize("f8", [False, True])
def test_hundreds_of_sequences(lib, f8):
    rng = random.Random(5)
    n = 300
    kv = [rng.choice((0, 1, 15, 16, 17, 40, 64, 65, 200, 300)) for _ in range(n)]
    for new in ([min(x, 1) for x in kv], [min(x, 30 if i % 9 == 0 else i % 3) for i, x in enumerate(kv)]):
        c = Cache(kv, new, 2, 64, 16, f8, "head", seed=50)
        q = _tokens(c.tokens, 8, 64, 51)
        lse = lse_of(c, q, 0.125, lambda b: causal_mask(c, b))
        w = torch.rand(c.n_pages, 2, 16, generator=torch.Generator().manual_seed(1)).cuda()
        ref, err = weigh(c, q, lse, 0.125, w, True, lambda b: causal_mask(c, b))
        lib.tr_cache_weigh(q, lse, c.pages["k"], c.table, c.kv_len, c.q_start, True, 0.125, w, True, c.scales["k"])
        _near(w, ref, err)
        sees = [tree_of([rng.randrange(-1, i) if i else -1 for i in range(x)]) for x in new]
        out, l = torch.zeros_like(q), torch.zeros(1, 8, c.tokens, device="cuda")
        tree = torch.cat([packed(x, 1) for x in sees if len(x)]).cuda()
        lib.tr_paged_attn_tree(q, *c.args(), c.q_start, tree, 0.125, out, l, *c.scale_args())
        check(attention_on(c, q, 0.125, lambda b: seen_in_tree(c, b, sees[b])), out, l)
    keys, count = torch.zeros(n, 2, 50, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    lib.tr_cache_select(w, c.table, c.kv_len, 2, 10, keys, count)
    lists = select(c, w.cpu(), 2, 10, 50)
    assert all(keys[b, h, :len(x)].tolist() == x for b in range(n) for h, x in enumerate(lists[b]))
    ref = keep(c, {x: t.cpu() for x, t in _tensors(c, w).items()}, lists, [min(x, 50) for x in kv], None)
    lib.tr_cache_keep(*c.args(), keys, count, None, *c.scale_args(), w)
    for x, t in _tensors(c, w).items():
        assert torch.equal(t.cpu(), ref[x]), x


def test_a_whole_step_captured(lib):
    """Drafts, their attention, weights, selection and moving in one graph, replayed on other lengths with eager work between."""
    D, H, n = 128, 2, 8
    c = Cache([600, 300], [n, n], H, D, 16, True, "head", seed=60, poison=False)
    q, k, v = _tokens(2 * n, 8, D, 61), _tokens(2 * n, H, D, 62), _tokens(2 * n, H, D, 63)
    sees = tree_of([-1, 0, 0, 1, 1, 2, 3, 3])
    tree = torch.cat([packed(sees, 1)] * 2).cuda()
    out, lse = torch.zeros_like(q), torch.zeros(1, 8, 2 * n, device="cuda")
    w = torch.zeros(c.n_pages, H, 16, device="cuda")
    keys, count = torch.zeros(2, H, 150, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ws = torch.empty(lib.tr_paged_attn_tree_workspace_bytes(q, c.pages["k"], c.table), dtype=torch.uint8, device="cuda")
    first = {x: t.clone() for x, t in _tensors(c, w).items()}

    def step():
        lib.tr_cache_write(k, v, *c.args(), c.q_start, *c.scale_args())
        lib.tr_paged_attn_tree(q, *c.args(), c.q_start, tree, D ** -0.5, out, lse, *c.scale_args(), workspace=ws)
        lib.tr_cache_weigh(q, lse, c.pages["k"], c.table, c.kv_len, c.q_start, True, D ** -0.5, w, False, c.scales["k"])
        lib.tr_cache_select(w, c.table, c.kv_len, 4, 16, keys, count)
        lib.tr_cache_keep(*c.args(), keys, count, None, *c.scale_args(), w)

    def state():
        return [x.clone() for x in (out, lse, keys, count, *_tensors(c, w).values())]

    def restart(kv):
        for x, t in _tensors(c, w).items():
            t.copy_(first[x])
        c.kv_len.copy_(_ints(*kv))
        for x in (out, lse, keys, count):
            x.zero_()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for kv in ([600, 300], [n, 299], [150, 151], [599, n]):
        restart(kv)
        step()
        torch.cuda.synchronize()
        eager = state()
        restart(kv)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, state()))


def test_calls_on_several_streams_at_once(lib):
    caches = [Cache([3000, 50], [1, 4], 2, 128, 16, i % 2 == 0, "head", seed=70 + i) for i in range(3)] + [Cache([700], [200], 1, 128, 16, False, "head", seed=79)]
    qs = [_tokens(c.tokens, 4 * c.Hkv, 128, 80 + i) for i, c in enumerate(caches)]
    lses = [lse_of(c, q, 0.1, lambda b: causal_mask(c, b)) for c, q in zip(caches, qs)]
    ws = [torch.zeros(c.n_pages, c.Hkv, 16, device="cuda") for c in caches]
    trees = [torch.cat([packed(tree_of([-1] * n), 7) for n in c.q]).cuda() for c in caches]
    outs = [(torch.zeros_like(q), torch.zeros(1, q.shape[1], q.shape[2], device="cuda")) for q in qs]
    streams = [torch.cuda.Stream() for _ in caches]
    spaces = [torch.empty(lib.tr_paged_attn_tree_workspace_bytes(q, c.pages["k"], c.table), dtype=torch.uint8, device="cuda") for c, q in zip(caches, qs)]
    torch.cuda.synchronize()
    for _ in range(4):
        for c, q, l, w, t, (o, l2), s, space in zip(caches, qs, lses, ws, trees, outs, streams, spaces):
            lib.tr_cache_weigh(q, l, c.pages["k"], c.table, c.kv_len, c.q_start, True, 0.1, w, False, c.scales["k"], stream=s)
            lib.tr_paged_attn_tree(q, *c.args(), c.q_start, t, 0.1, o, l2, *c.scale_args(), workspace=space, stream=s)
    torch.cuda.synchronize()
    for c, q, l, w, (o, l2) in zip(caches, qs, lses, ws, outs):
        once, err = weigh(c, q, l, 0.1, torch.zeros_like(w), False, lambda b: causal_mask(c, b))
        assert ((w.double() - 4 * once).abs() <= 4 * err + 8 * F32_STEP * once).all()
        check(attention_on(c, q, 0.1, lambda b: seen_in_tree(c, b, tree_of([-1] * c.q[b]))), o, l2)


def test_pages_past_32_bits(lib):
    """Pages more than 2^31 and more than 2^32 bytes from the first: weighed, chosen from, moved together."""
    page, H, D = 256, 8, 128
    n_pages = (9 << 29) // (page * H * D * 2) + 4          # 4.5 GiB of K, as much of V
    c = Cache([600], [20], H, D, page, False, "head", seed=71, poison=False)
    big = {x: torch.zeros(n_pages, H, page, D, dtype=torch.bfloat16, device="cuda") for x in "kv"}
    to = [n_pages - 1, 0, n_pages // 2 + 1]
    for i, p in enumerate(c.table[0].tolist()):
        for x in "kv":
            big[x][to[i]] = c.pages[x][p]
    c.table, c.pages, c.n_pages = _ints(*to).unsqueeze(0), big, n_pages
    q = _tokens(20, 16, D, 72)
    lse = lse_of(c, q, 0.1, lambda b: causal_mask(c, b))
    for rows in (20, 1):                                   # many rows and few
        c.q, c.starts, c.tokens, c.q_start = [rows], [0, rows], rows, _ints(0, rows)
        w = torch.zeros(n_pages, H, page, device="cuda")
        some, some_lse = q[:, :, 20 - rows:], lse[:, :, 20 - rows:]
        lib.tr_cache_weigh(some, some_lse, c.pages["k"], c.table, c.kv_len, c.q_start, True, 0.1, w)
        _near(w, *weigh(c, some, some_lse, 0.1, torch.zeros_like(w), True, lambda b: causal_mask(c, b)))
    keys, count = torch.zeros(1, H, 300, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.tr_cache_select(w, c.table, c.kv_len, 4, 30, keys, count)
    got = keys[0].tolist()
    assert got == select(c, w.cpu(), 4, 30, 300)[0]
    dense = lambda x: big[x][torch.tensor(to, device="cuda")].transpose(0, 1).reshape(H, -1, D)   # noqa: E731
    want = {x: torch.stack([dense(x)[h, torch.tensor(got[h], device="cuda")] for h in range(H)]) for x in "kv"}
    tree_out, tree_lse = torch.zeros(1, 16, 1, D, device="cuda"), torch.zeros(1, 16, 1, device="cuda")
    lib.tr_paged_attn_tree(q[:, :, :1], *c.args(), _ints(0, 1), _ints(1).view(1, 1), 0.1, tree_out, tree_lse)
    check(attention_on(c, q[:, :, :1], 0.1, lambda b: torch.ones(1, 600, dtype=torch.bool)), tree_out, tree_lse)
    lib.tr_cache_keep(*c.args(), keys, count, weights=w)
    for x in "kv":
        assert torch.equal(dense(x)[:, :300], want[x])


@pytest.mark.parametrize("gq", [17, 33, 40, 100])
@pytest.mark.parametrize("rows", ["few", "many", "long"])
def test_wide_groups(lib, gq, rows):
    """More query heads a K/V head than a tile of rows has rows, or a number that divides none."""
    kv, q = {"few": ([70, 300], [1, 0]), "many": ([70, 300, 1000], [3, 9, 2]), "long": ([400] * 110, [2] * 110)}[rows]
    c = Cache(kv, q, 1, 64, 16, rows == "many", "head", seed=gq)
    x = _tokens(c.tokens, gq, 64, 1)
    lse = lse_of(c, x, 0.125, lambda b: causal_mask(c, b))
    w = torch.rand(c.n_pages, 1, 16, generator=torch.Generator().manual_seed(1)).cuda()
    ref, err = weigh(c, x, lse, 0.125, w, True, lambda b: causal_mask(c, b))
    lib.tr_cache_weigh(x, lse, c.pages["k"], c.table, c.kv_len, c.q_start, True, 0.125, w, True, c.scales["k"])
    _near(w, ref, err)
    if rows != "long":
        sees = [tree_of([-1] * n) for n in q]
        out, l = torch.zeros_like(x), torch.zeros(1, gq, c.tokens, device="cuda")
        lib.tr_paged_attn_tree(x, *c.args(), c.q_start, torch.cat([packed(s, 1) for s in sees if len(s)]).cuda(), 0.125, out, l, *c.scale_args())
        check(attention_on(c, x, 0.125, lambda b: seen_in_tree(c, b, sees[b])), out, l)


def test_more_lists_than_a_grid_has_rows(lib):
    """70000 sequences of one page each: chosen from and moved."""
    n, D = 70000, 64
    g = torch.Generator().manual_seed(2)
    table = torch.randperm(n, generator=g).to(torch.int32).cuda().unsqueeze(1)
    kv_len = torch.randint(0, 17, (n,), generator=g).to(torch.int32).cuda()
    w = torch.rand(n, 1, 16, generator=g).cuda()
    k = torch.randint(-9, 9, (n, 1, 16, D), generator=g).bfloat16().cuda()
    v = k + 1
    keys, count = torch.full((n, 1, 5), -1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    lib.tr_cache_select(w, table, kv_len, 1, 1, keys, count)
    slots = torch.arange(16, device="cuda")
    at = table[:, 0].long()
    rank = w[at, 0].double()
    rank = torch.where((slots < 1) | (slots == kv_len[:, None] - 1), 2.0, rank)
    rank = torch.where(slots < kv_len[:, None], rank, -1.0)
    best = rank.sort(dim=-1, descending=True, stable=True).indices[:, :5]
    there = torch.arange(5, device="cuda") < kv_len.clamp(max=5)[:, None]
    best = torch.where(there, best, 99).sort(-1).values
    assert torch.equal(count, kv_len.clamp(max=5)) and torch.equal(keys[:, 0].long(), torch.where(there, best, -1))
    want_k, want_w = k.clone(), w.clone()
    seq, i = there.nonzero(as_tuple=True)
    want_k[at[seq], 0, i] = k[at[seq], 0, best[seq, i]]
    want_w[at[seq], 0, i] = w[at[seq], 0, best[seq, i]]
    lib.tr_cache_keep(k, v, table, kv_len, keys, count, weights=w)
    assert torch.equal(k, want_k) and torch.equal(v, want_k + 1) and torch.equal(w, want_w)


def test_refusals_in_python(lib):
    c = Cache([100], [2], 2, 64, 16, False, "head", seed=90)
    q, lse = _tokens(2, 8, 64, 91), torch.zeros(1, 8, 2, device="cuda")
    w = torch.zeros(c.n_pages, 2, 16, device="cuda")
    out = torch.zeros_like(q)
    with pytest.raises(lib.TokenRingError, match="TR_ERR_SHAPE"):
        lib.tr_paged_attn_tree(q, *c.args(), c.q_start, torch.zeros(3, 1, dtype=torch.int32, device="cuda"), 0.1, out, lse)
    with pytest.raises(TypeError, match="int32"):
        lib.tr_paged_attn_tree(q, *c.args(), c.q_start, torch.zeros(2, 1, dtype=torch.int64, device="cuda"), 0.1, out, lse)
    with pytest.raises(ValueError, match="dimension"):
        lib.tr_paged_attn_tree(q, *c.args(), c.q_start, torch.zeros(2, dtype=torch.int32, device="cuda"), 0.1, out, lse)
    with pytest.raises(lib.TokenRingError, match="TR_ERR_DTYPE"):
        lib.tr_cache_weigh(q, lse, c.pages["k"], c.table, c.kv_len, c.q_start, True, 0.1, w.bfloat16())
    with pytest.raises(lib.TokenRingError, match="TR_ERR_UNSUPPORTED"):
        lib.tr_cache_weigh(q, lse, c.pages["k"], c.table, c.kv_len, c.q_start, True, 0.0, w)
    with pytest.raises(ValueError, match="different devices"):
        lib.tr_cache_weigh(q, lse.cpu(), c.pages["k"], c.table, c.kv_len, c.q_start, True, 0.1, w)
    keys, count = torch.zeros(1, 2, 10, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(lib.TokenRingError, match="TR_ERR_SHAPE"):
        lib.tr_cache_select(w, c.table, c.kv_len, 6, 5, keys, count)
    with pytest.raises(ValueError, match="list for each"):
        lib.tr_cache_select(w, c.table, c.kv_len, 0, 0, keys.expand(2, 2, 10), count)
    with pytest.raises(lib.TokenRingError, match="TR_ERR_STRIDE"):
        lib.tr_cache_select(w, c.table, c.kv_len, 0, 0, keys[:, :1].expand(1, 2, 10), count)
    with pytest.raises(TypeError, match="int32"):
        lib.tr_cache_keep(*c.args(), keys.float(), count)
    with pytest.raises(ValueError, match="elements"):
        lib.tr_cache_keep(*c.args(), keys, count, torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(lib.TokenRingError, match="TR_ERR_SHAPE"):
        lib.tr_cache_keep(*c.args(), torch.zeros(1, 3, 10, dtype=torch.int32, device="cuda"), count)
