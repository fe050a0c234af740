"""tr_cache_select and tr_cache_keep against plain implementations: whole numbers and copies, equal to the last bit."""
import math
import random

import pytest
import torch

from evict_util import keep, select
from paged_util import Cache

pytestmark = pytest.mark.gpu


def _weights(c, seed, kind):
    g = torch.Generator().manual_seed(seed)
    shape = (c.n_pages, c.Hkv, c.page)
    x = torch.randn(shape, generator=g)
    if kind == "few":                 # many equal ones
        x = torch.randint(0, 4, shape, generator=g).float()
    elif kind == "zeros":
        x = torch.where(torch.rand(shape, generator=g) < 0.7, 0.0, x.exp())
        x = torch.where(torch.rand(shape, generator=g) < 0.5, -x * (x == 0), x)
    elif kind == "odd":               # infinities, NaN, the smallest numbers, both zeros
        pick = torch.tensor([math.inf, -math.inf, math.nan, -math.nan, 0.0, -0.0, 1e-45, -1e-45, 1e-38, 3.4e38, -3.4e38, 1.0])
        x = pick[torch.randint(0, len(pick), shape, generator=g)]
    elif kind == "near":              # differ in the last bits alone
        x = 1 + torch.randint(0, 3, shape, generator=g) * 2.0 ** -23
    return x.cuda()


def _select(lib, c, w, first, last, most):
    keys = torch.full((len(c.kv), c.Hkv, most), -5, dtype=torch.int32, device="cuda")
    count = torch.full((len(c.kv),), -5, dtype=torch.int32, device="cuda")
    lib.tr_cache_select(w, c.table, c.kv_len, first, last, keys, count)
    assert count.tolist() == [min(n, most) for n in c.kv]
    got = keys.tolist()
    for b, lists in enumerate(select(c, w.cpu(), first, last, most)):
        for h, ref in enumerate(lists):
            assert got[b][h][:len(ref)] == ref, (b, h)
            assert all(x == -5 for x in got[b][h][len(ref):])
    return keys, count


@pytest.mark.parametrize("kind", ["any", "few", "zeros", "odd", "near"])
@pytest.mark.parametrize("kv,most,first,last", [
    ([1], 1, 0, 0), ([17], 5, 0, 0), ([17], 5, 2, 3), ([17], 17, 4, 4), ([100, 0, 40, 41], 40, 4, 10), ([3000], 1, 0, 0), ([3000, 2999], 2999, 0, 0),
    ([4096, 4097, 4095], 2048, 4, 256), ([9000], 1234, 1, 0), ([500], 100, 0, 100), ([500], 0, 0, 0),
])
def test_select(lib, kv, most, first, last, kind):
    c = Cache(kv, [0] * len(kv), 2, 64, 16 if len(kv) > 1 else 48, False, seed=len(kv) + most)
    _select(lib, c, _weights(c, most, kind), first, last, most)


def test_select_of_strided_weights_and_missing_pages(lib):
    c = Cache([700, 650], [0, 0], 3, 64, 32, False, seed=3)
    big = torch.full((c.n_pages, 5, 64), math.nan, device="cuda")
    w = big[:, 1:4, 16:48]
    w.copy_(_weights(c, 1, "any"))
    c.table[0, 4], c.table[0, 9], c.table[1, 0] = -1, c.n_pages, -2 ** 31
    _select(lib, c, w, 4, 20, 300)
    _select(lib, c, w, 0, 0, 640)           # all that is there, and some of what is not


def test_select_long(lib):
    """More keys than fit any one turn of a workgroup."""
    c = Cache([70001], [0], 1, 64, 64, False, seed=4)
    g = torch.Generator().manual_seed(1)
    w = torch.randn(c.n_pages, 1, 64, generator=g).exp().cuda()
    keys, count = (torch.zeros(1, 1, 20000, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    lib.tr_cache_select(w, c.table, c.kv_len, 16, 1000, keys, count)
    x = w[c.table[0].long(), 0].flatten()[:70001].clone()
    x[:16] = math.inf
    x[-1000:] = math.inf
    ref = x.sort(descending=True, stable=True).indices[:20000].sort().values
    assert torch.equal(keys[0, 0].long(), ref) and count.tolist() == [20000]


@pytest.mark.parametrize("zeros", [0.0, 0.6])
@pytest.mark.parametrize("kv,most,table", [
    ([32768], 5000, 0), ([32769], 32768, 0), ([32800, 36864, 36865, 17], 20000, 0), ([65536, 65535, 0, 40000], 33000, 0), ([65537, 98304], 3, 0),
    ([5000, 32768, 30001], 2222, 40000),               # a table with room for more
    ([12289, 300, 12288] * 44, 6000, 0),               # more rows than compute units
])
def test_select_where_ranks_are_held(lib, kv, most, table, zeros):
    """Rows that LDS holds, that take registers too, and that are held nowhere from some key on; equal weights, and pages that are none."""
    c = Cache(kv, [0] * len(kv), 2, 64, 16, False, seed=6)
    g = torch.Generator().manual_seed(len(kv))
    w = torch.rand(c.n_pages, 2, 16, generator=g)
    w[torch.rand(w.shape, generator=g) < zeros] = 0
    w = (w * 500).round().div(500).cuda() if len(kv) % 2 else w.cuda()
    if table:
        c.table = torch.cat([c.table, torch.zeros(len(kv), table // 16 - c.table.shape[1], dtype=torch.int32, device="cuda")], 1)
    c.table[0, 2] = -1
    keys, count = torch.full((len(kv), 2, most), -7, dtype=torch.int32, device="cuda"), torch.zeros(len(kv), dtype=torch.int32, device="cuda")
    first, last = min(4, most // 2), min(100, most // 2)
    lib.tr_cache_select(w, c.table, c.kv_len, first, last, keys, count)
    assert count.tolist() == [min(n, most) for n in kv]
    for b, n in enumerate(kv):
        page = c.table[b].long().repeat_interleave(16)[:n]
        for h in range(2):
            x = torch.where(page >= 0, w[page.clamp(min=0), h, torch.arange(n, device="cuda") % 16], -1.0)
            x[:first] = math.inf
            x[n - min(last, n):] = math.inf
            m = min(n, most)
            ref = x.sort(descending=True, stable=True).indices[:m].sort().values
            assert torch.equal(keys[b, h, :m].long(), ref) and (keys[b, h, m:] == -7).all()


def _tensors(c, weights):
    t = {}
    for name in "kv":
        t[name] = c.pages[name].view(torch.uint8) if c.f8 else c.pages[name].view(torch.int16)
        if c.f8:
            t[name + "s"] = c.scales[name].view(torch.uint8)
    if weights is not None:
        t["w"] = weights
    return t


def _keep(lib, c, keys, count, start=None, weights=True):
    w = torch.rand(c.n_pages, c.Hkv, c.page, device="cuda") if weights else None
    cpu = {k: t.cpu() for k, t in _tensors(c, w).items()}
    ref = keep(c, cpu, keys, count, start)
    most = max([1] + [len(x) for s in keys for x in s])
    filled = [[x + [-1] * (most - len(x)) for x in s] for s in keys]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    lib.tr_cache_keep(c.pages["k"], c.pages["v"], c.table, c.kv_len, ints(filled), ints(count), None if start is None else ints(start), *c.scale_args(), w)
    for k, t in _tensors(c, w).items():
        assert torch.equal(t.cpu(), ref[k]), k


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("kv", [[1], [40], [300, 0, 299, 33], [2500, 1200], [64] * 40])
def test_keep(lib, kv, layout, D, f8):
    rng = random.Random(len(kv) + D)
    c = Cache(kv, [0] * len(kv), 4 if len(kv) > 20 else 2, D, 16, f8, layout, seed=5)
    keys = [[sorted(rng.sample(range(n), n * (h + 2) // (h + 4))) for h in range(c.Hkv)] for n in kv]
    n = [min(len(x) for x in s) for s in keys]
    _keep(lib, c, [[x[:n[b]] for x in s] for b, s in enumerate(keys)], n, weights=len(kv) != 2)


@pytest.mark.parametrize("f8", [False, True])
def test_keep_paths(lib, f8):
    """Accepted paths of drafts, one list for all heads: none of them, the first ones, some, all."""
    c = Cache([100, 50, 30, 77], [9] * 4, 2, 128, 16, f8, "token", seed=6)
    start = [n - 9 for n in c.kv]
    paths = [[], [0, 1, 2], [1, 4, 5, 8], list(range(9))]
    _keep(lib, c, [[[s + j for j in p]] for s, p in zip(start, paths)], [len(p) for p in paths], start)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seqs", [1, 64])
def test_keep_long_lists(lib, seqs, D, f8):
    """Lists that take several turns of a workgroup, whole rows and pieces of them."""
    kv, n, H = 3100 + 16 * (seqs == 1) * 400, 2900, 2
    c = Cache([kv] * seqs, [0] * seqs, H, D, 16, f8, "token" if D == 64 else "head", seed=10, poison=False)
    g = torch.Generator().manual_seed(seqs)
    keys = torch.rand(seqs, H, kv, generator=g).topk(n).indices.sort(-1).values
    w = torch.rand(c.n_pages, H, 16, generator=g).cuda()
    head = torch.arange(H)[None, :, None]
    place = lambda i: (c.table.cpu().long()[torch.arange(seqs)[:, None, None], i // 16], head, i % 16)   # noqa: E731
    ref = {}
    for k, t in _tensors(c, w).items():
        t = t.cpu()
        ref[k] = t.clone()
        ref[k][place(torch.arange(n).expand(seqs, H, n))] = t[place(keys)]
    lib.tr_cache_keep(c.pages["k"], c.pages["v"], c.table, c.kv_len, keys.to(torch.int32).cuda(), torch.full((seqs,), n, dtype=torch.int32, device="cuda"), None, *c.scale_args(), w)
    for k, t in _tensors(c, w).items():
        assert torch.equal(t.cpu(), ref[k]), k


def test_keep_skips_what_it_cannot_do(lib):
    """Entries beyond the keys, negative, that would move up, or that come from or go to no page; counts out of range."""
    c = Cache([100, 100, 100, 100], [0] * 4, 2, 64, 16, True, "head", seed=7)
    c.table[3, 1], c.table[3, 4] = -1, c.n_pages
    keys = [[[0, 5, 99, 100, 200, 2 ** 31 - 1], [-1, 2, 3, 50, 60, 2 ** 30]], [[1, 2, 3, 4, 5, 6]] * 2, [[3, 4, 5, 6, 7, 8]] * 2, [[i for i in range(0, 100, 2)]] * 2]
    keys = [[x + list(range(90, 90 + 50 - len(x))) if len(x) < 50 else x for x in s] for s in keys]
    _keep(lib, c, keys, [6, -3, 2 ** 31 - 1, 50], [0, 0, 0, 0])
    _keep(lib, c, keys, [6, 6, 6, 50], [-3, 3, -2 ** 31, 2 ** 31 - 1])


def test_keep_strided_and_side_by_side(lib):
    """K and V as the two halves of each row of one array, weights in a larger array."""
    c = Cache([400], [0], 2, 64, 16, False, "head", seed=8)
    both = torch.randn(c.n_pages, 2, 16, 128, device="cuda").bfloat16()
    c.pages["k"], c.pages["v"] = both[..., :64], both[..., 64:]
    keys = [[list(range(0, 400, 3)), list(range(100, 234))]]
    _keep(lib, c, keys, [134])


def test_captured_and_replayed_on_new_lists(lib):
    c = Cache([500, 300], [0, 0], 2, 128, 16, True, "head", seed=9)
    w = torch.rand(c.n_pages, 2, 16, device="cuda")
    keys, count = torch.zeros(2, 2, 200, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    first = {k: t.clone() for k, t in _tensors(c, w).items()}
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lib.tr_cache_select(w, c.table, c.kv_len, 4, 20, keys, count)
        lib.tr_cache_keep(c.pages["k"], c.pages["v"], c.table, c.kv_len, keys, count, None, *c.scale_args(), w)
    for seed in range(3):
        for k, t in _tensors(c, w).items():
            t.copy_(first[k])
        w.copy_(torch.rand(c.n_pages, 2, 16, generator=torch.Generator().manual_seed(seed)))
        before = {k: t.cpu() for k, t in _tensors(c, w).items()}
        lists = select(c, before["w"], 4, 20, 200)
        graph.replay()
        torch.cuda.synchronize()
        ref = keep(c, before, lists, [200, 200], None)
        for k, t in _tensors(c, w).items():
            assert torch.equal(t.cpu(), ref[k]), k
