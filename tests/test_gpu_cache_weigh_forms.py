"""tr_cache_weigh where a call's sequences have few and many rows, in each form that a launch may take (weigh_plan.h), against the 64-bit implementation and bounds of evict_util."""
import pytest
import torch

from evict_util import causal_mask, lse_of, weigh
from paged_util import Cache
from test_gpu_cache_weigh import _run

pytestmark = pytest.mark.gpu

AROUND = [33, 31, 32, 60, 1, 0, 8, 9]      # 132, 124, 128 rows of a K/V head in groups of 4: on both sides of the border between two launches; and of 32


def _widened(c, keys):
    """The same cache behind a table with room for `keys` keys."""
    more = keys // c.page - c.table.shape[1]
    c.table = torch.cat([c.table, torch.full((len(c.kv), more), -7, dtype=torch.int32, device="cuda")], 1)
    return c


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_two_launches(lib, causal, D, f8):
    """Many keys, few rows on average: sequences of more than 128 rows have a launch of their own."""
    q = AROUND + [1] * 22
    kv = [max(n, 100 + 157 * (i % 9)) for i, n in enumerate(q)]
    c = Cache(kv, q, 4, D, 32, f8, "head" if D == 64 else "token", seed=3)
    w = _run(lib, c, 16, causal, causal, behind=3)
    assert torch.equal(w, _run(lib, c, 16, causal, causal, behind=3))
    if causal:
        c.table[0, 1], c.table[3, 2] = -1, c.n_pages
        _run(lib, c, 16, True, True, [n // 2 if i % 2 else n + 3 for i, n in enumerate(kv)], layout="apart")


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("prompt", [96, 97, 98])
@pytest.mark.parametrize("room", [0, 16384])
def test_a_prompt_of_any_length(lib, room, prompt, f8):
    """112 tokens of 16 sequences are neither more nor less than 111 or 113; nor is a table wider than any sequence."""
    c = Cache([300] * 16, [prompt] + [1] * 15, 2, 128, 16, f8, "head", seed=4)
    if room:
        _widened(c, room)
    _run(lib, c, 8)


@pytest.mark.parametrize("gq", [1, 4, 7])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q", [[70, 1], [1, 200, 3], [129, 1, 1, 40], [3, 1, 1, 1, 1, 0, 150]])
def test_few_sequences(lib, q, D, gq):
    kv = [max(n, 90 + 333 * (i % 4)) for i, n in enumerate(q)]
    c = Cache(kv, q, 3, D, 16, len(q) % 2 == 1, "token" if gq == 4 else "head", seed=5)
    _run(lib, c, 3 * gq, behind=1)
    _run(lib, c, 3 * gq, False, False)


def test_replayed_with_other_lengths(lib):
    """A graph of two launches takes what its arrays hold: the prompt is another sequence's each time, and once there is none."""
    n, S, Hkv, gq = 40, 120, 4, 4
    c = _widened(Cache([700] * n, [S // n] * n, Hkv, 64, 16, True, "head", seed=6), 2048)
    g = torch.Generator().manual_seed(8)
    q = torch.randn(1, Hkv * gq, S, 64, generator=g).bfloat16().cuda()
    lse, w = torch.empty(1, Hkv * gq, S, device="cuda"), torch.rand(c.n_pages, Hkv, 16, generator=g).cuda()
    start = w.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.tr_cache_weigh(q, lse, c.pages["k"], c.table, c.kv_len, c.q_start, True, 0.125, w, True, c.scales["k"])
    for prompt in (0, 7, 39, None, 20):
        c.q = [3] * n if prompt is None else [81 if i == prompt else 1 for i in range(n)]
        c.starts = [sum(c.q[:i]) for i in range(n + 1)]
        c.q_start.copy_(torch.tensor(c.starts, dtype=torch.int32))
        seen_of = lambda b: causal_mask(c, b)   # noqa: E731
        lse.copy_(lse_of(c, q, 0.125, seen_of))
        w.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        ref, err = weigh(c, q, lse, 0.125, start, True, seen_of)
        same = err == 0
        assert torch.equal(w[same], start[same])
        assert (((w.double() - ref).abs() / err)[~same] <= 1).all()
