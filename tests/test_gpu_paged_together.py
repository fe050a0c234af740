"""The operators on a paged cache as a program uses them: a prompt in chunks and tokens one by one, written and attended; a cache that two devices share, folded with
the Update; a cache read back for block steps; captured and replayed; several streams; and the scratch of one launch for several calls."""
import pytest
import torch

from paged_util import BF16_STEP, Cache, attention, check

pytestmark = pytest.mark.gpu


def _tokens(n, H, D, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(1, n, H, D, generator=g).bfloat16().cuda().transpose(1, 2)


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Call:
    """tr_paged_attn on a cache with results of its own."""

    def __init__(self, lib, c, q, causal=True, pos=None, dtype=torch.bfloat16, workspace=None, stream=None):
        self.out = torch.zeros(1, q.shape[1], q.shape[2], c.D, dtype=dtype, device="cuda")
        self.lse = torch.zeros(1, q.shape[1], q.shape[2], device="cuda")
        if workspace is None:
            workspace = torch.empty(lib.tr_paged_attn_workspace_bytes(q, c.pages["k"], c.table), dtype=torch.uint8, device="cuda")
        self.run = lambda: lib.tr_paged_attn(q, *c.args(), c.q_start, causal, c.D ** -0.5, self.out, self.lse, *c.scale_args(), q_pos=pos, workspace=workspace, stream=stream)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_prompt_in_chunks_then_tokens(lib, D, f8):
    """Every step's keys are written, then attended with all before them: as one causal attention over what the cache holds."""
    total, Hkv, Hq = 333, 2, 8
    c = Cache([total], [total], Hkv, D, 16, f8, "token", seed=31)
    q, k, v = _tokens(total, Hq, D, 32), _tokens(total, Hkv, D, 33), _tokens(total, Hkv, D, 34)
    out, lse = torch.zeros(1, Hq, total, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, Hq, total, device="cuda")
    done = 0
    for n in (200, 100, 17, 1, 1, 5, 9):
        rows = slice(done, done + n)
        done += n
        where = (c.table, _ints(done), _ints(0, n))
        lib.tr_cache_write(k[:, :, rows], v[:, :, rows], *c.args()[:2], *where, *c.scale_args())
        lib.tr_paged_attn(q[:, :, rows], *c.args()[:2], *where, True, D ** -0.5, out[:, :, rows], lse[:, :, rows], *c.scale_args())
    assert done == total
    check(attention(c, q, D ** -0.5, True), out, lse)
    if not f8:      # what was written is what is attended
        got = c.rows("k", 0)[0].transpose(0, 1)
        assert torch.equal(got, k[0].double())


@pytest.mark.parametrize("f8", [False, True])
def test_a_cache_on_two_devices(lib, f8):
    """Each device writes the keys of its half and attends all queries to them; tr_merge folds the two block results (TokenRing's Update)."""
    n, total, cut, Hkv, Hq, D = 40, 700, 352, 2, 8, 128
    q, k, v = _tokens(n, Hq, D, 41), _tokens(total, Hkv, D, 42), _tokens(total, Hkv, D, 43)
    whole = Cache([total], [n], Hkv, D, 16, f8, "head", seed=44)
    lib.tr_cache_write(k, v, *whole.args()[:2], whole.table, whole.kv_len, _ints(0, total), *whole.scale_args())
    acc_o, acc_l = torch.zeros(1, Hq, n, D, device="cuda"), torch.full((1, Hq, n), float("-inf"), device="cuda")
    for first, kv in ((0, cut), (cut, total - cut)):
        part = Cache([kv], [n], Hkv, D, 32, f8, "head", seed=45 + first)
        # the new keys stand at the end of the sequence: this device writes those of all its keys that fall into its part
        lib.tr_cache_write(k, v, *part.args(), _ints(0, total), *part.scale_args(), q_pos=_ints(-first))
        step = Call(lib, part, q, True, _ints(total - n - first), torch.float32)
        step.run()
        lib.tr_merge(acc_o, acc_l, step.out, step.lse)
    found = attention(whole, q, D ** -0.5, True)
    check(found, acc_o, acc_l)


def test_read_back_for_block_steps(lib):
    """Keys handed on as dense tensors: a block step on them is the attention on the pages, up to the rounding of either."""
    c = Cache([500, 500], [64, 64], 2, 128, 48, True, "head", seed=51)
    q = _tokens(128, 8, 128, 52)
    k, v = (torch.empty(2, 2, 500, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lib.tr_cache_read(*c.args(), k, v, 0, *c.scale_args())
    step = Call(lib, c, q, True, None, torch.float32)
    step.run()
    found = attention(c, q, 128 ** -0.5, True)
    check(found, step.out, step.lse)
    dense_o, dense_l = torch.zeros(2, 8, 64, 128, device="cuda"), torch.zeros(2, 8, 64, device="cuda")
    dense_q = torch.cat([q[:, :, :64], q[:, :, 64:]], 0).contiguous()
    lib.tr_block_attn_causal_at(dense_q, k, v, 436, 0, 128 ** -0.5, dense_o, dense_l)
    for b, (rows, _, _, d_o, d_l) in enumerate(found):
        assert ((dense_o[b] - step.out[0, :, rows]).abs() <= 2 * d_o[0]).all() and ((dense_l[b] - step.lse[0, :, rows]).abs() <= 2 * d_l[0]).all()


@pytest.mark.parametrize("f8", [False, True])
def test_captured_and_replayed(lib, f8):
    """A step captured once and replayed on lengths, tokens and pages that change between the replays, with eager work of the same kind in between."""
    c = Cache([900, 33, 2000], [1, 40, 1], 2, 128, 16, f8, "head", seed=61)
    q, k, v = _tokens(42, 8, 128, 62), _tokens(42, 2, 128, 63), _tokens(42, 2, 128, 64)
    step, eager = Call(lib, c, q), Call(lib, c, q)

    def both():
        lib.tr_cache_write(k, v, *c.args(), c.q_start, *c.scale_args())
        step.run()
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i, kv in enumerate(([900, 33, 2000], [899, 40, 1], [1, 40, 1999], [900, 40, 2000])):
        c.kv = kv
        c.kv_len.copy_(_ints(*kv))
        k.copy_(_tokens(42, 2, 128, 70 + i))
        step.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = step.out.clone(), step.lse.clone()
        eager.run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], eager.out) and torch.equal(got[1], eager.lse)
        if kv[1] >= 40:     # (with fewer keys than new tokens the first ones stand in front of them)
            check(attention(c, q, 128 ** -0.5, True), *got)


def test_the_same_bits_again(lib):
    c = Cache([5000, 700, 64], [1, 130, 3], 2, 64, 32, True, "head", seed=81)
    q = _tokens(134, 8, 64, 82)
    a = Call(lib, c, q)
    a.run()
    was = a.out.clone(), a.lse.clone()
    for _ in range(3):
        a.run()
        assert torch.equal(a.out, was[0]) and torch.equal(a.lse, was[1])


def test_streams_and_one_workspace(lib):
    """Calls of different sizes in a row on one workspace; calls on other streams with workspaces of their own."""
    caches = [Cache([6000, 50], [1, 4], 2, 128, 16, i % 2 == 0, "head", seed=90 + i) for i in range(4)] + [Cache([3000], [300], 1, 128, 16, False, "head", seed=99)]
    qs = [_tokens(c.tokens, 4 * c.Hkv, 128, 95 + i) for i, c in enumerate(caches)]
    need = max(lib.tr_paged_attn_workspace_bytes(q, c.pages["k"], c.table) for q, c in zip(qs, caches))
    shared = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    for q, c in zip(qs, caches):
        one = Call(lib, c, q, workspace=shared)
        one.run()
        check(attention(c, q, 128 ** -0.5, True), one.out, one.lse)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in caches]
    calls = [Call(lib, c, q, stream=s) for c, q, s in zip(caches, qs, streams)]
    torch.cuda.synchronize()
    for _ in range(5):
        for call in calls:
            call.run()
    torch.cuda.synchronize()
    for call, c, q in zip(calls, caches, qs):
        check(attention(c, q, 128 ** -0.5, True), call.out, call.lse)


def test_long_caches_pass_32_bits(lib):
    """Pages more than 2^31 bytes and more than 2^32 bytes from the first: written, attended, read back."""
    page, H, D = 256, 8, 128
    n_pages = (9 << 29) // (page * H * D * 2) + 4          # 4.5 GiB of K, as much of V
    c = Cache([600], [20], H, D, page, False, "head", seed=71, poison=False)
    big = {x: torch.zeros(n_pages, H, page, D, dtype=torch.bfloat16, device="cuda") for x in "kv"}
    to = [n_pages - 1, 0, n_pages // 2 + 1]
    for i, p in enumerate(c.table[0].tolist()):
        for x in "kv":
            big[x][to[i]] = c.pages[x][p]
    c.table, c.pages, c.n_pages = _ints(*to).unsqueeze(0), big, n_pages
    q, k, v = _tokens(20, 16, D, 72), _tokens(20, H, D, 73), _tokens(20, H, D, 74)
    lib.tr_cache_write(k, v, *c.args(), c.q_start)
    step = Call(lib, c, q)
    step.run()
    check(attention(c, q, D ** -0.5, True), step.out, step.lse)
    out = [torch.zeros(1, H, 600, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lib.tr_cache_read(*c.args(), *out)
    assert torch.equal(out[0][0, :, 580:], k[0]) and torch.equal(out[1][0, :, 580:], v[0])


def test_quantised_attention_is_near(lib):
    """On an 8-bit cache the result is off by no more than what half a step of e4m3 in K and V can do."""
    kv, D, H = 400, 128, 2
    k, v = _tokens(kv, H, D, 101), _tokens(kv, H, D, 102)
    q = _tokens(1, 4, D, 103)
    outs = []
    for f8 in (False, True):
        c = Cache([kv], [1], H, D, 16, f8, "head", seed=104)
        lib.tr_cache_write(k, v, *c.args(), _ints(0, kv), *c.scale_args())
        step = Call(lib, c, q, True, None, torch.float32)
        step.run()
        outs.append((step.out, step.lse))
    # a score is off by at most e = scale * 2^-4 * sum |q k|; weights by a factor within exp(+-2 e), values by 2^-4 of themselves (and 2^-10 / 224 of the row's largest)
    qs, ks, vs = q[0].double().view(H, 2, 1, D), k[0].double().unsqueeze(1), v[0].double().unsqueeze(1)
    e = (qs.abs() @ (ks.abs() * 2.0 ** -4 + ks.abs().amax(-1, keepdim=True) * 2.0 ** -10 / 224).transpose(2, 3) * D ** -0.5).amax(-1).view(1, 4, 1)
    p = torch.softmax(qs @ ks.transpose(2, 3) * D ** -0.5, -1)
    mean = (p @ vs.abs()).view(1, 4, 1, D)
    largest = (p @ vs.abs().amax(-1, keepdim=True)).view(1, 4, 1, 1)
    grow = torch.exp(2 * e).unsqueeze(-1)
    bound = (grow - 1) * mean + grow * (2.0 ** -4 * mean + 2.0 ** -10 / 224 * largest) + 4 * BF16_STEP * grow * mean
    assert ((outs[0][0] - outs[1][0]).abs() <= bound).all() and ((outs[0][1] - outs[1][1]).abs() <= e + 1e-4).all()
