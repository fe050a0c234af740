"""tr_cache_write and tr_cache_read against their definition, bit by bit."""
import pytest
import torch

from paged_util import Cache, power, quantised

pytestmark = pytest.mark.gpu


def _tokens(T, H, D, seed, layout="token"):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(1, T, H, D, generator=g) * torch.exp(3 * torch.randn(1, T, H, 1, generator=g))).bfloat16()
    x = x.to("cuda")
    return x.transpose(1, 2) if layout == "token" else x.transpose(1, 2).contiguous()


def _bits(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16)


def _expected(c, name, x, pos=None):
    """(codes or values, scale bytes) of all pages after the tokens x have been written."""
    pages = _bits(c.pages[name]).clone()
    scales = c.scales[name].view(torch.uint8).clone() if c.f8 else None
    codes, e = quantised(x[0]) if c.f8 else (x[0], None)
    for b, n in enumerate(c.q):
        for i in range(n):
            key = (c.kv[b] - n if pos is None else pos[b]) + i
            if not 0 <= key < c.kv[b]:
                continue
            page = int(c.table[b, key // c.page])
            if not 0 <= page < c.n_pages:
                continue
            pages[page, :, key % c.page] = _bits(codes)[:, c.starts[b] + i]
            if c.f8:
                scales[page, :, key % c.page] = e[:, c.starts[b] + i]
    return pages, scales


CASES = [
    # kv, new tokens, Hkv, D, page, layout of the pages
    ([1], [1], 1, 64, 16, "head"),
    ([100, 16, 33], [5, 16, 1], 2, 128, 16, "head"),
    ([100, 0, 33, 64], [37, 0, 33, 0], 3, 128, 48, "token"),
    ([700] * 3, [7, 0, 300], 8, 64, 32, "token"),
    ([i % 5 for i in range(130)], [min(1, i % 5) for i in range(130)], 2, 128, 16, "head"),
]


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_write(lib, case, f8):
    kv, q, H, D, page, layout = case
    c = Cache(kv, q, H, D, page, f8, layout, seed=3)
    k, v = _tokens(c.tokens, H, D, 5), _tokens(c.tokens, H, D, 6)
    want = [_expected(c, name, x) for name, x in (("k", k), ("v", v))]
    lib.tr_cache_write(k, v, *c.args(), c.q_start, *c.scale_args())
    for name, (pages, scales) in zip("kv", want):
        assert torch.equal(_bits(c.pages[name]), pages)
        assert not f8 or torch.equal(c.scales[name].view(torch.uint8), scales)


@pytest.mark.parametrize("f8", [False, True])
def test_write_at_positions_and_beyond_the_pages(lib, f8):
    """Tokens in front of this cache's keys and behind them, entries that are no pages, tokens outside every sequence."""
    kv, q, pos = [40, 25, 64], [30, 20, 10], [-10, 15, 60]
    c = Cache(kv, q, 2, 128, 16, f8, "head", seed=4)
    c.table[0, 1], c.table[2, 3] = -1, c.n_pages
    k, v = _tokens(c.tokens + 9, 2, 128, 7), _tokens(c.tokens + 9, 2, 128, 8)      # 4 tokens in front, 5 behind
    c.q_start += 4
    c.starts = [s + 4 for s in c.starts]
    want = [_expected(c, name, x, pos) for name, x in (("k", k), ("v", v))]
    lib.tr_cache_write(k, v, *c.args(), c.q_start, *c.scale_args(), q_pos=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    for name, (pages, scales) in zip("kv", want):
        assert torch.equal(_bits(c.pages[name]), pages)
        assert not f8 or torch.equal(c.scales[name].view(torch.uint8), scales)


def test_scales_at_their_borders(lib):
    """The largest value at 448 and just above it, powers of two, zeros, the smallest and largest bf16, infinities and NaN."""
    inf, nan = float("inf"), float("nan")
    tops = [0.0, 448.0, 450.0, 1.0, 2.0, 1.75, 1.7578125, 2.0 ** -133, 2.0 ** -126, 2.0 ** -118, 1.75 * 2.0 ** -118, 3.3895e38, inf, nan, -448.0, -inf]
    x = torch.zeros(1, 1, len(tops), 64)
    x[0, 0, :, 0] = torch.tensor(tops, dtype=torch.float64).float()
    ramp = torch.linspace(-1, 1, 62)
    for i, t in enumerate(tops):
        x[0, 0, i, 2:] = ramp * (abs(t) if abs(t) < inf else 5.0)
    x = x.bfloat16().cuda()
    c = Cache([len(tops)], [len(tops)], 1, 64, 16, True, "head", seed=1)
    want = _expected(c, "k", x)
    lib.tr_cache_write(x, x, *c.args(), c.q_start, *c.scale_args())
    got = c.pages["k"].float()
    torch.testing.assert_close(got, want[0].view(torch.float8_e4m3fn).float(), rtol=0, atol=0, equal_nan=True)
    assert torch.equal(c.scales["k"].view(torch.uint8), want[1])


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("first", [0, 17])
def test_read(lib, case, f8, first):
    kv, q, H, D, page, layout = case
    c = Cache(kv, q, H, D, page, f8, layout, seed=9)
    S = max(0, max(kv) - first) + 3
    out = [torch.full((len(kv), S, H, D), 7.5, dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2)]
    want = [o.clone() for o in out]
    for name, w in zip("kv", want):
        for b, n in enumerate(kv):
            if n > first:
                w[b, :, :n - first] = c.rows(name, b)[0][first:].transpose(0, 1).bfloat16()
    lib.tr_cache_read(*c.args(), *out, first, *c.scale_args())
    for o, w in zip(out, want):
        assert torch.equal(o, w)


def test_every_code_and_scale(lib):
    """All 256 codes under all 256 scales come back as the values they stand for, rounded once to bf16."""
    c = Cache([1024], [0], 1, 64, 64, True, "head", seed=2, spare=0)
    codes = torch.arange(256, device="cuda").repeat(256).view(256 * 4, 64).to(torch.uint8)
    e = torch.arange(256, device="cuda").repeat_interleave(4).to(torch.uint8)
    page = c.table[0].long()
    for name in "kv":
        c.pages[name].view(torch.uint8)[page] = codes.view(16, 1, 64, 64)
        c.scales[name].view(torch.uint8)[page] = e.view(16, 1, 64)
    want = codes.view(torch.float8_e4m3fn).double() * torch.where(e == 255, float("nan"), power(e.long() - 127)).unsqueeze(-1)
    k, v = (torch.zeros(1, 1, 1024, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lib.tr_cache_read(*c.args(), k, v, 0, *c.scale_args())
    want = want.bfloat16()
    for x in (k, v):
        torch.testing.assert_close(x[0, 0], want, rtol=0, atol=0, equal_nan=True)
    q = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros(1, 1, 1, 64, device="cuda"), torch.zeros(1, 1, 1, device="cuda")
    c.kv_len.fill_(4 * 127)                     # scales 0 .. 126, values that a mean of all keeps apart
    c.pages["k"].view(torch.uint8).zero_()
    c.pages["v"].view(torch.uint8)[page] = torch.where((codes & 127) == 127, 0, codes).to(torch.uint8).view(16, 1, 64, 64)
    lib.tr_paged_attn(q, *c.args(), torch.tensor([0, 1], dtype=torch.int32, device="cuda"), False, 1.0, out, lse, *c.scale_args())
    assert torch.isfinite(out).all()


def test_values_come_back_as_near_as_their_type_allows(lib):
    """Written and read again: within half a step of e4m3 of the row's scale; once more written and read: the same."""
    c = Cache([300, 41], [300, 41], 4, 128, 16, True, "head", seed=11)
    k, v = _tokens(c.tokens, 4, 128, 21), _tokens(c.tokens, 4, 128, 22)
    back = [torch.zeros(2, 4, 300, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lib.tr_cache_write(k, v, *c.args(), c.q_start, *c.scale_args())
    lib.tr_cache_read(*c.args(), *back, 0, *c.scale_args())
    for x, y in ((k, back[0]), (v, back[1])):
        for b, (lo, n) in enumerate(((0, 300), (300, 41))):
            a, r = x[0, :, lo:lo + n].double(), y[b, :, :n].double()
            top = a.abs().amax(-1, keepdim=True)      # a scale is at most top / 224; below 2^-6 of it steps are all 2^-9 of it
            assert ((a - r).abs() <= torch.maximum(2.0 ** -4 * a.abs(), 2.0 ** -10 * top / 224)).all()
    again = [torch.cat([y[0, :, :300], y[1, :, :41]], 1).unsqueeze(0) for y in back]
    twice = [torch.zeros_like(y) for y in back]
    lib.tr_cache_write(*again, *c.args(), c.q_start, *c.scale_args())
    lib.tr_cache_read(*c.args(), *twice, 0, *c.scale_args())
    assert torch.equal(twice[0], back[0]) and torch.equal(twice[1], back[1])
