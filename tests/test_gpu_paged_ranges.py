"""Attention on a paged cache at the ends of its ranges: large V under growing scores, every code and scale in either product, millions of keys."""
import math

import pytest
import torch

from paged_util import F32_STEP, Cache, attention, check, power, quantised

pytestmark = pytest.mark.gpu


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _workspace(lib, q, pages, table):
    return torch.full((lib.tr_paged_attn_workspace_bytes(q, pages, table),), 255, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 70])
@pytest.mark.parametrize("growth", [12.0, 50.0, 300.0])
def test_large_values_under_growing_scores(lib, growth, n, D, f8):
    """V of about 2^92 under scores that rise by 12, 50 and 300 along the keys: finite results, and those of the formula."""
    kv = 3000
    c = Cache([kv], [n], 1, D, 16, f8, "head", seed=110)
    key = torch.arange(kv, device="cuda")
    page, slot = c.table[0].long()[key // 16], key % 16
    rows = torch.zeros(kv, D, device="cuda")
    rows[:, 0] = key * (growth / kv)
    if f8:
        codes, e = quantised(rows.bfloat16())
        c.pages["k"].view(torch.uint8)[page, 0, slot] = codes.view(torch.uint8)
        c.scales["k"].view(torch.uint8)[page, 0, slot] = e
        c.scales["v"].view(torch.uint8)[page, 0, slot] += 92
    else:
        c.pages["k"][page, 0, slot] = rows.bfloat16()
        c.pages["v"][page, 0, slot] *= 2.0 ** 92
    q = torch.zeros(1, 4, n, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = torch.tensor([1.0, 0.5, -1.0, 0.0], device="cuda").view(1, 4, 1)
    out, lse = torch.zeros(1, 4, n, D, device="cuda"), torch.zeros(1, 4, n, device="cuda")
    for ws in (None, _workspace(lib, q, c.pages["k"], c.table)):
        lib.tr_paged_attn(q, *c.args(), c.q_start, True, 1.0, out, lse, *c.scale_args(), workspace=ws)
        check(attention(c, q, 1.0, True), out, lse)


def _one_key_each(scale_bytes):
    """A sequence of one key for every 64 codes and every given scale, key 0 of a page of its own: cache, values [sequences, 64] as bf16 holds them."""
    n = 4 * len(scale_bytes)
    c = Cache([1] * n, [0] * n, 1, 64, 16, True, "head", seed=120, spare=0)
    codes = torch.arange(256, device="cuda").repeat(len(scale_bytes)).view(n, 64).to(torch.uint8)
    e = torch.tensor(scale_bytes, device="cuda").repeat_interleave(4)
    return c, c.table[:, 0].long(), codes, e


def _call(lib, c, q, tokens, scale, dtype=torch.float32):
    n = len(c.kv)
    out, lse = torch.zeros(1, q.shape[1], n * tokens, 64, dtype=dtype, device="cuda"), torch.zeros(1, q.shape[1], n * tokens, device="cuda")
    lib.tr_paged_attn(q, *c.args(), torch.arange(n + 1, dtype=torch.int32, device="cuda") * tokens, False, scale, out, lse, *c.scale_args())
    return out, lse


@pytest.mark.parametrize("heads", [1, 20, 64])      # 16, 32 and 256 rows a workgroup
def test_every_code_and_scale_of_v(lib, heads):
    """A token that sees one key gets that key's row of V: the weight is 1, so that the result is the value itself (below 2^-126, where products may count as 0, up to that)."""
    c, page, codes, e = _one_key_each(list(range(256)))
    c.pages["k"].view(torch.uint8).zero_()
    c.scales["k"].view(torch.uint8).fill_(127)
    c.pages["v"].view(torch.uint8)[page, 0, 0] = codes
    c.scales["v"].view(torch.uint8)[page, 0, 0] = e.to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double() * torch.where(e == 255, float("nan"), power(e.clamp(max=254) - 127)).unsqueeze(-1)
    want = want.bfloat16().double()
    out, lse = _call(lib, c, torch.zeros(1, heads, len(c.kv), 64, dtype=torch.bfloat16, device="cuda"), 1, 1.0)
    assert (lse == 0).all()
    out = out[0].double()
    fine = want.isfinite().expand_as(out)
    assert torch.equal(out.isnan(), want.isnan().expand_as(out)) and torch.equal(out.isposinf(), want.isposinf().expand_as(out))
    assert torch.equal(out.isneginf(), want.isneginf().expand_as(out))
    off = ((out - want).abs())[fine]
    assert (off <= torch.where(want.expand_as(out)[fine].abs() < 2.0 ** -126, 2.0 ** -126, 0.0)).all()


@pytest.mark.parametrize("tokens", [1, 2, 4])       # of 16 heads: 16, 32 and 256 rows a workgroup
def test_every_code_and_scale_of_k(lib, tokens):
    """A token that sees one key has its score as lse: with a query of one 1, a value of K (K near 0 as above).  Rounding: the score's product with `scale` in front of the exponential and
    in the result."""
    for e0 in (0, 3, 9, 10, 50, 100, 119, 120, 127, 128, 150, 200, 237, 238):
        c, page, codes, e = _one_key_each([e0])
        codes = torch.where((codes & 127) == 127, 0, codes).to(torch.uint8)      # (a NaN in any place makes all of the row's scores NaN)
        for name, x, s in (("k", codes, e0), ("v", codes * 0, 127)):
            c.pages[name].view(torch.uint8)[page, 0, 0] = x
            c.scales[name].view(torch.uint8)[page, 0, 0] = s
        scale = 2.0 ** min(120, 127 - e0)
        want = codes.view(torch.float8_e4m3fn).double() * power(e0 - 127) * scale      # [sequence, d]
        d = torch.arange(16 * tokens, device="cuda").view(tokens, 16)
        for first in range(0, 64, 16 * tokens):
            one = torch.nn.functional.one_hot(d + first, 64).transpose(0, 1)           # [head, token, 64]
            q = one.repeat(1, 4, 1).unsqueeze(0).bfloat16()
            _, lse = _call(lib, c, q, tokens, scale)
            got, ref = lse[0].view(16, 4, tokens).double(), want[:, d + first].permute(2, 0, 1)
            assert ((got - ref).abs() <= 4 * F32_STEP * ref.abs() + 2.0 ** -22 + 2.0 ** -126 * scale).all(), e0


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("kv,n,gq", [(2097152, 1, 4), (2097153, 40, 2), (5000001, 2, 8)])
def test_millions_of_keys(lib, kv, n, gq, f8):
    """Keys that repeat (a table of the same pages again and again): attention on the few there are, lse larger by the logarithm of the repeats; the keys behind the last whole repeat count on their own."""
    D, Hkv, page = 128, 2, 256
    c = Cache([5 * page], [n], Hkv, D, page, f8, "head", seed=130, poison=False)
    width = -(-kv // page)
    table = c.table[0].repeat(-(-width // 5))[:width].unsqueeze(0).contiguous()
    q = torch.randn(1, Hkv * gq, n, D, generator=torch.Generator().manual_seed(131)).bfloat16().cuda()
    out, lse = torch.zeros(1, Hkv * gq, n, D, device="cuda"), torch.zeros(1, Hkv * gq, n, device="cuda")
    ws = _workspace(lib, q, c.pages["k"], table)
    lib.tr_paged_attn(q, *c.args()[:2], table, _ints(kv), c.q_start, False, D ** -0.5, out, lse, *c.scale_args(), workspace=ws)
    times = torch.full((5 * page,), float(kv // (5 * page)), dtype=torch.float64, device="cuda")
    times[:kv % (5 * page)] += 1
    K, V = (c.rows(x, 0)[0].permute(1, 0, 2)[:, None] for x in "kv")
    qs = q[0].double().view(Hkv, gq, n, D)
    x = qs @ K.transpose(2, 3) * D ** -0.5 + times.log()
    ref_l = torch.logsumexp(x, -1)
    p = torch.exp(x - ref_l.unsqueeze(-1))
    ref_o, mean = p @ V, p @ V.abs()
    # rounding: weights to bf16; sums of up to 2^16 additions in 32 bits one after the other (a lane's, every fourth stretch of a part), each off by half a step
    size = float((qs.abs() @ K.abs().transpose(2, 3)).max()) * D ** -0.5
    d_l = (D + 16) * F32_STEP * size + 2.0 ** 16 * F32_STEP + 2.0 ** -20
    d_o = (2.0 ** -8 + 2 * d_l) * mean
    assert ((lse[0].view(Hkv, gq, n) - ref_l).abs() <= d_l).all()
    assert ((out[0].view(Hkv, gq, n, D) - ref_o).abs() <= d_o).all()
    assert math.isfinite(float(out.abs().max()))
