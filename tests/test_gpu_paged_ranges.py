"""Attention on a paged cache at the ends of its ranges."""
import math

import pytest
import torch

from paged_util import F32_STEP, Cache, attention, check, quantised

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
