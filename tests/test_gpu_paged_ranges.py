"""Attention on a paged cache at the ends of its ranges."""
import pytest
import torch

from paged_util import Cache, attention, check, quantised

pytestmark = pytest.mark.gpu


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
