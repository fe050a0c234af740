"""A tree without branches against the causal call, to the bit, where both take the same launch: tiles of as many rows, no keys shared out."""
import pytest
import torch

from evict_util import packed, tree_of
from paged_util import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kv,n", [
    ([1, 700, 3000], 1),          # 4 rows a K/V head: tiles of 16
    ([700], 3),                   # 12
    ([33, 700, 3000], 33),        # 132: of 256
    ([100, 700, 3000], 100),      # 400
    ([2000], 8),                  # 32: of 32
    ([2500], 300),
])
def test_a_chain_is_the_causal_call(lib, kv, n, D, f8):
    c = Cache(kv, [n] * len(kv), 2, D, 32, f8, "head", seed=8)
    sees = packed(tree_of(list(range(-1, n - 1))), (n + 31) // 32)
    q = torch.randn(1, 8, c.tokens, D, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    for dtype in (torch.bfloat16, torch.float32):
        of_tree, causal = ((torch.full(q.shape, 7.0, dtype=dtype, device="cuda"), torch.full((1, 8, c.tokens), 7.0, device="cuda")) for _ in range(2))
        lib.tr_paged_attn_tree(q, *c.args(), c.q_start, torch.cat([sees] * len(kv)).cuda(), 0.1, *of_tree, *c.scale_args())
        lib.tr_paged_attn(q, *c.args(), c.q_start, True, 0.1, *causal, *c.scale_args())
        assert torch.equal(of_tree[0], causal[0]) and torch.equal(of_tree[1], causal[1])
