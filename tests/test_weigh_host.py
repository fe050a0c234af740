"""tr_cache_weigh on a machine without a GPU: how much work a call may ask for."""
import pytest

from test_evict_host import SHAPE, Call, tr  # noqa: F401  (tr: a fixture)


@pytest.mark.parametrize("n_seqs,Hkv,stretches", [
    (14322, 3, 49981),      # 2^31 - 2 stretches of 64 keys: rounded up to eighths, their number would pass 2^31 - 1
    (1 << 16, 8, 1 << 12),  # 2^31
])
def test_more_keys_than_can_be_shared_out(tr, n_seqs, Hkv, stretches):  # noqa: F811
    assert n_seqs * Hkv * stretches >= 2 ** 31 - 8
    c = Call(tr, page=64)
    wide = lambda name, D: c.like(name, H=Hkv, stride_b=Hkv * 64 * D)   # noqa: E731
    q = c.like("q", H=Hkv, stride_b=Hkv * 7 * 128)
    st, msg = c("weigh", q=q, lse=c.like("lse", H=Hkv, stride_b=Hkv * 7), kp=wide("kp", 128), ks=wide("ks", 1), w=wide("w", 1),
                seqs=c.like("seqs", n_seqs=n_seqs, max_pages=stretches, table_stride=stretches))
    assert st == SHAPE and "too many keys" in msg, (st, msg)
