"""op_attention and op_kv_read at the ends of what scales, queries and caches may hold, against
the definitions in 64 bits; bounds as in test_gpu_kv_attention.py."""
import math

import pytest
import torch

from test_gpu_kv_attention import DEV, _gen, _i32, _pkg, attention64, batch, check, make_cache

pytestmark = pytest.mark.gpu

FEW, MANY = (4, 4), (32, 4)    # heads, heads of k and v: of 2 rows up to 16 vectors a head, or more


# ------------------------------------------------------------------ nothing to tell keys apart by
@pytest.mark.parametrize("prefix_len", [0, 200])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,Hk", [FEW, MANY], ids=["few", "many"])
@pytest.mark.parametrize("codes", [False, True])
def test_zero_queries(H, Hk, hd, codes, prefix_len):
    """Queries of zeros weigh what they see alike: rows of a sequence without slots (whose queries op_kv_append
    makes 0), keys of zeros as a new cache has them, and a scale of 0."""
    pkg = _pkg()
    starts, lens = [0, 5, 8], [0, 141]
    prefix = make_cache(codes, 1, Hk, prefix_len + 7, hd, seed=2) if prefix_len else None
    q = torch.zeros(8, H, hd, device=DEV, dtype=torch.bfloat16)
    for what in ("keys", "zero keys", "scale 0"):
        cache = make_cache(codes, 2, Hk, 150, hd, seed=1)
        if what == "zero keys":
            for t in cache.tensors[0:3:2]:
                if t is not None:
                    t.zero_()
        scale = 0.0 if what == "scale 0" else None
        for max_rows in (8, 5, 1):
            got = pkg.op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=max_rows, prefix=prefix,
                                   prefix_len=prefix_len or None, scale=scale)
            check(got, *attention64(q, cache, starts, lens, prefix=prefix, prefix_len=prefix_len, scale=scale,
                                    max_rows=max_rows))
            if not prefix_len:
                assert not got[:5].any()


def test_appended_rows_without_slots():
    """The same through the calls: a sequence of length 0 with rows, in a new cache of codes."""
    pkg, H, Hk, hd = _pkg(), 32, 4, 128
    cache = pkg.KVCache.zeros(2, Hk, 40, hd, dtype=torch.int8)
    s, l = _i32(0, 5, 8), _i32(0, 3)
    x = torch.randn(8, (H + 2 * Hk) * hd, device=DEV, generator=_gen(1))
    q = pkg.op_kv_append(x, cache, s, l, H)
    got = pkg.op_attention(q, cache, s, l, max_rows=5)
    assert not q[:5].any() and not got[:5].any()
    check(got, *attention64(q, cache, [0, 5, 8], [0, 3], max_rows=5))
