"""Kinds of arguments that the cache's and the attention's wrappers take, with host tensors that say
they are CUDA ones and a library that does nothing."""
import pytest
import torch

from paper_2608_10362_gb300 import KVCache
from test_kv_attention_cpu import BF, I32, _cache, _rows, _t, calls, kv_module  # noqa: F401
from test_wrapper_streams_cpu import allocations  # noqa: F401


class Paged(KVCache):
    """A caller's own kind of cache."""


def test_a_subclass_is_a_cache(calls):  # noqa: F811
    cache = Paged(*_cache(True).tensors)
    q, (s, l) = _t(3, 4, 64, dtype=BF), _rows()
    for prefix in (None, cache):
        assert kv_module.op_attention(q, cache, s, l, prefix=prefix).shape == q.shape
    assert kv_module.op_kv_append(_t(3, 4 * 64), cache, s, l, 2).shape == (3, 2, 64)
    assert kv_module.op_kv_read(cache, s, l, 3)[0].shape == (3, 1, 64)
    with pytest.raises(ValueError, match="KVCache"):
        kv_module.op_attention(q, cache.k, s, l)
