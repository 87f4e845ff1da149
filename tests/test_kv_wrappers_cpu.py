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


def test_what_is_no_tensor_is_refused(calls):  # noqa: F811
    """With the wrappers' own error, as an argument of the wrong kind is elsewhere."""
    cache, q, (s, l) = _cache(False), _t(3, 4, 64, dtype=BF), _rows()
    x = _t(3, 4 * 64)
    for bad in ([0, 1, 3], None, 7):
        for call in (lambda: kv_module.op_attention(q, cache, bad, l), lambda: kv_module.op_attention(q, cache, s, bad),
                     lambda: kv_module.op_kv_append(x, cache, bad, l, 2), lambda: kv_module.op_kv_append(x, cache, s, bad, 2),
                     lambda: kv_module.op_kv_read(cache, bad, l, 3), lambda: kv_module.op_kv_read(cache, s, bad, 3)):
            with pytest.raises(ValueError):
                call()
        if bad is not None:
            for kw in (dict(scratch=bad), dict(tree=bad), dict(out=bad), dict(prefix=bad)):
                with pytest.raises(ValueError):
                    kv_module.op_attention(q, cache, s, l, **kw)
            for kw in (dict(rope=bad), dict(offsets=bad), dict(q_gain=bad, k_gain=bad), dict(q=bad)):
                with pytest.raises(ValueError):
                    kv_module.op_kv_append(x, cache, s, l, 2, **kw)
            with pytest.raises(ValueError):
                kv_module.op_kv_read(cache, s, l, 3, k=bad)
            with pytest.raises(ValueError):
                KVCache(cache.k, bad)


def test_the_engines_cache_of_a_draft_that_is_none():
    """The wrapper's own error again, before anything is looked up."""
    import types

    from paper_2608_10362_gb300 import Engine
    engine = Engine.__new__(Engine)
    engine.ctx, engine.drafts, engine.kv = None, {}, None
    engine.shape = types.SimpleNamespace(n_layers=2, n_kv_heads=1, head_dim=64)
    for args in ((0, 3), (0, -1), (2,), (-1,), (0.5,), (None,)):
        with pytest.raises(ValueError):
            engine.kv_cache(*args)
