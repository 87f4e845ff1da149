"""Refusals of the cache's and the attention's calls, on a machine without a GPU: every check
comes before anything is enqueued, and the wrappers take no tensors from elsewhere."""
import ctypes as C

import pytest
import torch

from paper_2608_10362_gb300 import KVCache, _lib, op_rope_table


@pytest.fixture(scope="module")
def lib():
    from paper_2608_10362_gb300 import build
    build.build()
    return _lib.load()


AT = 1 << 20   # an aligned address that nothing follows: every call below is refused first


def good_kv(**kw):
    f = dict(k_dev=AT, v_dev=2 * AT, k_scale_dev=None, v_scale_dev=None, seq_stride=8 * 64 * 128, head_stride=64 * 128,
             pos_stride=128, scale_seq_stride=8 * 64, scale_head_stride=64, scale_pos_stride=1, n_seq=4, n_heads=8,
             max_pos=64, head_dim=128)
    return _lib.Kv(**{**f, **kw})


def good_batch(**kw):
    return _lib.Batch(**{**dict(starts_dev=AT, lens_dev=AT, n_seq=4, rows=16), **kw})


def good_append(**kw):
    f = dict(qkv_dev=AT, qkv_type=_lib.F32, n_heads=32, ld=48 * 128, rope_dev=AT, rope_positions=64, prefix_len=0,
             offsets_dev=None, q_gain_dev=AT, k_gain_dev=AT, eps=1e-5, q_dev=AT)
    return _lib.Append(**{**f, **kw})


def good_attention(**kw):
    f = dict(q_dev=AT, ldq=32 * 128, out_dev=2 * AT, ldo=32 * 128, n_heads=32, scale=0.1, tree_dev=None, prefix=None,
             prefix_len=0, max_rows=4)
    return _lib.Attention(**{**f, **kw})


def refused(lib, status):
    assert status == _lib.ERR_INVALID_ARG
    assert lib.memspec_op_last_error().decode()


KV_FAULTS = [dict(k_dev=None), dict(v_dev=None), dict(k_scale_dev=AT), dict(v_scale_dev=AT), dict(head_dim=96),
             dict(head_dim=0), dict(n_seq=0), dict(n_heads=0), dict(n_heads=1025), dict(max_pos=0), dict(max_pos=-1),
             dict(pos_stride=132), dict(head_stride=-128), dict(seq_stride=1 << 41), dict(k_dev=AT + 8),
             dict(k_scale_dev=AT, v_scale_dev=2 * AT, pos_stride=136), dict(k_scale_dev=AT + 2, v_scale_dev=2 * AT),
             dict(k_scale_dev=AT, v_scale_dev=2 * AT, scale_pos_stride=-1)]
BATCH_FAULTS = [dict(starts_dev=None), dict(lens_dev=None), dict(starts_dev=AT + 2), dict(n_seq=0), dict(n_seq=5),
                dict(n_seq=1025), dict(rows=0), dict(rows=65536)]


@pytest.mark.parametrize("fault", KV_FAULTS, ids=str)
def test_bad_caches(lib, fault):
    kv, b = good_kv(**fault), good_batch()
    refused(lib, lib.memspec_op_kv_append(C.byref(b), C.byref(kv), C.byref(good_append()), None))
    refused(lib, lib.memspec_op_kv_read(C.byref(b), C.byref(kv), AT, AT, None))
    refused(lib, lib.memspec_op_attention(C.byref(b), C.byref(kv), C.byref(good_attention()), AT, 1 << 40, None))
    prefix = good_attention(prefix=C.pointer(kv), prefix_len=1)
    refused(lib, lib.memspec_op_attention(C.byref(b), C.byref(good_kv()), C.byref(prefix), AT, 1 << 40, None))


@pytest.mark.parametrize("fault", BATCH_FAULTS, ids=str)
def test_bad_batches(lib, fault):
    kv, b = good_kv(n_seq=4 if fault.get("n_seq") != 1025 else 2000), good_batch(**fault)
    refused(lib, lib.memspec_op_kv_append(C.byref(b), C.byref(kv), C.byref(good_append()), None))
    refused(lib, lib.memspec_op_kv_read(C.byref(b), C.byref(kv), AT, AT, None))
    refused(lib, lib.memspec_op_attention(C.byref(b), C.byref(kv), C.byref(good_attention()), AT, 1 << 40, None))


@pytest.mark.parametrize("kv", [dict(pos_stride=64, head_dim=128), dict(seq_stride=0), dict(head_stride=32 * 128),
                                dict(v_dev=AT), dict(k_scale_dev=AT, v_scale_dev=AT),
                                dict(k_scale_dev=AT, v_scale_dev=2 * AT, scale_head_stride=32)], ids=str)
def test_caches_whose_vectors_overlap_are_not_written(lib, kv):
    refused(lib, lib.memspec_op_kv_append(C.byref(good_batch()), C.byref(good_kv(**kv)), C.byref(good_append()), None))


@pytest.mark.parametrize("fault", [dict(qkv_dev=None), dict(q_dev=None), dict(qkv_type=2), dict(n_heads=0),
                                   dict(n_heads=1025), dict(ld=48 * 128 - 2), dict(ld=48 * 128 + 1), dict(ld=1 << 41),
                                   dict(qkv_dev=AT + 4), dict(qkv_type=_lib.BF16, qkv_dev=AT + 2), dict(q_dev=AT + 2),
                                   dict(rope_positions=0), dict(prefix_len=-1), dict(q_gain_dev=None),
                                   dict(k_gain_dev=None), dict(eps=-1e-5), dict(eps=float("nan")),
                                   dict(eps=float("inf")), dict(offsets_dev=AT + 1)], ids=str)
def test_bad_appends(lib, fault):
    refused(lib, lib.memspec_op_kv_append(C.byref(good_batch()), C.byref(good_kv()), C.byref(good_append(**fault)), None))


@pytest.mark.parametrize("fault", [dict(q_dev=None), dict(out_dev=None), dict(out_dev=AT), dict(q_dev=AT + 8),
                                   dict(out_dev=2 * AT + 8), dict(ldq=32 * 128 - 8), dict(ldq=32 * 128 + 4),
                                   dict(ldo=1 << 41), dict(n_heads=0), dict(n_heads=36), dict(n_heads=8 * 65),
                                   dict(scale=float("nan")), dict(scale=float("inf")), dict(max_rows=0),
                                   dict(max_rows=17), dict(tree_dev=AT + 2)], ids=str)
def test_bad_attentions(lib, fault):
    a = good_attention(**fault)
    refused(lib, lib.memspec_op_attention(C.byref(good_batch()), C.byref(good_kv()), C.byref(a), AT, 1 << 40, None))


def test_bad_prefixes_and_scratch(lib):
    b, kv, n = good_batch(), good_kv(), C.c_size_t()
    for other, length in ((dict(n_heads=4), 8), (dict(head_dim=64), 8), ({}, -1), ({}, 65)):
        p = good_kv(**other)
        a = good_attention(prefix=C.pointer(p), prefix_len=length)
        refused(lib, lib.memspec_op_attention(C.byref(b), C.byref(kv), C.byref(a), AT, 1 << 40, None))
        refused(lib, lib.memspec_op_attention_scratch_bytes(C.byref(b), C.byref(kv), C.byref(a), C.byref(n)))
    a = good_attention()
    assert lib.memspec_op_attention_scratch_bytes(C.byref(b), C.byref(kv), C.byref(a), C.byref(n)) == 0
    refused(lib, lib.memspec_op_attention(C.byref(b), C.byref(kv), C.byref(a), AT, n.value - 1, None))
    refused(lib, lib.memspec_op_attention(C.byref(b), C.byref(kv), C.byref(a), AT + 8, n.value, None))
    refused(lib, lib.memspec_op_attention(C.byref(b), C.byref(kv), C.byref(a), None, n.value, None))
    for b_, kv_, a_ in ((None, kv, a), (b, None, a), (b, kv, None)):
        ptr = [None if x is None else C.byref(x) for x in (b_, kv_, a_)]
        refused(lib, lib.memspec_op_attention(*ptr, AT, n.value, None))


@pytest.mark.parametrize("args", [(0, 128, 1e4, AT), (8, 0, 1e4, AT), (8, 127, 1e4, AT), (8, 2048, 1e4, AT),
                                  (1 << 30, 128, 1e4, AT), (8, 128, 0.0, AT), (8, 128, float("nan"), AT),
                                  (8, 128, float("inf"), AT), (8, 128, 1e4, None), (8, 128, 1e4, AT + 2)], ids=str)
def test_bad_rope_tables(lib, args):
    refused(lib, lib.memspec_op_rope_table(*args, None))


def test_wrappers_take_no_host_tensors():
    k = torch.zeros(2, 2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        KVCache(k, k.clone())
    with pytest.raises(ValueError, match="scales"):
        KVCache(k, k.clone(), torch.zeros(2, 2, 8))
    with pytest.raises(ValueError, match="bfloat16 or int8"):
        KVCache.zeros(1, 1, 1, 64, dtype=torch.float32)
    with pytest.raises(ValueError, match="CUDA"):
        op_rope_table(8, 64, device="cpu")


# ------------------------------------------------------------------ memory, with a stream
from test_wrapper_streams_cpu import BF, CURRENT, LOG, SIDE, _t, allocations  # noqa: E402,F401
from paper_2608_10362_gb300 import kv as kv_module  # noqa: E402

I32 = torch.int32


def _cache(codes):
    t = [_t(2, 1, 8, 64, dtype=torch.int8 if codes else BF) for _ in (0, 1)]
    return KVCache(*t, *([_t(2, 1, 8), _t(2, 1, 8)] if codes else []))


def _rows():
    return [_t(3, dtype=I32), _t(2, dtype=I32)]


CALLS = {   # name: (the caches, the call's tensors, the call)
    "append": (lambda: [_cache(False)], lambda: [_t(3, 4 * 64), *_rows()],
               lambda st, c, x, s, l: kv_module.op_kv_append(x, c, s, l, 2, stream=st)),
    "append_codes": (lambda: [_cache(True)],
                     lambda: [_t(3, 4 * 64, dtype=BF), *_rows(), _t(2, 9, 32), _t(3, dtype=I32), _t(64, dtype=BF), _t(64, dtype=BF)],
                     lambda st, c, x, s, l, r, o, g, h: kv_module.op_kv_append(x, c, s, l, 2, r, o, 1, g, h, stream=st)),
    "read": (lambda: [_cache(True)], _rows, lambda st, c, s, l: kv_module.op_kv_read(c, s, l, 3, stream=st)[0]),
    "attention": (lambda: [_cache(False)], lambda: [_t(3, 4, 64, dtype=BF), *_rows()],
                  lambda st, c, q, s, l: kv_module.op_attention(q, c, s, l, stream=st)),
    "attention_prefix": (lambda: [_cache(False), _cache(True)], lambda: [_t(3, 4, 64, dtype=BF), *_rows(), _t(3, dtype=I32)],
                         lambda st, c, p, q, s, l, t: kv_module.op_attention(q, c, s, l, tree=t, prefix=p, stream=st)),
}


@pytest.fixture
def calls(allocations, monkeypatch):  # noqa: F811
    monkeypatch.setattr(kv_module, "_call_on", lambda dev, stream, fn, *args: 0)
    monkeypatch.setattr(kv_module, "_attention_scratch_bytes", lambda *a: 512)
    return allocations


@pytest.mark.parametrize("name", CALLS)
def test_memory_and_tensors_of_a_call_on_another_stream(calls, name):
    caches, tensors, call = CALLS[name]
    caches, tensors = caches(), tensors()
    calls.clear()
    LOG.clear()
    out = call(SIDE, *caches, *tensors)
    assert calls and all(s is SIDE for _, s in calls)
    assert ("record", out.data_ptr(), CURRENT) in LOG     # the caller goes on with it there
    used = [p for what, p, s in LOG if s is SIDE]
    assert all(t.data_ptr() in used for t in tensors + [t for c in caches for t in c.tensors if t is not None])
    calls.clear()
    LOG.clear()
    call(None, *caches, *tensors)
    assert calls and all(s is CURRENT for _, s in calls) and not LOG
