"""Pins of the sampling rules and the adapters in 64 bits, and the refusals of the calls
that implement them (which the library decides on the host, before any CUDA call)."""
import ctypes as C
import itertools
import os
import shutil

import numpy as np
import pytest

from oracle import filtering as F


def test_kept_worked_by_hand():
    # weights 8, 4, 2, 1, 1 in sixteenths of 16: ids 3, 0, 4, 1, 2
    z = np.log([4.0, 1.0, 1.0, 8.0, 2.0])
    z[2] = z[1]
    assert F.kept(z, 1.0).tolist() == [3, 0, 4, 1, 2]
    assert F.kept(z, 1.0, 4).tolist() == [3, 0, 4, 1]          # the tie goes to the lower id
    assert F.kept(z, 1.0, 0, 0.5).tolist() == [3]              # 8 of 16 are half
    assert F.kept(z, 1.0, 0, 0.51).tolist() == [3, 0]
    assert F.kept(z, 1.0, 2, 0.7).tolist() == [3, 0]           # 8 of 12 is less than 0.7
    assert F.kept(z, 1.0, 0, 1.0, 0.26).tolist() == [3, 0]
    assert F.kept(z, 1.0, 3, 0.9, 0.3).tolist() == [3, 0]
    assert F.kept(z, 0.0, 3, 0.9).tolist() == [3]
    # T = 2: weights are the square roots
    assert F.kept(z, 2.0, 0, 1.0, 0.51).tolist() == [3, 0]


def test_draw_follows_the_cumulative_weights_in_id_order():
    z = np.log([4.0, 1.0, 1.0, 8.0, 2.0])
    got = [F.draw(z, u, 1.0) for u in (0.0, 0.24, 0.26, 0.32, 0.38, 0.874, 0.876)]
    assert got == [0, 0, 1, 2, 3, 3, 4]
    assert [F.draw(z, u, 1.0, 2) for u in (0.0, 0.32, 0.34)] == [0, 0, 3]


def test_rows_without_a_finite_logit_and_odd_values():
    assert F.draw(np.full(4, -np.inf), 0.5, 1.0) == -1
    assert F.draw(np.array([np.nan, -np.inf]), 0.5, 0.0) == -1
    assert F.draw(np.array([np.nan, -3e38, -np.inf]), 0.5, 1.0) == 1
    assert F.kept(np.array([0.0, np.inf, 1.0, np.inf]), 1.0, 0, 0.6).tolist() == [1, 3]
    assert np.all(F.mask(np.full(3, -np.inf), 1.0, 2) == -np.inf)


def test_kept_mass_is_the_smallest_that_reaches_p():
    rng = np.random.default_rng(3)
    for _ in range(50):
        z = rng.normal(size=40)
        p = float(np.float32(rng.uniform(0.05, 0.99)))
        ids = F.kept(z, 0.8, 0, p)
        w = np.exp(z / float(np.float32(0.8)))
        assert w[ids].sum() >= p * w.sum() * (1 - 1e-12)
        assert w[ids[:-1]].sum() < p * w.sum()


def test_lora_oracle_is_the_merged_weight():
    rng = np.random.default_rng(4)
    x, a, b = rng.normal(size=(3, 16)), rng.normal(size=(2, 4, 16)), rng.normal(size=(2, 5, 4))
    y, size = F.lora(x, a, b, [1, -1, 0], [2.0, 0.5], [4, 3], np.ones((3, 5)))
    w = [2.0 * b[0] @ a[0], 0.5 * b[1][:, :3] @ a[1][:3]]
    np.testing.assert_allclose(y, 1 + np.stack([w[1] @ x[0], 0 * w[0] @ x[0], w[0] @ x[2]]), rtol=1e-13)
    assert np.all(size >= np.abs(y) - 1e-12)


# ------------------------------------------------------------------ refusals
needs_toolkit = pytest.mark.skipif(shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"),
                                   reason="CUDA toolkit not installed")
P = 0x10000     # an address that no call may touch


@pytest.fixture(scope="module")
def lib():
    from paper_2608_10362_gb300 import build, _lib
    build.build()
    return _lib.load()


def _rule(**kw):
    from paper_2608_10362_gb300._lib import Filter
    return Filter(**{**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **kw})


@needs_toolkit
@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(logits=P + 2), dict(rows=0), dict(rows=65536), dict(vocab=0), dict(vocab=131073),
    dict(ld=99), dict(ld=1 << 41), dict(rule=dict(temperature=-1.0)), dict(rule=dict(temperature=float("nan"))),
    dict(rule=dict(top_k=-1)), dict(rule=dict(top_p=0.0)), dict(rule=dict(top_p=1.5)),
    dict(rule=dict(top_p=float("nan"))), dict(rule=dict(min_p=-0.1)), dict(rule=dict(min_p=1.1)),
    dict(rule=dict(top_p_dev=P + 1)), dict(out=None), dict(out=P + 1), dict(u=None), dict(u=P + 3)])
def test_filter_calls_refuse(lib, bad):
    from paper_2608_10362_gb300 import _lib
    arg = {**dict(logits=P, ld=100, rows=4, vocab=100, rule={}, u=P, out=P + 0x1000), **bad}
    f = _rule(**arg["rule"])
    common = (arg["logits"], arg["ld"], arg["rows"], arg["vocab"], C.byref(f))
    assert lib.memspec_op_sample_filtered(*common, arg["u"], arg["out"], None) == _lib.ERR_INVALID_ARG
    assert lib.memspec_op_last_error()
    if "u" not in bad:
        ld = arg["vocab"] if arg["vocab"] > 100 else 100
        assert lib.memspec_op_filter_logits(*common, arg["out"], ld, None) == _lib.ERR_INVALID_ARG


@needs_toolkit
def test_filter_refuses_output_rows_that_do_not_fit(lib):
    from paper_2608_10362_gb300 import _lib
    f = _rule()
    for out, ld in ((P + 0x1000, 99), (P, 128)):    # shorter than a row; in place at another stride
        assert lib.memspec_op_filter_logits(P, 100, 4, 100, C.byref(f), out, ld, None) == _lib.ERR_INVALID_ARG
    assert lib.memspec_op_filter_logits(P, 100, 4, 100, None, P + 0x1000, 100, None) == _lib.ERR_INVALID_ARG


@needs_toolkit
@pytest.mark.parametrize("bad", [
    dict(a=None), dict(b=None), dict(x=None), dict(ids=None), dict(y=None), dict(scratch=None), dict(rows=0),
    dict(rows=257), dict(n=0), dict(n=(1 << 24) + 1), dict(k=12), dict(k=0), dict(rank=0), dict(rank=12),
    dict(rank=136), dict(adapters=0), dict(ldx=56), dict(ldx=68), dict(ldy=31), dict(ld_base=31),
    dict(base=P + 0x1000, ld_base=40), dict(x=P + 8), dict(a=P + 2), dict(b=P + 4), dict(scratch=P + 8),
    dict(y=P + 2), dict(base=P + 1), dict(ids=P + 1), dict(scales=P + 2), dict(ranks=P + 2), dict(nb=16),
    dict(adapters=(1 << 24) + 1), dict(adapters=(1 << 31) - 1), dict(ldx=1 << 41), dict(ldy=1 << 41), dict(ld_base=1 << 41)])
def test_lora_refuses(lib, bad):
    from paper_2608_10362_gb300 import _lib
    v = {**dict(a=P, b=P, x=P, ids=P, y=P + 0x1000, base=P + 0x2000, scratch=P, rows=4, n=32, k=64, rank=8, adapters=2,
                ldx=64, ldy=32, ld_base=32, scales=None, ranks=None, nb=1 << 20), **bad}
    f = _lib.Lora(v["a"], v["b"], v["scales"], v["ranks"], v["adapters"], v["rank"])
    st = lib.memspec_op_lora(C.byref(f), v["x"], v["ldx"], v["ids"], v["base"], v["ld_base"], v["y"], v["ldy"],
                             v["rows"], v["n"], v["k"], v["scratch"], v["nb"], None)
    assert st == _lib.ERR_INVALID_ARG
    assert lib.memspec_op_last_error()


@needs_toolkit
def test_lora_scratch_grows_with_the_call(lib):
    nb = C.c_size_t()
    sizes = []
    for rows, rank in itertools.product((1, 16, 256), (8, 128)):
        assert lib.memspec_op_lora_scratch_bytes(rows, 4096, 4096, rank, C.byref(nb)) == 0
        assert nb.value >= 4 * rows * rank
        sizes.append(nb.value)
    assert max(sizes) == sizes[-1]
    assert lib.memspec_op_lora_scratch_bytes(1, 1, 8, 8, None) != 0


@needs_toolkit
def test_wrappers_refuse_host_tensors(lib):
    import torch
    import paper_2608_10362_gb300 as pkg
    z, u = torch.zeros(2, 8), torch.zeros(2)
    for call in (lambda: pkg.op_sample_filtered(z, u), lambda: pkg.op_filter_logits(z),
                 lambda: pkg.op_lora(z.bfloat16(), torch.zeros(1, 8, 8).bfloat16(), torch.zeros(1, 8, 8).bfloat16(),
                                     torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()


def test_temperatures_below_the_lowest_count_as_it():
    z = np.array([0.0, -0.5, -1.0, -2.0]) * 1e-30           # weights 1, 0.61, 0.37, 0.14 at T = 1e-30
    for T in (1e-45, 1e-38, 1e-31, 1e-30):
        assert F.kept(z, T, 0, 1.0, 0.3).tolist() == [0, 1, 2]
        assert F.kept(z, T, 0, 0.7).tolist() == [0, 1]
        assert F.draw(z, 0.9, T) == 2
    assert F.kept(z, 0.0, 3).tolist() == [0]
