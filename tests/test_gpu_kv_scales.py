"""op_attention where its scale, queries, keys or values are near the ends of their types: each
product that stays in fp32 is right whatever its factors are, in both kernels.  Bounds as in
test_gpu_kv_attention.py, which count relative to scale sum|q k| and to the values."""
import math

import pytest
import torch

from test_gpu_kv_attention import DEV, _gen, _i32, _pkg, attention64, batch, check, make_cache

pytestmark = pytest.mark.gpu
HEADS = pytest.mark.parametrize("H,Hk", [(4, 4), (32, 4)], ids=["few", "many"])


def _times(cache, k=0, v=0):
    """The cache with its keys and values (of codes: their scales) times powers of two."""
    for i, e in ((0, k), (1, v)):
        t = cache.tensors[2 + i] if cache.codes else cache.tensors[i]
        t.mul_(2.0 ** (e // 2)).mul_(2.0 ** (e - e // 2))      # (2^e itself may be past fp32)
        assert torch.isfinite(t).all()
    return cache


def _attend(q, cache, starts, lens, **kw):
    for max_rows in (3, 1):
        got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=max_rows, **kw)
        check(got, *attention64(q, cache, starts, lens, max_rows=max_rows, **kw))


@HEADS
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("q_e,k_e,scale_e", [(55, 55, -110), (100, 0, -100), (-100, 0, 100), (0, -50, 50), (60, 0, -60),
                                             (0, 60, -60), (20, 100, -120), (-60, -55, 115)])
def test_scales_that_make_up_for_sizes(H, Hk, codes, q_e, k_e, scale_e):
    """Scores of size 1 from factors that are not."""
    starts, lens = batch([3, 1], [140, 20])
    cache = _times(make_cache(codes, 2, Hk, 150, 128, seed=3), k=k_e)
    q = (torch.randn(4, H, 128, device=DEV, generator=_gen(8)) * 2.0 ** q_e).bfloat16()
    _attend(q, cache, starts, lens, scale=0.09 * 2.0 ** scale_e)


@HEADS
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("scale", [0.0, 1e-38, -1e-32])
def test_small_scales_of_large_products(H, Hk, codes, scale):
    """q . k of 2^117 times 0 is 0, times 1e-38 is small: nothing stands in for the scale."""
    starts, lens = batch([3, 1], [140, 20])
    cache = _times(make_cache(codes, 2, Hk, 150, 128, seed=3), k=55)
    q = (torch.randn(4, H, 128, device=DEV, generator=_gen(8)) * 2.0 ** 55).bfloat16()
    _attend(q, cache, starts, lens, scale=scale)


@HEADS
@pytest.mark.parametrize("prefix_len", [0, 130])
@pytest.mark.parametrize("q_e,scale_e", [(-110, -15), (-20, -105), (0, -125), (-60, -65)])
def test_keys_of_the_largest_scales(H, Hk, q_e, scale_e, prefix_len):
    """Scales of K up to 2^120.2, keys up to 2^127.2: the largest that bf16 has too."""
    starts, lens = batch([3, 1], [140, 20])
    cache = _times(make_cache(True, 2, Hk, 150, 128, seed=3), k=125)
    prefix = _times(make_cache(True, 1, Hk, 150, 128, seed=4), k=125) if prefix_len else None
    assert cache.k_scale.max() > 2.0 ** 120
    q = (torch.randn(4, H, 128, device=DEV, generator=_gen(8)) * 2.0 ** q_e).bfloat16()
    _attend(q, cache, starts, lens, scale=0.09 * 2.0 ** scale_e, prefix=prefix, prefix_len=prefix_len)


@HEADS
def test_a_scale_of_0_over_the_largest_keys(H, Hk):
    """Codes never have q . k itself in fp32: 0 times 2^230 is 0."""
    starts, lens = batch([3, 1], [140, 20])
    cache = _times(make_cache(True, 2, Hk, 150, 128, seed=3), k=125)
    q = (torch.randn(4, H, 128, device=DEV, generator=_gen(8)) * 2.0 ** 100).bfloat16()
    _attend(q, cache, starts, lens, scale=0.0)


@HEADS
def test_the_largest_scale_over_keys_of_zeros(H, Hk):
    """2e38 q . 0 is 0, however large q is, and whatever the scale of a code of 0 is."""
    starts, lens = batch([3, 1], [140, 20])
    q = (torch.randn(4, H, 128, device=DEV, generator=_gen(8)) * 2.0 ** 20).bfloat16()
    for codes in (False, True):
        cache = make_cache(codes, 2, Hk, 150, 128, seed=3)
        cache.k.zero_()
        _attend(q, cache, starts, lens, scale=2e38)
        _attend(q, cache, starts, lens, scale=-2e38)
        if codes:
            cache.k_scale.fill_(2.0 ** -64)
            _attend(q, cache, starts, lens, scale=2e38)


@HEADS
@pytest.mark.parametrize("prefix_len", [0, 130])
@pytest.mark.parametrize("v_e,most", [(124, 127), (125, 127), (129, 2), (131, 1), (-58, 127)])
def test_values_of_the_largest_scales(H, Hk, v_e, most, prefix_len):
    """Scales of V up to 2^126.2 with codes that keep the values finite, and down to the smallest scale."""
    starts, lens = batch([3, 1], [140, 0])     # (the second row sees one key: its sum of weights is the least)
    cache = _times(make_cache(True, 2, Hk, 150, 128, seed=3), v=v_e)
    prefix = _times(make_cache(True, 1, Hk, 150, 128, seed=4), v=v_e) if prefix_len else None
    for c in (cache, prefix):
        if c is not None:
            c.v.clamp_(-most, most)
    q = torch.randn(4, H, 128, device=DEV, generator=_gen(8)).bfloat16()
    _attend(q, cache, starts, lens, prefix=prefix, prefix_len=prefix_len)


@HEADS
@pytest.mark.parametrize("prefix_len", [0, 130])
def test_values_at_the_end_of_bf16(H, Hk, prefix_len):
    """A weighted mean of values up to 2^126 is no larger than they are."""
    starts, lens = batch([3, 1], [140, 20])
    cache = _times(make_cache(False, 2, Hk, 150, 128, seed=3), v=123)
    prefix = _times(make_cache(False, 1, Hk, 150, 128, seed=4), v=123) if prefix_len else None
    cache.v.clamp_(-2.0 ** 126, 2.0 ** 126)
    q = (3 * torch.randn(4, H, 128, device=DEV, generator=_gen(8))).bfloat16()
    _attend(q, cache, starts, lens, prefix=prefix, prefix_len=prefix_len)


def test_read_counts_small_scales_as_attention_does():
    """A scale below 2^-64 counts as 2^-64, as the header has it."""
    pkg = _pkg()
    cache = make_cache(True, 1, 2, 8, 64, seed=3)
    cache.k_scale[:] = torch.tensor([0.0, 2.0 ** -70, 2.0 ** -64, 2.0 ** -63, -1.0, 1e-40, 0.5, math.nan], device=DEV)
    cache.v_scale[:] = cache.k_scale.flip(2)
    k, v = pkg.op_kv_read(cache, _i32(0, 8), _i32(8), 8)
    for got, codes, scale in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        s = torch.where(scale < 2.0 ** -64, torch.tensor(2.0 ** -64, device=DEV), scale)
        want = (codes.float() * s[..., None]).bfloat16()[0].transpose(0, 1)      # a product of 8 and 24 bits, rounded ...
        exact = (codes.double() * s.double()[..., None])[0].transpose(0, 1)
        ok = torch.isfinite(exact)
        assert ((got.double() - exact).abs()[ok] <= (2.0 ** -8 + 2.0 ** -24) * exact.abs()[ok]).all()   # ... to fp32, then bf16
        assert torch.equal(got[torch.isfinite(want)], want[torch.isfinite(want)])
        assert torch.isnan(got[~ok]).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_values_of_small_scales_beside_large_ones(hd):
    """Codes of many vectors a head enter as fp16: off by 2^-10 of themselves or, where fp16 runs out of bits, by what the
    header gives of the tile's largest scale.  A key's product and the subtrahend that takes 128 from its codes round at
    fp16's smallest step, 2^-24, each by half of it, of what the largest scale makes 2^-9: 2^-15 of that scale."""
    import os
    import re

    pkg = _pkg()
    header = os.path.join(os.path.dirname(os.path.dirname(pkg.__file__)), "include", "memspec_ops.h")
    with open(header) as fh:
        stated = 2.0 ** -int(re.search(r"themselves, or by 2\^-(\d+) of the", fh.read()).group(1))
    scales = torch.linspace(0, 1, 400, device=DEV).double().mul(6).sub(18).exp2().float()      # 2^-18 to 2^-12 of the largest
    n = len(scales)
    v = torch.zeros(n, 1, 2, hd, dtype=torch.int8, device=DEV)
    v[:, 0, 0] = torch.randint(-127, 128, (n, hd), device=DEV, generator=_gen(4), dtype=torch.int8)
    v_scale = torch.ones(n, 1, 2, device=DEV)
    v_scale[:, 0, 0] = scales
    cache = pkg.KVCache(torch.zeros_like(v), v, torch.ones_like(v_scale), v_scale)
    # 17 heads a row, one row a sequence, which weighs both keys alike: half of the first's value
    starts, lens = _i32(*range(n + 1)), _i32(*[2] * n)
    got = pkg.op_attention(torch.zeros(n, 17, hd, device=DEV, dtype=torch.bfloat16), cache, starts, lens, max_rows=1)
    want = 0.5 * v[:, :, 0].double() * scales.double()[:, None, None]
    bound = (2.0 ** -8 + 2.0 ** -10) * want.abs() + 0.5 * stated
    assert ((got.double() - want).abs() <= bound).all(), f"{((got.double() - want).abs() / bound).max():.2f} of the bound"
