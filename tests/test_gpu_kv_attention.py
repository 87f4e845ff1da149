"""op_kv_append, op_kv_read and op_attention against a plain implementation in 64 bits.

Bounds.  A result in bf16 is off by 2^-8 of itself.  Weights enter the product with v in 16
bits: off by 2^-8 (bf16 caches) or 2^-11 (codes) each, which moves a result by as much of
A = sum w|v| / sum w.  A score is an fp32 sum of head_dim products of magnitude S = scale sum
|q k| at most: off by (head_dim + 16) 2^-23 S (the tensor cores' sums may truncate: a whole
step each), which moves its weight, and so the result, by as much of A, twice (numerator and
denominator).  Keys and values of codes of more than 16 vectors a head enter as fp16, off by 2^-10
each, two roundings (their scales here lie within a factor of 7, so that nothing is near fp16's
small end): a score by 2^-10 S more, a result by 2^-10 A more.  Sums of weights and exponentials add (keys 2^-23 at most, in practice their
rounding averages out) 2^-18.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _pkg():
    import paper_2608_10362_gb300 as pkg
    return pkg


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def make_cache(codes, seqs, heads, positions, hd, seed=0, layout="bhsd"):
    g = _gen(seed)
    shape = {"bhsd": (seqs, heads, positions, hd), "bshd": (seqs, positions, heads, hd)}[layout]
    view = (lambda t: t) if layout == "bhsd" else (lambda t: t.transpose(1, 2))
    if not codes:
        return _pkg().KVCache(*(view(torch.randn(shape, device=DEV, generator=g).bfloat16()) for _ in (0, 1)))
    c = [view(torch.randint(-127, 128, shape, device=DEV, generator=g, dtype=torch.int8)) for _ in (0, 1)]
    s = [view(0.005 + 0.03 * torch.rand(*shape[:3], 1, device=DEV, generator=g))[..., 0] for _ in (0, 1)]
    return _pkg().KVCache(*c, *s)


def values(cache):
    k, v = cache.k.double(), cache.v.double()
    if cache.codes:
        k, v = k * cache.k_scale.double()[..., None], v * cache.v_scale.double()[..., None]
    return k, v


def attention64(q, cache, starts, lens, tree=None, prefix=None, prefix_len=0, scale=None, max_rows=None):
    """(result, bound) of every row, NaN where the row is in no sequence."""
    rows, H, hd = q.shape
    G = H // cache.n_heads
    scale = 1 / math.sqrt(hd) if scale is None else scale
    out = torch.full(q.shape, math.nan, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    kk, vv = values(cache)
    if prefix is not None:
        pk, pv = values(prefix)
    for b in range(len(lens)):
        lo, hi, L = starts[b], starts[b + 1], lens[b]
        n = hi - lo
        if n == 0:
            continue
        end = max(0, min(L, cache.max_pos))
        at = torch.arange(end, device=q.device)[None]
        first = L - n
        if tree is None:
            seen = at <= first + torch.arange(n, device=q.device)[:, None]
        else:
            bits = tree[lo:hi].long()[:, None] & 0xFFFFFFFF
            d = at - first
            seen = (at < first) | ((d >= 0) & (d < 32) & ((bits >> d.clamp(0, 31)) & 1 > 0))
        for h in range(cache.n_heads):
            k, v, s = kk[b, h, :end], vv[b, h, :end], seen
            if prefix is not None:
                k, v = torch.cat([pk[0, h, :prefix_len], k]), torch.cat([pv[0, h, :prefix_len], v])
                s = torch.cat([torch.ones(n, prefix_len, dtype=torch.bool, device=q.device), s], 1)
            x = q[lo:hi, h * G:(h + 1) * G].double()
            s = s[:, None].expand(n, G, s.shape[1])
            z = torch.where(s, torch.einsum("ngd,kd->ngk", x, k.nan_to_num(0, 0, 0)) * scale, -math.inf)
            any_ = s.any(2, keepdim=True)
            w = torch.where(any_, torch.softmax(torch.where(any_, z, 0.0), 2), 0.0)
            # a value that a row does not see does not count, whatever it is
            clean = v.nan_to_num(0, 0, 0)
            bad = (~torch.isfinite(v)).any(1) | (~torch.isfinite(k)).any(1)
            r = w @ clean
            r = torch.where((s & bad[None, None]).any(2, keepdim=True), math.nan, r)
            out[lo:hi, h * G:(h + 1) * G] = r
            A = w @ clean.abs()
            S = torch.where(s, torch.einsum("ngd,kd->ngk", x.abs(), k.nan_to_num(0, 0, 0).abs()) * abs(scale), 0.0)
            S = S.amax(2, keepdim=True) if S.shape[2] else S.sum(2, keepdim=True)
            weights = 2.0 ** -11 if cache.codes and (prefix is None or prefix.codes) else 2.0 ** -8
            many = max((max_rows or rows) if cache.codes else 0, rows if prefix is not None and prefix.codes else 0) * G > 16
            values16 = 2.0 ** -10 if many else 0.0
            bound[lo:hi, h * G:(h + 1) * G] = (2.0 ** -8 * (r.abs().nan_to_num(0) + weights * A)
                                               + (weights + values16 + 2 * ((hd + 16) * 2.0 ** -23 + values16) * S
                                                  + 2.0 ** -18) * A + 1e-30)
    return out, bound


def check(got, want, bound):
    """Rows of no sequence are not looked at; a NaN stands where one is wanted."""
    rows = ~torch.isnan(want)
    off = (got.double() - want).abs()
    assert torch.isfinite(got.double()[rows]).all()
    worst = (off[rows] / bound[rows]).max().item() if rows.any() else 0.0
    assert worst <= 1.0, f"off by {worst:.2f} of the bound"


def batch(rows_of, pasts):
    starts = np.concatenate([[0], np.cumsum(rows_of)]).astype(int)
    return list(map(int, starts)), [int(p + n) for p, n in zip(pasts, rows_of)]


SHAPES = [
    # heads, kv heads, head_dim, rows of each sequence, positions before them
    (1, 1, 64, [1], [0]),
    (4, 4, 128, [1], [1]),
    (8, 2, 128, [1, 1, 1], [126, 127, 128]),
    (32, 8, 128, [9] * 4, [511, 0, 77, 1200]),
    (32, 32, 128, [5], [2048]),
    (32, 4, 64, [21], [1003]),
    (40, 8, 128, [3, 0, 7, 1], [5, 900, 33, 15]),
    (6, 2, 128, [100, 28], [3, 250]),
    (16, 8, 64, [256], [300]),
    (6, 2, 64, [1] * 67, list(range(67))),
    (64, 1, 128, [2, 1], [63, 200]),
    (12, 12, 64, [2, 0, 0, 4], [16, 16, 16, 15]),
    (32, 8, 128, [1] * 8, [3000, 17, 4000, 1, 0, 2500, 129, 640]),
]


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}_{len(s[3])}seqs_{max(s[3])}rows_{max(s[4])}")
def test_attention_follows_the_definition(shape, codes):
    H, Hk, hd, rows_of, pasts = shape
    starts, lens = batch(rows_of, pasts)
    cache = make_cache(codes, len(lens), Hk, max(lens) + 3, hd, seed=H + hd)
    q = 2 * torch.randn(starts[-1], H, hd, device=DEV, generator=_gen(5))
    q = q.bfloat16()
    for max_rows in {max(rows_of), starts[-1]}:
        got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=max_rows)
        check(got, *attention64(q, cache, starts, lens, max_rows=max_rows))


@pytest.mark.parametrize("codes,pcodes", [(False, False), (True, True), (False, True), (True, False)])
@pytest.mark.parametrize("prefix_len", [1, 127, 1000])
@pytest.mark.parametrize("shape", [SHAPES[2], SHAPES[3], SHAPES[5], SHAPES[6], SHAPES[8]],
                         ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}_{len(s[3])}seqs")
def test_attention_behind_a_prefix(shape, codes, pcodes, prefix_len):
    H, Hk, hd, rows_of, pasts = shape
    starts, lens = batch(rows_of, pasts)
    cache = make_cache(codes, len(lens), Hk, max(lens) + 1, hd, seed=1)
    prefix = make_cache(pcodes, 2, Hk, prefix_len + 2, hd, seed=2)
    q = (2 * torch.randn(starts[-1], H, hd, device=DEV, generator=_gen(6))).bfloat16()
    got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=max(rows_of), prefix=prefix,
                              prefix_len=prefix_len)
    check(got, *attention64(q, cache, starts, lens, prefix=prefix, prefix_len=prefix_len, max_rows=max(rows_of)))
