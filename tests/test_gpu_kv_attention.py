"""op_kv_append, op_kv_read and op_attention against a plain implementation in 64 bits.

Bounds.  A result in bf16 is off by 2^-8 of itself.  Weights enter the product with v in 16
bits: off by 2^-8 (bf16 caches) or 2^-11 (codes) each, which moves a result by as much of
A = sum w|v| / sum w.  A score is an fp32 sum of head_dim products of magnitude S = scale sum
|q k| at most: off by (head_dim + 16) 2^-23 S (the tensor cores' sums may truncate: a whole
step each), which moves its weight, and so the result, by as much of A, twice (numerator and
denominator).  Keys and values of codes of more than 16 vectors a head enter as fp16, off by 2^-10
each (two roundings) or, where fp16 runs out (2^-25 of what the tile's largest scale makes 2^-9), by 2^-16 of the
largest scale: a score by 2^-10 S + 2^-16 scale sum|q| more, a result by 2^-10 A + 2^-16 scale more.  Weights of codes are fp16 that carry v's
scale too, the largest at least 2^6 (the maximum is taken again when it is passed by 2^14, and then set
2^6 below): what rounds at fp16's smallest step, 2^-24, is off by 2^-25, 2^-31 of the largest, so a
result by 2^-31 of the largest |v| for each key.  Sums of weights and exponentials add (keys 2^-23 at most, in practice their
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
    if cache.codes:   # a scale below 2^-64 counts as 2^-64
        k, v = (t * s.double().clamp(min=2.0 ** -64)[..., None] for t, s in ((k, cache.k_scale), (v, cache.v_scale)))
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
            if many:
                ends = [(c, e) for c, e in ((cache if cache.codes else None, end),
                                            (prefix if prefix is not None and prefix.codes else None, prefix_len)) if c and e]
                tops = [max(float(t[b if c is cache else 0, h, :e].nan_to_num(0, 0, 0).max()) for c, e in ends
                            for t in (c.tensors[i],)) if ends else 0.0 for i in (2, 3)]
                bound[lo:hi, h * G:(h + 1) * G] += 2.0 ** -16 * (
                    2 * tops[0] * abs(scale) * x.abs().nan_to_num(0).sum(2, keepdim=True) * A + tops[1])
            if cache.codes or prefix is not None and prefix.codes:
                bound[lo:hi, h * G:(h + 1) * G] += 2.0 ** -31 * clean.shape[0] * (clean.abs().max() if clean.numel() else 0.0)
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


# ------------------------------------------------------------------ masks and what lies behind them
@pytest.mark.parametrize("heads", [(8, 8, 64), (8, 2, 128), (32, 4, 128)], ids=str)
@pytest.mark.parametrize("codes", [False, True])
def test_trees_and_rows_that_see_nothing(heads, codes):
    H, Hk, hd = heads
    rng = np.random.default_rng(3)
    rows_of, pasts = [32, 7, 5, 1], [70, 0, 129, 0]
    starts, lens = batch(rows_of, pasts)
    bits = rng.integers(0, 1 << 32, starts[-1], dtype=np.uint32)
    bits[33] = 0                    # a sequence without a past: its row sees nothing
    bits[starts[3]] = 0
    bits[5] = 0                     # ... or the past alone
    tree = torch.from_numpy(bits.view(np.int32)).to(DEV)
    cache = make_cache(codes, 4, Hk, max(lens) + 40, hd, seed=9)
    q = torch.randn(starts[-1], H, hd, device=DEV, generator=_gen(1)).bfloat16()
    for max_rows in (32, 1):
        got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=max_rows, tree=tree)
        want, bound = attention64(q, cache, starts, lens, tree=tree, max_rows=max_rows)
        check(got, want, bound)
        assert not got[33].any() and not got[starts[3]].any()


@pytest.mark.parametrize("H,Hk", [(4, 4), (32, 4)])
@pytest.mark.parametrize("codes", [False, True])
def test_lengths_shorter_than_the_rows(H, Hk, codes):
    """Rows whose slots are before the first see nothing; a length past the cache is the cache's."""
    hd, starts, lens = 128, [0, 5, 8, 12], [2, 0, 1000]
    cache = make_cache(codes, 3, Hk, 40, hd, seed=4)
    q = torch.randn(12, H, hd, device=DEV, generator=_gen(2)).bfloat16()
    got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=5)
    want, bound = attention64(q, cache, starts, lens, max_rows=5)
    check(got, want, bound)
    assert not got[:3].any() and not got[5:8].any()


@pytest.mark.parametrize("H,Hk,hd", [(4, 4, 128), (8, 2, 64), (32, 4, 128), (32, 4, 64), (64, 1, 128)])
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_reach_it(H, Hk, hd, codes, what):
    """Slots past the length, and slots of later rows, hold infinities and NaN: rows that see none of
    them are as if they were not there, rows that do are not checked."""
    rows_of, pasts = [4, 6], [125, 256]
    starts, lens = batch(rows_of, pasts)
    cache = make_cache(codes, 2, Hk, max(lens) + 60, hd, seed=7)
    clean = [t.clone() for t in cache.tensors if t is not None]
    q = torch.randn(10, H, hd, device=DEV, generator=_gen(8)).bfloat16()
    want, bound = attention64(q, _pkg().KVCache(*clean), starts, lens, max_rows=6)
    bad = {0: 2, 1: 4}              # the first row of the sequence whose own slot is spoilt
    for b, L in enumerate(lens):
        first = L - rows_of[b] + bad[b]
        for t in (cache.tensors[2:] if codes else cache.tensors[:2]):
            t[b, :, first:] = what
    for max_rows in (6, 1):
        got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=max_rows)
        for b in (0, 1):
            rows = slice(starts[b], starts[b] + bad[b])
            check(got[rows], want[rows], bound[rows])
            if math.isnan(what):    # a NaN that is seen is not lost
                assert torch.isnan(got[starts[b] + bad[b]:starts[b + 1]].float()).all()


def test_values_alone_that_are_not_finite():
    """Only V is spoilt, at one element of one later row's slot; K is finite everywhere."""
    starts, lens = [0, 6], [200]
    for H, Hk in ((6, 6), (48, 6)):
        cache = make_cache(False, 1, Hk, 260, 128, seed=3)
        q = torch.randn(6, H, 128, device=DEV, generator=_gen(8)).bfloat16()
        want, bound = attention64(q, cache, starts, lens)
        cache.v[0, 1, 197, 77] = math.inf
        got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens))
        G = H // Hk
        check(got[:3], want[:3], bound[:3])
        others = [h for h in range(H) if h // G != 1]
        check(got[:, others], want[:, others], bound[:, others])
        assert not torch.isfinite(got[3:, G:2 * G].float()).all(2).any()


def test_a_row_with_nan_spoils_no_other():
    for H, Hk, codes in ((4, 4, False), (4, 4, True), (32, 4, False), (32, 4, True)):
        starts, lens = [0, 5], [300]
        cache = make_cache(codes, 1, Hk, 300, 128, seed=3)
        q = torch.randn(5, H, 128, device=DEV, generator=_gen(8)).bfloat16()
        want, bound = attention64(q, cache, starts, lens)
        q[2, 1, 5], q[3, 0] = math.nan, math.inf
        got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens))
        keep = torch.ones(5, H, dtype=torch.bool, device=DEV)
        keep[2, 1] = keep[3, 0] = False
        check(got[keep], want[keep], bound[keep])


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0, 1e-3])
@pytest.mark.parametrize("H,Hk,codes", [(4, 4, False), (4, 4, True), (32, 4, False), (32, 4, True)])
def test_scales_of_any_sign(H, Hk, codes, scale):
    starts, lens = batch([3, 6], [140, 20])
    cache = make_cache(codes, 2, Hk, 150, 128, seed=3)
    q = torch.randn(9, H, 128, device=DEV, generator=_gen(8)).bfloat16()
    got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), scale=scale)
    check(got, *attention64(q, cache, starts, lens, scale=scale))


@pytest.mark.parametrize("H,Hk", [(4, 4), (32, 4)])
def test_codes_whose_scales_are_far_apart(H, Hk):
    """From sequence to sequence and from tile to tile scales differ by powers that fp16 does not hold; within
    a tile by 2^10, where a value still has 2^-10 of itself."""
    seqs, L, hd = 3, 400, 128
    starts, lens = batch([2] * seqs, [L - 2] * seqs)
    cache = make_cache(True, seqs, Hk, L, hd, seed=6)
    power = torch.tensor([-60.0, 0.0, 40.0], device=DEV)[:, None, None] + 5 * (torch.arange(L, device=DEV) // 128)
    cache.v_scale.mul_(torch.exp2(power))
    cache.v_scale[:, :, ::7] *= 2.0 ** -10
    cache.k_scale[:, :, ::5] *= 2.0 ** -10
    q = torch.randn(2 * seqs, H, hd, device=DEV, generator=_gen(8)).bfloat16()
    got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens))
    check(got, *attention64(q, cache, starts, lens))


def test_queries_of_any_size():
    """fp16 does not hold what bf16 holds; products do."""
    starts, lens = batch([3], [140])
    for H, Hk in ((4, 4), (32, 4)):
        for size in (2.0 ** -60, 2.0 ** 60):
            cache = make_cache(True, 1, Hk, 150, 128, seed=3)
            q = (torch.randn(3, H, 128, device=DEV, generator=_gen(8)) * size).bfloat16()
            got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), scale=0.1 / size)
            check(got, *attention64(q, cache, starts, lens, scale=0.1 / size))


# ------------------------------------------------------------------ memory
@pytest.mark.parametrize("H,Hk", [(8, 8), (32, 4)])
@pytest.mark.parametrize("codes", [False, True])
def test_caches_and_rows_of_any_strides(H, Hk, codes):
    hd, rows_of, pasts = 128, [2, 0, 9], [130, 20, 64]
    starts, lens = batch(rows_of, pasts)
    q = torch.randn(starts[-1], 2 * H, hd, device=DEV, generator=_gen(8)).bfloat16()
    for kind in ("bshd", "wide", "kv together", "one head for all", "one sequence for all"):
        cache = make_cache(codes, 4, Hk, 160, hd, seed=5, layout="bshd" if kind == "bshd" else "bhsd")
        if kind == "wide":
            cut = [t[1:, :, 8:152] for t in cache.tensors if t is not None]
            cache = _pkg().KVCache(*cut)
        elif kind == "kv together":
            both = torch.stack([cache.k, cache.v], 2)
            scales = [] if not codes else list(torch.stack([cache.k_scale, cache.v_scale], 3).unbind(3))
            cache = _pkg().KVCache(both[:, :, 0], both[:, :, 1], *scales)
        elif kind != "bshd":
            dim = 1 if kind == "one head for all" else 0
            cut = [t.narrow(dim, 0, 1).expand(*t.shape[:dim], t.shape[dim], *t.shape[dim + 1:]) for t in cache.tensors
                   if t is not None]
            cache = _pkg().KVCache(*cut)
        x = q[:, H:] if kind == "wide" else q[:, :H]
        out = torch.full((starts[-1], H + 3, hd), 7.0, device=DEV, dtype=torch.bfloat16)
        got = _pkg().op_attention(x, cache, _i32(*starts), _i32(*lens), max_rows=9, out=out[:, 1:H + 1])
        check(got, *attention64(x, cache, starts, lens, max_rows=9))
        assert (out[:, 0] == 7).all() and (out[:, H + 1:] == 7).all()


@pytest.mark.parametrize("H,Hk", [(2, 2), (16, 2)])
@pytest.mark.parametrize("codes", [False, True])
def test_offsets_past_32_bits(H, Hk, codes):
    """Heads, positions and sequences more than 2^32 elements apart."""
    hd, far = 64, (1 << 32) // 64 + 3
    big = torch.empty(2 * far * 64 + (1 << 16), dtype=torch.int8 if codes else torch.bfloat16, device=DEV)
    L = 150
    # [2 sequences][2 heads][positions]: sequences far apart, heads interleaved by position
    view = lambda at: big.as_strided((2, 2, L, hd), (far * 64, hd, 4 * hd, 1), at)
    k, v = view(0), view(2 * hd)
    src = make_cache(codes, 2, 2, L, hd, seed=2)
    k.copy_(src.k), v.copy_(src.v)
    cache = _pkg().KVCache(k, v, *([] if not codes else [src.k_scale, src.v_scale]))
    starts, lens = batch([1, 3], [100, 147])
    q = torch.randn(4, H, hd, device=DEV, generator=_gen(8)).bfloat16()
    got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens))
    check(got, *attention64(q, src, starts, lens))


def test_rows_of_no_sequence_are_left():
    for H, Hk, prefix in ((4, 4, None), (32, 4, None), (32, 4, 50)):
        cache = make_cache(False, 2, Hk, 100, 64, seed=1)
        pre = None if prefix is None else make_cache(False, 1, Hk, prefix, 64, seed=2)
        q = torch.randn(9, H, 64, device=DEV, generator=_gen(8)).bfloat16()
        out = torch.full_like(q, 5.0)
        starts, lens = [1, 3, 6], [60, 9]
        _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), prefix=pre, out=out)
        assert (out[0] == 5).all() and (out[6:] == 5).all()
        want, bound = attention64(q[1:6].contiguous(), cache, [0, 2, 5], lens, prefix=pre, prefix_len=prefix or 0)
        check(out[1:6], want, bound)


def test_starts_that_make_no_sense_touch_nothing_else():
    """What the device's arrays hold cannot be refused: rows outside the call do not count."""
    cache = make_cache(False, 3, 4, 100, 64, seed=1)
    q = torch.randn(6, 32, 64, device=DEV, generator=_gen(8)).bfloat16()
    for starts, lens in (([0, 2, 4, 900], [50, 60, 70]), ([0, 4, 2, 6], [50, 60, 70]), ([-7, 2, 4, 6], [50, -3, 1 << 30])):
        out = torch.full((8, 32, 64), 5.0, device=DEV, dtype=torch.bfloat16)
        for max_rows in (6, 1):
            _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=max_rows, out=out[1:7])
        torch.cuda.synchronize()
        assert (out[0] == 5).all() and (out[7] == 5).all() and torch.isfinite(out.float()).all()


@pytest.mark.parametrize("H,Hk,codes,prefix", [(4, 4, False, 0), (4, 4, True, 90), (32, 4, False, 300), (32, 4, True, 300)])
def test_repeated_calls_and_shared_graphs(H, Hk, codes, prefix):
    """The same bits again and again; two captured graphs of different calls that share one scratch, replayed in
    turn on one stream, and eager calls between them."""
    pkg = _pkg()
    starts, lens = batch([3, 9, 1], [700, 20, 333])
    cache = make_cache(codes, 3, Hk, 720, 128, seed=1)
    pre = make_cache(codes, 1, Hk, prefix, 128, seed=2) if prefix else None
    q = [torch.randn(13, H, 128, device=DEV, generator=_gen(s)).bfloat16() for s in (1, 2)]
    s, l = _i32(*starts), _i32(*lens)
    scratch = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    call = lambda x, out: pkg.op_attention(x, cache, s, l, max_rows=9, prefix=pre, out=out, scratch=scratch)
    want = [call(x, torch.empty_like(x)).clone() for x in q]
    outs, graphs = [torch.empty_like(x) for x in q], []
    for x, out in zip(q, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(x, out)
        graphs.append(g)
    for _ in range(20):
        for i in (0, 1):
            outs[i].zero_()
            graphs[i].replay()
            again = call(q[1 - i], torch.empty_like(q[0]))
            assert torch.equal(outs[i], want[i]) and torch.equal(again, want[1 - i])
    l.sub_(1)                                  # lengths are read at replay
    graphs[0].replay()
    shorter = [n - 1 for n in lens]
    check(outs[0], *attention64(q[0], cache, starts, shorter, prefix=pre, prefix_len=prefix, max_rows=9))


def test_calls_on_other_streams_at_once():
    pkg = _pkg()
    starts, lens = batch([9] * 8, [500] * 8)
    cache = make_cache(True, 8, 4, 512, 128, seed=1)
    s, l = _i32(*starts), _i32(*lens)
    q = torch.randn(72, 32, 128, device=DEV, generator=_gen(1)).bfloat16()
    want = pkg.op_attention(q, cache, s, l, max_rows=9)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [pkg.op_attention(q, cache, s, l, max_rows=9, stream=streams[i % 3]) for i in range(9)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


# ------------------------------------------------------------------ the cache
def append64(x, starts, lens, H, Hk, hd, positions_of=None, rope=None, gains=None, eps=1e-5, prefix=0, offsets=None):
    """q, k, v of every row in 64 bits."""
    rows = x.shape[0]
    x = x.double().view(rows, H + 2 * Hk, hd)
    parts = list(x.split([H, Hk, Hk], 1))
    if gains is not None:
        for i in (0, 1):
            parts[i] = parts[i] / (parts[i].square().mean(2, keepdim=True) + eps).sqrt() * gains[i].double()
    if rope is not None:
        pos = torch.zeros(rows, dtype=torch.long, device=x.device)
        for b in range(len(lens)):
            n = starts[b + 1] - starts[b]
            for j in range(n):
                pos[starts[b] + j] = prefix + lens[b] - n + (j if offsets is None else int(offsets[starts[b] + j]))
        pos = pos.clamp(0, rope.shape[1] - 1)
        c, s = rope[0].double()[pos][:, None], rope[1].double()[pos][:, None]
        for i in (0, 1):
            lo, hi = parts[i][..., :hd // 2], parts[i][..., hd // 2:]
            parts[i] = torch.cat([lo * c - hi * s, lo * s + hi * c], 2)
    return parts


def append_bound(parts, hd):
    """fp32 arithmetic before the rounding: a norm's sum of hd squares in a tree (8 + 3 roundings of 2^-24), a
    square root's reciprocal (2^-22), three products, a turn of two products and a sum: within 2^-20 of the
    vector's largest pair, taken as its 2-norm over the pair."""
    out = []
    for p in parts:
        lo, hi = p[..., :hd // 2], p[..., hd // 2:]
        r = (lo.square() + hi.square()).sqrt()
        out.append(2.0 ** -20 * torch.cat([r, r], 2) + 1e-30)
    return out


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("bf16_in", [False, True])
@pytest.mark.parametrize("H,Hk,hd", [(1, 1, 64), (32, 8, 128), (32, 4, 64), (40, 40, 128), (6, 2, 128)])
@pytest.mark.parametrize("full", [False, True])
def test_append_and_read(H, Hk, hd, bf16_in, codes, full):
    pkg = _pkg()
    rows_of, pasts = [5, 0, 1, 30, 2], [0, 9, 33, 7, 62]
    starts, lens = batch(rows_of, pasts)
    rows = starts[-1]
    wide = torch.randn(rows, (H + 2 * Hk) * hd + 6, device=DEV, generator=_gen(1)) * 1.7
    if bf16_in:
        wide = wide.bfloat16()
    x = wide[:, 4:-2]
    cache = pkg.KVCache.zeros(6, Hk, 64, hd, dtype=torch.int8 if codes else torch.bfloat16)
    for t in cache.tensors:
        if t is not None:
            t.fill_(3)
    rope = pkg.op_rope_table(200, hd) if full else None
    gains = [(1 + 0.3 * torch.randn(hd, device=DEV, generator=_gen(i))).bfloat16() for i in (2, 3)] if full else None
    offsets = torch.randint(0, 6, (rows,), device=DEV, generator=_gen(4), dtype=torch.int32) if full else None
    q = pkg.op_kv_append(x, cache, _i32(*starts), _i32(*lens), H, rope=rope, offsets=offsets, prefix_len=100 if full else 0,
                         q_gain=gains[0] if full else None, k_gain=gains[1] if full else None, eps=1e-5)
    parts = append64(x.float(), starts, lens, H, Hk, hd, rope=rope, gains=gains, prefix=100, offsets=offsets)
    bounds = append_bound(parts, hd)
    off = (q.double() - parts[0]).abs()
    assert (off <= 2.0 ** -8 * parts[0].abs() + 1.01 * bounds[0]).all()
    kr, vr = pkg.op_kv_read(cache, _i32(*starts), _i32(*lens), rows)
    touched = torch.zeros(6, 64, dtype=torch.bool, device=DEV)
    for b in range(5):
        for j in range(rows_of[b]):
            r, slot = starts[b] + j, pasts[b] + j
            touched[b, slot] = True
            for which, t, got in ((1, cache.k, kr), (2, cache.v, vr)):
                want, bound = parts[which][r], bounds[which][r]
                if codes:
                    scale = (cache.k_scale if which == 1 else cache.v_scale)[b, :, slot].double()
                    top = want.abs().amax(1)
                    # the scale is the largest over 127, rounded once more; a code is the nearest whole number
                    assert ((scale * 127 - top).abs() <= 2.0 ** -19 * top).all()
                    held = t[b, :, slot].double()
                    assert held.abs().amax(1).eq(127).all()
                    assert ((held * scale[:, None] - want).abs() <= (0.5 + 2.0 ** -14) * scale[:, None] + 1.01 * bound).all()
                    assert ((got[r].double() - held * scale[:, None]).abs() <= 2.0 ** -8 * (held * scale[:, None]).abs()).all()
                else:
                    assert ((t[b, :, slot].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * bound).all()
                    assert torch.equal(got[r], t[b, :, slot])
    for t in cache.tensors:
        if t is not None:                      # nothing else was written
            assert (t.transpose(1, 2)[~touched] == 3).all()


def test_rows_out_of_range_leave_the_cache():
    """Slots before the first and past the last, positions past the table, rows of no sequence."""
    pkg = _pkg()
    H, Hk, hd, starts, lens = 4, 2, 64, [1, 5, 8, 9], [2, 41, 17]
    x = torch.randn(12, (H + 2 * Hk) * hd, device=DEV, generator=_gen(1))
    rope = pkg.op_rope_table(40, hd)
    offsets = torch.zeros(12, dtype=torch.int32, device=DEV)
    offsets[8] = 60                            # position 16 + 60
    for codes in (False, True):
        cache = pkg.KVCache.zeros(3, Hk, 40, hd, dtype=torch.int8 if codes else torch.bfloat16)
        q = torch.full((12, H, hd), 9.0, device=DEV, dtype=torch.bfloat16)
        pkg.op_kv_append(x, cache, _i32(*starts), _i32(*lens), H, rope=rope, offsets=offsets, q=q)
        assert (q[0] == 9).all() and (q[9:] == 9).all()
        zero = [1, 2, 3, 4, 7, 8]              # positions -2 (offsets are 0), slot 40, a position without an angle
        for r in range(1, 9):
            assert q[r].any().item() == (r not in zero)
        wrote = cache.k.transpose(1, 2).flatten(2).any(2)
        assert wrote.nonzero().tolist() == [[1, 38], [1, 39]]
        pkg.op_kv_append(x, cache, _i32(*starts), _i32(*lens), H, q=q)
        zero = [1, 2, 7]                       # slots -2, -1 and 40; without a table every position is one
        for r in range(1, 9):
            assert q[r].any().item() == (r not in zero)
        wrote = cache.k.transpose(1, 2).flatten(2).any(2)
        assert wrote.nonzero().tolist() == [[0, 0], [0, 1], [1, 38], [1, 39], [2, 16]]
        k, v = (torch.full((12, Hk, hd), 9.0, device=DEV, dtype=torch.bfloat16) for _ in (0, 1))
        pkg.op_kv_read(cache, _i32(*starts), _i32(*lens), 12, k=k, v=v)
        assert (k[0] == 9).all() and (v[9:] == 9).all() and not k[[1, 2, 7]].any() and k[3].any()


def test_vectors_that_codes_do_not_hold():
    """Zeros, the smallest and largest numbers, infinities and NaN: each stays in its own vector."""
    pkg = _pkg()
    x = torch.randn(1, 8 * 64, device=DEV, generator=_gen(1))
    v = x.view(8, 64)                          # 2 q, 3 k, 3 v heads
    v[2] = 0.0
    v[3] *= 1e-37
    v[4, 9] = math.nan
    v[5] *= 1e36
    v[6, 3] = -math.inf
    cache = pkg.KVCache.zeros(1, 3, 4, 64, dtype=torch.int8)
    pkg.op_kv_append(x, cache, _i32(0, 1), _i32(1), 2)
    k, val = pkg.op_kv_read(cache, _i32(0, 1), _i32(1), 1)
    assert not k[0, 0].any() and not k[0, 1].any() and cache.k_scale[0, 0, 0].item() == 2.0 ** -64
    assert not torch.isfinite(k[0, 2].float()).any()
    assert ((val[0, 0].double() - v[5].double()).abs() <= 0.51 * v[5].abs().max() / 127 + 2.0 ** -8 * v[5].abs().double()).all()
    assert not torch.isfinite(val[0, 1].float()).any()
    assert ((val[0, 2].double() - v[7].double()).abs() <= 0.51 * v[7].abs().max() / 127 + 2.0 ** -8 * v[7].abs().double()).all()


def test_rope_table_of_far_positions():
    t = _pkg().op_rope_table(1 << 20, 64, 1e6)
    pos = np.array([0, 1, 777777, (1 << 20) - 1])
    angle = pos[:, None] * 1e6 ** (-np.arange(0, 64, 2) / 64)
    got = t[:, torch.from_numpy(pos).to(DEV)].cpu().numpy()
    # an angle of up to 2^20 in 64 bits is off by 2^-32, cos and sin of it rounded once
    assert np.abs(got[0] - np.cos(angle)).max() <= 2.0 ** -24 + 2.0 ** -31
    assert np.abs(got[1] - np.sin(angle)).max() <= 2.0 ** -24 + 2.0 ** -31


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("codes", [False, True])
def test_decoding_row_by_row_is_one_pass(codes):
    """A layer as it is used: projection, norms and rotation into the cache, attention, O projection; a sequence
    taken at once and taken in pieces behind a shared prefix give the same up to their roundings."""
    pkg = _pkg()
    H, Hk, hd, d, total, cut = 8, 2, 64, 256, 90, 64
    width = (H + 2 * Hk) * hd
    x = torch.randn(total, d, device=DEV, generator=_gen(1)).bfloat16()
    w = (torch.randn(width, d, device=DEV, generator=_gen(2)) * d ** -0.5).bfloat16()
    wo = (torch.randn(d, H * hd, device=DEV, generator=_gen(3)) * (H * hd) ** -0.5).bfloat16()
    gains = [(1 + 0.2 * torch.randn(hd, device=DEV, generator=_gen(i))).bfloat16() for i in (4, 5)]
    rope = pkg.op_rope_table(128, hd)
    dtype = torch.int8 if codes else torch.bfloat16

    def layer(rows, cache, lens, prefix=None):
        qkv = pkg.op_linear(rows, w)
        s, l = _i32(0, rows.shape[0]), _i32(lens)
        q = pkg.op_kv_append(qkv, cache, s, l, H, rope=rope, prefix_len=prefix.max_pos if prefix else 0,
                             q_gain=gains[0], k_gain=gains[1])
        o = pkg.op_attention(q, cache, s, l, prefix=prefix)
        return o, pkg.op_linear(o.view(rows.shape[0], H * hd), wo)

    at_once = pkg.KVCache.zeros(1, Hk, total, hd, dtype=dtype)
    want, want_y = layer(x, at_once, total)
    prefix = pkg.KVCache(*[t[:, :, :cut] for t in at_once.tensors if t is not None])
    cache = pkg.KVCache.zeros(1, Hk, total - cut, hd, dtype=dtype)
    got, got_y, n = [], [], 0
    for rows in (1, 1, 5, 9, 1, 9):
        o, y = layer(x[cut + n:cut + n + rows], cache, n + rows, prefix=prefix)
        got.append(o), got_y.append(y)
        n += rows
    got, got_y = torch.cat(got), torch.cat(got_y)
    # op_linear of other row counts differs in the last bits: bf16 and code borders are crossed here and there, so a
    # few units of the largest step: 2^-7 (a code: 1/127 of a vector's largest) of typical sizes
    assert (got.double() - want[cut:].double()).abs().max() <= 2.0 ** -4 * want.abs().max()
    assert (got.double() - want[cut:].double()).norm() <= 2.0 ** -7 * want[cut:].double().norm()
    assert (got_y - want_y[cut:]).norm() <= 2.0 ** -7 * want_y[cut:].norm()


def test_the_engines_own_cache():
    """A layer of an engine's cache is a KVCache: attention over it is attention over what prefill left there."""
    from seeded_inputs import SHAPES, gen_weights
    pkg = _pkg()
    shape = SHAPES["tiny_target"]
    eng = pkg.Engine(shape, gen_weights(shape, 1), max_seq=128)
    prompt = np.random.default_rng(0).integers(0, shape.vocab, 70)
    eng.prefill(0, prompt)
    eng.sync()
    for layer in (0, shape.n_layers - 1):
        cache = eng.kv_cache(layer)
        assert cache.k.shape == (1, shape.n_kv_heads, 128, shape.head_dim)
        assert cache.k[0, :, :69].float().abs().amax(2).min() > 0     # every position but the last has been processed
        q = torch.randn(3, shape.n_heads, shape.head_dim, device=DEV, generator=_gen(1)).bfloat16()
        got = pkg.op_attention(q, cache, _i32(0, 3), _i32(69))
        check(got, *attention64(q, cache, [0, 3], [69]))
    with pytest.raises(ValueError, match="layer"):
        eng.kv_cache(shape.n_layers)
    eng.close()


# ------------------------------------------------------------------ refusals of the wrappers
def test_wrappers_refuse():
    pkg = _pkg()
    cache = make_cache(False, 2, 2, 16, 64)
    q = torch.zeros(3, 4, 64, device=DEV, dtype=torch.bfloat16)
    s, l = _i32(0, 1, 3), _i32(4, 5)
    ok = lambda **kw: pkg.op_attention(**{**dict(q=q, cache=cache, starts=s, lens=l), **kw})
    ok()
    for kw in (dict(q=q.float()), dict(q=q[0]), dict(q=q[:, :3]), dict(q=q[:, :, :32]), dict(q=q.cpu()), dict(cache=None),
               dict(starts=s.long()), dict(starts=s[:2]), dict(lens=l.cpu()), dict(lens=_i32(1, 2, 3), starts=_i32(0, 1, 2, 3)),
               dict(max_rows=0), dict(max_rows=4), dict(tree=_i32(1, 1)), dict(prefix_len=3),
               dict(prefix=cache, prefix_len=17), dict(prefix=cache.k), dict(out=q[:2]), dict(out=q.float()),
               dict(scratch=torch.empty(1 << 20, dtype=torch.uint8)), dict(q=q.transpose(0, 1)),
               dict(q=q[:0])):
        with pytest.raises(ValueError):
            ok(**kw)
    for kw in (dict(out=q), dict(scratch=torch.empty(8, dtype=torch.uint8, device=DEV)), dict(scale=math.nan),
               dict(prefix=make_cache(False, 1, 1, 16, 64))):
        with pytest.raises(pkg.MemSpecError):
            ok(**kw)
    x = torch.zeros(3, 8 * 64, device=DEV)
    gain = torch.ones(64, device=DEV, dtype=torch.bfloat16)
    rope = pkg.op_rope_table(16, 64)
    put = lambda **kw: pkg.op_kv_append(**{**dict(qkv=x, cache=cache, starts=s, lens=l, n_heads=4), **kw})
    put(rope=rope, q_gain=gain, k_gain=gain)
    for kw in (dict(qkv=x.half()), dict(qkv=x.cpu()), dict(qkv=x[:, :-1]), dict(qkv=x[0]), dict(n_heads=5), dict(n_heads=0),
               dict(rope=rope[0]), dict(rope=rope[:, :, :16]), dict(rope=rope.double()), dict(offsets=_i32(1)),
               dict(q_gain=gain), dict(q_gain=gain.float(), k_gain=gain.float()), dict(prefix_len=-1), dict(q=q[:2])):
        with pytest.raises(ValueError):
            put(**kw)
    with pytest.raises(pkg.MemSpecError):
        put(eps=-1.0)
    with pytest.raises(pkg.MemSpecError):      # rows at an odd stride
        put(qkv=torch.zeros(3, 8 * 64 + 1, device=DEV)[:, :-1])
    for kw in (dict(rows=0), dict(rows=3, k=q), dict(rows=3, starts=s[:2])):
        with pytest.raises(ValueError):
            pkg.op_kv_read(**{**dict(cache=cache, starts=s, lens=l), **kw})
    k = cache.k
    for bad in ((k, k[:1]), (k.float(), k.float()), (k, k.transpose(1, 2)), (k[..., ::2], k[..., ::2]), (k[0], k[0]),
                (k, k, torch.ones(2, 2, 16, device=DEV))):
        with pytest.raises(ValueError):
            pkg.KVCache(*bad)
    with pytest.raises(pkg.MemSpecError):      # k and v in one place are not written
        pkg.op_kv_append(x, pkg.KVCache(k, k), s, l, 4)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("H,Hk,hd,prefix", [(2, 2, 64, 0), (8, 1, 128, 0), (32, 1, 64, 0), (20, 1, 128, 130)])
def test_many_sequences_of_all_lengths(H, Hk, hd, prefix, codes):
    """1024 sequences, more than any table of the kernels holds, most with a row or none."""
    rng = np.random.default_rng(11)
    rows_of = rng.choice([0, 1, 1, 1, 2, 5], 1024)
    pasts = np.where(rng.random(1024) < 0.05, rng.integers(0, 900, 1024), rng.integers(0, 40, 1024))
    starts, lens = batch(rows_of, pasts)
    cache = make_cache(codes, 1024, Hk, max(lens), hd, seed=3)
    pre = make_cache(codes, 1, Hk, prefix, hd, seed=4) if prefix else None
    q = torch.randn(starts[-1], H, hd, device=DEV, generator=_gen(8)).bfloat16()
    got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=5, prefix=pre)
    some = list(range(0, 1024, 7)) + [1023]
    for b in some:
        rows = slice(starts[b], starts[b + 1])
        if rows.stop > rows.start:
            one = _pkg().KVCache(*[t[b:b + 1] for t in cache.tensors if t is not None])
            check(got[rows], *attention64(q[rows], one, [0, rows.stop - rows.start], [lens[b]], prefix=pre, prefix_len=prefix,
                                          max_rows=1 << 16))


@pytest.mark.parametrize("seed", range(12))
def test_drawn_batches(seed):
    """Shapes drawn from all that the calls take, each row against its definition."""
    rng = np.random.default_rng(1000 + seed)
    hd = int(rng.choice([64, 128]))
    Hk = int(rng.choice([1, 2, 3, 8]))
    H = Hk * int(rng.choice([1, 3, 4, 7, 16, 33, 64]))
    B = int(rng.integers(1, 9))
    rows_of = rng.integers(0, int(rng.choice([2, 10, 70])), B)
    rows_of[rng.integers(0, B)] += 1
    pasts = rng.integers(0, int(rng.choice([5, 300, 2500])), B)
    starts, lens = batch(rows_of, pasts)
    codes, pcodes = (bool(rng.integers(0, 2)) for _ in (0, 1))
    plen = int(rng.choice([0, 0, 1, 128, 777]))
    cache = make_cache(codes, B, Hk, max(lens) + 5, hd, seed=seed)
    pre = make_cache(pcodes, 1, Hk, plen + 1, hd, seed=seed + 50) if plen else None
    tree = torch.from_numpy(rng.integers(0, 1 << 32, starts[-1], dtype=np.uint32).view(np.int32)).to(DEV) \
        if max(rows_of) <= 32 and rng.integers(0, 2) else None
    q = (2 * torch.randn(starts[-1], H, hd, device=DEV, generator=_gen(seed))).bfloat16()
    max_rows = int(rng.integers(1, starts[-1] + 1))
    got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=max_rows, tree=tree, prefix=pre, prefix_len=plen)
    check(got, *attention64(q, cache, starts, lens, tree=tree, prefix=pre, prefix_len=plen, max_rows=1 << 16))


@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("H,Hk", [(4, 4), (32, 8), (32, 4)])
def test_a_vector_of_any_size_beside_others(H, Hk, codes):
    """Rows of one sequence whose queries are powers of 2^40 apart, and rows of no sequence (of which a prefix's
    units have the vectors too) with the largest values there are: each is as if it were alone."""
    starts, lens = batch([3], [140])
    cache = make_cache(codes, 1, Hk, 150, 128, seed=3)
    prefix = make_cache(codes, 1, Hk, 200, 128, seed=4)
    q = torch.randn(5, H, 128, device=DEV, generator=_gen(8))
    q[0] *= 2.0 ** 40
    q[2] *= 2.0 ** -40
    q[3:] = 3e38
    q = q.bfloat16()
    for pre in (None, prefix):
        got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens), max_rows=3, prefix=pre)
        for r in range(3):   # (a bound over the row's own sizes)
            want, bound = attention64(q, cache, starts, lens, prefix=pre, prefix_len=200, max_rows=3)
            check(got[r:r + 1], want[r:r + 1], bound[r:r + 1])


# ------------------------------------------------------------------ the ends of the ranges
@pytest.mark.parametrize("codes", [False, True])
def test_the_most_rows(codes):
    """65535 rows: of 1024 sequences, and of a single one."""
    pkg, hd = _pkg(), 64
    for rows_of, H in (([64] * 1023 + [63], 2), ([65535], 1)):
        starts, lens = batch(rows_of, [3] * len(rows_of))
        cache = pkg.KVCache.zeros(len(rows_of), 1, lens[0], hd, dtype=torch.int8 if codes else torch.bfloat16)
        x = torch.randn(65535, (H + 2) * hd, device=DEV, generator=_gen(3)).bfloat16()
        s, l = _i32(*starts), _i32(*lens)
        q = pkg.op_kv_append(x, cache, s, l, H)
        k, v = pkg.op_kv_read(cache, s, l, 65535)
        assert torch.equal(q, x.view(65535, H + 2, hd)[:, :H])
        if not codes:
            assert torch.equal(torch.cat([k, v], 1), x.view(65535, H + 2, hd)[:, H:])
        got = pkg.op_attention(q, cache, s, l)
        for row in (0, 1, 4097, 65471, 65533, 65534):
            b = np.searchsorted(starts, row, "right") - 1
            one = pkg.KVCache(*[t[b:b + 1] for t in cache.tensors if t is not None])
            check(got[row:row + 1], *attention64(q[row:row + 1], one, [0, 1], [lens[b] - (starts[b + 1] - 1 - row)],
                                                 max_rows=1 << 16))


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("H,Hk", [(1024, 1024), (4096, 64)])
def test_the_most_heads(H, Hk, codes):
    starts, lens = batch([1, 2], [40, 130])
    cache = make_cache(codes, 2, Hk, 140, 64, seed=3)
    q = torch.randn(3, H, 64, device=DEV, generator=_gen(8)).bfloat16()
    got = _pkg().op_attention(q, cache, _i32(*starts), _i32(*lens))
    check(got, *attention64(q, cache, starts, lens))


def test_a_layers_calls_on_a_side_stream_and_in_a_graph():
    """Append, attention and read, one after another on another stream, and captured there: replayed with the
    lengths of the next tokens they decode on."""
    pkg, H, Hk, hd = _pkg(), 8, 2, 128
    rope = pkg.op_rope_table(64, hd)
    caches = [pkg.KVCache.zeros(2, Hk, 64, hd, dtype=torch.int8) for _ in range(2)]
    s, l = _i32(0, 1, 2), _i32(5, 9)
    x = torch.randn(2, (H + 2 * Hk) * hd, device=DEV, generator=_gen(3))

    def layer(cache, stream=None):
        q = pkg.op_kv_append(x, cache, s, l, H, rope=rope, stream=stream)
        return pkg.op_attention(q, cache, s, l, max_rows=1, stream=stream), pkg.op_kv_read(cache, s, l, 2, stream=stream)[0]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for a, b in zip(layer(caches[0]), layer(caches[1], side)):
        torch.cuda.synchronize()
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = layer(caches[0])
    for _ in range(20):
        l.add_(1)
        x.normal_(generator=_gen(int(l[0])))
        graph.replay()
        for a, b in zip(outs, layer(caches[1])):
            assert torch.equal(a, b)
    assert all(torch.equal(a, b) for a, b in zip(caches[0].tensors, caches[1].tensors))


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("rows", [12, 64])
def test_calls_back_to_back_behind_a_prefix(rows, codes):
    """Rows by rows decoded behind a prefix: a call's launches may run beside one another, those of the next call
    on the same scratch, with queries written just before it, after them; eager and in one graph."""
    pkg, H, Hk, hd, P = _pkg(), 8, 4, 128, 700
    starts, lens = batch([1] * rows, [(37 * i) % 300 for i in range(rows)])
    cache = make_cache(codes, rows, Hk, 320, hd, seed=1)
    prefix = make_cache(codes, 1, Hk, P, hd, seed=2)
    s, l = _i32(*starts), _i32(*lens)
    qs = [torch.randn(rows, H, hd, device=DEV, generator=_gen(i)).bfloat16() for i in range(6)]
    scratch = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    q = torch.empty_like(qs[0])

    def run():
        outs = []
        for x in qs:
            q.copy_(x)
            outs.append(pkg.op_attention(q, cache, s, l, max_rows=1, prefix=prefix, scratch=scratch))
        return outs
    want = []
    for x in qs:
        want.append(pkg.op_attention(x, cache, s, l, max_rows=1, prefix=prefix))
        torch.cuda.synchronize()
    check(want[0], *attention64(qs[0], cache, starts, lens, prefix=prefix, prefix_len=P, max_rows=1))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for _ in range(30):
        graph.replay()
        for a, b, c in zip(run(), captured, want):
            assert torch.equal(a, c) and torch.equal(b, c)
