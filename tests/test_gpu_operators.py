"""Sampling rules (op_sample_filtered, op_filter_logits) and low-rank adapters (op_lora)
against their 64-bit definitions in oracle.filtering.

Draws and masks have to be equal.  The 64-bit form and the library's fixed-point weights
(off by 2^-34 of themselves in the mean square, at most 2^-31.8) can part only where a
border lies within that of u or p: with n kept ids in about n * 2^-33 of the draws, 2^-16
at the largest vocabulary kept whole.
"""
import math

import numpy as np
import pytest

from oracle import filtering as F

pytestmark = pytest.mark.gpu

RULES = [(1.0, 0, 1.0, 0.0), (0.8, 50, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.7, 40, 0.95, 0.0), (1.1, 0, 1.0, 0.05),
         (0.0, 0, 1.0, 0.0), (1.3, 1000, 0.98, 0.001), (1.0, 1, 1.0, 0.0), (0.9, 3, 0.5, 0.3), (0.05, 0, 0.999, 0.0),
         (50.0, 0, 0.5, 0.0), (1.0, 1 << 30, 1e-9, 0.0), (1.0, 0, 1.0, 1.0), (2.0, 5000, 0.6, 0.0)]


def _logits(kind, rows, vocab, seed=0):
    rng = np.random.default_rng([seed, rows, vocab, len(kind)])
    z = rng.normal(size=(rows, vocab))
    if kind != "flat":
        z = 12.0 - 1.4 * np.log1p(np.argsort(rng.random((rows, vocab)), axis=1)) + 0.7 * z
    z = z.astype(np.float32)
    if kind == "coarse":        # many equal logits, on both sides of zero
        z = np.round(z * 4).astype(np.float32) / 4
    elif kind == "equal":
        z[:] = -2.5
    elif kind == "masked":      # -inf, the type's lowest value, NaN; a row that leaves nothing
        z[rng.random(z.shape) < 0.7] = -np.inf
        z[rng.random(z.shape) < 0.2] = -F.LARGEST
        z[rng.random(z.shape) < 0.05] = np.nan
        z[0] = -np.inf
        if rows > 1:
            z[1] = np.nan
        if rows > 2:            # a single id left
            z[2] = -np.inf
            z[2, vocab // 2] = 1.0
    elif kind == "infinite":    # +inf ties with the largest finite number
        z[:, ::7] = np.inf
        z[:, 0] = F.LARGEST
    return z


def _uniforms(rows, seed=0):
    u = (2 * np.random.default_rng([seed, rows]).integers(0, 1 << 23, rows) + 1) * 2.0 ** -24
    if rows > 3:
        u[1], u[2] = 0.0, 1 - 2.0 ** -24
    return u.astype(np.float32)


def _rows_at(z, ld, offset):
    """z on the GPU with rows ld apart, the first one `offset` floats past an aligned
    address; everything around the rows is a large logit."""
    import torch
    rows, vocab = z.shape
    raw = torch.full((offset + rows * ld + 8,), 1e30, device="cuda")
    v = raw[offset:offset + rows * ld].view(rows, ld)[:, :vocab]
    v.copy_(torch.from_numpy(z))
    return raw, v


SHAPES = [(1, 1), (3, 2), (4, 31), (2, 513), (5, 2048), (3, 4097), (14, 9999), (2, 32003), (9, 32000), (2, 65536),
          (3, 100001), (2, 128256), (2, 131072), (40, 700), (170, 1500)]


@pytest.mark.parametrize("kind", ["peaked", "flat", "coarse", "equal", "masked", "infinite"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_draws_and_masks_follow_the_definition(rows, vocab, kind):
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    z, u = _logits(kind, rows, vocab), _uniforms(rows)
    rules = [RULES[(r + rows + vocab) % len(RULES)] for r in range(rows)]
    raw, zt = _rows_at(z, vocab + (rows * 3) % 8, (rows + vocab) % 4)
    before = raw.clone()
    per = [torch.tensor([r[i] for r in rules], dtype=torch.int32 if i == 1 else torch.float32, device="cuda")
           for i in range(4)]
    got = op_sample_filtered(zt, torch.from_numpy(u).cuda(), *per).cpu().numpy()
    masked = op_filter_logits(zt, *per).cpu().numpy()
    assert torch.equal(raw.nan_to_num(7.0), before.nan_to_num(7.0))
    for r in range(min(rows, 40)):
        want = F.mask(z[r], *rules[r])
        bad = np.flatnonzero(masked[r] != want)
        assert bad.size == 0, (r, rules[r], bad[:5], np.isfinite(masked[r]).sum(), np.isfinite(want).sum())
        assert got[r] == F.draw(z[r], u[r], *rules[r]), (r, rules[r], u[r])


@pytest.mark.parametrize("rule", RULES)
def test_one_rule_for_all_rows(rule):
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    z, u = np.concatenate([_logits("peaked", 3, 20000), _logits("flat", 3, 20000)]), _uniforms(6)
    zt = torch.from_numpy(z).cuda()
    T, k, p, m = rule
    got = op_sample_filtered(zt, torch.from_numpy(u).cuda(), temperature=T, top_k=k, top_p=p, min_p=m)
    assert got.cpu().tolist() == [F.draw(z[r], u[r], *rule) for r in range(6)]
    masked = op_filter_logits(zt, temperature=T, top_k=k, top_p=p, min_p=m).cpu().numpy()
    assert all(np.array_equal(masked[r], F.mask(z[r], *rule)) for r in range(6))


@pytest.mark.parametrize("vocab", [1000, 5000, 131072])
def test_borders_among_equal_weights_are_exact(vocab):
    """All weights are equal, so every sum is a whole number: u = j / vocab lands on the
    border after id j - 1 and draws id j; top-p = j / vocab keeps j ids where the float
    holds it exactly, else the next whole number."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    j = np.unique(np.concatenate([np.arange(0, vocab, vocab // 60), [1, vocab - 1]]))
    f = (j / vocab).astype(np.float32)
    zt = torch.full((len(j), vocab), 0.25, device="cuda")
    got = op_sample_filtered(zt, torch.from_numpy(f).cuda()).cpu().numpy()
    exact = np.floor(f.astype(np.float64) * vocab).astype(int)     # 24 + 17 bits: exact
    assert got.tolist() == exact.tolist()
    p = torch.from_numpy(f).cuda()
    n = torch.isfinite(op_filter_logits(zt, top_p=p)).sum(1).cpu().numpy()
    assert n.tolist() == np.maximum(1, np.ceil(f.astype(np.float64) * vocab)).astype(int).tolist()


@pytest.mark.parametrize("T,first,step,last", [(0.6, 0, 3, 200), (1.0, 20, 60, 1500)])
@pytest.mark.parametrize("vocab", [4000, 15000, 50000, 128256])
def test_top_p_next_to_a_border(vocab, T, first, step, last):
    """p is the float nearest to the share of the first j ids: above it or below by some 1e-8,
    where the weights of the ids behind the candidates decide to their last bits."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    rows, T = 24, float(np.float32(T))
    z, u, p = _logits("peaked", rows, vocab, 3), _uniforms(rows), np.empty(rows, np.float32)
    for r in range(rows):
        w = np.sort(np.exp((z[r].astype(np.float64) - z[r].max()) / T))[::-1]
        share = np.cumsum(w) / np.sum(w)
        j = next(j for j in range(first + step * r % last, last) if 2.0 ** -30 < abs(np.float32(share[j]) - share[j]) < 2.0 ** -24)
        p[r] = share[j]
    zt, pt = torch.from_numpy(z).cuda(), torch.from_numpy(p).cuda()
    got = op_sample_filtered(zt, torch.from_numpy(u).cuda(), temperature=T, top_p=pt).cpu().numpy()
    masked = op_filter_logits(zt, temperature=T, top_p=pt).cpu().numpy()
    for r in range(rows):
        assert np.array_equal(masked[r], F.mask(z[r], T, 0, p[r])), r
        assert got[r] == F.draw(z[r], u[r], T, 0, p[r]), r
    assert op_filter_logits(zt, temperature=T, top_p=pt, out=zt) is zt
    assert np.array_equal(zt.cpu().numpy(), masked)


@pytest.mark.parametrize("kind", ["peaked", "flat", "coarse", "equal", "masked", "infinite"])
@pytest.mark.parametrize("rows,vocab", [(64, 900), (64, 15000), (160, 15000), (48, 32003), (160, 32000), (32, 70000),
                                        (96, 65537), (8, 131072), (64, 128256)])
def test_draws_are_those_from_the_mask(rows, vocab, kind):
    """A draw under a rule is the draw without one from the logits that the mask keeps: the
    maximum and so every kept weight is the same, and both have to be equal to the last bit.
    Temperatures that leave one id up to all of them, top-k below, at and above what the
    candidates hold."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    z = torch.from_numpy(_logits(kind, min(rows, 16), vocab, 7)).cuda().repeat(rows // min(rows, 16), 1)
    u = torch.from_numpy(_uniforms(rows, 7)).cuda()
    rules = []
    for T in (1e-20, 0.02, 0.3, 0.6, 1.0, 1.5, 20.0, 1e20, math.inf):
        for p in (1e-6, 0.1, 0.5, 0.9, 0.95, 0.99, 0.9999):
            for min_p in (0.0, 0.02):
                rules.append(dict(temperature=T, top_p=p, min_p=min_p))
        for k in (60, 257, 449, 1000, 1600, 5000):
            for p in (1.0, 0.98, 0.6):
                rules.append(dict(temperature=T, top_k=k, top_p=p))
    for rule in rules:
        got = op_sample_filtered(z, u, **rule)
        want = op_sample_filtered(op_filter_logits(z, **rule), u, temperature=rule["temperature"])
        assert torch.equal(got, want), (rule, torch.nonzero(got != want)[:5])


def test_rule_arrays_out_of_range_mean_what_the_header_says():
    import torch
    from paper_2608_10362_gb300 import op_filter_logits
    z = _logits("peaked", 1, 3000)
    nan = float("nan")
    odd = [(-1.0, 5, 1.0, 0.0), (nan, 5, 1.0, 0.0), (1.0, -3, 1.0, 0.0), (1.0, 0, 2.0, 0.0), (1.0, 0, nan, 0.0),
           (1.0, 0, 0.0, 0.0), (1.0, 0, -1.0, 0.0), (1.0, 0, 1.0, -1.0), (1.0, 0, 1.0, nan), (1.0, 0, 1.0, 7.0),
           (math.inf, 0, 0.5, 0.0), (1e-40, 0, 0.5, 0.0), (1e30, 0, 1.0, 0.5)]
    keeps = [1, 1, 3000, 3000, 3000, 1, 1, 3000, 3000, 1, 1500, 1, 3000]
    per = [torch.tensor([o[i] for o in odd], dtype=torch.int32 if i == 1 else torch.float32, device="cuda")
           for i in range(4)]
    m = op_filter_logits(torch.from_numpy(z).cuda().expand(len(odd), -1).contiguous(), *per)
    assert torch.isfinite(m).sum(1).tolist() == keeps


def test_mask_in_place_and_into_rows_of_a_larger_tensor():
    import torch
    from paper_2608_10362_gb300 import op_filter_logits
    z = _logits("peaked", 7, 5001)
    rule = dict(temperature=0.9, top_k=77, top_p=0.97)
    want = np.stack([F.mask(r, 0.9, 77, 0.97) for r in z])
    zt = torch.from_numpy(z).cuda()
    big = torch.full((7, 5100), 3.0, device="cuda")
    out = op_filter_logits(zt, **rule, out=big[:, 50:5051])
    assert np.array_equal(out.cpu().numpy(), want)
    assert bool((big[:, :50] == 3).all()) and bool((big[:, 5051:] == 3).all())
    assert op_filter_logits(zt, **rule, out=zt) is zt
    assert np.array_equal(zt.cpu().numpy(), want)
    # a second time nothing more is cut by top-k
    assert np.array_equal(op_filter_logits(zt, temperature=0.9, top_k=77).cpu().numpy(), want)
    with pytest.raises(ValueError):
        op_filter_logits(big[:, :5001], out=big[:, 1:5002])


def test_filtered_draws_repeat_and_run_under_a_graph():
    """The same bits from call to call, on another stream, and from two captured graphs
    that run at once and are replayed on new inputs."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    z = [torch.from_numpy(_logits(k, 24, 50257, 5)).cuda() for k in ("peaked", "flat")]
    u = torch.from_numpy(_uniforms(24, 1)).cuda()
    rule = dict(temperature=0.9, top_k=2000, top_p=0.9)
    first = [(op_sample_filtered(x, u, **rule), op_filter_logits(x, **rule)) for x in z]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for x, (t, m) in zip(z, first):
            assert torch.equal(op_sample_filtered(x, u, **rule), t)
            assert torch.equal(op_filter_logits(x, **rule), m)
            t2 = op_sample_filtered(x, u, **rule, stream=side)
            side.synchronize()
            assert torch.equal(t2, t)
    static = [x.clone() for x in z]
    graphs, outs = [], []
    torch.cuda.synchronize()
    for x in static:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append((op_sample_filtered(x, u, **rule), op_filter_logits(x, **rule)))
        graphs.append(g)
    for swap in (False, True, False):
        for x, src in zip(static, z[::-1] if swap else z):
            x.copy_(src)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        for (t, m), (wt, wm) in zip(outs, first[::-1] if swap else first):
            assert torch.equal(t, wt) and torch.equal(m, wm)


def test_many_rows_and_rows_far_apart():
    """More rows than the chip holds at once; row strides past 2^31 elements; a mask beside the
    logits in the rows of one tensor."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    z, u = _logits("peaked", 50, 97), _uniforms(50)
    many = torch.from_numpy(z).cuda().repeat(800, 1)
    got = op_sample_filtered(many, torch.from_numpy(u).cuda().repeat(800), temperature=0.8, top_k=20, top_p=0.9)
    want = [F.draw(z[r], u[r], 0.8, 20, 0.9) for r in range(50)]
    assert torch.equal(got.cpu().view(800, 50), torch.tensor(want, dtype=torch.int32).expand(800, 50))
    far = 1 << 30
    raw = torch.zeros(2 * far + 97, device="cuda")
    rows = torch.as_strided(raw, (3, 97), (far, 1))
    rows.copy_(torch.from_numpy(z[:3]))
    assert op_sample_filtered(rows, torch.from_numpy(u[:3]).cuda(), temperature=0.8, top_k=20, top_p=0.9).tolist() == want[:3]
    op_filter_logits(rows, top_k=5, out=rows)
    assert np.array_equal(rows.cpu().numpy(), np.stack([F.mask(r, 1.0, 5) for r in z[:3]]))
    del raw, rows
    both = torch.zeros(50, 200, device="cuda")
    both[:, :97] = torch.from_numpy(z)
    op_filter_logits(both[:, :97], top_k=5, out=both[:, 100:197])
    assert np.array_equal(both[:, 100:197].cpu().numpy(), np.stack([F.mask(r, 1.0, 5) for r in z]))
    assert np.array_equal(both[:, :97].cpu().numpy(), z) and bool((both[:, 97:100] == 0).all())
    # uniforms outside [0, 1): the first kept id, the last
    ids = np.sort(F.kept(z[0], 1.0, 7))
    odd = torch.tensor([-1.0, 1.0, math.inf, float("nan")], device="cuda")
    four = torch.from_numpy(z[:1]).cuda().repeat(4, 1)
    assert op_sample_filtered(four, odd, top_k=7).tolist() == [ids[0], ids[-1], ids[-1], ids[0]]


def test_filter_arguments_are_refused():
    import torch
    from paper_2608_10362_gb300 import MemSpecError, op_filter_logits, op_sample_filtered
    z, u = torch.zeros(3, 40, device="cuda"), torch.full((3,), 0.5, device="cuda")
    ids = torch.empty(3, dtype=torch.int32, device="cuda")
    for bad in (dict(temperature=-1.0), dict(top_p=0.0), dict(top_p=1.2), dict(min_p=1.5)):
        with pytest.raises(MemSpecError):
            op_sample_filtered(z, u, **bad)
    for call in (lambda: op_sample_filtered(z.half(), u), lambda: op_sample_filtered(z[0], u),
                 lambda: op_sample_filtered(z.t(), torch.zeros(40, device="cuda")),
                 lambda: op_sample_filtered(z[:1].expand(3, 40), u), lambda: op_sample_filtered(z, u[:2]),
                 lambda: op_sample_filtered(z, u.double()), lambda: op_sample_filtered(z, u, top_k=-1),
                 lambda: op_sample_filtered(z, u, top_k=1 << 32), lambda: op_sample_filtered(z, u, top_k=1.5),
                 lambda: op_sample_filtered(z, u, top_k=u), lambda: op_sample_filtered(z, u, top_p=u[:2]),
                 lambda: op_sample_filtered(z, u, out=ids[:2]), lambda: op_sample_filtered(z[:0], u[:0]),
                 lambda: op_filter_logits(z, out=z[:, :39]), lambda: op_filter_logits(z[:, :0])):
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------ adapters
def _lora_case(rows, n, k, rank, adapters, who, seed=0, whole=False):
    """Seeded inputs; `whole`: small whole numbers, whose products and sums fp32 holds exactly."""
    rng = np.random.default_rng([seed, rows, n, k, rank, adapters])
    bf = lambda v: (np.ascontiguousarray(v, dtype=np.float32).view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
    if whole:
        x = rng.integers(-2, 3, (rows, k)).astype(np.float32)
        a = rng.integers(-1, 2, (adapters, rank, k)).astype(np.float32)
        b = rng.integers(-2, 3, (adapters, n, rank)).astype(np.float32)
        base = rng.integers(-100, 101, (rows, n)).astype(np.float32)
        scales = (2.0 ** rng.integers(-2, 3, adapters)).astype(np.float32)
    else:
        x, base = bf(rng.normal(size=(rows, k))), rng.normal(size=(rows, n)).astype(np.float32)
        a, b = bf(rng.normal(size=(adapters, rank, k)) * k ** -0.5), bf(rng.normal(size=(adapters, n, rank)) * 0.05)
        scales = rng.uniform(0.5, 2.0, adapters).astype(np.float32)
    ids = {"one": np.zeros(rows, int), "each": np.arange(rows) % adapters,
           "random": rng.integers(-1, adapters + 1, rows), "none": np.full(rows, -1)}[who]
    ranks = rng.integers(0, rank + 3, adapters)     # 0: an empty adapter; past rank: clamped
    return x, a, b, ids.astype(np.int32), scales, ranks.astype(np.int32), base


def _cuda(v):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(v)).cuda()
    return t


LORA = [(1, 64, 64, 8, 1, "one"), (1, 1, 8, 8, 1, "one"), (3, 33, 72, 16, 2, "each"), (5, 4096, 1024, 16, 3, "random"),
        (16, 1000, 4096, 16, 16, "each"), (17, 513, 520, 24, 4, "one"), (21, 3001, 2048, 40, 8, "random"),
        (64, 256, 1032, 64, 5, "random"), (144, 1536, 768, 64, 16, "each"), (255, 130, 264, 128, 3, "random"),
        (256, 768, 2304, 128, 2, "one"), (256, 95, 64, 8, 256, "each"), (12, 640, 640, 48, 4, "none"),
        (2, 8192, 14336, 128, 2, "each"), (33, 100, 40, 56, 40, "random"), (30, 9001, 136, 16, 3, "random"),
        (200, 700, 512, 32, 1, "one"), (256, 4096, 256, 8, 16, "each"), (256, 4100, 64, 16, 1, "one"),
        (20, 90, 640, 64, 20, "each"), (40, 200, 320, 72, 30, "random"), (32, 64, 2000, 120, 32, "each"),
        (150, 40, 2048, 32, 2, "random"), (7, 16400, 3000, 24, 2, "each")]


@pytest.mark.parametrize("with_ranks", [True, False])
@pytest.mark.parametrize("rows,n,k,rank,adapters,who", LORA)
def test_lora_is_exact_on_whole_numbers(rows, n, k, rank, adapters, who, with_ranks):
    """The absolute values of all products sum to less than 2^24 - 400 before the scale, so
    every partial sum in any order is exact; scales are powers of two (1/4 to 4), so that
    base + scale * sum is a whole number of units of min(1, scale), fewer than 2^24."""
    import torch
    from paper_2608_10362_gb300 import op_lora
    x, a, b, ids, scales, ranks, base = _lora_case(rows, n, k, rank, adapters, who, whole=True)
    ranks = ranks if with_ranks else None
    want, size = F.lora(x, a, b, ids, scales, ranks, base)
    assert F.lora(x, a, b, ids, None, ranks)[1].max() < 2 ** 24 - 400 and size.max() < 2 ** 24
    got = op_lora(_cuda(x).bfloat16(), _cuda(a).bfloat16(), _cuda(b).bfloat16(), _cuda(ids), _cuda(scales),
                  None if ranks is None else _cuda(ranks), _cuda(base))
    assert np.array_equal(got.cpu().numpy().astype(np.float64), want)


@pytest.mark.parametrize("rows,n,k,rank,adapters,who", LORA)
def test_lora_matches_64_bits(rows, n, k, rank, adapters, who):
    """Products of bf16 values are exact in fp32.  A sum of m of them in any order is off by
    at most m units of 2^-23 (additions that may truncate) of the sum of their absolute
    values: k for A x, rank and the two last operations for the rest."""
    from paper_2608_10362_gb300 import op_lora
    x, a, b, ids, scales, ranks, base = _lora_case(rows, n, k, rank, adapters, who)
    want, size = F.lora(x, a, b, ids, scales, ranks, base)
    got = op_lora(_cuda(x).bfloat16(), _cuda(a).bfloat16(), _cuda(b).bfloat16(), _cuda(ids), _cuda(scales), _cuda(ranks),
                  _cuda(base)).cpu().numpy().astype(np.float64)
    err = np.abs(got - want)
    assert np.all(err <= (k + rank + 4) * 2.0 ** -23 * size)
    # and in the mean the roundings do not add up: within 1e-6 of the result's size
    assert np.linalg.norm(err) <= 1e-6 * np.linalg.norm(want) + 1e-12


def test_lora_keeps_what_it_does_not_own():
    """Strided x, base and y, in place and not; rows without an adapter get the base's bits;
    nothing beside the rows is written; NaN in unused ranks and unused adapters is not read
    into the result."""
    import torch
    from paper_2608_10362_gb300 import op_lora
    rows, n, k, rank, adapters = 19, 300, 200, 32, 6
    x, a, b, ids, scales, ranks, base = _lora_case(rows, n, k, rank, adapters, "random", seed=9)
    ranks = np.array([32, 0, 5, 31, 16, 32], dtype=np.int32)
    ids[:6] = [-1, 0, 1, 2, 3, 4]
    ids[ids == 5] = 0                           # adapter 5 is nobody's
    want, size = F.lora(x, a, b, ids, scales, ranks, base)
    a, b = a.copy(), b.copy()
    for i, r in enumerate(ranks):
        a[i, r:], b[i, :, r:] = np.nan, np.nan
    a[5], b[5], scales[5] = np.nan, np.nan, np.nan
    xs = torch.full((rows, k + 24), 1e30, device="cuda", dtype=torch.bfloat16)
    xs[:, 8:8 + k] = _cuda(x)
    ys = torch.full((rows, n + 13), 7.0, device="cuda")
    ys[:, 5:5 + n] = _cuda(base)
    args = (xs[:, 8:8 + k], _cuda(a).bfloat16(), _cuda(b).bfloat16(), _cuda(ids), _cuda(scales), _cuda(ranks))
    out = torch.full((rows, n + 3), 7.0, device="cuda")
    got = op_lora(*args, base=ys[:, 5:5 + n], y=out[:, 1:1 + n])
    assert bool((out[:, 0] == 7).all()) and bool((out[:, 1 + n:] == 7).all())
    none = np.flatnonzero((ids < 0) | (ids >= adapters))
    assert len(none) and torch.equal(got[none], ys[none, 5:5 + n])
    assert np.all(np.abs(got.cpu().numpy() - want) <= (k + rank + 4) * 2.0 ** -23 * size)
    y = ys[:, 5:5 + n]
    assert op_lora(*args, base=y, y=y) is y
    assert torch.equal(y, got) and bool((ys[:, :5] == 7).all()) and bool((ys[:, 5 + n:] == 7).all())
    bare = op_lora(*args)
    want0, size0 = F.lora(x, np.nan_to_num(a), np.nan_to_num(b), ids, scales, ranks)
    assert np.all(np.abs(bare.cpu().numpy() - want0) <= (k + rank + 4) * 2.0 ** -23 * size0)
    with pytest.raises(ValueError):
        op_lora(*args, base=ys[:, 5:5 + n], y=ys[:, 6:6 + n])


def test_lora_repeats_on_one_scratch_of_any_content_and_under_graphs():
    """The same bits whatever the scratch held; two graphs with scratches of their own run at
    once; replays see new inputs."""
    import torch
    from paper_2608_10362_gb300 import op_lora
    from paper_2608_10362_gb300.engine import _lora_scratch_bytes
    cases = [_lora_case(48, 2048, 1024, 32, 8, "random", s) for s in (1, 2)]
    dev = [[_cuda(v).bfloat16() if i < 3 else _cuda(v) for i, v in enumerate(c)] for c in cases]
    nb = max(_lora_scratch_bytes(r, 2048, 1024, 32) for r in range(1, 257))
    scratch = [torch.empty(nb, dtype=torch.uint8, device="cuda") for _ in range(2)]
    call = lambda d, s: op_lora(d[0], d[1], d[2], d[3], d[4], d[5], d[6], scratch=s)
    first = [call(d, scratch[0]).clone() for d in dev]
    for fill in (0, 255, 127):
        scratch[1].fill_(fill)
        for d, f in zip(dev, first):
            assert torch.equal(call(d, scratch[1]), f)
    assert torch.equal(call([v[:7] if i in (0, 3, 6) else v for i, v in enumerate(dev[0])], scratch[1]), first[0][:7])
    static = [[v.clone() for v in d] for d in dev]
    graphs, outs = [], []
    torch.cuda.synchronize()
    for d, s in zip(static, scratch):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(d, s))
        graphs.append(g)
    side = torch.cuda.Stream()
    for swap in (False, True):
        for d, src in zip(static, dev[::-1] if swap else dev):
            for v, w in zip(d, src):
                v.copy_(w)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        for o, f in zip(outs, first[::-1] if swap else first):
            assert torch.equal(o, f)


def test_lora_single_rows_at_any_stride_and_rows_far_apart():
    import torch
    from paper_2608_10362_gb300 import op_lora
    x, a, b, ids, scales, ranks, base = _lora_case(3, 100, 64, 16, 2, "each", whole=True)
    want, _ = F.lora(x, a, b, ids, scales, ranks, base)
    rest = (_cuda(a).bfloat16(), _cuda(b).bfloat16(), _cuda(ids)[1:2].clone(), _cuda(scales), _cuda(ranks))
    one = torch.zeros(3, 67, device="cuda", dtype=torch.bfloat16)
    one[0, :64] = _cuda(x)[1]
    odd = torch.zeros(3, 103, device="cuda")
    odd[0, :100] = _cuda(base)[1]
    got = op_lora(one[:1, :64], *rest, base=odd[:1, :100])
    assert np.array_equal(got.cpu().numpy(), want[1:2].astype(np.float32))
    got = op_lora(one[:1, :64].expand(1, 64), *rest, base=odd[0, :100].unsqueeze(0).expand(1, 100))
    assert np.array_equal(got.cpu().numpy(), want[1:2].astype(np.float32))
    far = 1 << 30
    raw, rawx = torch.zeros(2 * far + 100, device="cuda"), torch.zeros(2 * far + 64, device="cuda", dtype=torch.bfloat16)
    y, xs = torch.as_strided(raw, (3, 100), (far, 1)), torch.as_strided(rawx, (3, 64), (far, 1))
    y.copy_(_cuda(base))
    xs.copy_(_cuda(x))
    op_lora(xs, _cuda(a).bfloat16(), _cuda(b).bfloat16(), _cuda(ids), _cuda(scales), _cuda(ranks), base=y, y=y)
    assert np.array_equal(y.cpu().numpy(), want.astype(np.float32))


def test_lora_infinities_stay_in_their_rows():
    import torch
    from paper_2608_10362_gb300 import op_lora
    x, a, b, ids, scales, ranks, base = _lora_case(20, 200, 128, 16, 4, "each", seed=6)
    ranks[:] = 16
    want, size = F.lora(x, a, b, ids, scales, ranks, base)
    x[5, 17], x[9, 3] = np.inf, np.nan
    a[2, 3, 5], b[3, 100, 2] = np.nan, np.inf
    got = op_lora(_cuda(x).bfloat16(), _cuda(a).bfloat16(), _cuda(b).bfloat16(), _cuda(ids), _cuda(scales), _cuda(ranks),
                  _cuda(base)).cpu().numpy()
    fine = np.array([r for r in range(20) if ids[r] in (0, 1) and r not in (5, 9)])
    assert np.all(np.abs(got[fine] - want[fine]) <= (128 + 16 + 4) * 2.0 ** -23 * size[fine])
    assert np.all(np.isfinite(np.delete(got[ids == 3], 100, axis=1)))


def test_lora_arguments_are_refused():
    import torch
    from paper_2608_10362_gb300 import MemSpecError, op_lora
    mk = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    x, a, b = mk(4, 64), mk(2, 16, 64), mk(2, 32, 16)
    ids, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    base = torch.zeros(4, 32, device="cuda")
    for call in (lambda: op_lora(mk(257, 64), a, b, ids.new_zeros(257)), lambda: op_lora(x, mk(2, 12, 64), mk(2, 32, 12), ids),
                 lambda: op_lora(mk(4, 60), mk(2, 16, 60), b, ids),
                 lambda: op_lora(x, a, b, ids, scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(MemSpecError):
            call()
    for call in (lambda: op_lora(x.float(), a, b, ids), lambda: op_lora(x, a[0], b, ids), lambda: op_lora(x, a, b[:1], ids),
                 lambda: op_lora(x, a, b.transpose(1, 2), ids), lambda: op_lora(x, mk(2, 16, 72), b, ids),
                 lambda: op_lora(x, a, b, ids.long()), lambda: op_lora(x, a, b, ids[:3]),
                 lambda: op_lora(x, a, b, ids, f[:1]), lambda: op_lora(x, a, b, ids, f, f),
                 lambda: op_lora(x, a, b, ids, base=base[:, :31]), lambda: op_lora(x, a, b, ids, y=base.double()),
                 lambda: op_lora(x, a, b, ids, base=base.cpu())):
        with pytest.raises(ValueError):
            call()


def test_adapters_and_rules_of_a_batch_together():
    """What a batched pass does at its end: the shared LM head, each request's adapter beside
    it, each request's rule on its rows - through the bf16 and the INT4 head."""
    import torch
    from paper_2608_10362_gb300 import int4_pack, op_linear, op_linear_int4, op_lora, op_sample_filtered
    rows, vocab, k, rank, adapters = 12, 4003, 512, 16, 4
    x, a, b, ids, scales, ranks, _ = _lora_case(rows, vocab, k, rank, adapters, "random", seed=3)
    rng = np.random.default_rng(8)
    w = _cuda(rng.normal(size=(vocab, k)).astype(np.float32) * 0.2).bfloat16()
    q = torch.from_numpy(rng.integers(0, 256, (vocab, k // 2), dtype=np.uint8)).cuda()
    s = torch.full((vocab, k // 128), 0.02, device="cuda").bfloat16()
    zp = torch.full((vocab, k // 128), 8, dtype=torch.uint8, device="cuda")
    xt = _cuda(x).bfloat16()
    rules = [RULES[r % len(RULES)] for r in range(rows)]
    per = [torch.tensor([r[i] for r in rules], dtype=torch.int32 if i == 1 else torch.float32, device="cuda")
           for i in range(4)]
    u = _uniforms(rows, 4)
    for shared in (op_linear(xt, w), op_linear_int4(xt, int4_pack(q, s, zp), vocab)):
        z = op_lora(xt, _cuda(a).bfloat16(), _cuda(b).bfloat16(), _cuda(ids), _cuda(scales), _cuda(ranks), base=shared,
                    y=shared)
        got = op_sample_filtered(z, torch.from_numpy(u).cuda(), *per).cpu().tolist()
        zh = z.cpu().numpy()
        assert got == [F.draw(zh[r], u[r], *rules[r]) for r in range(rows)]
