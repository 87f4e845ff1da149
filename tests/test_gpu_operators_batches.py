"""Sampling rules over batches whose rows do not all fit the chip at once (kernels of 256 threads,
few rows take those of 512) against their 64-bit definition."""
import numpy as np
import pytest

from oracle import filtering as F
from test_gpu_operators import RULES, _logits, _rows_at, _uniforms

pytestmark = pytest.mark.gpu


# 256 threads: 35 rows and more of 8 CTAs, 73 of 4, 153 of 2 and 305 of one; 170 x 1500: 512, every row
@pytest.mark.parametrize("kind", ["peaked", "flat", "coarse", "equal", "masked", "infinite"])
@pytest.mark.parametrize("rows,vocab,every", [(42, 128256, 1), (100, 65537, 5), (75, 40000, 1), (160, 20000, 5),
                                              (320, 9000, 5), (170, 1500, 1)])
def test_batches_follow_the_definition(rows, vocab, every, kind):
    """Every `every`-th row, with each of the 14 rules on some of them."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    few = min(rows, 30)
    z = np.tile(_logits(kind, few, vocab, 11), (-(-rows // few), 1))[:rows]
    u = _uniforms(rows, 11)
    rules = [RULES[(r // every) % len(RULES)] for r in range(rows)]
    raw, zt = _rows_at(z, vocab + (rows * 3) % 8, (rows + vocab) % 4)
    per = [torch.tensor([r[i] for r in rules], dtype=torch.int32 if i == 1 else torch.float32, device="cuda")
           for i in range(4)]
    got = op_sample_filtered(zt, torch.from_numpy(u).cuda(), *per).cpu().numpy()
    masked = op_filter_logits(zt, *per).cpu().numpy()
    for r in range(0, rows, every):
        want = F.mask(z[r], *rules[r])
        bad = np.flatnonzero(masked[r] != want)
        assert bad.size == 0, (r, rules[r], bad[:5], np.isfinite(masked[r]).sum(), np.isfinite(want).sum())
        assert got[r] == F.draw(z[r], u[r], *rules[r]), (r, rules[r], u[r])


@pytest.mark.parametrize("rule", RULES)
def test_one_rule_for_a_batch(rule):
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    rows, vocab = 84, 65536
    z = np.tile(np.concatenate([_logits("peaked", 3, vocab, 12), _logits("flat", 3, vocab, 12)]), (rows // 6, 1))
    u = _uniforms(rows, 12)
    zt = torch.from_numpy(z).cuda()
    kw = dict(zip(("temperature", "top_k", "top_p", "min_p"), rule))
    got = op_sample_filtered(zt, torch.from_numpy(u).cuda(), **kw).cpu().tolist()
    masked = op_filter_logits(zt, **kw).cpu().numpy()
    for r in range(6):
        want = F.mask(z[r], *rule)
        assert all(np.array_equal(masked[q], want) for q in range(r, rows, 6)), r
    assert got == [F.draw(z[r], u[r], *rule) for r in range(rows)]


@pytest.mark.parametrize("T,first,step,last", [(0.6, 0, 3, 200), (1.0, 20, 60, 1500)])
@pytest.mark.parametrize("rows,vocab", [(80, 50000), (40, 128256)])
def test_top_p_next_to_a_border_in_a_batch(rows, vocab, T, first, step, last):
    """p is the float nearest to the share of a row's first j ids, above it or below by some 1e-8."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    T = float(np.float32(T))
    z, u, p = _logits("peaked", rows, vocab, 13), _uniforms(rows, 13), np.empty(rows, np.float32)
    for r in range(rows):
        w = np.sort(np.exp((z[r].astype(np.float64) - z[r].max()) / T))[::-1]
        share = np.cumsum(w) / np.sum(w)
        p[r] = share[next(j for j in range(first + step * r % last, last)
                          if 2.0 ** -30 < abs(np.float32(share[j]) - share[j]) < 2.0 ** -24)]
    zt, pt = torch.from_numpy(z).cuda(), torch.from_numpy(p).cuda()
    got = op_sample_filtered(zt, torch.from_numpy(u).cuda(), temperature=T, top_p=pt).cpu().numpy()
    masked = op_filter_logits(zt, temperature=T, top_p=pt).cpu().numpy()
    for r in range(rows):
        assert np.array_equal(masked[r], F.mask(z[r], T, 0, p[r])), r
        assert got[r] == F.draw(z[r], u[r], T, 0, p[r]), r


@pytest.mark.parametrize("rows,rank,vocab", [(4, 16, 4096), (16, 64, 9000), (100, 32, 4003), (144, 128, 32000)])
def test_calls_back_to_back_give_what_calls_apart_give(rows, rank, vocab):
    """Shared projection, adapters in place, mask in place, draw: each reads what the call before it
    writes and starts before that has ended; the same with the GPU waited for after each."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_linear, op_lora, op_sample_filtered
    g = torch.Generator(device="cuda").manual_seed(rows)
    mk = lambda *s: torch.randn(*s, device="cuda", generator=g)
    k, n = 512, 5
    xs = [mk(rows, k).bfloat16() for _ in range(n)]
    w, a, b = (mk(vocab, k) * 0.1).bfloat16(), (mk(n, rank, k) * 0.05).bfloat16(), mk(n, vocab, rank).bfloat16()
    ids = torch.randint(-1, n, (rows,), device="cuda", generator=g, dtype=torch.int32)
    u = torch.rand(rows, device="cuda", generator=g)
    T = 0.5 + torch.rand(rows, device="cuda", generator=g)
    scratch = torch.empty(rows * rank * 4, dtype=torch.uint8, device="cuda")

    def run(x, wait):
        z = op_linear(x, w)
        wait()
        op_lora(x, a, b, ids, base=z, y=z, scratch=scratch)
        wait()
        first = op_sample_filtered(z, u, T, top_p=0.9)
        wait()
        op_filter_logits(z, T, top_p=0.9, out=z)
        wait()
        return first, op_sample_filtered(z, u, T), z

    want = [run(x, torch.cuda.synchronize) for x in xs]
    for _ in range(8):
        got = [run(x, lambda: None) for x in xs]
        torch.cuda.synchronize()
        for one, other in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(one, other))
    for first, second, _ in want:
        assert torch.equal(first, second)        # a draw under a rule is one from its mask
