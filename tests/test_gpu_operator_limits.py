"""Sampling rules at the ends of what 32 bits hold, against their 64-bit definition."""
import numpy as np
import pytest

from oracle import filtering as F

pytestmark = pytest.mark.gpu

HOT = [1e19, 2e19, 1e28, 1e36, 1e37, 3e37, 1e38, 2e38, F.LARGEST, np.inf]


def _wide(kind, rows, vocab, seed=0):
    """Logits over all that fp32 holds: steps (infinities, the largest and the lowest finite
    number, NaN and some between, many equal) or spread evenly."""
    rng = np.random.default_rng([seed, rows, vocab])
    if kind == "steps":
        v = np.array([np.inf, F.LARGEST, 2e38, 12.0, 0.0, -1e38, -F.LARGEST, -np.inf, np.nan], np.float32)
        return v[rng.choice(len(v), (rows, vocab), p=[.02, .02, .1, .2, .2, .2, .2, .03, .03])]
    return (rng.uniform(-1, 1, (rows, vocab)) * F.LARGEST).astype(np.float32)


def _both(z, u, rules):
    """Draws and masks on the GPU, one rule per row."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    per = [torch.tensor([float(r[i]) if i != 1 else r[i] for r in rules], dtype=torch.int32 if i == 1 else torch.float32,
                        device="cuda") for i in range(4)]
    zt = torch.from_numpy(z).cuda()
    return (op_sample_filtered(zt, torch.from_numpy(u).cuda(), *per).cpu().numpy(),
            op_filter_logits(zt, *per).cpu().numpy())


def _uniforms(rows, seed=0):
    return ((2 * np.random.default_rng([seed, rows]).integers(0, 1 << 23, rows) + 1) * 2.0 ** -24).astype(np.float32)


def _compare(z, u, rules):
    drawn, masked = _both(z, u, rules)
    for r, rule in enumerate(rules):
        assert np.array_equal(masked[r], F.mask(z[r], *rule)), (r, rule)
        assert drawn[r] == F.draw(z[r], u[r], *rule), (r, rule)


@pytest.mark.parametrize("kind", ["steps", "spread"])
@pytest.mark.parametrize("vocab", [300, 5000, 40000])
def test_temperatures_up_to_infinity_over_logits_of_any_size(kind, vocab):
    """max - z passes the largest float, 1 / T falls below the smallest normal one."""
    rules = [(T, k, p, 0.0) for T in HOT for k, p in ((0, 1.0), (0, 0.9), (0, 0.3), (100, 1.0), (150, 0.8), (1200, 0.7))]
    _compare(_wide(kind, len(rules), vocab), _uniforms(len(rules)), rules)


@pytest.mark.parametrize("kind", ["steps", "spread"])
@pytest.mark.parametrize("vocab", [300, 5000, 40000])
def test_min_p_at_temperatures_up_to_infinity(kind, vocab):
    """T log(min_p) passes the largest float where the bound max + T log(min_p) does not."""
    rules = [(T, k, p, m) for T in HOT for m in (1e-30, 0.01, 0.1, 0.5, 0.9, 1 - 2.0 ** -24, 1.0)
             for k, p in ((0, 1.0), (120, 0.9))]
    _compare(_wide(kind, len(rules), vocab, 1), _uniforms(len(rules), 1), rules)


def test_temperatures_below_the_lowest_count_as_it():
    """All parts of a rule take 1e-30 for a smaller temperature above 0: logits some 1e-31 apart."""
    rng = np.random.default_rng(4)
    z = (np.round(rng.normal(size=(40, 3000)) * 8) * 1e-31).astype(np.float32)
    rules = [(T, k, p, m) for T in (1e-45, 1e-38, 1e-33, 9e-31, 1e-30) for m in (0.0, 0.3)
             for k, p in ((0, 1.0), (0, 0.9), (100, 1.0), (900, 0.8))]
    _compare(z, _uniforms(len(rules), 2), rules)


@pytest.mark.parametrize("vocab", [1, 2, 3, 4, 5])
def test_single_ids_at_every_alignment(vocab):
    """The shortest rows under every kind of rule, in place and not, wherever they begin."""
    import torch
    from paper_2608_10362_gb300 import op_filter_logits, op_sample_filtered
    z = np.array([[0.5, -1.0, 0.5, 2.0, np.nan], [-np.inf, 3.0, np.inf, -F.LARGEST, 0.0]], np.float32)[:, :vocab]
    rules = [(1.0, 0, 0.9, 0.0), (1.0, 0, 1e-3, 0.0), (0.7, 1, 0.9, 0.0), (0.7, 2, 0.5, 0.1), (2.0, 0, 1.0, 0.4),
             (0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.0)]
    u = torch.tensor([0.3], device="cuda")
    for at in range(4):
        for row in z:
            raw = torch.full((at + vocab + 4,), 1e30, device="cuda")
            zt = raw[at:at + vocab].view(1, vocab)
            for rule in rules:
                zt.copy_(torch.from_numpy(row))
                kw = dict(zip(("temperature", "top_k", "top_p", "min_p"), rule))
                want = F.mask(row, *rule)
                assert op_sample_filtered(zt, u, **kw).tolist() == [F.draw(row, float(u[0]), *rule)]
                assert np.array_equal(op_filter_logits(zt, **kw).cpu().numpy()[0], want)
                op_filter_logits(zt, **kw, out=zt)
                assert np.array_equal(zt.cpu().numpy()[0], want)
                assert bool((raw[:at] == 1e30).all()) and bool((raw[at + vocab:] == 1e30).all())


def _sparse_lora(adapters, rank, k, n, rows, ids, seed):
    """A call on zeros but for some whole numbers in the adapters that the rows have: the result by
    picking those out."""
    import torch
    from paper_2608_10362_gb300 import op_lora
    rng = np.random.default_rng(seed)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    a, b = torch.zeros(adapters, rank, k, **bf), torch.zeros(adapters, n, rank, **bf)
    x = torch.zeros(rows, k, **bf)
    cols = np.unique(np.concatenate([[0, k - 1], rng.integers(0, k, 60)]))
    outs = np.unique(np.concatenate([[0, n - 1], rng.integers(0, n, 60)]))
    xv = rng.integers(-3, 4, (rows, len(cols)))
    x[:, torch.from_numpy(cols).cuda()] = torch.from_numpy(xv).to(**bf)
    base = torch.from_numpy(rng.integers(-50, 51, (rows, n)).astype(np.float32)).cuda()
    want = base.clone()
    for i in sorted({i for i in ids if 0 <= i < adapters}):
        av, bv = rng.integers(-3, 4, (rank, len(cols))), rng.integers(-3, 4, (len(outs), rank))
        a[i, :, torch.from_numpy(cols).cuda()] = torch.from_numpy(av).to(**bf)
        b[i, torch.from_numpy(outs).cuda()] = torch.from_numpy(bv).to(**bf)
        for r in np.flatnonzero(np.array(ids) == i):
            want[int(r), torch.from_numpy(outs).cuda()] += torch.from_numpy(bv @ (av @ xv[r])).float().cuda()
    got = op_lora(x, a, b, torch.tensor(ids, dtype=torch.int32, device="cuda"), base=base)
    assert torch.equal(got, want)


@pytest.mark.parametrize("adapters,rank,k,n,rows", [
    (70, 128, 262144, 64, 3),          # A past 2^31 elements
    (70, 128, 64, 262144, 3),          # B
    (300, 32, 262144, 40, 40), (300, 16, 64, 524288, 2),
    (1, 8, 1 << 24, 32, 2), (2, 8, 64, 1 << 24, 2), (1, 32, 64, (1 << 24) - 3, 1),   # the longest rows
    (1 << 24, 8, 8, 1, 5)])            # the most adapters
def test_adapters_past_what_32_bits_address(adapters, rank, k, n, rows):
    ids = [adapters - 1, 0, adapters, adapters - 1, adapters // 2][:rows] + [adapters - 1 - r % 3 for r in range(max(0, rows - 5))]
    _sparse_lora(adapters, rank, k, n, rows, ids, rank + rows)
