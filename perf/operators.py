"""The operators of a batch whose requests differ, as a program calls them: each request's
own sampling rule on its rows of logits, and each request's own low-rank adapter beside a
projection that all of them share.

Kinds of case (the "kind" of a case):

* sample   op_sample_filtered: one draw per row from softmax(z / T) cut down by the row's
           top-k, top-p and min-p, with uniforms that are given;
* filter   op_filter_logits: the same cut as a mask on the logits (what the acceptance
           test of a speculative step compares has to be cut on both sides);
* lora     op_lora: y = base + scale[a] (x A[a]^T) B[a]^T, a = the row's adapter or none.

The kept ids of a row are a prefix of its ids by descending logit (equal logits: by
ascending id), the shortest of three:
  top-k   the first k;
  top-p   of those, the shortest whose weights exp((z - max) / T) sum to at least
          p times the sum over the first k (over all ids without top-k);
  min-p   the ids with exp((z - max) / T) >= min_p.
The draw is the first id, ascending, at which the running sum of the kept weights passes
u times their sum.  T = 0: the first id of the largest logit.  NaN logits count as -inf,
+inf as the largest finite number; a row without any finite logit draws -1 and keeps
nothing.
"""
import dataclasses
import math

import numpy as np
import torch

own = False
DEV = "cuda"
LARGEST = torch.finfo(torch.float32).max

# T, top-k (0: off), top-p (1: off), min-p (0: off): rules that requests of one batch carry
RULES = {
    "off": [(1.0, 0, 1.0, 0.0)],
    "topk": [(0.8, 50, 1.0, 0.0)],
    "topp": [(1.0, 0, 0.9, 0.0)],
    "topk_topp": [(0.7, 50, 0.95, 0.0)],
    "minp": [(1.1, 0, 1.0, 0.05)],
    "mixed": [(0.7, 50, 0.95, 0.0), (1.0, 0, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.05), (1.3, 0, 1.0, 0.0),
              (0.8, 40, 1.0, 0.0), (1.0, 1000, 0.98, 0.02), (0.6, 0, 0.8, 0.1), (1.0, 1, 1.0, 0.0)],
}


def listed():
    return [
        # one token of one request (the 7B target's vocabulary) under the usual top-k and top-p
        dict(name="sample_one", kind="sample", rows=1, vocab=32000, rule="topk_topp", logits="peaked"),
        # sixteen requests decoding together at a 128K vocabulary, nucleus sampling
        dict(name="sample_16_topp", kind="sample", rows=16, vocab=128256, rule="topp", logits="peaked"),
        # the flat logits of a random-init model: the nucleus is most of an odd vocabulary
        dict(name="sample_21_flat", kind="sample", rows=21, vocab=32003, rule="topp", logits="flat"),
        # every row of a batched verify pass (16 requests x 9 rows), a rule per request
        dict(name="sample_144_mixed", kind="sample", rows=144, vocab=128256, rule="mixed", logits="peaked"),
        # the K + 1 target rows of one request's verify pass before acceptance
        dict(name="filter_5", kind="filter", rows=5, vocab=32000, rule="topk_topp", logits="peaked"),
        # the target rows of 16 requests x 9, logits that were rounded to bf16 (many equal ones)
        dict(name="filter_144_bf16", kind="filter", rows=144, vocab=128256, rule="mixed", logits="bf16"),
        # one decoded row with one adapter on the 7B target's O projection: the smallest call
        dict(name="lora_one", kind="lora", rows=1, n=4096, k=4096, rank=16, adapters=1, who="one", strided=False),
        # sixteen requests with an adapter each on the 8B target's Q projection, whose output is
        # a part of the fused Q/K/V rows
        dict(name="lora_16_q", kind="lora", rows=16, n=4096, k=4096, rank=16, adapters=16, who="each", strided=True),
        # gate/up of the 8B target at 16 requests x 9 rows, ranks up to 64, some requests without one
        dict(name="lora_144_gate_up", kind="lora", rows=144, n=28672, k=4096, rank=64, adapters=16, who="some", strided=False),
        # a prefill pass of 256 rows of one request through the down projection
        dict(name="lora_256_down", kind="lora", rows=256, n=4096, k=14336, rank=128, adapters=4, who="one", strided=False),
        # an LM head of odd size at the rows of a draft tree
        dict(name="lora_21_lm_head", kind="lora", rows=21, n=32003, k=2048, rank=24, adapters=8, who="some", strided=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "filter", "lora", "lora"])
    if kind == "lora":
        return dict(kind=kind, rows=_log(rng, 1, 256), n=_log(rng, 64, 32768), k=8 * _log(rng, 16, 1792),
                    rank=8 * rng.randint(1, 16), adapters=rng.randint(1, 32), who=rng.choice(["one", "each", "some"]),
                    strided=rng.choice([False, True]))
    rows, vocab = _log(rng, 1, 256), _log(rng, 2000, 131072)
    while rows * vocab > 144 * 128256:
        rows -= 1
    return dict(kind=kind, rows=rows, vocab=vocab, rule=rng.choice(sorted(RULES)),
                logits=rng.choice(["peaked", "flat", "bf16", "masked"]))


# ------------------------------------------------------------------ inputs
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((seed * 1000003 + what * 7919) & 0x7FFFFFFFFFFF)


def _logits(case, seed):
    """peaked: weights that fall by rank as a trained model's do, with noise; flat: a
    random-init model's; bf16: peaked ones rounded to bf16; masked: nine tenths of the ids
    ruled out (-inf), and in the first row of four or more all of them."""
    R, V = case["rows"], case["vocab"]
    g = _gen(seed, 1)
    z = torch.randn(R, V, device=DEV, generator=g)
    if case["logits"] == "flat":
        return z
    order = torch.rand(R, V, device=DEV, generator=g).argsort(1).float()
    z = 12.0 - 1.4 * torch.log1p(order) + 0.7 * z
    if case["logits"] == "bf16":
        z = z.to(torch.bfloat16).float()
    if case["logits"] == "masked":
        z = z.masked_fill(torch.rand(R, V, device=DEV, generator=g) < 0.9, -math.inf)
        if R >= 4:
            z[0] = -math.inf
    return z


def _uniforms(case, seed):
    g = _gen(seed, 2)
    return (2 * torch.randint(0, 1 << 23, (case["rows"],), device=DEV, generator=g) + 1).double().mul(2.0 ** -24).float()


def _rule(case):
    """temperature, top_k, top_p, min_p: numbers, or where the requests differ a value per row."""
    rules = RULES[case["rule"]]
    if len(rules) == 1:
        return rules[0]
    per = [rules[r % len(rules)] for r in range(case["rows"])]
    kinds = (torch.float32, torch.int32, torch.float32, torch.float32)
    return tuple(torch.tensor([p[i] for p in per], dtype=kinds[i], device=DEV) for i in range(4))


def _lora_rows(case):
    """Each row's adapter (-1: none) and each adapter's rank: of the case, not of the seed."""
    R, N = case["rows"], case["adapters"]
    r = np.random.default_rng([R, case["n"], case["k"], N])
    if case["who"] == "one":
        ids = np.full(R, int(r.integers(N)))
    else:
        each = max(1, R // max(N, 1))               # rows of one request stand together
        ids = r.permutation(N)[(np.arange(R) // each) % N]
        if case["who"] == "some":
            ids = np.where((np.arange(R) // each) % 4 == 3, -1, ids)
            ids[0] = max(ids[0], 0)
    ranks = np.maximum(1, case["rank"] // r.choice([1, 1, 2, 4], size=N)) if N > 1 else np.array([case["rank"]])
    return ids.astype(np.int32), ranks.astype(np.int32)


@dataclasses.dataclass
class State:
    case: dict
    z: torch.Tensor = None
    u: torch.Tensor = None
    rule: tuple = None
    x: torch.Tensor = None
    a: torch.Tensor = None
    b: torch.Tensor = None
    ids: torch.Tensor = None
    ranks: torch.Tensor = None
    scales: torch.Tensor = None
    base: torch.Tensor = None
    scratch: torch.Tensor = None


def prepare(case, seed):
    if case["kind"] != "lora":
        return State(case, z=_logits(case, seed), u=_uniforms(case, seed), rule=_rule(case))
    R, n, k, rank, N = (case[w] for w in ("rows", "n", "k", "rank", "adapters"))
    ids, ranks = _lora_rows(case)
    normal = lambda what, shape, std: torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(
        0.0, std, generator=_gen(seed, what))
    base = torch.randn(R, n + (1024 if case["strided"] else 0), device=DEV, generator=_gen(seed, 3))
    return State(case, x=normal(4, (R, k), 1.0), a=normal(5, (N, rank, k), k ** -0.5), b=normal(6, (N, n, rank), 0.05),
                 ids=torch.from_numpy(ids).to(DEV), ranks=torch.from_numpy(ranks).to(DEV),
                 scales=0.5 + 1.5 * torch.rand(N, device=DEV, generator=_gen(seed, 7)), base=base[:, :n],
                 scratch=torch.empty(32 << 20, dtype=torch.uint8, device=DEV))


# ------------------------------------------------------------------ the operators
def _kept(z, rule):
    """Plain form of the cut: (ids by descending logit, their weights, whether each is kept)."""
    T, k, p, m = (torch.as_tensor(v, device=DEV).view(-1, 1) for v in rule)
    zs, order = torch.sort(z, dim=1, descending=True, stable=True)
    top = zs[:, :1]
    live = zs > -math.inf
    greedy = T <= 0
    # exp((z - max) / T) in 64 bits: what decides stands next to borders
    w = torch.exp((zs.double() - top.double()) / torch.where(greedy, 1.0, T).double())
    w = torch.where(live, w, 0.0)
    place = torch.arange(zs.shape[1], device=DEV)[None]
    keep = live & ((k <= 0) | (place < k))
    wk = torch.where(keep, w, 0.0)
    cum = torch.cumsum(wk, 1)
    enough = p.double() * cum[:, -1:]
    keep &= (p >= 1) | (cum - wk < enough) | (place == 0)
    keep &= w >= m.double()
    return order, w, torch.where(greedy, place == 0, keep) & live


def _sane(z):
    return torch.where(torch.isnan(z), -math.inf, z).clamp(max=LARGEST)


def _plain_sample(s):
    order, w, keep = _kept(_sane(s.z), s.rule)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))
    cum = torch.cumsum(w, 1)
    passed = cum > s.u.double().view(-1, 1) * cum[:, -1:]
    return torch.where(passed.any(1), passed.to(torch.uint8).argmax(1), -1).int()


def _plain_filter(s):
    z = _sane(s.z)
    order, _, keep = _kept(z, s.rule)
    return torch.where(torch.zeros_like(keep).scatter_(1, order, keep), z, -math.inf)


def _plain_lora(s):
    N, rank, k = s.a.shape
    n = s.b.shape[1]
    t = (s.x.float() @ s.a.float().view(N * rank, k).T).view(-1, N, rank)
    mine = torch.arange(N, device=DEV)[None] == s.ids[:, None]
    used = torch.arange(rank, device=DEV)[None] < s.ranks[:, None]
    t = torch.where(mine[:, :, None] & used[None], t, 0.0) * s.scales[None, :, None]
    return s.base + t.view(-1, N * rank) @ s.b.float().transpose(1, 2).reshape(N * rank, n)


def run(state):
    s, kind = state, state.case["kind"]
    if own:
        import paper_2608_10362_gb300 as pkg
        if kind == "lora":
            return pkg.op_lora(s.x, s.a, s.b, s.ids, scales=s.scales, ranks=s.ranks, base=s.base, scratch=s.scratch)
        T, k, p, m = s.rule
        if kind == "sample":
            return pkg.op_sample_filtered(s.z, s.u, temperature=T, top_k=k, top_p=p, min_p=m)
        return pkg.op_filter_logits(s.z, temperature=T, top_k=k, top_p=p, min_p=m)
    return {"sample": _plain_sample, "filter": _plain_filter, "lora": _plain_lora}[kind](s)


def work(case):
    if case["kind"] != "lora":
        values = case["rows"] * case["vocab"]
        return {"bytes": (4 if case["kind"] == "sample" else 8) * values + 8 * case["rows"], "flops": 2 * values}
    ids, ranks = _lora_rows(case)
    R, n, k = case["rows"], case["n"], case["k"]
    weights = sum(2 * int(ranks[i]) * (n + k) for i in set(ids.tolist()) if i >= 0)
    rows = [int(ranks[i]) for i in ids if i >= 0]
    return {"bytes": weights + 2 * len(rows) * k + 8 * R * n, "flops": 2 * sum(rows) * (n + k)}


# ------------------------------------------------------------------ 64-bit values
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return None          # whole numbers: a draw has no value in more bits
    if case["kind"] == "filter":
        # row by row from the definition, the ids ranked by (-logit, id) as one list
        out = torch.full(s.z.shape, -math.inf, dtype=torch.float64, device=DEV)
        rules = RULES[case["rule"]]
        for r in range(case["rows"]):
            T, k, p, m = rules[r % len(rules)]
            p, m, T = float(np.float32(p)), float(np.float32(m)), float(np.float32(T))
            z = s.z[r].double()
            ids = torch.argsort(-z, stable=True)
            ids = ids[torch.isfinite(z[ids])]
            if ids.numel() == 0:
                continue
            if T == 0:
                k, p, m, T = 1, 1.0, 0.0, 1.0
            ids = ids[:k] if k > 0 else ids
            w = ((z[ids] - z[ids[0]]) / T).exp()
            n = ids.numel()
            if p < 1:
                n = min(n, 1 + int((w.cumsum(0) < p * w.sum()).sum()))
            ids = ids[:n][w[:n] >= m]
            out[r, ids] = z[ids]
        return out
    out = s.base.double()
    ids, ranks = _lora_rows(case)
    for i in sorted(set(ids.tolist()) - {-1}):
        rows = torch.from_numpy(np.nonzero(ids == i)[0]).to(DEV)
        rk = int(ranks[i])
        t = s.x[rows].double() @ s.a[i, :rk].double().T
        out[rows] += float(s.scales[i]) * (t @ s.b[i, :, :rk].double().T)
    return out
