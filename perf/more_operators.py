"""A layer's keys and values between its Q/K/V projection and its O projection, as a program
calls the operators: the projection's rows made into queries, keys and values and put into a
cache, of bf16 or of 8-bit codes; and the attention of the rows over what the cache holds,
also where all sequences of a batch begin with one prefix.

Kinds of case (the "kind" of a case):

* append   op_kv_append, and for a cache of codes op_kv_read of the rows just put there;
* attend   op_attention, with or without a prefix that the batch shares.

Rows starts[b] .. starts[b+1]-1 of a call belong to sequence b, whose cache holds lens[b]
positions, the rows' own at the end: row j of n sits in slot s = lens[b] - n + j.

append: of a row of [q heads | k heads | v heads], each head's q and k are
  x / sqrt(mean(x^2) + eps) * gain        (where there are gains),
then rotated: the pair (x_i, x_{i+hd/2}) by the angle pos * base^(-2i/hd), with pos =
prefix + lens[b] - n + offset, the row's offset being j, in a draft tree the row's depth.
q is rounded to bf16.  A cache of bf16 takes k and v rounded; one of codes takes for each
head's vector scale = max(max|x|, 127 * 2^-64) / 127 and rint(x / scale).

attend: row j's head h gives sum_i w_i v_i / sum_i w_i, w_i = exp(q . k_i / sqrt(hd)), over
the prefix's positions and the slots up to its own; in a tree over the slots before the
rows' own and those of the rows whose bit is set in the row's mask.  Heads of one group
share a head of k and v.  A row that sees nothing gives zeros.
"""
import dataclasses
import functools
import math

import numpy as np
import torch

own = False
DEV = "cuda"
EPS = 1e-5
BASE = 10000.0
SMALLEST = 127.0 * 2.0 ** -64


def _append(name, **kw):
    base = dict(kind="append", name=name, seqs=1, rows=1, ragged=False, heads=32, kv_heads=32, hd=128, past=512, prefix=0,
                codes=False, norm=False, bf16_in=False, tree=False)
    return {**base, **kw}


def _attend(name, **kw):
    base = dict(kind="attend", name=name, seqs=1, rows=1, ragged=False, heads=32, kv_heads=32, hd=128, past=512, prefix=0,
                codes=False, tree=False, masked=False)
    return {**base, **kw}


def listed():
    return [
        # one decoded token of the 7B target (as many k/v heads as q heads) into its bf16 cache
        _append("append_one", past=2047),
        # the verify rows of sixteen requests of the 8B target (four heads to a group), K = 8, with
        # norms of q and k, into a cache of codes, and read back
        _append("append_144_codes", seqs=16, rows=9, kv_heads=8, past=2000, codes=True, norm=True),
        # a prompt of the 7B target in one call, q/k/v of 16 bits
        _append("append_2047", rows=2047, past=0, bf16_in=True, norm=True),
        # a draft tree of 21 rows of the 1.1B target (heads of 64), codes, read back
        _append("append_tree_21", rows=21, kv_heads=4, hd=64, past=1003, codes=True, norm=True, tree=True),
        # one decoded token of the 7B target: the smallest call
        _attend("attend_one", past=2047),
        # the verify rows of one request of the 7B target, K = 4, over a cache of codes
        _attend("attend_verify_5", rows=5, past=2048, codes=True),
        # a draft tree of the 1.1B target (eight heads to a group, heads of 64), an odd past
        _attend("attend_tree_21", rows=21, kv_heads=4, hd=64, past=1003, tree=True),
        # sixteen requests of the 8B target, prefixes of 512 to 4096, K = 8, a cache of codes
        _attend("attend_16x9_codes", seqs=16, rows=9, kv_heads=8, past=4096, ragged=True, codes=True),
        # a prefill pass: 256 rows of one prompt of the 8B target behind 4099 others
        _attend("attend_256_rows", rows=256, kv_heads=8, past=4099),
        # 64 requests decoding together, contexts up to 32768, codes: what fills a card
        _attend("attend_64_long", seqs=64, rows=1, kv_heads=8, past=32767, ragged=True, codes=True),
        # sixteen requests that begin with the same 8192 positions, K = 8
        _attend("attend_prefix_16x9", seqs=16, rows=9, kv_heads=8, past=512, ragged=True, prefix=8192),
        # 64 requests behind a prefix of 32768 in codes, decoding; some of them have no rows now
        _attend("attend_prefix_64", seqs=64, rows=1, kv_heads=8, past=1024, ragged=True, prefix=32768, codes=True,
                masked=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend"])
    hd = rng.choice([64, 128, 128])
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (32, 4), (12, 12), (16, 8), (40, 8), (6, 2)])
    case = dict(kind=kind, hd=hd, heads=heads, kv_heads=kv_heads, codes=rng.choice([False, True]))
    if kind == "append":
        rows = _log(rng, 1, 2047)
        seqs = rng.choice([1, _log(rng, 1, min(rows, 64))])
        case.update(seqs=seqs, rows=rows // seqs, ragged=rng.choice([False, True]), past=_log(rng, 1, 2048), prefix=0,
                    norm=rng.choice([False, True]), bf16_in=rng.choice([False, True]), tree=False)
        return case
    tree = rng.random() < 0.2
    seqs = _log(rng, 1, 64)
    rows = rng.randint(2, 32) if tree else rng.choice([1, rng.randint(1, 16), _log(rng, 1, 256)])
    prefix = rng.choice([0, 0, _log(rng, 1, 32768)])
    past = _log(rng, 1, 16384)
    case.update(seqs=seqs, rows=rows, ragged=rng.choice([False, True]), past=past, prefix=prefix, tree=tree,
                masked=rng.choice([False, True]))
    most = next(c for c in listed() if c["name"] == "attend_64_long")
    while _cost(case) > _cost(most):
        if case["seqs"] > 1:
            case["seqs"] -= 1
        else:
            case["past"] = case["past"] // 2 + 1
            case["prefix"] //= 2
    return case


def _cost(case):
    """A pass's cost, roughly: the bytes of its keys and values and the products of the plain form."""
    per = case["seqs"] * (case["past"] + case["rows"]) + case["prefix"]
    pairs = case["seqs"] * case["rows"] * (case["past"] + case["rows"] + case["prefix"])
    return per * case["kv_heads"] * case["hd"] * 4 + pairs * case["heads"] * case["hd"] / 20


def _case_rng(case):
    return np.random.default_rng([case["seqs"], case["rows"], case["past"], case["heads"], case["kv_heads"], case["prefix"]])


def _batch(case):
    """starts and lens of the sequences: of the case, not of the seed."""
    r, B, n, past = _case_rng(case), case["seqs"], case["rows"], case["past"]
    rows = np.full(B, n)
    pasts = np.full(B, past)
    if case["ragged"]:
        pasts = np.exp(r.uniform(math.log(max(1, past // 8)), math.log(past + 1), B)).astype(np.int64) if past else pasts
        if case["kind"] == "append" and n > 1:
            rows = r.integers(1, n + 1, B)
    if case.get("masked"):
        rows = np.where(np.arange(B) % 5 == 4, 0, rows)      # requests that wait
        pasts = np.where(np.arange(B) % 7 == 6, 0, pasts)    # requests that begin
    return np.concatenate([[0], np.cumsum(rows)]).astype(np.int32), (pasts + rows).astype(np.int32)


def _trees(case, starts):
    """Each row's offset (its depth) and the rows of its own sequence that it sees, as bits."""
    r = _case_rng(case)
    offsets, masks = np.zeros(starts[-1], np.int32), np.zeros(starts[-1], np.int32)
    for a, b in zip(starts[:-1], starts[1:]):
        for j in range(b - a):
            if j == 0:
                offsets[a], masks[a] = 0, 1
                continue
            p = int(r.integers(0, j))
            offsets[a + j] = offsets[a + p] + 1
            masks[a + j] = np.array([int(np.uint32(masks[a + p])) | 1 << j], np.uint32).view(np.int32)[0]
    return offsets, masks


# ------------------------------------------------------------------ inputs
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((seed * 1000003 + what * 7919) & 0x7FFFFFFFFFFF)


def _normal(seed, what, shape, std, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=_gen(seed, what))


@functools.lru_cache(maxsize=8)
def _rope(positions, hd):
    """cos and sin of pos * base^(-2i/hd), angles in 64 bits: fp32 [2][positions][hd/2]."""
    angle = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * BASE ** (
        -torch.arange(0, hd, 2, device=DEV, dtype=torch.float64)[None] / hd)
    return torch.stack([angle.cos(), angle.sin()]).float()


def _store(case, seed, what, seqs, positions):
    """k, v and (of codes) their scales: what a cache holds after earlier calls."""
    shape = (seqs, case["kv_heads"], positions, case["hd"])
    if not case["codes"]:
        return [_normal(seed, what, shape, 1.0), _normal(seed, what + 1, shape, 1.0)]
    # codes of normal vectors: the largest of a vector is 127 and stands for about 2.7
    codes = [torch.randint(0, 256, shape, device=DEV, generator=_gen(seed, what + i), dtype=torch.uint8) for i in (0, 1)]
    codes = [(_quantile()[c.int()] if c.numel() < 1 << 24 else _by_parts(c)) for c in codes]
    scales = [(0.017 + 0.01 * torch.rand(shape[:3], device=DEV, generator=_gen(seed, what + 2 + i))) for i in (0, 1)]
    return codes + scales


@functools.lru_cache(maxsize=1)
def _quantile():
    """256 codes that fall as a normal variable's do."""
    p = (torch.arange(256, device=DEV, dtype=torch.float64) + 0.5) / 256
    return (torch.erfinv(2 * p - 1) * math.sqrt(2) * 47).round().clamp(-127, 127).to(torch.int8)


def _by_parts(c):
    out = torch.empty(c.shape, dtype=torch.int8, device=DEV)
    for i in range(c.shape[0]):
        out[i] = _quantile()[c[i].int()]
    return out


@dataclasses.dataclass
class State:
    case: dict
    starts: torch.Tensor
    lens: torch.Tensor
    kv: list                       # k, v [, k_scale, v_scale]
    rows: int
    longest: int                   # rows of the longest sequence
    keys: int                      # positions of the longest sequence
    x: torch.Tensor = None         # append: the projection's rows
    rope: torch.Tensor = None
    gains: tuple = (None, None)
    offsets: torch.Tensor = None
    q: torch.Tensor = None         # attend
    mask: torch.Tensor = None
    prefix: list = None
    scratch: torch.Tensor = None
    handles: tuple = None          # the framework's views of kv and prefix, made once


def prepare(case, seed):
    starts, lens = _batch(case)
    n, hd, H, Hk = int(starts[-1]), case["hd"], case["heads"], case["kv_heads"]
    positions = -(-(int(lens.max()) + 8) // 8) * 8
    dev = lambda a: torch.from_numpy(a).to(DEV)
    offsets, mask = _trees(case, starts) if case["tree"] else (None, None)
    s = State(case, dev(starts), dev(lens), [], n, int(np.diff(starts).max()), int(lens.max()))
    if case["kind"] == "append":
        shape = (case["seqs"], Hk, positions, hd)
        s.kv = [torch.zeros(shape, dtype=torch.int8 if case["codes"] else torch.bfloat16, device=DEV) for _ in (0, 1)]
        if case["codes"]:
            s.kv += [torch.zeros(shape[:3], device=DEV) for _ in (0, 1)]
        s.x = _normal(seed, 1, (n, (H + 2 * Hk) * hd), 1.5, torch.bfloat16 if case["bf16_in"] else torch.float32)
        s.rope = _rope(positions + case["prefix"], hd)
        if case["norm"]:
            s.gains = tuple((1.0 + 0.2 * torch.randn(hd, device=DEV, generator=_gen(seed, w))).bfloat16() for w in (2, 3))
        s.offsets = None if offsets is None else dev(offsets)
        return s
    s.kv = _store(case, seed, 10, case["seqs"], positions)
    if case["prefix"]:
        s.prefix = _store(case, seed, 20, 1, case["prefix"])
    s.q = _normal(seed, 1, (n, H, hd), 2.0)
    s.mask = None if mask is None else dev(mask)
    s.scratch = torch.empty((64 << 20) + 16 * n * H * (hd + 8), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------ the operators
def _where(s):
    """Of each row: its sequence, its place among the sequence's rows, its slot."""
    rows = torch.arange(s.rows, device=DEV)
    b = torch.searchsorted(s.starts[1:].long(), rows, right=True)
    n = (s.starts[1:] - s.starts[:-1])[b].long()
    j = rows - s.starts[b]
    return b, j, s.lens[b].long() - n + j, n


def _plain_append(s):
    c = s.case
    H, Hk, hd = c["heads"], c["kv_heads"], c["hd"]
    b, j, slot, n = _where(s)
    q, k, v = s.x.float().view(s.rows, H + 2 * Hk, hd).split([H, Hk, Hk], 1)
    if s.gains[0] is not None:
        unit = lambda t, g: t * torch.rsqrt(t.square().mean(2, keepdim=True) + EPS) * g.float()
        q, k = unit(q, s.gains[0]), unit(k, s.gains[1])
    pos = c["prefix"] + slot - j + (j if s.offsets is None else s.offsets.long())
    cos, sin = s.rope[0][pos][:, None], s.rope[1][pos][:, None]

    def turn(t):
        lo, hi = t[..., :hd // 2], t[..., hd // 2:]
        return torch.cat([lo * cos - hi * sin, lo * sin + hi * cos], 2)

    q, k = turn(q).bfloat16(), turn(k)
    if not c["codes"]:
        s.kv[0][b, :, slot], s.kv[1][b, :, slot] = k.bfloat16(), v.bfloat16()
        return [q, s.kv[0], s.kv[1]]
    for i, t in enumerate((k, v)):
        scale = t.abs().amax(2).clamp(min=SMALLEST) / 127.0
        s.kv[i][b, :, slot] = torch.round(t / scale[:, :, None]).to(torch.int8)
        s.kv[2 + i][b, :, slot] = scale
    back = [(s.kv[i][b, :, slot].float() * s.kv[2 + i][b, :, slot][:, :, None]).bfloat16() for i in (0, 1)]
    return [q, *back]


def _values(kv, end):
    """k and v as they count, up to position `end`, in 32 bits."""
    k, v = kv[0][:, :, :end].float(), kv[1][:, :, :end].float()
    if len(kv) == 4:
        k, v = k * kv[2][:, :, :end, None], v * kv[3][:, :, :end, None]
    return k, v


def _plain_attend(s):
    c = s.case
    B, R, H, Hk, hd, L = c["seqs"], s.longest, c["heads"], c["kv_heads"], c["hd"], s.keys
    b, j, slot, n = _where(s)
    q = torch.zeros(B, R, H, hd, device=DEV)
    q[b, j] = s.q.float() * hd ** -0.5
    q = q.view(B, R, Hk, H // Hk, hd).permute(0, 2, 1, 3, 4)          # [seq][kv head][row][of the group][hd]
    k, v = _values(s.kv, L)
    z = (q.reshape(B, Hk, -1, hd) @ k.transpose(2, 3)).view(B, Hk, R, H // Hk, L)
    first = (s.lens - (s.starts[1:] - s.starts[:-1])).long()[:, None, None]
    at = torch.arange(L, device=DEV)[None, None]
    if s.mask is None:
        seen = at <= first + torch.arange(R, device=DEV)[None, :, None]
    else:
        bits = torch.zeros(B, R, dtype=torch.int64, device=DEV)
        bits[b, j] = s.mask.long()
        seen = (at < first) | ((bits[:, :, None] >> (at - first).clamp(0, 31)) & 1 > 0)
    seen = seen & (at < s.lens.long()[:, None, None])
    z = z.masked_fill(~seen[:, None, :, None], -math.inf)
    if s.prefix is not None:
        pk, pv = _values(s.prefix, c["prefix"])
        flat = q.permute(1, 0, 2, 3, 4).reshape(Hk, -1, hd)
        zp = (flat @ pk[0].transpose(1, 2)).view(Hk, B, R, H // Hk, -1).transpose(0, 1)
        top = torch.maximum(z.amax(4, keepdim=True), zp.amax(4, keepdim=True))
        wp = torch.exp(zp - top)
    else:
        top = z.amax(4, keepdim=True)
        top = torch.where(top > -math.inf, top, 0.0)
    w = torch.exp(z - top)
    total = w.sum(4)
    out = (w.view(B, Hk, -1, L) @ v).view(B, Hk, R, H // Hk, hd)
    if s.prefix is not None:
        total = total + wp.sum(4)
        out = out + (wp.transpose(0, 1).reshape(Hk, -1, c["prefix"]) @ pv[0]).view(Hk, B, R, H // Hk, hd).transpose(0, 1)
    out = torch.where(total[..., None] > 0, out / total[..., None], 0.0)
    return out.permute(0, 2, 1, 3, 4).reshape(B, R, H, hd)[b, j].bfloat16()


def run(state):
    s, c = state, state.case
    if own:
        import paper_2608_10362_gb300 as pkg
        if s.handles is None:
            s.handles = (pkg.KVCache(*s.kv), pkg.KVCache(*s.prefix) if s.prefix else None)
        cache, prefix = s.handles
        if c["kind"] == "attend":
            return pkg.op_attention(s.q, cache, s.starts, s.lens, max_rows=s.longest, tree=s.mask, prefix=prefix,
                                    scratch=s.scratch)
        q = pkg.op_kv_append(s.x, cache, s.starts, s.lens, c["heads"], rope=s.rope, offsets=s.offsets,
                             prefix_len=c["prefix"], q_gain=s.gains[0], k_gain=s.gains[1], eps=EPS)
        if c["codes"]:
            return [q, *pkg.op_kv_read(cache, s.starts, s.lens, s.rows)]
        return [q, *s.kv]
    return (_plain_append if c["kind"] == "append" else _plain_attend)(s)


def work(case):
    starts, lens = _batch(case)
    n, hd, H, Hk = int(starts[-1]), case["hd"], case["heads"], case["kv_heads"]
    vector = hd + 4 if case["codes"] else 2 * hd
    if case["kind"] == "append":
        values = n * (H + 2 * Hk) * hd
        put = 2 * n * Hk * (vector + (vector + 2 * hd if case["codes"] else 0))    # written; of codes read back too
        return {"bytes": values * (2 if case["bf16_in"] else 4) + 2 * n * H * hd + put + 4 * n * hd,
                "flops": values * 8}
    rows = np.diff(starts)
    own_keys = int(lens[rows > 0].sum())
    pairs = int((rows * (lens - rows) + (rows * (rows + 1)) // 2).sum()) + n * case["prefix"]
    return {"bytes": 4 * n * H * hd + 2 * (own_keys + case["prefix"]) * Hk * vector, "flops": 4 * pairs * H * hd}


# ------------------------------------------------------------------ 64-bit values
def _exact_append(case, s):
    """Row by row in NumPy, from the definition."""
    H, Hk, hd, half = case["heads"], case["kv_heads"], case["hd"], case["hd"] // 2
    starts, lens = _batch(case)
    x = s.x.double().cpu().numpy().reshape(s.rows, H + 2 * Hk, hd)
    offsets = None if s.offsets is None else s.offsets.cpu().numpy()
    cache = [np.zeros(tuple(s.kv[0].shape)) for _ in (0, 1)] if not case["codes"] else None
    q = np.empty((s.rows, H, hd))
    back = [np.empty((s.rows, Hk, hd)) for _ in (0, 1)]
    theta = BASE ** (-2.0 * np.arange(half) / hd)
    gains = [None if g is None else g.double().cpu().numpy() for g in s.gains]
    for b in range(case["seqs"]):
        for r in range(starts[b], starts[b + 1]):
            j = r - starts[b]
            slot = lens[b] - (starts[b + 1] - starts[b]) + j
            pos = case["prefix"] + slot - j + (j if offsets is None else offsets[r])
            heads = x[r].copy()
            if gains[0] is not None:
                heads[:H + Hk] /= np.sqrt((heads[:H + Hk] ** 2).mean(1, keepdims=True) + EPS)
                heads[:H] *= gains[0]
                heads[H:H + Hk] *= gains[1]
            turn = np.exp(1j * pos * theta)
            z = (heads[:H + Hk, :half] + 1j * heads[:H + Hk, half:]) * turn
            heads[:H + Hk, :half], heads[:H + Hk, half:] = z.real, z.imag
            q[r] = heads[:H]
            for i, t in enumerate((heads[H:H + Hk], heads[H + Hk:])):
                if case["codes"]:
                    scale = np.maximum(np.abs(t).max(1, keepdims=True), SMALLEST) / 127.0
                    back[i][r] = np.rint(t / scale) * scale
                else:
                    cache[i][b, :, slot] = t
    return [torch.from_numpy(t) for t in ([q, *back] if case["codes"] else [q, *cache])]


def _exact_attend(case, s):
    """Sequence by sequence and head by head of k and v, in 64 bits."""
    H, Hk, hd = case["heads"], case["kv_heads"], case["hd"]
    starts, lens = _batch(case)
    masks = None if s.mask is None else s.mask.cpu().numpy().view(np.uint32)
    out = torch.zeros(s.rows, H, hd, dtype=torch.float64, device=DEV)

    def as_counts(kv, b, h, i, end):
        t = kv[i][b, h, :end].double()
        return t * kv[2 + i][b, h, :end].double()[:, None] if len(kv) == 4 else t

    for b in range(case["seqs"]):
        lo, hi, L = int(starts[b]), int(starts[b + 1]), int(lens[b])
        n = hi - lo
        if n == 0:
            continue
        seen = np.arange(L)[None] <= (L - n + np.arange(n))[:, None]
        if masks is not None:
            bits = (masks[lo:hi, None] >> np.arange(n, dtype=np.uint32)[None]) & 1
            seen[:, L - n:] = bits.astype(bool)
        seen = np.concatenate([np.ones((n, case["prefix"]), bool), seen], 1)
        seen = torch.from_numpy(np.repeat(seen, H // Hk, 0)).to(DEV)
        for h in range(Hk):
            k, v = (as_counts(s.kv, b, h, i, L) for i in (0, 1))
            if s.prefix is not None:
                k, v = (torch.cat([as_counts(s.prefix, 0, h, i, case["prefix"]), t]) for i, t in ((0, k), (1, v)))
            q = s.q[lo:hi, h * (H // Hk):(h + 1) * (H // Hk)].double().reshape(-1, hd)
            z = torch.where(seen, q @ k.T / math.sqrt(hd), -math.inf)
            w = torch.softmax(z, 1) if L + case["prefix"] else z
            out[lo:hi, h * (H // Hk):(h + 1) * (H // Hk)] = (torch.nan_to_num(w) @ v).view(n, H // Hk, hd)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(case, s)
    if case["seqs"] * case["kv_heads"] > 2048:
        return None
    return _exact_attend(case, s)
