"""Every row that a step with sampling rules leaves behind, against the same row of a step
without them: a draft's later rows and all of a tree's."""
import numpy as np
import pytest
import torch

from oracle import filtering as F
from oracle.philox import uniform
from oracle.speculative import softmax_t
from seeded_inputs import gen_prompt
from test_gpu_sampling_rules import _engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1.0, 0.03, 0.015])
def test_draft_rows_are_cut_by_their_requests_rule(T):
    """As long as a request's draws are those without a rule (the uniforms are the same), the next
    draft row before the cut is the same too; mostly so at low temperatures, where few ids of
    these random-init models hold nearly all of the sum."""
    K, B = 4, 4
    eng, plain = _engine(use_graphs=True), _engine(use_graphs=False)
    compared = np.zeros((B, K), int)
    sets = [[(0, 0.97, 0.0), (12, 1.0, 0.0), (0, 1.0, 0.02), (300, 0.98, 0.01)],
            [(60, 1.0, 0.0), (0, 0.95, 0.0), (150, 0.95, 0.0), (0, 1.0, 0.01)]]
    for case in range(16):
        rules = sets[case % 2]
        for e in (eng, plain):
            for b in range(B):
                e.prefill(b, gen_prompt(300 + 10 * case + b, 20 + 9 * b, e.vocab), seed=40 + case)
            e.set_batch(B)
        for b, rule in enumerate(rules):
            eng.set_sampling(b, *rule)
        for e in (eng, plain):
            e.draft_step(K, T)
            assert e.sync() == 0
        cut, whole = eng.draft_logits(B, K), plain.draft_logits(B, K)
        x, y = eng.draft_tokens(B), plain.draft_tokens(B)
        for b in range(B):
            for j in range(K):
                assert np.array_equal(cut[b, j], F.mask(whole[b, j], T, *rules[b])), (case, b, j)
                assert np.isfinite(cut[b, j, x[b, j]])
                compared[b, j] += 1
                if x[b, j] != y[b, j]:
                    break
    assert T == 1.0 or np.all(compared[:, 1:] >= 3), compared
    eng.close()
    plain.close()


def _slot(z, T, rule, u):
    """The draw from a row's cut, and whether u lies within a rounding of a border."""
    cut = F.mask(z, T, *rule)
    c = np.cumsum(softmax_t(cut, T))
    return F.draw(z, u, T, *rule), np.min(np.abs(c - u)) < 1e-5


@pytest.mark.parametrize("graphs", [False, True])
@pytest.mark.parametrize("rule", [(30, 0.9, 0.0), (0, 0.6, 0.0), (0, 1.0, 0.3), (500, 1.0, 0.0), (64, 0.95, 0.05)])
def test_tree_rows_and_the_walk_are_cut(rule, graphs):
    from paper_2608_10362_gb300 import _lib
    T, seed = 0.8, 2
    eng, plain = _engine(batch=1, use_graphs=graphs), _engine(batch=1, use_graphs=False)
    res = torch.zeros(66, dtype=torch.int32, pin_memory=True)

    def rows(e, tokens, parents, cut):
        e.prefill(0, gen_prompt(4, 50, e.vocab), seed=seed)
        if cut:
            e.set_sampling(0, *rule)
        e.tree_step(tokens, parents, T, res)
        assert e.sync() == 0
        n = len(tokens) + 1
        return e.read_buffer(_lib.BUF_TREE_LOGITS, np.float32, n * e.vocab).reshape(n, -1)

    # a path of the rule's own draws, with another child beside each node
    tokens, parents, node = [], [], -1
    for e in range(4):
        z = rows(plain, tokens + [0], parents + [node], False)[node + 1]
        x, _ = _slot(z, T, rule, uniform(seed, 0, 0, 64 + e))
        tokens += [int(x), (int(x) + 1) % plain.vocab]
        parents += [node, node]
        node = len(tokens) - 2
    whole = rows(plain, tokens, parents, False)
    cut = rows(eng, tokens, parents, True)
    for r in range(len(tokens) + 1):
        assert np.array_equal(cut[r], F.mask(whole[r], T, *rule)), r
    r, near, want = 0, False, []
    while True:
        x, close = _slot(whole[r], T, rule, uniform(seed, 0, 0, 64 + len(want)))
        near |= close
        want.append(x)
        child = [i for i, (t, p) in enumerate(zip(tokens, parents)) if p == r - 1 and t == x]
        if not child:
            break
        r = child[0] + 1
    got = res[2:2 + int(res[0])].tolist()
    assert got == want or near
    assert len(want) >= 3
    eng.close()
    plain.close()


def test_rules_of_some_requests_shorter_steps_and_smaller_batches():
    """K below max_k; a rule on one request of the batch, or on one past it; a rule that changes
    between replays of one graph."""
    T, K = 0.9, 2
    eng = _engine(batch=4, use_graphs=True)
    for b in range(4):
        eng.prefill(b, gen_prompt(70 + b, 25 + 3 * b, eng.vocab), seed=8 + b)
    off = (0, 1.0, 0.0)
    for batch, rules in ((2, {2: (7, 1.0, 0.0)}), (4, {2: (7, 1.0, 0.0)}), (3, {1: (0, 0.5, 0.0)}),
                         (4, {0: (0, 1.0, 0.8), 1: (9, 0.9, 0.0)}), (4, {}), (1, {0: (3, 1.0, 0.0)})):
        eng.set_batch(batch)
        for b in range(4):
            eng.set_sampling(b, *rules.get(b, off))
        for _ in range(2):
            eng.draft_step(K, T)
            eng.verify_step(K)
            assert eng.sync() == 0
            whole, drafts = eng.target_logits(batch, K), eng.draft_logits(batch, K)
            assert np.isfinite(whole).all()
            eng.accept_commit(K, T, eng.results_host)
            assert eng.sync() == 0
            cut = eng.target_logits(batch, K)
            for b in range(batch):
                for i in range(K + 1):
                    assert np.array_equal(cut[b, i], F.mask(whole[b, i], T, *rules.get(b, off))), (batch, b, i)
                for j in range(K):
                    assert np.isfinite(drafts[b, j]).all() == (b not in rules)
    eng.close()
