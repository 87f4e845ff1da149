"""Sampling rules in the engine's steps (memspec_set_sampling): the draft's draws, both
sides of the acceptance test and a tree's draws are cut by each request's own rule."""
import numpy as np
import pytest
import torch

from oracle import filtering as F
from oracle.philox import step_uniforms
from oracle.speculative import accept, softmax_t
from seeded_inputs import SHAPES, gen_logits, gen_prompt, gen_weights

pytestmark = pytest.mark.gpu

RULES = [(0, 1.0, 0.0), (40, 1.0, 0.0), (0, 0.9, 0.0), (200, 0.8, 0.02), (0, 1.0, 0.1), (1, 1.0, 0.0)]


def _engine(batch=4, **kw):
    from paper_2608_10362_gb300 import Engine
    t, d = SHAPES["tiny_target"], SHAPES["tiny_draft"]
    eng = Engine(t, gen_weights(t, 0), max_batch=batch, max_seq=512, max_k=4, max_drafts=1, draft_shape_max=d,
                 draft_budget_bytes=32 << 20, **kw)
    eng.register_draft(0, d, gen_weights(d, 1))
    eng.load_draft_async(0)
    eng.set_active_draft(0)
    return eng


def _start(eng, rules):
    for b, rule in enumerate(rules):
        eng.prefill(b, gen_prompt(20 + b, 30 + 7 * b, eng.vocab), seed=5 + b)
        eng.set_sampling(b, *rule)
    eng.set_batch(len(rules))


def _decision(zt, zd, x, T, u_a, u_f, n, y):
    """The oracle's decision on the cut logits, or one that a rounding explains."""
    K = len(x)
    ro = accept(zt.astype(np.float64), zd.astype(np.float64), x, T, u_a, u_f)
    if n != ro.n_accepted:
        i = min(n, ro.n_accepted)
        return abs(u_a[i] - ro.p_of_x[i] / ro.q_of_x[i]) < 1e-4
    if y != ro.token:
        w = softmax_t(zt[n], T)
        if n < K:
            w = np.maximum(w - softmax_t(zd[n], T), 0)
        c = np.cumsum(w) / w.sum()
        return abs(u_f - c[min(y, ro.token)]) < 1e-4
    return True


@pytest.mark.parametrize("graphs", [False, True])
@pytest.mark.parametrize("T", [1.0, 0.6])
def test_steps_follow_each_requests_rule(graphs, T):
    eng = _engine(use_graphs=graphs)
    plain = _engine(use_graphs=False)
    K, B = 4, 4
    accepted = 0
    for rules in (RULES[:4], RULES[2:]):
        _start(eng, rules)
        for step in range(6):
            state = eng.seq_state()
            # the same state in an engine without rules: the first draft row before the cut
            _start(plain, [(0, 1.0, 0.0)] * B)
            toks = [eng.committed_tokens(b) for b in range(B)]
            for b in range(B):
                plain.prefill(b, toks[b], seed=5 + b)
            plain.draft_step(K, T)
            assert plain.sync() == 0
            eng.draft_step(K, T)
            eng.verify_step(K)
            assert eng.sync() == 0
            whole = eng.target_logits(B, K)
            zd, x = eng.draft_logits(B, K), eng.draft_tokens(B)[:, :K]
            first = plain.draft_logits(B, K)[:, 0]
            eng.accept_commit(K, T, eng.results_host)
            assert eng.sync() == 0
            zt = eng.target_logits(B, K)
            res = eng.results_host.numpy()[:B * (K + 2)].reshape(B, K + 2)
            for b in range(B):
                for i in range(K + 1):
                    assert np.array_equal(zt[b, i], F.mask(whole[b, i], T, *rules[b])), (step, b, i)
                u_d, u_a, u_f = step_uniforms(5 + b, b, int(state[b, 2]), K)
                if step == 0:      # later the drafts' caches were filled by passes of other shapes
                    assert np.array_equal(zd[b, 0], F.mask(first[b], T, *rules[b])), (step, b)
                for j in range(K):
                    kept = np.flatnonzero(np.isfinite(zd[b, j]))
                    if rules[b][0] and rules[b][1] == 1 and rules[b][2] == 0:
                        assert len(kept) == rules[b][0]
                    want = F.draw(zd[b, j], u_d[j], T)
                    if x[b, j] != want:   # 32-bit sums: u within a rounding of the border
                        w = softmax_t(zd[b, j], T)
                        assert abs(u_d[j] - np.cumsum(w)[min(x[b, j], want)]) < 1e-5, (step, b, j)
                n, y = int(res[b, 0]), int(res[b, int(res[b, 0]) + 1])
                accepted += n
                assert _decision(zt[b], zd[b], x[b], T, u_a, u_f, n, y), (step, b)
                assert np.isfinite(zt[b, n, y])    # the emitted token was kept
    assert accepted > 0
    eng.close()
    plain.close()


def test_rules_change_between_steps_and_end_with_the_request():
    """Without a rule a step does what it did; the same engine with one does not; a prefill
    ends the rule; greedy steps never cut."""
    eng = _engine(batch=1, use_graphs=True)
    K = 3

    def stream(rule, T, reset_by_prefill=True):
        eng.prefill(0, gen_prompt(9, 40, eng.vocab), seed=11)
        if rule:
            eng.set_sampling(0, *rule)
        for _ in range(5):
            eng.step(K, T, eng.results_host)
        assert eng.sync() == 0
        return eng.committed_tokens(0).tolist(), np.isfinite(eng.target_logits(1, K)).all()

    free, whole = stream(None, 1.0)
    assert whole
    cut, whole = stream((5, 1.0, 0.0), 1.0)
    assert cut != free and not whole
    assert stream(None, 1.0) == (free, True)
    assert stream((0, 1.0, 0.0), 1.0) == (free, True)
    greedy = stream(None, 0.0)
    assert stream((5, 0.5, 0.5), 0.0) == greedy and greedy[1]
    # top-1 at any temperature is the greedy stream
    assert stream((1, 1.0, 0.0), 0.9)[0] == greedy[0]
    eng.close()


def test_tree_steps_draw_from_the_cut_rows():
    eng = _engine(batch=1, use_graphs=False)
    res = torch.zeros(66, dtype=torch.int32, pin_memory=True)
    rule, T = (30, 0.9, 0.0), 0.8
    from paper_2608_10362_gb300 import _lib
    from oracle.philox import uniform
    eng.prefill(0, gen_prompt(4, 50, eng.vocab), seed=2)
    eng.set_sampling(0, *rule)
    nodes = [3, 7, 9, 11, 13]
    parents = [-1, -1, 0, 0, 2]
    eng.tree_step(nodes, parents, T, res)
    assert eng.sync() == 0
    z = eng.read_buffer(_lib.BUF_TREE_LOGITS, np.float32, 6 * eng.vocab).reshape(6, -1)
    kept = np.isfinite(z).sum(1)
    assert np.all((kept >= 1) & (kept <= 30))
    emitted = int(res[2])
    assert np.isfinite(z[0, emitted])
    want = F.draw(z[0], uniform(2, 0, 0, 64), T)
    w = softmax_t(z[0], T)
    assert emitted == want or abs(uniform(2, 0, 0, 64) - np.cumsum(w)[min(emitted, want)]) < 1e-5
    eng.close()


def test_rules_are_refused():
    from paper_2608_10362_gb300 import MemSpecError, _lib
    eng = _engine(batch=2)
    for bad in ((2, 5, 1.0, 0.0), (-1, 5, 1.0, 0.0), (0, 0, 0.0, 0.0), (0, 0, 1.1, 0.0), (0, 0, float("nan"), 0.0),
                (0, 0, 1.0, -0.1), (0, 0, 1.0, 1.1)):
        with pytest.raises(MemSpecError) as e:
            eng.set_sampling(*bad)
        assert e.value.status == _lib.ERR_INVALID_ARG
    for bad in (-1, 2.5, 1 << 31):
        with pytest.raises(ValueError):
            eng.set_sampling(0, bad)
    eng.close()
    for kw in (dict(launch_mode="pass"), dict(draft_kernel="fused")):
        eng = _engine(batch=1, **kw)
        eng.prefill(0, gen_prompt(4, 20, eng.vocab), seed=2)
        eng.set_sampling(0, 5)
        with pytest.raises(MemSpecError) as e:
            eng.draft_step(2, 1.0)
        assert e.value.status == _lib.ERR_UNSUPPORTED
        eng.step(2, 0.0)                 # greedy: no cut needed
        eng.set_sampling(0)
        eng.step(2, 1.0)
        assert eng.sync() == 0
        eng.close()
