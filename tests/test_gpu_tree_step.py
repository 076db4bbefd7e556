"""shard_step_tree against the fp64 oracle and the drafted-tree decoder on top of
it (shard_step_tree, head_sample, shard_tree_accept as they are used together).

A node's hidden state is, by definition, what the decode step gives for the last
token of its path from the root; the oracle runs each path as the new tokens of
one request.  The bar is the fixed one of the step (relative L2 1e-3, max-abs
2e-2 with one fp16 ulp where that is larger)."""
import dataclasses

import numpy as np
import pytest
import torch

import oracle
import paper_2608_19147_gb300 as pkg
import synth
from gpu_engine import GpuEngine, GpuShard, to_dev
from paper_2608_19147_gb300.spec import TreeDecoder, tree_depths
from scenarios import OracleEngine, f16, prefill
from test_gpu_layers import assert_fixed_bar, fp16_ulp

pytestmark = pytest.mark.gpu
SEED = 4711


def random_tree(n, g):
    return [-1] + [int(g.integers(max(0, i - 6), i)) for i in range(1, n)]


def run_tree(g, n, parents, pos, mask, hidden_in=None, token_ids=None, check=True):
    N = sum(n)
    keep = [to_dev(np.asarray(x, np.int32)) for x in (parents, pos)] + [to_dev(mask)]
    d_h = to_dev(hidden_in) if hidden_in is not None else None
    d_t = to_dev(np.asarray(token_ids, np.int32)) if token_ids is not None else None
    out = torch.empty((max(N, 1), g.shape.hidden), dtype=torch.int16, device="cuda")
    rc = pkg.shard_step_tree(g.shard.h, g.st, d_h.data_ptr() if d_h is not None else None, d_t.data_ptr() if d_t is not None else None, n,
                             keep[0].data_ptr(), keep[1].data_ptr(), keep[2].data_ptr(), mask.shape[1], out.data_ptr(), g.stream, check=check)
    if rc == 0:
        rc = pkg.shard_sync_status(g.shard.h, g.stream, check=check)
    return out.cpu().numpy().view(np.uint16) if rc == 0 else rc


@pytest.fixture(scope="module")
def tiny():
    w = synth.make_weights(synth.TINY, SEED)
    sh = GpuShard(synth.TINY, w)
    yield w, sh
    sh.close()


def path_of(parents, i):
    p = []
    while i >= 0:
        p.append(i)
        i = parents[i]
    return p[::-1]


def against_paths(shape, w, sh, n, P, holes, tokens):
    rng = np.random.default_rng(sum(n) + P[0])
    B, cap = len(n), max(P) + max(n) + 4
    g = GpuEngine(sh, B, cap)
    trees = [random_tree(k, rng) if k else [] for k in n]
    mask = np.ones((B, cap), np.uint8)
    for b in range(B):
        prefill(g, shape, SEED, b, P[b])
        mask[b, :P[b]] = rng.random(P[b]) >= holes
    N = sum(n)
    h = None if tokens else synth.hidden_in(shape, SEED, 3, N)
    ids = rng.integers(0, shape.vocab, N) if tokens else None
    pos = [P[b] + d for b in range(B) for d in tree_depths(trees[b])]
    try:
        got = run_tree(g, n, sum(trees, []), pos, mask, hidden_in=h, token_ids=ids)
        first = 0
        for b in range(B):
            assert g.length(b) == P[b] + n[b]
            done = set()
            for i in range(n[b]):
                if i in done or any(p == i for p in trees[b]):  # every node is on the path to some leaf
                    continue
                path = path_of(trees[b], i)
                o = OracleEngine(shape, w, 1, cap)
                prefill(o, shape, SEED, 0, P[b], src_row=b)
                row = np.concatenate([mask[b, :P[b]], np.ones(len(path), np.uint8)])
                at = [first + j for j in path]
                want = o.step([len(path)], np.asarray(pos)[at].astype(np.int32), row, hidden_in=None if h is None else np.ascontiguousarray(h[at]),
                              token_ids=None if ids is None else ids[at].astype(np.int32))
                assert_fixed_bar(got[at], want, "row %d leaf %d" % (b, i))
                for layer in range(shape.n_layers):
                    kg, vg = g.read(b, layer, P[b], n[b])
                    ko, vo = o.read(0, layer, P[b], len(path))
                    for a, c in ((kg[path], ko), (vg[path], vo)):
                        assert (np.abs(f16(a) - f16(c)) <= np.maximum(2e-2, fp16_ulp(f16(c)))).all()
                done.update(path)
            first += n[b]
    finally:
        g.close()


@pytest.mark.parametrize("n,P,holes,tokens", [([1], [70], 0.0, True), ([9], [0], 0.0, False), ([13, 0, 6, 1], [40, 17, 0, 130], 0.2, True),
                                              ([40, 24], [129, 200], 0.1, False)])
def test_tree_step_matches_the_oracle_along_every_path(tiny, n, P, holes, tokens):
    w, sh = tiny
    against_paths(synth.TINY, w, sh, n, P, holes, tokens)


def test_tree_step_at_8b_width():
    shape = dataclasses.replace(synth.LLAMA8B_STAGE, name="8b-2L", n_layers=2, vocab=0)
    w = synth.make_weights(shape, SEED)
    sh = GpuShard(shape, w)
    try:
        against_paths(shape, w, sh, [7, 4], [72, 300], 0.1, False)
    finally:
        sh.close()


def test_a_chain_continues_like_steps_and_prefill_after_it(tiny):
    """A chain, then a packed-step's worth of plain steps: the row goes on as if the chain had been steps."""
    w, sh = tiny
    shape = synth.TINY
    g, o = GpuEngine(sh, 1, 120), OracleEngine(shape, w, 1, 120)
    try:
        for e in (g, o):
            prefill(e, shape, SEED, 0, 33)
        n = 12
        h = synth.hidden_in(shape, SEED, 9, n)
        mask = np.ones((1, 120), np.uint8)
        got = run_tree(g, [n], list(range(-1, n - 1)), np.arange(33, 33 + n), mask, hidden_in=h)
        want = o.step([n], np.arange(33, 33 + n, dtype=np.int32), mask[0, :33 + n], hidden_in=h)
        assert_fixed_bar(got, want, "chain")
        for s in range(3):
            h1 = synth.hidden_in(shape, SEED, 20 + s, 1)
            L = 33 + n + s
            a = g.step([1], np.array([L], np.int32), mask[0, :L + 1], hidden_in=h1)
            assert_fixed_bar(a, o.step([1], np.array([L], np.int32), mask[0, :L + 1], hidden_in=h1), "step %d" % s)
    finally:
        g.close()


def test_tree_step_refusals_and_guards(tiny):
    w, sh = tiny
    shape = synth.TINY
    g = GpuEngine(sh, 2, 64)
    try:
        mask, par, pos = np.ones((2, 64), np.uint8), [-1, 0, -1], [0, 1, 0]
        h = synth.hidden_in(shape, SEED, 1, 3)
        E = pkg.SHARD_EINVAL
        assert run_tree(g, [2, 1, 0], par, pos, mask, hidden_in=h, check=False) == E
        assert run_tree(g, [0, 0], par, pos, mask, hidden_in=h, check=False) == E
        assert run_tree(g, [-1, 2], par, pos, mask, hidden_in=h, check=False) == E
        assert run_tree(g, [257, 1], par, pos, mask, hidden_in=h, check=False) == E
        assert run_tree(g, [2, 1], par, pos, mask, check=False) == E
        assert run_tree(g, [2, 1], par, pos, np.ones((2, 1), np.uint8), hidden_in=h, check=False) == E
        assert run_tree(g, [65, 1], par, pos, mask, hidden_in=h, check=False) == pkg.SHARD_ECAPACITY
        good = run_tree(g, [2, 1], par, pos, mask, hidden_in=h)
        # values on the device: reported, and the state is to be reset
        for bad in (dict(parents=[-1, 1, -1]), dict(pos=[0, shape.max_position, 0]), dict(mask=np.zeros((2, 64), np.uint8)), dict(tokens=[0, shape.vocab, 0])):
            pkg.kv_state_reset(g.st, -1)
            a = dict(parents=par, pos=pos, mask=mask)
            tokens = bad.pop("tokens", None)
            a.update(bad)
            assert run_tree(g, [2, 1], a["parents"], a["pos"], a["mask"], hidden_in=None if tokens else h, token_ids=tokens, check=False) == E
            assert "device guard" in pkg.shard_last_error()
            assert run_tree(g, [2, 1], par, pos, mask, hidden_in=h, check=False) == E  # poisoned
        pkg.kv_state_reset(g.st, -1)
        assert np.array_equal(run_tree(g, [2, 1], par, pos, mask, hidden_in=h), good)
    finally:
        g.close()


def test_tree_step_refuses_arrays_that_are_not_aligned_to_their_values(tiny):
    w, sh = tiny
    g = GpuEngine(sh, 2, 64)
    try:
        dev = [to_dev(np.asarray(x, np.int32)) for x in ([-1, 0, -1, 0], [0, 1, 0, 0])] + [to_dev(np.ones((2, 64), np.uint8))]
        dev += [to_dev(synth.hidden_in(synth.TINY, SEED, 1, 4)), torch.empty((4, synth.TINY.hidden), dtype=torch.int16, device="cuda")]
        p = [x.data_ptr() for x in dev]
        good = dict(hidden_in=p[3], token_ids=None, n_new=[2, 1], parents=p[0], position_ids=p[1], attention_mask=p[2], mask_stride=64, hidden_out=p[4])
        for over in (dict(parents=p[0] + 2), dict(position_ids=p[1] + 1), dict(hidden_in=p[3] + 1), dict(hidden_out=p[4] + 1),
                     dict(hidden_in=None, token_ids=p[0] + 2)):
            assert pkg.shard_step_tree(g.shard.h, g.st, **{**good, **over}, stream=g.stream, check=False) == pkg.SHARD_EINVAL, over
            assert "aligned" in pkg.shard_last_error()
        pkg.shard_step_tree(g.shard.h, g.st, **{**good, "hidden_in": p[3] + 2}, stream=g.stream)  # to its values is enough
        pkg.shard_sync_status(g.shard.h, g.stream)
    finally:
        g.close()


def test_a_request_does_not_see_the_others(tiny):
    w, sh = tiny
    shape = synth.TINY
    outs = []
    for other in (1, 2):
        g = GpuEngine(sh, 2, 64)
        prefill(g, shape, SEED, 0, 20)
        prefill(g, shape, SEED, 1, 20, src_row=other)
        h = np.concatenate([synth.hidden_in(shape, SEED, 1, 5), synth.hidden_in(shape, SEED, 10 + other, 5)])
        par = [-1, 0, 0, 1, 2] * 2
        pos = [20 + d for d in (0, 1, 1, 2, 2)] * 2
        outs.append(run_tree(g, [5, 5], par, pos, np.ones((2, 64), np.uint8), hidden_in=h))
        g.close()
    assert np.array_equal(outs[0][:5], outs[1][:5]) and not np.array_equal(outs[0][5:], outs[1][5:])


# ---------------------------------------------------------------------------
# the decoder
# ---------------------------------------------------------------------------

@pytest.fixture(scope="module")
def model():
    w = synth.make_weights(synth.TINY, SEED)
    s0 = dataclasses.replace(synth.TINY, name="tiny-stage0", n_layers=1)
    s1 = dataclasses.replace(synth.TINY, name="tiny-stage1", n_layers=1, vocab=0)
    stages = [GpuShard(s0, synth.ShardWeights(s0, SEED, [w.layers[0]], w.embedding)), GpuShard(s1, synth.ShardWeights(s1, SEED, [w.layers[1]], None))]
    hw = synth.make_head(synth.TINY.hidden, synth.TINY.vocab, synth.TINY.group, SEED + 1)
    head = pkg.head_create(hw.hidden, hw.vocab, hw.group, hw.rms_eps, hw.lm_head, hw.norm)
    yield [s.h for s in stages], head
    pkg.head_destroy(head)
    for s in stages:
        s.close()


def decode(model, prompts, n, trees=None, **settings):
    """n tokens or more of each request; trees(b, tokens so far, step) -> (drafts, parents)"""
    stages, head = model
    d = TreeDecoder(stages, synth.TINY.hidden, head, len(prompts), 400, **settings)
    try:
        out = [[t] for t in d.prefill(prompts)]
        step = 0
        while min(len(o) for o in out) < n:
            got = d.step(None if trees is None else [trees(b, out[b], step) for b in range(len(prompts))])
            for o, t in zip(out, got):
                o += t
            step += 1
        return out, d
    finally:
        d.close()


PROMPTS = [[3, 14, 15, 92, 65], [35], [89, 79, 32, 38, 46, 26, 43, 38, 32, 79, 50]]


def test_greedy_trees_give_the_greedy_tokens(model):
    n = 24
    plain, _ = decode(model, PROMPTS, n, temperature=0)

    def trees(b, out, step):
        g = np.random.default_rng(100 * b + step)
        truth = plain[b]
        drafts, parents = [], []
        at = 0  # the node that holds the truth so far
        for k in range(int(g.integers(0, 5))):
            want = truth[len(out) + k] if len(out) + k < len(truth) else 0
            wrong = [int(t) for t in g.integers(0, 512, 2)]
            here = wrong[:1] + [want if g.random() < 0.75 else wrong[1]] + wrong[1:]
            for t in here:
                drafts.append(t)
                parents.append(at)
            at = len(drafts) - 1
        return drafts, parents

    spec, d = decode(model, PROMPTS, n, trees, temperature=0)
    # the projections sum in another order for other numbers of tokens: a near tie may fall the other way, and the
    # texts part there; before that they are the same
    for a, b in zip(plain, spec):
        m = min(len(a), len(b))
        same = next((i for i in range(m) if a[i] != b[i]), m)
        assert same >= 12, (same, a, b)
    assert 0 < d.accepted < d.proposed


def test_sampled_decoding_is_repeatable_and_follows_its_draws(model):
    def draws(seed):
        g = np.random.default_rng(seed)
        return lambda n: g.random(n)

    a, _ = decode(model, PROMPTS, 12, temperature=0.9, top_p=0.95, draws=draws(1))
    b, _ = decode(model, PROMPTS, 12, temperature=0.9, top_p=0.95, draws=draws(1))
    c, _ = decode(model, PROMPTS, 12, temperature=0.9, top_p=0.95, draws=draws(2))
    assert a == b and a != c


def test_decoder_refuses(model):
    stages, head = model
    d = TreeDecoder(stages, synth.TINY.hidden, head, 1, 40)
    try:
        with pytest.raises(RuntimeError):
            d.step()
        with pytest.raises(ValueError):
            d.prefill([[]])
        d.prefill([[1, 2, 3]])
        for drafts, parents in (([5], [1]), ([5, 6], [0, 2]), ([5], [-1]), ([5], [])):
            with pytest.raises(ValueError):
                d.step([(drafts, parents)])
        with pytest.raises(ValueError):
            d.step([([1] * 38, list(range(38)))])
        assert len(d.step([([5, 6], [0, 0])])[0]) in (1, 2)
    finally:
        d.close()


def test_a_request_without_a_token_is_an_error_and_changes_nothing(model):
    """Draws that are no numbers: prefill and step raise, and the decoder goes on as one that never had them."""
    stages, head = model
    nan, trees = (lambda n: np.full(n, np.nan)), [([7, 8, 9], [0, 0, 1]), ([5], [0]), ((), ())]
    outs = []
    for spoil in (False, True):
        d = TreeDecoder(stages, synth.TINY.hidden, head, len(PROMPTS), 60, temperature=0.8, draws=lambda n: np.full(n, 0.4))
        try:
            good, out = d.draws, []

            def call(f, *a):
                if spoil:
                    d.draws = nan
                    with pytest.raises(RuntimeError, match="request 0, 1, 2"):
                        f(*a)
                    d.draws = good
                out.append(f(*a))

            with pytest.raises(ValueError):
                d.prefill(PROMPTS[:2] + [[1] * 61])
            call(d.prefill, PROMPTS)
            for _ in range(3):
                call(d.step, trees)
            for st in d.states:
                assert [pkg.kv_state_length(st, b) for b in range(3)] == d.length
            outs.append((out, d.length, d.position))
        finally:
            d.close()
    assert outs[0] == outs[1]


def test_draws_of_another_count_are_refused_before_anything_runs(model):
    stages, head = model
    d = TreeDecoder(stages, synth.TINY.hidden, head, 2, 40, draws=lambda n: np.full(n, 0.3))
    good = d.draws
    try:
        for f in (lambda: d.prefill([[1, 2], [3]]), lambda: d.step([([5], [0]), ((), ())])):
            for bad in (lambda n: np.zeros(n - 1), lambda n: np.zeros(n + 1), lambda n: np.zeros((1, n)), lambda n: 0.5):
                d.draws, before = bad, (list(d.length), list(d.current))
                with pytest.raises(ValueError, match="draws"):
                    f()
                assert (d.length, d.current) == before
                assert [[pkg.kv_state_length(st, b) for b in range(2)] for st in d.states] == [d.length] * 2
            d.draws = good
            f()
    finally:
        d.close()


def test_sampled_trees_emit_the_models_draws(model):
    """Sixteen requests of one text with trees of likely drafts: every emitted token is the draw of the model's distribution (the oracle's)
    after the path before it, with the random number that its node was given, and a path goes on as long as the tree has the draw.
    Logits differ from the oracle's by e at most: the head's bar (2e-3 and 1e-4 of the largest) and, for the step's 1e-3 of the hidden
    state, four times that of the logits' spread; at temperature T a sum of weights then differs by exp(2 e / T) - 1 of the whole."""
    stages, head = model
    w, hw = synth.make_weights(synth.TINY, SEED), synth.make_head(synth.TINY.hidden, synth.TINY.vocab, synth.TINY.group, SEED + 1)
    T, B, known, g = 0.1, 16, {}, np.random.default_rng(17)

    def after(tokens):
        """(weights that sum to 1, their sums by id, how far a sum may be off) after these tokens"""
        key = tuple(tokens)
        if key not in known:
            n = len(key)
            h = OracleEngine(synth.TINY, w, 1, 32).step([n], np.arange(n, dtype=np.int32), np.ones(n, np.uint8), token_ids=np.array(key, np.int32))
            lg = oracle.head_top1(h[-1:], hw.norm, hw.lm_head, hw.rms_eps)[3][0]
            x = np.exp((lg - lg.max()) / T)
            e = 2e-3 + 1e-4 * np.abs(lg).max() + 4e-3 * lg.std()
            known[key] = x / x.sum(), np.cumsum(x) / x.sum(), np.exp(2 * e / T) - 1
        return known[key]

    def is_draw(token, u, tokens):
        p, upto, off = after(tokens)
        return upto[token] - p[token] - off <= u <= upto[token] + off

    given = [np.full(B, 0.4)]
    d = TreeDecoder(stages, synth.TINY.hidden, head, B, 80, temperature=T, draws=lambda n: given[-1][:n])
    try:
        text = PROMPTS[0]
        first = d.prefill([text] * B)
        assert len(set(first)) == 1 and is_draw(first[0], 0.4, text)
        text = text + first[:1]
        p, upto, _ = after(text)
        kids = [int(t) for t in np.argsort(-p)[:3]]
        drafts, parents = list(kids), [0] * 3
        for k, t in enumerate(kids):
            for c in np.argsort(-after(text + [t])[0])[:3]:
                drafts.append(int(c))
                parents.append(1 + k)
        n = 1 + len(drafts)
        u = g.random((B, n))
        for b in range(3):  # the middle of a draft's share, further from its ends than sums are off: surely that draft
            u[b, 0] = upto[kids[b]] - p[kids[b]] / 2
        given.append(u.reshape(-1))
        out = d.step([(drafts, parents)] * B)
        lengths = set()
        for b in range(B):
            node, path = 0, []
            for k, token in enumerate(out[b]):
                assert is_draw(token, np.float32(u[b, node]), text + path), (b, k)
                path.append(token)
                node = next((1 + i for i in range(len(drafts)) if parents[i] == node and drafts[i] == token), None)
                assert (node is None) == (k + 1 == len(out[b])), (b, k)
            lengths.add(len(out[b]))
        for b in range(3):
            assert p[kids[b]] / 2 <= after(text)[2] or out[b][0] == kids[b]
        assert len(lengths) > 1 and any(p[t] / 2 > after(text)[2] for t in kids)
        given.append(g.random(B))
        for b, token in enumerate(d.step()):
            assert is_draw(token[0], np.float32(given[-1][b]), text + out[b]), b
    finally:
        d.close()
