"""Decoding by sampling with drafting heads held in 4 bits: heads -> candidates -> tree -> verify -> acceptance -> commit, step after step,
every acceptance checked against the double-precision oracle on the logits that the step produced."""
import numpy as np
import pytest

import oracle
import workloads as wl
from oracle import mx4 as omx
from oracle import sampling as osam

pytestmark = pytest.mark.gpu

SHAPE = wl.scaled(wl.TINY, name="sampled", d_model=512, n_heads=4, d_head=128, d_ffn=1408, vocab=1500, n_layers=2, dtype="f16")
HEADS, TEMP, DRAFT_TEMP = 3, 0.9, 1.1
# node -> parent, level, rank among its parent's children (the candidates of a level in the order of their draws)
PARENT = [-1, 0, 0, 0, 1, 1, 2, 4, 4, 6, 7]


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.fixture(scope="module")
def ghd():
    import paper_2505_23219_b200 as g
    return g


def test_decode_loop(ghd):
    import torch
    n, L, steps = len(PARENT), 40, 5
    level, rank, seen = [0] * n, [0] * n, {}
    for i in range(1, n):
        level[i], rank[i] = level[PARENT[i]] + 1, seen.get(PARENT[i], 0)
        seen[PARENT[i]] = rank[i] + 1
    Lmax = L + n * (steps + 1)
    head = wl.head_weights(SHAPE, 5)
    head["lm_head"] = (head["lm_head"].astype(np.float32) * 6).astype(np.float16)        # logits a few units apart
    ctx = ghd.ghd_create(ghd.ModelCfg(SHAPE.d_model, SHAPE.n_heads, SHAPE.d_head, SHAPE.d_ffn, SHAPE.vocab, SHAPE.n_layers, Lmax, 16, "f16", SHAPE.rms_eps, SHAPE.rope_theta))
    weights = ghd.ModelWeights(dev(head["embed"]), [ghd.LayerWeights(**{k: dev(w[k]) for k in ghd.LayerWeights.FIELDS}) for w in
                               (wl.layer_weights(SHAPE, 5, l) for l in range(SHAPE.n_layers))], dev(head["rms_final"]), dev(head["lm_head"]))
    caches = [wl.kv_cache(SHAPE, 5, l, L, Lmax) for l in range(SHAPE.n_layers)]
    kvs = [ghd.KvLayer(dev(k), dev(v), ghd.KV_LEN_DEVICE) for k, v in caches]
    ghd.ghd_kv_len_set(ctx, L)
    tree = ghd.ghd_tree_build(ctx, PARENT, ghd.KV_LEN_DEVICE)
    r = np.random.RandomState(8)
    # the heads are the model's own lm_head behind a small layer, in 4 bits: drafts that are right now and then
    w1 = [ghd.ghd_mx4_quantize(ctx, dev((r.randn(512, 512) * 0.01).astype(np.float16))) for _ in range(HEADS)]
    w2 = ghd.ghd_mx4_quantize(ctx, weights.lm_head)
    codes, scales = w2.codes.cpu().numpy(), w2.scales.cpu().numpy()
    lv, rk = dev(np.array(level, np.int32)), dev(np.array(rank, np.int32))
    drow = dev(np.array([l if l < HEADS else -1 for l in level], np.int32))
    tokens = dev(wl.draft_tokens(PARENT, SHAPE.vocab, 9).astype(np.int32))
    draft = torch.zeros(HEADS, SHAPE.vocab, device="cuda")
    draft_row = None                                             # the first step's candidates were not drawn
    emitted, accepted = [], 0
    for step in range(steps):
        logits, amax = ghd.ghd_verify_step(ctx, weights, kvs, tree, tokens)
        u = torch.rand(n, device="cuda")
        more = {} if draft_row is None else dict(draft_row=draft_row, draft_logits=draft, draft_temperature=DRAFT_TEMP)
        res = ghd.ghd_accept_sampled(ctx, ghd.SampledRows(tree.parent[:n], tokens, logits, u, temperature=TEMP, **more))
        nodes, toks = osam.verify(PARENT, tokens.cpu().numpy(), logits.cpu().numpy(), u.cpu().numpy(), TEMP, None if draft_row is None else draft_row.cpu().numpy(),
                                  draft.cpu().numpy(), DRAFT_TEMP)
        got = res[0].cpu().numpy()
        assert got[0] == len(nodes) - 1 and list(got[2:2 + len(nodes)]) == nodes and list(got[258:258 + len(toks)]) == toks
        emitted += toks
        accepted += len(nodes) - 1
        before = ghd.ghd_kv_len_get(ctx)
        ghd.ghd_kv_commit(ctx, kvs, ghd.KV_LEN_DEVICE, res[0])
        assert ghd.ghd_kv_len_get(ctx) == before + len(nodes)
        # next candidates: the heads at the last accepted node
        hidden = ghd.ghd_copy_hidden(ctx, n)[nodes[-1]:nodes[-1] + 1]
        h = ghd.ghd_rmsnorm(ctx, hidden.contiguous(), weights.rms_final)
        for k in range(HEADS):
            a = ghd.ghd_mx4_linear(ctx, h, w1[k])
            y = (h.float() + a * torch.sigmoid(a)).half()
            ghd.ghd_mx4_linear(ctx, y, w2, y=draft[k:k + 1])
            want = omx.product(y.cpu().numpy(), codes, scales, SHAPE.vocab, 512)
            assert np.abs(draft[k].cpu().numpy() - want[0]).max() <= 2.0 ** -15 * np.abs(want).max()
        uc = torch.rand(HEADS, 16, device="cuda")
        cand = ghd.ghd_draft_sample(ctx, draft, uc, 3, DRAFT_TEMP)
        for k in range(HEADS):
            assert np.array_equal(cand[k].cpu().numpy(), osam.draw(draft[k].cpu().numpy(), DRAFT_TEMP, 3, uc[k].cpu().numpy()))
        full = torch.full((max(level) + 1, 16), 0, dtype=torch.int32, device="cuda")
        full[:HEADS] = cand
        tokens = ghd.ghd_tree_fill_tokens(ctx, full, res[0], lv, rk)
        draft_row = drow
        tree = ghd.ghd_tree_build(ctx, PARENT, ghd.KV_LEN_DEVICE, tree)
        assert int(tokens[0]) == toks[-1]
    ghd.ghd_sync_status(ctx)
    assert len(emitted) == accepted + steps and all(0 <= t < SHAPE.vocab for t in emitted)


def test_oracle_is_the_one_of_greedy_acceptance_when_cold(ghd):
    """Near temperature 0 the sampled acceptance of candidates that were not drawn is the greedy one."""
    import torch
    r = np.random.RandomState(12)
    V, n = 600, 30
    ctx = ghd.ghd_create(ghd.ModelCfg(512, 4, 128, 512, V, 1, 512, 32, "f16"))
    for seed in range(5):
        parent = wl.random_tree(n, 5, 40 + seed, max_children=4)
        logits = r.randn(n, V).astype(np.float32)
        amax = logits.argmax(1).astype(np.int32)
        # siblings unlike each other, half of the nodes' first children right
        tokens = np.zeros(n, np.int32)
        kids = {}
        for i in range(1, n):
            k = kids.get(parent[i], 0)
            kids[parent[i]] = k + 1
            tokens[i] = amax[parent[i]] if k == 0 and r.rand() < 0.7 else (amax[parent[i]] + 1 + k) % V
        tree = ghd.ghd_tree_build(ctx, parent, 10)
        greedy = ghd.ghd_accept(ctx, tree, dev(tokens), dev(amax)).cpu().numpy()
        cold = ghd.ghd_accept_sampled(ctx, ghd.SampledRows(tree.parent[:n], dev(tokens), dev(logits), torch.rand(n, device="cuda"), temperature=1e-4))[0].cpu().numpy()
        m = cold[0]
        assert greedy[0] >= m and list(cold[258:259 + m]) == [amax[x] for x in cold[2:3 + m]]
        want = oracle.accept(parent, tokens, amax)
        assert want[0] == greedy[0] == m


def test_decode_loop_of_the_drafting_heads(ghd):
    """Step, sampled acceptance, commit, the framework's own heads, draws from their logits, next tree.  What is allowed between the step and the heads
    (acceptance, draws, products with 4-bit matrices) leaves the heads' input alone: a second context does the step and the heads only."""
    import torch
    n, L, steps, K = len(PARENT), 40, 4, 3
    level, rank, seen = [0] * n, [0] * n, {}
    for i in range(1, n):
        level[i], rank[i] = level[PARENT[i]] + 1, seen.get(PARENT[i], 0)
        seen[PARENT[i]] = rank[i] + 1
    Lmax = L + n * (steps + 1)
    head = wl.head_weights(SHAPE, 7)
    head["lm_head"] = (head["lm_head"].astype(np.float32) * 6).astype(np.float16)
    r = np.random.RandomState(18)
    weights = ghd.ModelWeights(dev(head["embed"]), [ghd.LayerWeights(**{k: dev(w[k]) for k in ghd.LayerWeights.FIELDS}) for w in
                               (wl.layer_weights(SHAPE, 7, l) for l in range(SHAPE.n_layers))], dev(head["rms_final"]), dev(head["lm_head"]))
    heads = ghd.MedusaWeights(dev((r.randn(K, 512, 512) * 0.01).astype(np.float16)), dev(np.tile(head["lm_head"], (K, 1, 1))))
    held = ghd.ghd_mx4_quantize(ghd.ghd_create(ghd.ModelCfg(512, 4, 128, 512, 100, 1, 512, 16, "f16")), weights.lm_head)
    caches = [wl.kv_cache(SHAPE, 7, l, L, Lmax) for l in range(SHAPE.n_layers)]
    both = []
    for _ in range(2):
        ctx = ghd.ghd_create(ghd.ModelCfg(SHAPE.d_model, SHAPE.n_heads, SHAPE.d_head, SHAPE.d_ffn, SHAPE.vocab, SHAPE.n_layers, Lmax, 16, "f16", SHAPE.rms_eps, SHAPE.rope_theta))
        ghd.ghd_kv_len_set(ctx, L)
        both.append([ctx, [ghd.KvLayer(dev(k), dev(v), ghd.KV_LEN_DEVICE) for k, v in caches], ghd.ghd_tree_build(ctx, PARENT, ghd.KV_LEN_DEVICE)])
    (ctx, kvs, tree), (ctx2, kvs2, tree2) = both
    lv, rk = dev(np.array(level, np.int32)), dev(np.array(rank, np.int32))
    drow = dev(np.array([l if l < K else -1 for l in level], np.int32))
    tokens = dev(wl.draft_tokens(PARENT, SHAPE.vocab, 9).astype(np.int32))
    draft = draft_row = None
    x = torch.randn(16, 512, device="cuda").half()
    for step in range(steps):
        logits, _ = ghd.ghd_verify_step(ctx, weights, kvs, tree, tokens)
        u = torch.rand(n, device="cuda")
        more = {} if draft is None else dict(draft_row=draft_row, draft_logits=draft, draft_temperature=DRAFT_TEMP)
        res = ghd.ghd_accept_sampled(ctx, ghd.SampledRows(tree.parent[:n], tokens, logits, u, temperature=TEMP, **more))
        nodes, toks = osam.verify(PARENT, tokens.cpu().numpy(), logits.cpu().numpy(), u.cpu().numpy(), TEMP, None if draft is None else draft_row.cpu().numpy(),
                                  None if draft is None else draft.cpu().numpy(), DRAFT_TEMP)
        got = res[0].cpu().numpy()
        assert got[0] == len(nodes) - 1 and list(got[2:2 + len(nodes)]) == nodes and list(got[258:258 + len(toks)]) == toks
        ghd.ghd_mx4_linear(ctx, x, held)
        ghd.ghd_mx4_gate_up(ctx, x, held, held)
        ghd.ghd_draft_sample(ctx, logits, torch.rand(n, 16, device="cuda"), 5)
        ghd.ghd_kv_commit(ctx, kvs, ghd.KV_LEN_DEVICE, res[0])
        _, draft = ghd.ghd_medusa_draft(ctx, heads, res[0], [1] * K, want_logits=True)
        logits2, _ = ghd.ghd_verify_step(ctx2, weights, kvs2, tree2, tokens)
        _, draft2 = ghd.ghd_medusa_draft(ctx2, heads, res[0], [1] * K, want_logits=True)
        ghd.ghd_kv_commit(ctx2, kvs2, ghd.KV_LEN_DEVICE, res[0])
        assert torch.equal(logits, logits2) and torch.equal(draft, draft2)
        uc = torch.rand(K, 16, device="cuda")
        cand = ghd.ghd_draft_sample(ctx, draft, uc, 3, DRAFT_TEMP)
        for k in range(K):
            assert np.array_equal(cand[k].cpu().numpy(), osam.draw(draft[k].cpu().numpy(), DRAFT_TEMP, 3, uc[k].cpu().numpy()))
        full = torch.zeros(max(level) + 1, 16, dtype=torch.int32, device="cuda")
        full[:K] = cand
        tokens = ghd.ghd_tree_fill_tokens(ctx, full, res[0], lv, rk)
        assert int(tokens[0]) == toks[-1]
        draft_row = drow
        tree, tree2 = ghd.ghd_tree_build(ctx, PARENT, ghd.KV_LEN_DEVICE, tree), ghd.ghd_tree_build(ctx2, PARENT, ghd.KV_LEN_DEVICE, tree2)
    ghd.ghd_sync_status(ctx)
    ghd.ghd_sync_status(ctx2)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_slots_without_a_candidate(ghd, dtype):
    """A drafter with one likely token only: its further draws are -1, and so are the tree's slots that take them.  The step works them out as token 0,
    the other nodes do not see them, and no acceptance takes them."""
    import torch
    shape = wl.scaled(SHAPE, dtype=dtype)
    n, L = len(PARENT), 30
    head = wl.head_weights(shape, 9)
    T = np.float16 if dtype == "f16" else np.float32
    weights = ghd.ModelWeights(dev(head["embed"]), [ghd.LayerWeights(**{k: dev(w[k]) for k in ghd.LayerWeights.FIELDS}) for w in
                               (wl.layer_weights(shape, 9, l) for l in range(shape.n_layers))], dev(head["rms_final"]), dev(head["lm_head"]))
    ctx = ghd.ghd_create(ghd.ModelCfg(shape.d_model, shape.n_heads, shape.d_head, shape.d_ffn, shape.vocab, shape.n_layers, L + n, 16, dtype, shape.rms_eps, shape.rope_theta))
    caches = [wl.kv_cache(shape, 9, l, L, L + n) for l in range(shape.n_layers)]
    kvs = [ghd.KvLayer(dev(k.astype(T)), dev(v.astype(T)), L) for k, v in caches]
    tree = ghd.ghd_tree_build(ctx, PARENT, L)
    draft = torch.full((3, shape.vocab), -np.inf, device="cuda")
    draft[0, 40], draft[1, 41], draft[2, [42, 43]] = 1.0, 2.0, 3.0
    cand = ghd.ghd_draft_sample(ctx, draft, torch.rand(3, 16, device="cuda"), 3)
    assert (cand[:2, 1:] == -1).all() and (cand[2, 2:] == -1).all() and (cand[:, 0] >= 40).all()
    level, rank, seen = [0] * n, [0] * n, {}
    for i in range(1, n):
        level[i], rank[i] = level[PARENT[i]] + 1, seen.get(PARENT[i], 0)
        seen[PARENT[i]] = rank[i] + 1
    cand = torch.cat((cand, torch.full((max(level), 16), -1, dtype=torch.int32, device="cuda")))
    res = torch.full((514,), -1, dtype=torch.int32, device="cuda")
    res[0], res[258] = 0, 5
    tokens = ghd.ghd_tree_fill_tokens(ctx, cand, res, dev(np.array(level, np.int32)), dev(np.array(rank, np.int32)))
    none = [i for i in range(n) if int(tokens[i]) == -1]
    assert none and int(tokens[1]) == 40
    for bad in (-1, shape.vocab, 2 ** 31 - 1, -2 ** 31):
        t = tokens.clone()
        t[none] = bad
        logits, amax = ghd.ghd_verify_step(ctx, weights, kvs, tree, t)
        zero = t.clone()
        zero[none] = 0
        assert torch.equal(logits, ghd.ghd_verify_step(ctx, weights, kvs, tree, zero)[0])
        drow = dev(np.array([l if l < 3 else -1 for l in level], np.int32))
        u = torch.rand(n, device="cuda")
        got = ghd.ghd_accept_sampled(ctx, ghd.SampledRows(tree.parent[:n], t, logits, u, draft_row=drow, draft_logits=draft))[0].cpu().numpy()
        nodes, toks = osam.verify(PARENT, t.cpu().numpy(), logits.cpu().numpy(), u.cpu().numpy(), 1.0, drow.cpu().numpy(), draft.cpu().numpy(), 1.0)
        assert list(got[2:2 + len(nodes)]) == nodes and list(got[258:258 + len(toks)]) == toks and not set(nodes) & set(none)
        greedy = ghd.ghd_accept(ctx, tree, t, amax).cpu().numpy()
        assert not set(greedy[2:3 + greedy[0]]) & set(none)
    ghd.ghd_sync_status(ctx)
