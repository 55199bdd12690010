"""Drafting and verifying by sampling on the GPU against the double-precision oracle (oracle/sampling.py)."""
import math

import numpy as np
import pytest

from oracle import sampling as osam

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ghd():
    import paper_2505_23219_b200 as g
    return g


_CTX = {}


def ctx_for(ghd, vocab):
    if vocab not in _CTX:
        _CTX[vocab] = ghd.ghd_create(ghd.ModelCfg(512, 4, 128, 512, vocab, 1, 512, 16, "f16"))
    return _CTX[vocab]


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def logits_of(r, rows, vocab, strong=3.0):
    x = r.randn(rows, vocab) * 1.5
    k = max(1, min(20, vocab // 4))
    for i in range(rows):
        x[i, r.choice(vocab, k, replace=False)] += strong + 6 * r.rand(k)
    return x.astype(np.float32)


# ------------------------------------------------------------------ candidates
@pytest.mark.parametrize("vocab", [1, 2, 31, 32, 33, 100, 1000, 4097, 32000, 100003])
@pytest.mark.parametrize("rows", [1, 5, 40, 200])
def test_draw(ghd, vocab, rows):
    if rows * vocab > 4e6:
        rows = max(1, 4000000 // vocab)
    r = np.random.RandomState(vocab + rows)
    logits, u = logits_of(r, rows, vocab), r.rand(rows, 16).astype(np.float32)
    draws, temp = 1 + (vocab + rows) % 16, [0.5, 0.8, 1.0, 1.7][rows % 4]
    got = ghd.ghd_draft_sample(ctx_for(ghd, vocab), dev(logits), dev(u), draws, temp).cpu().numpy()
    ghd.ghd_sync_status(ctx_for(ghd, vocab))
    for i in range(rows):
        assert np.array_equal(got[i], osam.draw(logits[i], temp, draws, u[i])), i


def test_draw_from_many_rows(ghd):
    r = np.random.RandomState(6)
    for rows, vocab in ((700, 300), (450, 2050)):
        logits, u = logits_of(r, rows, vocab), r.rand(rows, 16).astype(np.float32)
        got = ghd.ghd_draft_sample(ctx_for(ghd, vocab), dev(logits), dev(u), 5, 0.9).cpu().numpy()
        for i in range(rows):
            assert np.array_equal(got[i], osam.draw(logits[i], 0.9, 5, u[i])), i


def test_draw_at_the_ends(ghd):
    """Numbers at and outside the ends of [0, 1), masked tokens, rows that run out of tokens, extreme logits."""
    V = 300
    r = np.random.RandomState(1)
    ctx = ctx_for(ghd, V)
    logits = logits_of(r, 10, V)
    logits[1, :] = -np.inf
    logits[1, [5, 250, 299]] = [0.0, 1.0, -2.0]                   # three tokens for sixteen draws
    logits[2, :] = -np.inf
    logits[2, 299] = -3e38
    logits[3, :] = 3e38
    logits[4, :] = 0.0
    logits[4, 17] = 1e30                                          # one token has it all, the others round to nothing
    logits[5, :] = np.where(np.arange(V) % 2, -np.inf, 1.0)
    logits[6, :] = 0.0                                            # equal tokens
    u = r.rand(10, 16).astype(np.float32)
    u[0, :6] = [0.0, 1.0, -1.0, 2.0, np.nan, np.nextafter(np.float32(1), np.float32(0))]
    u[5, ::2], u[5, 1::2] = 0.0, 1.0
    got = ghd.ghd_draft_sample(ctx, dev(logits), dev(u), 16, 1.0).cpu().numpy()
    ghd.ghd_sync_status(ctx)
    for i in range(10):
        assert np.array_equal(got[i], osam.draw(logits[i], 1.0, 16, u[i])), i
    assert sorted(got[1, :3]) == [5, 250, 299] and (got[1, 3:] == -1).all() and (got[4, 1:] == -1).all()


@pytest.mark.parametrize("bad", ["nan", "inf", "none"])
def test_draw_from_what_is_no_distribution(ghd, bad):
    V = 5000
    ctx = ctx_for(ghd, V)
    r = np.random.RandomState(3)
    logits, u = logits_of(r, 4, V), r.rand(4, 16).astype(np.float32)
    if bad == "nan":
        logits[2, 4321] = np.nan
    elif bad == "inf":
        logits[2, 77] = np.inf
    else:
        logits[2] = -np.inf
    got = ghd.ghd_draft_sample(ctx, dev(logits), dev(u), 5, 1.0).cpu().numpy()
    with pytest.raises(ghd.GhdError, match="distribution"):
        ghd.ghd_sync_status(ctx)
    ghd.ghd_sync_status(ctx)                                      # reported once
    assert (got[2] == -1).all()
    for i in (0, 1, 3):
        assert np.array_equal(got[i], osam.draw(logits[i], 1.0, 5, u[i]))


# ------------------------------------------------------------------ verification
def random_parents(r, n, wide):
    return [-1] + [int(r.randint(max(0, (i - 1) // wide), max(1, (i + 1) // 2))) for i in range(1, n)]


class Batch:
    """Trees of several sequences; nodes of one depth share draws from their level's draft row."""

    def __init__(self, r, cnt, vocab, temp, drawn, noise=0.7, share=1.0, wide=4):
        self.cnt, self.vocab, self.temp, self.drawn = cnt, vocab, temp, drawn
        parent, tokens, drow, logits, draft = [], [], [], [], []
        for n in cnt:
            p = random_parents(r, n, wide) if n else []
            depth = [0] * n
            for i in range(1, n):
                depth[i] = depth[p[i]] + 1
            deep = max(depth) if n else 0
            base = len(draft)
            rows = logits_of(r, deep + 1, vocab, 5.0)
            draft.extend(rows)
            kids = np.bincount([x for x in p if x >= 0], minlength=1).max() if n > 1 else 1
            cand = []
            for d in range(deep + 1):
                w = osam.distribution(rows[d], temp).copy()
                if drawn:
                    c = [int(x) for x in r.choice(vocab, min(kids, int((w > 0).sum())), replace=False, p=w)]
                else:
                    c = [int(x) for x in np.argsort(-rows[d], kind="stable")[:kids]]
                cand.append(c + [-1] * (kids - len(c)))
            seen = {}
            for i in range(n):
                parent.append(p[i])
                rank = seen.get(p[i], 0)
                seen[p[i]] = rank + 1
                tokens.append(cand[depth[i] - 1][rank] if i else 7 % vocab)
                drow.append(base + depth[i])
                logits.append(share * rows[depth[i]] + noise * r.randn(vocab))
        self.start = np.concatenate(([0], np.cumsum(cnt))).astype(np.int32)
        self.n = int(self.start[-1])
        self.parent, self.tokens, self.drow = np.array(parent, np.int32), np.array(tokens, np.int32), np.array(drow, np.int32)
        self.logits = np.array(logits, np.float32).reshape(self.n, vocab)
        self.draft = np.array(draft, np.float32).reshape(-1, vocab)
        self.u = r.rand(self.n).astype(np.float32)

    def rows(self, ghd, **kw):
        more = dict(draft_row=dev(self.drow), draft_logits=dev(self.draft), draft_temperature=self.temp) if self.drawn else {}
        args = dict(row_start=dev(self.start), temperature=self.temp, **more)
        args.update(kw)
        return ghd.SampledRows(dev(self.parent), dev(self.tokens), dev(self.logits), dev(self.u), **args)

    def check(self, got, only=None):
        longest = 0
        for s, n in enumerate(self.cnt):
            a, b = self.start[s], self.start[s] + n
            nodes, toks = osam.verify(self.parent[a:b], self.tokens[a:b], self.logits[a:b], self.u[a:b], self.temp,
                                      self.drow[a:b] if self.drawn else None, self.draft, self.temp)
            want = np.full(514, -1, np.int32)
            want[0], want[1] = max(0, len(nodes) - 1), len(nodes)
            want[2:2 + len(nodes)], want[258:258 + len(toks)] = nodes, toks
            assert np.array_equal(got[s], want), (s, got[s][:8], want[:8], got[s][258:264], want[258:264])
            longest = max(longest, len(nodes) - 1)
        return longest


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("cnt,vocab", [([1], 50), ([2], 1), ([7], 33), ([64], 32000), ([256], 1000), ([5, 0, 1, 30], 100), ([20] * 20, 997), ([3] * 200, 64),
                                       ([40, 17, 64, 9], 4099), ([12, 12], 70001), ([20] * 40, 33000)])
@pytest.mark.parametrize("temp", [0.6, 1.0])
def test_verify(ghd, drawn, cnt, vocab, temp):
    r = np.random.RandomState(len(cnt) * 100 + cnt[0] + vocab + 3 * drawn)
    b = Batch(r, cnt, vocab, temp, drawn)
    ctx = ctx_for(ghd, vocab)
    rows = b.rows(ghd)
    got = ghd.ghd_accept_sampled(ctx, rows)
    again = ghd.ghd_accept_sampled(ctx, rows)
    ghd.ghd_sync_status(ctx)
    b.check(got.cpu().numpy())
    assert (got == again).all()


@pytest.mark.parametrize("noise,share", [(0.0, 1.0), (0.05, 1.0), (2.0, 0.5), (1.0, 0.0)])
def test_verify_of_near_and_far_drafters(ghd, noise, share):
    """A draft distribution that is the target's (all accepted), nearly (differences cancel), or has nothing to do with it."""
    r = np.random.RandomState(int(noise * 100) + 7)
    b = Batch(r, [30] * 24, 2000, 1.0, True, noise=noise, share=share)
    ctx = ctx_for(ghd, 2000)
    longest = b.check(ghd.ghd_accept_sampled(ctx, b.rows(ghd)).cpu().numpy())
    assert longest >= 3 if share == 1.0 else longest >= 0
    ghd.ghd_sync_status(ctx)


def test_verify_of_wide_nodes_and_repeated_tokens(ghd):
    """Every node hangs on the root; siblings repeat, lie outside the vocabulary, or have no probability in either distribution."""
    V = 400
    ctx = ctx_for(ghd, V)
    r = np.random.RandomState(11)
    for drawn in (True, False):
        b = Batch(r, [200, 200, 200, 200], V, 1.0, drawn)
        b.parent[:] = np.tile([-1] + [0] * 199, 4)
        b.tokens[:] = r.randint(0, V, 800)
        b.tokens[r.choice(800, 60, replace=False)] = [-1, V, 2**31 - 1] * 20
        b.logits[:, r.choice(V, 150, replace=False)] = -np.inf
        b.draft[:, r.choice(V, 150, replace=False)] = -np.inf
        b.u[:] = np.where(r.rand(800) < 0.7, 0.999, b.u)
        b.u[[0, 200]] = [0.0, 1.0]
        b.check(ghd.ghd_accept_sampled(ctx, b.rows(ghd)).cpu().numpy())
        ghd.ghd_sync_status(ctx)


@pytest.mark.parametrize("cnt,vocab", [([64], 100), ([256, 0, 1], 250), ([9] * 60, 300), ([30] * 7, 513)])
def test_verify_row_by_row(ghd, cnt, vocab):
    """Where there are too many rows to weigh them all ahead of the walk (draft rows that nobody uses make them many here)."""
    import torch
    r = np.random.RandomState(vocab)
    for drawn in (True, False):
        b = Batch(r, cnt, vocab, 0.8, True)
        if not drawn:
            b.drow[:] = -1
        rest = torch.zeros(49152, vocab, device="cuda")
        got = ghd.ghd_accept_sampled(ctx_for(ghd, vocab), b.rows(ghd, draft_logits=torch.cat((dev(b.draft), rest))))
        ghd.ghd_sync_status(ctx_for(ghd, vocab))
        b.check(got.cpu().numpy())
        assert (got == ghd.ghd_accept_sampled(ctx_for(ghd, vocab), b.rows(ghd))).all()


def test_verify_of_many_rows(ghd):
    r = np.random.RandomState(31)
    V = 6000
    for drawn in (True, False):
        b = Batch(r, [150] * 14 + [3], V, 1.0, drawn)
        b.check(ghd.ghd_accept_sampled(ctx_for(ghd, V), b.rows(ghd)).cpu().numpy())
    ghd.ghd_sync_status(ctx_for(ghd, V))


def test_largest_vocabulary(ghd):
    import torch
    r = np.random.RandomState(32)
    V = 1 << 20
    ctx = ghd.ghd_create(ghd.ModelCfg(512, 4, 128, 512, V, 1, 512, 1, "f16"))
    b = Batch(r, [4], V, 1.0, True)
    b.check(ghd.ghd_accept_sampled(ctx, b.rows(ghd)).cpu().numpy())
    u = r.rand(2, 16).astype(np.float32)
    got = ghd.ghd_draft_sample(ctx, dev(b.logits[:2]), dev(u), 3).cpu().numpy()
    for i in range(2):
        assert np.array_equal(got[i], osam.draw(b.logits[i], 1.0, 3, u[i]))
    ghd.ghd_sync_status(ctx)
    big = ghd.ghd_create(ghd.ModelCfg(512, 4, 128, 512, V + 1, 1, 512, 1, "f16"))
    with pytest.raises(ghd.GhdError, match="GHD_ESHAPE"):
        ghd.ghd_draft_sample(big, torch.zeros(1, V + 1, device="cuda"), torch.zeros(1, 16, device="cuda"), 1)


def test_extreme_temperatures_and_logits(ghd):
    """Cold: the largest token; hot: all alike; logits near the ends of their type."""
    V = 700
    ctx = ctx_for(ghd, V)
    r = np.random.RandomState(33)
    logits, u = logits_of(r, 6, V), r.rand(6, 16).astype(np.float32)
    logits[4] = np.where(r.rand(V) < 0.5, 3.4e38, -3.4e38)
    logits[5] = r.randn(V) * 1e-40
    for temp in (1e-30, 1e-3, 1e10, 2.0 ** 64):
        got = ghd.ghd_draft_sample(ctx, dev(logits), dev(u), 1, temp).cpu().numpy()
        ghd.ghd_sync_status(ctx)
        for i in range(6):
            if temp == 1e-30 and i < 4:
                assert got[i, 0] == logits[i].argmax()
            elif i == 4 and temp < 1e30:
                assert logits[4, got[4, 0]] > 0
            else:
                assert got[i, 0] == osam.draw(logits[i], temp, 1, u[i])[0]


def test_streams_and_graphs(ghd):
    """A context on its own stream, results asked for on another; calls recorded once and replayed with other inputs."""
    import torch
    V = 2000
    r = np.random.RandomState(34)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = ghd.ghd_create(ghd.ModelCfg(512, 4, 128, 512, V, 1, 512, 16, "f16"))
    b, b2 = Batch(r, [40] * 3, V, 1.0, True), Batch(r, [40] * 3, V, 1.0, True)
    rows = b.rows(ghd)
    torch.cuda.synchronize()
    got = ghd.ghd_accept_sampled(ctx, rows)                    # (from the default stream)
    side.synchronize()
    b.check(got.cpu().numpy())
    u = torch.rand(3, 16, device="cuda")
    lg = dev(b.logits[:3])
    torch.cuda.synchronize()
    cand, out = torch.empty(3, 16, dtype=torch.int32, device="cuda"), torch.empty(3, 514, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ghd.ghd_accept_sampled(ctx, rows, out=out)
        ghd.ghd_draft_sample(ctx, lg, u, 5, cand=cand)
    for t, a in zip(rows.tensors, (b2.parent, b2.tokens, b2.logits, b2.u, b2.start, b2.drow, None)):
        if a is not None:
            t.copy_(dev(a))
    if rows.tensors[6].shape[0] == b2.draft.shape[0]:
        rows.tensors[6].copy_(dev(b2.draft))
    else:
        b2.draft = rows.tensors[6].cpu().numpy()
        b2.drow = np.minimum(b2.drow, len(b2.draft) - 1)
        rows.tensors[5].copy_(dev(b2.drow))
    lg.copy_(dev(b2.logits[:3]))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        g.replay()
    side.synchronize()
    b2.check(out.cpu().numpy())
    for i in range(3):
        assert np.array_equal(cand[i].cpu().numpy(), osam.draw(b2.logits[i], 1.0, 5, u[i].cpu().numpy()))
    ghd.ghd_sync_status(ctx)


def test_verify_mixes_drawn_and_other_children(ghd):
    V = 600
    ctx = ctx_for(ghd, V)
    r = np.random.RandomState(12)
    b = Batch(r, [50] * 10, V, 0.9, True)
    b.drow[r.choice(500, 200, replace=False)] = -1
    b.check(ghd.ghd_accept_sampled(ctx, b.rows(ghd)).cpu().numpy())
    one = ghd.SampledRows(*(dev(x[:50]) for x in (b.parent, b.tokens, b.logits, b.u)), temperature=0.9, draft_row=dev(b.drow[:50]), draft_logits=dev(b.draft), draft_temperature=0.9)
    assert (ghd.ghd_accept_sampled(ctx, one)[0] == ghd.ghd_accept_sampled(ctx, b.rows(ghd))[0]).all()


def test_temperatures_of_target_and_drafter(ghd):
    V = 800
    ctx = ctx_for(ghd, V)
    r = np.random.RandomState(13)
    b = Batch(r, [40] * 8, V, 1.0, True)
    got = ghd.ghd_accept_sampled(ctx, b.rows(ghd, temperature=0.7, draft_temperature=1.4)).cpu().numpy()
    for s in range(8):
        a, e = b.start[s], b.start[s + 1]
        nodes, toks = osam.verify(b.parent[a:e], b.tokens[a:e], b.logits[a:e], b.u[a:e], 0.7, b.drow[a:e], b.draft, 1.4)
        assert list(got[s, 2:2 + len(nodes)]) == nodes and list(got[s, 258:258 + len(toks)]) == toks


def test_bad_rows_are_recorded(ghd):
    V = 500
    ctx = ctx_for(ghd, V)
    r = np.random.RandomState(14)
    for what, status in [("start", "GHD_ETREE"), ("many", "GHD_ETREE"), ("parent", "GHD_ETREE"), ("draft", "GHD_EINVAL"), ("target nan", "distribution"), ("draft nan", "distribution")]:
        b = Batch(r, [20, 20, 20], V, 1.0, True)
        start = b.start.copy()
        if what == "start":
            start[1], start[2] = 40, 20                            # sequence 1 runs backwards, 0 and 2 have 40 rows
        if what == "many":
            b = Batch(r, [20, 250, 20], V, 1.0, True)
            start = np.array([0, 0, 270, 290], np.int32)
        if what == "parent":
            b.parent[25], b.parent[40] = 9, 3                      # a child before its parent; a root with one
        if what == "draft":
            b.drow[20] = len(b.draft)
        if what == "target nan":
            b.logits[20, 3] = np.nan
        if what == "draft nan":
            b.draft[b.drow[20], 3] = np.inf
        got = ghd.ghd_accept_sampled(ctx, b.rows(ghd, row_start=dev(start))).cpu().numpy()
        with pytest.raises(ghd.GhdError, match=status):
            ghd.ghd_sync_status(ctx)
        ghd.ghd_sync_status(ctx)
        if what == "start":
            assert got[1, 1] == 0 and (got[1, 2:] == -1).all()
            continue
        if what == "many":
            assert list(got[:2, 1]) == [0, 0]
            a, e = 270, 290
            nodes, toks = osam.verify(b.parent[a:e], b.tokens[a:e], b.logits[a:e], b.u[a:e], 1.0, b.drow[a:e], b.draft, 1.0)
            assert list(got[2, 2:2 + len(nodes)]) == nodes and list(got[2, 258:258 + len(toks)]) == toks
            continue
        if what == "parent":
            b.parent[25] = -1                                      # (passed over: nobody's child)
        b.check(got)


@pytest.mark.parametrize("vocab", [400, 402])
def test_rows_off_the_16_byte_boundaries(ghd, vocab):
    """Logits anywhere in a buffer, in both ways through the calls."""
    import torch
    r = np.random.RandomState(41)
    ctx = ctx_for(ghd, vocab)
    b = Batch(r, [30] * 3, vocab, 1.0, True)
    lazy = np.concatenate((b.draft, np.zeros((49152 // (vocab // 256 + 1) + 1, vocab), np.float32)))
    for off in (1, 2, 3):
        def at(x):
            t = torch.zeros(x.size + off, device="cuda")
            t[off:] = dev(x.reshape(-1))
            return t[off:].view(x.shape)
        for draft in (b.draft, lazy):
            rows = ghd.SampledRows(dev(b.parent), dev(b.tokens), at(b.logits), at(b.u), row_start=dev(b.start), draft_row=dev(b.drow), draft_logits=at(draft))
            b.check(ghd.ghd_accept_sampled(ctx, rows).cpu().numpy())
        u = r.rand(5, 16).astype(np.float32)
        got = ghd.ghd_draft_sample(ctx, at(b.logits[:5]), at(u), 7).cpu().numpy()
        for i in range(5):
            assert np.array_equal(got[i], osam.draw(b.logits[i], 1.0, 7, u[i]))
    ghd.ghd_sync_status(ctx)


def test_draft_rows_of_leaves_are_not_looked_at(ghd):
    V = 300
    ctx = ctx_for(ghd, V)
    b = Batch(np.random.RandomState(42), [30] * 6, V, 1.0, True)
    for s in range(6):
        for i in range(30):
            if i not in b.parent[30 * s:30 * s + 30]:
                b.drow[30 * s + i] = 10 ** 9
    got = ghd.ghd_accept_sampled(ctx, b.rows(ghd)).cpu().numpy()
    ghd.ghd_sync_status(ctx)
    b.drow[b.drow == 10 ** 9] = -1
    b.check(got)


def test_first_call_of_a_context_is_recorded(ghd):
    import torch
    V = 900
    r = np.random.RandomState(43)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = ghd.ghd_create(ghd.ModelCfg(512, 4, 128, 512, V, 1, 512, 16, "f16"))
    b = Batch(r, [40] * 3, V, 1.0, True)
    rows = b.rows(ghd)
    out = torch.empty(3, 514, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ghd.ghd_accept_sampled(ctx, rows, out=out)
    with torch.cuda.stream(side):
        g.replay()
    side.synchronize()
    b.check(out.cpu().numpy())


def test_nothing_to_do(ghd):
    import torch
    V = 100
    ctx = ctx_for(ghd, V)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    none = torch.empty(0, V, device="cuda")
    for start in (None, i32(0, 0, 0)):
        rows = ghd.SampledRows(i32(), i32(), none, torch.empty(0, device="cuda"), row_start=start)
        got = ghd.ghd_accept_sampled(ctx, rows).cpu().numpy()
        assert (got[:, :2] == 0).all() and (got[:, 2:] == -1).all()
    ghd.ghd_sync_status(ctx)


def test_refusals(ghd):
    import torch
    V = 100
    ctx = ctx_for(ghd, V)
    r = np.random.RandomState(15)
    b = Batch(r, [5, 5], V, 1.0, True)
    lg, u = dev(b.logits), torch.rand(10, 16, device="cuda")
    for temp in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(ghd.GhdError, match="temperature"):
            ghd.ghd_draft_sample(ctx, lg, u, 3, temp)
        with pytest.raises(ghd.GhdError, match="temperature"):
            ghd.ghd_accept_sampled(ctx, b.rows(ghd, temperature=temp))
        with pytest.raises(ghd.GhdError, match="temperature"):
            ghd.ghd_accept_sampled(ctx, b.rows(ghd, draft_temperature=temp))
    for draws in (0, 17, -1):
        with pytest.raises(ghd.GhdError, match="n_draws"):
            ghd.ghd_draft_sample(ctx, lg, u, draws)
    with pytest.raises(ghd.GhdError, match="logits"):
        ghd.ghd_draft_sample(ctx, lg[:, :99], u, 3)
    with pytest.raises(ghd.GhdError, match="uniforms"):
        ghd.ghd_draft_sample(ctx, lg, u[:9], 3)
    with pytest.raises(ghd.GhdError, match="both"):
        b.rows(ghd, draft_logits=None)
    with pytest.raises(ghd.GhdError, match="logits a row"):
        ghd.ghd_accept_sampled(ctx_for(ghd, 50), b.rows(ghd))
    with pytest.raises(ghd.GhdError, match="n_seqs"):
        ghd.ghd_accept_sampled(ctx, b.rows(ghd, row_start=torch.zeros(1026, dtype=torch.int32, device="cuda")))
    with pytest.raises(ghd.GhdError, match="out"):
        ghd.ghd_accept_sampled(ctx, b.rows(ghd), out=torch.zeros(1, 514, dtype=torch.int32, device="cuda"))
    big = Batch(r, [1], V, 1.0, False)
    n = 257
    rows = ghd.SampledRows(torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, V, device="cuda"), torch.zeros(n, device="cuda"))
    with pytest.raises(ghd.GhdError, match="256"):
        ghd.ghd_accept_sampled(ctx, rows)
    assert (ghd.ghd_draft_sample(ctx, lg[:0], u[:0], 3).shape == (0, 16))
    ghd.ghd_sync_status(ctx)
    assert big.n == 1


# ------------------------------------------------------------------ cold drafters
# (lead of the likeliest draft token over the others in logits, draft temperature): from a lead that rounding does not see to one in
# front of which the rest is nothing in 64 bits (40 at 0.05: 800 nats; the others stay clear of the 693 that the calls hold and the 745 that the
# oracle's exponential holds)
COLD = [(3, 0.05), (3, 0.5), (8, 0.2), (10, 0.2), (10, 0.25), (16, 0.4), (20, 0.5), (20, 0.1), (30, 0.05), (40, 0.4), (40, 0.05)]


def cold_batch(r, seqs, kids, vocab, lead, temp_q):
    """seqs trees of a root with `kids` children drawn from a draft row with one token far ahead, which the target mostly rejects."""
    b = Batch(r, [1 + kids] * seqs, vocab, 1.0, False)
    n = 1 + kids
    b.parent = np.tile(np.array([-1] + [0] * kids, np.int32), seqs)
    b.logits = (r.randn(b.n, vocab) * 1.2).astype(np.float32)
    b.draft = (r.uniform(-0.5, 0.5, (seqs, vocab))).astype(np.float32)
    top = r.randint(0, vocab, seqs)
    b.draft[np.arange(seqs), top] += np.float32(lead)
    b.logits[np.arange(seqs) * n, top] -= np.float32(4)
    b.drow = np.repeat(np.arange(seqs), n).astype(np.int32)
    for s in range(seqs):
        b.tokens[n * s + 1:n * (s + 1)] = osam.draw(b.draft[s], temp_q, kids, r.rand(kids).astype(np.float32))[:kids]
    # the first child is rejected in most of the trees, the later ones meet any number
    b.u[1::n] = np.where(r.rand(seqs) < 0.9, np.float32(0.97), b.u[1::n])
    return b


def check_cold(b, got, temp_q):
    rejected = 0
    for s, n in enumerate(b.cnt):
        a, e = b.start[s], b.start[s] + n
        nodes, toks = osam.verify(b.parent[a:e], b.tokens[a:e], b.logits[a:e], b.u[a:e], 1.0, b.drow[a:e], b.draft, temp_q)
        assert list(got[s, :2]) == [len(nodes) - 1, len(nodes)] and list(got[s, 2:2 + len(nodes)]) == nodes and list(got[s, 258:258 + len(toks)]) == toks, (s, nodes, toks)
        rejected += nodes[1:2] != [1]
    return rejected


@pytest.mark.parametrize("lead,temp_q", COLD)
@pytest.mark.parametrize("vocab,seqs,kids", [(5, 400, 2), (600, 100, 3), (4100, 12, 5), (8000, 150, 4)])
def test_verify_of_cold_drafters(ghd, lead, temp_q, vocab, seqs, kids):
    """One draft token holds nearly all of its distribution and is rejected: what is left of it decides, however little that is.
    All rows weighed ahead and row by row (unused draft rows make them many), with a node's probabilities kept and (8000) worked out again."""
    import torch
    r = np.random.RandomState(int(lead * 100 + temp_q * 1000) + vocab + kids)
    b = cold_batch(r, seqs, kids, vocab, lead, temp_q)
    ctx = ctx_for(ghd, vocab)
    more = dict(draft_row=dev(b.drow), draft_temperature=temp_q)
    got = ghd.ghd_accept_sampled(ctx, b.rows(ghd, draft_logits=dev(b.draft), **more))
    assert check_cold(b, got.cpu().numpy(), temp_q) > seqs // 2
    rest = torch.zeros(49152 * 256 // vocab + 1 if vocab > 256 else 49152, vocab, device="cuda")
    assert (got == ghd.ghd_accept_sampled(ctx, b.rows(ghd, draft_logits=torch.cat((dev(b.draft), rest)), **more))).all()
    ghd.ghd_sync_status(ctx)


@pytest.mark.parametrize("lead,temp_q", [(10, 0.25), (10, 0.2), (16, 0.4), (37, 1.0), (40, 0.05)])
def test_cold_drafters_leave_the_distribution_as_it_is(ghd, lead, temp_q):
    """Draws and their verification together: the first token is the target's over many random numbers."""
    import torch
    V, seqs, calls = 5, 1024, 40
    ctx = ctx_for(ghd, V)
    p = np.array([0.02, 0.10, 0.60, 0.20, 0.08])
    logits = torch.log(torch.tensor(np.tile(p, (3 * seqs, 1)), device="cuda")).float()
    draft = torch.tensor([[lead, 0.6, -0.5, -0.2, 0.1]], device="cuda").float().repeat(seqs, 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(lead * 10 + temp_q * 100))
    i32 = dict(dtype=torch.int32, device="cuda")
    parent = torch.tensor([-1, 0, 0] * seqs, **i32)
    start, drow = torch.arange(0, 3 * seqs + 1, 3, **i32), torch.arange(0, seqs, **i32).repeat_interleave(3)
    count = torch.zeros(V, device="cuda")
    for _ in range(calls):
        cand = ghd.ghd_draft_sample(ctx, draft, torch.rand(seqs, 16, generator=g, device="cuda"), 2, temp_q)
        tokens = torch.cat((torch.zeros(seqs, 1, **i32), cand[:, :2]), 1).reshape(-1).contiguous()
        rows = ghd.SampledRows(parent, tokens, logits, torch.rand(3 * seqs, generator=g, device="cuda"), row_start=start, draft_row=drow, draft_logits=draft, draft_temperature=temp_q)
        first = ghd.ghd_accept_sampled(ctx, rows)[:, 258]
        count += torch.bincount(first.long(), minlength=V)
    ghd.ghd_sync_status(ctx)
    n = seqs * calls
    assert (np.abs(count.cpu().numpy() / n - p) <= 5 * np.sqrt(p * (1 - p) / n)).all(), count / n


@pytest.mark.parametrize("vocab", [5, 700, 9000])
def test_candidates_that_were_not_drawn_and_hold_nearly_all(ghd, vocab):
    """Each child holds all but some 1e-7 of what is left of the target and is rejected all the same (its number is close to one): what is
    left after three of them is less than rounding leaves of 1 - their sum."""
    r = np.random.RandomState(vocab)
    ctx, seqs, kids = ctx_for(ghd, vocab), 60, 5
    b = Batch(r, [1 + kids] * seqs, vocab, 1.0, True)
    n, most = 1 + kids, np.float32(osam.U_MOST)
    b.parent = np.tile(np.array([-1] + [0] * kids, np.int32), seqs)
    b.drow[:] = -1
    for s in range(seqs):
        order = r.choice(vocab, 5, replace=False)
        b.logits[n * s] = -110.0 + r.rand(vocab)
        b.logits[n * s, order] = -16.0 * np.arange(5)
        b.tokens[n * s + 1:n * (s + 1)] = order
        b.u[n * s + 1:n * (s + 1)] = np.where(np.arange(kids) < s % 5, most, r.rand(kids))
    many = np.concatenate((b.draft, np.zeros((49152 // (vocab // 256 + 1) + 1, vocab), np.float32)))
    for draft in (b.draft, many):
        got = ghd.ghd_accept_sampled(ctx, b.rows(ghd, draft_logits=dev(draft))).cpu().numpy()
        b.check(got)
    assert {1, 2, 3, 4, 5} <= set(got[:, 3])
    ghd.ghd_sync_status(ctx)


# ------------------------------------------------------------------ the ends of what 64 bits hold
def held(logits, temp):
    """The calls' reading of logits: a token with less than 2^-1000 of the likeliest one's weight (which is 1 in these tests) is left out."""
    z = logits.astype(np.float64) / float(np.float32(temp)) / math.log(2)
    assert z.max() == 0 and not (np.abs(z + 1000) < 0.2).any()
    return np.where(z < -1000, -np.inf, logits).astype(np.float32)


def far(rows, vocab, temp, top, below):
    """Token `top` alone at the top, the others `below` (binary orders) under it."""
    z = np.array(below, np.float64) + np.zeros((rows, vocab))
    z[:, top] = 0
    return (-z * (math.log(2) * float(np.float32(temp)))).astype(np.float32)


@pytest.mark.parametrize("V,top", [(1024, 700), (9000, 8000)])
@pytest.mark.parametrize("below", [940.5, 985.5, 998.5, 999.5, 1000.5, 1010.5])
def test_tokens_at_the_end_of_64_bits(ghd, below, V, top):
    """Segments (and whole CTAs' shares) in front whose tokens are some 2^-1000 of the likeliest: the number 0 takes the first token that has
    weight, and there is one.  Draws go on into such tokens as long as they have weight."""
    import torch
    temp, seqs = 0.01, 3
    ctx = ctx_for(ghd, V)
    r = np.random.RandomState(int(below))
    logits = far(seqs, V, temp, top, below)
    logits[2, :top] = far(1, top + 1, temp, top, below - 6.25 + 0.5 * r.randint(0, 20, top + 1))[0, :top]      # some have weight, some have none
    zero = np.zeros((seqs, 16), np.float32)
    u = np.stack((zero[0], r.rand(16), r.rand(16))).astype(np.float32)
    for us in (zero, u):
        got = ghd.ghd_draft_sample(ctx, dev(logits), dev(us), 8, temp).cpu().numpy()
        for i in range(seqs):
            assert np.array_equal(got[i], osam.draw(held(logits[i], temp), temp, 8, us[i])), i
    lazy = torch.zeros(49152 * 256 // V + 1, V, device="cuda")
    one = np.full(seqs, -1, np.int32)
    for draft in (lazy[:1], lazy):
        for u0 in (0.0, 0.5):
            rows = ghd.SampledRows(dev(one), dev(one), dev(logits), dev(np.full(seqs, u0, np.float32)), row_start=dev(np.arange(seqs + 1, dtype=np.int32)), temperature=temp,
                                   draft_row=dev(one), draft_logits=draft)
            res = ghd.ghd_accept_sampled(ctx, rows).cpu().numpy()
            for i in range(seqs):
                assert res[i, 258] == osam.first_over(osam.distribution(held(logits[i], temp), temp), u0), (i, u0)
    ghd.ghd_sync_status(ctx)


@pytest.mark.parametrize("temp", [2.0 ** -149, 2.0 ** -140, 1e-38, 1e-36, 1e-30])
def test_smallest_temperatures(ghd, temp):
    """Zeros of both signs are equal and numbers below 2^-126 are what they are, whatever the temperature divides them by."""
    V = 600
    ctx = ctx_for(ghd, V)
    r = np.random.RandomState(35)
    x = np.full((5, V), -np.inf)
    x[0, :] = np.where(r.rand(V) < 0.5, 0.0, -0.0)
    x[1, :] = -1e-3
    x[1, r.choice(V, 9, replace=False)] = [0.0, -0.0, 0.0, -0.0, 0.0, -0.0, 0.0, -0.0, 0.0]
    x[2, :] = -np.abs(r.randn(V)) * 3 * temp                                 # (rounded to the numbers that there are)
    x[3, :] = r.randn(V) * 3 * temp
    x[4, [3, 300, 599]] = [0.0, temp, 2 * temp]
    logits, u = x.astype(np.float32), r.rand(5, 16).astype(np.float32)
    got = ghd.ghd_draft_sample(ctx, dev(logits), dev(u), 8, temp).cpu().numpy()
    one = np.full(5, -1, np.int32)
    rows = ghd.SampledRows(dev(one), dev(one), dev(logits), dev(u[:, 9].copy()), row_start=dev(np.arange(6, dtype=np.int32)), temperature=temp)
    res = ghd.ghd_accept_sampled(ctx, rows).cpu().numpy()
    ghd.ghd_sync_status(ctx)
    for i in range(5):
        assert np.array_equal(got[i], osam.draw(logits[i], temp, 8, u[i])), i
        assert res[i, 258] == osam.first_over(osam.distribution(logits[i], temp), u[i, 9]), i


def test_verify_at_the_smallest_temperatures(ghd):
    """Trees whose logits and temperatures are both about 1e-37, below 2^-126 in part; in both ways through the call."""
    import torch
    V, temp = 700, float(np.float32(1e-37))
    ctx = ctx_for(ghd, V)
    for drawn in (True, False):
        b = Batch(np.random.RandomState(36), [20] * 8, V, 1.0, drawn)
        b.logits, b.draft, b.temp = (b.logits * temp).astype(np.float32), (b.draft * temp).astype(np.float32), temp
        assert (np.abs(b.logits) < 2.0 ** -126).any() and (np.abs(b.logits) > 2.0 ** -126).any()
        b.check(ghd.ghd_accept_sampled(ctx, b.rows(ghd)).cpu().numpy())
        if drawn:
            many = torch.cat((dev(b.draft), torch.zeros(49152, V, device="cuda")))
            b.check(ghd.ghd_accept_sampled(ctx, b.rows(ghd, draft_logits=many)).cpu().numpy())
    ghd.ghd_sync_status(ctx)


def improbable_batch(r, seqs, kids, vocab, both):
    """Drafter and target agree but for some 1e-5: the tokens behind the first one or two (`both`) are all but impossible for the target, and are what the
    children hold.  Each is rejected, and each time all but some 1e-5 of what was left is taken away."""
    b = Batch(r, [1 + kids] * seqs, vocab, 1.0, False)
    n = 1 + kids
    b.parent = np.tile(np.array([-1] + [0] * kids, np.int32), seqs)
    b.drow = np.repeat(np.arange(seqs), n).astype(np.int32)
    b.draft = (np.full((seqs, vocab), -np.inf)).astype(np.float32)
    b.logits = np.full((b.n, vocab), -60.0, np.float32) - (3 * r.rand(b.n, vocab)).astype(np.float32)
    for s in range(seqs):
        order = r.choice(vocab, kids + 4, replace=False)
        top = order[:1 + both]
        b.draft[s, order] = -11 - 2 * r.rand(kids + 4)
        b.draft[s, top] = [0.0, 0.4][:len(top)]
        b.logits[n * s, top] = [0.0, 0.4 + r.choice([-1e-4, 1e-4])][:len(top)]
        b.tokens[n * s + 1:n * (s + 1)] = order[2:2 + kids]
        b.u[n * s + 1:n * (s + 1)] = 0.3 + 0.7 * r.rand(kids)
    return b


@pytest.mark.parametrize("both", [0, 1])
@pytest.mark.parametrize("vocab,seqs,kids", [(20, 200, 6), (700, 60, 3), (8000, 150, 5)])
def test_children_that_are_all_but_impossible(ghd, vocab, seqs, kids, both):
    """What is left of the target shrinks by 1e-5 with each rejection, and keeps its digits; there always is a last token."""
    import torch
    r = np.random.RandomState(vocab + kids + both)
    b = improbable_batch(r, seqs, kids, vocab, both)
    ctx = ctx_for(ghd, vocab)
    got = ghd.ghd_accept_sampled(ctx, b.rows(ghd, draft_row=dev(b.drow), draft_logits=dev(b.draft)))
    rest = torch.zeros(49152 * 256 // vocab + 1 if vocab > 256 else 49152, vocab, device="cuda")
    assert (got == ghd.ghd_accept_sampled(ctx, b.rows(ghd, draft_row=dev(b.drow), draft_logits=torch.cat((dev(b.draft), rest))))).all()
    ghd.ghd_sync_status(ctx)
    assert check_cold(b, got.cpu().numpy(), 1.0) == seqs
    assert (got[:, 258] >= 0).all()
