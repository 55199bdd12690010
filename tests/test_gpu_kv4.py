"""The paged 4-bit cache on the GPU against the double-precision oracle (oracle/kv4.py)."""
import numpy as np
import pytest

import workloads as wl
from oracle import kv4 as okv4

pytestmark = pytest.mark.gpu

THETA = 10000.0


@pytest.fixture(scope="module")
def ghd():
    import paper_2505_23219_b200 as g
    return g


def make_ctx(ghd, H, d, dtype, max_nodes=64):
    return ghd.ghd_create(ghd.ModelCfg(H * d, H, d, 256, 100, 1, 512, max_nodes, dtype, 1e-6, THETA))


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Setup:
    """A cache with random rows, pages in random order, every other byte of the pool random too (NaN scales among it)."""

    def __init__(self, ghd, H, Hk, d, dtype, R, lens, cnt, seed, spare=3, behind=0, garbage=True):
        r = np.random.RandomState(seed)
        self.H, self.Hk, self.d, self.dtype, self.R = H, Hk, d, dtype, R
        self.np_t = np.float16 if dtype == "f16" else np.float32
        S = len(lens)
        self.lens, self.cnt = list(lens), list(cnt)
        self.start = np.concatenate(([0], np.cumsum(cnt))).astype(np.int32)
        self.n, self.n_rows = int(self.start[-1]), int(self.start[-1]) + behind
        need = [-(-(a + b) // R) for a, b in zip(lens, cnt)]
        n_pages = sum(need) + spare
        order = r.permutation(n_pages)
        self.table = np.full((S, max(need) + 1), -7, np.int32)              # entries past a sequence's rows are not ids
        at = 0
        for s in range(S):
            self.table[s, :need[s]] = order[at:at + need[s]]
            at += need[s]
        self.pool = okv4.Pool(n_pages, Hk, R, d, dtype)
        if garbage:
            self.pool.data[:] = r.randint(0, 256, self.pool.data.shape)
        strong = np.exp(0.6 * r.randn(d))
        for s in range(S):
            for t in range(lens[s] + cnt[s]):
                page, row = okv4.slots(self.table, R, s, t)
                for h in range(Hk):
                    self.pool.put(0, page, row, h, *okv4.quantise((r.randn(d) * strong).astype(np.float32), dtype))
                    self.pool.put(1, page, row, h, *okv4.quantise((r.randn(d) * 0.6 + 0.1).astype(np.float32), dtype))
        self.r = r
        self.ctx = make_ctx(ghd, H, d, dtype)
        self.kv_len = dev(np.array(lens, np.int32))
        self.kv = ghd.Kv4Cache(dev(self.table), self.kv_len, R, Hk, n_pages)
        self.dpool = dev(self.pool.data.reshape(-1))
        assert ghd.ghd_kv4_pool_bytes(self.ctx, self.kv) == self.pool.data.size

    def trees(self, words=None):
        vis = []
        W = words or (max(max(self.cnt), 1) + 63) // 64
        mask = np.zeros((max(self.n_rows, 1), W * 64), np.uint8)
        for s, n in enumerate(self.cnt):
            v = np.eye(n, dtype=bool)
            for i in range(1, n):
                v[i] |= v[self.r.randint(max(0, i - 7), i)]
            vis.append(v)
            mask[self.start[s]:self.start[s] + n, :n] = v
        return vis, np.packbits(mask, axis=1, bitorder="little").view(np.int64).reshape(len(mask), W)


def attention_tolerance(su, q):
    """Absolute bound per output element, from the arithmetic (nothing measured).
    Scores: q . c is summed in 32 bits over d products of |q_i| and at most 8, each of up to d additions off by 2^-23 of
    the running sum (the tensor cores may truncate); scaled by scale / sqrt d; the minimum's term by 2^-22.  A score off by
    e moves a weight by a factor 1 +- 2 e, hence the output by at most 4 e max |v|.  exp2 and the 32-bit weights: 2^-20.
    Values: the weight times scale is rounded to half (2^-11, plus 2^-25 below the normal range) in f16, to 24 bits in
    f32, and meets codes of at most 8; the sums run over L keys in 32 bits.  Output: half a step of its type."""
    f16 = su.dtype == "f16"
    K, V = su.pool_values
    d, L = su.d, max(a + b for a, b in zip(su.lens, su.cnt))
    par = np.array([np.abs(x).max() for x in (K, V)])
    qsum = np.abs(q.astype(np.float64)).sum(-1).max()
    s_k, s_v, m_k = su.max_scale[0], su.max_scale[1], par[0]
    e = (d * 2.0 ** -23 * 8 * s_k * qsum + 2.0 ** -22 * 2 * m_k * qsum) / np.sqrt(d) + 2.0 ** -20
    e += 2.0 ** -23 * 16 * par[0] * qsum / np.sqrt(d) if not f16 else 0.0            # q in three terms: 2^-24 each
    w = 2.0 ** -11 if f16 else 2.0 ** -23
    a = 8 * s_v * (w + L * 2.0 ** -23) + (8 * 2.0 ** -25 * L if f16 else 0.0) + 4 * e * par[1] + L * 2.0 ** -23 * par[1]
    return lambda want: a + (2.0 ** -11 if f16 else 2.0 ** -23) * np.abs(want)


def collect(su):
    """Largest scales and all finite values of the sequences' rows, for the tolerance."""
    K, V, sc = [], [], np.zeros(2)
    for s in range(len(su.lens)):
        k, v = okv4.rows(su.pool, su.table, s, 0, su.lens[s] + su.cnt[s])
        K.append(k.reshape(-1)), V.append(v.reshape(-1))
        for t in range(su.lens[s] + su.cnt[s]):
            page, row = okv4.slots(su.table, su.R, s, t)
            for w in (0, 1):
                for h in range(su.Hk):
                    x = float(su.pool.params(w, page, row, h)[0])
                    sc[w] = max(sc[w], x) if np.isfinite(x) else sc[w]
    K, V = np.concatenate(K), np.concatenate(V)
    su.pool_values = (K[np.isfinite(K)], V[np.isfinite(V)])
    su.max_scale = sc


def run_attention(ghd, su, vis, words, want_status=True):
    import torch
    q = su.r.randn(su.n_rows, su.H, su.d).astype(su.np_t)
    rows = ghd.Kv4Rows(dev(su.start), su.n_rows, mask=None if words is None else dev(words))
    out = torch.full((su.n_rows, su.H * su.d), 7.0, dtype=su.ctx.cfg.torch_dtype, device="cuda")
    ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, dev(q.reshape(su.n_rows, -1)), out=out)
    if want_status:
        ghd.ghd_sync_status(su.ctx)
    got = out.float().cpu().numpy().astype(np.float64).reshape(su.n_rows, su.H, su.d)
    assert (got[su.n:] == 7.0).all()                                      # rows behind the last sequence
    want = okv4.attention(su.pool, su.table, su.lens, su.start, vis, q[: su.n])
    return q, got[: su.n], want


def check_attention(ghd, su, vis, words):
    collect(su)
    q, got, want = run_attention(ghd, su, vis, words)
    tol = attention_tolerance(su, q)(want)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


CASES = [
    # heads, kv heads, d, type, page rows, lengths, new rows
    (4, 4, 128, "f16", 64, [130], [1]),
    (4, 4, 128, "f16", 16, [0], [1]),
    (4, 4, 128, "f16", 32, [63, 64, 65, 0], [1, 1, 1, 1]),
    (8, 2, 128, "f16", 16, [200, 0, 17], [3, 0, 9]),
    (7, 1, 64, "f16", 128, [255, 1], [5, 2]),
    (4, 4, 64, "f16", 16, [90], [70]),
    (4, 4, 128, "f16", 128, [300, 10], [33, 64]),
    (4, 4, 128, "f16", 64, [40], [200]),
    (4, 4, 64, "f32", 32, [129, 0, 3], [7, 5, 1]),
    (6, 2, 128, "f32", 16, [50], [11]),
    (4, 1, 128, "f16", 16, [700], [1]),
]


@pytest.mark.parametrize("tree", [True, False], ids=["tree", "causal"])
@pytest.mark.parametrize("H,Hk,d,dtype,R,lens,cnt", CASES)
def test_attention_against_the_oracle(ghd, H, Hk, d, dtype, R, lens, cnt, tree):
    su = Setup(ghd, H, Hk, d, dtype, R, lens, cnt, 17 * H + R + len(lens), behind=2)
    if tree:
        vis, words = su.trees()
    else:
        vis, words = [np.ones((n, n), bool) for n in cnt], None
    check_attention(ghd, su, vis, words)


TILED = [
    (4, 4, 128, "f16", 64, [130], [1]),
    (2, 2, 128, "f16", 128, [0, 1], [17, 64]),
    (2, 2, 64, "f16", 16, [127, 0, 128, 129, 5], [63, 64, 0, 65, 1]),
    (6, 2, 128, "f16", 32, [300, 0], [21, 22]),               # 63 and 66 rows of a head: tiles that end inside a node's group
    (5, 1, 64, "f16", 128, [640, 383], [1, 30]),
    (2, 1, 128, "f16", 16, [33], [256]),
    (3, 3, 64, "f16", 64, [1100], [40]),                      # a head's keys over several blocks
    (16, 16, 128, "f16", 32, [0, 3, 90, 0, 31], [2, 1, 9, 33, 70]),
]


@pytest.mark.parametrize("path", [1, 2], ids=["rows", "tcgen05"])
@pytest.mark.parametrize("tree", [True, False], ids=["tree", "causal"])
@pytest.mark.parametrize("H,Hk,d,dtype,R,lens,cnt", TILED)
def test_both_kernels_on_tiles_of_many_rows(ghd, H, Hk, d, dtype, R, lens, cnt, tree, path):
    su = Setup(ghd, H, Hk, d, dtype, R, lens, cnt, 29 * H + R + len(lens), behind=3)
    ghd.ghd_set_option(su.ctx, 2, path)
    if tree:
        vis, words = su.trees()
    else:
        vis, words = [np.ones((n, n), bool) for n in cnt], None
    check_attention(ghd, su, vis, words)


@pytest.mark.parametrize("tree", [True, False], ids=["tree", "causal"])
@pytest.mark.parametrize("H,Hk,d,R,lens,cnt", [(4, 1, 64, 16, [100, 0], [30, 20]), (2, 2, 128, 32, [200], [90]), (3, 1, 128, 128, [129, 5, 0], [64, 1, 33]), (2, 2, 64, 64, [900], [70])])
def test_many_rows_in_float_mode(ghd, H, Hk, d, R, lens, cnt, tree):
    su = Setup(ghd, H, Hk, d, "f32", R, lens, cnt, 31 * H + R + len(lens), behind=3)
    vis, words = su.trees() if tree else ([np.ones((n, n), bool) for n in cnt], None)
    check_attention(ghd, su, vis, words)


def test_more_sequences_than_blocks(ghd):
    """1024 sequences, the most a call takes, of no, one or a few rows each."""
    r = np.random.RandomState(3)
    lens, cnt = r.randint(0, 40, 1024).tolist(), r.randint(0, 4, 1024).tolist()
    for path in (1, 2):
        su = Setup(ghd, 2, 1, 64, "f16", 16, lens, cnt, 37, behind=1)
        ghd.ghd_set_option(su.ctx, 2, path)
        check_attention(ghd, su, [np.ones((n, n), bool) for n in cnt], None)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_rows_that_see_nothing_get_zeros_and_bits_above_the_diagonal_count_for_nothing(ghd, dtype):
    su = Setup(ghd, 4, 2, 64, dtype, 16, [0, 20], [6, 6], 5)
    vis, words = su.trees()
    words[2] = 0                                                          # row 2 of the first sequence: no cache, no node
    words[4] |= 1 << 5                                                    # a later node
    words[8] = 0                                                          # second sequence: only the cache is left
    vis[0][2] = False
    vis[1][2] = False
    collect(su)
    q, got, want = run_attention(ghd, su, vis, words)
    assert (got[2] == 0).all() and (want[2] == 0).all()
    assert (np.abs(got - want) <= attention_tolerance(su, q)(want)).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_nan_and_infinity_reach_only_the_rows_that_see_them(ghd, dtype):
    """Node 1 of a tree has a NaN key row and node 2 an infinite value row; node 3 sees neither, 4 sees 1, 5 sees 2.
    A query of NaN touches its own row alone.  What lies past the sequence's rows is random bytes."""
    su = Setup(ghd, 4, 2, 128, dtype, 32, [37], [6], 9)
    vis = [np.eye(6, dtype=bool)]
    vis[0][:, 0] = True
    vis[0][4, 1] = vis[0][5, 2] = True
    mask = np.zeros((6, 64), np.uint8)
    mask[:, :6] = vis[0]
    words = np.packbits(mask, axis=1, bitorder="little").view(np.int64)
    for node, which in ((1, 0), (2, 1)):
        page, row = okv4.slots(su.table, su.R, 0, 37 + node)
        for h in range(2):
            su.pool.put(which, page, row, h, su.pool.codes(which, page, row, h), np.nan if which == 0 else np.inf, 0.5)
    su.dpool.copy_(dev(su.pool.data.reshape(-1)))
    collect(su)
    with np.errstate(all="ignore"):
        q, got, want = run_attention(ghd, su, vis, words)
    bad = np.array([False, True, True, False, True, True])
    assert np.isfinite(got[~bad]).all() and np.isnan(got[[1, 4]]).all() and (~np.isfinite(got[[2, 5]])).any(-1).all()
    tol = attention_tolerance(su, q)
    assert (np.abs(got - want)[~bad] <= tol(want)[~bad]).all()


def test_a_nan_query_stays_in_its_row(ghd):
    import torch
    su = Setup(ghd, 4, 4, 128, "f16", 64, [100], [5], 10)
    vis, words = su.trees()
    collect(su)
    q = su.r.randn(5, 4, 128).astype(np.float16)
    q[3, 1, 17] = np.nan
    out = ghd.ghd_kv4_attention(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), 5, mask=dev(words)), su.dpool, dev(q.reshape(5, -1)))
    ghd.ghd_sync_status(su.ctx)
    got = out.float().cpu().numpy().reshape(5, 4, 128)
    assert np.isnan(got[3, 1]).all()
    got[3, 1] = 0
    q[3, 1] = 0
    want = okv4.attention(su.pool, su.table, su.lens, su.start, vis, q)
    want[3, 1] = 0
    assert (np.abs(got - want) <= attention_tolerance(su, q)(want)).all()
    assert torch.isfinite(torch.from_numpy(got)).all()


def test_extreme_scales_of_values_and_scores(ghd):
    """Values near the largest half, and scores that grow along the cache (the reference has to follow)."""
    su = Setup(ghd, 2, 2, 128, "f16", 16, [150], [2], 11, garbage=False)
    for t in range(152):
        page, row = okv4.slots(su.table, 16, 0, t)
        for h in range(2):
            su.pool.put(1, page, row, h, su.pool.codes(1, page, row, h), 8000.0, -60000.0)
            x = np.full(128, 0.02 * t, np.float32)
            x[::2] += 0.5
            su.pool.put(0, page, row, h, *okv4.quantise(x, "f16"))
    su.dpool.copy_(dev(su.pool.data.reshape(-1)))
    collect(su)
    vis = [np.ones((2, 2), bool)]
    q = np.abs(su.r.randn(2, 2, 128)).astype(np.float16)
    out = ghd.ghd_kv4_attention(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), 2), su.dpool, dev(q.reshape(2, -1)))
    ghd.ghd_sync_status(su.ctx)
    got = out.double().cpu().numpy().reshape(2, 2, 128)
    want = okv4.attention(su.pool, su.table, su.lens, su.start, vis, q)
    tol = np.minimum(attention_tolerance(su, q)(want), 400.0)
    assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("H,Hk,n", [(2, 2, 1), (4, 1, 9), (2, 2, 32), (2, 2, 70)])
def test_scales_behind_the_rows_cost_no_precision(ghd, H, Hk, n):
    """The page's rows behind a sequence hold the largest scales there are.  All scores are equal, so the tolerance is that of
    the weights alone."""
    su = Setup(ghd, H, Hk, 128, "f16", 128, [0, 3], [n, n], 13, garbage=False)
    collect(su)
    for s in range(2):
        for t in range(su.lens[s] + n, -(-(su.lens[s] + n) // 128) * 128):
            page, row = okv4.slots(su.table, 128, s, t)
            for h in range(Hk):
                for which in (0, 1):
                    su.pool.put(which, page, row, h, su.pool.codes(which, page, row, h), 65504.0, -65504.0)
    su.dpool.copy_(dev(su.pool.data.reshape(-1)))
    vis, words = su.trees()
    q = np.zeros((2 * n, H, 128), np.float16)
    out = ghd.ghd_kv4_attention(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), 2 * n, mask=dev(words)), su.dpool, dev(q.reshape(2 * n, -1)))
    ghd.ghd_sync_status(su.ctx)
    got = out.double().cpu().numpy().reshape(2 * n, H, 128)
    want = okv4.attention(su.pool, su.table, su.lens, su.start, vis, q)
    assert (np.abs(got - want) <= attention_tolerance(su, q)(want)).all()


def test_the_same_call_gives_the_same_bits_and_leaves_its_scratch_clean(ghd):
    su = Setup(ghd, 4, 4, 128, "f16", 64, [1500, 10], [9, 3], 12)
    vis, words = su.trees()
    q = dev(su.r.randn(12, 4 * 128).astype(np.float16))
    rows = ghd.Kv4Rows(dev(su.start), 12, mask=dev(words))
    first = ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q).clone()
    for _ in range(20):
        assert bool((ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q) == first).all())
    ghd.ghd_sync_status(su.ctx)


@pytest.mark.parametrize("H,Hk,d,dtype,R,lens,cnt", [
    (4, 4, 128, "f16", 64, [130], [1]),
    (8, 2, 128, "f16", 16, [0, 13, 40], [20, 0, 7]),
    (4, 4, 64, "f16", 32, [31, 5], [2, 40]),
    (4, 2, 64, "f32", 16, [0, 100000 % 97], [33, 3]),
    (2, 2, 128, "f32", 128, [127], [130]),
])
@pytest.mark.parametrize("with_pos", [True, False], ids=["pos", "slots"])
def test_append_and_read_back(ghd, H, Hk, d, dtype, R, lens, cnt, with_pos):
    import torch
    su = Setup(ghd, H, Hk, d, dtype, R, lens, cnt, 23 + H + R, behind=2)
    n = su.n_rows
    pos = su.r.randint(0, 200000, n).astype(np.int32) if with_pos else None
    # q, k and v side by side in one buffer
    qkv = su.r.randn(n, (H + 2 * Hk) * d).astype(su.np_t)
    qkv[0, H * d: H * d + d] = 0.25                                          # a constant row: scale 0 after position 0, else a rotated one
    x = dev(qkv)
    q, k, v = x.split((H * d, Hk * d, Hk * d), 1)
    before = su.dpool.clone()
    q_out = torch.full((n, H * d), 9.0, dtype=x.dtype, device="cuda")
    rows = ghd.Kv4Rows(dev(su.start), n, pos=None if pos is None else dev(pos))
    ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, q, k, v, q_out=q_out)
    ghd.ghd_sync_status(su.ctx)
    a = qkv[: su.n].reshape(su.n, H + 2 * Hk, d)
    want_q = okv4.append(su.pool, su.table, su.lens, su.start, pos, a[:, :H], a[:, H:H + Hk], a[:, H + Hk:], THETA)
    got_q = q_out.double().cpu().numpy().reshape(n, H, d)
    assert (got_q[su.n:] == 9.0).all()
    # rotated in 32 bits (angle's cosine and sine rounded, two products, one sum: 2^-22 of |a| + |b|), then rounded once
    amp = np.abs(a[:, :H].astype(np.float64))
    amp = amp + np.concatenate([amp[..., d // 2:], amp[..., : d // 2]], -1)
    half = 2.0 ** -11 if dtype == "f16" else 2.0 ** -24
    assert (np.abs(got_q[: su.n] - want_q) <= half * np.abs(want_q) + 2.0 ** -22 * amp + (2.0 ** -25 if dtype == "f16" else 0)).all()
    # codes, scales and minima bit for bit, and not one other byte of the pool
    assert np.array_equal(su.dpool.cpu().numpy(), su.pool.data.reshape(-1))
    assert before.numel() == su.dpool.numel() and int(su.kv_len[0]) == lens[0]
    # read back
    kb, vb = ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, dev(su.start), n)
    ghd.ghd_sync_status(su.ctx)
    for w, got in ((0, kb), (1, vb)):
        got = got.double().cpu().numpy()[: su.n].reshape(su.n, Hk, d)
        want = np.concatenate([okv4.rows(su.pool, su.table, s, lens[s], cnt[s])[w] for s in range(len(lens))])
        # one fused 32-bit operation, then the rounding to T
        assert (np.abs(got - want) <= (half + 2.0 ** -24) * np.abs(want) + 2.0 ** -25).all()


def test_append_of_keys_and_values_alone_and_in_place_queries(ghd):
    su = Setup(ghd, 4, 4, 128, "f16", 16, [5], [9], 31)
    k, v, q = (su.r.randn(9, 4 * 128).astype(np.float16) for _ in range(3))
    rows = ghd.Kv4Rows(dev(su.start), 9)
    assert ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, None, dev(k), dev(v)) is None
    r = lambda a: a.reshape(9, 4, 128)  # noqa: E731
    want = okv4.append(su.pool, su.table, su.lens, su.start, None, r(q), r(k), r(v), THETA)
    assert np.array_equal(su.dpool.cpu().numpy(), su.pool.data.reshape(-1))
    qd = dev(q)
    other = ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, qd.clone(), dev(k), dev(v))
    ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, qd, dev(k), dev(v), q_out=qd)
    assert bool((other == qd).all())
    assert np.abs(qd.double().cpu().numpy().reshape(9, 4, 128) - want).max() <= 2.0 ** -11 * np.abs(want).max() + 2.0 ** -20 * 8
    ghd.ghd_sync_status(su.ctx)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_append_of_rows_that_are_not_finite_reads_back_as_nan(ghd, dtype):
    su = Setup(ghd, 2, 2, 64, dtype, 16, [3], [4], 33)
    k, v, q = (su.r.randn(4, 2 * 64).astype(su.np_t) for _ in range(3))
    v[0, 5], v[1, 70], v[2, 3], k[3, 9] = np.nan, np.inf, -np.inf, np.nan
    rows = ghd.Kv4Rows(dev(su.start), 4)
    ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, dev(q), dev(k), dev(v))
    kb, vb = (x.float().cpu().numpy().reshape(4, 2, 64) for x in ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, dev(su.start), 4))
    ghd.ghd_sync_status(su.ctx)
    bad_v = np.array([[1, 0], [0, 1], [1, 0], [0, 0]], bool)
    bad_k = np.array([[0, 0], [0, 0], [0, 0], [1, 0]], bool)
    assert np.isnan(vb[bad_v]).all() and np.isfinite(vb[~bad_v]).all()
    assert np.isnan(kb[bad_k]).all() and np.isfinite(kb[~bad_k]).all()


@pytest.mark.parametrize("dtype,d,R", [("f16", 128, 16), ("f16", 64, 64), ("f32", 64, 16), ("f32", 128, 32)])
def test_commit_moves_the_accepted_rows(ghd, dtype, d, R):
    import torch
    lens, cnt = [30, 0, 5, 64], [12, 9, 0, 40]
    su = Setup(ghd, 4, 2, d, dtype, R, lens, cnt, 41)
    pools = torch.stack([su.dpool, torch.from_numpy(su.r.randint(0, 256, su.dpool.numel()).astype(np.uint8)).cuda()])
    host = [okv4.Pool(su.pool.data.shape[0], 2, R, d, dtype, data=p.cpu().numpy().reshape(su.pool.data.shape)) for p in pools]
    paths = [(3, [0, 1, 4, 11]), (0, [0]), (0, [0]), (5, [0, 2, 3, 9, 20, 39])]
    res = np.zeros((4, 514), np.int32)
    for s, (m, nodes) in enumerate(paths):
        res[s, 0], res[s, 1], res[s, 2:3 + m] = m, m + 1, nodes
    rows = ghd.Kv4Rows(dev(su.start), su.n)
    ghd.ghd_kv4_commit(su.ctx, su.kv, rows, pools, dev(res))
    ghd.ghd_sync_status(su.ctx)
    new = okv4.commit(host, su.table, lens, su.start, paths)
    assert su.kv_len.cpu().tolist() == new == [34, 1, 5, 70]
    assert np.array_equal(pools.cpu().numpy(), np.stack([h.data.reshape(-1) for h in host]))
    ghd.ghd_kv4_commit(su.ctx, su.kv, ghd.Kv4Rows(dev(np.array([0, 1, 3, 3, 4], np.int32)), 4), None)     # a prompt: all rows stay
    assert su.kv_len.cpu().tolist() == [35, 3, 5, 71]
    ghd.ghd_sync_status(su.ctx)


def test_pages_behind_four_gigabytes(ghd):
    """Page ids whose byte offsets pass 32 bits (signed and unsigned)."""
    import torch
    H, d, R = 32, 128, 128
    ctx = make_ctx(ghd, H, d, "f16")
    page_bytes = H * okv4.block_bytes(R, d, "f16")
    n_pages = (1 << 32) // page_bytes + 40
    pool = torch.zeros(n_pages * page_bytes, dtype=torch.uint8, device="cuda")
    ids = [n_pages - 1, (1 << 31) // page_bytes + 1, 3]
    kv = ghd.Kv4Cache(dev(np.array([ids], np.int32)), dev(np.array([0], np.int32)), R, H, n_pages)
    small = torch.zeros(3 * page_bytes, dtype=torch.uint8, device="cuda")
    kv2 = ghd.Kv4Cache(dev(np.array([[1, 0, 2]], np.int32)), dev(np.array([0], np.int32)), R, H, 3)
    r = np.random.RandomState(3)
    n = 300
    q, k, v = (dev(r.randn(n, H * d).astype(np.float16)) for _ in range(3))
    rows = ghd.Kv4Rows(dev(np.array([0, n], np.int32)), n)
    outs = []
    for c, p in ((kv, pool), (kv2, small)):
        qr = ghd.ghd_kv4_append(ctx, c, rows, p, q, k, v)
        ghd.ghd_kv4_commit(ctx, c, rows, None)
        one = ghd.Kv4Rows(dev(np.array([0, 0], np.int32)), 0)
        assert one.n_rows == 0
        c.kv_len.sub_(5)
        last = ghd.Kv4Rows(dev(np.array([0, 5], np.int32)), 5)
        outs.append([ghd.ghd_kv4_attention(ctx, c, last, p, qr[-5:].contiguous()), *ghd.ghd_kv4_read(ctx, c, p, dev(np.array([0, n], np.int32)), n, first=dev(np.array([0], np.int32)))])
    ghd.ghd_sync_status(ctx)
    for a, b in zip(*outs):
        assert bool((a == b).all()) and float(a.abs().max()) > 0


def test_bad_pages_and_rows_are_skipped_and_reported(ghd):
    import torch
    su = Setup(ghd, 4, 4, 64, "f16", 16, [40, 20], [2, 2], 51, garbage=False)
    rows = ghd.Kv4Rows(dev(su.start), 4)
    q = dev(su.r.randn(4, 256).astype(np.float16))
    k = dev(su.r.randn(4, 256).astype(np.float16))
    good = ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q).clone()
    ghd.ghd_sync_status(su.ctx)
    for bad in (-1, su.kv.c.n_pages, 2**31 - 1):
        su.kv.page_table[0, 1] = bad
        out = ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q)
        with pytest.raises(ghd.GhdError) as e:
            ghd.ghd_sync_status(su.ctx)
        assert e.value.name == "GHD_EINVAL" and "page id" in str(e.value)
        assert bool(torch.isfinite(out).all()) and bool((out[2:] == good[2:]).all())
        ghd.ghd_sync_status(su.ctx)                                       # reported once
    su.kv.page_table[0, 1] = int(su.table[0, 1])
    su.kv.page_table[1, 1] = -3                                           # where the second sequence's new rows go
    before = su.dpool.clone()
    ghd.ghd_kv4_append(su.ctx, su.kv, ghd.Kv4Rows(dev(np.array([0, 0, 4], np.int32)), 4), su.dpool, None, k, k)
    with pytest.raises(ghd.GhdError):
        ghd.ghd_sync_status(su.ctx)
    assert bool((su.dpool == before).all())
    su.kv.page_table[1, 1] = int(su.table[1, 1])
    for bad_len in (-4, 16 * su.table.shape[1] - 1, 2**31 - 1):             # no room for two rows
        su.kv_len[0] = bad_len
        for call in (lambda: ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q), lambda: ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, q, k, k),
                     lambda: ghd.ghd_kv4_commit(su.ctx, su.kv, rows, None)):
            su.kv_len[0] = bad_len
            call()
            with pytest.raises(ghd.GhdError) as e:
                ghd.ghd_sync_status(su.ctx)
            assert e.value.name in ("GHD_ENOSPACE", "GHD_EINVAL")
    su.kv_len.copy_(dev(np.array([40, 20], np.int32)))
    with pytest.raises(ghd.GhdError):
        ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, dev(su.start), 4, first=dev(np.array([0, 10**6], np.int32)))
        ghd.ghd_sync_status(su.ctx)


def test_refusals(ghd):
    import torch
    su = Setup(ghd, 4, 4, 64, "f16", 16, [4], [2], 61)
    rows = ghd.Kv4Rows(dev(su.start), 2)
    h = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")  # noqa: E731
    good = (su.kv.page_table, su.kv_len)

    def refused(name, fn):
        launches = ghd.ghd_launch_count(su.ctx)
        with pytest.raises(ghd.GhdError) as e:
            fn()
        assert e.value.name == name
        assert ghd.ghd_launch_count(su.ctx) == launches

    att = lambda kv, rows_=rows, q=None: ghd.ghd_kv4_attention(su.ctx, kv, rows_, torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), h(2, 256) if q is None else q)  # noqa: E731
    refused("GHD_EINVAL", lambda: att(ghd.Kv4Cache(*good, 24, 4, 4)))
    refused("GHD_ESHAPE", lambda: att(ghd.Kv4Cache(*good, 16, 3, 4)))
    refused("GHD_EINVAL", lambda: att(ghd.Kv4Cache(*good, 16, 4, 0)))
    refused("GHD_EINVAL", lambda: att(su.kv, q=h(1, 256)))
    refused("GHD_EINVAL", lambda: att(su.kv, q=torch.zeros(2, 256, device="cuda")))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool[1:], h(2, 256)))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, h(3, 256).view(-1)[1:513].view(2, 256)))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, None, h(2, 256), h(2, 260)[:, :256]))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, h(2, 128), h(2, 256), h(2, 256)))
    big = torch.zeros((1025, 1), dtype=torch.int32, device="cuda")
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_attention(su.ctx, ghd.Kv4Cache(big, big.view(-1), 16, 4, 1), ghd.Kv4Rows(torch.zeros(1026, dtype=torch.int32, device="cuda"), 2),
                                                        su.dpool, h(2, 256)))
    refused("GHD_EINVAL", lambda: ghd.Kv4Rows(dev(su.start), 2, pos=torch.zeros(1, dtype=torch.int32, device="cuda")))
    refused("GHD_EINVAL", lambda: ghd.Kv4Rows(dev(su.start), 2, mask=torch.zeros((1, 1), dtype=torch.int64, device="cuda")))
    assert ghd.ghd_kv4_attention(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), 0), su.dpool, h(2, 256)).abs().sum() == 0      # no rows: nothing to do
    ghd.ghd_sync_status(su.ctx)


def test_steps_captured_in_one_graph_on_a_stream_of_their_own(ghd):
    """append -> attention -> accept's result -> commit, three steps recorded once and replayed twice, against the same
    steps called one by one: lengths, pools and outputs equal to the bit."""
    import torch
    H, Hk, d, R, S, n = 4, 2, 128, 16, 3, 9
    r = np.random.RandomState(71)
    stream = torch.cuda.Stream()
    steps = 3
    lens0 = np.array([0, 33, 200], np.int32)
    paths = r.randint(1, 3, (steps, S))
    res = np.zeros((steps, S, 514), np.int32)
    for t in range(steps):
        for s in range(S):
            m = int(paths[t, s])
            res[t, s, 0], res[t, s, 1] = m, m + 1
            res[t, s, 3:3 + m] = np.sort(r.choice(np.arange(1, n), m, replace=False))
    with torch.cuda.stream(stream):
        ctx = make_ctx(ghd, H, d, "f16")
        pages = 20
        table = dev(np.arange(S * pages, dtype=np.int32).reshape(pages, S).T.copy())
        kv_len = dev(lens0)
        kv = ghd.Kv4Cache(table, kv_len, R, Hk, S * pages)
        pool = ghd.ghd_kv4_pool(ctx, kv, 2)
        rows = ghd.Kv4Rows(dev(np.arange(S + 1, dtype=np.int32) * n), S * n)
        fill = ghd.Kv4Rows(dev(np.concatenate(([0], np.cumsum(lens0))).astype(np.int32)), int(lens0.sum()))
        big = dev(r.randn(int(lens0.sum()), Hk * d).astype(np.float16))
        kv_len.zero_()
        for p in pool:
            ghd.ghd_kv4_append(ctx, kv, fill, p, None, big, big)
        ghd.ghd_kv4_commit(ctx, kv, fill, None)
        assert kv_len.cpu().tolist() == lens0.tolist()
        x = [[dev(r.randn(S * n, w * d).astype(np.float16)) for w in (H, Hk, Hk)] for _ in range(steps)]
        resd = dev(res)
        outs = torch.zeros((steps, 2, S * n, H * d), dtype=torch.float16, device="cuda")
        qr = torch.zeros((S * n, H * d), dtype=torch.float16, device="cuda")
        pool0 = pool.clone()

        def go(t):
            for l in range(2):
                ghd.ghd_kv4_append(ctx, kv, rows, pool[l], *x[t], q_out=qr)
                ghd.ghd_kv4_attention(ctx, kv, rows, pool[l], qr, out=outs[t, l])
            ghd.ghd_kv4_commit(ctx, kv, rows, pool, resd[t])

        for t in range(steps):
            go(t)
        ghd.ghd_sync_status(ctx)
        want = (outs.clone(), pool.clone(), kv_len.clone())
        assert want[2].cpu().tolist() == (lens0 + (paths + 1).sum(0)).tolist()
        graph = torch.cuda.CUDAGraph()
        kv_len.copy_(dev(lens0))
        with torch.cuda.graph(graph, stream=stream):
            for t in range(steps):
                go(t)
        for _ in range(2):
            kv_len.copy_(dev(lens0))
            pool.copy_(pool0)
            outs.zero_()
            graph.replay()
            ghd.ghd_sync_status(ctx)
            for a, b in zip((outs, pool, kv_len), want):
                assert bool((a == b).all())


def test_a_decode_loop_over_the_paged_cache_agrees_with_decoding_one_row_at_a_time(ghd):
    """A chain of rows verified as one tree gives each row what decoding it alone gives (the same cache rows are read),
    and the path accepted out of a branching tree leaves the cache that appending its rows in sequence leaves."""
    import torch
    H, Hk, d, R = 4, 2, 64, 16
    ctx = make_ctx(ghd, H, d, "f32")
    r = np.random.RandomState(81)
    table = dev(np.array([[4, 2, 7, 0]], np.int32))
    q, k, v = (dev(r.randn(30, w * d).astype(np.float32)) for w in (H, Hk, Hk))

    def fresh():
        kv = ghd.Kv4Cache(table, dev(np.array([0], np.int32)), R, Hk, 8)
        return kv, ghd.ghd_kv4_pool(ctx, kv)

    one_row = ghd.Kv4Rows(dev(np.array([0, 1], np.int32)), 1)
    kv_a, pool_a = fresh()
    alone = []
    for i in range(30):
        qr = ghd.ghd_kv4_append(ctx, kv_a, one_row, pool_a[0], q[i:i + 1], k[i:i + 1], v[i:i + 1])
        alone.append(ghd.ghd_kv4_attention(ctx, kv_a, one_row, pool_a[0], qr))
        ghd.ghd_kv4_commit(ctx, kv_a, one_row, None)
    kv_b, pool_b = fresh()
    rows = ghd.Kv4Rows(dev(np.array([0, 30], np.int32)), 30)
    qr = ghd.ghd_kv4_append(ctx, kv_b, rows, pool_b[0], q, k, v)
    chain = ghd.ghd_kv4_attention(ctx, kv_b, rows, pool_b[0], qr)
    assert bool((pool_a == pool_b).all())
    a, b = torch.cat(alone).double(), chain.double()
    assert float((a - b).abs().max()) <= 2.0 ** -17 * float(a.abs().max())     # both within the bounds of the 32-bit sums
    # tree: rows 0, 1, 2 are the accepted path at nodes 0, 3, 5; the others are alternatives
    kv_c, pool_c = fresh()
    pick = torch.tensor([0, 7, 8, 1, 9, 2], device="cuda")
    pos = dev(np.array([0, 1, 1, 1, 2, 2], np.int32))
    vis = np.eye(6, dtype=np.uint8)
    vis[:, 0] = 1
    vis[4, 1] = vis[5, 3] = 1
    mask = np.zeros((6, 64), np.uint8)
    mask[:, :6] = vis
    rows = ghd.Kv4Rows(dev(np.array([0, 6], np.int32)), 6, pos=pos, mask=dev(np.packbits(mask, axis=1, bitorder="little").view(np.int64)))
    qr = ghd.ghd_kv4_append(ctx, kv_c, rows, pool_c[0], q[pick], k[pick], v[pick])
    out = ghd.ghd_kv4_attention(ctx, kv_c, rows, pool_c[0], qr)
    assert float((out[[0, 3, 5]].double() - a[:3]).abs().max()) <= 2.0 ** -17 * float(a.abs().max())
    res = np.zeros((1, 514), np.int32)
    res[0, :5] = [2, 3, 0, 3, 5]
    ghd.ghd_kv4_commit(ctx, kv_c, rows, pool_c, dev(res))
    ghd.ghd_sync_status(ctx)
    assert int(kv_c.kv_len[0]) == 3
    three, first = dev(np.array([0, 3], np.int32)), dev(np.array([0], np.int32))
    for x, y in zip(ghd.ghd_kv4_read(ctx, kv_c, pool_c[0], three, 3, first=first), ghd.ghd_kv4_read(ctx, kv_a, pool_a[0], three, 3, first=first)):
        assert bool((x == y).all())


def on_path(ghd, ctx, path):
    ghd.ghd_set_option(ctx, 2, path)


def test_special_rows_in_the_tcgen05_kernel(ghd):
    """A row that sees nothing, one that sees the cache alone, a key of NaN, a value of infinity and a query of NaN, among 40 rows."""
    su = Setup(ghd, 4, 2, 128, "f16", 32, [0, 37], [40, 40], 91)
    on_path(ghd, su.ctx, 2)
    vis, words = su.trees()
    words[7] = 0
    vis[0][7] = False
    words[40 + 11] = 0
    vis[1][11] = False
    for node, which in ((1, 0), (2, 1)):
        page, row = okv4.slots(su.table, su.R, 1, 37 + node)
        for h in range(2):
            su.pool.put(which, page, row, h, su.pool.codes(which, page, row, h), np.nan if which == 0 else np.inf, 0.5)
    su.dpool.copy_(dev(su.pool.data.reshape(-1)))
    collect(su)
    q = su.r.randn(80, 4, 128).astype(np.float16)
    q[20, 1, 5] = np.nan
    out = ghd.ghd_kv4_attention(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), 80, mask=dev(words)), su.dpool, dev(q.reshape(80, -1)))
    ghd.ghd_sync_status(su.ctx)
    got = out.double().cpu().numpy().reshape(80, 4, 128)
    assert (got[7] == 0).all() and np.isnan(got[20, 1]).all()
    clean = np.ones((80, 4), bool)
    clean[20, 1] = False
    sees_nan = np.tril(vis[1])[:, 1] | np.tril(vis[1])[:, 2]
    clean[40:][sees_nan] = False
    assert not np.isfinite(got[40:][sees_nan]).all(-1).any() and clean.sum() > 200
    q[20, 1] = 0
    with np.errstate(all="ignore"):
        want = okv4.attention(su.pool, su.table, su.lens, su.start, vis, q)
    assert (np.abs(got - want) <= attention_tolerance(su, np.nan_to_num(q))(want))[clean].all()


@pytest.mark.parametrize("path", [1, 2], ids=["rows", "tcgen05"])
def test_scores_and_scales_that_grow_along_the_cache(ghd, path):
    """Scores rise by far more than the reference's slack every few keys, and V's scales by a factor of 10^4: references and the
    exponent have to follow.  Late keys carry nearly all weight, so the output is close to their values."""
    su = Setup(ghd, 2, 2, 128, "f16", 16, [700], [70], 93, garbage=False)
    on_path(ghd, su.ctx, path)
    for t in range(770):
        page, row = okv4.slots(su.table, 16, 0, t)
        for h in range(2):
            x = np.full(128, 0.004 * t, np.float32)
            x[::2] += 0.5
            su.pool.put(0, page, row, h, *okv4.quantise(x, "f16"))
            su.pool.put(1, page, row, h, su.pool.codes(1, page, row, h), 0.01 * 10 ** (4 * t / 770), -0.07 * 10 ** (4 * t / 770))
    su.dpool.copy_(dev(su.pool.data.reshape(-1)))
    collect(su)
    vis = [np.tril(np.ones((70, 70), bool))]
    q = np.abs(su.r.randn(70, 2, 128)).astype(np.float16)
    out = ghd.ghd_kv4_attention(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), 70), su.dpool, dev(q.reshape(70, -1)))
    ghd.ghd_sync_status(su.ctx)
    got = out.double().cpu().numpy().reshape(70, 2, 128)
    want = okv4.attention(su.pool, su.table, su.lens, su.start, vis, q)
    assert np.isfinite(got).all() and (np.abs(got - want) <= attention_tolerance(su, q)(want)).all()


@pytest.mark.parametrize("path", [1, 2], ids=["rows", "tcgen05"])
def test_the_same_bits_every_time_over_many_blocks(ghd, path):
    su = Setup(ghd, 4, 4, 128, "f16", 64, [900, 10, 0, 333], [33, 64, 5, 0], 95)
    on_path(ghd, su.ctx, path)
    vis, words = su.trees()
    n = su.n
    q = dev(su.r.randn(n, 4 * 128).astype(np.float16))
    rows = ghd.Kv4Rows(dev(su.start), n, mask=dev(words))
    first = ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q).clone()
    for _ in range(20):
        assert bool((ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q) == first).all())
    ghd.ghd_sync_status(su.ctx)


@pytest.mark.parametrize("offset", [-8.0, 0.01, 8.0])
@pytest.mark.parametrize("dtype,path,n", [("f16", 1, 3), ("f16", 1, 12), ("f16", 2, 40), ("f32", 0, 3)])
def test_keys_without_a_page_before_those_with_one(ghd, dtype, path, n, offset):
    """The first 320 rows have page ids that no pool has: the call reports it, and gives what the other rows alone give, whether
    their scores are far below 0, near it or far above.  64 sequences share the pages, so that a block walks on from rows without
    a page to rows with one."""
    H, d, R, gone, S = 2, 128, 32, 10, 64
    su = Setup(ghd, H, H, d, dtype, R, [1000], [n], 99, garbage=False)
    for t in range(1000 + n):
        page, row = okv4.slots(su.table, R, 0, t)
        for h in range(H):
            su.pool.put(0, page, row, h, *okv4.quantise((offset + 0.1 * su.r.randn(d)).astype(np.float32), dtype))
    su.dpool.copy_(dev(su.pool.data.reshape(-1)))
    on_path(ghd, su.ctx, path)
    table = np.repeat(su.table, S, 0)
    table[:, :gone] = -1
    kv = ghd.Kv4Cache(dev(table), dev(np.full(S, 1000, np.int32)), R, H, su.kv.c.n_pages)
    q = (1.0 + 0.2 * su.r.randn(n, H, d)).astype(su.np_t)
    vis, words = su.trees()
    rows = ghd.Kv4Rows(dev(np.arange(S + 1, dtype=np.int32) * n), S * n, mask=dev(np.tile(words[:n], (S, 1))))
    out = ghd.ghd_kv4_attention(su.ctx, kv, rows, su.dpool, dev(np.tile(q.reshape(n, -1), (S, 1))))
    with pytest.raises(ghd.GhdError):
        ghd.ghd_sync_status(su.ctx)
    su.table, su.lens = su.table[:, gone:].copy(), [1000 - gone * R]
    collect(su)
    want = okv4.attention(su.pool, su.table, su.lens, su.start, vis, q)
    got = out.double().cpu().numpy().reshape(S, n, H, d)
    assert (np.abs(got - want) <= attention_tolerance(su, q)(want)).all()


def test_two_contexts_on_two_streams_at_once(ghd):
    """Each context has its own workspace, so calls of two of them may overlap."""
    import torch
    sets = []
    for i in range(2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            su = Setup(ghd, 4, 4, 128, "f16", 64, [800 + 100 * i, 10], [70, 3], 96 + i)
            vis, words = su.trees()
            q = dev(su.r.randn(su.n, 4 * 128).astype(np.float16))
            rows = ghd.Kv4Rows(dev(su.start), su.n, mask=dev(words))
            alone = ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q).clone()
            stream.synchronize()
            sets.append((stream, su, q, rows, alone, torch.empty_like(q)))
    for _ in range(10):
        for stream, su, q, rows, alone, out in sets:
            with torch.cuda.stream(stream):
                ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q, out=out)
    torch.cuda.synchronize()
    for stream, su, q, rows, alone, out in sets:
        ghd.ghd_sync_status(su.ctx)
        assert bool((out == alone).all())


@pytest.mark.parametrize("dtype,d", [("f16", 64), ("f16", 128), ("f32", 64), ("f32", 128)])
def test_append_of_ties_and_of_the_ends_of_the_range(ghd, dtype, d):
    """Quotients that are exactly a half, rows of one value, of the largest and of the smallest values: codes bit for bit."""
    su = Setup(ghd, 2, 2, d, dtype, 16, [0], [9], 97, garbage=False)
    r = np.random.RandomState(5)
    top = 60000.0 if dtype == "f16" else 3.0e38
    tiny = 6e-8 if dtype == "f16" else 1.4e-45
    v = np.zeros((9, 2, d), np.float64)
    v[0] = r.randint(0, 31, (2, d)) * 0.5                          # with ends 0 and 15: scale 1, halves
    v[0, :, 0], v[0, :, 1] = 0, 15
    v[1] = -v[0] * 0.25 - 3
    v[2] = 0.75
    v[3] = r.uniform(-top, top, (2, d))
    v[3, :, 0], v[3, :, 1] = -top, top
    v[4] = r.randint(0, 40, (2, d)) * tiny                         # below the normal range
    v[5] = r.randint(0, 2, (2, d)) * tiny                          # the scale rounds to 0
    v[6] = 1000 + r.randint(0, 3, (2, d))                          # the minimum's rounding against a small scale
    v[7] = np.where(r.rand(2, d) < 0.5, -0.0, 0.0)
    v[8] = r.randn(2, d) * np.exp2(r.randint(-12, 12, (2, d)))
    v = v.astype(su.np_t)
    rows = ghd.Kv4Rows(dev(su.start), 9)
    flat = dev(v.reshape(9, -1))
    pos = dev(np.zeros(9, np.int32))                               # no rotation: K gets the same rows
    ghd.ghd_kv4_append(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), 9, pos=pos), su.dpool, None, flat, flat)
    ghd.ghd_sync_status(su.ctx)
    okv4.append(su.pool, su.table, su.lens, su.start, np.zeros(9, np.int32), v, v, v, THETA)
    got = okv4.Pool(su.pool.data.shape[0], 2, 16, d, dtype, data=su.dpool.cpu().numpy().reshape(su.pool.data.shape))
    page, row = okv4.slots(su.table, 16, 0, 7)
    for which in (0, 1):
        for h in (0, 1):                                           # of zeros of both signs either is the lowest: equal, but not the same bits
            scale, mn = got.params(which, page, row, h)
            assert scale == 0 and mn == 0
            su.pool.put(which, page, row, h, su.pool.codes(which, page, row, h), scale, mn)
    assert np.array_equal(got.data, su.pool.data)


def test_more_refusals(ghd):
    import torch
    su = Setup(ghd, 4, 4, 64, "f32", 16, [4], [2], 98)
    rows = ghd.Kv4Rows(dev(su.start), 2)
    q = torch.zeros((2, 256), device="cuda")

    def refused(name, fn):
        launches = ghd.ghd_launch_count(su.ctx)
        with pytest.raises(ghd.GhdError) as e:
            fn()
        assert e.value.name == name and ghd.ghd_launch_count(su.ctx) == launches

    on_path(ghd, su.ctx, 2)
    refused("GHD_EUNSUPPORTED", lambda: ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q))
    on_path(ghd, su.ctx, 0)
    res = torch.zeros((1, 514), dtype=torch.int32, device="cuda")
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_commit(su.ctx, su.kv, rows, [su.dpool, su.dpool], res))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_commit(su.ctx, su.kv, rows, [], res))
    long = ghd.Kv4Cache(torch.zeros((1, (1 << 23) + 1), dtype=torch.int32, device="cuda"), su.kv_len, 128, 4, 1)
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_attention(su.ctx, long, rows, su.dpool, q))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool.cpu(), q))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q, out=q.cpu()))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, dev(su.start), 2, k_out=q[:1]))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_commit(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), -1), None))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q, out=q))
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, dev(su.start), 2, k_out=q, v_out=q))
    odd = ghd.Kv4Rows(dev(su.start), 2, mask=torch.ones((2, 1), dtype=torch.int64, device="cuda"))
    odd.c.mask += 4                                                # what only a C caller can pass
    refused("GHD_EINVAL", lambda: ghd.ghd_kv4_attention(su.ctx, su.kv, odd, su.dpool, q))
    with pytest.raises(ghd.GhdError):
        ghd.Kv4Rows(torch.zeros(2, dtype=torch.int32), 2)
    with pytest.raises(ghd.GhdError):
        ghd.Kv4Rows(dev(np.zeros(4, np.int32))[::2], 2)


@pytest.mark.parametrize("dtype,d", [("f16", 128), ("f32", 64)])
def test_commit_of_long_paths_that_overlap_themselves(ghd, dtype, d):
    """Paths of 8, 9 and 70 rows whose sources are the places of rows moved earlier, over page borders."""
    lens, cnt = [13, 0, 100], [10, 40, 80]
    su = Setup(ghd, 2, 1, d, dtype, 16, lens, cnt, 43)
    paths = [(8, [0] + list(range(2, 10))), (9, [0] + sorted(np.random.RandomState(4).choice(np.arange(9, 40), 9, replace=False).tolist())), (70, [0] + list(range(9, 79)))]
    host = [okv4.Pool(su.pool.data.shape[0], 1, 16, d, dtype, data=su.pool.data.copy())]
    res = np.zeros((3, 514), np.int32)
    for s, (m, nodes) in enumerate(paths):
        res[s, 0], res[s, 1], res[s, 2:3 + m] = m, m + 1, nodes
    ghd.ghd_kv4_commit(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), su.n), [su.dpool], dev(res))
    ghd.ghd_sync_status(su.ctx)
    assert su.kv_len.cpu().tolist() == okv4.commit(host, su.table, lens, su.start, paths) == [22, 10, 171]
    assert np.array_equal(su.dpool.cpu().numpy(), host[0].data.reshape(-1))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_long_call_is_its_pieces(ghd, dtype):
    """12,000 rows of five sequences appended and read at once (a warp has several rows, and queries and keys of each) against a
    call for every 300 of them: queries, pool and rows read equal to the bit; queries in place too."""
    import torch
    H, Hk, d, R, n = 4, 2, 64, 32, 12000
    ctx = make_ctx(ghd, H, d, dtype)
    r = np.random.RandomState(101)
    cnt = np.array([5000, 0, 1, 6000, 999])
    start = np.concatenate(([0], np.cumsum(cnt)))
    lens = np.array([3, 7, 0, 40, 100])
    pages = -(-(lens + cnt) // R)
    table = np.zeros((5, pages.max()), np.int32)
    order = r.permutation(pages.sum())
    for s in range(5):
        table[s, :pages[s]] = order[pages[:s].sum():pages[: s + 1].sum()]
    T = torch.float16 if dtype == "f16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(n, (H + 2 * Hk) * d, device="cuda", generator=gen).to(T)
    pos = dev(r.randint(0, 5000, n).astype(np.int32))
    q, k, v = (t.contiguous() for t in x.split((H * d, Hk * d, Hk * d), 1))
    kv = ghd.Kv4Cache(dev(table), dev(lens.astype(np.int32)), R, Hk, int(pages.sum()))
    whole = ghd.ghd_kv4_pool(ctx, kv)[0]
    all_rows = dev(start.astype(np.int32))
    qa = ghd.ghd_kv4_append(ctx, kv, ghd.Kv4Rows(all_rows, n, pos=pos), whole, q, k, v)
    ka, va = ghd.ghd_kv4_read(ctx, kv, whole, all_rows, n)
    parts, qb, kb, vb = torch.zeros_like(whole), torch.empty_like(qa), torch.empty_like(ka), torch.empty_like(va)
    for s in range(5):
        for i in range(0, cnt[s], 300):
            m = min(300, cnt[s] - i)
            at = slice(start[s] + i, start[s] + i + m)
            one = ghd.Kv4Cache(dev(table[s:s + 1]), dev(np.array([lens[s] + i], np.int32)), R, Hk, int(pages.sum()))
            few = dev(np.array([0, m], np.int32))
            qb[at] = ghd.ghd_kv4_append(ctx, one, ghd.Kv4Rows(few, m, pos=pos[at].contiguous()), parts, q[at], k[at], v[at])
            kb[at], vb[at] = ghd.ghd_kv4_read(ctx, one, parts, few, m)
    ghd.ghd_sync_status(ctx)
    for a, b in ((qa, qb), (whole, parts), (ka, kb), (va, vb)):
        assert bool((a == b).all())
    qc = q.clone()
    ghd.ghd_kv4_append(ctx, kv, ghd.Kv4Rows(all_rows, n, pos=pos), whole, qc, k, v, q_out=qc)
    assert bool((qc == qa).all()) and bool((whole == parts).all())
    ghd.ghd_sync_status(ctx)


def test_commit_of_more_layers_than_one_launch_takes(ghd):
    import torch
    su = Setup(ghd, 2, 1, 64, "f16", 16, [20, 3], [6, 5], 47)
    L = 70
    pools = torch.from_numpy(su.r.randint(0, 256, (L, su.dpool.numel())).astype(np.uint8)).cuda()
    host = [okv4.Pool(su.pool.data.shape[0], 1, 16, 64, "f16", data=p.cpu().numpy().reshape(su.pool.data.shape)) for p in pools]
    paths = [(2, [0, 3, 5]), (1, [0, 4])]
    res = np.zeros((2, 514), np.int32)
    for s, (m, nodes) in enumerate(paths):
        res[s, 0], res[s, 1], res[s, 2:3 + m] = m, m + 1, nodes
    ghd.ghd_kv4_commit(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), su.n), pools, dev(res))
    ghd.ghd_sync_status(su.ctx)
    assert su.kv_len.cpu().tolist() == okv4.commit(host, su.table, [20, 3], su.start, paths)
    assert np.array_equal(pools.cpu().numpy(), np.stack([h.data.reshape(-1) for h in host]))


def test_keys_that_the_rotation_takes_below_the_range(ghd):
    su = Setup(ghd, 2, 1, 128, "f16", 16, [0], [3], 49)
    k = su.r.randn(3, 128).astype(np.float16)
    k[1, :64], k[1, 64:] = -60000, 60000                            # by 0.75 radians: -60000 (cos + sin) = -84800
    ghd.ghd_kv4_append(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), 3, pos=dev(np.ones(3, np.int32))), su.dpool, None, dev(k), dev(su.r.randn(3, 128).astype(np.float16)))
    kb, vb = (x.float().cpu().numpy() for x in ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, dev(su.start), 3))
    ghd.ghd_sync_status(su.ctx)
    assert np.isneginf(kb[1]).all() and np.isfinite(kb[[0, 2]]).all() and np.isfinite(vb).all()


def test_broadcast_rows_are_refused_before_a_launch(ghd):
    import torch
    su = Setup(ghd, 4, 2, 64, "f16", 16, [4], [2], 62)
    rows = ghd.Kv4Rows(dev(su.start), 2)
    q, k = torch.zeros((2, 256), dtype=torch.float16, device="cuda"), torch.zeros((2, 128), dtype=torch.float16, device="cuda")
    before, launches = su.dpool.clone(), ghd.ghd_launch_count(su.ctx)
    for args in ((q[:1].expand(2, 256), k, k), (q, k[:1].expand(2, 128), k[:1].expand(2, 128)), (None, k, k[:1].expand(2, 128))):
        with pytest.raises(ghd.GhdError) as e:
            ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, *args)
        assert e.value.name == "GHD_EINVAL"
    assert ghd.ghd_launch_count(su.ctx) == launches and bool((su.dpool == before).all())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_append_of_one_row_takes_any_row_stride(ghd, dtype):
    """q of one row in a wider buffer, rotated in place; k a transposed column; v a column block: as contiguous copies give."""
    import torch
    H, Hk, d = 4, 2, 64
    su = Setup(ghd, H, Hk, d, dtype, 16, [9], [1], 63, garbage=False)
    rows = ghd.Kv4Rows(dev(su.start), 1)
    q, k, v = (dev(su.r.randn(1, w * d).astype(su.np_t)) for w in (H, Hk, Hk))
    want_pool = su.dpool.clone()
    want_q = ghd.ghd_kv4_append(su.ctx, su.kv, rows, want_pool, q, k, v)
    wide = torch.zeros((1, 1024), dtype=q.dtype, device="cuda")
    wide[:, 256:512], wide[:, 512:640] = q, v
    qi = wide[:, 256:512]
    got = ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, qi, k.reshape(Hk * d, 1).clone().t(), wide[:, 512:640], q_out=qi)
    ghd.ghd_sync_status(su.ctx)
    assert got.data_ptr() == qi.data_ptr() and bool((qi == want_q).all()) and bool((su.dpool == want_pool).all())
    assert not wide[:, :256].any() and bool((wide[:, 512:640] == v).all()) and not wide[:, 640:].any()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_outputs_made_under_another_current_stream_are_the_kernels(ghd, dtype):
    """The context's kernels run on its own stream.  A call under another current stream, busy with a long kernel and then with
    writes to memory that is free again, gives what it gives under the context's."""
    import torch
    H, Hk, d = 4, 2, 64
    su = Setup(ghd, H, Hk, d, dtype, 16, [40, 7], [5, 3], 64, garbage=False)
    rows = ghd.Kv4Rows(dev(su.start), su.n)
    q, k, v = (dev(su.r.randn(su.n, w * d).astype(su.np_t)) for w in (H, Hk, Hk))
    pool0, other = su.dpool.clone(), torch.cuda.Stream()

    def busy(*shapes):                                          # writes that come late, to memory that the next such tensor gets
        if torch.cuda.current_stream() == su.ctx.stream:
            return
        for t in [torch.empty(s, dtype=q.dtype, device="cuda") for s in shapes]:
            torch.cuda._sleep(20_000_000)
            t.fill_(9.0)

    def calls():
        busy(q.shape)
        qr = ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, q, k, v)
        busy(q.shape)
        out = ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q)
        busy(k.shape, k.shape)
        kb, vb = ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, rows.row_start, su.n)
        busy()
        torch.cuda._sleep(20_000_000)
        pool = ghd.ghd_kv4_pool(su.ctx, su.kv, 2)
        ghd.ghd_kv4_append(su.ctx, su.kv, rows, pool[1], None, k, v)
        return [qr, out, kb, vb, pool]

    want = [x.clone() for x in calls()]
    torch.cuda.synchronize()
    assert all(bool(x.any()) for x in want)
    su.dpool.copy_(pool0)
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        got = calls()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert a.shape == b.shape and bool((a.view(torch.uint8) == b.view(torch.uint8)).all())


def test_a_bad_page_does_not_hide_a_wait_that_ran_out(ghd):
    """A bad page id is reported, and the kernel runs on.  A wait that runs out after that has to be reported too, and what it left
    in the workspace (arrival counters) be cleared.  The wait is played by the words that it would have left."""
    import torch
    su = Setup(ghd, 2, 2, 64, "f16", 16, [1500], [2], 65, garbage=False)
    rows = ghd.Kv4Rows(dev(su.start), 2)
    q = dev(su.r.randn(2, 128).astype(np.float16))
    good = ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q).clone()
    ghd.ghd_sync_status(su.ctx)
    first = int(su.kv.page_table[0, 0])
    su.kv.page_table[0, 0] = -1
    ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q)
    su.kv.page_table[0, 0] = first
    words = su.ctx.workspace[:256 + 4 * 4096].view(torch.int32)       # status words, then the counters
    words[:1] = torch.where(words[:1] == 0, 3, words[:1])             # a kernel records it where nothing stands
    words[64:] = 5
    with pytest.raises(ghd.GhdError) as e:
        ghd.ghd_sync_status(su.ctx)
    assert e.value.name == "GHD_ETIMEOUT"
    ghd.ghd_sync_status(su.ctx)                                       # reported once
    assert not words.any()
    assert bool((ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q) == good).all())
    su.kv.page_table[0, 0] = -1
    ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, q)
    with pytest.raises(ghd.GhdError, match="page id"):
        ghd.ghd_sync_status(su.ctx)


SINKS = [(1, 1, 1), (1, 1, 9), (1, 4, 3), (2, 1, 40), (2, 4, 17)]       # kernel, query heads a key head, new rows


@pytest.mark.parametrize("behind", [9.0, 13.0], ids=["9 below", "13 below"])
@pytest.mark.parametrize("size", [1e-3, 1e-2, 0.1])
@pytest.mark.parametrize("path,g,n", SINKS)
@pytest.mark.parametrize("d", [64, 128])
def test_small_weights_keep_their_bits(ghd, d, path, g, n, size, behind):
    """One key has nearly all the weight and values of 0; the others, `behind` nats below it, make the output.  Queries have one
    channel that is not 0, so scores are sums of three exact products.

    Bound of an element, with the weights of the oracle: each weight times scale is rounded to half (2^-11) and its score and exponential
    are off by 2^-18 at most (scores below 32 in powers of two, in 32 bits: a few times 2^-19 each), times |code - 8|; the middles
    min + 8 scale are off by 2^-18 likewise; sums of L terms in 32 bits (2^-23 each, tensor cores may truncate), taken relative to the sum
    of their sizes; output half a step of half, 2^-25 below the normal range.  A weight rounded below half's normal range is off by
    up to half of itself: far above this bound."""
    import torch
    H, Hk, L = g, 1, 2048
    r = np.random.RandomState(100 * n + d)
    su = Setup(ghd, H, Hk, d, "f16", 64, [0], [1], 17, spare=0, garbage=False)
    n_pages = (L + n + 63) // 64
    pool = okv4.Pool(n_pages, Hk, 64, d, "f16")
    table = r.permutation(n_pages).astype(np.int32)[None]
    q = np.zeros((n, H, d), np.float16)
    q[:, :, 0] = 8.0
    top = int(r.randint(0, L))
    scale = 1.0 if d == 64 else 1.5
    step = 8.0 * scale / np.sqrt(d)                            # nats of one code of channel 0
    score = 15 - np.rint((behind + r.rand(L + n) * 1.5) / step)
    assert 0 <= score.min() and score.max() < 8
    for t in range(L + n):
        page, row = okv4.slots(table, 64, 0, t)
        c = r.randint(0, 16, d)
        c[0] = 15 if t == top else int(score[t])
        pool.put(0, page, row, 0, c.astype(np.uint8), scale, -2.0)
        pool.put(1, page, row, 0, *okv4.quantise((r.randn(d) * size * (t != top)).astype(np.float32), "f16"))
    on_path(ghd, su.ctx, path)
    kv = ghd.Kv4Cache(dev(table), dev(np.array([L], np.int32)), 64, Hk, n_pages)
    out = ghd.ghd_kv4_attention(su.ctx, kv, ghd.Kv4Rows(dev(np.array([0, n], np.int32)), n), dev(pool.data.reshape(-1)), dev(q.reshape(n, -1)))
    ghd.ghd_sync_status(su.ctx)
    got = out.double().cpu().numpy().reshape(n, H, d)
    K, V = okv4.rows(pool, table, 0, 0, L + n)
    par = np.array([pool.params(1, *okv4.slots(table, 64, 0, t), 0).astype(np.float64) for t in range(L + n)])
    code = (V[:, 0] - par[:, 1:]) / np.where(par[:, :1] == 0, 1.0, par[:, :1])
    for i in range(n):
        see = np.arange(L + n) <= L + i
        w = np.exp(K[see, 0, 0] * 8.0 / np.sqrt(d) - (K[see, 0, 0] * 8.0 / np.sqrt(d)).max())
        w /= w.sum()
        assert w[top] > 0.5
        part, middle = par[see, :1] * np.abs(code[see] - 8), np.abs(par[see, 1:] + 8 * par[see, :1])
        want = w @ V[see, 0]
        tol = w @ (part * (2.0 ** -11 + 2.0 ** -18 + L * 2.0 ** -23) + middle * (2.0 ** -18 + L * 2.0 ** -23)) + np.maximum(2.0 ** -11 * np.abs(want), 2.0 ** -25)
        assert (np.abs(got[i] - want) <= tol).all(), (i, float((np.abs(got[i] - want) / tol).max()))


@pytest.mark.parametrize("dtype,d,path,g,n", [("f16", 128, 1, 2, 3), ("f16", 64, 1, 1, 12), ("f16", 128, 2, 1, 40), ("f16", 64, 2, 2, 20)])
def test_rows_that_see_a_key_of_minus_infinity_get_nan(ghd, dtype, d, path, g, n):
    """The rotation takes cache row 70 and, in another sequence, new row 1 below half's range: they read back as -inf, whose product
    with a query is no number, whatever the sign of the query's sum.  Rows that do not see them are what they are without them."""
    Hk, R = 2, 32
    H = g * Hk
    su = Setup(ghd, H, Hk, d, dtype, R, [90, 50], [n, n], 19, garbage=False)
    on_path(ghd, su.ctx, path)
    for s, t in ((0, 70), (1, 51)):
        page, row = okv4.slots(su.table, R, s, t)
        for h in range(Hk):
            su.pool.put(0, page, row, h, su.pool.codes(0, page, row, h), 7000.0, -np.inf)
    su.dpool.copy_(dev(su.pool.data.reshape(-1)))
    vis = [np.ones((n, n), bool), np.ones((n, n), bool)]
    vis[1][2:, 1] = np.arange(2, n) % 2 == 0                           # some rows behind new row 1 do not see it
    mask = np.zeros((2 * n, 64), np.uint8)
    mask[:n, :n], mask[n:, :n] = vis[0], vis[1]
    words = np.packbits(mask, axis=1, bitorder="little").view(np.int64)
    q = su.r.randn(2 * n, H, d).astype(su.np_t)
    q[::2] += np.float16(0.5)                                           # sums of both signs, channels of both signs in every row
    q[1::2] -= np.float16(0.5)
    assert (q.min(-1) < 0).all() and (q.max(-1) > 0).all() and (q.astype(np.float64).sum(-1) > 0).any() and (q.astype(np.float64).sum(-1) < 0).any()
    out = ghd.ghd_kv4_attention(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), 2 * n, mask=dev(words)), su.dpool, dev(q.reshape(2 * n, -1)))
    ghd.ghd_sync_status(su.ctx)
    got = out.double().cpu().numpy().reshape(2 * n, H, d)
    with np.errstate(all="ignore"):
        collect(su)
        want = okv4.attention(su.pool, su.table, su.lens, su.start, vis, q)
    bad = np.ones(2 * n, bool)
    bad[n] = False                                                      # new row 0 comes before it
    bad[n:] &= np.tril(vis[1])[:, 1]
    assert np.isnan(want[bad]).all() and np.isfinite(want[~bad]).all() and (n <= 3 or (~bad).sum() > 2)
    assert np.isnan(got[bad]).all()
    assert (np.abs(got - want)[~bad] <= attention_tolerance(su, q)(want)[~bad]).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_calls_without_rows_take_buffers_without_elements(ghd, dtype):
    """A step in which no sequence has a new row: tensors of no rows have no memory, and the calls do nothing."""
    import torch
    su = Setup(ghd, 4, 2, 64, dtype, 16, [20, 3], [0, 0], 66, garbage=False)
    e = lambda *s, t=su.ctx.cfg.torch_dtype: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    rows = ghd.Kv4Rows(dev(su.start), 0, pos=e(0, t=torch.int32), mask=e(0, 1, t=torch.int64))
    before, launches = su.dpool.clone(), ghd.ghd_launch_count(su.ctx)
    assert ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, e(0, 256), e(0, 128), e(0, 128)).shape == (0, 256)
    assert ghd.ghd_kv4_append(su.ctx, su.kv, rows, su.dpool, None, e(0, 128), e(0, 128)) is None
    assert ghd.ghd_kv4_attention(su.ctx, su.kv, rows, su.dpool, e(0, 256)).shape == (0, 256)
    assert [x.shape for x in ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, rows.row_start, 0)] == [(0, 128), (0, 128)]
    ghd.ghd_kv4_commit(su.ctx, su.kv, rows, None)
    ghd.ghd_sync_status(su.ctx)
    assert ghd.ghd_launch_count(su.ctx) == launches and bool((su.dpool == before).all()) and su.kv_len.cpu().tolist() == [20, 3]


def test_a_cache_that_the_calls_refuse_has_no_pool(ghd):
    import torch
    su = Setup(ghd, 4, 2, 64, "f16", 16, [4], [2], 67, garbage=False)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    good = ghd.ghd_kv4_pool_bytes(su.ctx, ghd.Kv4Cache(z(1024, 2), z(1024), 128, 2, 3))
    assert good == 3 * 2 * okv4.block_bytes(128, 64, "f16")
    for table, args in ((z(1025, 2), (128, 2, 3)), (z(0, 2), (128, 2, 3)), (z(2, 0), (128, 2, 3)), (z(1, (1 << 23) + 1), (128, 2, 3)), (z(2, 2), (24, 2, 3)), (z(2, 2), (128, 3, 3)),
                        (z(2, 2), (128, 0, 3)), (z(2, 2), (128, 2, 0)), (z(2, 2), (128, 2, -1))):
        assert ghd.ghd_kv4_pool_bytes(su.ctx, ghd.Kv4Cache(table, z(table.shape[0]), *args)) == 0, (tuple(table.shape), args)


@pytest.mark.parametrize("dtype,d", [("f16", 128), ("f32", 64)])
def test_keys_alone_or_values_alone_are_read(ghd, dtype, d):
    import torch
    su = Setup(ghd, 2, 2, d, dtype, 16, [40, 0, 9], [1, 1, 1], 68)
    start, first, n = dev(np.array([0, 5, 5, 12], np.int32)), dev(np.array([30, 0, 2], np.int32)), 12
    k, v = ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, start, n, first=first)
    only_k, no_v = ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, start, n, first=first, values=False)
    no_k, only_v = ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, start, n, first=first, keys=False)
    ghd.ghd_sync_status(su.ctx)
    assert no_v is None and no_k is None and bool((only_k == k).all()) and bool((only_v == v).all())
    out = torch.zeros_like(v)
    assert ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, start, n, first=first, v_out=out, keys=False)[1] is out and bool((out == v).all())
    for kw in (dict(keys=False, values=False), dict(keys=False, k_out=out), dict(values=False, v_out=out)):
        with pytest.raises(ghd.GhdError) as e:
            ghd.ghd_kv4_read(su.ctx, su.kv, su.dpool, start, n, first=first, **kw)
        assert e.value.name == "GHD_EINVAL"


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_which_kernel_ran_is_counted(ghd, dtype):
    """Few rows take the kernel of narrow tiles, many in half mode the tcgen05 kernel, and the option picks one of the two."""
    ctx = make_ctx(ghd, 4, 64, dtype)
    few, many = (Setup(ghd, 4, 4, 64, dtype, 16, [30], [n], 69, garbage=False) for n in (1, 100))
    want = [0, 0]
    for path in (0, 1, 2):
        for su, tc in ((few, path == 2), (many, path == 2 or (path == 0 and dtype == "f16"))):
            if path == 2 and dtype == "f32":                    # refused: nothing runs
                continue
            on_path(ghd, ctx, path)
            ghd.ghd_kv4_attention(ctx, su.kv, ghd.Kv4Rows(dev(su.start), su.n), su.dpool, dev(su.r.randn(su.n, 256).astype(su.np_t)))
            want[tc] += 1
            assert [ghd.ghd_path_count(ctx, p) for p in (ghd.PATH_KV4_ROWS, ghd.PATH_KV4_TC)] == want
    ghd.ghd_sync_status(ctx)


@pytest.mark.parametrize("tree", [True, False], ids=["tree", "causal"])
@pytest.mark.parametrize("H,Hk,d,R,lens,cnt", [(4, 1, 64, 16, [100, 0], [45, 31]), (2, 1, 128, 32, [77], [90]), (24, 24, 128, 16, [33, 0], [90, 70]), (40, 20, 64, 64, [20], [44])])
def test_two_tiles_at_a_time_in_float_mode(ghd, H, Hk, d, R, lens, cnt, tree):
    """More than 128 rows a key head, or more than 64 and many heads."""
    su = Setup(ghd, H, Hk, d, "f32", R, lens, cnt, 37 * H + R + len(lens), behind=3)
    vis, words = su.trees() if tree else ([np.ones((n, n), bool) for n in cnt], None)
    check_attention(ghd, su, vis, words)


@pytest.mark.parametrize("path", [0, 1, 2], ids=["auto", "rows", "tcgen05"])
@pytest.mark.parametrize("H,Hk,d,R,lens,cnt", [
    (2, 1, 128, 64, [0], [700]),                                        # a prompt
    (2, 2, 64, 16, [300, 0], [1, 513]),                                 # a prompt beside a token
    (2, 2, 128, 32, [200] + [40 + 7 * i for i in range(31)], [256] + [1] * 31),      # a wide tree beside tokens
    (4, 1, 64, 128, [130, 5, 1000, 0], [300, 1, 0, 33]),
])
def test_long_prompts_and_batches_of_unlike_sequences(ghd, H, Hk, d, R, lens, cnt, path):
    su = Setup(ghd, H, Hk, d, "f16", R, lens, cnt, 41 * H + R + len(lens), behind=2)
    on_path(ghd, su.ctx, path)
    if cnt[0] == 256:
        vis, words = su.trees()
    else:
        vis, words = [np.ones((n, n), bool) for n in cnt], None
    check_attention(ghd, su, vis, words)


@pytest.mark.parametrize("H,Hk,d,lens,cnt", [(2, 1, 128, [0], [600]), (2, 2, 64, [300, 0], [1, 290])])
def test_long_prompts_in_float_mode(ghd, H, Hk, d, lens, cnt):
    su = Setup(ghd, H, Hk, d, "f32", 32, lens, cnt, 43 * H + len(lens), behind=2)
    check_attention(ghd, su, [np.ones((n, n), bool) for n in cnt], None)


@pytest.mark.parametrize("H,Hk,d,n", [(4, 4, 64, 1), (28, 4, 128, 3), (32, 32, 128, 200), (8, 8, 64, 700)])
def test_float_queries_are_rotated_in_64_bits_and_rounded_once(ghd, H, Hk, d, n):
    """Half a step of the result, and what differs between two ways to the angle in 64 bits: positions below 2^18 times a frequency
    that two functions may round apart, 2^18 * 2^-51 with the products of the angle, and 2^-51 for sine, cosine and the two sums."""
    r = np.random.RandomState(d + n)
    ctx = make_ctx(ghd, H, d, "f32")
    R, pages = 64, (n + 63) // 64
    kv = ghd.Kv4Cache(dev(np.arange(pages, dtype=np.int32)[None]), dev(np.zeros(1, np.int32)), R, Hk, pages)
    q, k = r.randn(n, H, d).astype(np.float32), r.randn(n, Hk * d).astype(np.float32)
    pos = r.randint(0, 1 << 18, n).astype(np.int32)
    got = ghd.ghd_kv4_append(ctx, kv, ghd.Kv4Rows(dev(np.array([0, n], np.int32)), n, pos=dev(pos)), ghd.ghd_kv4_pool(ctx, kv)[0], dev(q.reshape(n, -1)), dev(k), dev(k))
    ghd.ghd_sync_status(ctx)
    got = got.double().cpu().numpy().reshape(n, H, d)
    want = np.stack([okv4.rotate(q[i].astype(np.float64), pos[i], THETA) for i in range(n)])
    amp = np.abs(q.astype(np.float64))
    amp = amp + np.concatenate([amp[..., d // 2:], amp[..., : d // 2]], -1)
    assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -32 * amp).all()


@pytest.mark.parametrize("own", [False, True], ids=["by nobody", "by themselves"])
@pytest.mark.parametrize("path,H,Hk,n", [(1, 2, 2, 5), (1, 4, 2, 9), (2, 2, 2, 40), (2, 4, 2, 33)])
def test_values_of_keys_that_a_row_does_not_see_cost_it_no_precision(ghd, path, H, Hk, n, own):
    """New rows 1 and n - 2 are seen by no row, or by themselves alone, and have the largest values there are; all others are near
    0.001.  All scores are equal, so the bound is that of the weights alone: 2^-11 for the weight times scale, 2^-18 for the exponential
    and 32-bit sums of fewer than 128 terms, against codes of at most 8; output half a step of half, 2^-25 below the normal range."""
    d, L = 128, 60
    big = (1, n - 2)
    su = Setup(ghd, H, Hk, d, "f16", 32, [L], [n], 21, garbage=False)
    on_path(ghd, su.ctx, path)
    part = middle = 0.0
    for t in range(L + n):
        page, row = okv4.slots(su.table, 32, 0, t)
        for h in range(Hk):
            c, s, m = okv4.quantise((su.r.randn(d) * (25000.0 if t - L in big else 1e-3)).clip(-65000, 65000).astype(np.float32), "f16")
            su.pool.put(1, page, row, h, c, s, m)
            if t - L not in big:
                part, middle = max(part, 8 * float(s)), max(middle, abs(float(m) + 8 * float(s)))
    su.dpool.copy_(dev(su.pool.data.reshape(-1)))
    vis = [np.ones((n, n), bool)]
    for i in big:
        vis[0][:, i] = False
        vis[0][i, i] = own
    mask = np.zeros((n, 64), np.uint8)
    mask[:, :n] = vis[0]
    words = np.packbits(mask, axis=1, bitorder="little").view(np.int64)
    q = np.zeros((n, H, d), np.float16)
    out = ghd.ghd_kv4_attention(su.ctx, su.kv, ghd.Kv4Rows(dev(su.start), n, mask=dev(words)), su.dpool, dev(q.reshape(n, -1)))
    ghd.ghd_sync_status(su.ctx)
    got = out.double().cpu().numpy().reshape(n, H, d)
    want = okv4.attention(su.pool, su.table, su.lens, su.start, vis, q)
    tol = part * (2.0 ** -11 + 2.0 ** -15) + middle * 2.0 ** -15 + np.maximum(2.0 ** -11 * np.abs(want), 2.0 ** -25)
    small = np.ones(n, bool)
    small[list(big)] = not own
    assert (np.abs(got - want) <= tol)[small].all(), float((np.abs(got - want) / tol)[small].max())
    assert np.isfinite(got).all() and (small.all() or (np.abs(got - want) <= 2.0 ** -9 * np.abs(want).max())[~small].all())
