"""Cases of the operators of a paged key/value cache held in 4 bits.

Four operators work on the same cache: new rows are rotated, quantised and appended; the tree attention reads
the pages; rows come back in the storage type; the rows of an accepted path are committed.  Every case is one of
them at sizes of the 7B / 13B / tiny shapes that the benchmark and the sweeps use, or at grouped heads.

The cache.  A pool is bytes [n_pages][n_kv_heads][block]; a block holds R = page_rows rows:
    K codes [R][d/2] | V codes [R][d/2] | K (scale, min) [R][2] | V (scale, min) [R][2]
with the scales and minima in the storage type.  Channel 2b of a row is the low half of byte b, channel 2b + 1 the
high half; the value of code c is min + scale * c.  Row t of sequence s is row t % R of page table[s][t // R].
Quantising a row of d values x (rounded to 32 bits after the rotation): min = T(lo), scale = T((hi - lo) / 15),
c = round-to-even((x - min) / scale) held in [0, 15]; scale 0 gives code 0.
"""
import math
import random

import numpy as np
import torch

own = False

_THETA = 10000.0
_CTX = {}


# ------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one sequence decodes one token on the 7B shape: latency
        dict(name="append 1 token 7b", op="append", dtype="f16", heads=32, kv_heads=32, dh=128, page=64, seqs=1, rows=1, kv=2048, tree=False),
        # a few drafted trees of the tiny shape in float mode, odd row counts
        dict(name="append trees tiny f32", op="append", dtype="f32", heads=8, kv_heads=8, dh=64, page=32, seqs=5, rows=49, kv=257, tree=True),
        # prompts of a batch imported at once, ragged, grouped heads, small pages
        dict(name="append prompts grouped", op="append", dtype="f16", heads=32, kv_heads=8, dh=128, page=16, seqs=8, rows=2048, kv=0, tree=False),
        # plain decoding of one sequence on the 7B shape
        dict(name="attend 1 token 7b 2048", op="attend", dtype="f16", heads=32, kv_heads=32, dh=128, page=64, seqs=1, rows=1, kv=2048, tree=False),
        # a serving batch of ragged sequences, one token each, grouped heads
        dict(name="attend 32 seqs grouped 8192", op="attend", dtype="f16", heads=32, kv_heads=8, dh=128, page=16, seqs=32, rows=1, kv=8192, tree=False),
        # a batch of verification trees on the 7B shape, up to 64 nodes each, ragged caches
        dict(name="attend 8 trees of 64 7b 8192", op="attend", dtype="f16", heads=32, kv_heads=32, dh=128, page=64, seqs=8, rows=64, kv=8192, tree=True),
        # one wide tree on the 13B shape
        dict(name="attend tree of 256 13b 4096", op="attend", dtype="f16", heads=40, kv_heads=40, dh=128, page=128, seqs=1, rows=256, kv=4096, tree=True),
        # small trees in float mode, odd lengths
        dict(name="attend trees tiny f32", op="attend", dtype="f32", heads=8, kv_heads=8, dh=64, page=32, seqs=4, rows=7, kv=301, tree=True),
        # a few rows looked at again, odd count
        dict(name="read 13 rows 13b", op="read", dtype="f16", heads=40, kv_heads=40, dh=128, page=64, seqs=1, rows=13, kv=512, tree=False),
        # whole sequences leave the cache for one in the storage type
        dict(name="read 8 seqs of 2048 7b", op="read", dtype="f16", heads=32, kv_heads=32, dh=128, page=64, seqs=8, rows=2048, kv=2048, tree=False),
        # one accepted path after a step of the 7B shape, a few layers
        dict(name="commit 1 path 7b", op="commit", dtype="f16", heads=32, kv_heads=32, dh=128, page=64, seqs=1, rows=64, kv=2048, tree=True, layers=4, path=3),
        # accepted paths of a batch in float mode
        dict(name="commit 16 paths f32", op="commit", dtype="f32", heads=8, kv_heads=8, dh=64, page=16, seqs=16, rows=49, kv=257, tree=True, layers=8, path=5),
    ]


_SHAPES = [(32, 32, 128), (40, 40, 128), (32, 8, 128), (28, 4, 128), (8, 8, 64), (12, 4, 64)]


def draw(rng):
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["append", "attend", "attend", "attend", "read", "commit"])
        h, hk, d = rng.choice(_SHAPES)
        c = dict(op=op, dtype=rng.choice(["f16", "f16", "f16", "f32"]), heads=h, kv_heads=hk, dh=d, page=rng.choice([16, 32, 64, 128]), seqs=span(1, 32))
        if op == "append":
            c.update(tree=rng.random() < 0.5, kv=span(1, 8192) - 1)
            c.update(rows=span(1, 256) if c["tree"] else span(1, 2048))
        elif op == "attend":
            c.update(tree=rng.random() < 0.7, kv=span(1, 16384) - 1, rows=span(1, 256))
        elif op == "read":
            c.update(tree=False, kv=span(1, 8192), rows=0)
            c["rows"] = min(c["kv"], span(1, 8192))
        else:
            c.update(tree=True, kv=span(1, 8192) - 1, rows=rng.randint(16, 128), layers=rng.randint(1, 8), path=rng.randint(1, 6))
        w = work(c)
        rows = c["seqs"] * (c["kv"] + c["rows"]) * hk * d                          # values of the cache
        held = c["seqs"] * h * c["rows"] * (c["kv"] + c["rows"])                   # scores that the plain form holds at once
        if w["bytes"] <= 3.2e8 and rows <= 2.7e8 and (op != "attend" or (w["bytes"] <= 1.45e8 and w["flops"] <= 2.3e10 and held <= 2.6e8)):
            return c


# ------------------------------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.float16 if case["dtype"] == "f16" else torch.float32


def _plan(case):
    """Lengths of the sequences, on the host: the longest has what the case says, the others less."""
    S, kv, rows = case["seqs"], case["kv"], case["rows"]
    r = np.random.RandomState(7919 * S + 31 * kv + rows)
    lens = [kv] + [int(x) for x in r.randint(kv // 8, kv + 1, S - 1)]
    if case["op"] == "read":
        cnt = [rows] + [int(x) for x in r.randint(rows // 2, rows + 1, S - 1)]
        cnt = [min(a, b) for a, b in zip(cnt, lens)]
    elif case["op"] == "commit":
        cnt = [rows] * S
    else:
        cnt = [rows] + [int(x) for x in r.randint((rows + 1) // 2, rows + 1, S - 1)]
    if S > 2 and case["op"] != "commit":
        lens[1], cnt[1] = 0, cnt[1] if case["op"] != "read" else 0      # one sequence starts from nothing
    return lens, cnt


def _tree(r, n):
    """Parents of a tree of n nodes (parent[i] < i) and its visibility, bool [n][n]."""
    parent = [-1] + [int(r.randint(max(0, (i - 1) // 4), i)) for i in range(1, n)]
    vis = np.eye(n, dtype=bool)
    depth = np.zeros(n, dtype=np.int64)
    for i in range(1, n):
        vis[i] |= vis[parent[i]]
        depth[i] = depth[parent[i]] + 1
    return vis, depth


def _words(vis, W):
    n = vis.shape[0]
    bits = np.zeros((n, W * 64), dtype=np.uint8)
    bits[:, :n] = vis
    return np.packbits(bits, axis=1, bitorder="little").view(np.int64)


def _fill_pool(pool, case, gen, T):
    """Rows of normal values (the keys with a few strong channels), quantised the way the cache holds them."""
    d, R, es = case["dh"], case["page"], 2 if T == torch.float16 else 4
    n = pool.shape[0]
    strong = torch.exp(0.5 * torch.randn(d, device="cuda", generator=gen))
    step = max(1, (1 << 25) // (case["kv_heads"] * R * d))
    for which in (0, 1):
        for p in range(0, n, step):
            part = pool[p:p + step]
            x = torch.randn(part.shape[0], case["kv_heads"], R, d, device="cuda", generator=gen)
            x = x * strong if which == 0 else x * 0.6 + 0.05
            lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
            mn, sc = lo.to(T), ((hi - lo) / 15).to(T)
            c = ((x - mn.float()) / sc.float()).round().clamp(0, 15).to(torch.uint8)
            part[:, :, which * R * d // 2:(which + 1) * R * d // 2] = (c[..., 0::2] | (c[..., 1::2] << 4)).flatten(2)
            at = R * d + which * 2 * es * R
            part[:, :, at:at + 2 * es * R] = torch.cat((sc, mn), -1).flatten(2).contiguous().view(torch.uint8)


def prepare(case, seed):
    lens, cnt = _plan(case)
    r = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T = _dtype(case)
    S, H, Hk, d, R = case["seqs"], case["heads"], case["kv_heads"], case["dh"], case["page"]
    es = 2 if T == torch.float16 else 4
    block = R * d + 4 * R * es
    extra = 0 if case["op"] == "read" else max(cnt)
    max_pages = (max(a + b for a, b in zip(lens, cnt)) + extra) // R + 1
    n_pages = sum((a + b + R - 1) // R for a, b in zip(lens, cnt)) + 3
    order = r.permutation(n_pages)
    table = np.zeros((S, max_pages), dtype=np.int32)
    at = 0
    for s in range(S):
        k = (lens[s] + cnt[s] + R - 1) // R
        table[s, :k] = order[at:at + k]
        at += k
    layers = case.get("layers", 1)
    pools = torch.zeros(layers, n_pages, Hk, block, dtype=torch.uint8, device="cuda")
    for l in range(layers):
        _fill_pool(pools[l], case, gen, T)
    start = np.concatenate(([0], np.cumsum(cnt)))
    n_rows = int(start[-1])
    dev = lambda a, t: torch.tensor(a, dtype=t, device="cuda")  # noqa: E731
    st = dict(case=case, T=T, pools=pools, table=dev(table, torch.int32), kv_len=dev(lens, torch.int32), start=dev(start, torch.int32),
              n_rows=n_rows, max_len=max(a + b for a, b in zip(lens, cnt)), max_rows=max(cnt), mask=None)
    if case["op"] in ("append", "attend"):
        W = (max(cnt) + 63) // 64
        pos, words = [], []
        for s in range(S):
            if case["tree"]:
                vis, depth = _tree(r, cnt[s])
                pos += list(lens[s] + depth)
                words.append(_words(vis, W))
            else:
                pos += list(range(lens[s], lens[s] + cnt[s]))
        st["pos"] = dev(pos, torch.int32)
        if case["tree"]:
            behind = 3 if case["op"] == "attend" and S > 1 else 0
            st["mask"] = dev(np.concatenate(words + [np.zeros((behind, W), dtype=np.int64)]), torch.int64)
    if case["op"] == "append":       # q, k and v of one projection, side by side
        st["qkv"] = torch.randn(n_rows, (H + 2 * Hk) * d, device="cuda", generator=gen).to(T)
        st["q_out"] = torch.empty(n_rows, H * d, dtype=T, device="cuda")
    if case["op"] == "attend":       # rotated queries; the last rows of the batch belong to nobody
        pad = 3 if S > 1 else 0
        st["q"] = torch.randn(n_rows + pad, H * d, device="cuda", generator=gen).to(T)
        st["out"] = torch.zeros(n_rows + pad, H * d, dtype=T, device="cuda")
        st["n_rows"] = n_rows + pad
    if case["op"] == "read":
        st["first"] = dev([int(r.randint(0, a - b + 1)) for a, b in zip(lens, cnt)], torch.int32)
    if case["op"] == "commit":       # what the acceptance of each tree left: a root path deep in the tree
        m = case["path"]
        res = np.zeros((S, 514), dtype=np.int32)
        for s in range(S):
            res[s, 0], res[s, 1] = m, m + 1
            res[s, 3:3 + m] = np.sort(r.choice(np.arange(m + 1, case["rows"]), m, replace=False))
            res[s, 258:258 + m + 1] = r.randint(0, 1000, m + 1)
        st["results"] = dev(res, torch.int32)
        st["kept"] = dev(np.arange(S + 1) * (m + 1), torch.int32)
    return st


# ------------------------------------------------------------------------------------------------- plain form
def _parts(pool, case, T):
    """Views of a pool: codes [pages][heads][R][d/2] and (scale, min) [pages][heads][R][2], for K and for V."""
    d, R, es = case["dh"], case["page"], 2 if T == torch.float16 else 4
    half = R * d // 2
    codes = [pool[..., i * half:(i + 1) * half].unflatten(-1, (R, d // 2)) for i in (0, 1)]
    par = [pool[..., 2 * half + i * 2 * es * R:2 * half + (i + 1) * 2 * es * R].view(T).unflatten(-1, (R, 2)) for i in (0, 1)]
    return codes, par


def _values(codes, par):
    """Codes [..., d/2] and (scale, min) [..., 2] -> 32-bit values [..., d]."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
    p = par.float()
    return p[..., 1:2] + p[..., 0:1] * c


def _rows_of(start, n):
    """Row numbers 0 .. n - 1 -> (sequence, index in its rows); rows behind the last sequence are clamped to it."""
    i = torch.arange(n, device="cuda", dtype=torch.int32)
    s = (torch.searchsorted(start, i, right=True) - 1).clamp(max=start.numel() - 2)
    return s, i.long() - start[s].long()


def _fetch(pool, case, T, table, s, slot):
    codes, par = _parts(pool, case, T)
    page, r = table[s, slot // case["page"]].long(), slot % case["page"]
    return [_values(codes[i][page, :, r], par[i][page, :, r]) for i in (0, 1)]


def _plain_append(st):
    case, T = st["case"], st["T"]
    H, Hk, d, n = case["heads"], case["kv_heads"], case["dh"], st["n_rows"]
    q, k, v = st["qkv"].split((H * d, Hk * d, Hk * d), 1)
    freq = _THETA ** (torch.arange(d // 2, device="cuda", dtype=torch.float64) * (-2.0 / d))
    ang = st["pos"].double()[:, None, None] * freq
    c, s = ang.cos(), ang.sin()

    def turn(x):
        a, b = x.double().unflatten(1, (-1, 2, d // 2)).unbind(2)
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    st["q_out"].copy_(turn(q).flatten(1))
    seq, i = _rows_of(st["start"], n)
    slot = st["kv_len"][seq].long() + i
    page, r = st["table"][seq, slot // case["page"]].long(), slot % case["page"]
    codes, par = _parts(st["pools"][0], case, T)
    for which, x in enumerate((turn(k).float(), v.float().unflatten(1, (Hk, d)))):
        lo, hi = x.amin(-1, keepdim=True).double(), x.amax(-1, keepdim=True).double()
        mn, sc = lo.to(T), ((hi - lo) / 15).to(T)
        t = (x.double() - mn.double()) / sc.double()
        code = torch.where(sc == 0, torch.zeros_like(t), t).round().clamp(0, 15).to(torch.uint8)
        codes[which][page, :, r] = code[..., 0::2] | (code[..., 1::2] << 4)
        par[which][page, :, r] = torch.cat((sc, mn), -1)
    return [st["q_out"]] + [x.to(T).flatten(1) for x in _fetch(st["pools"][0], case, T, st["table"], seq, slot)]


def _plain_attend(st):
    case, T = st["case"], st["T"]
    H, Hk, d, S = case["heads"], case["kv_heads"], case["dh"], case["seqs"]
    g, L, N = H // Hk, st["max_len"], st["max_rows"]
    kv, start = st["kv_len"].long(), st["start"].long()
    cnt = start[1:] - start[:-1]
    key = torch.arange(L, device="cuda")
    slot = torch.minimum(key[None, :], (kv + cnt - 1).clamp(min=0)[:, None])
    K, V = _fetch(st["pools"][0], case, T, st["table"], torch.arange(S, device="cuda")[:, None].expand(S, L), slot)      # [S, L, Hk, d]
    row = torch.arange(N, device="cuda")
    live = row[None, :] < cnt[:, None]                                              # [S, N]
    at = (start[:-1, None] + row[None, :]).clamp(max=st["n_rows"] - 1)
    q = st["q"][at].float().view(S, N, Hk, g, d).permute(0, 2, 1, 3, 4).reshape(S, Hk, N * g, d)
    w = torch.matmul(q, K.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))               # [S, Hk, N g, L]
    j = (key[None, :] - kv[:, None])                                                # [S, L]: number among the new rows
    see = (j[:, None, :] >= 0) & (j[:, None, :] <= row[None, :, None])              # [S, N, L]
    if st["mask"] is not None:
        m = st["mask"][at]                                                          # [S, N, W]
        jj = j.clamp(0, m.shape[2] * 64 - 1)[:, None, :].expand(S, N, L)
        see = see & (((m.gather(2, jj >> 6) >> (jj & 63)) & 1) == 1)
    see = (see | (j[:, None, :] < 0)) & (j[:, None, :] < cnt[:, None, None])
    see = see[:, None, :, None, :].expand(S, Hk, N, g, L).reshape(S, Hk, N * g, L)
    w = torch.where(see, w, -math.inf)
    top = w.amax(-1, keepdim=True)
    w = torch.exp(w - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w, V.permute(0, 2, 1, 3)) / torch.where(total == 0, 1.0, total)
    o = o.view(S, Hk, N, g, d).permute(0, 2, 1, 3, 4).reshape(S * N, H * d)
    live = live.reshape(-1)
    st["out"][at.reshape(-1)[live]] = o[live].to(T)
    return st["out"]


def _plain_read(st):
    seq, i = _rows_of(st["start"], st["n_rows"])
    return [x.to(st["T"]).flatten(1) for x in _fetch(st["pools"][0], st["case"], st["T"], st["table"], seq, st["first"][seq].long() + i)]


def _plain_commit(st):
    case, T, m = st["case"], st["T"], st["case"]["path"]
    S, R = case["seqs"], case["page"]
    seq = torch.arange(S, device="cuda")[:, None].expand(S, m + 1)
    kv = st["kv_len"].long()[:, None]
    src, dst = kv + st["results"][:, 2:3 + m].long(), kv + torch.arange(m + 1, device="cuda")
    ps, rs, pd, rd = st["table"][seq, src // R].long(), src % R, st["table"][seq, dst // R].long(), dst % R
    codes, par = _parts(st["pools"], case, T)
    for x in codes + par:
        x[:, pd, :, rd] = x[:, ps, :, rs]
    new_len = st["kv_len"] + st["results"][:, 0] + 1
    got = [_values(codes[i][:, pd, :, rd], par[i][:, pd, :, rd]) for i in (0, 1)]       # [S, m + 1, layers, Hk, d]
    return [new_len] + [[x.to(T) for x in y.permute(2, 0, 1, 3, 4).reshape(case["layers"], S * (m + 1), -1)] for y in got]


# ------------------------------------------------------------------------------------------------- the framework's operators
def _ctx(case):
    """The context a program keeps for its model shape."""
    import paper_2505_23219_b200 as ghd
    key = (case["heads"], case["dh"], case["dtype"])
    if key not in _CTX:
        _CTX[key] = ghd.ghd_create(ghd.ModelCfg(case["heads"] * case["dh"], case["heads"], case["dh"], 256, 1000, 1, 4096, 256, case["dtype"], 1e-6, _THETA))
    return ghd, _CTX[key]


def _own(st):
    case = st["case"]
    ghd, ctx = _ctx(case)
    if case["op"] == "commit":
        kv_len = st["kv_len"].clone()
        kv = ghd.Kv4Cache(st["table"], kv_len, case["page"], case["kv_heads"], st["pools"].shape[1])
        ghd.ghd_kv4_commit(ctx, kv, ghd.Kv4Rows(st["start"], st["n_rows"]), st["pools"], st["results"])
        back = [ghd.ghd_kv4_read(ctx, kv, p, st["kept"], case["seqs"] * (case["path"] + 1), first=st["kv_len"]) for p in st["pools"]]
        return [kv_len, [k for k, _ in back], [v for _, v in back]]
    kv = ghd.Kv4Cache(st["table"], st["kv_len"], case["page"], case["kv_heads"], st["pools"].shape[1])
    pool = st["pools"][0]
    if case["op"] == "read":
        return list(ghd.ghd_kv4_read(ctx, kv, pool, st["start"], st["n_rows"], first=st["first"]))
    rows = ghd.Kv4Rows(st["start"], st["n_rows"], pos=st["pos"] if case["op"] == "append" else None, mask=st["mask"])
    if case["op"] == "attend":
        return ghd.ghd_kv4_attention(ctx, kv, rows, pool, st["q"], out=st["out"])
    H, Hk, d = case["heads"], case["kv_heads"], case["dh"]
    q, k, v = st["qkv"].split((H * d, Hk * d, Hk * d), 1)
    ghd.ghd_kv4_append(ctx, kv, rows, pool, q, k, v, q_out=st["q_out"])
    return [st["q_out"]] + list(ghd.ghd_kv4_read(ctx, kv, pool, st["start"], st["n_rows"], first=st["kv_len"]))


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "attend": _plain_attend, "read": _plain_read, "commit": _plain_commit}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------- bytes and operations
def work(case):
    """Each input read once, each output written once; the attention's products over the rows it may see."""
    lens, cnt = _plan(case)
    es = 2 if case["dtype"] == "f16" else 4
    H, Hk, d, n = case["heads"], case["kv_heads"], case["dh"], sum(cnt)
    row4 = Hk * (d + 4 * es)                       # K and V of one row in the cache: codes, scales and minima
    rowT = 2 * Hk * d * es                         # ... in the storage type
    if case["op"] == "append":                     # q in and out, k and v in, the cache rows out; and the rows read back
        return {"bytes": n * (2 * H * d * es + rowT + row4 + row4 + rowT), "flops": n * (6 * (H + Hk) * d + 8 * Hk * d)}
    if case["op"] == "read":
        return {"bytes": n * (row4 + rowT), "flops": n * 4 * Hk * d}
    if case["op"] == "commit":
        moved, kept = case["seqs"] * case["path"] * case["layers"], case["seqs"] * (case["path"] + 1) * case["layers"]
        return {"bytes": 2 * moved * row4 + kept * (row4 + rowT), "flops": kept * 4 * Hk * d}
    nbytes = sum(a + b for a, b in zip(lens, cnt)) * row4 + 2 * n * H * d * es
    pairs = sum(b * a + b * (b + 1) // 2 for a, b in zip(lens, cnt))
    return {"bytes": nbytes, "flops": 4 * pairs * H * d}


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_rows(pool, case, T, pages, rows):
    """K and V of the given (page, row) places, one list entry each, in 64 bits: [n][heads][d]."""
    d, R, es = case["dh"], case["page"], 2 if T == torch.float16 else 4
    blocks = pool[pages.long()]                                                       # [n][heads][block]
    n, heads = blocks.shape[:2]
    r = rows.long()
    out = []
    for which in (0, 1):
        byte_at = which * R * d // 2 + r[:, None] * (d // 2) + torch.arange(d // 2, device="cuda")
        b = torch.gather(blocks, 2, byte_at[:, None, :].expand(n, heads, d // 2))
        x = torch.empty(n, heads, d, dtype=torch.float64, device="cuda")
        x[:, :, 0::2] = (b % 16).double()
        x[:, :, 1::2] = torch.div(b, 16, rounding_mode="floor").double()
        p_at = R * d + which * 2 * es * R + r[:, None] * 2 * es + torch.arange(2 * es, device="cuda")
        p = torch.gather(blocks, 2, p_at[:, None, :].expand(n, heads, 2 * es)).contiguous().view(T).double()
        out.append(x * p[:, :, :1] + p[:, :, 1:])
    return out


def _exact_seq(st, pool, s, slots):
    R = st["case"]["page"]
    page = st["table"][s].long()[torch.div(slots, R, rounding_mode="floor")]
    parts = [_exact_rows(pool, st["case"], st["T"], page[i:i + 512], (slots % R)[i:i + 512]) for i in range(0, slots.numel(), 512)]
    return [torch.cat(x) for x in zip(*parts)]


def exact(case, seed):
    st = prepare(case, seed)
    T, H, Hk, d = st["T"], case["heads"], case["kv_heads"], case["dh"]
    start, lens = st["start"].tolist(), st["kv_len"].tolist()
    arange = lambda a, b: torch.arange(a, b, device="cuda")  # noqa: E731
    if case["op"] == "read":
        first = st["first"].tolist()
        got = [_exact_seq(st, st["pools"][0], s, arange(first[s], first[s] + start[s + 1] - start[s])) for s in range(case["seqs"]) if start[s + 1] > start[s]]
        return [torch.cat([x[i] for x in got]).flatten(1) for i in (0, 1)]
    if case["op"] == "commit":
        m, res = case["path"], st["results"].tolist()
        back = [[], []]
        for pool in st["pools"]:
            got = [_exact_seq(st, pool, s, lens[s] + torch.tensor(res[s][2:3 + m], device="cuda")) for s in range(case["seqs"])]
            for i in (0, 1):
                back[i].append(torch.cat([x[i] for x in got]).flatten(1))
        return [torch.tensor([a + m + 1 for a in lens], dtype=torch.int32, device="cuda")] + back
    if case["op"] == "append":
        n = st["n_rows"]
        x = st["qkv"].double().view(n, H + 2 * Hk, d)
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                        st["pos"].double()[:, None] * torch.pow(torch.tensor(_THETA, dtype=torch.float64, device="cuda"), arange(0, d // 2).double() / (-d / 2)))
        rot = torch.complex(x[:, :H + Hk, :d // 2], x[:, :H + Hk, d // 2:]) * z[:, None, :]
        rot = torch.cat((rot.real, rot.imag), 2)
        out = [rot[:, :H].flatten(1)]
        for y in (rot[:, H:].float().double(), x[:, H + Hk:]):          # the codes are those of values rounded to 32 bits
            low, high = y.min(2, keepdim=True).values, y.max(2, keepdim=True).values
            scale = torch.div(high - low, 15.0).to(T).double()
            low = low.to(T).double()
            code = torch.where(scale > 0, torch.round((y - low) / scale), torch.zeros((), dtype=torch.float64, device="cuda"))
            out.append((low + scale * torch.minimum(torch.maximum(code, torch.zeros_like(code)), torch.full_like(code, 15.0))).flatten(1))
        return out
    out = st["out"].double()
    g = H // Hk
    for s in range(case["seqs"]):
        a, n = lens[s], start[s + 1] - start[s]
        if n == 0:
            continue
        K, V = _exact_seq(st, st["pools"][0], s, arange(0, a + n))
        see = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        if st["mask"] is not None:
            bits = st["mask"][start[s]:start[s] + n].cpu().numpy().view(np.uint8)
            see &= torch.tensor(np.unpackbits(bits, axis=1, bitorder="little")[:, :n] != 0, device="cuda")
        see = torch.cat((torch.ones(n, a, dtype=torch.bool, device="cuda"), see), 1)
        q = st["q"][start[s]:start[s] + n].double().view(n, H, d)
        for h in range(H):
            p = torch.softmax((q[:, h] @ K[:, h // g].T / math.sqrt(d)).masked_fill(~see, -math.inf), 1)
            out[start[s]:start[s] + n, h * d:(h + 1) * d] = p @ V[:, h // g]
    return out


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(k)) for k in range(6)]:
        print(c.get("name", "drawn"), work(c), {k: v for k, v in c.items() if k != "name"})
