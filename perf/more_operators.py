"""Cases of two pairs of operators: weights in microscaled 4-bit floating point and their product, and drafting and
verifying tokens by sampling from given random numbers.

Matrices in 4 bits.  A matrix [m][k] is held in tiles of 128 x 128 (m and k rounded up, zeros behind them):
    codes  [m/128][k/128][128 rows][64 bytes], element 2b of a row in the low half of byte b, element 2b + 1 in the high half;
    scales [m/128][k/128][512]: byte (r % 32) * 16 + (r / 32) * 4 + j is that of row r, elements 32 j .. 32 j + 31.
A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; a scale byte s stands for 2^(s - 127), 255 for NaN.  Quantising 32 elements:
    E = floor(log2(largest magnitude)) - 2, -127 at least (-127 for zeros), code = x / 2^E rounded to the nearest (ties to the even
    code) and held within +-6.

Sampling.  w_s = exp(l_s / temperature) over a row of logits (-inf: not in the distribution).
Draws without replacement: draw j is the first token t whose running sum of the weights not yet drawn exceeds u_j times their total.
Verification walks a tree from its root.  P: the node's distribution, Q: the one that its children were drawn from.  Children in order:
    accepted if u Q(x) < P(x); otherwise P <- max(P - Q, 0) / its sum, Q <- Q without x / its sum.
    Candidates that nobody drew: accepted if u < P(x), otherwise P <- P without x / its sum.
When no child is left the last token is drawn from P with the root's random number.
"""
import math
import random

import numpy as np
import torch

own = False

_CTX = {}
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the gate and up weights of a 13B layer are laid out when the model is loaded (the largest matrix of a layer)
        dict(name="quantise 13b gate up", op="quantise", dtype="f16", m=27648, k=5120),
        # an odd matrix in float mode: rows and columns that fill no tile
        dict(name="quantise odd f32", op="quantise", dtype="f32", m=1000, k=1376),
        # one token through a square projection of the 7B shape: latency
        dict(name="product 1 row 7b", op="product", dtype="f16", n=1, m=4096, k=4096),
        # a small tree's logits (lm_head of the 7B shape)
        dict(name="product 16 rows lm_head 7b", op="product", dtype="f16", n=16, m=32000, k=4096),
        # a tree of 64 nodes through the projection out of the MLP
        dict(name="product 64 rows down 7b", op="product", dtype="f16", n=64, m=4096, k=11008),
        # float mode, tiny shape, odd row count
        dict(name="product 49 rows tiny f32", op="product", dtype="f32", n=49, m=1000, k=512),
        # the first half of the MLP with its activation: a tree of 64 nodes on the 7B shape
        dict(name="gate up 64 rows 7b", op="gate_up", dtype="f16", n=64, m=11008, k=4096),
        # ... and the widest tree on the 13B shape
        dict(name="gate up 256 rows 13b", op="gate_up", dtype="f16", n=256, m=13824, k=5120),
        # five drafting heads of one sequence, ten candidates each
        dict(name="draw 10 of 5 heads", op="draw", rows=5, vocab=32000, draws=10, temp=0.8),
        # the heads of a batch of sequences
        dict(name="draw 4 of 320 heads", op="draw", rows=320, vocab=32000, draws=4, temp=1.0),
        # one tree of 64 nodes whose candidates were drawn
        dict(name="verify 1 tree of 64", op="verify", seqs=1, nodes=64, vocab=32000, temp=0.8, drawn=True),
        # a batch of ragged trees, candidates not drawn (the heads' best)
        dict(name="verify 48 trees of 64", op="verify", seqs=48, nodes=64, vocab=32000, temp=1.0, drawn=False),
    ]


def draw(rng):
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["quantise", "product", "product", "gate_up", "draw", "verify", "verify"])
        c = dict(op=op)
        if op == "quantise":
            c.update(dtype=rng.choice(["f16", "f16", "f32"]), m=span(64, 32768), k=span(64, 16384))
            if c["m"] * c["k"] > 14e7 or (c["dtype"] == "f32" and c["m"] * c["k"] > 7e7):
                continue
        elif op in ("product", "gate_up"):
            c.update(dtype=rng.choice(["f16", "f16", "f16", "f32"]), n=span(1, 256), m=span(64, 32768), k=span(64, 14336))
            if rng.random() < 0.5:                          # whole tiles, as most models have
                c.update(m=-(-c["m"] // 128) * 128, k=-(-c["k"] // 128) * 128)
            if c["m"] * c["k"] > (7e7 if op == "gate_up" else 14e7) or (c["dtype"] == "f32" and c["n"] * c["m"] * c["k"] > 4e9):
                continue
        elif op == "draw":
            c.update(rows=span(1, 400), vocab=span(300, 131072), draws=rng.randint(1, 16), temp=rng.choice([0.5, 0.8, 1.0, 1.3]))
            if c["rows"] * c["vocab"] > 1e7:
                continue
        else:
            c.update(seqs=span(1, 64), nodes=span(1, 256), vocab=span(300, 131072), temp=rng.choice([0.5, 0.8, 1.0, 1.3]), drawn=rng.random() < 0.6)
            if c["seqs"] * c["nodes"] * c["vocab"] > 9e7:
                continue
        return c


# ------------------------------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.float16 if case["dtype"] == "f16" else torch.float32


def _up(x):
    return -(-x // 128) * 128


def _blocks(x):
    """[m][k] -> 32-bit [m/128 up][k/128 up ...] rows of 32 elements: [M][K/32][32]."""
    m, k = x.shape
    return torch.nn.functional.pad(x.float(), (0, _up(k) - k, 0, _up(m) - m)).unflatten(1, (-1, 32))


def _quantise(x):
    """-> codes uint8 [M][K/32][32] and scale bytes uint8 [M][K/32]."""
    b = _blocks(x)
    top = b.abs().amax(-1)
    E = torch.where(top == 0, -127, (torch.frexp(top)[1] - 3).clamp(min=-127))
    t = torch.ldexp(b.double(), -E[..., None]).float()
    a = t.abs()
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5).byte())
    return code | (torch.signbit(t).byte() << 3), torch.where(torch.isfinite(top), E + 127, 255).to(torch.uint8)


def _tiled(code, scale):
    M, KB = scale.shape
    c = code.flatten(1)
    c = (c[:, 0::2] | (c[:, 1::2] << 4)).view(M // 128, 128, KB // 4, 64).transpose(1, 2).contiguous()
    s = scale.view(M // 128, 4, 32, KB // 4, 4).permute(0, 3, 2, 1, 4).contiguous()
    return c, s.flatten(2)


def _weights(gen, m, k):
    """A matrix as a model's are, held in 4 bits: normal, with rows and columns of unlike strength."""
    M, K = _up(m), _up(k)
    codes = torch.empty(M // 128, K // 128, 128, 64, dtype=torch.uint8, device="cuda")
    scales = torch.empty(M // 128, K // 128, 512, dtype=torch.uint8, device="cuda")
    cols = torch.exp(0.3 * torch.randn(k, device="cuda", generator=gen)) / math.sqrt(k)
    step = 128 * max(1, (1 << 25) // (128 * K))
    for r in range(0, m, step):
        rows = min(step, m - r)
        w = torch.randn(rows, k, device="cuda", generator=gen) * cols * torch.exp(0.2 * torch.randn(rows, 1, device="cuda", generator=gen))
        c, s = _tiled(*_quantise(w))
        codes[r // 128:r // 128 + c.shape[0]], scales[r // 128:r // 128 + c.shape[0]] = c, s
    return codes, scales


def _parents(r, n):
    """A tree of n nodes: parent[i] < i, and its depths."""
    parent, depth = [-1], [0]
    for i in range(1, n):
        p = int(r.randint(max(0, (i - 1) // 5), max(1, (i + 1) // 2)))
        parent.append(p)
        depth.append(depth[p] + 1)
    return parent, depth


def _logits(rows, vocab, randn, rand):
    """Rows as a model's are: most tokens far below two dozen that hold nearly all of the probability."""
    x = 1.5 * randn(rows, vocab)
    strong = max(1, min(24, vocab // 8))
    return x.scatter_add_(1, (rand(rows, strong) * vocab).long().clamp(max=vocab - 1), 8 + 6 * rand(rows, strong))


def _trees(case):
    """The trees of a case, on the host: the first has all nodes, the others some of them."""
    r = np.random.RandomState(7919 * case["seqs"] + 31 * case["nodes"] + case["vocab"])
    cnt = [case["nodes"]] + [int(x) for x in r.randint((case["nodes"] + 1) // 2, case["nodes"] + 1, case["seqs"] - 1)]
    return cnt, [_parents(r, n) for n in cnt]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    rand = lambda *s: torch.rand(*s, device="cuda", generator=gen)  # noqa: E731
    st = dict(case=case)
    if case["op"] in ("quantise", "product", "gate_up"):
        T = st["T"] = _dtype(case)
    if case["op"] == "quantise":
        m, k = case["m"], case["k"]
        st["x"] = torch.empty(m, k, dtype=T, device="cuda")
        cols = torch.exp(0.3 * randn(k)) / math.sqrt(k)
        for r in range(0, m, 2048):
            st["x"][r:r + 2048] = randn(min(2048, m - r), k) * cols
        st["codes"] = torch.zeros(_up(m) // 128, _up(k) // 128, 128, 64, dtype=torch.uint8, device="cuda")
        st["scales"] = torch.zeros(_up(m) // 128, _up(k) // 128, 512, dtype=torch.uint8, device="cuda")
        st["out"] = torch.empty(m, k, dtype=T, device="cuda")
    elif case["op"] == "product":
        st["w"] = [_weights(gen, case["m"], case["k"])]
        st["x"] = (randn(case["n"], case["k"]) * torch.exp(0.5 * randn(case["k"]))).to(T)       # a few strong channels
        st["out"] = torch.empty(case["n"], case["m"], dtype=torch.float32, device="cuda")
    elif case["op"] == "gate_up":
        st["w"] = [_weights(gen, case["m"], case["k"]) for _ in range(2)]
        st["x"] = (randn(case["n"], case["k"]) * torch.exp(0.5 * randn(case["k"]))).to(T)
        st["out"] = torch.empty(case["n"], case["m"], dtype=T, device="cuda")
    elif case["op"] == "draw":
        st["logits"] = _logits(case["rows"], case["vocab"], randn, rand)
        st["u"] = rand(case["rows"], 16)
        st["out"] = torch.full((case["rows"], 16), -1, dtype=torch.int32, device="cuda")
    else:
        _prepare_trees(st, case, seed, randn, rand)
    return st


def _prepare_trees(st, case, seed, randn, rand):
    """Trees whose nodes on one level share candidates: the best of the level's draft distribution, or draws from it."""
    S, V = case["seqs"], case["vocab"]
    cnt, trees = _trees(case)
    deep = max(max(d) for _, d in trees)
    wide = 1
    parent, level, rank, seq = [], [], [], []
    for s, (p, d) in enumerate(trees):
        seen = {}
        for i, x in enumerate(p):
            parent.append(x)
            level.append(d[i])
            rank.append(seen.get(x, 0))
            seen[x] = seen.get(x, 0) + 1
            seq.append(s)
        wide = max(wide, max(seen[x] for x in seen))
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    lv, rk, sq = dev(level).long(), dev(rank).long(), dev(seq).long()
    draft = _logits(S * (deep + 1), V, randn, rand)
    row = sq * (deep + 1) + lv                                  # the draft row that a node's children come from
    wide = min(wide, V)
    if case["drawn"]:
        best = torch.argsort(draft / case["temp"] - torch.log(-torch.log(rand(S * (deep + 1), V).double().clamp(1e-12, 1 - 1e-12))).float(), 1, descending=True)[:, :wide]
    else:
        best = torch.topk(draft, wide, 1).indices
    n = len(parent)
    logits = torch.empty(n, V, device="cuda")
    for r in range(0, n, 512):
        at = row[r:r + 512]
        logits[r:r + 512] = 0.95 * draft[at] + 0.7 * randn(at.numel(), V)
    up = torch.where(lv > 0, row - 1, 0)
    st["tokens"] = best[up, rk.clamp(max=wide - 1)].int()
    st.update(parent=dev(parent), logits=logits, draft=draft, draft_row=row.int(), u=rand(n), start=dev(np.concatenate(([0], np.cumsum(cnt)))), n_rows=n,
              deep=deep, wide=wide, out=torch.full((S, 514), -1, dtype=torch.int32, device="cuda"))


# ------------------------------------------------------------------------------------------------- plain form
def _values(codes, scales):
    """The tiles -> 32-bit values [M][K]."""
    mt, kt = codes.shape[:2]
    c = codes.transpose(1, 2).reshape(mt * 128, kt * 64)
    c = torch.stack((c & 15, c >> 4), -1).flatten(1)
    s = scales.view(mt, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(mt * 128, kt * 4)
    table = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device="cuda")
    scale = torch.where(s == 255, math.nan, torch.ldexp(torch.ones((), device="cuda"), s.int() - 127))
    return (table[c.int()].unflatten(1, (-1, 32)) * scale[..., None]).flatten(1)


def _plain_quantise(st):
    m, k = st["x"].shape
    st["codes"], st["scales"] = _tiled(*_quantise(st["x"]))
    return _values(st["codes"], st["scales"])[:m, :k].to(st["T"])


def _plain_product(st):
    case = st["case"]
    y = [torch.matmul(st["x"].float(), _values(*w)[:case["m"], :case["k"]].T) for w in st["w"]]
    if case["op"] == "product":
        return y[0]
    return (y[0] / (1 + torch.exp(-y[0])) * y[1]).to(st["T"])


def _first_over(w, u):
    """Per row: the first place whose running sum exceeds u times the total; the last one with weight where rounding leaves none."""
    run = w.cumsum(-1)
    t = (run <= u[:, None] * run[:, -1:]).sum(-1)
    last = w.shape[-1] - 1 - (w.flip(-1) > 0).int().argmax(-1)
    return torch.minimum(t, last)


def _plain_draw(st):
    case = st["case"]
    z = st["logits"].double() / case["temp"]
    w = torch.exp(z - z.amax(-1, keepdim=True))
    out = torch.full_like(st["out"], -1)
    for j in range(case["draws"]):
        t = _first_over(w, st["u"][:, j].double())
        out[:, j] = torch.where(w.sum(-1) > 0, t, -1)
        w = w.scatter(1, t[:, None], 0.0)
    return out


def _plain_verify(st):
    case, n = st["case"], st["n_rows"]
    start, parent, u = st["start"].long(), st["parent"].long(), st["u"].double()
    S = start.numel() - 1
    rows = torch.arange(n, device="cuda")
    seq = torch.searchsorted(start, rows, right=True) - 1
    up = torch.where(parent < 0, n, start[seq] + parent)                     # the parent's row; n: none
    order = torch.argsort(up, stable=True)                                   # children of one node side by side, in order
    first = torch.searchsorted(up[order], torch.arange(n + 1, device="cuda"))
    first = torch.cat((first, first.new_full((1,), n)))
    P_of = lambda x, t: torch.softmax(x.double() / t, -1)  # noqa: E731
    at, live = start[:-1].clone(), start[1:] > start[:-1]
    at = at.clamp(max=n - 1)
    out = torch.full_like(st["out"], -1)
    out[:, 0], out[:, 1] = 0, live.int()
    out[:, 2] = torch.where(live, 0, -1)
    ids = torch.arange(S, device="cuda")
    left = P_of(st["logits"][at], case["temp"])
    for level in range(st["deep"] + 1):
        P = P_of(st["logits"][at], case["temp"])
        Q = P_of(st["draft"][st["draft_row"][at].long()], case["temp"]) if case["drawn"] else None
        moved = torch.zeros_like(live)
        nxt = at.clone()
        for j in range(st["wide"]):
            have = live & ~moved & (first[at] + j < first[at + 1])
            child = order[torch.where(have, first[at] + j, 0)]
            x = st["tokens"][child].long()
            p = P[ids, x]
            q = Q[ids, x] if case["drawn"] else torch.ones_like(p)
            ok = have & (q > 0) & (u[child] * q < p)
            no = have & ~ok & ((q > 0) if case["drawn"] else (p > 0))
            nxt = torch.where(ok, child, nxt)
            moved = moved | ok
            rest = torch.clamp(P - Q, min=0) if case["drawn"] else P.scatter(1, x[:, None], 0.0)
            total = rest.sum(-1, keepdim=True)
            P = torch.where((no[:, None]) & (total > 0), rest / total, P)
            if case["drawn"]:
                rest = Q.scatter(1, x[:, None], 0.0)
                total = rest.sum(-1, keepdim=True)
                Q = torch.where(no[:, None] & (total > 0), rest / total, torch.where(no[:, None], 0.0, Q))
        ended = live & ~moved
        left = torch.where(ended[:, None], P, left)
        m = out[:, 0].long()
        out[ids, 3 + m] = torch.where(moved, (nxt - start[:-1]).int(), out[ids, 3 + m])
        out[ids, 258 + m] = torch.where(moved, st["tokens"][nxt], out[ids, 258 + m])
        out[:, 0] += moved.int()
        out[:, 1] += moved.int()
        at, live = torch.where(moved, nxt, at), moved
    last = _first_over(left, u[start[:-1].clamp(max=n - 1)])
    m = out[:, 0].long()
    out[ids, 258 + m] = torch.where(start[1:] > start[:-1], last.int(), -1)
    return out


# ------------------------------------------------------------------------------------------------- the framework's operators
def _ctx(case):
    """The context a program keeps for its model shape."""
    import paper_2505_23219_b200 as ghd
    if case["op"] in ("quantise", "product", "gate_up"):
        key = (case["dtype"], _up(case["k"]), case.get("n", 1))
        make = lambda: ghd.ModelCfg(512, 4, 128, _up(case["k"]), 1000, 1, 512, case.get("n", 1), case["dtype"])  # noqa: E731
    else:
        key = case["vocab"]
        make = lambda: ghd.ModelCfg(512, 4, 128, 512, case["vocab"], 1, 512, 1, "f16")  # noqa: E731
    if key not in _CTX:
        _CTX[key] = ghd.ghd_create(make())
    return ghd, _CTX[key]


def _own(st):
    case = st["case"]
    ghd, ctx = _ctx(case)
    if case["op"] == "quantise":
        if "held" not in st:
            st["held"] = ghd.Mx4(st["codes"], st["scales"], case["m"], case["k"])
        ghd.ghd_mx4_quantize(ctx, st["x"], st["held"])
        return ghd.ghd_mx4_read(ctx, st["held"], out=st["out"])
    if case["op"] in ("product", "gate_up"):
        if "held" not in st:
            st["held"] = [ghd.Mx4(c, s, case["m"], case["k"]) for c, s in st["w"]]
        if case["op"] == "product":
            return ghd.ghd_mx4_linear(ctx, st["x"], st["held"][0], y=st["out"])
        return ghd.ghd_mx4_gate_up(ctx, st["x"], *st["held"], u=st["out"])
    if case["op"] == "draw":
        return ghd.ghd_draft_sample(ctx, st["logits"], st["u"], case["draws"], case["temp"], cand=st["out"])
    if "held" not in st:
        more = dict(draft_logits=st["draft"], draft_row=st["draft_row"], draft_temperature=case["temp"]) if case["drawn"] else {}
        st["held"] = ghd.SampledRows(st["parent"], st["tokens"], st["logits"], st["u"], row_start=st["start"], temperature=case["temp"], **more)
    return ghd.ghd_accept_sampled(ctx, st["held"], out=st["out"])


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_quantise(state) if op == "quantise" else _plain_draw(state) if op == "draw" else _plain_verify(state) if op == "verify" else _plain_product(state)


# ------------------------------------------------------------------------------------------------- bytes and operations
def work(case):
    """Each input read once, each output written once."""
    es = 2 if case.get("dtype") == "f16" else 4
    if case["op"] == "quantise":        # the matrix in, codes and scales out; and the values they stand for
        mk = case["m"] * case["k"]
        return {"bytes": mk * 2 * es + mk * 17 // 16, "flops": 4 * mk}
    if case["op"] in ("product", "gate_up"):
        n, m, k, two = case["n"], case["m"], case["k"], 2 if case["op"] == "gate_up" else 1
        return {"bytes": two * m * k * 17 // 32 + n * k * es + n * m * (4 if two == 1 else es), "flops": 2 * two * n * m * k}
    if case["op"] == "draw":
        return {"bytes": case["rows"] * (case["vocab"] * 4 + 128), "flops": 4 * case["rows"] * case["vocab"]}
    # at the least the root's row, and the one that its children come from; further rows only where a child is accepted
    rows = case["seqs"] * (2 if case["drawn"] else 1)
    return {"bytes": rows * case["vocab"] * 4 + case["seqs"] * (case["nodes"] * 12 + 514 * 4), "flops": 4 * rows * case["vocab"]}


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_matrix(codes, scales, m, k):
    """Element by element from where the layout puts it, in 64 bits."""
    r, c = torch.arange(m, device="cuda")[:, None], torch.arange(k, device="cuda")[None, :]
    kt = codes.shape[1]
    out = torch.empty(m, k, dtype=torch.float64, device="cuda")
    levels = torch.tensor(_LEVELS, dtype=torch.float64, device="cuda")
    for a in range(0, m, 1024):
        rr = r[a:a + 1024]
        tile = torch.div(rr, 128, rounding_mode="floor") * kt + torch.div(c, 128, rounding_mode="floor")
        in_row, in_col = rr % 128, c % 128
        byte = codes.view(-1)[tile * 8192 + in_row * 64 + torch.div(in_col, 2, rounding_mode="floor")].long()
        nib = torch.where(in_col % 2 == 1, byte // 16, byte % 16)
        s = scales.view(-1)[tile * 512 + (in_row % 32) * 16 + torch.div(in_row, 32, rounding_mode="floor") * 4 + torch.div(in_col, 32, rounding_mode="floor")].double()
        out[a:a + 1024] = levels[nib % 8] * torch.where(nib >= 8, -1.0, 1.0) * torch.pow(2.0, s - 127)
    return out


def _exact_verify(st):
    """One sequence after the other, the distributions written out, on the host."""
    case = st["case"]
    start, parent, tokens, u = (st[x].tolist() for x in ("start", "parent", "tokens", "u"))
    out = np.full((len(start) - 1, 514), -1, dtype=np.int32)

    def dist(row):
        z = row.double().cpu().numpy() / case["temp"]
        e = np.exp(z - z.max())
        return e / math.fsum(e)

    for s in range(len(start) - 1):
        a, b = start[s], start[s + 1]
        if a == b:
            out[s, 0] = out[s, 1] = 0
            continue
        at, nodes, toks = a, [0], []
        while True:
            p = dist(st["logits"][at])
            q = dist(st["draft"][int(st["draft_row"][at])]) if case["drawn"] else None
            step = None
            for c in range(at + 1, b):
                if parent[c] != at - a:
                    continue
                x = tokens[c]
                if q is None:
                    if u[c] < p[x]:
                        step = c
                        break
                    if p[x] > 0:
                        p[x] = 0
                        p = p / p.sum()
                elif q[x] > 0:
                    if u[c] * q[x] < p[x]:
                        step = c
                        break
                    p = np.maximum(p - q, 0)
                    p = p / p.sum()
                    q[x] = 0
                    q = q / q.sum() if q.sum() > 0 else q
            if step is None:
                run = np.cumsum(p)
                toks.append(min(int(np.sum(run <= u[a] * run[-1])), int(np.flatnonzero(p)[-1])))
                break
            nodes.append(step - a)
            toks.append(tokens[step])
            at = step
        out[s, 0], out[s, 1] = len(nodes) - 1, len(nodes)
        out[s, 2:2 + len(nodes)] = nodes
        out[s, 258:258 + len(toks)] = toks
    return torch.tensor(out, device="cuda")


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "quantise":
        m, k = case["m"], case["k"]
        out = torch.empty(m, k, dtype=torch.float64, device="cuda")
        level = torch.tensor(_LEVELS, dtype=torch.float64, device="cuda")
        half = (level[1:] + level[:-1]) / 2
        for a in range(0, m, 1024):
            x = torch.nn.functional.pad(st["x"][a:a + 1024].double(), (0, -k % 32)).unflatten(1, (-1, 32))
            top = x.abs().max(-1, keepdim=True).values
            E = torch.floor(torch.log2(top.clamp(min=2.0 ** -126)))
            E = torch.where(torch.pow(2.0, E) > top, E - 1, torch.where(torch.pow(2.0, E + 1) <= top, E + 1, E)) - 2
            unit = torch.pow(2.0, E.clamp(min=-127))
            y = x.abs() / unit
            low, high = torch.bucketize(y, half), torch.bucketize(y, half, right=True)      # they differ on a tie
            code = torch.where(low % 2 == 0, low, high)
            out[a:a + 1024] = (level[code] * unit * torch.sign(x)).flatten(1)[:, :k]
        return out
    if case["op"] in ("product", "gate_up"):
        x = st["x"].double()
        y = [torch.cat([x @ _exact_matrix(c[i:i + 32], s[i:i + 32], min(4096, case["m"] - 128 * i), case["k"]).T for i in range(0, c.shape[0], 32)], 1) for c, s in st["w"]]
        return y[0] if case["op"] == "product" else y[0] * torch.sigmoid(y[0]) * y[1]
    if case["op"] == "draw":
        out = np.full((case["rows"], 16), -1, dtype=np.int32)
        u = st["u"].tolist()
        for r in range(case["rows"]):
            z = st["logits"][r].double().cpu().numpy() / case["temp"]
            w = np.exp(z - z.max())
            for j in range(min(case["draws"], case["vocab"])):
                run = np.cumsum(w)
                out[r, j] = min(int(np.searchsorted(run, u[r][j] * run[-1], side="right")), int(np.flatnonzero(w)[-1]))
                w[out[r, j]] = 0
        return torch.tensor(out, device="cuda")
    return _exact_verify(st)


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(k)) for k in range(6)]:
        print(c.get("name", "drawn"), work(c), {k: v for k, v in c.items() if k != "name"})
