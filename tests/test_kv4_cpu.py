"""The paged 4-bit cache without a GPU: index arithmetic of the kernels (compiled for the host), the oracle's
pins, and the refusals of the binding."""
import ctypes as C
import subprocess
from pathlib import Path

import numpy as np
import pytest

from oracle import kv4 as okv4

ROOT = Path(__file__).resolve().parent.parent

_HARNESS = r"""
#include "kv4_layout.h"
#include <vector>
using namespace ghd;
extern "C" {
unsigned block_bytes(int R, int d, int es) { return kv4_block_bytes(R, d, es); }
unsigned code_at(int R, int d, int w, int r) { return kv4_code_at(R, d, w, r); }
unsigned param_at(int R, int d, int es, int w, int r) { return kv4_param_at(R, d, es, w, r); }
void seq(int start, int end, int n_rows, int len, long long cap, int* out) {
    Kv4Seq q = kv4_seq(start, end, n_rows, len, cap);
    out[0] = q.row0; out[1] = q.n; out[2] = q.len; out[3] = q.n_new; out[4] = q.bad;
}
// Deals the units of a batch over `ctas` runs as the kernels do.  out: (seq, head, tile, chunk0, take, chunks, cta, first lo) per piece.
long long deal(int n_seqs, const int* start, const int* len, int n_rows, long long cap, int heads, int group, int tile_rows, int chunk,
               int lead, int ctas, long long* out, long long most) {
    Kv4Tiling t{heads, group, tile_rows, chunk, lead};
    std::vector<int64_t> sums(n_seqs + 1, 0);
    auto seq_of = [&](int s) { return kv4_seq(start[s], start[s + 1], n_rows, len[s], cap); };
    for (int s = 0; s < n_seqs; ++s) sums[s + 1] = sums[s] + heads * kv4_head_units(t, seq_of(s));
    const int64_t units = sums[n_seqs], per = kv4_units_per_cta(units, ctas);
    long long n = 0;
    for (int c = 0; c < ctas; ++c) {
        int64_t u = per * c;
        const int64_t e = u + per < units ? u + per : units;
        while (u < e) {
            Kv4Item it = kv4_find_item(t, sums.data(), n_seqs, seq_of, u, e);
            if (n >= most || it.next <= u || it.next > e) return -1;
            u = it.next;
            if (it.take == 0) continue;
            long long* o = out + 9 * n++;
            o[0] = it.seq; o[1] = it.head; o[2] = it.tile; o[3] = it.chunk0; o[4] = it.take; o[5] = it.chunks; o[6] = c; o[7] = it.first; o[8] = kv4_tile_keys(t, it.q, it.tile);
        }
    }
    return n;
}
// Walks every run item by item: by a search for each and by going on from the one before.  -> items, or -1 where the two differ
long long walk(int n_seqs, const int* start, const int* len, int n_rows, long long cap, int heads, int group, int tile_rows, int chunk, int lead, int ctas) {
    Kv4Tiling t{heads, group, tile_rows, chunk, lead};
    std::vector<int64_t> sums(n_seqs + 1, 0);
    auto seq_of = [&](int s) { return kv4_seq(start[s], start[s + 1], n_rows, len[s], cap); };
    for (int s = 0; s < n_seqs; ++s) sums[s + 1] = sums[s] + heads * kv4_head_units(t, seq_of(s));
    const int64_t units = sums[n_seqs], per = kv4_units_per_cta(units, ctas);
    long long n = 0;
    for (int c = 0; c < ctas; ++c) {
        const int64_t u = per * c, e = u + per < units ? u + per : units;
        if (u >= e) continue;
        Kv4Item b = kv4_find_item(t, sums.data(), n_seqs, seq_of, u, e);
        for (;;) {
            ++n;
            if (b.take == 0 && b.next < e) return -1;             // only a run's last item may be without chunks
            if (b.next >= e) break;
            const Kv4Item a = kv4_find_item(t, sums.data(), n_seqs, seq_of, b.next, e);
            kv4_next_item(t, seq_of, b, e);
            if (a.seq != b.seq || a.head != b.head || a.tile != b.tile || a.chunk0 != b.chunk0 || a.chunks != b.chunks || a.take != b.take ||
                a.first != b.first || a.next != b.next || a.q.row0 != b.q.row0 || a.q.n != b.q.n || a.q.len != b.q.len || a.q.n_new != b.q.n_new) return -1;
        }
    }
    return n;
}
}
"""


@pytest.fixture(scope="module")
def lay(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv4")
    (d / "h.cpp").write_text(_HARNESS)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", f"-I{ROOT}/paper_2505_23219_b200/csrc", "-o", str(d / "h.so"), str(d / "h.cpp")])
    lib = C.CDLL(str(d / "h.so"))
    lib.deal.restype = lib.walk.restype = C.c_longlong
    return lib


@pytest.mark.parametrize("R", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("es", [2, 4])
def test_a_block_holds_its_rows_once_and_nothing_else(lay, R, d, es):
    size = lay.block_bytes(R, d, es)
    assert size % 16 == 0                                      # 16-byte pieces and bulk copies of whole blocks
    used = np.zeros(size, np.int32)
    for w in (0, 1):
        for r in range(R):
            c = lay.code_at(R, d, w, r)
            assert c % 16 == 0 and lay.code_at(R, d, w, r - r % 16) % 16 == 0
            used[c:c + d // 2] += 1
            p = lay.param_at(R, d, es, w, r)
            assert p % (2 * es) == 0
            used[p:p + 2 * es] += 1
    assert (used == 1).all()
    assert size == okv4.block_bytes(R, d, "f16" if es == 2 else "f32")
    pool = okv4.Pool(1, 1, R, d, "f16" if es == 2 else "f32")
    for w in (0, 1):
        for r in (0, R - 1):
            assert pool._at(w, r) == (lay.code_at(R, d, w, r), lay.param_at(R, d, es, w, r))


def test_numbers_out_of_range_are_held_inside_the_buffers(lay):
    out = (C.c_int * 5)()
    rng = np.random.RandomState(3)
    for _ in range(4000):
        n_rows, cap = int(rng.randint(0, 50)), int(rng.randint(16, 200))
        a, b, ln = int(rng.randint(-20, 80)), int(rng.randint(-20, 80)), int(rng.choice([-5, 0, 3, 190, 2**31 - 1, -2**31, rng.randint(0, 200)]))
        lay.seq(a, b, n_rows, ln, C.c_longlong(cap), out)
        row0, n, length, n_new, bad = out
        assert 0 <= row0 <= n_rows and 0 <= n and row0 + n <= n_rows
        assert 0 <= length <= cap and 0 <= n_new <= n and length + n_new <= cap
        fine = 0 <= a <= b <= n_rows and 0 <= ln and ln + (b - a) <= cap
        assert bool(bad) != fine
        if fine:
            assert (row0, n, length, n_new) == (a, b - a, ln, b - a)


@pytest.mark.parametrize("group,tile_rows,chunk", [(1, 8, 64), (1, 16, 64), (4, 8, 64), (7, 16, 64), (1, 64, 128), (5, 128, 128)])
@pytest.mark.parametrize("lead", [0, 3, 6])
def test_the_work_split_takes_every_chunk_once(lay, group, tile_rows, chunk, lead):
    rng = np.random.RandomState(group * 100 + tile_rows)
    buf = (C.c_longlong * (9 * 200000))()
    for trial in range(25):
        n_seqs = int(rng.choice([1, 2, 5, 17]))
        cnt = rng.choice([0, 1, 2, 7, 33, 200], n_seqs)
        lens = rng.choice([0, 1, 15, 63, 64, 65, 500, 3000], n_seqs).astype(np.int32)
        start = np.concatenate(([0], np.cumsum(cnt))).astype(np.int32)
        heads, ctas = int(rng.choice([1, 3, 8])), int(rng.choice([1, 7, 148, 592]))
        n = lay.deal(n_seqs, start.ctypes.data_as(C.c_void_p), lens.ctypes.data_as(C.c_void_p), int(start[-1]), C.c_longlong(1 << 20), heads, group, tile_rows, chunk,
                     lead, ctas, buf, C.c_longlong(200000))
        assert n >= 0
        pieces = np.array(buf[: 9 * n], np.int64).reshape(n, 9)
        seen = {}
        for s, h, tile, c0, take, chunks, cta, first, keys in pieces:
            want_keys = min(lens[s] + cnt[s], lens[s] + ((tile + 1) * tile_rows - 1) // group + 1)
            assert keys == want_keys and chunks == max(1, -(-want_keys // chunk))
            got = seen.setdefault((s, h, tile), [0, int(first), []])
            assert got[0] == c0 and got[1] == first             # pieces of an item come in order, without holes
            got[0] += take
            got[2].append(int(cta))
            assert got[0] <= chunks
        items = {(s, h, tl) for s in range(n_seqs) for h in range(heads) for tl in range(-(-int(cnt[s]) * group // tile_rows))}
        assert set(seen) == items
        units = sum(v[0] + lead for v in seen.values())
        per = max(1, -(-units // ctas))
        cont, begun = {}, {}
        for key, (total, first, ctas_of) in seen.items():
            chunks = max(1, -(-min(lens[key[0]] + cnt[key[0]], lens[key[0]] + ((key[2] + 1) * tile_rows - 1) // group + 1) // chunk))
            assert total == chunks
            # contributors are consecutive, and what the finisher derives from the unit numbers
            assert ctas_of == list(range(first // per, (first + chunks - 1) // per + 1))
            if len(ctas_of) > 1:                                # scratch: one slot for an item begun, one for an item continued
                assert ctas_of[0] not in begun
                begun[ctas_of[0]] = key
                for c in ctas_of[1:]:
                    assert c not in cont
                    cont[c] = key


def test_oracle_quantisation_pins():
    x = np.arange(16, dtype=np.float32)
    for dt in ("f16", "f32"):
        c, s, m = okv4.quantise(x, dt)                           # 0 .. 15 in steps of one: codes are the values
        assert list(c) == list(range(16)) and s == 1 and m == 0
        c, s, m = okv4.quantise(np.full(64, 3.25, np.float32), dt)
        assert not c.any() and s == 0 and m == 3.25
        for bad in (np.nan, np.inf, -np.inf):
            y = x.copy()
            y[5] = bad
            c, s, m = okv4.quantise(y, dt)
            with np.errstate(all="ignore"):
                assert np.isnan(np.float64(m) + np.float64(s) * c.astype(np.float64)).all()
    y = np.random.RandomState(0).randn(128).astype(np.float32)
    c, s, m = okv4.quantise(y, "f32")
    assert np.abs(m + s * c.astype(np.float64) - y).max() <= float(s) * (0.5 + 1e-6)


def test_oracle_rotation_keeps_lengths_and_relative_angles():
    r = np.random.RandomState(1)
    a, b = r.randn(1, 64), r.randn(1, 64)
    for p in (0, 1, 77, 100000):
        assert np.allclose(np.linalg.norm(okv4.rotate(a, p, 1e4)), np.linalg.norm(a))
        assert np.isclose((okv4.rotate(a, p + 5, 1e4) * okv4.rotate(b, p, 1e4)).sum(), (okv4.rotate(a, 5, 1e4) * b).sum())
    assert np.allclose(okv4.rotate(a, 0, 1e4), a)


def test_oracle_attention_pins():
    pool = okv4.Pool(4, 2, 16, 64, "f32")
    table, r = np.array([[2, 0]]), np.random.RandomState(2)
    for t in range(20):
        page, row = okv4.slots(table, 16, 0, t)
        for h in range(2):
            pool.put(0, page, row, h, np.zeros(64, np.uint8), 0.0, 0.0)                 # zero keys: the mean of the visible values
            pool.put(1, page, row, h, np.zeros(64, np.uint8), 0.0, float(t))
    q = r.randn(3, 4, 64).astype(np.float32)
    vis = np.array([[1, 0, 0], [0, 0, 0], [1, 1, 1]], bool)
    out = okv4.attention(pool, table, [17], [0, 3], [vis], q)
    assert np.allclose(out[0], np.arange(18).mean()) and np.allclose(out[1], np.arange(17).mean()) and np.allclose(out[2], np.arange(20).mean())
    assert not okv4.attention(pool, table, [0], [0, 3], [np.zeros((3, 3), bool)], q).any()
    new = okv4.commit([pool], table, [15], [0, 5], [(2, [0, 2, 4])])
    assert new == [18]
    assert okv4.rows(pool, table, 0, 15, 3)[1][:, 0, 0].tolist() == [15.0, 17.0, 19.0]


def test_binding_refuses_what_is_no_device_tensor():
    import torch
    import paper_2505_23219_b200 as ghd
    table, lens = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ghd.GhdError, match="device tensor"):
        ghd.Kv4Cache(table, lens, 16, 2, 8)
    with pytest.raises(ghd.GhdError, match="n_seqs"):
        ghd.Kv4Cache(lens, lens, 16, 2, 8)
    with pytest.raises(ghd.GhdError, match="device tensor"):
        ghd.Kv4Rows(torch.zeros(3, dtype=torch.int32), 4)


def test_null_contexts_are_refused_without_a_gpu():
    import ctypes
    from paper_2505_23219_b200 import build
    lib = ctypes.CDLL(str(build.build()))
    lib.ghd_kv4_pool_bytes.restype = ctypes.c_size_t
    assert lib.ghd_kv4_pool_bytes(None, None) == 0
    n = [None] * 12
    assert lib.ghd_kv4_append(*n[:10]) == 1 and lib.ghd_kv4_attention(*n[:6]) == 1 and lib.ghd_kv4_read(*n[:7]) == 1 and lib.ghd_kv4_commit(*n[:6]) == 1


@pytest.mark.parametrize("seed", range(8))
def test_going_on_to_the_next_item_is_the_search_for_it(lay, seed):
    r = np.random.RandomState(seed)
    for _ in range(8):
        S = r.randint(1, 9)
        cnt = np.where(r.rand(S) < 0.3, 0, r.randint(1, 90, S))
        start = np.concatenate(([0], np.cumsum(cnt))).astype(np.int32)
        ln = np.where(r.rand(S) < 0.2, 0, r.randint(1, 3000, S)).astype(np.int32)
        heads, group, rows, lead, ctas = int(r.randint(1, 6)), int(r.randint(1, 9)), int(r.choice([8, 16, 64])), int(r.randint(0, 8)), int(r.choice([1, 3, 148, 444]))
        p = lambda a: a.ctypes.data_as(C.c_void_p)  # noqa: E731
        n = lay.walk(S, p(start), p(ln), int(start[-1]), C.c_longlong(4000), heads, group, rows, 128, lead, ctas)
        assert n >= 0 and (n > 0) == (start[-1] > 0)


def _host_ctx(dtype="f16"):
    """What the checks of a call's tensors look at, for tensors on the host (device -1)."""
    import types
    import torch
    return types.SimpleNamespace(dtype=torch.float16 if dtype == "f16" else torch.float32, dev=-1)


def test_rows_that_overlap_are_refused():
    """A broadcast row has stride 0: the call would take it for contiguous rows and read behind it."""
    import torch
    import paper_2505_23219_b200 as ghd
    from paper_2505_23219_b200 import binding
    x = torch.zeros((1, 256), dtype=torch.float16)
    for bad in (x.expand(64, 256), torch.zeros(64 * 256, dtype=torch.float16).as_strided((64, 256), (128, 1)), torch.zeros(400, dtype=torch.float16).as_strided((2, 256), (8, 1))):
        with pytest.raises(ghd.GhdError, match="overlap"):
            binding._kv4_strided(_host_ctx(), bad, bad.shape[0], 256, "k")
    wide = torch.zeros((64, 768), dtype=torch.float16)
    for at in (0, 256, 512):
        assert binding._kv4_strided(_host_ctx(), wide[:, at:at + 256], 64, 256, "k") == (wide.data_ptr() + 2 * at, 768)


def test_the_stride_of_a_single_row_says_nothing():
    import torch
    from paper_2505_23219_b200 import binding
    wide = torch.zeros((5, 768), dtype=torch.float16)
    column = torch.zeros((256, 1), dtype=torch.float16)
    for x in (wide[:1, :256], wide[3:4, 256:512], wide[:, 512:], column.t(), wide[:1, :256].expand(4, 256)):
        assert binding._kv4_strided(_host_ctx(), x, 1, 256, "k") == (x.data_ptr(), 0)


@pytest.fixture
def host_binding(monkeypatch):
    """The binding with descriptions of tensors on the host."""
    from paper_2505_23219_b200 import binding

    def need(t, dtype, what, numel, dev=None):
        assert t.dtype is dtype and t.numel() >= numel
        return t.data_ptr()
    monkeypatch.setattr(binding, "_need", need)
    return binding


def test_descriptions_keep_the_tensors_they_point_to(host_binding):
    """The struct has the pointers from the start: another tensor, or another size, needs another description."""
    import torch
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    kv = host_binding.Kv4Cache(i32(2, 4), i32(2), 16, 2, 8)
    rows = host_binding.Kv4Rows(i32(3), 4, pos=i32(4), mask=torch.zeros((4, 1), dtype=torch.int64))
    for x, names in ((kv, ("kv_len", "page_table", "n_seqs", "n_kv_heads", "n_rows", "dev", "c", "ref")), (rows, ("row_start", "pos", "mask", "n_rows", "n_starts", "dev", "c", "ref"))):
        for name in names:
            with pytest.raises(AttributeError):
                setattr(x, name, i32(2))
            with pytest.raises(AttributeError):
                delattr(x, name)
    kv.kv_len[1] = 7                                            # contents are the caller's
    assert kv.c.kv_len == kv.kv_len.data_ptr() and kv.c.page_table == kv.page_table.data_ptr()
    assert (rows.c.row_start, rows.c.pos, rows.c.mask) == (rows.row_start.data_ptr(), rows.pos.data_ptr(), rows.mask.data_ptr())


def test_numbers_beyond_the_struct_are_refused(host_binding):
    """Cut off to 32 bits they would be others: 8 - 2^32 pages are 8 for the kernels and none for the check of the pool's size."""
    import torch
    table, lens, start = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for args in ((16, 2, 8 - 2**32), (16, 2 - 2**32, 8), (16 - 2**32, 2, 8), (16, 2, 2**31), (2**32 + 16, 2, 8)):
        with pytest.raises(host_binding.GhdError, match="32 bits"):
            host_binding.Kv4Cache(table, lens, *args)
    for n in (2**32 + 4, 2**31, -2**31 - 1):
        with pytest.raises(host_binding.GhdError, match="32 bits"):
            host_binding.Kv4Rows(start, n)
    assert host_binding.Kv4Cache(table, lens, 16, 2, 8).c.n_pages == 8 and host_binding.Kv4Rows(start, -1).c.n_rows == -1      # (the calls refuse that)
