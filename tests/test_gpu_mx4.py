"""Matrices in microscaled 4-bit floating point on the GPU against the double-precision oracle (oracle/mx4.py)."""
import math

import numpy as np
import pytest

from oracle import mx4 as omx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ghd():
    import paper_2505_23219_b200 as g
    return g


def make_ctx(ghd, dtype, k, n=64):
    return ghd.ghd_create(ghd.ModelCfg(512, 4, 128, max(512, -(-k // 8) * 8), 100, 1, 512, n, dtype))


def np_t(dtype):
    return np.float16 if dtype == "f16" else np.float32


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def matrix(r, m, k, dtype):
    return (r.randn(m, k) * np.exp(1.5 * r.randn(m, 1)) * np.exp(0.7 * r.randn(1, k)) * 0.05).astype(np_t(dtype))


def random_held(ghd, r, m, k, lo=118, hi=132):
    """Any codes, scales of a narrow range: what another program may have quantised."""
    codes = r.randint(0, 256, omx.code_bytes(m, k)).astype(np.uint8)
    scales = r.randint(lo, hi, omx.scale_bytes(m, k)).astype(np.uint8)
    # elements past m and k have code 0
    rows, cols = np.arange(omx.up(m))[:, None], np.arange(0, omx.up(k), 2)[None, :]
    tile = (rows // 128) * (omx.up(k) // 128) + cols // 128
    at = tile * 8192 + (rows % 128) * 64 + (cols % 128) // 2
    byte = codes[at]
    byte = np.where(cols + 1 < k, byte, byte & 15)
    codes[at] = np.where((rows < m) & (cols < k), byte, 0)
    return ghd.Mx4(dev(codes), dev(scales), m, k), codes, scales


# ------------------------------------------------------------------ quantise, read back
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("m,k", [(1, 1), (1, 31), (3, 33), (128, 128), (129, 127), (5, 1000), (200, 264), (64, 520)])
def test_quantise_codes_and_scales(ghd, dtype, m, k):
    r = np.random.RandomState(m * 1000 + k)
    ctx = make_ctx(ghd, dtype, k)
    x = matrix(r, m, k, dtype)
    w = ghd.ghd_mx4_quantize(ctx, dev(x))
    codes, scales = omx.quantise(x.astype(np.float64))
    got = w.codes.cpu().numpy()
    # a negative zero's sign is the only freedom
    assert np.array_equal(got, codes) and np.array_equal(w.scales.cpu().numpy(), scales)
    back = ghd.ghd_mx4_read(ctx, w).cpu().numpy()
    assert np.array_equal(back, omx.values(codes, scales, m, k).astype(np_t(dtype)))
    ghd.ghd_sync_status(ctx)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_quantise_ties_limits_and_special_values(ghd, dtype):
    T = np_t(dtype)
    m, k = 12, 96
    x = np.zeros((m, k), T)
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.5]
    for r_, e in enumerate([0, -3, 5]):
        x[r_, :1] = 4.0 * 2.0 ** e
        x[r_, 1:1 + len(mids)] = np.array(mids) * 2.0 ** e
        x[r_, 32] = 7.0 * 2.0 ** e
        x[r_, 33:33 + len(mids)] = -np.array(mids) * 2.0 ** e
        x[r_, 64] = -4.0 * 2.0 ** e
        x[r_, 65:65 + len(mids)] = np.nextafter(np.array(mids, T), T(0)) * T(2.0 ** e)
    tiny, big = np.finfo(T).smallest_subnormal, np.finfo(T).max
    x[3, :] = tiny
    x[4, ::3] = 3 * tiny
    x[5, :] = big
    x[6, 1], x[6, 40], x[6, 70] = np.inf, -np.inf, np.nan
    x[7, 31], x[7, 32] = np.nan, 1.0
    x[8, :] = -0.0
    x[9, ::2], x[9, 1::2] = big, tiny
    ctx = make_ctx(ghd, dtype, k)
    w = ghd.ghd_mx4_quantize(ctx, dev(x))
    codes, scales = omx.quantise(x.astype(np.float64))
    assert np.array_equal(w.scales.cpu().numpy(), scales)
    want = omx.values(codes, scales, m, k)
    back = ghd.ghd_mx4_read(ctx, w).cpu().numpy()
    with np.errstate(over="ignore"):
        assert np.array_equal(back, want.astype(T), equal_nan=True)
    assert np.isnan(back[6]).all() and np.isnan(back[7, :32]).all() and not np.isnan(back[7, 32:]).any()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("off,ld", [(0, 200), (1, 200), (8, 203), (3, 137)])
def test_strides_and_alignment(ghd, dtype, off, ld):
    import torch
    r = np.random.RandomState(off + ld)
    m, k = 37, 130
    ctx = make_ctx(ghd, dtype, k)
    flat = dev(matrix(r, 1, m * ld + off, dtype)[0])
    x = flat[off:off + m * ld].view(m, ld)[:, :k]
    w = ghd.ghd_mx4_quantize(ctx, x)
    codes, scales = omx.quantise(x.cpu().numpy().astype(np.float64))
    assert np.array_equal(w.codes.cpu().numpy(), codes) and np.array_equal(w.scales.cpu().numpy(), scales)
    out = torch.full((off + m * ld,), 7.0, dtype=x.dtype, device="cuda")
    view = out[off:].view(m, ld)
    ghd.ghd_mx4_read(ctx, w, out=view[:, :k])
    assert np.array_equal(view[:, :k].cpu().numpy(), omx.values(codes, scales, m, k).astype(np_t(dtype)))
    assert (view[:, k:] == 7.0).all() and (out[:off] == 7.0).all()
    y = ghd.ghd_mx4_linear(ctx, x, w).cpu().numpy()
    check_product(x.cpu().numpy(), codes, scales, m, k, y)


def test_read_of_scales_out_of_the_type(ghd):
    """Scales that another program wrote: every one of them, rounded once (to infinity and to zero too)."""
    for dtype in ("f16", "f32"):
        m, k = 8, 1024
        codes = np.tile(np.array([0x10, 0x32, 0x54, 0x76, 0x98, 0xba, 0xdc, 0xfe], np.uint8), omx.code_bytes(m, k) // 8)
        scales = np.zeros(omx.scale_bytes(m, k), np.uint8)
        for r in range(m):
            for b in range(k // 32):
                scales[omx.scale_place(m, k, r, 32 * b)] = r * 32 + b
        ctx = make_ctx(ghd, dtype, k)
        got = ghd.ghd_mx4_read(ctx, ghd.Mx4(dev(codes), dev(scales), m, k)).cpu().numpy()
        with np.errstate(over="ignore", under="ignore"):
            want = omx.values(codes, scales, m, k).astype(np_t(dtype))
        assert np.array_equal(got, want, equal_nan=True)


# ------------------------------------------------------------------ product
def product_bound(x, w, k):
    """Absolute bound per element, from the arithmetic.  Products of an element of x (split without loss but for 2^-27 of the largest of 32)
    and a code are exact.  k of them are summed in 32 bits: groups of 32 are aligned to the largest and cut at 2^-24 of it at the
    least, and added to a running sum that is rounded (or cut: 2^-23) each time; the terms of an element, the parts of a split sum and the
    last roundings add a dozen such steps.  Every intermediate sum is at most S = sum |x| |w|."""
    S = np.abs(x) @ np.abs(w).T
    top = np.zeros((x.shape[0], omx.up(k)))
    top[:, :k] = np.abs(x)
    top = np.repeat(top.reshape(x.shape[0], -1, 32).max(-1), 32, axis=1)[:, :k]
    return (math.ceil(k / 32) + 16) * 2.0 ** -22 * S + 2.0 ** -26 * (top @ np.abs(w).T) + 1e-37


def check_product(x, codes, scales, m, k, y):
    x = x.astype(np.float64)
    w = omx.values(codes, scales, m, k)
    err, bound = np.abs(y.astype(np.float64) - x @ w.T), product_bound(x, w, k)
    assert (err <= bound).all(), f"{(err / bound).max()} of the bound"


SHAPES = [(1, 1, 1), (1, 128, 128), (2, 130, 100), (3, 64, 33), (15, 300, 256), (16, 257, 384), (17, 1000, 520), (31, 128, 1376), (32, 129, 640), (33, 700, 512),
          (48, 384, 1024), (64, 512, 2048), (65, 256, 512), (100, 640, 128), (128, 128, 4096), (200, 300, 513), (256, 1152, 256)]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n,m,k", SHAPES)
def test_linear(ghd, dtype, n, m, k):
    r = np.random.RandomState(n * 7 + m * 3 + k)
    ctx = make_ctx(ghd, dtype, k, n)
    w, codes, scales = random_held(ghd, r, m, k)
    x = (r.randn(n, k) * np.exp(1.5 * r.randn(n, k))).astype(np_t(dtype))
    y = ghd.ghd_mx4_linear(ctx, dev(x), w)
    again = ghd.ghd_mx4_linear(ctx, dev(x), w)
    ghd.ghd_sync_status(ctx)
    check_product(x, codes, scales, m, k, y.cpu().numpy())
    assert (y == again).all()


# clusters of single tiles and of pairs, with an odd number of tiles, several groups of rows, one k-step, more CTAs than k-steps
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n,m,k", [(96, 2400, 7000), (24, 2400, 7000), (64, 300, 1100), (22, 9400, 300), (40, 9600, 300), (64, 700, 100), (256, 1100, 130)])
def test_linear_shared_units(ghd, dtype, n, m, k):
    r = np.random.RandomState(n * 11 + m + k)
    ctx = make_ctx(ghd, dtype, k, n)
    w, codes, scales = random_held(ghd, r, m, k)
    x = r.randn(n, k).astype(np_t(dtype))
    y = ghd.ghd_mx4_linear(ctx, dev(x), w)
    again = ghd.ghd_mx4_linear(ctx, dev(x), w)
    ghd.ghd_sync_status(ctx)
    check_product(x, codes, scales, m, k, y.cpu().numpy())
    assert (y == again).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n,m,k", [(1, 1, 1), (1, 11008, 512), (16, 130, 100), (33, 300, 384), (64, 512, 1000), (70, 1376, 512), (256, 257, 256)])
def test_gate_up(ghd, dtype, n, m, k):
    r = np.random.RandomState(n * 5 + m + k)
    ctx = make_ctx(ghd, dtype, k, n)
    (wg, gc, gs), (wu, uc, us) = random_held(ghd, r, m, k, 116, 124), random_held(ghd, r, m, k, 116, 124)
    x = (r.randn(n, k) * 0.2).astype(np_t(dtype))
    u = ghd.ghd_mx4_gate_up(ctx, dev(x), wg, wu).cpu().numpy().astype(np.float64)
    ghd.ghd_sync_status(ctx)
    x = x.astype(np.float64)
    G, U = omx.values(gc, gs, m, k), omx.values(uc, us, m, k)
    g, up = x @ G.T, x @ U.T
    sig = 1 / (1 + np.exp(-g))
    want = g * sig * up
    # d(SiLU) <= 1.1 dg; a few roundings of the functions in 32 bits (|g| enters the exponential's argument); half a step of the output
    bound = 1.1 * product_bound(x, G, k) * np.abs(up) + np.abs(g * sig) * product_bound(x, U, k) + 1.1 * product_bound(x, G, k) * product_bound(x, U, k)
    bound = bound + np.abs(want) * (2.0 ** -20 + np.abs(g) * 2.0 ** -22)
    half = 2.0 ** -11 if dtype == "f16" else 2.0 ** -24
    bound = bound * (1 + half) + half * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 1e-37)
    fine = np.abs(want) < (65504 if dtype == "f16" else 3e38)
    assert fine.mean() > 0.99 and (np.abs(u - want)[fine] <= bound[fine]).all(), f"{(np.abs(u - want)[fine] / bound[fine]).max()} of the bound"


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_rows_of_wide_range_keep_their_bits(ghd, dtype):
    """Elements of one 32 far apart, subnormal ones, the largest numbers: each alone against a matrix that picks it out."""
    k = 64
    T = np_t(dtype)
    ctx = make_ctx(ghd, dtype, k, 40)
    r = np.random.RandomState(2)
    x = np.zeros((40, k), T)
    for i in range(40):
        x[i, i % 32] = r.randn() * 2.0 ** (-12 if dtype == "f16" else -60)
        x[i, 32 + i % 32] = r.randn() * 2.0 ** (14 if dtype == "f16" else 100)
    x[0, 0], x[1, 1] = np.finfo(T).max, np.finfo(T).smallest_subnormal * 5
    x[2, :32] = np.float16(1) + np.arange(32).astype(T) * np.finfo(T).eps
    eye = np.zeros((k, k), np.float64)
    eye[np.arange(k), np.arange(k)] = 1.0
    codes, scales = omx.quantise(eye)
    w = ghd.Mx4(dev(codes), dev(scales), k, k)
    y = ghd.ghd_mx4_linear(ctx, dev(x), w).cpu().numpy().astype(np.float64)
    X = x.astype(np.float64)
    top = np.repeat(np.abs(X).reshape(40, 2, 32).max(-1), 32, axis=1)
    # the least number that a term and its scale can hold is 2^-9 * 2^-127, so an element of x may be off by half of 2^-136
    # besides (no half is that small: 2^-24 is its least)
    assert (np.abs(y - X) <= 2.0 ** -22 * np.abs(X) + 2.0 ** -26 * top + (0 if dtype == "f16" else 2.0 ** -137)).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_nan_and_infinity_stay_in_their_rows(ghd, dtype):
    n, m, k = 20, 200, 256
    r = np.random.RandomState(9)
    ctx = make_ctx(ghd, dtype, k, n)
    w, codes, scales = random_held(ghd, r, m, k)
    scales[omx.scale_place(m, k, 77, 64)] = 255
    w = ghd.Mx4(dev(codes), dev(scales), m, k)
    x = r.randn(n, k).astype(np_t(dtype))
    x[3, 7], x[8, 200] = np.nan, np.inf
    y = ghd.ghd_mx4_linear(ctx, dev(x), w).cpu().numpy()
    nan = np.isnan(y)
    assert nan[:, 77].all() and nan[3].all() and (nan[8] | np.isinf(y[8])).all()
    nan[:, 77] = nan[3] = nan[8] = True
    assert nan.sum() == 200 * 2 + 18
    rest = [i for i in range(n) if i not in (3, 8)]
    scales[omx.scale_place(m, k, 77, 64)] = 127
    keep = np.ones(m, bool)
    keep[77] = False
    W = omx.values(codes, scales, m, k)
    X = x[rest].astype(np.float64)
    assert (np.abs(y[rest] - X @ W.T) <= product_bound(X, W, k))[:, keep].all()


def test_streams_graphs_and_a_shared_workspace(ghd):
    """Calls of many shapes one after the other through one workspace; a context on its own stream; calls recorded and replayed with other inputs."""
    import torch
    r = np.random.RandomState(21)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = make_ctx(ghd, "f16", 2048, 200)
    shapes = [(1, 300, 2048), (200, 513, 640), (3, 4096, 128), (64, 128, 1000), (33, 2000, 2048), (1, 1, 1)]
    held = [random_held(ghd, r, m, k) for _, m, k in shapes]
    xs = [r.randn(n, k).astype(np.float16) for n, _, k in shapes]
    dx = [dev(x) for x in xs]
    torch.cuda.synchronize()
    ys = [ghd.ghd_mx4_linear(ctx, x, w[0]) for x, w in zip(dx, held)]        # (asked for on the default stream)
    side.synchronize()
    for (n, m, k), x, w, y in zip(shapes, xs, held, ys):
        check_product(x, w[1], w[2], m, k, y.cpu().numpy())
    outs = [torch.zeros_like(y) for y in ys]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        for x, w, y in zip(dx, held, outs):
            ghd.ghd_mx4_linear(ctx, x, w[0], y=y)
    xs = [r.randn(*x.shape).astype(np.float16) for x in xs]
    for t, x in zip(dx, xs):
        t.copy_(dev(x))
    torch.cuda.synchronize()
    for _ in range(2):
        with torch.cuda.stream(side):
            g.replay()
    side.synchronize()
    for (n, m, k), x, w, y in zip(shapes, xs, held, outs):
        check_product(x, w[1], w[2], m, k, y.cpu().numpy())
    ghd.ghd_sync_status(ctx)


def test_first_call_of_a_context_is_recorded(ghd):
    import torch
    r = np.random.RandomState(23)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = make_ctx(ghd, "f16", 512, 32)
    w, codes, scales = random_held(ghd, r, 300, 500)
    x, y = r.randn(20, 500).astype(np.float16), torch.empty(20, 300, device="cuda")
    dx = dev(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ghd.ghd_mx4_linear(ctx, dx, w, y=y)
    with torch.cuda.stream(side):
        g.replay()
    side.synchronize()
    check_product(x, codes, scales, 300, 500, y.cpu().numpy())


@pytest.mark.parametrize("lo,hi,e", [(240, 255, -110), (0, 20, 100), (60, 70, 60), (200, 254, -127)])
def test_scales_far_from_one(ghd, lo, hi, e):
    """Large scales with small x and the other way round: the products are ordinary numbers."""
    r = np.random.RandomState(lo)
    n, m, k = 9, 140, 300
    ctx = make_ctx(ghd, "f32", k, n)
    w, codes, scales = random_held(ghd, r, m, k, lo, hi)
    x = np.ldexp(r.randn(n, k), e).astype(np.float32)
    y = ghd.ghd_mx4_linear(ctx, dev(x), w).cpu().numpy()
    X, W = x.astype(np.float64), omx.values(codes, scales, m, k)
    # besides product_bound's: an element of x may be off by 2^-137, half of the least number that a term and its scale hold
    bound = product_bound(X, W, k) + 2.0 ** -137 * np.abs(W).sum(1)[None, :]
    want = X @ W.T
    fine = np.abs(want) + bound < 3e38
    assert fine.all() and (np.abs(y - want) <= bound).all(), f"{(np.abs(y - want) / bound).max()} of the bound"


def test_outputs_end_where_they_should(ghd):
    """Nothing behind the output is written, whatever the last tile holds."""
    import torch
    r = np.random.RandomState(22)
    for dtype in ("f16", "f32"):
        for n, m, k in [(1, 1, 5), (5, 129, 300), (40, 383, 128), (100, 130, 256)]:
            ctx = make_ctx(ghd, dtype, k, n)
            w, codes, scales = random_held(ghd, r, m, k, 118, 124)
            x = (r.randn(n, k) * 0.3).astype(np_t(dtype))
            y = torch.full((n * m + 64,), 7.0, device="cuda")
            ghd.ghd_mx4_linear(ctx, dev(x), w, y=y)
            u = torch.full((n * m + 64,), 7.0, dtype=ctx.dtype, device="cuda")
            ghd.ghd_mx4_gate_up(ctx, dev(x), w, w, u=u)
            ghd.ghd_sync_status(ctx)
            assert (y[n * m:] == 7.0).all() and (u[n * m:] == 7.0).all()
            check_product(x, codes, scales, m, k, y[:n * m].view(n, m).cpu().numpy())


@pytest.mark.parametrize("m,k", [(20000, 128), (128, 8192), (9000, 1152), (12928, 640), (25600, 384)])
def test_linear_of_many_units_and_long_sums(ghd, m, k):
    r = np.random.RandomState(m + k)
    for n in (7, 50):
        ctx = make_ctx(ghd, "f16", k, n)
        w, codes, scales = random_held(ghd, r, m, k)
        x = r.randn(n, k).astype(np.float16)
        check_product(x, codes, scales, m, k, ghd.ghd_mx4_linear(ctx, dev(x), w).cpu().numpy())
        ghd.ghd_sync_status(ctx)


def test_refusals(ghd):
    import torch
    ctx = make_ctx(ghd, "f16", 512, 16)
    w = ghd.ghd_mx4(ctx, 40, 256)
    x = torch.zeros(16, 256, dtype=torch.float16, device="cuda")
    for bad in (x.float(), x[:, :255], x.t(), x[0], x.cpu(), x[:1].expand(16, 256)):
        with pytest.raises((ghd.GhdError, IndexError)):
            ghd.ghd_mx4_linear(ctx, bad, w)
    with pytest.raises(ghd.GhdError, match="max_nodes"):
        ghd.ghd_mx4_linear(ctx, torch.zeros(17, 256, dtype=torch.float16, device="cuda"), w)
    with pytest.raises(ghd.GhdError, match="n < 1"):
        ghd.ghd_mx4_linear(ctx, x[:0], w)
    with pytest.raises(ghd.GhdError, match="y"):
        ghd.ghd_mx4_linear(ctx, x, w, y=torch.zeros(16, 39, device="cuda"))
    with pytest.raises(ghd.GhdError, match="GHD_ENOSPACE"):
        wide = ghd.ghd_mx4(ctx, 4, 640)
        ghd.ghd_mx4_linear(ctx, torch.zeros(2, 640, dtype=torch.float16, device="cuda"), wide)
    with pytest.raises(ghd.GhdError, match="differ"):
        ghd.ghd_mx4_gate_up(ctx, x, w, ghd.ghd_mx4(ctx, 41, 256))
    with pytest.raises(ghd.GhdError, match="codes"):
        ghd.Mx4(w.codes[:-1], w.scales, 40, 256)
    with pytest.raises(ghd.GhdError, match="aligned"):
        odd = torch.zeros(w.codes.numel() + 32, dtype=torch.uint8, device="cuda")[16:16 + w.codes.numel()]
        ghd.ghd_mx4_quantize(ctx, x[:, :256], ghd.Mx4(odd, w.scales, 16, 256))
    with pytest.raises(ghd.GhdError, match="x"):
        ghd.ghd_mx4_quantize(ctx, x, w)
    with pytest.raises(AttributeError):
        w.codes = None
    assert ctx.lib.ghd_mx4_linear(ctx.handle, x.data_ptr(), 100, w.ref, 16, x.data_ptr()) == 1          # ld < k
    assert ctx.lib.ghd_mx4_linear(ctx.handle, x.data_ptr() + 1, 0, w.ref, 16, x.data_ptr()) == 1
    ghd.ghd_sync_status(ctx)


def picked(cols, k, scale):
    """A matrix whose row i has `scale` (a power of two) in column cols[i] and nothing else -> codes, scale bytes."""
    w = np.zeros((len(cols), k))
    w[np.arange(len(cols)), cols] = scale
    return omx.quantise(w)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_gate_up_far_from_zero(ghd, dtype):
    """Strongly negative and positive gates next to large and small up values: finite, and as exact as the functions are."""
    gates = np.array([-3e4, -1000, -206.5, -180.25, -120, -95.5, -89, -88, -87.25, -81, -80, -79.875, -50, -30, -20, -8, -2, -0.5, 0, 0.5, 3, 20, 89, 200], np.float32)
    ups = np.array([1.0, -1.0, 3.0], np.float32)
    n, k = len(gates) * len(ups), 64
    x = np.zeros((n, k), np_t(dtype))
    x[:, 0], x[:, 32] = np.repeat(gates, len(ups)), np.tile(ups, len(gates))          # (32 apart: neither is small next to the other)
    ctx = make_ctx(ghd, dtype, k, n)
    m, worst = 5, 0.0
    wide = [(1.0, 2.0 ** 125), (1.0, 2.0 ** 60), (1.0, 1.0), (1.0, 2.0 ** -30)]
    if dtype == "f32":
        wide += [(2.0 ** 60, 2.0 ** 60), (2.0 ** 100, 2.0 ** -100)]
    for a, b in wide:
        (gc, gs), (uc, us) = picked([0] * m, k, a), picked([32] * m, k, b)
        u = ghd.ghd_mx4_gate_up(ctx, dev(x), ghd.Mx4(dev(gc), dev(gs), m, k), ghd.Mx4(dev(uc), dev(us), m, k)).cpu().numpy().astype(np.float64)
        g, up = x[:, 0].astype(np.float64) * a, x[:, 32].astype(np.float64) * b
        with np.errstate(over="ignore"):
            want = (g / (1 + np.exp(-g)) * up)[:, None] + np.zeros((n, m))
        big = 65504.0 if dtype == "f16" else float(np.finfo(np.float32).max)
        fine = np.abs(want) < big
        assert np.array_equal(u[~fine], np.where(want > 0, np.inf, -np.inf)[~fine])
        # Both sums are exact here.  Above -80: the exponential of a float (one unit, 2^-23), a sum, a quotient and a product (2^-24 each).  Below,
        # 1 + e^-g is e^-g: four factors of the exponential of g / 4 and five products.  At the end half a step of the output, and of its smallest numbers
        # (which the products before the last pass as well).
        # (half: its exponential is exp2's, whose argument -1.44 g is rounded: |g| 2^-23 besides, and a quotient of 2 units)
        err = 14 * 2.0 ** -24 + (2.0 ** -23 * np.abs(np.clip(g, -80, 80))[:, None] + 2.0 ** -22 if dtype == "f16" else 0.0)
        half, least = (2.0 ** -11, 2.0 ** -24) if dtype == "f16" else (2.0 ** -24, 2.0 ** -149)
        bound = np.abs(want) * (err + half) + 4 * least
        assert np.isfinite(u[fine]).all() and (np.abs(u - want)[fine] <= bound[fine]).all(), (a, b, (np.abs(u - want) / bound)[fine].max())
        worst = max(worst, float((np.abs(u - want) / bound)[fine].max()))
    ghd.ghd_sync_status(ctx)
    assert worst <= 1


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("k", [4096, 8192, 14336])
@pytest.mark.parametrize("signs", [1, 2])
def test_long_sums_lose_little(ghd, dtype, k, signs):
    """Relative error of the norm over outputs whose whole sum one CTA works out.  An accumulator takes 4 x 32 (halves) or 4 x 16 (floats) sums
    of 32 products; the running sum is half of the last one on average, and an addition cuts off up to some 2^-28.5 of it on average: for one sign
    64 (32) x 2^-28.5 = 2^-22.5 (2^-23.5).  Besides, each is rounded, half a unit at most, without a sign.  The bound does not depend on k.
    For both signs the running sums are short and the cuts have no sign.  (Without x's last term it is above 2^-21.5 in floats.)"""
    import torch
    n, m = 16, 19000
    g = torch.Generator(device="cuda")
    g.manual_seed(k + signs)
    ctx = make_ctx(ghd, dtype, k, n)
    w, x = torch.randn(m, k, generator=g, device="cuda") * 0.05, torch.randn(n, k, generator=g, device="cuda")
    if signs == 1:
        w, x = w.abs(), x.abs()
    held, x = ghd.ghd_mx4_quantize(ctx, w.to(ctx.dtype)), x.to(ctx.dtype)
    want = x.double() @ ghd.ghd_mx4_read(ctx, held).double().T
    err = float((ghd.ghd_mx4_linear(ctx, x, held).double() - want).norm() / want.norm())
    ghd.ghd_sync_status(ctx)
    assert err <= (2.0 ** -23 if signs == 2 or dtype == "f32" else 2.0 ** -22)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_two_contexts_at_once(ghd, dtype):
    """Products of two contexts on two streams, each with units that several CTAs share, while a third stream keeps SMs busy by turns."""
    import torch
    r = np.random.RandomState(61)
    shapes, sides, jobs = [(50, 12928, 640), (16, 25600, 384)], [torch.cuda.Stream() for _ in range(3)], []
    for (n, m, k), side in zip(shapes, sides):
        with torch.cuda.stream(side):
            ctx = make_ctx(ghd, dtype, k, n)
        w, codes, scales = random_held(ghd, r, m, k)
        x = r.randn(n, k).astype(np_t(dtype))
        jobs.append((ctx, dev(x), w, x, codes, scales, [torch.empty(n, m, device="cuda") for _ in range(30)]))
    a = torch.randn(2048, 2048, device="cuda")
    b = torch.empty_like(a)
    torch.cuda.synchronize()
    for i in range(30):
        for ctx, dx, w, *_, ys in jobs:
            ghd.ghd_mx4_linear(ctx, dx, w, y=ys[i])
        with torch.cuda.stream(sides[2]):
            torch.mul(a, a, out=b)
    torch.cuda.synchronize()
    for (n, m, k), (ctx, dx, w, x, codes, scales, ys) in zip(shapes, jobs):
        ghd.ghd_sync_status(ctx)
        check_product(x, codes, scales, m, k, ys[0].cpu().numpy())
        assert all(torch.equal(ys[0], y) for y in ys[1:])
