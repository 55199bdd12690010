"""Microscaled 4-bit matrices and sampling without a GPU: the oracles' pins and the refusals of the library and the binding."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import mx4, sampling


@pytest.fixture(scope="module")
def lib():
    from paper_2505_23219_b200 import build
    from paper_2505_23219_b200 import binding
    return binding.load_library(build.build())


# ------------------------------------------------------------------ the oracles
def test_levels_and_ties():
    for mid, want in [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6)]:
        x = np.zeros(32)
        x[0], x[1], x[2] = 4.0, mid, -mid                # the largest is 4: E = 0
        codes, s = mx4.quantise_block(x)
        assert s == 127 and codes[0] == 6 and codes[1] == want and codes[2] == want + 8
    x = np.zeros(32)
    x[:2] = 7.99, -6.2                                    # still E = 0: held at 6
    codes, s = mx4.quantise_block(x)
    assert s == 127 and list(codes[:2]) == [7, 15]


@pytest.mark.parametrize("top,byte", [(0.0, 0), (2.0 ** -149, 0), (2.0 ** -125, 0), (2.0 ** -124, 1), (1.0, 125), (4.0, 127), (7.9, 127), (8.0, 128),
                                      (float(np.finfo(np.float32).max), 252), (math.inf, 255), (math.nan, 255)])
def test_scale_bytes(top, byte):
    x = np.zeros(32)
    x[5] = top
    assert mx4.quantise_block(x)[1] == byte


@pytest.mark.parametrize("m,k", [(1, 1), (3, 33), (128, 128), (130, 200)])
def test_layout_places_every_element_once(m, k):
    seen = set()
    for r in range(mx4.up(m)):
        for c in range(mx4.up(k)):
            seen.add(mx4.code_place(m, k, r, c))
    assert len(seen) == 2 * mx4.code_bytes(m, k) and max(b for b, _ in seen) == mx4.code_bytes(m, k) - 1
    assert len({mx4.scale_place(m, k, r, c) for r in range(mx4.up(m)) for c in range(0, mx4.up(k), 32)}) == mx4.scale_bytes(m, k)


def test_values_of_quantised_are_within_half_a_step():
    r = np.random.RandomState(3)
    x = r.randn(70, 150) * np.exp(2 * r.randn(70, 1))
    codes, scales = mx4.quantise(x)
    v = mx4.values(codes, scales, 70, 150)
    pad = np.zeros((70, 160))
    pad[:, :150] = np.abs(x)
    top = np.repeat(pad.reshape(70, -1, 32).max(-1), 32, axis=1)[:, :150]
    # the largest magnitude has 4 to 8 units: half of the widest step (2 units) is at most a quarter of it, and so is what lies past 6
    assert (np.abs(v - x) <= top / 4).all() and (v != 0).mean() > 0.7


def test_verification_is_exact_for_any_drafter():
    """Over a fine grid of random numbers the emitted first token has the target's distribution, whatever the candidates' was."""
    r = np.random.RandomState(5)
    V = 4
    logits, draft = r.randn(3, V) * 1.5, r.randn(1, V) * 1.5
    p, q = sampling.distribution(logits[0], 1.0), sampling.distribution(draft[0], 1.0)
    grid = (np.arange(24) + 0.5) / 24
    got = np.zeros(V)
    for a in range(V):                                    # two candidates without replacement, every ordered pair by its probability
        for b in range(V):
            if a == b:
                continue
            weight = q[a] * q[b] / (1 - q[a])
            hit = np.zeros(V)
            for ua in grid:
                for ub in grid:
                    for u0 in grid:
                        nodes, toks = sampling.verify([-1, 0, 0], [0, a, b], logits, [u0, ua, ub], 1.0, [0, -1, -1], draft)
                        hit[toks[0]] += 1
            got += weight * hit / hit.sum()
    # every number decides between two outcomes at a border: the grid is off by at most half a cell at each of the three
    assert np.abs(got - p).max() <= 3 * 0.5 / 24


def test_draws_are_without_replacement_and_end():
    logits = np.array([0.0, -np.inf, 1.0, -np.inf], np.float32)
    out = sampling.draw(logits, 1.0, 4, [0.99, 0.0, 0.5, 0.5])
    assert list(out[:4]) == [2, 0, -1, -1]


# ------------------------------------------------------------------ refusals
def test_sizes(lib):
    assert lib.ghd_mx4_code_bytes(1, 1) == 8192 and lib.ghd_mx4_scale_bytes(1, 1) == 512
    for m, k in [(129, 128), (4096, 11008), (1000, 1376)]:
        assert lib.ghd_mx4_code_bytes(m, k) == mx4.code_bytes(m, k) and lib.ghd_mx4_scale_bytes(m, k) == mx4.scale_bytes(m, k)
    for m, k in [(0, 5), (5, 0), (-1, 5), ((1 << 20) + 1, 5), (5, (1 << 20) + 1), (1 << 20, 1 << 20)]:
        assert lib.ghd_mx4_code_bytes(m, k) == 0 and lib.ghd_mx4_scale_bytes(m, k) == 0


def test_null_contexts(lib):
    assert lib.ghd_mx4_quantize(None, None, 0, None) == 1 and lib.ghd_mx4_read(None, None, None, 0) == 1
    assert lib.ghd_mx4_linear(None, None, 0, None, 1, None) == 1 and lib.ghd_mx4_gate_up(None, None, 0, None, None, 1, None) == 1
    assert lib.ghd_draft_sample(None, None, 1, 1.0, 1, None, None) == 1 and lib.ghd_accept_sampled(None, None, None) == 1


def test_binding_refuses_what_is_not_on_a_device(lib):
    import torch
    import paper_2505_23219_b200 as ghd
    with pytest.raises(ghd.GhdError, match="codes"):
        ghd.Mx4(torch.zeros(8192, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 1, 1)
    with pytest.raises(ghd.GhdError, match="GHD_ESHAPE"):
        ghd.Mx4(torch.zeros(8192, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 1 << 21, 1)
    with pytest.raises(ghd.GhdError, match="outside"):
        ghd.Mx4(torch.zeros(8192, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 0, 1)
    z = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ghd.GhdError, match="parent"):
        ghd.SampledRows(z, z, torch.zeros(3, 5), torch.zeros(3))
    with pytest.raises(ghd.GhdError, match="logits"):
        ghd.SampledRows(z, z, torch.zeros(2, 5), torch.zeros(3))


def test_descriptions_have_the_header_layout():
    from paper_2505_23219_b200 import binding
    assert C.sizeof(binding._Mx4) == 24 and binding._Mx4.codes.offset == 8
    assert C.sizeof(binding._Sampled) == 80 and binding._Sampled.n_draft.offset == 64 and binding._Sampled.draft_temperature.offset == 72


@pytest.mark.parametrize("bits,terms", [(11, 3), (24, 5)])
def test_terms_hold_every_bit_and_the_last_one_is_needed(bits, terms):
    """x as a sum of e4m3 numbers, each with 2^5 times what the ones before it left: what the product makes of rows of halves and floats.  One term
    less shows in the norm of a long sum (2^-23 is what the tests of the product allow there)."""
    import torch
    r = np.random.RandomState(bits)
    x = torch.from_numpy(r.randn(128, 32).astype(np.float16 if bits == 11 else np.float32)).double()
    top = torch.floor(torch.log2(x.abs().amax(1, keepdim=True)))
    left, held, after = x * 2.0 ** (7 - top), torch.zeros_like(x), []
    for p in range(terms):
        t = left.float().clamp(-448, 448).to(torch.float8_e4m3fn).double()
        held, left = held + t * 2.0 ** (top - 7 - 5 * p), (left - t) * 32
        after.append(float((held - x).norm() / x.norm()))
    assert ((held - x).abs() <= 2.0 ** (top + 1) * 2.0 ** (-27 if bits == 11 else -37)).all()
    assert after[-2] > 2.0 ** -21.5
