"""Sequence layers and 4-bit products at the ends of their values' and sizes' range: activations and weights that overflow, states
that grow or vanish by more than fp32 holds on the way, numbers of sequences beyond what one launch takes.

The bounds of finite results are those of the layers' own tests (test_gpu_q4.py, test_gpu_sequence.py)."""
import numpy as np
import pytest
import torch

import paper_1905_00571_amd as cad
from test_gpu_sequence import TYPES, U, check, dev, half_step, run_scan, scan_inputs, scan_reference, starts_of

# ---- SiLU -----------------------------------------------------------------------------------------

ENDS = np.array([np.inf, np.finfo(np.float32).max, 3e38, 2.4e38, 2.3e38, 6e4, 1e4, 151.0, 150.0, 149.0, 88.0, 17.0, 1.0, 0.0, -0.0, -1e-3, -1.0, -20.0, -80.0,
                 -149.0, -150.0, -151.0, -6e4, -2.4e38, np.finfo(np.float32).min, -np.inf, np.nan], np.float32)


def check_silu(y, v, dtype):
    """y of v / (1 + exp(-v)): no numbers and infinities where that has them in 64 bits, rounded to the type; a finite value to 8 half steps of
    fp32 (and, below 2^-100, to 1e-30)."""
    with np.errstate(all="ignore"):
        ref = v.astype(np.float64) / (1 + np.exp(-v.astype(np.float64)))
        held = ref.astype(np.float16 if dtype == "f16" else np.float32)
    got = y.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref)), (got, ref)
    infinite = np.isinf(held)
    assert np.array_equal(got[infinite], held[infinite].astype(np.float64))
    f = np.isfinite(held)
    assert (np.abs(got[f] - ref[f]) <= 8 * U * np.abs(ref[f]) + half_step(ref[f], dtype) + 1e-30).all(), (got, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n,cin", [(1, 64), (1, 2304), (20, 64), (300, 64)])
def test_silu_of_a_product_at_the_ends_of_its_range(dtype, n, cin):
    tt, flag, _ = TYPES[dtype]
    h = cad.cadnn_q4_pack_codes(np.ones((len(ENDS), cin), np.int8), np.ones((len(ENDS), -(-cin // 32)), np.float32), 32, flag)
    x = torch.zeros(n, cin, dtype=tt, device="cuda")
    y = cad.cadnn_q4_fc(h, x, dev(ENDS), cad.ACT_SILU)
    for row in {0, n // 2, n - 1}:
        check_silu(y[row], ENDS, dtype)
    x[0, 3] = float("inf")                  # an activation that has overflowed
    y = cad.cadnn_q4_fc(h, x, None, cad.ACT_SILU)
    assert bool((y[0] == float("inf")).all()) and bool((y[1:] == 0).all())
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("channels", [1, 16])
def test_silu_of_a_convolution_at_the_ends_of_its_range(dtype, channels):
    tt, flag, npt = TYPES[dtype]
    with np.errstate(over="ignore"):
        x = np.repeat(ENDS.astype(npt)[:, None], channels, 1)
    for w in (np.ones((channels, 1, 1, 1), np.float32), np.tile(np.float32([0, 1]), (channels, 1)).reshape(channels, 1, 1, 2)):      # (all taps, a tap of zero)
        h = cad.cadnn_pack_weights(w, flag)
        y = cad.cadnn_causal_conv1d(h, dev(x), act=cad.ACT_SILU)
        check_silu(y, x.astype(np.float32), dtype)
        h.free()


# ---- states that grow and vanish ---------------------------------------------------------------------

LENS = [[200], [400], [900], [2100], [200, 1500]]


def check_with_and_without_pieces(v, lens, softplus):
    starts = starts_of(lens)
    ref, bound, last, off = scan_reference(v, starts, softplus, True, False)
    for how in ({}, {"longest": max(lens)}, {"workspace": torch.empty(0, dtype=torch.uint8, device="cuda")}):
        y, kept = run_scan(v, dev(starts), len(lens), softplus, True, False, **how)
        check(kept, last, off, "f32", f"state, {lens}, {list(how)}")
        check(y, ref, bound, "f32", f"{lens}, {list(how)}")


@pytest.mark.gpu
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("rows", [16, 64])
def test_small_states_that_grow_by_more_than_fp32_holds(lens, rows):
    """States of 1e-30 times exp(110) to exp(128), over 16 rows and over 64 (rows of one piece, and of several)."""
    v = scan_inputs(lens, 20, 16, 1, np.float32, 13)
    v["a"] = (v["a"] * 0.0 + np.random.default_rng(1).uniform(110, 128, v["a"].shape) / 128).astype(np.float32)
    v["x"][:] = 0.0
    v["dt"][:] = 0.0
    for lo in starts_of(lens)[:-1]:
        v["dt"][lo + 96:lo + 96 + rows] = 128.0 / rows
    v["state"] *= 1e-30
    check_with_and_without_pieces(v, lens, False)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("first", [1.0, 1e20])
def test_states_that_vanish_stay_so_when_later_rows_grow(lens, first):
    """A factor of exp(-256), over 32 rows, and then one of exp(128) over as many: nothing is left of the state."""
    v = scan_inputs(lens, 20, 16, 1, np.float32, 14)
    v["a"][:] = -1.0
    v["x"][:] = 0.0
    v["dt"][:] = 0.0
    for lo in starts_of(lens)[:-1]:
        v["dt"][lo + 16:lo + 48] = 8.0
        v["dt"][lo + 64:lo + 96] = -4.0
    v["state"] *= first
    check_with_and_without_pieces(v, lens, False)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", LENS)
def test_large_states_that_vanish(lens):
    """States of 1e36 (times ten, outputs would pass what fp32 holds by themselves: sums over the states up to 2e37 and gates up to 5)."""
    v = scan_inputs(lens, 20, 16, 1, np.float32, 15)
    v["a"][:] = -1.0
    v["dt"][:] = 0.0
    for lo, hi in zip(starts_of(lens), starts_of(lens)[1:]):
        v["dt"][lo + 16:lo + 48] = 8.0
        v["x"][lo:lo + 100] = 0.0
        v["dt"][lo + 100:hi] = 0.1
    v["state"] *= 1e36
    check_with_and_without_pieces(v, lens, False)


# ---- decay rates of the largest magnitude --------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[2], [1, 3, 0, 2], [300], [40, 500]])
def test_rates_of_the_lowest_value(lens):
    """a of the type's lowest value: a state is forgotten by a row with a step, and kept by one whose step is zero."""
    v = scan_inputs(lens, 36, 24, 1, np.float32, 16)
    v["a"][::3] = np.finfo(np.float32).min
    v["a"][1, ::2] = -2.0 ** 127
    v["dt"][::2] = -np.inf                    # (softplus gives zero)
    starts = starts_of(lens)
    f = {k: a.copy() for k, a in v.items()}
    f["dt"][::2] = -300.0
    ref, bound, last, off = scan_reference(f, starts, True, True, False)
    for how in ({}, {"longest": max(lens)}, {"workspace": torch.empty(0, dtype=torch.uint8, device="cuda")}):
        y, kept = run_scan(v, dev(starts), len(lens), True, True, False, **how)
        check(y, ref, bound, "f32", str(how))
        check(kept, last, off, "f32", str(how))
        w = dict(v, a=v["a"].copy())
        w["a"][5, 3] = np.nan
        z, held = run_scan(w, dev(starts), len(lens), True, True, False, **how)
        ran = [s for s, m in enumerate(lens) if m]
        assert bool(torch.isnan(z[:, 5]).all()) and bool(torch.isnan(held[ran, 5, 3]).all())
        z[:, 5], held[:, 5, 3] = y[:, 5], kept[:, 5, 3]
        assert torch.equal(y, z) and torch.equal(kept, held)


# ---- activations of 4-bit products ------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("n,cin", [(1, 300), (1, 2304), (5, 2304), (20, 300), (300, 300), (1500, 300)])
def test_every_no_number_stays_one(n, cin):
    """fp32 no-numbers whose payload lies in their low 16 bits alone, of either sign."""
    codes = np.random.default_rng(17).integers(1, 8, (300, cin)).astype(np.int8)
    h = cad.cadnn_q4_pack_codes(codes, np.full((300, -(-cin // 64)), 0.25, np.float32), 64, cad.F32)
    x = torch.ones(n, cin, device="cuda")
    clean = cad.cadnn_q4_fc(h, x)
    for bits in (0x7f800001, 0x7f80ffff, 0x7fc00000, 0xff800001 - 2 ** 32, 0xffffffff - 2 ** 32):
        x.fill_(1.0)
        x.view(torch.int32)[n // 2, 5] = bits
        y = cad.cadnn_q4_fc(h, x)
        assert bool(torch.isnan(y[n // 2]).all()), hex(bits)
        y[n // 2] = clean[n // 2]
        assert torch.equal(y, clean)
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("n,cin", [(1, 300), (3, 2304), (13, 2304), (20, 300), (300, 304), (300, 301), (1500, 304)])
def test_fp16_activations_below_the_normal_numbers_count(n, cin):
    """Products of codes and multiples of 2^-24, whose sums fp32 holds exactly; an fp16 result is rounded to such a multiple once."""
    g = np.random.default_rng(18)
    codes = g.integers(-8, 8, (300, cin)).astype(np.int8)
    h = cad.cadnn_q4_pack_codes(codes, np.full((300, -(-cin // 128)), 0.25, np.float32), 128, cad.F16)
    x = (g.integers(-1023, 1024, (n, cin)) * 2.0 ** -24).astype(np.float16)
    y = cad.cadnn_q4_fc(h, dev(x))
    ref = 0.25 * (x.astype(np.float64) @ codes.astype(np.float64).T)
    assert (np.abs(y.double().cpu().numpy() - ref) <= half_step(ref, "f16")).all()
    h.free()


# ---- more work than one launch takes ------------------------------------------------------------------------

@pytest.mark.gpu
def test_causal_conv1d_of_more_sequences_than_one_launch_has_workgroups_for():
    """2^24 sequences, all but a few of them empty: 2^24 workgroups of 256 threads are one launch's limit."""
    seqs, tokens, channels = 1 << 24, 40, 2048
    g = np.random.default_rng(19)
    first, middle, end = 7, 9, 24                  # rows of the first sequence, of one in the middle, of the last
    starts = torch.full((seqs + 1,), first, dtype=torch.int32, device="cuda")
    starts[0] = 0
    starts[9_000_001:] = first + middle
    starts[seqs] = tokens
    x = g.standard_normal((tokens, channels)).astype(np.float16)
    w = g.uniform(-1, 1, (channels, 4)).astype(np.float16).astype(np.float32)
    h = cad.cadnn_pack_weights(w.reshape(channels, 1, 1, 4), cad.F16)
    want = cad.cadnn_causal_conv1d(h, dev(x), None, dev(np.array([0, first, first + middle, tokens], np.int32)), 3)
    y = cad.cadnn_causal_conv1d(h, dev(x), None, starts, seqs)
    assert torch.equal(y, want)
    h.free()


# ---- gates of a scan -------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("tokens", [1, 3, 20, 400])
@pytest.mark.parametrize("dstate", [4, 40])
def test_gate_of_a_scan_at_the_ends_of_its_range(dtype, tokens, dstate):
    """Outputs that are the gate alone (d x = 1, c = 0): in fp32 as exact as the other layers' SiLU, in fp16 to a half step and 3 |z| half steps of fp32."""
    tt, flag, npt = TYPES[dtype]
    with np.errstate(over="ignore"):
        z = np.concatenate([ENDS, np.linspace(-87, 87, 229)]).astype(npt)
    v = scan_inputs([tokens], len(z), dstate, 1, npt, 20)
    v["x"][:], v["c"][:], v["z"][:], v["d"][:] = 1.0, 0.0, z, 1.0
    for how in ({}, {"workspace": torch.empty(0, dtype=torch.uint8, device="cuda")}):
        y, _ = run_scan(v, None, 1, **how)
        for row in {0, tokens // 2, tokens - 1}:
            if dtype == "f32":
                check_silu(y[row], z, dtype)
            else:
                f = np.isfinite(z) & (np.abs(z) < 65504)
                zf, got = z[f].astype(np.float64), y[row].double().cpu().numpy()
                ref = zf / (1 + np.exp(-np.clip(zf, -700, None)))
                assert (np.abs(got[f] - ref) <= (8 + 3 * np.abs(zf)) * U * np.abs(ref) + half_step(ref, dtype)).all()
                assert np.array_equal(np.isnan(got), np.isnan(z) | (z == -np.inf)) and (got[z == np.inf] == np.inf).all()
