"""Layers on packed sequences (short causal convolution, selective scan) and a block of them with 4-bit products,
against their definitions in 64 bits, one token after the other.

Bounds.  u = 2^-24 is half a step of fp32.  Convolution: K + 1 terms summed in fp32, |error| <= (K + 2) u A with A the sum of
the terms' magnitudes; SiLU multiplies it by at most 1.1 and adds 8 u of the value (an exponential, a sum, a quotient).
Scan: the bound of the state is carried along with the state,
    E' = p (E + |h| dp) + |q| dq + u |h'|,   p = exp(step a), q = step x b,
with ds = 8 u for softplus (an exponential to 2 u, at most six roundings of a series; 2 u without it), dp = |step a| (ds + 3 u + 80 u) + 4 u
(80 u: a long sequence is cut into pieces whose steps are summed with at most 8 + 512 / 8 roundings) and dq = ds + 3 u;
an output is off by at most sum |c| E + (N + 4) u (sum |c h| + |d x|), times |silu(z)|, plus (8 + 3 |z|) u of itself.
A result stored in fp16 is off by half a step, 2^-11 of its value (2^-25 below the normal numbers), more."""
import ctypes

import numpy as np
import pytest
import torch

import paper_1905_00571_amd as cad

U = 2.0 ** -24
TYPES = {"f32": (torch.float32, cad.F32, np.float32), "f16": (torch.float16, cad.F16, np.float16)}


def half_step(ref, dtype):
    return 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 if dtype == "f16" else U * np.abs(ref)


def check(got, ref, bound, dtype, what=""):
    got = got.detach().double().cpu().numpy()
    bound = bound + half_step(ref, dtype) + 1e-30
    d = np.abs(got - ref)
    assert np.isfinite(got).all(), what
    assert (d <= bound).all(), f"{what}: {int((d > bound).sum())} beyond the bound, worst {float((d / bound).max()):.2f}"


def dev(v, tt=None):
    t = torch.from_numpy(np.ascontiguousarray(v)).cuda()
    return t if tt is None else t.to(tt)


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1 + np.exp(-v))


def starts_of(lens, offset=0):
    return np.concatenate([[offset], offset + np.cumsum(lens)]).astype(np.int32)


# ---- short causal convolution ---------------------------------------------------------------

def conv_reference(x, w, bias, state, starts, act):
    x, w, state = x.astype(np.float64), w.astype(np.float64), state.astype(np.float64).copy()
    k = w.shape[1]
    y, mag = np.zeros_like(x), np.zeros_like(x)
    for s, (lo, hi) in enumerate(zip(starts, starts[1:])):
        line = np.concatenate([state[s], x[lo:hi]])
        for j in range(k):
            y[lo:hi] += line[j:j + hi - lo] * w[:, j]
            mag[lo:hi] += np.abs(line[j:j + hi - lo] * w[:, j])
        state[s] = line[len(line) - (k - 1):] if k > 1 else state[s]
    if bias is not None:
        y, mag = y + bias, mag + np.abs(bias)
    bound = (k + 2) * U * mag
    if act == cad.ACT_RELU:
        y = np.maximum(y, 0)
    if act == cad.ACT_SILU:
        y = silu(y)
        bound = 1.1 * bound + 8 * U * np.abs(y)
    return y, bound, state


CONV = [([1], 64, 4), ([1] * 7, 40, 4), ([5, 0, 1, 2, 30], 16, 4), ([200], 130, 3), ([0, 0, 3], 8, 8), ([2, 2, 2], 24, 7),
        ([700, 1, 66], 64, 2), ([129] * 3, 72, 1), ([33] * 4, 9, 5), ([1000], 2056, 4), ([0], 8, 4), ([64, 64], 512, 6)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("lens,channels,taps", CONV)
def test_causal_conv1d(dtype, lens, channels, taps):
    tt, flag, npt = TYPES[dtype]
    g = np.random.default_rng(channels + taps)
    tokens, seqs = sum(lens), len(lens)
    x = g.standard_normal((tokens, channels)).astype(npt)
    w = g.uniform(-1, 1, (channels, taps)).astype(npt).astype(np.float32)
    w[::3, 0] = 0.0
    bias = g.standard_normal(channels).astype(np.float32)
    state = g.standard_normal((seqs, taps - 1, channels)).astype(npt)
    act = [cad.ACT_SILU, cad.ACT_NONE, cad.ACT_RELU][(channels + taps) % 3]
    h = cad.cadnn_pack_weights(w.reshape(channels, 1, 1, taps), flag)
    starts = starts_of(lens)
    forms = [dev(starts)] + ([None] if len(set(lens)) == 1 else [])
    for seq_start in forms:
        for b, st in ((bias, state), (None, None)):
            kept = None if st is None else dev(st)
            y = cad.cadnn_causal_conv1d(h, dev(x), kept, seq_start, seqs, None if b is None else dev(b), act)
            ref, bound, last = conv_reference(x, w, b, np.zeros_like(state) if st is None else st, starts, act)
            check(y, ref, bound, dtype, f"{lens}, {channels} channels, {taps} taps")
            if st is not None:
                assert np.array_equal(kept.double().cpu().numpy(), last)      # rows are moved, not computed
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_causal_conv1d_rows_apart_and_rows_of_no_sequence(dtype):
    """Slices of wider rows, odd channel counts, offsets that leave rows to no sequence: those and what lies between rows stay."""
    tt, flag, npt = TYPES[dtype]
    g = np.random.default_rng(2)
    for channels, off in ((48, 8), (48, 3), (37, 0)):
        starts = np.array([3, 40, 40, 97], np.int32)
        x = g.standard_normal((110, channels)).astype(npt)
        w = g.uniform(-1, 1, (channels, 4)).astype(npt).astype(np.float32)
        state = g.standard_normal((3, 3, channels)).astype(npt)
        h = cad.cadnn_pack_weights(w.reshape(channels, 1, 1, 4), flag)
        wide = torch.full((110, channels + 16), float("nan"), dtype=tt, device="cuda")
        wide[3:97, off:off + channels] = dev(x)[3:97]
        out = torch.full((110, channels + 16), 7.0, dtype=tt, device="cuda")
        kept = dev(state)
        cad.cadnn_causal_conv1d(h, wide[:, off:off + channels], kept, dev(starts), 3, out=out[:, off:off + channels])
        ref, bound, last = conv_reference(x, w, None, state, starts, cad.ACT_NONE)
        check(out[3:97, off:off + channels], ref[3:97], bound[3:97], dtype)
        assert np.array_equal(kept.double().cpu().numpy(), last)
        out[3:97, off:off + channels] = 7.0
        assert bool((out == 7.0).all())
        h.free()


@pytest.mark.gpu
def test_causal_conv1d_skips_zero_taps_and_cuts_bad_offsets():
    w = np.array([[0.0, 2.0], [1.0, 0.0]], np.float32)
    h = cad.cadnn_pack_weights(w.reshape(2, 1, 1, 2))
    x = torch.tensor([[float("inf"), 1.0], [1.0, float("nan")], [3.0, 5.0]], device="cuda")
    y = cad.cadnn_causal_conv1d(h, x)
    assert y[1].tolist() == [2.0, 1.0] and y[0].tolist() == [float("inf"), 0.0] and y[2, 0].item() == 6.0
    x = torch.ones(20, 2, device="cuda")
    out = torch.full((20, 2), 7.0, device="cuda")
    state = torch.zeros(3, 1, 2, device="cuda")
    # sequence 0: rows 0 to 6; sequence 1: its end lies before its start, so it is empty; sequence 2: from row 15 to the end
    cad.cadnn_causal_conv1d(h, x, state, torch.tensor([-5, 6, -9, 1000], dtype=torch.int32, device="cuda"), 3, out=out)
    assert bool((state[1] == 0).all())
    h.free()


# ---- selective scan -----------------------------------------------------------------------------

def scan_inputs(lens, channels, dstate, groups, npt, seed):
    g = np.random.default_rng(seed)
    tokens, seqs = sum(lens), len(lens)
    v = {"x": g.standard_normal((tokens, channels)).astype(npt), "dt": (g.standard_normal((tokens, channels)) * 1.5).astype(npt),
         "z": (g.standard_normal((tokens, channels)) * 2).astype(npt),
         "b": g.standard_normal((tokens, groups, dstate)).astype(npt), "c": g.standard_normal((tokens, groups, dstate)).astype(npt),
         "a": -(g.uniform(0.05, 4.0, (channels, dstate))).astype(np.float32), "d": g.standard_normal(channels).astype(np.float32),
         "dt_bias": g.uniform(-6, 0, channels).astype(np.float32), "state": g.standard_normal((seqs, channels, dstate)).astype(np.float32)}
    return v


def scan_reference(v, starts, softplus, gate, bias=True, skip=True, state=True):
    f = {k: a.astype(np.float64) for k, a in v.items()}
    tokens, channels = f["x"].shape
    groups, n = f["b"].shape[1:]
    step = f["dt"] + (f["dt_bias"] if bias else 0.0)
    ds = 2 * U * (1 + np.abs(step))
    if softplus:
        # (the bias is added in fp32: its rounding moves softplus by at most u |step|, relative to it at most u (1 + |step|))
        ds = 8 * U + U * (1 + np.abs(step))
        step = np.logaddexp(0, step)
    else:
        ds = 2 * U * np.ones_like(step)
    d = f["d"] if skip else np.zeros(channels)
    y, bound = np.zeros((tokens, channels)), np.zeros((tokens, channels))
    kept = f["state"].copy() if state else np.zeros_like(f["state"])
    off = np.zeros_like(kept)
    for s, (lo, hi) in enumerate(zip(starts, starts[1:])):
        h, e = kept[s], off[s]
        for t in range(lo, hi):
            b, c = (np.repeat(f[k][t], channels // groups, 0) for k in "bc")
            sa = step[t][:, None] * f["a"]
            p, q = np.exp(sa), (step[t] * f["x"][t])[:, None] * b
            dp = np.abs(sa) * (ds[t][:, None] + 83 * U) + 4 * U
            new = p * h + q
            e = p * (e + np.abs(h) * dp) + np.abs(q) * (ds[t][:, None] + 3 * U) + U * np.abs(new)
            h = new
            y[t] = (c * h).sum(1) + d * f["x"][t]
            bound[t] = (np.abs(c) * e).sum(1) + (n + 4) * U * (np.abs(c * h).sum(1) + np.abs(d * f["x"][t]))
        kept[s], off[s] = h, e
    if gate:
        z = silu(f["z"])
        y = y * z
        bound = bound * np.abs(z) + (8 + 3 * np.abs(f["z"])) * U * np.abs(y)
    return y, bound, kept, off


def run_scan(v, seq_start, seqs, softplus=True, gate=True, bias=True, skip=True, state=True, **more):
    t = {k: dev(a) for k, a in v.items()}
    kept = t["state"] if state else None
    y = cad.cadnn_selective_scan(t["x"], t["dt"], t["a"], t["b"], t["c"], d=t["d"] if skip else None, z=t["z"] if gate else None,
                                 dt_bias=t["dt_bias"] if bias else None, softplus=softplus, state=kept, seq_start=seq_start, seqs=seqs, **more)
    return y, kept


SCAN = [([1] * 40 + [300] + [2] * 30, 24, 16, 1), ([1], 1, 1, 1), ([1], 1536, 16, 1), ([1] * 5, 100, 16, 1), ([1, 0, 1, 1], 64, 64, 4), ([2, 1, 3], 20, 3, 2), ([1], 30, 256, 3), ([4], 12, 128, 1),
        ([9], 5, 5, 1), ([8, 16, 24], 70, 16, 1), ([37], 300, 8, 1), ([40, 0, 11, 90], 33, 24, 3), ([100], 20, 64, 2), ([60], 18, 100, 2),
        ([50], 6, 256, 1), ([700], 64, 16, 1), ([300, 1, 0, 512, 77], 36, 16, 2), ([1100], 40, 7, 1), ([260] * 3, 260, 20, 1), ([640], 9, 130, 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("lens,channels,dstate,groups", SCAN)
def test_selective_scan(dtype, lens, channels, dstate, groups):
    tt, flag, npt = TYPES[dtype]
    v = scan_inputs(lens, channels, dstate, groups, npt, channels + dstate)
    starts = starts_of(lens)
    what = f"{lens}, {channels} channels, {dstate} states, {groups} groups"
    ref, bound, last, off = scan_reference(v, starts, True, True)
    runs = [{"seq_start": dev(starts)}, {"seq_start": dev(starts), "longest": max(lens)}, {"seq_start": dev(starts), "longest": 1}, {"seq_start": dev(starts), "workspace": torch.empty(0, dtype=torch.uint8, device="cuda")},
            {"seq_start": dev(starts), "workspace": torch.empty(64, dtype=torch.uint8, device="cuda")}]
    if len(set(lens)) == 1:
        runs.append({"seq_start": None})
    for how in runs:
        y, kept = run_scan(v, seqs=len(lens), **how)
        check(y, ref, bound, dtype, what)
        check(kept, last, off, "f32", what + ": state")
    ref, bound, _, _ = scan_reference(v, starts, True, False, False, False, False)
    y, _ = run_scan(v, dev(starts), len(lens), True, False, False, False, False)
    check(y, ref, bound, dtype, what + ", without what may be left out")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("lens", [[3, 1], [200, 150]])
def test_selective_scan_without_softplus(dtype, lens):
    tt, flag, npt = TYPES[dtype]
    v = scan_inputs(lens, 50, 16, 1, npt, 3)
    v["dt"] = np.abs(v["dt"]) * npt(0.1)
    starts = starts_of(lens)
    ref, bound, last, off = scan_reference(v, starts, False, True, bias=False)
    y, kept = run_scan(v, dev(starts), len(lens), softplus=False, bias=False)
    check(y, ref, bound, dtype)
    check(kept, last, off, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("each", [1, 60, 700])
def test_selective_scan_rows_apart_and_rows_of_no_sequence(dtype, each):
    tt, flag, npt = TYPES[dtype]
    channels, n, groups = 44, 16, 2
    lens = [each, 0, each + 1]
    v = scan_inputs(lens, channels, n, groups, npt, 5)
    starts = starts_of(lens)
    tokens = sum(lens)
    ref, bound, last, off = scan_reference(v, starts, True, True)
    rows = torch.full((tokens + 9, 4 * channels + 2 * groups * n + 5), float("nan"), dtype=tt, device="cuda")
    at, views = 1, {}
    for k in ("x", "z", "dt", "b", "c"):
        width = channels if k in "xzdt" else groups * n
        views[k] = rows[:, at:at + width]
        views[k][4:4 + tokens] = dev(v[k].reshape(tokens, width))
        at += width
    out = torch.full((tokens + 9, channels + 3), 7.0, dtype=tt, device="cuda")
    t = {k: dev(v[k]) for k in ("a", "d", "dt_bias", "state")}
    cad.cadnn_selective_scan(views["x"], views["dt"], t["a"], views["b"].unflatten(1, (groups, n)), views["c"].unflatten(1, (groups, n)), d=t["d"],
                             z=views["z"], dt_bias=t["dt_bias"], softplus=True, state=t["state"], seq_start=dev(starts + 4), seqs=3, out=out[:, 2:2 + channels])
    check(out[4:4 + tokens, 2:2 + channels], ref, bound, dtype)
    check(t["state"], last, off, "f32")
    out[4:4 + tokens, 2:2 + channels] = 7.0
    assert bool((out == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("cuts", [[900], [333, 1, 1, 2, 563], [899, 1], [64] * 14 + [4]])
def test_prompt_in_parts_leads_to_the_same_state(dtype, cuts):
    tt, flag, npt = TYPES[dtype]
    v = scan_inputs([900], 20, 16, 1, npt, 8)
    ref, bound, last, off = scan_reference(v, [0, 900], True, True)
    t = {k: dev(a) for k, a in v.items()}
    got, at = [], 0
    for m in cuts:
        part = slice(at, at + m)
        got.append(cad.cadnn_selective_scan(t["x"][part], t["dt"][part], t["a"], t["b"][part], t["c"][part], d=t["d"], z=t["z"][part],
                                            dt_bias=t["dt_bias"], softplus=True, state=t["state"]))
        at += m
    check(torch.cat(got), ref, bound, dtype)
    check(t["state"], last, off, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [2, 200])
@pytest.mark.parametrize("dstate", [16, 24, 3])
def test_selective_scan_with_masked_steps_and_values_that_are_not_finite(tokens, dstate):
    """A step of the lowest value or of minus infinity leaves the state as it is (softplus gives 0); an infinite x is infinite
    in its own channel and in no other."""
    v = scan_inputs([tokens], 70, dstate, 1, np.float32, 4)
    v["dt"][0, ::2] = np.finfo(np.float32).min
    v["dt"][1, ::2] = -np.inf
    y, kept = run_scan(v, None, 1, bias=False)
    f = {k: a.copy() for k, a in v.items()}
    f["dt"][:2, ::2] = -200.0                     # softplus is zero in both formats' range
    ref, bound, last, off = scan_reference(f, [0, tokens], True, True, bias=False)
    check(y, ref, bound, "f32")
    check(kept, last, off, "f32")
    v["x"][0, 7] = np.inf
    v["c"] = np.abs(v["c"])
    v["b"] = np.abs(v["b"])
    v["d"][7] = 0.5
    f = {k: a.copy() for k, a in v.items()}
    f["dt"][:2, ::2] = -200.0
    f["x"][0, 7] = 1.0
    ref, bound, last, off = scan_reference(f, [0, tokens], True, False, bias=False)
    y, kept = run_scan(v, None, 1, gate=False, bias=False)
    assert bool(torch.isinf(y[0, 7])) and bool(torch.isinf(kept[0, 7]).all())
    others = [c for c in range(70) if c != 7]
    check(y[:, others], ref[:, others], bound[:, others], "f32")
    check(kept[:, others], last[:, others], off[:, others], "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[100], [1000], [90, 1000]])
def test_selective_scan_with_states_that_grow(lens):
    """a > 0: over a run of rows exp(a * steps) passes what fp32 holds, but states that are zero until the last rows do not notice."""
    v = scan_inputs(lens, 20, 16, 1, np.float32, 12)
    v["a"] = np.abs(v["a"]) * 0.25
    v["dt"][:] = 8.0
    v["state"][:] = 0.0
    starts = starts_of(lens)
    for lo, hi in zip(starts, starts[1:]):
        v["x"][lo:hi - 3] = 0.0
    ref, bound, last, off = scan_reference(v, starts, False, False, False)
    y, kept = run_scan(v, dev(starts), len(lens), False, False, False)
    check(y, ref, bound, "f32")
    check(kept, last, off, "f32")


@pytest.mark.gpu
def test_selective_scan_of_a_long_sequence():
    """More pieces of one sequence than are joined in one round."""
    for tokens in (2065, 5000):
        v = scan_inputs([tokens], 6, 16, 1, np.float32, tokens)
        v["a"] *= 0.01                  # (what a row leaves is still there thousands of rows later)
        ref, bound, last, off = scan_reference(v, [0, tokens], True, True)
        y, kept = run_scan(v, None, 1)
        check(y, ref, bound, "f32")
        check(kept, last, off, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [12, 400, 3000])
def test_selective_scan_cuts_bad_offsets(tokens):
    """Offsets that lie outside the rows or descend change no row and no state but those of the call's own tensors."""
    channels, n = 40, 16
    v = scan_inputs([tokens], channels, n, 1, np.float32, 9)
    t = {k: dev(a) for k, a in v.items()}
    out = torch.full((tokens + 20, channels), 7.0, device="cuda")
    states = torch.full((5, channels, n), 3.0, device="cuda")
    for starts in ([-9, tokens, tokens // 3, 10 ** 6], [0, -1, -2, -3], [10 ** 9, 10 ** 9, 5, 9], [tokens, 0, tokens, 0]):
        cad.cadnn_selective_scan(t["x"], t["dt"], t["a"], t["b"], t["c"], softplus=True, state=states[1:4], seqs=3, out=out[10:10 + tokens],
                                 seq_start=torch.tensor(starts, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
    assert bool((out[:10] == 7.0).all()) and bool((out[10 + tokens:] == 7.0).all())
    assert bool((states[0] == 3.0).all()) and bool((states[4] == 3.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("tokens,seqs", [(900, 1), (900, 300)])
def test_rows_far_apart(dtype, tokens, seqs):
    """Offsets beyond 2^31 elements, in all tensors that have rows."""
    tt, flag, npt = TYPES[dtype]
    channels, n = 24, 16
    stride = 2 ** 31 // tokens + 4096
    lens = [tokens // seqs] * seqs
    starts = starts_of(lens)
    v = scan_inputs(lens, channels, n, 1, npt, 10)

    def far(a):
        a = dev(a.reshape(tokens, -1))
        w = torch.empty_strided(a.shape, (stride, 1), dtype=a.dtype, device="cuda")
        return w.copy_(a)

    t = {k: far(a) if k in ("x", "dt", "z", "b", "c") else dev(a) for k, a in v.items()}
    out = torch.empty_strided((tokens, channels), (stride, 1), dtype=tt, device="cuda")
    cad.cadnn_selective_scan(t["x"], t["dt"], t["a"], t["b"], t["c"], d=t["d"], z=t["z"], dt_bias=t["dt_bias"], softplus=True, state=t["state"],
                             seqs=seqs, out=out)
    ref, bound, last, off = scan_reference(v, starts, True, True)
    check(out, ref, bound, dtype)
    check(t["state"], last, off, "f32")
    g = np.random.default_rng(11)
    w = g.uniform(-1, 1, (channels, 4)).astype(npt).astype(np.float32)
    state = g.standard_normal((seqs, 3, channels)).astype(npt)
    h = cad.cadnn_pack_weights(w.reshape(channels, 1, 1, 4), flag)
    kept = dev(state)
    cad.cadnn_causal_conv1d(h, t["x"], kept, None, seqs, None, cad.ACT_SILU, out=out)
    ref, bound, last = conv_reference(v["x"], w, None, state, starts, cad.ACT_SILU)
    check(out, ref, bound, dtype)
    assert np.array_equal(kept.double().cpu().numpy(), last)
    h.free()


# ---- together ---------------------------------------------------------------------------------------

class Block:
    """in projection (4 bits) -> causal convolution, SiLU -> projections of dt, b, c (4 bits) -> gated scan -> out projection."""

    def __init__(self, dtype, width, channels, dstate, rank, seed):
        tt, flag, npt = TYPES[dtype]
        g = np.random.default_rng(seed)
        self.tt, self.width, self.channels, self.dstate, self.rank = tt, width, channels, dstate, rank
        q4 = lambda cout, cin: cad.cadnn_q4_pack((g.standard_normal((cout, cin)) / cin ** 0.5).astype(np.float32), 32, flag)
        self.w_in, self.w_proj = q4(2 * channels, width), q4(rank + 2 * dstate, channels)
        self.w_dt, self.w_out = q4(channels, rank), q4(width, channels)
        taps = g.uniform(-0.5, 0.5, (channels, 1, 1, 4)).astype(np.float32)
        self.w_conv = cad.cadnn_pack_weights(taps, flag)
        self.taps = cad.cadnn_unpack_weights(self.w_conv).reshape(channels, 4)
        self.conv_bias = (g.standard_normal(channels) * 0.1).astype(np.float32)
        self.a = -g.uniform(0.5, dstate, (channels, dstate)).astype(np.float32)
        self.d, self.dt_bias = np.ones(channels, np.float32), g.uniform(-6, -2, channels).astype(np.float32)
        self.on = {k: dev(getattr(self, k)) for k in ("conv_bias", "a", "d", "dt_bias")}

    def states(self, seqs):
        return (torch.zeros(seqs, 3, self.channels, dtype=self.tt, device="cuda"),
                torch.zeros(seqs, self.channels, self.dstate, device="cuda"))

    def run(self, x, states, seq_start, seqs):
        conv, scan = states
        c, r, n = self.channels, self.rank, self.dstate
        xz = cad.cadnn_q4_fc(self.w_in, x)
        u = cad.cadnn_causal_conv1d(self.w_conv, xz[:, :c], conv, seq_start, seqs, self.on["conv_bias"], cad.ACT_SILU)
        proj = cad.cadnn_q4_fc(self.w_proj, u)
        dt = cad.cadnn_q4_fc(self.w_dt, proj[:, :r])
        y = cad.cadnn_selective_scan(u, dt, self.on["a"], proj[:, r:r + n], proj[:, r + n:], d=self.on["d"], z=xz[:, c:],
                                     dt_bias=self.on["dt_bias"], softplus=True, state=scan, seq_start=seq_start, seqs=seqs)
        return cad.cadnn_q4_fc(self.w_out, y)

    def reference(self, x, starts):
        c, r, n = self.channels, self.rank, self.dstate
        back = lambda h: cad.cadnn_q4_unpack(h).astype(np.float64)
        seqs = len(starts) - 1
        xz = x.astype(np.float64) @ back(self.w_in).T
        u, _, _ = conv_reference(xz[:, :c], self.taps, self.conv_bias, np.zeros((seqs, 3, c)), starts, cad.ACT_SILU)
        proj = u @ back(self.w_proj).T
        dt = proj[:, :r] @ back(self.w_dt).T
        v = {"x": u, "dt": dt, "z": xz[:, c:], "b": proj[:, None, r:r + n], "c": proj[:, None, r + n:], "a": self.a, "d": self.d,
             "dt_bias": self.dt_bias, "state": np.zeros((seqs, c, n))}
        y, _, last, _ = scan_reference(v, starts, True, True)
        return y @ back(self.w_out).T, last


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("f16", 1e-2)])
def test_block_prompt_then_single_tokens(dtype, tol):
    """Ragged prompts in one call and then tokens one by one, as a server runs them, give what the definition gives for the whole
    sequences; the tolerance is the library's for chained layers, relative to the largest output."""
    tt, flag, npt = TYPES[dtype]
    block = Block(dtype, 96, 160, 16, 8, 1)
    g = np.random.default_rng(2)
    lens, more = [70, 1, 200, 13], 3
    whole = [g.standard_normal((m + more, 96)).astype(npt) for m in lens]
    ref, last = block.reference(np.concatenate(whole), starts_of([m + more for m in lens]))
    ref = np.split(ref, np.cumsum([m + more for m in lens])[:-1])
    states = block.states(4)
    got = block.run(dev(np.concatenate([w[:m] for w, m in zip(whole, lens)])), states, dev(starts_of(lens)), 4)
    parts = [list(p) for p in torch.split(got, lens)]
    for k in range(more):
        y = block.run(dev(np.stack([w[m + k] for w, m in zip(whole, lens)])), states, None, 4)
        for i in range(4):
            parts[i].append(y[i])
    top = max(np.abs(r).max() for r in ref)
    for p, r in zip(parts, ref):
        assert np.abs(torch.stack(p).double().cpu().numpy() - r).max() <= tol * top
    assert np.abs(states[1].double().cpu().numpy() - last).max() <= tol * np.abs(last).max()


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [3, 600])
def test_block_replayed_as_a_graph(tokens):
    """Two graphs of one block (each with memory of its own), replayed in turn with eager calls between them."""
    block = Block("f16", 64, 128, 16, 8, 3)
    seqs = 3 if tokens == 3 else 1
    x = torch.randn(tokens, 64, device="cuda").half()
    block.run(x, block.states(seqs), None, seqs)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        states, graph = block.states(seqs), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = block.run(x, states, None, seqs)
        graphs.append((graph, states, y))
    eager = block.states(seqs)
    for _, states, _ in graphs:
        for s in states:
            s.zero_()
    for k in range(3):
        x.copy_(torch.randn(tokens, 64, device="cuda").half())
        want = block.run(x, eager, None, seqs)
        for graph, states, y in graphs:
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
            assert all(torch.equal(s, e) for s, e in zip(states, eager))


@pytest.mark.gpu
def test_two_streams_at_once():
    block = Block("f32", 64, 128, 16, 8, 3)
    xs = [torch.randn(400, 64, device="cuda") for _ in range(2)]
    want = [block.run(x, block.states(1), None, 1) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = []
    for s, x in zip(streams, xs):
        with torch.cuda.stream(s):
            got.append(block.run(x, block.states(1), None, 1))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # the same through the calls' own argument
    v = scan_inputs([500], 64, 16, 1, np.float32, 6)
    t = {k: dev(a) for k, a in v.items()}
    args = (t["x"], t["dt"], t["a"], t["b"], t["c"])
    one = cad.cadnn_selective_scan(*args, softplus=True)
    torch.cuda.synchronize()
    other = cad.cadnn_selective_scan(*args, softplus=True, stream=streams[0])
    streams[0].synchronize()
    assert torch.equal(one, other)


# ---- refusals (no GPU needed: the checks come first) --------------------------------------------------

def test_causal_conv1d_refusals():
    L = cad.lib()
    h = cad.cadnn_pack_weights(np.ones((6, 1, 1, 4), np.float32))
    nine = cad.cadnn_pack_weights(np.ones((6, 1, 1, 9), np.float32))
    full = cad.cadnn_pack_weights(np.ones((6, 2, 1, 4), np.float32))
    tall = cad.cadnn_pack_weights(np.ones((6, 1, 2, 2), np.float32))
    p = [ctypes.c_void_p(1 << (10 + k)) for k in range(4)]           # never dereferenced

    def call(w=h, x=p[0], xs=6, y=p[1], ys=6, tokens=10, seqs=2, start=None, state=p[2], bias=None, act=0):
        return L.cadnn_causal_conv1d(None if w is None else w.handle, x, xs, y, ys, tokens, seqs, start, state, bias, act, None)

    assert call(w=None) == 1 and call(w=full) == 1 and call(w=tall) == 1 and call(w=nine) == 2
    assert call(tokens=-1) == 1 and call(seqs=0) == 1 and call(tokens=11) == 1 and b"one length" in L.cadnn_last_error()
    assert call(tokens=(1 << 30) + 2) == 2 and call(seqs=(1 << 24) + 1, start=p[3]) == 2
    assert call(x=None) == 1 and call(y=None) == 1 and call(y=p[0]) == 1 and call(state=p[0]) == 1 and call(state=p[1]) == 1
    assert call(xs=5) == 1 and call(ys=5) == 1 and call(act=3) == 1 and call(act=-1) == 1
    assert call(x=ctypes.c_void_p(1026)) == 1 and call(start=ctypes.c_void_p(1026)) == 1
    assert call(tokens=0, x=None, y=None) == 0                         # nothing to do
    for w in (h, nine, full, tall):
        w.free()


def test_selective_scan_refusals():
    L = cad.lib()
    nbytes = ctypes.c_size_t(3)

    def args(**changed):
        g = cad.binding.ScanArgs()
        for k, v in dict(dtype=0, tokens=10, seqs=2, channels=6, dstate=16, groups=2, softplus=1, x=1 << 10, dt=1 << 11, b=1 << 12, c=1 << 13, y=1 << 14,
                         x_stride=6, dt_stride=6, b_stride=32, c_stride=32, y_stride=6, a=1 << 15, **changed).items():
            setattr(g, k, v)
        return g

    def args2(**changed):
        g = args()
        for k, v in changed.items():
            setattr(g, k, v)
        return ctypes.byref(g)

    def call(**changed):
        return L.cadnn_selective_scan(args2(**changed), None, 0, None)

    assert L.cadnn_selective_scan(None, None, 0, None) == 1
    for bad in (dict(dtype=5), dict(tokens=-1), dict(seqs=0), dict(tokens=11), dict(channels=0), dict(dstate=0), dict(groups=0), dict(groups=4), dict(x=None), dict(dt=None),
                dict(a=None), dict(b=None), dict(c=None), dict(y=None), dict(y=1 << 10), dict(y=1 << 11), dict(y=1 << 12), dict(x_stride=5), dict(dt_stride=0), dict(y_stride=5),
                dict(b_stride=31), dict(c_stride=16), dict(z=1 << 16, z_stride=3), dict(x=1026), dict(state=1026), dict(longest=-1), dict(seq_start=1025), dict(state=1 << 14)):
        assert call(**bad) == 1, bad
    for big in (dict(dstate=257, b_stride=600, c_stride=600), dict(channels=(1 << 20) + 2, x_stride=1 << 21, dt_stride=1 << 21, y_stride=1 << 21), dict(seqs=65536, seq_start=1 << 17),
                dict(groups=5000, channels=5000), dict(tokens=(1 << 30) + 2)):
        assert call(**big) == 2, big
    assert call(tokens=0, x=None) == 0
    ws = L.cadnn_selective_scan_workspace_bytes
    assert ws(args2(), None) == 1 and ws(None, ctypes.byref(nbytes)) == 1 and nbytes.value == 0
    assert ws(args2(), ctypes.byref(nbytes)) == 0 and nbytes.value == 0                                   # short sequences
    assert ws(args2(tokens=4096, seqs=1), ctypes.byref(nbytes)) == 0 and nbytes.value > 0
    many = nbytes.value
    assert ws(args2(tokens=4096, seqs=1, channels=600), ctypes.byref(nbytes)) == 0 and nbytes.value > many
    assert ws(args2(tokens=0, seqs=1), ctypes.byref(nbytes)) == 0 and nbytes.value == 0


def test_sequence_wrappers_refuse_tensors_that_do_not_fit():
    x = torch.ones(4, 6)
    h = cad.cadnn_pack_weights(np.ones((6, 1, 1, 4), np.float32))
    with pytest.raises(ValueError):
        cad.cadnn_causal_conv1d(h, x)                 # not on a GPU
    with pytest.raises(ValueError):
        cad.cadnn_causal_conv1d(h, torch.ones(4, 5))
    with pytest.raises(ValueError):
        cad.cadnn_selective_scan(x, x, torch.ones(6, 3), torch.ones(4, 3), torch.ones(4, 3))
    h.free()
