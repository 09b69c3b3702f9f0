"""Which kernel serves a fully connected layer with 4-bit weights, and every one of them against the definition.

The bounds are those of test_gpu_q4.py."""
import ctypes

import numpy as np
import pytest
import torch

import paper_1905_00571_amd as cad
from test_gpu_q4 import TYPES, check, layer, reference


def dev(v):
    return torch.from_numpy(np.ascontiguousarray(v)).cuda()


# (what a handle of zeros costs is its size alone: the choice goes by sizes, type and alignment)


def blank(cout, cin, group, dtype):
    return cad.cadnn_q4_pack_codes(np.zeros((cout, cin), np.int8), np.ones((cout, -(-cin // group)), np.float32), group, cad.F16 if dtype == "f16" else cad.F32)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_tile_through_registers_is_chosen_for_some_layer(group):
    """fp16 rows that cannot go straight to LDS: an odd number of inputs, a row length or an address that is no multiple of 16 bytes."""
    names = {}
    for cout in (515, 4095):
        h = blank(cout, 391, group, "f16")
        for n in (33, 64, 300, 400, 515, 2047):
            names[n, cout] = cad.cadnn_q4_fc_variant_name(h, n)
        h.free()
    assert {"tile_64x32", "tile_128x64", "tile_128x64_whole"} <= set(names.values())
    assert names[2047, 4095] == "tile_128x64_whole" and names[33, 515].startswith("few_")
    h = blank(4096, 392, group, "f16")
    straight = cad.cadnn_q4_fc_variant_name(h, 2047)
    assert straight == "tile_128x128_lds"
    for how in ({"x_stride": 393}, {"address": 8}, {"x_stride": 1 << 22}):
        assert cad.cadnn_q4_fc_variant_name(h, 2047, **how) == "tile_128x64_whole"
    assert cad.cadnn_q4_fc_variant_name(h, 2047, x_stride=400, address=32) == straight
    h.free()


def test_variant_name_refusals():
    h = blank(8, 40, 32, "f32")
    f, buf = cad.lib().cadnn_q4_fc_variant_name, ctypes.create_string_buffer(4)
    assert f(None, None, 40, 1, buf, 4) == 1 and f(h.handle, None, 40, 1, None, 4) == 1 and f(h.handle, None, 40, 1, buf, 0) == 1
    assert f(h.handle, None, 40, 0, buf, 4) == 1 and f(h.handle, None, 39, 1, buf, 4) == 1
    assert f(h.handle, None, 40, 1, buf, 4) == 0 and buf.value == b"few"            # cut to the buffer, as the other names are
    h.free()


# ---- every kernel against the definition ---------------------------------------------------------------

# (rows, filters) by kernel, chosen for all three group sizes; neither is a multiple of a tile's
KERNELS = {"f32": {"columns_4": (3, 515), "columns_5": (5, 33), "few_16x16": (3, 33), "few_32x16": (17, 2051), "few_64x16": (17, 4099), "few_64x32": (33, 8190),
                   "tile_128x32": (100, 5003), "tile_256x32": (200, 5003), "tile_256x64": (1501, 2051)},
           "f16": {"columns_4": (1, 515), "columns_16": (13, 33), "few_16x16": (3, 33), "few_32x16": (17, 2051), "few_64x16": (17, 4099),
                   "tile_64x32_lds": (1501, 130), "tile_128x64_lds": (1300, 3001), "tile_128x128_lds": (1000, 6002),
                   "tile_64x32": (1501, 130), "tile_128x64": (300, 5003), "tile_128x64_whole": (300, 8190)}}
ALL = [(d, k) for d in KERNELS for k in KERNELS[d]]


def widths(kernel):
    """Numbers of inputs: a last block of its own size, one block alone, whole blocks.  (Staged columns serve long rows only, copies straight to
    LDS multiples of eight.)"""
    return (2057, 2100, 2304) if kernel.startswith("columns") else (392, 104, 512) if kernel.endswith("_lds") else (391, 97, 512)


def case(dtype, kernel, cin, group, seed):
    """Weights, rows, bias, and the handle, which `kernel` serves."""
    n, cout = KERNELS[dtype][kernel]
    codes, scales = layer(cout, cin, group, dtype, seed)
    g = np.random.default_rng(seed + 1)
    x = g.standard_normal((n, cin)).astype(np.float16 if dtype == "f16" else np.float32)
    return codes, scales, x, g.standard_normal(cout).astype(np.float32), cad.cadnn_q4_pack_codes(codes, scales, group, TYPES[dtype][1])


def aligned(kernel, cin):
    """A row length, in elements, for rows that lie apart, and the first row's offset: as the kernel needs them, or odd ones."""
    return (cin + 24, 8) if kernel.endswith("_lds") else (cin + 8 - cin % 2, 3)


def named(h, kernel, x):
    return cad.cadnn_q4_fc_variant_name(h, x.shape[0], x.stride(0), x.data_ptr()) == kernel


def test_every_kernel_is_among_those_tested():
    """The rules' kernels over many sizes are those that KERNELS names, for every type and group size."""
    for dtype in KERNELS:
        for group in (32, 64, 128):
            seen = set()
            for cout in (33, 130, 777, 2051, 3001, 4099, 5003, 6002, 8190):
                for cin in (391, 392, 2057):
                    h = blank(cout, cin, group, dtype)
                    seen |= {cad.cadnn_q4_fc_variant_name(h, n) for n in (1, 3, 5, 13, 17, 33, 64, 100, 129, 200, 300, 600, 1000, 1300, 1501, 2047)}
                    h.free()
            assert seen == set(KERNELS[dtype]), (dtype, group)


@pytest.mark.gpu
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype,kernel", ALL)
def test_every_kernel(dtype, kernel, group):
    for i, cin in enumerate(widths(kernel)):
        codes, scales, x, bias, h = case(dtype, kernel, cin, group, 31 + i)
        xd = dev(x)
        if dtype == "f16" and kernel.startswith("tile") and not kernel.endswith("_lds") and cin % 8 == 0:
            xd = torch.nn.functional.pad(xd, (0, 1))[:, :cin]          # (rows that cannot go straight to LDS)
        assert named(h, kernel, xd)
        act = [cad.ACT_SILU, cad.ACT_NONE, cad.ACT_RELU][(i + group // 32) % 3]
        b = bias if i != 1 else None
        y = cad.cadnn_q4_fc(h, xd, None if b is None else dev(b), act)
        ref, mag = reference(codes, scales, group, x, b, act)
        check(y, ref, mag, cin, dtype, f"{kernel}, {cin} inputs, groups of {group}, act {act}")
        h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kernel", ALL)
def test_every_kernel_on_slices_of_wider_rows(dtype, kernel):
    """Rows apart in x and y: what lies between them is no number in x, and stays in y."""
    tt = TYPES[dtype][0]
    cin = widths(kernel)[0]
    codes, scales, x, bias, h = case(dtype, kernel, cin, 64, 41)
    n, cout = KERNELS[dtype][kernel]
    length, at = aligned(kernel, cin)
    wide = torch.full((n, length), float("nan"), dtype=tt, device="cuda")
    view = wide[:, at:at + cin]
    view.copy_(dev(x))
    assert named(h, kernel, view)
    out = torch.full((n, cout + 9), 7.0, dtype=tt, device="cuda")
    cad.cadnn_q4_fc(h, view, dev(bias), out=out[:, 5:5 + cout])
    ref, mag = reference(codes, scales, 64, x, bias, cad.ACT_NONE)
    check(out[:, 5:5 + cout], ref, mag, cin, dtype, kernel)
    assert bool((out[:, :5] == 7.0).all()) and bool((out[:, 5 + cout:] == 7.0).all())
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kernel", ALL)
def test_every_kernel_keeps_values_that_are_not_finite_to_their_row(dtype, kernel):
    cin = widths(kernel)[0]
    codes, scales, x, _, h = case(dtype, kernel, cin, 32, 51)
    n = len(x)
    ref, mag = reference(codes, scales, 32, x, None, cad.ACT_NONE)
    sign = torch.where(torch.from_numpy(codes[:, cin - 1]) > 0, float("inf"), float("-inf"))
    moved = codes[:, cin - 1] != 0
    for row in {0, n // 2, n - 1}:
        for value in (np.inf, np.nan):
            v = x.copy()
            v[row, cin - 1] = value
            y = cad.cadnn_q4_fc(h, dev(v)).float().cpu()
            others = [r for r in {0, n // 2, n - 1, max(row - 1, 0), min(row + 1, n - 1)} if r != row]
            if others:
                check(y[others], ref[others], mag[others], cin, dtype, kernel)
            assert bool(torch.isfinite(y[[r for r in range(n) if r != row]]).all())
            if value == np.inf:                    # (a code of zero meets it: no number)
                assert torch.equal(y[row][moved], sign[moved]) and bool(torch.isnan(y[row][~moved]).all())
            else:
                assert bool(torch.isnan(y[row]).all())
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kernel", ALL)
def test_every_kernel_on_rows_far_apart(dtype, kernel):
    """Offsets beyond 2^31 bytes in x and beyond 2^31 elements in y (copies straight to LDS: rows as far apart as they serve)."""
    tt = TYPES[dtype][0]
    cin = widths(kernel)[0]
    codes, scales, x, _, h = case(dtype, kernel, cin, 128, 61)
    n, cout = KERNELS[dtype][kernel]
    stride = (1 << 22) - 8 if kernel.endswith("_lds") else 2 ** 31 // n + 4097
    view = torch.empty_strided((n, cin), (stride, 1), dtype=tt, device="cuda")
    out = torch.empty_strided((n, cout), (2 ** 31 // n + 8192, 1), dtype=tt, device="cuda")
    view.copy_(dev(x))
    assert named(h, kernel, view)
    cad.cadnn_q4_fc(h, view, out=out)
    ref, mag = reference(codes, scales, 128, x, None, cad.ACT_NONE)
    check(out, ref, mag, cin, dtype, kernel)
    h.free()
