"""Which kernel serves a fully connected layer with 4-bit weights."""
import ctypes

import numpy as np
import pytest

import paper_1905_00571_amd as cad

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
