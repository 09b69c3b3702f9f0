"""Fully connected layers with 4-bit weights and group scales against the definition in 64 bits.

Bounds.  Codes are exact, a group's sum of k products is an fp32 sum and so is the sum over groups, so with any order of
additions |error| <= (cin + 4) * 2^-24 * A, A = sum |s q x| + |bias|; the orders used here add at most eight waves' parts of
trees over 32 products and stay far below (16 + sqrt(cin)) * 2^-24 * A, which is what is asked.  A result stored in fp16 is
off by half a step, 2^-11 of its value, more.  SiLU multiplies an error by at most 1.1 and adds 2^-22 of the value."""
import ctypes

import numpy as np
import pytest
import torch

import paper_1905_00571_amd as cad

TYPES = {"f32": (torch.float32, cad.F32), "f16": (torch.float16, cad.F16)}


def layer(cout, cin, group, dtype, seed):
    g = np.random.default_rng(seed)
    codes = np.clip(np.rint(g.standard_normal((cout, cin)) * 3), -8, 7).astype(np.int8)
    scales = (g.uniform(0.2, 1.0, (cout, -(-cin // group))) / cin ** 0.5).astype(np.float32)
    if dtype == "f16":
        scales = scales.astype(np.float16).astype(np.float32)
    return codes, scales


def reference(codes, scales, group, x, bias, act):
    w = codes.astype(np.float64) * np.repeat(scales.astype(np.float64), group, 1)[:, :codes.shape[1]]
    y = x.astype(np.float64) @ w.T
    mag = np.abs(x).astype(np.float64) @ np.abs(w).T
    if bias is not None:
        y, mag = y + bias, mag + np.abs(bias)
    if act == cad.ACT_RELU:
        y = np.maximum(y, 0)
    if act == cad.ACT_SILU:
        y = y / (1 + np.exp(-y))
    return y, mag


def check(y, ref, mag, cin, dtype, what=""):
    got = y.double().cpu().numpy()
    bound = 1.1 * (16 + cin ** 0.5) * 2.0 ** -24 * mag + (2.0 ** -11 * np.abs(ref) + 2.0 ** -25 if dtype == "f16" else 2.0 ** -22 * np.abs(ref)) + 1e-30
    d = np.abs(got - ref)
    assert np.isfinite(got).all(), what
    assert (d <= bound).all(), f"{what}: {int((d > bound).sum())} beyond the bound, worst {float((d / bound).max()):.2f}"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,cin,cout", [(1, 1, 1), (1, 128, 16), (1, 2048, 1000), (2, 127, 33), (3, 129, 17), (5, 1000, 4099), (13, 5003, 70),
                                        (16, 256, 48), (17, 260, 50), (33, 1536, 257), (64, 640, 130), (65, 384, 100), (100, 4100, 64),
                                        (129, 512, 512), (300, 96, 1030), (1000, 777, 300)])
def test_q4_fc(dtype, group, n, cin, cout):
    tt, flag = TYPES[dtype]
    codes, scales = layer(cout, cin, group, dtype, 7 * cin + cout + group)
    g = np.random.default_rng(cin + n)
    x = torch.from_numpy(g.standard_normal((n, cin)).astype(np.float32)).to(tt)
    bias = g.standard_normal(cout).astype(np.float32)
    h = cad.cadnn_q4_pack_codes(codes, scales, group, flag)
    act = [cad.ACT_NONE, cad.ACT_RELU, cad.ACT_SILU][(n + cin + cout) % 3]
    for b in (bias, None):
        y = cad.cadnn_q4_fc(h, x.cuda(), None if b is None else torch.from_numpy(b).cuda(), act)
        ref, mag = reference(codes, scales, group, x.float().numpy(), b, act)
        check(y, ref, mag, cin, dtype, f"n {n}, {cin} -> {cout}, groups of {group}, act {act}")
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n,cin,cout,pad_x,off_x,pad_y,off_y", [(3, 256, 64, 24, 8, 16, 4), (70, 256, 64, 24, 8, 16, 4), (2, 130, 50, 3, 1, 5, 1),
                                                                (90, 391, 65, 1, 1, 3, 1), (200, 512, 256, 7, 3, 0, 0), (200, 512, 256, 0, 0, 2, 1)])
def test_q4_fc_slices_of_wider_rows(dtype, n, cin, cout, pad_x, off_x, pad_y, off_y):
    """Strided and misaligned rows; what lies between the rows of y stays, and what lies between those of x is not read
    (it holds values that are no numbers)."""
    tt, flag = TYPES[dtype]
    codes, scales = layer(cout, cin, 64, dtype, 5)
    g = np.random.default_rng(6)
    wide = torch.full((n, cin + pad_x + off_x), float("nan"), dtype=tt, device="cuda")
    x = torch.from_numpy(g.standard_normal((n, cin)).astype(np.float32)).to(tt)
    wide[:, off_x:off_x + cin] = x.cuda()
    out = torch.full((n, cout + pad_y + off_y), 7.0, dtype=tt, device="cuda")
    h = cad.cadnn_q4_pack_codes(codes, scales, 64, flag)
    cad.cadnn_q4_fc(h, wide[:, off_x:off_x + cin], out=out[:, off_y:off_y + cout])
    ref, mag = reference(codes, scales, 64, x.float().numpy(), None, cad.ACT_NONE)
    check(out[:, off_y:off_y + cout], ref, mag, cin, dtype)
    rest = torch.cat([out[:, :off_y], out[:, off_y + cout:]], 1)
    assert bool((rest == 7.0).all())
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n", [1, 20, 200])
def test_q4_fc_values_that_are_not_finite_reach_their_row_alone(dtype, n):
    tt, flag = TYPES[dtype]
    cin, cout = 300, 40
    codes, scales = layer(cout, cin, 32, dtype, 9)
    codes[:, 5] = np.where(codes[:, 5] == 0, 3, codes[:, 5])
    x = torch.from_numpy(np.random.default_rng(10).standard_normal((n, cin)).astype(np.float32)).to(tt)
    x[0, 5] = float("inf")
    h = cad.cadnn_q4_pack_codes(codes, scales, 32, flag)
    y = cad.cadnn_q4_fc(h, x.cuda()).cpu()
    assert torch.equal(y[0], torch.where(torch.from_numpy(codes[:, 5]) > 0, float("inf"), float("-inf")).to(tt))
    if n > 1:
        ref, mag = reference(codes, scales, 32, x[1:].float().numpy(), None, cad.ACT_NONE)
        check(y[1:], ref, mag, cin, dtype)
    x[0, 5] = float("nan")
    assert bool(torch.isnan(cad.cadnn_q4_fc(h, x.cuda())[0]).all())
    if dtype == "f32":              # the largest values stay finite where their products are
        x[0] = 0.0
        x[0, 5] = torch.finfo(tt).max
        y = cad.cadnn_q4_fc(h, x.cuda()).double().cpu().numpy()
        ref, mag = reference(codes, scales, 32, x.float().numpy(), None, cad.ACT_NONE)
        fine = np.abs(codes[:, 5].astype(np.float64) * float(x[0, 5])) <= torch.finfo(tt).max     # (a code of one: the product is that value itself)
        d = np.abs(y[0] - ref[0])[fine]
        assert fine.any() and (d <= 1e-6 * mag[0][fine]).all()
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_q4_pack_on_the_gpu_is_what_unpack_says(dtype):
    tt, flag = TYPES[dtype]
    g = np.random.default_rng(3)
    w = (g.standard_normal((75, 200)) * 0.1).astype(np.float32)
    h = cad.cadnn_q4_pack(w, 64, flag)
    x = torch.from_numpy(g.standard_normal((4, 200)).astype(np.float32)).to(tt)
    y = cad.cadnn_q4_fc(h, x.cuda())
    back = cad.cadnn_q4_unpack(h).astype(np.float64)
    xd = x.double().numpy()
    check(y, xd @ back.T, np.abs(xd) @ np.abs(back).T, 200, dtype)
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 100])
def test_q4_fc_on_another_stream_and_in_a_graph(n):
    codes, scales = layer(500, 1000, 128, "f16", 4)
    h = cad.cadnn_q4_pack_codes(codes, scales, 128, cad.F16)
    x = torch.randn(n, 1000, device="cuda").half()
    bias = torch.randn(500, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(cad.CadnnError, match="captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            cad.cadnn_q4_fc(h, x, bias)
    torch.cuda.synchronize()
    eager = cad.cadnn_q4_fc(h, x, bias)
    side.wait_stream(torch.cuda.current_stream())
    y = cad.cadnn_q4_fc(h, x, bias, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(eager, y)
    with torch.cuda.graph(graph):
        z = cad.cadnn_q4_fc(h, x, bias, cad.ACT_RELU)
    for k in range(3):
        x.copy_(torch.randn(n, 1000, device="cuda").half())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, cad.cadnn_q4_fc(h, x, bias, cad.ACT_RELU))
    h.free()


def test_q4_pack_codes_round_trip():
    for dtype, flag in (("f32", cad.F32), ("f16", cad.F16)):
        for cout, cin, group in ((1, 1, 32), (3, 33, 32), (5, 256, 128), (17, 131, 64)):
            codes, scales = layer(cout, cin, group, dtype, cin)
            h = cad.cadnn_q4_pack_codes(codes, scales, group, flag)
            got = cad.cadnn_q4_export(h)
            assert np.array_equal(got["codes"], codes) and np.array_equal(got["scales"], scales)
            assert np.array_equal(cad.cadnn_q4_unpack(h), codes.astype(np.float32) * np.repeat(scales, group, 1)[:, :cin])
            h.free()


@pytest.mark.parametrize("flag", [cad.F32, cad.F16])
def test_q4_pack_takes_the_nearest_code(flag):
    g = np.random.default_rng(1)
    w = g.standard_normal((9, 300)).astype(np.float32)
    w[2] = 0.0
    w[3, :64] *= 1e-3
    h = cad.cadnn_q4_pack(w, 64, flag)
    e = cad.cadnn_q4_export(h)
    s = np.repeat(e["scales"], 64, 1)[:, :300]
    assert (e["scales"][2] == 0).all() and (e["codes"][2] == 0).all()
    top = np.abs(np.pad(w, ((0, 0), (0, 20))).reshape(9, 5, 64)).max(2) / np.float32(7)
    # one rounding of the quotient, and one to the storage type
    assert (np.abs(e["scales"] - top) <= (2.0 ** -11 if flag == cad.F16 else 2.0 ** -23) * top).all()
    back = cad.cadnn_q4_unpack(h)
    assert (np.abs(back - w) <= s * np.float32(0.5 + 7 * 2.0 ** -10)).all()      # half a code, and what the scale's rounding costs the largest
    h.free()


def test_q4_refusals():
    L = cad.lib()
    out = ctypes.c_void_p(5)
    w = np.ones((2, 40), np.float32)
    pw = w.ctypes.data_as(ctypes.POINTER(ctypes.c_float))
    codes = np.ones((2, 40), np.int8)
    pc = codes.ctypes.data_as(ctypes.POINTER(ctypes.c_int8))
    assert L.cadnn_q4_pack(None, 2, 40, 32, 0, ctypes.byref(out)) == 1 and out.value is None
    assert L.cadnn_q4_pack(pw, 2, 40, 32, 0, None) == 1
    assert L.cadnn_q4_pack(pw, 0, 40, 32, 0, ctypes.byref(out)) == 1
    assert L.cadnn_q4_pack(pw, 2, -1, 32, 0, ctypes.byref(out)) == 1
    assert L.cadnn_q4_pack(pw, 2, 40, 32, 9, ctypes.byref(out)) == 1
    for group in (0, 16, 33, 256, -32):
        assert L.cadnn_q4_pack(pw, 2, 40, group, 0, ctypes.byref(out)) == 2
    assert L.cadnn_q4_pack(pw, 2, (1 << 24) + 1, 32, 0, ctypes.byref(out)) == 2
    for bad in (np.inf, np.nan, 1e38):
        w[1, 3] = bad
        assert L.cadnn_q4_pack(pw, 2, 40, 32, 0, ctypes.byref(out)) == 1 and b"row 1" in L.cadnn_last_error()
    w[1, 3] = 1e6
    assert L.cadnn_q4_pack(pw, 2, 40, 32, 1, ctypes.byref(out)) == 1          # a scale beyond binary16
    for bad in (np.nan, np.inf, 2.0 ** 120):
        with pytest.raises(cad.CadnnError, match="scale 1"):
            cad.cadnn_q4_pack_codes(codes, np.array([[1, bad], [1, 1]]), 32)
    with pytest.raises(cad.CadnnError, match="finite"):
        cad.cadnn_q4_pack_codes(codes, np.full((2, 2), 7e4), 32, cad.F16)
    for bad in (8, -9, 127, -128):
        c = codes.copy()
        c[1, 39] = bad
        with pytest.raises(cad.CadnnError, match="row 1"):
            cad.cadnn_q4_pack_codes(c, np.ones((2, 2)), 32)
    with pytest.raises(ValueError):
        cad.cadnn_q4_pack_codes(codes.astype(np.int32) * 300, np.ones((2, 2)), 32)
    with pytest.raises(ValueError):
        cad.cadnn_q4_pack_codes(codes, np.ones((2, 1)), 32)
    with pytest.raises(ValueError):
        cad.cadnn_q4_pack(np.ones(8, np.float32))
    h = cad.cadnn_q4_pack_codes(codes, np.ones((2, 2)), 32)
    x, y = ctypes.c_void_p(64), ctypes.c_void_p(128)      # never dereferenced: the checks come first
    fc = L.cadnn_q4_fc
    assert fc(None, x, 40, y, 2, 1, None, 0, None) == 1
    assert fc(h.handle, None, 40, y, 2, 1, None, 0, None) == 1
    assert fc(h.handle, x, 40, None, 2, 1, None, 0, None) == 1
    assert fc(h.handle, x, 40, y, 2, 0, None, 0, None) == 1
    assert fc(h.handle, x, 39, y, 2, 1, None, 0, None) == 1
    assert fc(h.handle, x, 40, y, 1, 1, None, 0, None) == 1
    assert fc(h.handle, x, 40, y, 2, 1, None, 3, None) == 1 and b"activation" in L.cadnn_last_error()
    assert fc(h.handle, x, 40, x, 2, 1, None, 0, None) == 1
    assert fc(h.handle, ctypes.c_void_p(66), 40, y, 2, 1, None, 0, None) == 1
    assert fc(h.handle, x, 40, y, 2, (1 << 24) + 1, None, 0, None) == 2
    assert L.cadnn_q4_free(None) == 0 and L.cadnn_q4_prepare(None) == 1 and L.cadnn_q4_export(None, None, None) == 1
    assert L.cadnn_q4_unpack(h.handle, None) == 1
    h.free()


@pytest.mark.gpu
def test_q4_fc_refuses_tensors_that_do_not_fit():
    h = cad.cadnn_q4_pack_codes(np.ones((8, 40), np.int8), np.ones((8, 2)), 32)
    x = torch.ones(3, 40, device="cuda")
    for bad in (torch.ones(3, 39, device="cuda"), x.half(), torch.ones(40, 3, device="cuda").t(), x.cpu(), x[0]):
        with pytest.raises((ValueError, RuntimeError)):
            cad.cadnn_q4_fc(h, bad)
    with pytest.raises(ValueError):
        cad.cadnn_q4_fc(h, x, torch.ones(7, device="cuda"))
    with pytest.raises(ValueError):
        cad.cadnn_q4_fc(h, x, out=torch.ones(3, 8, device="cuda").half())
    with pytest.raises(cad.CadnnError):
        cad.cadnn_q4_fc(h, x[:0])
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_q4_fc_with_negative_and_vanishing_scales(dtype):
    tt, flag = TYPES[dtype]
    codes, scales = layer(50, 384, 128, dtype, 21)
    scales[::2, 1] *= -1
    scales[3:9] = 0.0
    scales[11] = 2.0 ** -24 if dtype == "f16" else 2.0 ** -140          # below the normal numbers
    h = cad.cadnn_q4_pack_codes(codes, scales, 128, flag)
    x = torch.from_numpy(np.random.default_rng(22).standard_normal((40, 384)).astype(np.float32)).to(tt)
    for n in (1, 40):
        y = cad.cadnn_q4_fc(h, x[:n].cuda())
        ref, mag = reference(codes, scales, 128, x[:n].float().numpy(), None, cad.ACT_NONE)
        rows = [r for r in range(50) if r != 11]
        check(y[:, rows], ref[:, rows], mag[:, rows], 384, dtype)
        # (row 11: sums of products below the normal numbers, rounded to their steps at most once a group and once in the end)
        step = 2.0 ** -24 if dtype == "f16" else 2.0 ** -149
        assert (np.abs(y[:, 11].double().cpu().numpy() - ref[:, 11]) <= 3 * step + 2.0 ** -10 * np.abs(ref[:, 11])).all()
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n", [("f16", 1100), ("f32", 600), ("f16", 9), ("f32", 4)])
def test_q4_fc_rows_far_apart(dtype, n):
    """Offsets beyond 2^31 elements, in x and in y."""
    tt, flag = TYPES[dtype]
    stride = 2 ** 31 // n + 4096 + (1 if n < 16 else 0)
    codes, scales = layer(130, 256, 64, dtype, 23)
    h = cad.cadnn_q4_pack_codes(codes, scales, 64, flag)
    values = torch.from_numpy(np.random.default_rng(24).standard_normal((n, 256)).astype(np.float32)).to(tt)
    x = torch.empty_strided((n, 256), (stride, 1), dtype=tt, device="cuda")
    out = torch.empty_strided((n, 130), (stride, 1), dtype=tt, device="cuda")
    x.copy_(values)
    cad.cadnn_q4_fc(h, x, out=out)
    ref, mag = reference(codes, scales, 64, values.float().numpy(), None, cad.ACT_NONE)
    check(out, ref, mag, 256, dtype)
    h.free()


@pytest.mark.gpu
@pytest.mark.parametrize("n,cin,cout", [(1500, 300, 2100), (2000, 512, 1024)])
def test_q4_fc_first_call_of_a_kernel_in_a_graph(n, cin, cout):
    """Prepared weights are enough for a call to be captured, whatever its kernel asks of the device."""
    codes, scales = layer(cout, cin, 32, "f32", 25)
    h = cad.cadnn_q4_pack_codes(codes, scales, 32, cad.F32)
    cad.cadnn_q4_prepare(h)
    x = torch.randn(n, cin, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = cad.cadnn_q4_fc(h, x, None, cad.ACT_SILU)
    for k in range(3):
        x.copy_(torch.randn(n, cin, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, cad.cadnn_q4_fc(h, x, None, cad.ACT_SILU))
    ref, mag = reference(codes, scales, 32, x.cpu().numpy(), None, cad.ACT_SILU)
    check(y, ref, mag, cin, "f32")
    h.free()


@pytest.mark.gpu
def test_q4_fc_from_two_threads_at_once():
    """The first calls on a handle, side by side: one of them uploads the weights, both use them."""
    import threading
    codes, scales = layer(600, 1024, 64, "f16", 26)
    x = torch.randn(20, 1024, device="cuda").half()
    for _ in range(3):
        h = cad.cadnn_q4_pack_codes(codes, scales, 64, cad.F16)
        torch.cuda.synchronize()
        got = [None, None]

        def work(i):
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                got[i] = cad.cadnn_q4_fc(h, x)
            s.synchronize()

        threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], cad.cadnn_q4_fc(h, x))
        h.free()
