"""GPU parity of the 8-bit floating-point operators against the numpy oracle: quantised matrices bit for bit in both orientations, products
within the bound that their additions have (f8_util.product_bound)."""
import numpy as np
import pytest
import torch

from oracle import f8
from paper_2407_09453_b200 import bsp, synth
from f8_util import FTYPE, XTYPE, codes_of, device, held, launches, product_bound, random_held, template, values

pytestmark = pytest.mark.gpu


def quantize_both(X, ftype, colsum=None, ldx=None):
    P, I = X.shape
    act = bsp.F8Activations(P, I, FTYPE[ftype])
    for m in (act.rows, act.cols):
        m.data.view(torch.uint8).fill_(0xEE)
        m.scale.fill_(0xEE)
    bsp.bsp_quantize_f8(X, bsp.dtype_code(X.dtype), P, I, I if ldx is None else ldx, act.rows.m, act.cols.m, colsum, act.ws)
    return act


def assert_forms(act, x, ftype):
    for m, t in ((act.rows, x), (act.cols, x.T)):
        codes, scales = f8.quantize(t, ftype)
        got_codes, got_scales = codes_of(m)
        assert np.array_equal(got_scales, scales)
        assert np.array_equal(got_codes, codes)


@pytest.mark.parametrize("P,I,dtype,ftype", [(1, 8, "bf16", "e4m3"), (1, 1, "f32", "e5m2"), (128, 128, "bf16", "e4m3"), (127, 129, "f32", "e4m3"), (130, 200, "bf16", "e5m2"),
                                             (64, 2048, "bf16", "e4m3"), (5, 1003, "bf16", "e4m3"), (300, 77, "f32", "e5m2"), (1023, 264, "bf16", "e4m3")])
def test_quantize_both_orientations(P, I, dtype, ftype):
    x = values(2000 + P, P, I, dtype)
    act = quantize_both(device(x, dtype), ftype)
    assert_forms(act, x, ftype)


def test_quantize_one_orientation_leaves_the_other():
    x = values(2100, 140, 300, "bf16")
    X = device(x, "bf16")
    for which in ("rows", "cols"):
        act = bsp.F8Activations(140, 300)
        other = act.cols if which == "rows" else act.rows
        other.data.view(torch.uint8).fill_(0xAB)
        bsp.bsp_quantize_f8(X, bsp.BF16, 140, 300, 300, act.rows.m if which == "rows" else None, act.cols.m if which == "cols" else None, None, None)
        codes, scales = f8.quantize(x if which == "rows" else x.T, "e4m3")
        got = codes_of(getattr(act, which))
        assert np.array_equal(got[0], codes) and np.array_equal(got[1], scales)
        assert bool((other.data.view(torch.uint8) == 0xAB).all())


@pytest.mark.parametrize("dtype,off,ldx", [("bf16", 0, 264), ("bf16", 3, 261), ("f32", 0, 260), ("f32", 1, 259), ("bf16", 8, 512)])
def test_quantize_strides_and_alignment(dtype, off, ldx):
    """Rows that are not packed and buffers that start off a 16-byte boundary; what lies between the rows is not read as data."""
    P, I = 133, 250
    x = values(2200 + off, P, I, dtype)
    store = torch.full((P * ldx + off,), float("nan"), dtype=XTYPE[dtype], device="cuda")
    view = torch.as_strided(store, (P, I), (ldx, 1), off)
    view.copy_(device(x, dtype))
    act = quantize_both(view, "e4m3", None, ldx)
    assert_forms(act, x, "e4m3")


@pytest.mark.parametrize("ftype", ["e4m3", "e5m2"])
def test_quantize_extremes(ftype):
    """Blocks of zeros, NaN and infinities (NaN in 8 bits, in no scale), subnormals, the largest floats, entries exactly at a scale's border."""
    x = values(2300, 256, 384, "f32")
    x[0] = 0.0
    x[:, 1] = 0.0
    x[3, 5], x[3, 200], x[7, 300] = np.nan, np.inf, -np.inf
    x[9] = np.nan
    x[11] = np.inf
    x[13] = 2.0 ** -149
    x[15] = np.finfo(np.float32).max
    x[17, :128] = f8.MAX[ftype]
    x[18, :128] = np.nextafter(np.float32(f8.MAX[ftype]), np.float32(np.inf))
    x[19, :128] = np.float32(2.0 ** -126)
    act = quantize_both(device(x, "f32"), ftype)
    assert_forms(act, x, ftype)


@pytest.mark.parametrize("P,I,dtype", [(1, 16, "bf16"), (129, 100, "f32"), (1500, 513, "bf16")])
def test_column_sums(P, I, dtype):
    x = values(2400 + P, P, I, dtype)
    sums = torch.full((I,), float("nan"), device="cuda")
    act = quantize_both(device(x, dtype), "e4m3", sums)
    assert_forms(act, x, "e4m3")
    want = x.astype(np.float64).sum(0)
    # a sum of P terms, at most 8 + 16 + tiles additions deep, each off by half a step of what can have been summed
    depth = 8 + 1 + 8 + -(-P // 1024) + 8
    assert (np.abs(sums.cpu().numpy() - want) <= depth * 2.0 ** -24 * np.abs(x.astype(np.float64)).sum(0) * 1.01).all()
    again = torch.empty_like(sums)
    bsp.bsp_quantize_f8(device(x, dtype), bsp.dtype_code(XTYPE[dtype]), P, I, I, act.rows.m, None, again, act.ws)
    assert torch.equal(again, sums)                                       # always the same order


@pytest.mark.parametrize("O,I,bo,bi,dtype", [(8, 8, 8, 8, "bf16"), (136, 264, 8, 8, "f32"), (1000, 304, 4, 16, "bf16"), (272, 132, 16, 4, "f32"), (128, 128, 8, 8, "bf16")])
def test_quantize_weights(O, I, bo, bi, dtype):
    w = values(2500 + O, O, I, dtype, 0.05)
    gamma = synth.random_gamma(2501, O // bo, I // bi, (O // bo) * (I // bi) // 2)
    gamma[0] = 0                                                           # a row of Gamma that keeps nothing
    hidden = np.where(f8.spread_gamma(gamma, O, I, bo, bi), w, np.where(np.arange(I) % 3 == 0, np.nan, np.inf)).astype(np.float32)
    lay = bsp.F8Layer(O, I, bo, bi, XTYPE[dtype])
    g = torch.from_numpy(np.ascontiguousarray(gamma, dtype=np.uint8)).cuda()
    lay.quantize(device(hidden, dtype), g)
    want = f8.masked(w.astype(np.float64), gamma, bo, bi)
    codes, scales = f8.quantize(want, "e4m3", 128)
    got = codes_of(lay.w)
    assert np.array_equal(got[1], scales) and np.array_equal(got[0] & 0x7F, codes & 0x7F)
    back = f8.dequantize(*got, "e4m3")
    assert np.array_equal(back, f8.dequantize(codes, scales, "e4m3"))
    assert np.array_equal(f8.dequantize(*codes_of(lay.wt), "e4m3"), back.T)      # both orientations hold the same values
    lay.quantize(device(w, dtype))
    codes, scales = f8.quantize(w, "e4m3", 128)
    got = codes_of(lay.w)
    assert np.array_equal(got[0], codes) and np.array_equal(got[1], scales)


@pytest.mark.parametrize("R,K,dtype,ftype", [(1, 1, "f32", "e4m3"), (130, 260, "bf16", "e4m3"), (257, 100, "f32", "e5m2"), (33, 1000, "bf16", "e5m2")])
@pytest.mark.parametrize("transpose", [False, True])
def test_dequantize(R, K, dtype, ftype, transpose):
    codes, scales = f8.quantize(values(2600 + R, R, K, "f32"), ftype)
    m = held(codes, scales, ftype)
    shape = (K, R) if transpose else (R, K)
    ld = shape[1] + 5
    store = torch.full((shape[0], ld), -7.0, dtype=XTYPE[dtype], device="cuda")
    bsp.bsp_dequantize_f8(m.m, store, bsp.dtype_code(XTYPE[dtype]), ld, transpose)
    want = f8.dequantize(codes, scales, ftype)
    got = store.float().cpu().numpy()
    assert np.array_equal(got[:, :shape[1]], (want.T if transpose else want).astype(np.float32))     # (a value has few bits: bf16 holds it)
    assert (got[:, shape[1]:] == -7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,K,extra,off", [(1, 1, 0, 0), (131, 257, 0, 0), (129, 300, 1, 1), (130, 131, 3, 2), (300, 63, 2, 3), (255, 15, 0, 5)])
def test_dequantize_any_alignment(R, K, extra, off, dtype):
    """Rows of X that begin anywhere, in both orientations; nothing between or around them is written."""
    codes, scales = f8.quantize(values(2650 + R, R, K, "f32"), "e4m3")
    m, want = held(codes, scales, "e4m3"), f8.dequantize(codes, scales, "e4m3")
    for w, transpose in ((want, False), (want.T, True)):
        ld = w.shape[1] + extra
        store = torch.full((off + w.shape[0] * ld + 8,), -7.0, dtype=XTYPE[dtype], device="cuda")
        view = torch.as_strided(store, w.shape, (ld, 1), off)
        bsp.bsp_dequantize_f8(m.m, view, bsp.dtype_code(XTYPE[dtype]), ld, transpose)
        expect = torch.full_like(store, -7.0)
        torch.as_strided(expect, w.shape, (ld, 1), off).copy_(device(w, dtype))
        assert torch.equal(store, expect)


@pytest.mark.parametrize("dtype,off,ldx", [("bf16", 1, 257), ("f32", 3, 257), ("bf16", 0, 257), ("bf16", 5, 258)])
def test_quantize_any_alignment(dtype, off, ldx):
    P, I = 260, 257
    x = values(2660 + off, P, I, dtype)
    store = torch.full((P * ldx + off,), float("nan"), dtype=XTYPE[dtype], device="cuda")
    view = torch.as_strided(store, (P, I), (ldx, 1), off)
    view.copy_(device(x, dtype))
    assert_forms(quantize_both(view, "e4m3", None, ldx), x, "e4m3")


def test_dequantize_transposed_many_tiles():
    R, K = 2050, 2120
    codes, scales = f8.quantize(values(2680, R, K, "f32"), "e4m3")
    m, want = held(codes, scales, "e4m3"), f8.dequantize(codes, scales, "e4m3")
    ld = 2056
    X = torch.full((K, ld), -7.0, dtype=torch.bfloat16, device="cuda")
    bsp.bsp_dequantize_f8(m.m, X, bsp.BF16, ld, True)
    got = X.float().cpu().numpy()
    assert np.array_equal(got[:, :R], want.T.astype(np.float32)) and (got[:, R:] == -7.0).all()


def test_dequantize_every_code_and_scale():
    for ftype in ("e4m3", "e5m2"):
        codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
        scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 2, axis=1)
        m = held(codes, scales, ftype)
        X = torch.empty((256, 256), device="cuda")
        bsp.bsp_dequantize_f8(m.m, X, bsp.F32, 256)
        with np.errstate(over="ignore", invalid="ignore"):
            want = f8.dequantize(codes, scales, ftype).astype(np.float32)
        want[255] = np.nan
        assert np.array_equal(X.cpu().numpy(), want, equal_nan=True)


def gemm(A, a, B, b, bias, out):
    M, N = a.shape[0], b.shape[0]
    ws = bsp.new_workspace(256)
    guard = 64
    store = torch.full((M * N + guard,), -7.0, dtype=XTYPE[out], device="cuda")
    Y = store[:M * N].view(M, N)
    bsp.bsp_gemm_f8(A.m, B.m, None if bias is None else torch.from_numpy(bias).cuda(), Y, bsp.dtype_code(XTYPE[out]), ws)
    bsp.bsp_check(ws)
    want = a @ b.T + (0.0 if bias is None else bias.astype(np.float64))
    got = Y.float().cpu().numpy()
    assert bool((store[M * N:] == -7.0).all())
    return got, want


@pytest.mark.parametrize("M,N,K,at,bt,out", [
    (1, 8, 16, "e4m3", "e4m3", "f32"), (1, 1, 1, "e4m3", "e4m3", "f32"), (128, 128, 128, "e4m3", "e4m3", "f32"), (3, 5, 200, "e5m2", "e4m3", "f32"),
    (16, 128, 512, "e4m3", "e4m3", "bf16"), (17, 136, 640, "e4m3", "e5m2", "f32"), (33, 257, 1000, "e4m3", "e4m3", "bf16"), (64, 1000, 2048, "e4m3", "e4m3", "f32"),
    (65, 24, 130, "e5m2", "e5m2", "f32"), (129, 300, 1024, "e4m3", "e4m3", "f32"), (1000, 264, 8192, "e5m2", "e4m3", "f32"), (1023, 2048, 384, "e4m3", "e4m3", "bf16"),
    (1, 4096, 4096, "e4m3", "e4m3", "f32"), (20000, 128, 72, "e4m3", "e4m3", "bf16")])
def test_gemm(M, N, K, at, bt, out):
    A, a = random_held(3000 + M, M, K, at)
    B, b = random_held(3100 + N, N, K, bt, 0.05)
    bias = synth.normal(3200, (N,), 1.0).astype(np.float32)
    got, want = gemm(A, a, B, b, bias, out)
    assert (np.abs(got - want) <= product_bound(a, b, want, out)).all()
    got, want = gemm(A, a, B, b, None, out)
    assert (np.abs(got - want) <= product_bound(a, b, want, out)).all()


@pytest.mark.parametrize("M,N,K,at,bt,out", [(2300, 2056, 400, "e4m3", "e4m3", "bf16"), (2300, 2056, 4400, "e5m2", "e4m3", "f32"), (20000, 264, 136, "e4m3", "e5m2", "f32"),
                                             (130, 20000, 2048, "e4m3", "e4m3", "bf16"), (2049, 2564, 2050, "e4m3", "e4m3", "f32"),
                                             (2560, 2560, 300, "e4m3", "e4m3", "bf16"), (2500, 2440, 2400, "e4m3", "e4m3", "f32"), (1030, 1000, 4096, "e4m3", "e4m3", "bf16")])
def test_gemm_large(M, N, K, at, bt, out):
    """Products that take pairs of CTAs: ragged in both directions, one and several sums of 2048 entries, more tiles than pairs."""
    A, a = random_held(3050 + M, M, K, at)
    B, b = random_held(3150 + N, N, K, bt, 0.05)
    bias = synth.normal(3250, (N,), 1.0).astype(np.float32)
    got, want = gemm(A, a, B, b, bias, out)
    assert (np.abs(got - want) <= product_bound(a, b, want, out)).all()


def test_weight_gradient_large():
    O, I, P = 2304, 2312, 2700
    A, a = random_held(3510, O, P, "e5m2", 1e-3)
    B, b = random_held(3610, I, P, "e4m3")
    gamma = synth.random_gamma(3710, O // 8, I // 8, (O // 8) * (I // 8) // 2)
    dW, ws = torch.full((O, I), float("nan"), device="cuda"), bsp.new_workspace(256)
    bsp.bsp_gemm_f8_dw(bsp.wdesc(O, I, 1, 1, 8, 8, bsp.F32), torch.from_numpy(np.ascontiguousarray(gamma, dtype=np.uint8)).cuda(), A.m, B.m, dW, ws)
    bsp.bsp_check(ws)
    want = f8.masked(a @ b.T, gamma, 8, 8)
    assert (np.abs(dW.cpu().numpy() - want) <= product_bound(a, b, want, "f32")).all()


def test_gemm_scales_across_their_range():
    """Scales that differ from row to row and block to block by up to 2^80."""
    M, N, K = 200, 150, 700
    codes, _ = f8.quantize(values(3300, M, K, "f32"), "e4m3")
    wcodes, _ = f8.quantize(values(3301, N, K, "f32"), "e4m3")
    s, t = synth.uniform_int(3302, (M, 6), 87, 167).astype(np.uint8), synth.uniform_int(3303, (N, 6), 87, 167).astype(np.uint8)
    a, b = f8.dequantize(codes, s, "e4m3"), f8.dequantize(wcodes, t, "e4m3")
    got, want = gemm(held(codes, s, "e4m3"), a, held(wcodes, t, "e4m3"), b, None, "f32")
    assert (np.abs(got - want) <= product_bound(a, b, want, "f32")).all()


@pytest.mark.parametrize("M,N,K,out", [(40, 200, 20000, "f32"), (100, 32, 9000, "f32"), (128, 64, 3000, "bf16"), (70, 61, 5000, "f32"), (500, 66, 300, "bf16"), (700, 1026, 128, "f32"),
                                       (5000, 136, 2304, "f32"), (300, 7, 2000, "bf16")])
def test_gemm_shared_sums_and_narrow_tiles(M, N, K, out):
    """Long sums over clusters and in several chunks, tiles of every width, outputs whose rows are not 16-byte multiples."""
    A, a = random_held(3060 + M, M, K, "e4m3")
    B, b = random_held(3160 + N, N, K, "e5m2", 0.05)
    bias = synth.normal(3260, (N,), 1.0).astype(np.float32)
    got, want = gemm(A, a, B, b, bias, out)
    assert (np.abs(got - want) <= product_bound(a, b, want, out)).all()


def test_gemm_nan_stays_in_its_row_and_column():
    M, N, K = 150, 140, 260
    codes, s = f8.quantize(values(3400, M, K, "f32"), "e4m3")
    wcodes, t = f8.quantize(values(3401, N, K, "f32"), "e4m3")
    codes[5, 259], wcodes[131, 0] = 0x7F, 0xFF
    A, B = held(codes, s, "e4m3"), held(wcodes, t, "e4m3")
    a, b = f8.dequantize(codes, s, "e4m3"), f8.dequantize(wcodes, t, "e4m3")
    got, _ = gemm(A, a, B, b, None, "f32")
    assert np.isnan(got[5]).all() and np.isnan(got[:, 131]).all()
    rows, cols = np.arange(M) != 5, np.arange(N) != 131
    a, b = a[rows], b[cols]
    want = a @ b.T
    assert (np.abs(got[rows][:, cols] - want) <= product_bound(a, b, want, "f32")).all()


@pytest.mark.parametrize("O,I,P,bo,bi,at", [(8, 8, 1, 8, 8, "e4m3"), (64, 64, 333, 8, 8, "e5m2"), (256, 80, 5000, 4, 16, "e4m3"), (144, 260, 129, 16, 4, "e5m2"),
                                            (1024, 256, 1000, 8, 8, "e4m3")])
def test_weight_gradient(O, I, P, bo, bi, at):
    A, a = random_held(3500 + O, O, P, at, 1e-3)
    B, b = random_held(3600 + I, I, P, "e4m3")
    gamma = synth.random_gamma(3700, O // bo, I // bi, (O // bo) * (I // bi) // 2)
    wd, ws = bsp.wdesc(O, I, 1, 1, bo, bi, bsp.F32), bsp.new_workspace(256)
    for g in (gamma, None):
        dW = torch.full((O, I), float("nan"), device="cuda")
        bsp.bsp_gemm_f8_dw(wd, None if g is None else torch.from_numpy(np.ascontiguousarray(g, dtype=np.uint8)).cuda(), A.m, B.m, dW, ws)
        bsp.bsp_check(ws)
        want = f8.masked(a @ b.T, g, bo, bi)
        got = dW.cpu().numpy()
        assert (np.abs(got - want) <= product_bound(a, b, want, "f32")).all()
        if g is not None:
            assert (got[~f8.spread_gamma(g, O, I, bo, bi)] == 0).all()


def test_weight_gradient_of_dropped_blocks_is_zero_even_where_sums_are_nan():
    O, I, P = 64, 64, 200
    codes, s = f8.quantize(values(3800, O, P, "f32"), "e5m2")
    codes[:] = 0x7F
    xcodes, t = f8.quantize(values(3801, I, P, "f32"), "e4m3")
    gamma = synth.random_gamma(3802, 8, 8, 40)
    dW = torch.full((O, I), 3.0, device="cuda")
    ws = bsp.new_workspace(256)
    bsp.bsp_gemm_f8_dw(bsp.wdesc(O, I, 1, 1, 8, 8, bsp.BF16), torch.from_numpy(np.ascontiguousarray(gamma, dtype=np.uint8)).cuda(), held(codes, s, "e5m2").m, held(xcodes, t, "e4m3").m, dW, ws)
    keep = f8.spread_gamma(gamma, O, I, 8, 8)
    got = dW.cpu().numpy()
    assert np.isnan(got[keep]).all() and (got[~keep] == 0).all()


@pytest.mark.parametrize("P,I,O,dtype,out", [(1, 8, 8, "bf16", "f32"), (1, 4096, 1000, "bf16", "bf16"), (7, 1003, 72, "f32", "f32"), (16, 512, 640, "bf16", "f32"), (33, 264, 40, "f32", "bf16"),
                                             (64, 2048, 1000, "f32", "f32"), (200, 136, 264, "bf16", "bf16")])
def test_linear(P, I, O, dtype, out):
    x = values(3900 + P, P, I, dtype)
    B, b = random_held(3901 + O, O, I, "e4m3", 0.05)
    a = f8.dequantize(*f8.quantize(x, "e4m3"), "e4m3")
    bias = synth.normal(3902, (O,), 1.0).astype(np.float32)
    ldx = I + 8
    X = torch.full((P, ldx), float("nan"), dtype=XTYPE[dtype], device="cuda")
    X[:, :I] = device(x, dtype)
    Y = torch.full((P, O), -7.0, dtype=XTYPE[out], device="cuda")
    ws = bsp.new_workspace(bsp.bsp_linear_f8_workspace_bytes(B.m, P))
    bsp.bsp_linear_f8(B.m, X, bsp.dtype_code(XTYPE[dtype]), P, ldx, torch.from_numpy(bias).cuda(), Y, bsp.dtype_code(XTYPE[out]), ws)
    bsp.bsp_check(ws)
    want = a @ b.T + bias.astype(np.float64)
    assert (np.abs(Y.float().cpu().numpy() - want) <= product_bound(a, b, want, out)).all()


@pytest.mark.parametrize("P,I,O", [(64, 40000, 136), (2, 70000, 24), (64, 8192, 4100), (40, 129, 128)])
def test_linear_long_rows(P, I, O):
    """Rows that a CTA cannot hold in 8 bits, and ones that it can."""
    x = values(3950 + P, P, I, "bf16")
    B, b = random_held(3951 + O, O, I, "e4m3", 0.05)
    a = f8.dequantize(*f8.quantize(x, "e4m3"), "e4m3")
    Y = torch.full((P, O), -7.0, device="cuda")
    ws = bsp.new_workspace(bsp.bsp_linear_f8_workspace_bytes(B.m, P))
    bsp.bsp_linear_f8(B.m, device(x, "bf16"), bsp.BF16, P, I, None, Y, bsp.F32, ws)
    bsp.bsp_check(ws)
    want = a @ b.T
    assert (np.abs(Y.cpu().numpy() - want) <= product_bound(a, b, want, "f32")).all()


def test_linear_extremes():
    """NaN, infinities, zeros and subnormals in the rows that a server hands over come out as from the quantiser and the product."""
    P, I, O = 9, 1000, 200
    x = values(3960, P, I, "f32")
    x[1] = 0.0
    x[2, 5], x[3, 700], x[4, 130] = np.nan, np.inf, -np.inf
    x[5] = 2.0 ** -140
    x[6] = np.inf
    B, b = random_held(3961, O, I, "e4m3", 0.05)
    lay = bsp.F8Layer(O, I, 8, 8, torch.float32)
    lay.w.data.copy_(B.data); lay.w.scale.copy_(B.scale)
    Y, act, Z = torch.empty((P, O), device="cuda"), bsp.F8Activations(P, I), torch.empty((P, O), device="cuda")
    lay.linear(device(x, "f32"), None, Y)
    lay.forward(device(x, "f32"), act, None, Z)
    a = f8.dequantize(*f8.quantize(x, "e4m3"), "e4m3")
    bad = np.isnan(a).any(1)
    for got in (Y.cpu().numpy(), Z.cpu().numpy()):
        assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
        want = a[~bad] @ b.T
        assert (np.abs(got[~bad] - want) <= product_bound(a[~bad], b, want, "f32")).all()


def step_tensors(P, O, I):
    w, x, dy = values(4000, O, I, "f32", 0.05), values(4001, P, I, "bf16"), values(4002, P, O, "bf16", 1e-3)
    bias = synth.normal(4003, (O,), 1.0).astype(np.float32)
    return w, x, dy, bias


def test_training_step_with_gamma_from_the_mask_builder():
    """Mask, quantised weights, forward, backward as a program runs them; the gradients against the formulas and against differences of the
    loss sum(Y dY) of the layer that the 8-bit tensors define (which is linear, so a difference is exact but for rounding)."""
    P, O, I = 700, 264, 392
    w, x, dy, bias = step_tensors(P, O, I)
    W, X, dY, b = device(w, "f32"), device(x, "bf16"), device(dy, "bf16"), torch.from_numpy(bias).cuda()
    prune = bsp.SparseLayer(O, I, 1, 1, 8, 8, torch.float32)
    prune.mask(W, (O // 8) * (I // 8) // 2)
    lay = bsp.F8Layer(O, I, 8, 8, torch.float32)
    act, grad = bsp.F8Activations(P, I), bsp.F8Activations(P, O, torch.float8_e5m2)
    Y, dX, dW, db = torch.empty((P, O), device="cuda"), torch.empty((P, I), dtype=torch.bfloat16, device="cuda"), torch.empty((O, I), device="cuda"), torch.empty(O, device="cuda")
    lay.quantize(W, prune.gamma)
    lay.forward(X, act, b, Y)
    lay.backward(dY, act, grad, dX, dW, db)
    lay.check()
    gamma = prune.gamma.cpu().numpy()
    keep = f8.spread_gamma(gamma, O, I, 8, 8)
    back = lambda t, f, rows=1: f8.dequantize(*f8.quantize(t, f, rows), f)  # noqa: E731
    wq, xq, xqt = back(f8.masked(w.astype(np.float64), gamma, 8, 8), "e4m3", 128), back(x, "e4m3"), back(x.T, "e4m3")
    gq, gqt = back(dy, "e5m2"), back(dy.T, "e5m2")
    for got, want, p, q, out in ((Y, xq @ wq.T + bias.astype(np.float64), xq, wq, "f32"), (dX, gq @ wq, gq, wq.T, "bf16"), (dW, np.where(keep, gqt @ xqt.T, 0.0), gqt, xqt, "f32")):
        assert (np.abs(got.float().cpu().numpy() - want) <= product_bound(p, q, want, out)).all()
    assert (np.abs(db.cpu().numpy() - dy.astype(np.float64).sum(0)) <= 40 * 2.0 ** -24 * np.abs(dy.astype(np.float64)).sum(0)).all()
    # differences: loss(W) = sum over p of (xhat W^t) . dyhat in 64 bits, with the tensors' own 8-bit values
    loss = lambda m: float(((xqt.T @ m.T) * gqt.T).sum())  # noqa: E731
    for o, i in ((0, 0), (100, 200), (263, 391)):
        for k in range(8):
            o1, i1 = o // 8 * 8 + k, i // 8 * 8 + k
            d = np.zeros_like(wq)
            d[o1, i1] = 1.0 if keep[o1, i1] else 0.0
            diff = (loss(d) - loss(-d)) / 2
            bound = product_bound(gqt[o1:o1 + 1], xqt[i1:i1 + 1], np.array([[diff]]), "f32")[0, 0]
            assert abs(float(dW[o1, i1]) - diff) <= bound + 1e-9 * abs(diff)


def test_step_is_captured_into_a_graph_and_replayed_on_new_inputs():
    P, O, I = 130, 136, 264
    w, x, dy, bias = step_tensors(P, O, I)
    lay = bsp.F8Layer(O, I, 8, 8, torch.float32)
    act, grad = bsp.F8Activations(P, I), bsp.F8Activations(P, O, torch.float8_e5m2)
    W, X, dY, b = device(w, "f32"), device(x, "bf16"), device(dy, "bf16"), torch.from_numpy(bias).cuda()
    Y, dX, dW, db = torch.empty((P, O), device="cuda"), torch.empty((P, I), device="cuda"), torch.empty((O, I), device="cuda"), torch.empty(O, device="cuda")

    def step():
        lay.quantize(W)
        lay.forward(X, act, b, Y)
        lay.backward(dY, act, grad, dX, dW, db)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    X.copy_(device(values(4100, P, I, "bf16"), "bf16"))
    W.copy_(device(values(4101, O, I, "f32", 0.05), "f32"))
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (Y, dX, dW, db)]
    for t in (Y, dX, dW, db):
        t.fill_(float("nan"))
    step()
    lay.check()
    assert all(torch.equal(a, b) for a, b in zip(got, (Y, dX, dW, db)))


def test_calls_of_two_streams_side_by_side():
    """Layers with workspaces of their own on two streams, many calls deep: each gives what it gives alone."""
    P, O, I = 64, 1000, 1024
    lays, outs, xs, alone = [], [], [], []
    for k in range(2):
        lay = bsp.F8Layer(O, I, 8, 8, torch.float32)
        lay.quantize(device(values(4200 + k, O, I, "f32", 0.05), "f32"))
        X = device(values(4210 + k, P, I, "bf16"), "bf16")
        Y = torch.empty((P, O), device="cuda")
        lay.linear(X, None, Y)
        torch.cuda.synchronize()
        lays.append(lay); xs.append(X); outs.append([torch.empty_like(Y) for _ in range(20)]); alone.append(Y.clone())
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for n in range(20):
        for k in range(2):
            lays[k].linear(xs[k], None, outs[k][n], streams[k])
    torch.cuda.synchronize()
    for k in range(2):
        lays[k].check()
        assert all(torch.equal(y, alone[k]) for y in outs[k])


def test_clusters_of_two_streams_side_by_side():
    """Products that share sums over clusters, layers that quantise their rows in place and pairs of CTAs, on two streams at once, each with
    workspaces of its own: each call gives what it gives alone."""
    jobs = []
    for k, (M, N, K, out) in enumerate([(144, 260, 5000, "f32"), (1024, 256, 6000, "f32"), (16, 4096, 4096, "bf16"), (300, 520, 2048, "f32"), (2304, 2304, 512, "bf16"), (40, 72, 9000, "f32")]):
        A, _ = random_held(4300 + k, M, K, "e4m3")
        B, _ = random_held(4320 + k, N, K, "e4m3", 0.05)
        ws = [bsp.new_workspace(256) for _ in range(2)]
        jobs.append((M, N, XTYPE[out], lambda s, Y, which, A=A, B=B, out=out, ws=ws: bsp.bsp_gemm_f8(A.m, B.m, None, Y, bsp.dtype_code(XTYPE[out]), ws[which], s)))
    for k, (P, O, I) in enumerate([(1, 4096, 4096), (16, 1000, 2048)]):
        B, _ = random_held(4340 + k, O, I, "e4m3", 0.05)
        X = device(values(4350 + k, P, I, "bf16"), "bf16")
        ws = [bsp.new_workspace(bsp.bsp_linear_f8_workspace_bytes(B.m, P)) for _ in range(2)]
        jobs.append((P, O, torch.float32, lambda s, Y, which, B=B, X=X, P=P, I=I, ws=ws: bsp.bsp_linear_f8(B.m, X, bsp.BF16, P, I, None, Y, bsp.F32, ws[which], s)))
    alone = []
    for rows, cols, t, call in jobs:
        alone.append(torch.full((rows, cols), -7.0, dtype=t, device="cuda"))
        call(None, alone[-1], 0)
    order = [j for j in range(len(jobs)) for _ in range(4)]
    order = [order, order[::-1]]                                             # (the streams go through the jobs in opposite orders)
    outs = [[torch.full(alone[j].shape, -7.0, dtype=alone[j].dtype, device="cuda") for j in o] for o in order]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for n in range(len(order[0])):
        for which, s in enumerate(streams):
            jobs[order[which][n]][3](s, outs[which][n], which)
    torch.cuda.synchronize()
    for which in range(2):
        assert all(torch.equal(Y, alone[j]) for j, Y in zip(order[which], outs[which]))


def test_linear_is_captured_into_a_graph():
    for P, O, I in ((1, 520, 1000), (64, 264, 4096)):
        lay = bsp.F8Layer(O, I, 8, 8, torch.float32)
        lay.quantize(device(values(4400 + P, O, I, "f32", 0.05), "f32"))
        X, Y = device(values(4401 + P, P, I, "bf16"), "bf16"), torch.empty((P, O), device="cuda")
        lay.linear(X, None, Y)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lay.linear(X, None, Y)
        X.copy_(device(values(4402 + P, P, I, "bf16"), "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        got = Y.clone()
        lay.linear(X, None, Y)
        lay.check()
        assert torch.equal(got, Y)


def test_offsets_past_32_bits():
    """Matrices of more than 2^31 bytes, and an output of more than 2^32: the last rows and columns are where they belong."""
    P, I = 66000, 33000
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    X = torch.randn((P, I), device="cuda", dtype=torch.bfloat16, generator=g)
    act = bsp.F8Activations(P, I)
    bsp.bsp_quantize_f8(X, bsp.BF16, P, I, I, act.rows.m, act.cols.m, None, None)
    for r in (0, P - 3):
        codes, scales = f8.quantize(X[r:r + 3].float().cpu().numpy(), "e4m3")
        assert np.array_equal(act.rows.data[r:r + 3, :I].view(torch.uint8).cpu().numpy(), codes)
    for c in (0, I - 3):
        codes, scales = f8.quantize(X[:, c:c + 3].T.float().cpu().numpy(), "e4m3")
        assert np.array_equal(act.cols.data[c:c + 3, :P].view(torch.uint8).cpu().numpy(), codes)
    back = torch.empty_like(X)
    for m, transpose in ((act.rows, False), (act.cols, True)):
        back.zero_()
        bsp.bsp_dequantize_f8(m.m, back, bsp.BF16, I, transpose)
        for r in (0, P - 2):
            x = X[r:r + 2].double()
            assert bool(((back[r:r + 2].double() - x).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -10 * 2.0 ** 3).all())
    del X, back
    M, N, K = 70000, 16400, 16
    A, B = bsp.F8Matrix(M, K), bsp.F8Matrix(N, K)
    for m in (A, B):
        m.data.copy_(torch.randn(m.data.shape, device="cuda", generator=g).to(torch.float8_e4m3fn))
        m.scale.fill_(127)
    Y, ws = torch.empty((M, N), device="cuda"), bsp.new_workspace(256)
    bsp.bsp_gemm_f8(A.m, B.m, None, Y, bsp.F32, ws)
    bsp.bsp_check(ws)
    for r in (0, M // 2, M - 2):
        a, b = A.data[r:r + 2].double().cpu().numpy(), B.data.double().cpu().numpy()
        want = a @ b.T
        assert (np.abs(Y[r:r + 2].cpu().numpy() - want) <= product_bound(a, b, want, "f32")).all()
    Z = torch.empty((M, N), device="cuda", dtype=torch.float32)
    act = bsp.F8Matrix(N, M)
    bsp.bsp_quantize_f8(Y, bsp.F32, M, N, N, None, act.m, None, None)
    bsp.bsp_dequantize_f8(act.m, Z, bsp.F32, N, True)
    assert bool(((Z[-1] - Y[-1]).abs() <= 2.0 ** -4 * Y[-1].abs() + 2.0 ** -9).all())


@pytest.mark.parametrize("stream", [False, True])
def test_gradient_is_under_the_gamma_that_the_weights_were_quantised_under(stream):
    """The mask builder writes a new Gamma to its buffer between quantize() and backward(): the gradient is still that of the layer whose
    weights answered."""
    P, O, I = 100, 64, 48
    w, x, dy, _ = step_tensors(P, O, I)
    W, X, dY = device(w, "f32"), device(x, "bf16"), device(dy, "bf16")
    prune = bsp.SparseLayer(O, I, 1, 1, 8, 8, torch.float32)
    lay = bsp.F8Layer(O, I, 8, 8, torch.float32)
    act, grad = bsp.F8Activations(P, I), bsp.F8Activations(P, O)
    Y, dW = torch.empty((P, O), device="cuda"), torch.empty((O, I), device="cuda")
    s = torch.cuda.Stream() if stream else None
    torch.cuda.synchronize()
    prune.mask(W, 24, stream=s)
    lay.quantize(W, prune.gamma, s)
    first = prune.gamma.clone() if s is None else None
    prune.mask(-W.flip(0).contiguous(), 24, stream=s)
    lay.forward(X, act, None, Y, s)
    lay.backward(dY, act, grad, dW=dW, stream=s)
    torch.cuda.synchronize()
    if first is None:
        prune.mask(W, 24)
        first = prune.gamma.clone()
    keep = f8.spread_gamma(first.cpu().numpy(), O, I, 8, 8)
    a, b = f8.dequantize(*f8.quantize(dy.T, "e4m3"), "e4m3"), f8.dequantize(*f8.quantize(x.T, "e4m3"), "e4m3")
    want = np.where(keep, a @ b.T, 0.0)
    assert (np.abs(dW.cpu().numpy() - want) <= product_bound(a, b, want, "f32")).all()
    lay.quantize(W)                                                      # without a Gamma all weights have a gradient
    lay.forward(X, act, None, Y)
    lay.backward(dY, act, grad, dW=dW)
    assert (np.abs(dW.cpu().numpy() - a @ b.T) <= product_bound(a, b, a @ b.T, "f32")).all()


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_long_sums_of_pairs_do_not_lose_bits(out):
    """Products of one sign, cancelled by the bias: what is left of Y is the error of the sums.  No instruction of a sum of 8192 entries (256
    instructions; 2048 and 64 for a float32 output) is off by more than one step of what has been summed by then, 2^-23 i / 256 of the sum, which
    makes 128.5 steps of it; joining up to 128 of them, and the bias, half a step of the whole each."""
    M, N, K = 2304, 2304, 262144
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    A, B = bsp.F8Matrix(M, K), bsp.F8Matrix(N, K)
    A.data.view(torch.uint8).copy_(torch.randint(0x30, 0x40, (1, K), device="cuda", dtype=torch.uint8, generator=g).expand(M, K))
    B.data.view(torch.uint8).copy_(torch.randint(0x30, 0x40, (N, K), device="cuda", dtype=torch.uint8, generator=g))
    for m in (A, B):
        m.scale.fill_(127)
    a = A.data[0].double()
    exact = torch.cat([B.data[n:n + 128].double() @ a for n in range(0, N, 128)])
    bias = (-exact).float()
    Y, ws = torch.empty((M, N), dtype=XTYPE[out], device="cuda"), bsp.new_workspace(256)
    call = lambda: bsp.bsp_gemm_f8(A.m, B.m, bias, Y, bsp.dtype_code(XTYPE[out]), ws)  # noqa: E731
    call()
    bsp.bsp_check(ws)
    assert [template(n)[0] for n, _ in launches(call)] == ["gemm_f8_pair_kernel"]
    instructions, joined = (256, 32) if out == "bf16" else (64, 128)
    bound = ((instructions + 1) / 2 * 2.0 ** -23 + (joined + 1) * 2.0 ** -24) * 1.01
    left = (Y.double() - (exact + bias.double())).abs() / exact
    assert float(left.max()) <= bound, (float(left.max()), bound)


@pytest.mark.parametrize("M,N,K,at,bt", [(1500, 1480, 8193, "e4m3", "e4m3"), (2300, 2056, 8300, "e5m2", "e4m3"), (1500, 1480, 16500, "e4m3", "e5m2"), (2300, 2056, 16400, "e4m3", "e4m3")])
def test_gemm_bf16_in_several_sums(M, N, K, at, bt):
    """bfloat16 outputs of pairs whose sums are joined in registers: two and three chunks a tile, whole and halved tiles, one and two tiles a pair."""
    A, a = random_held(3080 + M, M, K, at)
    B, b = random_held(3180 + K, N, K, bt, 0.05)
    bias = synth.normal(3280, (N,), 1.0).astype(np.float32)
    got, want = gemm(A, a, B, b, bias, "bf16")
    assert (np.abs(got - want) <= product_bound(a, b, want, "bf16")).all()
    Y, ws = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), bsp.new_workspace(256)
    assert [template(n) for n, _ in launches(lambda: bsp.bsp_gemm_f8(A.m, B.m, None, Y, bsp.BF16, ws))] == [("gemm_f8_pair_kernel", "Lb0ELb1E")]
