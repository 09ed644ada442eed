"""The paths of the 8-bit floating-point operators that depend on sizes and values: rows quantised in place by tiles of every width, NaN, infinities
and subnormals in bfloat16, one form alone, long sums, a first call that is captured.  Each test says which kernel it means to run."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import f8
from paper_2407_09453_b200 import bsp, synth
from f8_util import EPS2, FTYPE, XTYPE, codes_of, device, held, launches, product_bound, random_held, template, values

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MANGLED = {"bf16": "13__nv_bfloat16", "f32": "f"}


@pytest.mark.parametrize("P,I,O,dtype,off,extra,split", [
    # up to 16 positions, tiles of 16 columns: up to 64 rows of 128 entries a CTA, and more
    (7, 4096, 4096, "bf16", 0, 0, 4), (5, 4095, 4096, "f32", 1, 2, 4), (3, 16384, 4096, "bf16", 0, 0, 4), (2, 40000, 264, "f32", 0, 0, 8), (3, 39999, 136, "bf16", 3, 5, 8),
    # 17..32 positions, tiles of 32 columns: up to 32 rows of 128 entries a CTA, and up to 64
    (17, 8, 264, "bf16", 0, 0, 1), (24, 112, 1000, "f32", 0, 4, 1), (31, 99, 136, "bf16", 1, 2, 1), (32, 129, 1408, "bf16", 0, 7, 1), (27, 200, 264, "f32", 1, 3, 1),
    (20, 500, 1000, "bf16", 3, 1, 2), (32, 500, 264, "f32", 0, 0, 2), (32, 1001, 1408, "bf16", 0, 7, 4), (17, 2048, 1000, "f32", 0, 0, 8), (32, 2048, 264, "bf16", 0, 8, 8),
    # 33..64 positions, tiles of 64 columns, the scales of whose rows take two columns
    (33, 8, 8, "f32", 0, 0, 1), (40, 72, 264, "bf16", 5, 3, 1), (50, 112, 1088, "f32", 0, 0, 1), (63, 101, 1000, "bf16", 0, 3, 1), (64, 112, 4096, "bf16", 0, 0, 1), (64, 127, 136, "f32", 2, 0, 1)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_linear_in_place(P, I, O, dtype, off, extra, split, out):
    """One launch that quantises its rows itself, over clusters of 1 to 8 CTAs; rows that begin anywhere, with NaN between them."""
    x = values(5000 + P + I, P, I, dtype)
    B, b = random_held(5001 + O, O, I, "e4m3", 0.05)
    a = f8.dequantize(*f8.quantize(x, "e4m3"), "e4m3")
    bias = synth.normal(5002, (O,), 1.0).astype(np.float32)
    ldx = I + extra
    X = torch.full((P * ldx + off,), float("nan"), dtype=XTYPE[dtype], device="cuda").as_strided((P, I), (ldx, 1), off)
    X.copy_(device(x, dtype))
    Y = torch.full((P * O + 64,), -7.0, dtype=XTYPE[out], device="cuda")
    ws, bd = bsp.new_workspace(bsp.bsp_linear_f8_workspace_bytes(B.m, P)), torch.from_numpy(bias).cuda()
    call = lambda: bsp.bsp_linear_f8(B.m, X, bsp.dtype_code(XTYPE[dtype]), P, ldx, bd, Y, bsp.dtype_code(XTYPE[out]), ws)  # noqa: E731
    call()
    bsp.bsp_check(ws)
    want = a @ b.T + bias.astype(np.float64)
    assert (np.abs(Y[:P * O].view(P, O).float().cpu().numpy() - want) <= product_bound(a, b, want, out)).all()
    assert bool((Y[P * O:] == -7.0).all())
    assert [(template(n), ctas) for n, ctas in launches(call)] == [(("gemm_f8_tile_kernel", MANGLED[dtype]), -(-O // 128) * split)]


def odd_values(P, I, dtype, ftype):
    """Rows and columns with NaN, infinities (in even and odd places), zeros, subnormals, the largest finite value, and entries at a scale's border."""
    big = float(torch.finfo(XTYPE[dtype]).max)
    tiny = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149
    step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    x = values(5100, P, I, dtype)
    x[0], x[1] = 0.0, np.nan
    x[2] = np.inf
    x[3] = -np.inf
    x[4, 0::2], x[5, 1::2], x[6, 0::3], x[7, 1::5] = np.nan, np.nan, np.inf, -np.inf
    x[8, 4], x[8, 5] = np.inf, np.nan
    x[9, 6], x[9, 7] = -np.nan, -np.inf
    x[10], x[11] = tiny, 2.0 ** -126
    x[12] = big
    x[13, :64], x[13, 64:] = -big, tiny
    x[14] = f8.MAX[ftype]
    x[15] = f8.MAX[ftype] * (1 + step / 1.75)                            # the next value of the type
    if P > 20 and I > 70:
        x[:, 33], x[:, 34], x[:, 35], x[:, 64] = np.nan, np.inf, 0.0, -np.inf
        x[16:, 40], x[16:, 41] = tiny, -big
    assert np.array_equal(x, torch.from_numpy(x).to(XTYPE[dtype]).float().numpy(), equal_nan=True)
    return x


def same_codes(got, want):
    """Codes are equal; the sign of a NaN is not."""
    nan = (want & 0x7F) == 0x7F
    return np.array_equal(got[~nan], want[~nan]) and bool(((got[nan] & 0x7F) == 0x7F).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,I,ftype", [(256, 384, "e4m3"), (200, 300, "e5m2"), (131, 77, "e4m3"), (16, 130, "e5m2")])
def test_quantize_odd_values(P, I, ftype, dtype):
    x = odd_values(P, I, dtype, ftype)
    act = bsp.F8Activations(P, I, FTYPE[ftype])
    bsp.bsp_quantize_f8(device(x, dtype), bsp.dtype_code(XTYPE[dtype]), P, I, I, act.rows.m, act.cols.m, None, None)
    for m, t in ((act.rows, x), (act.cols, x.T)):
        codes, scales = f8.quantize(t, ftype)
        got_codes, got_scales = codes_of(m)
        assert np.array_equal(got_scales, scales)
        if ftype == "e4m3":
            assert same_codes(got_codes, codes)
        else:                                                              # (e5m2 has several NaN)
            assert np.array_equal(f8.dequantize(got_codes, got_scales, ftype), f8.dequantize(codes, scales, ftype), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_weights_odd_values(dtype):
    O, I = 256, 384
    w = odd_values(O, I, dtype, "e4m3")
    w[128:, 128:256] = np.nan                                              # a tile of nothing else
    lay = bsp.F8Layer(O, I, 8, 8, XTYPE[dtype])
    lay.quantize(device(w, dtype))
    codes, scales = f8.quantize(w, "e4m3", 128)
    for m, c in ((lay.w, codes), (lay.wt, codes.T)):
        assert same_codes(codes_of(m)[0], c)
    assert np.array_equal(codes_of(lay.w)[1], scales)
    assert np.array_equal(codes_of(lay.wt)[1], np.repeat(scales[::128].T, 128, axis=0)[:I])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,I,O,kernels", [(16, 1000, 200, 1), (24, 130, 200, 1), (40, 100, 136, 1), (40, 1000, 136, 2), (70, 300, 136, 2)])
def test_linear_odd_values(P, I, O, kernels, dtype):
    x = odd_values(P, I, dtype, "e4m3")
    B, b = random_held(5201, O, I, "e4m3", 0.05)
    a = f8.dequantize(*f8.quantize(x, "e4m3"), "e4m3")
    X, Y, ws = device(x, dtype), torch.full((P, O), -7.0, device="cuda"), bsp.new_workspace(bsp.bsp_linear_f8_workspace_bytes(B.m, P))
    call = lambda: bsp.bsp_linear_f8(B.m, X, bsp.dtype_code(XTYPE[dtype]), P, I, None, Y, bsp.F32, ws)  # noqa: E731
    call()
    bsp.bsp_check(ws)
    bad, got = np.isnan(a).any(1), Y.cpu().numpy()
    assert np.isnan(got[bad]).all()
    with np.errstate(over="ignore"):
        want = a[~bad] @ b.T
        fits = np.abs(a[~bad]) @ np.abs(b).T <= np.finfo(np.float32).max / 2    # (what passes the largest float32 on its way is not compared)
        assert (np.abs(got[~bad] - want) <= product_bound(a[~bad], b, want, "f32"))[fits].all()
    assert len(launches(call)) == kernels


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("O,I,bo,bi", [(136, 264, 8, 8), (128, 128, 4, 16), (272, 132, 16, 4)])
def test_quantize_weights_in_one_orientation(O, I, bo, bi, dtype):
    """Either form alone is the one that both give, and the other's buffers are left as they were."""
    w = values(5300 + O, O, I, dtype, 0.05)
    gamma = synth.random_gamma(5301, O // bo, I // bi, (O // bo) * (I // bi) // 2)
    W, g = device(w, dtype), torch.from_numpy(np.ascontiguousarray(gamma, dtype=np.uint8)).cuda()
    wd = bsp.wdesc(O, I, 1, 1, bo, bi, XTYPE[dtype])
    codes, scales = f8.quantize(f8.masked(w.astype(np.float64), gamma, bo, bi), "e4m3", 128)
    for which in ("rows", "cols"):
        forms = {"rows": bsp.F8Matrix(O, I), "cols": bsp.F8Matrix(I, O)}
        for m in forms.values():
            m.data.view(torch.uint8).fill_(0xAB)
            m.scale.fill_(0xAB)
        bsp.bsp_quantize_weights_f8(wd, W, g, forms["rows"].m if which == "rows" else None, forms["cols"].m if which == "cols" else None)
        other = forms["cols" if which == "rows" else "rows"]
        assert bool((other.data.view(torch.uint8) == 0xAB).all()) and bool((other.scale == 0xAB).all())
        got = f8.dequantize(*codes_of(forms[which]), "e4m3")
        want = f8.dequantize(codes, scales, "e4m3")
        assert np.array_equal(got, want if which == "rows" else want.T)


@pytest.mark.parametrize("M,N,out,kernel", [(300, 200, "f32", "gemm_f8_tile_kernel"), (300, 200, "bf16", "gemm_f8_tile_kernel"), (40, 200, "f32", "gemm_f8_tile_kernel"),
                                            (40, 200, "bf16", "gemm_f8_tile_kernel"), (2304, 2304, "f32", "gemm_f8_pair_kernel"), (2304, 2304, "bf16", "gemm_f8_pair_kernel")])
def test_long_sums_keep_their_bits(M, N, out, kernel):
    """Products of one sign and of many sizes, cancelled by the bias: what is left of Y is the error of the sums.  An instruction is off by at most
    one step of what has been summed by then, 2^-23 i / n of a sum of n instructions, (n + 1) / 2 steps of it in all; n = 64 (2048 entries; 256
    for a bfloat16 output of pairs).  Joining those sums, eight ranges of k and the bias costs half a step of the whole each."""
    K = 262144
    g = torch.Generator(device="cuda")
    g.manual_seed(13)
    A, B = bsp.F8Matrix(M, K), bsp.F8Matrix(N, K)
    A.data.view(torch.uint8).copy_(torch.randint(0x20, 0x68, (1, K), device="cuda", dtype=torch.uint8, generator=g).expand(M, K))
    B.data.view(torch.uint8).copy_(torch.randint(0x20, 0x68, (N, K), device="cuda", dtype=torch.uint8, generator=g))
    for m in (A, B):
        m.scale.fill_(127)
    a = A.data[0].double()
    exact = torch.cat([B.data[n:n + 128].double() @ a for n in range(0, N, 128)])
    bias = (-exact).float()
    Y, ws = torch.empty((M, N), dtype=XTYPE[out], device="cuda"), bsp.new_workspace(256)
    call = lambda: bsp.bsp_gemm_f8(A.m, B.m, bias, Y, bsp.dtype_code(XTYPE[out]), ws)  # noqa: E731
    call()
    bsp.bsp_check(ws)
    n = 256 if (out, kernel) == ("bf16", "gemm_f8_pair_kernel") else 64
    bound = ((n + 1) / 2 * 2.0 ** -23 + (K / 32 / n + 8 + 1) * 2.0 ** -24) * (1 + EPS2[out]) * 1.01
    left = (Y.double() - (exact + bias.double())).abs() / exact
    assert float(left.max()) <= bound, (float(left.max()), bound)
    assert [template(name)[0] for name, _ in launches(call)] == [kernel]


FIRST = r"""
import torch
from paper_2407_09453_b200 import bsp
P, O, I = 130, 136, 264
g = torch.Generator(device="cuda")
g.manual_seed(1)
W, X, dY, b = (torch.randn(s, device="cuda", generator=g) for s in ((O, I), (P, I), (P, O), (O,)))
lay = bsp.F8Layer(O, I, 8, 8, torch.float32)
gamma = (torch.rand(O // 8 * (I // 8), device="cuda", generator=g) < 0.5).to(torch.uint8)
act, grad = bsp.F8Activations(P, I), bsp.F8Activations(P, O, torch.float8_e5m2)
outs = [torch.empty(s, device="cuda") for s in ((P, O), (P, I), (O, I), (O,), (1, O), (P, I), (2304, 2304))]
Y, dX, dW, db, Z, back, large = outs
big = bsp.F8Matrix(2304, 512)
big.data.copy_(torch.randn(big.data.shape, device="cuda", generator=g).to(torch.float8_e4m3fn))
big.scale.fill_(127)

def step():
    lay.quantize(W, gamma)
    lay.forward(X, act, b, Y)
    lay.backward(dY, act, grad, dX, dW, db)
    lay.linear(X[:1], b, Z)
    bsp.bsp_dequantize_f8(act.cols.m, back, bsp.F32, I, True)
    bsp.bsp_gemm_f8(big.m, big.m, None, large, bsp.F32, lay.ws)

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
for t in outs:
    t.fill_(float("nan"))
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in outs]
for t in outs:
    t.fill_(float("nan"))
step()
lay.check()
assert all(torch.equal(a, b) and bool(a.isfinite().all()) for a, b in zip(got, outs))
"""


def test_first_calls_of_a_process_are_captured():
    """No call needs one before it that is not captured."""
    subprocess.run([sys.executable, "-c", FIRST], check=True, timeout=300, cwd=ROOT)


@pytest.mark.parametrize("R,K,wide", [(2048, 2304, False), (2056, 2300, True), (2560, 2560, True), (2048, 2304 + 128, True)])
def test_transposed_restore_on_both_sides_of_its_rule(R, K, wide):
    """288 tiles and 304 to 400: the same values by both forms, nothing behind the rows written."""
    codes, scales = f8.quantize(values(5400 + R, R, K, "f32"), "e5m2")
    m, want = held(codes, scales, "e5m2"), f8.dequantize(codes, scales, "e5m2").T
    X = torch.full((K, R + 8), -7.0, dtype=torch.bfloat16, device="cuda")
    call = lambda: bsp.bsp_dequantize_f8(m.m, X, bsp.BF16, R + 8, True)  # noqa: E731
    call()
    got = X.float().cpu().numpy()
    assert np.array_equal(got[:, :R], want.astype(np.float32)) and (got[:, R:] == -7.0).all()
    assert [template(n) for n, _ in launches(call)] == [("dequantize_f8_kernel", "13__nv_bfloat16Lb1ELb1ELb%dE" % wide)]


@pytest.mark.parametrize("P,I,O", [(1, 520, 264), (20, 272, 136), (50, 112, 264), (64, 2048, 136), (100, 300, 264)])
def test_linear_on_e5m2_weights(P, I, O):
    x = values(5500 + P, P, I, "bf16")
    B, b = random_held(5501 + O, O, I, "e5m2", 0.05)
    a = f8.dequantize(*f8.quantize(x, "e4m3"), "e4m3")
    Y, ws = torch.full((P, O), -7.0, device="cuda"), bsp.new_workspace(bsp.bsp_linear_f8_workspace_bytes(B.m, P))
    bsp.bsp_linear_f8(B.m, device(x, "bf16"), bsp.BF16, P, I, None, Y, bsp.F32, ws)
    bsp.bsp_check(ws)
    want = a @ b.T
    assert (np.abs(Y.cpu().numpy() - want) <= product_bound(a, b, want, "f32")).all()


def test_step_in_one_call_after_another_on_strided_and_single_rows():
    """Views that describe themselves by their stride, and a single row whose stride says nothing, give what packed copies give."""
    O, I = 72, 40
    lay = bsp.F8Layer(O, I, 8, 8, torch.float32)
    lay.quantize(device(values(5600, O, I, "f32", 0.05), "f32"))
    wide = device(values(5601, 70, I + 24, "bf16"), "bf16")
    for X in (wide[:, 8:8 + I], wide[::3, :I], wide[:1, :I], wide[:1, :I].expand(1, I), wide[:, :1].t()[:, :I]):
        P = X.shape[0]
        outs = []
        for x in (X, X.contiguous()):
            act, Y, Z = bsp.F8Activations(P, I), torch.empty((P, O), device="cuda"), torch.empty((P, O), device="cuda")
            if x.stride(1) != 1:
                with pytest.raises(ValueError):
                    lay.linear(x, None, Z)
                x = x.contiguous()
            lay.forward(x, act, None, Y)
            lay.linear(x, None, Z)
            lay.check()
            outs.append((Y, Z, codes_of(act.rows)))
        (Y, Z, r), (y, z, s) = outs
        assert torch.equal(Y, y) and torch.equal(Z, z) and np.array_equal(r[0], s[0]) and np.array_equal(r[1], s[1])
