"""Host side of the 8-bit floating-point operators: sizes, and every refusal before anything is launched (no GPU needed)."""
import pytest
import torch

from oracle import f8
from paper_2407_09453_b200 import bsp, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


class Stream:
    cuda_stream = 0


S = Stream()


def buffer(n=4096, dtype=torch.uint8):
    t = torch.zeros(n + 64, dtype=dtype)
    off = (-t.data_ptr() % 64) // t.element_size()
    return t[off:off + n]


def matrix(R, K, t=torch.float8_e4m3fn, data=None, scale=None):
    return bsp.f8matrix(t, R, K, buffer() if data is None else data, buffer() if scale is None else scale)


@pytest.mark.parametrize("R,K", [(1, 1), (128, 128), (129, 513), (1000, 2048), (3, 511), (128, 512)])
def test_sizes(R, K):
    assert bsp.bsp_f8_pitch(K) == -(-K // 16) * 16
    assert bsp.bsp_f8_data_bytes(R, K) == R * bsp.bsp_f8_pitch(K)
    assert bsp.bsp_f8_scale_bytes(R, K) == f8.scale_bytes(R, K)
    m = bsp.F8Matrix(R, K, torch.float8_e5m2, device="cpu")
    assert (m.m.type, m.m.rows, m.m.cols, m.m.data, m.m.scale) == (bsp.E5M2, R, K, m.data.data_ptr(), m.scale.data_ptr())
    assert m.data.shape == (R, bsp.bsp_f8_pitch(K)) and m.scale.numel() == f8.scale_bytes(R, K)
    assert bsp.bsp_quantize_f8_workspace_bytes(R, K) >= 256 + -(-R // 128) * K * 4
    assert bsp.bsp_linear_f8_workspace_bytes(matrix(8, K), R) >= 256 + R * bsp.bsp_f8_pitch(K) + f8.scale_bytes(R, K)


def test_sizes_that_are_none():
    assert [f(0, 5) for f in (bsp.bsp_f8_data_bytes, bsp.bsp_f8_scale_bytes, bsp.bsp_quantize_f8_workspace_bytes)] == [0, 0, 0]
    assert bsp.bsp_f8_data_bytes(5, -1) == 0 and bsp.bsp_linear_f8_workspace_bytes(matrix(8, 8), 0) == 0


def refused(status, call):
    with pytest.raises(bsp.BspError) as e:
        call()
    assert e.value.status == status


def test_quantize_refusals():
    x, ws = buffer(4096, torch.float32), buffer()
    rows, cols = matrix(8, 32), matrix(32, 8)
    q = lambda X=x, t=bsp.F32, P=8, I=32, ldx=32, r=rows, c=cols, s=None, w=ws: bsp.bsp_quantize_f8(X, t, P, I, ldx, r, c, s, w, S)  # noqa: E731
    refused(bsp.ERR_NULL, lambda: q(X=None))
    refused(bsp.ERR_NULL, lambda: q(r=None, c=None))
    refused(bsp.ERR_NULL, lambda: q(s=x, w=None))
    refused(bsp.ERR_DTYPE, lambda: q(t=bsp.I8))
    refused(bsp.ERR_DTYPE, lambda: q(r=matrix(8, 32, torch.float8_e5m2)))
    refused(bsp.ERR_DTYPE, lambda: q(r=matrix(8, 32, bsp.BF16), c=None))
    refused(bsp.ERR_SHAPE, lambda: q(P=0))
    refused(bsp.ERR_SHAPE, lambda: q(P=2 ** 31))
    refused(bsp.ERR_SHAPE, lambda: q(ldx=31))
    refused(bsp.ERR_SHAPE, lambda: q(r=cols))
    refused(bsp.ERR_SHAPE, lambda: q(c=rows))
    refused(bsp.ERR_SHAPE, lambda: q(r=matrix(8, 32, data=buffer()[4:]), c=None))
    refused(bsp.ERR_SHAPE, lambda: q(X=x.view(torch.uint8)[2:]))
    refused(bsp.ERR_NULL, lambda: q(r=bsp.F8(bsp.E4M3, 8, 32, None, x.data_ptr()), c=None))
    refused(bsp.ERR_SHAPE, lambda: q(s=x.view(torch.uint8)[2:]))


def test_weights_and_back_refusals():
    w, g = buffer(4096, torch.float32), buffer()
    rows, cols = matrix(64, 32), matrix(32, 64)
    q = lambda wd, W=w, r=rows, c=cols: bsp.bsp_quantize_weights_f8(wd, W, g, r, c, S)  # noqa: E731
    good = bsp.wdesc(64, 32, 1, 1, 8, 8, bsp.F32)
    refused(bsp.ERR_DTYPE, lambda: q(bsp.wdesc(64, 32, 1, 1, 8, 8, bsp.I8)))
    refused(bsp.ERR_BLOCK, lambda: q(bsp.wdesc(64, 32, 1, 1, 8, 4, bsp.F32)))
    refused(bsp.ERR_SHAPE, lambda: q(bsp.wdesc(64, 32, 3, 1, 8, 8, bsp.F32)))
    refused(bsp.ERR_SHAPE, lambda: q(bsp.wdesc(64, 40, 1, 1, 8, 8, bsp.F32)))
    refused(bsp.ERR_NULL, lambda: q(good, W=None))
    refused(bsp.ERR_NULL, lambda: q(good, r=None, c=None))
    d = lambda m=rows, X=w, t=bsp.F32, ldx=32, tr=False: bsp.bsp_dequantize_f8(m, X, t, ldx, tr, S)  # noqa: E731
    refused(bsp.ERR_NULL, lambda: d(m=None))
    refused(bsp.ERR_NULL, lambda: d(X=None))
    refused(bsp.ERR_DTYPE, lambda: d(t=bsp.I32))
    refused(bsp.ERR_SHAPE, lambda: d(ldx=31))
    refused(bsp.ERR_SHAPE, lambda: d(tr=True))                          # rows of 64 entries then


def test_product_refusals():
    y, ws = buffer(4096, torch.float32), buffer()
    x, w = matrix(8, 32), matrix(64, 32, torch.float8_e5m2)
    p = lambda a=x, b=w, bias=None, Y=y, t=bsp.F32, s=ws: bsp.bsp_gemm_f8(a, b, bias, Y, t, s, S)  # noqa: E731
    refused(bsp.ERR_NULL, lambda: p(a=None))
    refused(bsp.ERR_NULL, lambda: p(Y=None))
    refused(bsp.ERR_NULL, lambda: p(s=None))
    refused(bsp.ERR_DTYPE, lambda: p(t=bsp.I32))
    refused(bsp.ERR_SHAPE, lambda: p(b=matrix(64, 33)))
    refused(bsp.ERR_SHAPE, lambda: p(Y=y[1:]))
    refused(bsp.ERR_SHAPE, lambda: p(bias=y.view(torch.uint8)[2:]))
    refused(bsp.ERR_SHAPE, lambda: p(a=matrix(8, 32, scale=buffer()[4:])))
    g = lambda wd, a=matrix(64, 100), b=matrix(32, 100): bsp.bsp_gemm_f8_dw(wd, ws, a, b, y, ws, S)  # noqa: E731
    refused(bsp.ERR_SHAPE, lambda: g(bsp.wdesc(64, 40, 1, 1, 8, 8, bsp.F32)))
    refused(bsp.ERR_SHAPE, lambda: g(bsp.wdesc(32, 32, 1, 1, 8, 8, bsp.F32)))
    refused(bsp.ERR_SHAPE, lambda: g(bsp.wdesc(64, 32, 1, 3, 8, 8, bsp.F32)))
    refused(bsp.ERR_BLOCK, lambda: g(bsp.wdesc(64, 32, 1, 1, 1, 1, bsp.F32)))
    l = lambda m=w, X=y, t=bsp.F32, P=8, ldx=32, Y=y, s=ws: bsp.bsp_linear_f8(m, X, t, P, ldx, None, Y, bsp.F32, s, S)  # noqa: E731, E741
    refused(bsp.ERR_NULL, lambda: l(m=None))
    refused(bsp.ERR_NULL, lambda: l(s=None))
    refused(bsp.ERR_DTYPE, lambda: l(t=bsp.I8))
    refused(bsp.ERR_SHAPE, lambda: l(P=0))
    refused(bsp.ERR_SHAPE, lambda: l(ldx=8))
    refused(bsp.ERR_SHAPE, lambda: l(Y=y[1:]))


def test_layer_refuses_tensors_that_it_would_misread():
    lay = bsp.F8Layer(64, 32, 8, 8, torch.float32, device="cpu")
    x, y = torch.zeros(8, 32), torch.zeros(8, 64)
    for call in (lambda: lay.quantize(torch.zeros(32, 64).t()), lambda: lay.linear(torch.zeros(32, 8).t(), None, y, S), lambda: lay.linear(x, None, torch.zeros(64, 8).t(), S),
                 lambda: lay.linear(torch.zeros(8, 40), None, y, S), lambda: lay.linear(x, None, torch.zeros(8, 32), S),
                 lambda: lay.forward(x, None, None, torch.zeros(9, 64), S), lambda: lay.backward(y, None, None, dX=torch.zeros(8, 64), stream=S)):
        with pytest.raises(ValueError):
            call()
    gamma = torch.ones(32, dtype=torch.uint8)
    for call in (lambda: lay.quantize(torch.zeros(64, 32, dtype=torch.bfloat16)), lambda: lay.quantize(torch.zeros(64, 32), gamma[:31]), lambda: lay.quantize(torch.zeros(64, 32), gamma.bool()),
                 lambda: lay.linear(x, torch.zeros(64, dtype=torch.bfloat16), y, S), lambda: lay.linear(x, torch.zeros(63), y, S), lambda: lay.linear(torch.zeros(1025, 32), None, torch.zeros(1025, 64), S),
                 lambda: lay.backward(y, None, None, dW=torch.zeros(64, 32, dtype=torch.bfloat16), stream=S), lambda: lay.backward(y, None, None, db=torch.zeros(32), stream=S),
                 lambda: lay.linear(x.to("meta"), None, y, S)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        bsp.bsp_gemm_f8(bsp.wdesc(8, 8, 1, 1, 8, 8, bsp.F32), matrix(8, 8), None, y, bsp.F32, y, S)


@pytest.mark.parametrize("P,C,stride", [(8, 32, (0, 1)), (8, 32, (4, 1)), (8, 32, (31, 1)), (2, 32, (0, 1)), (8, 1, (0, 1)), (8, 1, (0, 0))])
def test_layer_refuses_rows_that_overlap(P, C, stride):
    """Expanded and overlapping matrices, whose rows are fewer entries apart than they are long (the gradient of a sum over positions has
    stride (0, 1)): no distance of rows describes them to the library."""
    x = torch.zeros(P * 32).as_strided((P, C), stride)
    with pytest.raises(ValueError, match="X: .*rows"):
        bsp._row_distance(x, "X")
    if C == 1:
        return
    lay, sq, y = bsp.F8Layer(64, 32, 8, 8, torch.float32, device="cpu"), bsp.F8Layer(32, 32, 8, 8, torch.float32, device="cpu"), torch.zeros(P, 64)
    act = bsp.F8Activations(P, 32, device="cpu")
    for call in (lambda: lay.linear(x, None, y, S), lambda: lay.forward(x, act, None, y, S), lambda: sq.backward(x, act, bsp.F8Activations(P, 32, device="cpu"), dX=torch.zeros(P, 32), stream=S)):
        with pytest.raises(ValueError, match="rows"):
            call()


def test_row_distance():
    assert bsp._row_distance(torch.zeros(8, 32), "X") == 32
    assert bsp._row_distance(torch.zeros(8, 40)[:, :32], "X") == 40
    assert bsp._row_distance(torch.zeros(8 * 50).as_strided((8, 1), (50, 7)), "X") == 50
    for first in (0, 1, 32, 100):                                        # of a single row it is not used
        assert bsp._row_distance(torch.zeros(200).as_strided((1, 32), (first, 1)), "X") >= 32
    assert bsp._row_distance(torch.zeros(1, 32).expand(1, 32), "X") == 32


def test_layer_takes_buffers_of_the_right_size_and_device_only():
    """What a step keeps in 8 bits, `act` and `grad`: made for other sizes, on another device, missing or one in place of the other, they are
    refused before anything is enqueued."""
    P, O, I = 8, 64, 32
    lay = bsp.F8Layer(O, I, 8, 8, torch.float32, device="cpu")
    held = lambda p, c, d="cpu": bsp.F8Activations(p, c, device=d)  # noqa: E731
    x, y, dy, dx, dw = torch.zeros(P, I), torch.zeros(P, O), torch.zeros(P, O), torch.zeros(P, I), torch.zeros(O, I)
    act, grad = held(P, I), held(P, O)
    forward = lambda a: lay.forward(x, a, None, y, S)  # noqa: E731
    backward = lambda a, g, **k: lay.backward(dy, a, g, stream=S, **k)  # noqa: E731
    calls = [lambda a=a: forward(a) for a in (None, held(P + 1, I), held(P, I + 8), held(P, I, "meta"), act.rows)]
    calls += [lambda g=g: backward(act, g, dX=dx) for g in (None, held(P + 1, O), held(P, O + 8), held(P, O, "meta"), act)]
    calls += [lambda a=a: backward(a, grad, dX=dx, dW=dw) for a in (None, held(P + 1, I), held(P, I + 8), held(P, I, "meta"))]
    square, both = bsp.F8Layer(I, I, 8, 8, torch.float32, device="cpu"), held(P, I)
    calls.append(lambda: square.backward(x, both, both, dW=torch.zeros(I, I), stream=S))         # dY would be written over the checkpoint
    for call in calls:
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("t", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_8_bit_types_are_those_of_8_bit_matrices_only(t):
    """A tensor of plain entries has none of them: refused where its type is named, as every type is that the library does not know."""
    for make in (lambda: bsp.SparseLayer(64, 64, 1, 1, 8, 8, t, device="cpu"), lambda: bsp.F8Layer(64, 64, 8, 8, t, device="cpu"),
                 lambda: bsp.wdesc(64, 64, 1, 1, 8, 8, t), lambda: bsp.dtype_code(t)):
        with pytest.raises(KeyError):
            make()
    lay = bsp.SparseLayer(64, 64, 1, 1, 8, 8, torch.bfloat16, device="cpu")
    with pytest.raises(KeyError):
        lay.gemm(torch.zeros(8, 64, dtype=torch.bfloat16), None, torch.zeros(8, 64).to(t), S)
    assert bsp.F8Matrix(4, 4, t, device="cpu").m.type == (bsp.E4M3 if t == torch.float8_e4m3fn else bsp.E5M2)


def test_misaligned_workspaces_are_refused():
    """The quantiser writes words to its workspace, the products a status word and (the layer) 16-byte pieces: none of it off its alignment."""
    odd, y = buffer()[2:], buffer(4096, torch.float32)
    x, w = matrix(8, 32), matrix(64, 32)
    refused(bsp.ERR_SHAPE, lambda: bsp.bsp_quantize_f8(y, bsp.F32, 8, 32, 32, x, None, y, odd, S))
    refused(bsp.ERR_SHAPE, lambda: bsp.bsp_gemm_f8(x, w, None, y, bsp.F32, odd, S))
    refused(bsp.ERR_SHAPE, lambda: bsp.bsp_gemm_f8_dw(bsp.wdesc(64, 32, 1, 1, 8, 8, bsp.F32), None, matrix(64, 100), matrix(32, 100), y, odd, S))
    refused(bsp.ERR_SHAPE, lambda: bsp.bsp_linear_f8(w, y, bsp.F32, 8, 32, None, y, bsp.F32, odd, S))
