"""Helpers for the tests of the 8-bit floating-point operators: 8-bit matrices between numpy codes and the device, inputs, tolerances."""
import re

import numpy as np
import torch

from oracle import f8
from paper_2407_09453_b200 import bsp, synth

FTYPE = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
XTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS2 = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}          # half a step, relative


def values(seed, R, K, dtype, std=1.0):
    """Normal entries whose rows and stretches of 64 columns differ in size, rounded to their storage type."""
    x = synth.normal(seed, (R, K), std)
    x = x * np.exp2(synth.uniform_int(seed + 1, (R, 1), -6, 6)) * np.repeat(np.exp2(synth.uniform_int(seed + 2, (1, -(-K // 64)), -4, 4)), 64, axis=1)[:, :K]
    x = x.astype(np.float32)
    return synth.round_to_bf16(x) if dtype == "bf16" else x


def device(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(XTYPE[dtype])


def held(codes, scales, ftype, junk=0x55):
    """An F8Matrix with these codes and scales, junk in the padding of its rows."""
    R, K = codes.shape
    m = bsp.F8Matrix(R, K, FTYPE[ftype])
    data = np.full((R, m.data.shape[1]), junk, np.uint8)
    data[:, :K] = codes
    m.data.view(torch.uint8).copy_(torch.from_numpy(data))
    m.scale.copy_(torch.from_numpy(f8.pack_scales(scales, K)))
    return m


def codes_of(m):
    """Codes and scale bytes of an F8Matrix."""
    return m.data.view(torch.uint8).cpu().numpy()[:, :m.cols], f8.unpack_scales(m.scale.cpu().numpy(), m.rows, m.cols)


def random_held(seed, R, K, ftype, std=1.0):
    """A random 8-bit matrix: its device form and its values in float64."""
    codes, scales = f8.quantize(values(seed, R, K, "f32", std), ftype)
    return held(codes, scales, ftype), f8.dequantize(codes, scales, ftype)


def product_bound(x, w, want, out):
    """How far Y = x w^t may be off: the products are exact, and each of the additions (32 products an instruction, then up to eight ranges and the
    bias) is off by at most one step of float32, 2^-23, of what can have been summed by then, which the sum of the magnitudes
    bounds; and half a step of the output's type."""
    steps = -(-x.shape[1] // 32) + 9
    return steps * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T) * 1.01 + EPS2[out] * np.abs(want) * 1.01 + 1e-37


def launches(call):
    """The kernels that `call` launches, in order, as (name, CTAs): captured into a graph, whose nodes are read and which never runs."""
    from cuda.bindings import driver

    def ok(r):
        assert int(r[0]) == 0, r[0]
        return r[1:] if len(r) != 2 else r[1]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw = driver.CUgraph(int(graph.raw_cuda_graph()))
    nodes, count = ok(driver.cuGraphGetNodes(raw, 64))
    found = []
    for n in nodes[:count]:
        if ok(driver.cuGraphNodeGetType(n)) != driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            continue
        k = ok(driver.cuGraphKernelNodeGetParams(n))
        name = ok(driver.cuFuncGetName(k.func)) if int(k.func) else ok(driver.cuKernelGetName(k.kern))
        found.append((name.decode(), k.gridDimX))
    return found


def template(name):
    """`kernel<arguments>` of a mangled name, arguments as mangled: ("gemm_f8_pair_kernel", "Lb1ELb1E")."""
    m = re.search(r"\d+((?:gemm|quantize|dequantize)_f8_(?:any_)?(?:tile_|pair_)?kernel)I(.*?)EEv", name)
    return m.groups() if m else (name, "")
