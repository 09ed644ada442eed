"""Plain numpy oracle of the 8-bit floating-point operators, in 64 bits: formats by their definition, scales, both orientations, products.
Shares nothing with the CUDA path (test infrastructure)."""
import numpy as np

E4M3, E5M2 = "e4m3", "e5m2"
MAX = {E4M3: 448.0, E5M2: 57344.0}


def value(code: int, f8: str) -> float:
    """The value of one byte: sign, 4 (5) exponent bits with bias 7 (15), 3 (2) fraction bits; e4m3 has no infinity and one NaN."""
    ebits, mbits, bias = (4, 3, 7) if f8 == E4M3 else (5, 2, 15)
    s, e, m = code >> 7, code >> mbits & (1 << ebits) - 1, code & (1 << mbits) - 1
    if f8 == E4M3 and (code & 0x7F) == 0x7F:
        return float("nan")
    if f8 == E5M2 and e == 31:
        return float("nan") if m else (-1.0) ** s * float("inf")
    v = m * 2.0 ** (1 - bias - mbits) if e == 0 else (1 + m / (1 << mbits)) * 2.0 ** (e - bias)
    return -v if s else v


TABLE = {f: np.array([value(c, f) for c in range(256)]) for f in (E4M3, E5M2)}


def encode(x: np.ndarray, f8: str) -> np.ndarray:
    """Codes of the nearest finite values (ties to the even code), 0x7F for NaN; |x| is at most MAX."""
    grid = TABLE[f8][:128]
    grid = grid[np.isfinite(grid)]
    v = np.where(np.isnan(x), 0.0, np.abs(x))
    up = np.minimum(np.searchsorted(grid, v), len(grid) - 1)
    down = np.maximum(up - 1, 0)
    du, dd = grid[up] - v, v - grid[down]
    code = np.where((dd < du) | ((dd == du) & (down % 2 == 0)), down, up).astype(np.uint8)
    code = np.where(np.signbit(x), code | 0x80, code).astype(np.uint8)
    return np.where(np.isnan(x), np.uint8(0x7F), code).astype(np.uint8)


def scale_byte(amax, f8: str):
    """Smallest b with amax <= MAX 2^(b - 127), b >= 0; 127 for 0."""
    limits = np.ldexp(MAX[f8], np.arange(255) - 127)
    return np.where(np.asarray(amax) == 0.0, 127, np.searchsorted(limits, amax))


def quantize(x: np.ndarray, f8: str, tile_rows: int = 1):
    """x [R][K] with a scale for tile_rows x 128 entries: codes [R][K] and scale bytes [R][ceil(K / 128)]."""
    x = np.asarray(x, dtype=np.float64)
    x = np.where(np.isinf(x), np.nan, x)
    R, K = x.shape
    tiles = np.pad(x, ((0, -R % tile_rows), (0, -K % 128))).reshape(-(-R // tile_rows), tile_rows, -(-K // 128), 128)
    scales = np.repeat(scale_byte(np.where(np.isnan(tiles), 0.0, np.abs(tiles)).max(axis=(1, 3)), f8), tile_rows, axis=0)[:R]
    return encode(np.ldexp(x, 127 - np.repeat(scales, 128, axis=1)[:, :K]), f8), scales.astype(np.uint8)


def dequantize(codes: np.ndarray, scales: np.ndarray, f8: str) -> np.ndarray:
    K = codes.shape[1]
    return np.ldexp(TABLE[f8][codes], np.repeat(scales.astype(np.int64), 128, axis=1)[:, :K] - 127)


def scale_bytes(rows: int, cols: int) -> int:
    return -(-rows // 128) * -(-cols // 512) * 512


def scale_at(r, b, cols):
    """Place of the scale of row r and block b (bsp_f8 of bsp.h)."""
    return ((r // 128) * -(-cols // 512) + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4


def pack_scales(scales: np.ndarray, cols: int) -> np.ndarray:
    R, nb = scales.shape
    out = np.full(scale_bytes(R, cols), 127, np.uint8)
    r, b = np.meshgrid(np.arange(R), np.arange(nb), indexing="ij")
    out[scale_at(r, b, cols)] = scales
    return out


def unpack_scales(packed: np.ndarray, R: int, cols: int) -> np.ndarray:
    r, b = np.meshgrid(np.arange(R), np.arange(-(-cols // 128)), indexing="ij")
    return packed[scale_at(r, b, cols)]


def spread_gamma(gamma: np.ndarray, O: int, I: int, bo: int, bi: int) -> np.ndarray:
    return np.repeat(np.repeat(gamma.reshape(O // bo, I // bi), bo, axis=0), bi, axis=1) != 0


def masked(w: np.ndarray, gamma, bo: int, bi: int) -> np.ndarray:
    """Gamma (.) W: a dropped weight is zero whatever it holds."""
    return w if gamma is None else np.where(spread_gamma(gamma, *w.shape, bo, bi), w, 0.0)
