"""The expert layer's operators in 64 bits on the CPU, from their definitions: numpy only, slot by slot where the order
matters, and independent of the library."""
import numpy as np

BLOCK = 128
MIN = 2.0 ** -126


def width(cols):
    return -(-cols // BLOCK) * BLOCK


def pitch(cols):
    return -(-(width(cols) // BLOCK) // 4) * 4


def cols_width(rows, groups):
    return BLOCK * (rows // BLOCK + groups)


def sort(topk, first, experts):
    T, k = topk.shape
    rows = [[] for _ in range(experts)]
    for s, e in enumerate(topk.reshape(-1).astype(np.int64)):
        if first <= e < first + experts:
            rows[e - first].append(s)
    order = [s for r in rows for s in r]
    offsets = np.concatenate([[0], np.cumsum([len(r) for r in rows])]).astype(np.int32)
    slot_of = np.full(T * k, -1, dtype=np.int32)
    slot_of[:len(order)] = order
    row_of = np.full(T * k, -1, dtype=np.int32)
    row_of[order] = np.arange(len(order))
    return offsets, slot_of, row_of.reshape(T, k)


# The 256 values of e4m3.
def _e4m3(b):
    s, e, m = b >> 7, b >> 3 & 15, b & 7
    if b & 127 == 127:
        return np.nan
    v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
    return -v if s else v


E4M3 = np.array([_e4m3(b) for b in range(256)])


def round_e4m3(v):
    """Nearest e4m3 values of float64 values of magnitude up to 448, ties to even."""
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 1e-300))), -6)
    step = 2.0 ** (e - 3)
    return np.round(v / step) * step


def scale_of(amax, kind):
    """fp32 scale of blocks with these largest magnitudes, by the stated rule (the division is fp32)."""
    with np.errstate(all="ignore"):
        s = np.maximum((amax.astype(np.float32) / np.float32(448)).astype(np.float32), np.float32(MIN))
        if kind == "e8m0":
            m, e = np.frexp(s.astype(np.float64))
            s = np.ldexp(1.0, np.where(m == 0.5, e - 1, e))
        return np.where(np.isfinite(amax), s, np.nan).astype(np.float64)


def quantize(x, kind, rows_block=1):
    """x float64 [n, k]: (values before their scale, scales [ceil(n / rows_block), k blocks])."""
    n, k = x.shape
    v = np.zeros((n, width(k)))
    v[:, :k] = x
    v = v.reshape(n, -1, BLOCK)
    amax = np.where(np.isfinite(v).all(2), np.abs(np.where(np.isfinite(v), v, 0)).max(2), np.inf)
    if rows_block > 1:
        amax = np.stack([amax[i:i + rows_block].max(0) for i in range(0, n, rows_block)])
    s = scale_of(amax, kind)
    each = np.repeat(s, rows_block, 0)[:n][:, :, None]
    r = (np.float32(1) / each.astype(np.float32)).astype(np.float64)
    with np.errstate(all="ignore"):
        q = round_e4m3((v.astype(np.float32) * r.astype(np.float32)).astype(np.float64))
        q = np.where(np.isnan(each), np.nan, q)
    return q.reshape(n, -1), s


def dequantize(q, s, rows_block=1):
    n = q.shape[0]
    return q * np.repeat(np.repeat(s, rows_block, 0)[:n], BLOCK, 1)


def columns(x, offsets, rows):
    """x [rows, H] of grouped rows laid out along the rows: [H, cols_width], zeros where no row falls."""
    groups = len(offsets) - 1
    out = np.zeros((x.shape[1], cols_width(rows, groups)))
    for g in range(groups):
        at = BLOCK * (offsets[g] // BLOCK + g)
        out[:, at:at + offsets[g + 1] - offsets[g]] = x[offsets[g]:offsets[g + 1]].T
    return out
