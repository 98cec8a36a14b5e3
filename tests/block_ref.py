"""The operators around the expert layer in 64 bits on the CPU, from their definitions: numpy only, and independent of the
library."""
import numpy as np

import expert_ref as ref

EPS = 2.0 ** -24  # half a step of fp32


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else EPS


def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1 / (1 + e), e / (1 + e))


def choose(z, topk, bias=None):
    """int32 [T, k] by repeated search: the largest score, the first among equals, -1 where none can be chosen."""
    T, E = z.shape
    key = z if bias is None else sigmoid(z) + bias
    out = np.full((T, topk), -1, dtype=np.int32)
    for t in range(T):
        left = [(np.inf if np.isnan(key[t, e]) else key[t, e], int(np.isnan(key[t, e])), e) for e in range(E)
                if z[t, e] != -np.inf and (bias is None or bias[e] != -np.inf)]
        left.sort(key=lambda v: (-v[1], -v[0], v[2]))
        for j, v in enumerate(left[:topk]):
            out[t, j] = v[2]
    return out


def gate(z, idx, score, normalize):
    """(scores of all experts, weights [T, k] before the factor), from logarithms, so that nothing vanishes."""
    with np.errstate(all="ignore"):
        if score == "softmax":
            top = z.max(1, keepdims=True)
            top = np.where(np.isfinite(top), top, 0)
            logp = z - top - np.log(np.exp(z - top).sum(1, keepdims=True))
        else:
            logp = np.where(z >= 0, -np.log1p(np.exp(-np.abs(z))), z - np.log1p(np.exp(-np.abs(z))))
        chosen = np.where(idx >= 0, np.take_along_axis(logp, np.maximum(idx, 0), 1), -np.inf)
        if normalize:
            top = chosen.max(1, keepdims=True)
            top = np.where(np.isfinite(top), top, 0)
            chosen = chosen - top - np.log(np.exp(chosen - top).sum(1, keepdims=True))
        w = np.where(np.isneginf(chosen) | (idx < 0), 0.0, np.exp(chosen))
        return np.exp(logp), w


def route_grad(g, z, idx, score, normalize, factor):
    p, q = gate(z, idx, score, normalize)
    T, E = z.shape
    d = np.zeros((T, E))
    for t in range(T):
        s = sum(q[t, j] * g[t, j] for j in range(idx.shape[1]))
        for j, e in enumerate(idx[t]):
            if e < 0:
                continue
            if normalize:
                d[t, e] += q[t, j] * (g[t, j] - s) * (1 if score == "softmax" else 1 - p[t, e])
            elif score == "sigmoid":
                d[t, e] += g[t, j] * p[t, e] * (1 - p[t, e])
            else:
                d[t, e] += p[t, e] * g[t, j]
        if score == "softmax" and not normalize:
            d[t] -= np.where(z[t] == -np.inf, 0, p[t]) * s
    return factor * d


def swiglu(gu):
    g, u = np.split(gu, 2, 1)
    return g * sigmoid(g) * u


def swiglu_grad(dout, gu):
    g, u = np.split(gu, 2, 1)
    s = sigmoid(g)
    return np.concatenate([dout * u * s * (1 + g * (1 - s)), dout * g * s], 1)


def weights8(values, kind):
    """A weight matrix [E, n, k] as the library keeps it: (float64 values, e4m3 bytes [E, n, width], scales)."""
    E, n, k = values.shape
    q, s, v = [], [], []
    for m in values:
        qe, se = ref.quantize(m, kind, 128)
        q.append(qe)
        s.append(se)
        v.append(ref.dequantize(qe, se, 128)[:, :k])
    return np.stack(v), np.stack(q), np.stack(s)


def few(x, idx, w, w1, w2, first, h_bits=None):
    """(out, bound) of the layer on these values; bound: what fp32 sums and a rounding of h to `h_bits` can cost, without
    the last rounding of out.  Sums of m products lose (m + 8) 2^-24 of their magnitudes; the sigmoid and the products of h
    14 units of 2^-24; silu's slope is below 1.1."""
    T, H = x.shape
    E, _, I = w2.shape
    out, bound = np.zeros((T, w2.shape[1])), np.zeros((T, w2.shape[1]))
    for e in range(E):
        hit = (idx.astype(np.int64) == first + e)
        for t in np.nonzero(hit.any(1))[0]:
            weight = w[t][hit[t]].sum()
            gu, mag = w1[e] @ x[t], np.abs(w1[e]) @ np.abs(x[t])
            g, u = gu[:I], gu[I:]
            dg, du = (H + 8) * EPS * mag[:I], (H + 8) * EPS * mag[I:]
            silu = g * sigmoid(g)
            h = weight * silu * u
            dh = abs(weight) * (1.1 * np.abs(u) * dg + np.abs(silu) * du + 1.1 * dg * du) + 16 * EPS * np.abs(h) + \
                (0 if h_bits is None else 2.0 ** -h_bits * np.abs(h))
            out[t] += w2[e] @ h
            bound[t] += np.abs(w2[e]) @ (dh + (I * idx.shape[1] + 24) * EPS * np.abs(h))
    return out, bound
