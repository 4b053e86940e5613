"""Plain 64-bit forms of the operators in include/gptq_w4a16_serving.h, and bounds of their rounding errors (numpy)."""
import numpy as np

U16, U32 = 2.0 ** -11, 2.0 ** -24  # half a unit in the last place, relative: fp16, fp32


def dequant64(qweight, qzeros, scales):
    """float64 [K, N] = scale * (q - z), not rounded."""
    shift = np.arange(0, 32, 4, dtype=np.uint32)
    q = (qweight.view(np.uint32)[:, None, :] >> shift[None, :, None] & 15).reshape(-1, qweight.shape[1]).astype(np.int64)
    z = (qzeros.view(np.uint32)[:, :, None] >> shift & 15).reshape(qzeros.shape[0], -1).astype(np.int64)
    per = q.shape[0] // z.shape[0]
    return (q - np.repeat(z, per, 0)) * np.repeat(scales.astype(np.float64), per, 0)


def random_packed(rng, K, N, group, *lead):
    words = lambda *s: rng.integers(0, 2 ** 32, size=s, dtype=np.uint32).view(np.int32)  # noqa: E731
    return (words(*lead, K // 8, N), words(*lead, K // group, N // 8),
            rng.uniform(0.001, 0.01, size=(*lead, K // group, N)).astype(np.float16))


def route64(logits, top_k, renormalize):
    """ids and weights by definition: masked are NaN and -inf; infinities of the top share the weight."""
    M, E = logits.shape
    ids, weights = np.full((M, top_k), -1, np.int32), np.zeros((M, top_k))
    for m in range(M):
        l = [float(v) for v in logits[m]]
        order = sorted((e for e in range(E) if l[e] > -np.inf), key=lambda e: (-l[e], e))
        if not order:
            continue
        top = l[order[0]]
        share = {e: 1.0 if l[e] == top else np.exp(l[e] - top) for e in order}
        chosen = order[:top_k]
        total = sum(share[e] for e in (chosen if renormalize else order))
        for j, e in enumerate(chosen):
            ids[m, j], weights[m, j] = e, share[e] / total
    return ids, weights


def experts64(x, ids, weights, gate_up, down):
    """The layer's output, and a bound of its error.  With a = sums of absolute products: fp32 sums of n terms are off by n U32
    of a at most; the activation moves with gate (slope of silu at most 1.1) and up, and is rounded to fp16; the products of
    down are summed alike; the output is rounded to fp16."""
    M, hidden = x.shape
    E, inter = gate_up[0].shape[0], gate_up[0].shape[2] // 2
    out, off = np.zeros((M, hidden)), np.zeros((M, hidden))
    x = x.astype(np.float64)
    for e in range(E):
        rows, places = np.nonzero(ids == e)
        if len(rows) == 0:
            continue
        w13 = dequant64(*(t[e] for t in gate_up))
        w2 = dequant64(*(t[e] for t in down))
        with np.errstate(over="ignore"):
            gu, agu = x[rows] @ w13, np.abs(x[rows]) @ np.abs(w13)
            g, u = gu[:, :inter], gu[:, inter:]
            d = (hidden + 8) * U32
            dg, du = d * agu[:, :inter], d * agu[:, inter:]
            silu = g / (1 + np.exp(-g))
        h = silu * u
        dh = 1.1 * dg * np.abs(u) + (np.abs(silu) + dg) * du + np.abs(h) * (U16 + 16 * U32) + 2.0 ** -25
        wt = weights[rows, places].astype(np.float64)[:, None]
        np.add.at(out, rows, wt * (h @ w2))
        np.add.at(off, rows, np.abs(wt) * (dh @ np.abs(w2) + (inter + 8) * U32 * (np.abs(h) @ np.abs(w2))))
    return out, off + U16 * (np.abs(out) + off) + 2.0 ** -25


def lora64(x, a, b, scaling, adapter, base):
    """base plus every row's adapter, and a bound of the error: two fp32 sums, then one rounding to fp16."""
    out = base.astype(np.float64).copy()
    off = np.zeros_like(out)
    x = x.astype(np.float64)
    K, rank = a.shape[2], a.shape[1]
    for m, l in enumerate(adapter):
        if not 0 <= l < len(scaling):
            continue
        al, bl, s = a[l].astype(np.float64), b[l].astype(np.float64), float(scaling[l])
        out[m] += s * (bl @ (al @ x[m]))
        off[m] = abs(s) * (K + rank + 16) * U32 * (np.abs(bl) @ (np.abs(al) @ np.abs(x[m])))
    rounded = np.array([0 <= l < len(scaling) for l in adapter])[:, None]
    return out, np.where(rounded, off + 4 * U32 * np.abs(base.astype(np.float64)) + U16 * (np.abs(out) + off) + 2.0 ** -25, 0.0)
