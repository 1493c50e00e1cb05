"""Plain CPU definitions of the operators around a sparse block with group-scaled weights, in float64.

Independent of the CUDA path: loops and elementary numpy operations, written from the definitions in the C header.
"""
import numpy as np

from .singlequant_oracle import rotate

# nibble position of channel c within a 32-bit word of eight channels (weight-only order)
POSITION = (0, 4, 1, 5, 2, 6, 3, 7)


def rotate_rows(W, R1, R2):
    return W.astype(np.float64) if R1 is None else rotate(W, R1, R2)


def quantise_groups(Z, group, bits, offset):
    """Rows of fp32 values -> (codes [N, K], sg [G, N] fp16, bg [G, N] fp16 or None); the decision in fp32, as the library states it."""
    Z = np.asarray(Z, np.float32)
    N, K = Z.shape
    G = -(-K // group)
    cmin, cmax = -(1 << (bits - 1)), (1 << (bits - 1)) - 1
    codes = np.zeros((N, K), np.int64)
    sg, bg = np.zeros((G, N), np.float16), np.zeros((G, N), np.float16)
    for g in range(G):
        part = Z[:, g * group:(g + 1) * group]
        if offset:
            lo, hi = part.min(1), part.max(1)
            sg[g] = ((hi - lo) / np.float32(cmax - cmin)).astype(np.float16)
            bg[g] = (lo - np.float32(cmin) * sg[g].astype(np.float32)).astype(np.float16)
        else:
            sg[g] = (np.abs(part).max(1) / np.float32(cmax)).astype(np.float16)
        step = sg[g].astype(np.float32)[:, None]
        with np.errstate(divide="ignore"):
            inv = np.where(step > 0, np.float32(1) / step, np.float32(0)).astype(np.float32)
        t = (part - bg[g].astype(np.float32)[:, None]) * inv + np.float32(0.5)
        codes[:, g * group:(g + 1) * group] = np.clip(np.floor(t), cmin, cmax)
    return codes, sg, (bg if offset else None)


def pack_codes(codes):
    """Codes [N, K] -> bytes [N, K/2] in the weight-only order."""
    N, K = codes.shape
    words = np.zeros((N, K // 8), np.uint32)
    for c in range(8):
        words |= (codes[:, c::8] & 15).astype(np.uint32) << np.uint32(4 * POSITION[c])
    return words.view(np.uint8).reshape(N, K // 2)


def weights(codes, sg, bg, group):
    """w[c, k] = code * sg[k / group, c] + bg[k / group, c] in float64."""
    g = np.arange(codes.shape[1]) // group
    w = codes * sg.astype(np.float64)[g].T
    return w if bg is None else w + bg.astype(np.float64)[g].T


def experts(Z, w, row_token, offsets, M):
    """Rows offsets[e] .. offsets[e + 1] - 1 times expert e's weights; rows behind the last are NaN."""
    Y = np.full((M, w[0].shape[0]), np.nan)
    for e in range(len(w)):
        for r in range(offsets[e], offsets[e + 1]):
            Y[r] = w[e] @ Z[row_token[r]].astype(np.float64)
    return Y


def route(logits, k, renorm, mask=None):
    x = np.array(logits, np.float64)
    x[np.isnan(x)] = -np.inf
    T, E = x.shape
    ids, gates = np.full((T, k), -1), np.zeros((T, k))
    p, n = np.zeros((T, E)), 0
    for t in range(T):
        if (mask is not None and not mask[t]) or x[t].max() == -np.inf:
            continue
        n += 1
        m = x[t].max()
        with np.errstate(invalid="ignore"):
            e = np.where(x[t] == m, 1.0, np.exp(x[t] - m))
        p[t] = e / e.sum()
        order = sorted(range(E), key=lambda i: (-x[t, i], i))
        order = [i for i in order if x[t, i] > -np.inf][:k]
        ids[t, :len(order)] = order
        gates[t, :len(order)] = p[t, order] if not renorm else e[order] / e[order].sum()
    counts = np.array([(ids == e).sum() for e in range(E)])
    offsets = np.concatenate([[0], np.cumsum(counts)])
    pos, row_token, nxt = np.full((T, k), -1), np.full(T * k, -1), offsets[:-1].copy()
    for t in range(T):
        for j in range(k):
            if ids[t, j] >= 0:
                pos[t, j] = nxt[ids[t, j]]
                row_token[pos[t, j]] = t
                nxt[ids[t, j]] += 1
    loss = E * np.sum(counts / (k * n) * p.sum(0) / n) if n else 0.0
    return {"ids": ids, "gates": gates, "counts": np.append(counts, n), "offsets": offsets, "row_token": row_token, "pos": pos,
            "loss": loss, "p": p}


def route_backward(r, renorm, dgates, dloss):
    """The gradient for the result `r` of route, from the Jacobian of every token's softmax."""
    p, ids = r["p"], r["ids"]
    T, E = p.shape
    k, n = ids.shape[1], r["counts"][-1]
    out = np.zeros((T, E))
    for t in range(T):
        if p[t].sum() == 0:
            continue
        J = np.diag(p[t]) - np.outer(p[t], p[t])                    # dp / dl
        d = dloss * E * r["counts"][:E] / (k * n) / n
        sel = ids[t][ids[t] >= 0]
        dg = dgates[t][ids[t] >= 0]
        if renorm:
            q = r["gates"][t][ids[t] >= 0]
            out[t, sel] += (np.diag(q) - np.outer(q, q)) @ dg
        else:
            d = d.copy()
            d[sel] += dg
        out[t] += J @ d
    return out


def combine(Y, pos, gates):
    T, k = pos.shape
    out = np.zeros((T, Y.shape[1]))
    for t in range(T):
        for j in range(k):
            if 0 <= pos[t, j] < len(Y):
                out[t] += gates[t, j] * Y[pos[t, j]].astype(np.float64)
    return out


def combine_backward(dout, Y, pos, gates):
    """(dY with NaN in the rows that no slot names, dgates)."""
    T, k = pos.shape
    dY, dg = np.full(Y.shape, np.nan), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            if 0 <= pos[t, j] < len(Y):
                dY[pos[t, j]] = np.float64(gates[t, j]) * dout[t].astype(np.float64)
                dg[t, j] = dout[t].astype(np.float64) @ Y[pos[t, j]].astype(np.float64)
    return dY, dg
