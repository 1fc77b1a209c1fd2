"""Plain fp64 forms of the history operators: sampling with sinks, the quantised row cache, attention of one query per root
and head with a time bias by buckets, and its gradients.  One loop per root and head, no blocking; used by tests only."""
from __future__ import annotations

import numpy as np


def visible(ts, a, b, t, window, sinks):
    """Entries of the slice [a, b) that a root of time t sees: (len, [window, most recent first], [sinks, oldest first])."""
    n = 0
    while a + n < b and ts[a + n] < t:
        n += 1
    recent = [n - 1 - j for j in range(min(n, window))]
    return n, recent, list(range(min(sinks, n - len(recent))))


def sample_window(indptr, nbr, eid, ts, nodes, times, window, sinks):
    R, S = len(nodes), window + sinks
    out = dict(nbr=np.full((R, S), -1, np.int32), eid=np.full((R, S), -1, np.int32), ts=np.zeros((R, S)),
               cnt=np.zeros(R, np.int32), first=np.zeros(R, np.int64), len=np.zeros(R, np.int32))
    for i in range(R):
        if not 0 <= nodes[i] < len(indptr) - 1:
            continue
        a, b = int(indptr[nodes[i]]), int(indptr[nodes[i] + 1])
        n, recent, first = visible(ts, a, b, times[i], window, sinks)
        at = [a + j for j in recent + first]
        out["first"][i], out["len"][i], out["cnt"][i] = a, n, len(at)
        out["nbr"][i, :len(at)], out["eid"][i, :len(at)], out["ts"][i, :len(at)] = nbr[at], eid[at], ts[at]
    return out


def bf16_up(s):
    """The least bf16 number that is not below the fp32 numbers s >= 0."""
    bits = np.asarray(s, np.float32).view(np.uint32).astype(np.uint64)
    return ((bits + 0xFFFF) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def quantise(x, bits):
    """Codes (int) and scales (fp32 values of bf16) of the groups along the last axis of x (fp32-valued)."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        amax = np.abs(x).max(-1)
        bad = ~np.isfinite(x).all(-1)
        s = bf16_up((np.where(bad, 0.0, amax).astype(np.float32) * (np.float32(1) / np.float32(7 if bits == 4 else 127))).astype(np.float32))
        s = np.where(amax < 2.0 ** -100, np.float32(0), s).astype(np.float32)
        r = np.where(s > 0, np.float32(1) / s, np.float32(0)).astype(np.float32)
        codes = np.rint(np.where(bad[..., None], 0.0, x) * r[..., None].astype(np.float64))
    return codes.astype(np.int64), np.where(bad, np.float32(np.nan), s).astype(np.float32)


def dequantise(codes, scales, most=float(np.finfo(np.float32).max)):
    """Code times scale.  The scale is rounded up to bf16, so the product may pass the row type's largest finite value `most` by 2^-7 of
    it: it is held there; what is further out is left as it is."""
    x = codes.astype(np.float64) * scales[..., None].astype(np.float64)
    return np.where((np.abs(x) > most) & (np.abs(x) <= most * (1 + 2.0 ** -7) * (1 + 2.0 ** -20)), np.copysign(most, x), x)


def bucket(bounds, dt):
    return int(sum(1 for b in bounds if b <= dt))


def softmax(z):
    """Weights of logits; all zero where there is no logit above -infinity."""
    if len(z) == 0 or np.max(z) == -np.inf:
        return np.zeros(len(z))
    e = np.exp(z - np.max(z))
    return e / e.sum()


def attend(q, rows_k, rows_v, seen, bias, buckets, scale):
    """q [R, H, D]; rows_k, rows_v [N, KV, D]; seen[r]: row numbers; buckets[r]: their buckets (or bias None) -> out [R, H, D]."""
    R, H, D = q.shape
    G = H // rows_k.shape[1]
    out = np.zeros((R, H, D))
    for r in range(R):
        for h in range(H):
            k, v = rows_k[seen[r], h // G], rows_v[seen[r], h // G]
            z = scale * (k @ q[r, h])
            if bias is not None:
                z = z + bias[h][buckets[r]]
            p = softmax(z)
            out[r, h] = p @ v if len(p) else 0.0
    return out


def slot_attend(q, k, v, cnt, bias, buckets, scale):
    """k, v [R, S, KV, D], the first cnt[r] slots count; buckets [R, S]."""
    R, H, D = q.shape
    G = H // k.shape[2]
    out = np.zeros((R, H, D))
    for r in range(R):
        n = cnt[r]
        for h in range(H):
            z = scale * (k[r, :n, h // G] @ q[r, h])
            if bias is not None:
                z = z + bias[h][buckets[r, :n]]
            out[r, h] = softmax(z) @ v[r, :n, h // G] if n else 0.0
    return out


def slot_attend_backward(q, k, v, cnt, bias, buckets, scale, dout):
    """(dq, dk, dv, dbias) and, for error bounds, the sum of the magnitudes of dbias's terms."""
    R, H, D = q.shape
    G = H // k.shape[2]
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    db = None if bias is None else np.zeros(bias.shape)
    mag = None if bias is None else np.zeros(bias.shape)
    for r in range(R):
        n = cnt[r]
        for h in range(H):
            kv = h // G
            z = scale * (k[r, :n, kv] @ q[r, h])
            if bias is not None:
                z = z + bias[h][buckets[r, :n]]
            p = softmax(z)
            dp = v[r, :n, kv] @ dout[r, h]
            dz = p * (dp - (p * dp).sum())
            dq[r, h] = scale * (dz @ k[r, :n, kv]) if n else 0.0
            dk[r, :n, kv] += scale * np.outer(dz, q[r, h])
            dv[r, :n, kv] += np.outer(p, dout[r, h])
            if bias is not None:
                np.add.at(db[h], buckets[r, :n], dz)
                np.add.at(mag[h], buckets[r, :n], p * (np.abs(dp) + abs((p * dp).sum())))
    return dq, dk, dv, db, mag
