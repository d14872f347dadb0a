"""The operators around a verification round by their definitions, in 64 bits on the CPU (numpy), one row at a time."""
import math

import numpy as np


def clean_parents(parents, tq):
    """Parent indices of the nodes that exist; anything that is not an earlier node counts as the committed token."""
    return [p if -1 <= p < i else -1 for i, p in enumerate(parents[:tq])]


def ancestors(parents, tq):
    lines = []
    for i, p in enumerate(clean_parents(parents, tq)):
        lines.append([i] + (lines[p] if p >= 0 else []))
    return lines


def prefix_attention(q, kp, vp, k, v, plens, lens, nq, parents, scale):
    """q [B,T,H,dk]; kp, vp [G,Hkv,P,d]; k, v [B,Hkv,S,d]; all float64.  Returns out and, per output value, the sum of
    p |v| (what relative errors of the probabilities act on) and the largest sum of |q_i k_i| scale of a row."""
    B, T, H, _ = q.shape
    G, Hk, dv = kp.shape[0] if kp is not None else B, k.shape[1], v.shape[3]
    out, mass, size = np.zeros((B, T, H, dv)), np.zeros((B, T, H, dv)), np.zeros((B, T, H, 1))
    for b in range(B):
        g = b // (B // G)
        lines = ancestors(parents[b] if parents is not None else list(range(-1, T - 1)), nq[b])
        for h in range(H):
            c = h // (H // Hk)
            ks, vs = (([kp[g, c, :plens[g]]], [vp[g, c, :plens[g]]]) if kp is not None else ([], []))
            for i in range(nq[b]):
                rows = list(range(lens[b])) + sorted(lens[b] + a for a in lines[i])
                keys, vals = np.concatenate(ks + [k[b, c, rows]]), np.concatenate(vs + [v[b, c, rows]])
                x = scale * (keys @ q[b, i, h])
                p = np.exp(x - x.max())
                p /= p.sum()
                out[b, i, h], mass[b, i, h] = p @ vals, p @ np.abs(vals)
                size[b, i, h] = scale * (np.abs(keys) @ np.abs(q[b, i, h])).max()
    return out, mass, size


def sample(x, t, top_k, top_p, min_p, u):
    """(token, probability, margin): margin is how near u's target lies to a border, relative to the kept sum."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    top = x.max()
    if top == -np.inf:
        return -1, 0.0, 1.0
    if not t > 0:
        return int(np.argmax(x)), 1.0, 1.0
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        w = np.where(x == top, 1.0, np.where(x == -np.inf, 0.0, np.exp((x - top) / t)))
    order = np.argsort(-x, kind="stable")
    ws = w[order]
    n_k = top_k if 0 < top_k < len(x) else len(x)
    n = n_k
    if not (top_p >= 1 or math.isnan(top_p)):
        upto = np.cumsum(ws[:n_k])
        n = 1 if top_p <= 0 else min(n_k, int(np.sum(upto < top_p * upto[-1])) + 1)
    if min_p > 0:
        n = min(n, int(np.sum(x == top)) if min_p >= 1 else int(np.sum(ws >= min_p)))
    kept = np.zeros(len(x))
    kept[order[:n]] = ws[:n]
    c = np.cumsum(kept)
    u = 0.0 if not u >= 0 else u
    target = u * c[-1]
    over = np.nonzero(c > target)[0] if u < 1 else []
    token = int(over[0]) if len(over) else int(np.nonzero(kept)[0][-1])
    return token, kept[token] / c[-1], float(np.min(np.abs(c - target)) / c[-1]) if 0 < u < 1 else 1.0


def accept(draft, root, sampled, length, nq, parents):
    """(path, next token, committed length) of one sequence."""
    parents = clean_parents(parents, nq)
    at, want, path = -1, int(root), []
    while want >= 0:
        fit = [i for i in range(nq) if parents[i] == at and draft[i] == want]
        if not fit:
            break
        at = fit[0]
        path.append(at)
        want = int(sampled[at])
    return path, want, length + len(path)


def commit(rows, path, n, length, T, cap):
    """rows [rows, d] of one (layer, sequence, KV head), moved."""
    out, before = rows.copy(), -1
    for j in range(min(n, T)):
        if not (before < path[j] < T) or length < 0 or length + path[j] >= cap:
            break
        out[length + j] = rows[length + path[j]]
        before = path[j]
    return out
