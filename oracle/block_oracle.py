"""CPU float64 oracle of what a layer has between its shard GEMMs.  TEST INFRASTRUCTURE ONLY.

The definitions written out with numpy in float64: the norms of a block with its gate and residual (forward and
backward), the rotation of query and key heads with the paged cache they are appended to, and the attention of
one new token per sequence over that cache.  Pinned by tests/test_oracle_block.py against closed forms, finite
differences and the attention core of ntp_oracle.  Imports nothing from the product.
"""
from __future__ import annotations

import numpy as np

RMS, LAYER = 0, 1


def norm_stats(t, kind, eps):
    """Mean (0 for the RMS norm) and reciprocal deviation of every row."""
    mean = t.mean(1) if kind == LAYER else np.zeros(t.shape[0])
    return mean, 1.0 / np.sqrt(((t - mean[:, None]) ** 2).mean(1) + eps)


def _hat(t, stats):
    return (t - stats[0][:, None]) * stats[1][:, None]


def block_norm_fwd(X, Z, w, kind, eps, a=1.0, b=1.0):
    """X' = a X + b gate * post(Z), Y = pre(X'); w: dict of post_gamma, post_beta, gate, pre_gamma, pre_beta (absent: left out).
    Returns (X', Y or None, stats [4, M])."""
    stats = np.zeros((4, X.shape[0]))
    out, Y = X, None
    if Z is not None:
        r = Z
        if "post_gamma" in w:
            stats[0], stats[1] = norm_stats(Z, kind, eps)
            r = _hat(Z, stats[:2]) * w["post_gamma"] + w.get("post_beta", 0.0)
        out = a * X + b * (w.get("gate", 1.0) * r)
    if "pre_gamma" in w:
        stats[2], stats[3] = norm_stats(out, kind, eps)
        Y = _hat(out, stats[2:]) * w["pre_gamma"] + w.get("pre_beta", 0.0)
    return out, Y, stats


def _norm_bwd(up, t, stats, kind):
    """Gradient at t of a row's normalised values whose gradient is `up`."""
    hat = _hat(t, stats)
    d = up - hat * (up * hat).mean(1, keepdims=True)
    if kind == LAYER:
        d = d - up.mean(1, keepdims=True)
    return d * stats[1][:, None]


def block_norm_bwd(dXout, dY, Xout, Z, stats, w, kind, a=1.0, b=1.0, branch=True):
    """Gradients of block_norm_fwd as a dict: dX, dZ (branch) and those of the vectors in w (the gate's as it was given: [H] or [M, H])."""
    G = 0.0 if dXout is None else dXout
    out = {}
    if "pre_gamma" in w:
        hat = _hat(Xout, stats[2:])
        out["pre_gamma"] = (dY * hat).sum(0)
        if "pre_beta" in w:
            out["pre_beta"] = dY.sum(0)
        G = G + _norm_bwd(dY * w["pre_gamma"], Xout, stats[2:], kind)
    out["dX"] = a * G if branch else G
    if branch:
        dr, hat = b * G, Z
        if "post_gamma" in w:
            hat = _hat(Z, stats[:2])
        if "gate" in w:
            r = hat * w["post_gamma"] + w.get("post_beta", 0.0) if "post_gamma" in w else Z
            dg = dr * r
            out["gate"] = dg.sum(0) if w["gate"].ndim == 1 else dg
            dr = dr * w["gate"]
        if "post_gamma" in w:
            out["post_gamma"] = (dr * hat).sum(0)
            if "post_beta" in w:
                out["post_beta"] = dr.sum(0)
            dr = _norm_bwd(dr * w["post_gamma"], Z, stats[:2], kind)
        out["dZ"] = dr
    return out


def rotate(x, positions, inv_freq, interleaved):
    """Heads x [M, heads, d], the first 2 len(inv_freq) elements rotated in pairs by positions * inv_freq."""
    n = len(inv_freq)
    out = np.array(x, dtype=np.float64)
    if n == 0:
        return out
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * np.asarray(inv_freq)[None, None, :]
    c, s = np.cos(angle), np.sin(angle)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    x1, x2 = x[..., first], x[..., second]
    out[..., first], out[..., second] = x1 * c - x2 * s, x2 * c + x1 * s
    return out


def kv_append(QKV, q_cnt, kv_cnt, d, positions, slots, inv_freq, interleaved, K, V):
    """Rotated queries and keys of QKV [M, (q_cnt + 2 kv_cnt) d]; K, V [pages, kv_cnt, page, d] get the keys and values of the rows whose slot
    exists (copies are returned).  Returns (Q [M, q_cnt d], Krot [M, kv_cnt d], K, V)."""
    M = QKV.shape[0]
    x = QKV.reshape(M, q_cnt + 2 * kv_cnt, d)
    qk = rotate(x[:, :q_cnt + kv_cnt], positions, inv_freq, interleaved)
    K, V = K.copy(), V.copy()
    page = K.shape[2]
    for m in range(M):
        s = int(slots[m])
        if 0 <= s < K.shape[0] * page:
            K[s // page, :, s % page] = qk[m, q_cnt:]
            V[s // page, :, s % page] = x[m, q_cnt + kv_cnt:]
    return qk[:, :q_cnt].reshape(M, -1), qk[:, q_cnt:].reshape(M, -1), K, V


def attn_decode(Q, K, V, table, lengths, max_len, q_off, kv_off, group):
    """One new token per sequence: (C [n_seq, q_cnt d], LSE [q_cnt, n_seq], A) with A [n_seq, q_cnt d] = sum p |V| / sum p, the size of what is added."""
    n_seq = Q.shape[0]
    pages, _, page, d = K.shape
    q_cnt = Q.shape[1] // d
    C, A, LSE = np.zeros((n_seq, q_cnt, d)), np.zeros((n_seq, q_cnt, d)), np.full((q_cnt, n_seq), -np.inf)
    for s in range(n_seq):
        at = [(int(table[s][t // page]), t % page) for t in range(min(int(lengths[s]), max_len))]
        at = [(p, t) for p, t in at if 0 <= p < pages]
        if not at:
            continue
        p_of, t_of = np.array([p for p, _ in at]), np.array([t for _, t in at])
        for j in range(q_cnt):
            g = (q_off + j) // group - kv_off
            k, v = K[p_of, g, t_of].astype(np.float64), V[p_of, g, t_of].astype(np.float64)
            score = k @ Q[s, j * d:(j + 1) * d] / np.sqrt(d)
            top = score.max()
            w = np.exp(score - top)
            C[s, j], A[s, j] = w @ v / w.sum(), w @ np.abs(v) / w.sum()
            LSE[j, s] = top + np.log(w.sum())
    return C.reshape(n_seq, -1), LSE, A.reshape(n_seq, -1)


def head_norm(x, gamma, eps):
    """Heads x [..., d] divided by the root of their mean square, times gamma [d] (None: as they are)."""
    return x if gamma is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gamma


def qk_norm(QKV, q_cnt, kv_cnt, d, q_gamma, k_gamma, eps, positions, inv_freq, interleaved):
    """Normed and rotated query heads [M, q_cnt, d] and key heads [M, kv_cnt, d] of QKV, and its value heads."""
    x = QKV.reshape(QKV.shape[0], q_cnt + 2 * kv_cnt, d)
    q, k = head_norm(x[:, :q_cnt], q_gamma, eps), head_norm(x[:, q_cnt:q_cnt + kv_cnt], k_gamma, eps)
    return rotate(q, positions, inv_freq, interleaved), rotate(k, positions, inv_freq, interleaved), x[:, q_cnt + kv_cnt:]


def qk_norm_bwd(QKV, q_cnt, kv_cnt, d, q_gamma, k_gamma, eps, positions, inv_freq, interleaved, dQ, dK):
    """Gradients of qk_norm: at the query and key columns of QKV [M, (q_cnt + kv_cnt) d], and of the gammas (None where there is none)."""
    M = QKV.shape[0]
    x = QKV.reshape(M, q_cnt + 2 * kv_cnt, d)
    out, dg = [], []
    for t, gamma, up in ((x[:, :q_cnt], q_gamma, dQ.reshape(M, q_cnt, d)), (x[:, q_cnt:q_cnt + kv_cnt], k_gamma, dK.reshape(M, kv_cnt, d))):
        u = rotate(up, positions, -np.asarray(inv_freq), interleaved)
        if gamma is None:
            out.append(u), dg.append(None)
            continue
        rstd = 1.0 / np.sqrt((t * t).mean(-1, keepdims=True) + eps)
        hat = t * rstd
        dg.append((u * hat).sum((0, 1)))
        w = u * gamma
        out.append((w - hat * (w * hat).mean(-1, keepdims=True)) * rstd)
    return np.concatenate(out, 1).reshape(M, -1), dg[0], dg[1]


def e4m3_code(top):
    """Byte of the smallest power of two 2^(b - 127), b >= 16, whose 448-fold is not below `top`; 127 for 0."""
    top = np.asarray(top, dtype=np.float64)
    part, e = np.frexp(np.where(top > 0, top, 1.0))
    return np.where(top > 0, np.maximum(e - 9 + (part > 0.875) + 127, 16), 127)


def to_e4m3(u):
    """Numbers of at most 448 to the nearest e4m3 number, ties to the even one: 3 bits behind the first, from 2^-6 down in steps of 2^-9."""
    step = np.ldexp(1.0, np.maximum(np.frexp(u)[1] - 1, -6) - 3)
    return np.rint(u / step) * step


def heads_to_8_bits(x):
    """e4m3 numbers and bytes of heads x [..., d]: values above the type's range of the head's largest finite one, NaN for what is not finite.  At byte 247 numbers of at most 240: 256 2^120 is no
    number of bf16."""
    fine = np.isfinite(x)
    code = e4m3_code(np.where(fine, np.abs(x), 0.0).max(-1))
    u = np.where(fine, x, 0.0) * np.ldexp(1.0, 127 - code)[..., None]
    top = np.where(code > 246, 240.0, 448.0)[..., None]
    return np.where(fine, np.clip(to_e4m3(u), -top, top), np.nan), code


def attn_chunk(Q, K, V, starts, table, lengths, max_new, max_len, q_off, kv_off, group):
    """Attention of each sequence's newest rows over its pages (K, V [pages, kv_cnt, page, d] as numbers): C [M, q_cnt d], LSE [q_cnt, M], A [M, q_cnt d] =
    sum p |V| / sum p, and which rows are written."""
    M = Q.shape[0]
    pages, _, page, d = K.shape
    q_cnt = Q.shape[1] // d
    C, A, LSE, written = np.zeros((M, q_cnt, d)), np.zeros((M, q_cnt, d)), np.full((q_cnt, M), -np.inf), np.zeros(M, dtype=bool)
    if starts is None:
        starts = list(range(M + 1))
    for s in range(len(lengths)):
        lo, hi = (min(max(int(x), 0), M) for x in starts[s:s + 2])
        n = max(hi - lo, 0)
        rows = min(n, max_new)
        written[lo:lo + rows] = True
        length = min(int(lengths[s]), max_len)
        at = np.arange(max(length, 0))
        p_of = np.asarray(table[s], dtype=np.int64)[at // page] if len(at) else at
        there = (p_of >= 0) & (p_of < pages)
        at, p_of = at[there], p_of[there]
        if rows == 0 or len(at) == 0:
            continue
        seen = at[None, :] <= (length - n + np.arange(rows))[:, None]
        for j in range(q_cnt):
            g = (q_off + j) // group - kv_off
            k, v = K[p_of, g, at % page].astype(np.float64), V[p_of, g, at % page].astype(np.float64)
            score = np.where(seen, Q[lo:lo + rows, j * d:(j + 1) * d] @ k.T / np.sqrt(d), -np.inf)
            top = score.max(1, keepdims=True)
            top = np.where(np.isneginf(top), 0.0, top)
            w = np.exp(score - top)
            total = w.sum(1)
            inv = np.where(total > 0, 1.0 / np.where(total > 0, total, 1.0), 0.0)[:, None]
            C[lo:lo + rows, j], A[lo:lo + rows, j] = w @ v * inv, w @ np.abs(v) * inv
            with np.errstate(divide="ignore"):
                LSE[j, lo:lo + rows] = top[:, 0] + np.log(total)
    return C.reshape(M, -1), LSE, A.reshape(M, -1), written
