"""One layer's serving step in fp64 -- TEST INFRASTRUCTURE (see oracle/__init__.py).

The cache of the block format as logical arrays: codes uint8 [B][cap][Hkv][dh]
and scale exponents [B][cap / block][Hkv]; an element is
decode(code) * 2^(e - 127).  Rows of new tokens are packed, sequence after
sequence: sequence b's are [start[b], start[b + 1]) and take its slots from
seq_len[b] on.
"""
import numpy as np

from .fp8 import e4m3_decode, e4m3_encode
from .refresh import rope_inv_freq

E_MIN, E_MAX, E_ONE = 10, 247, 127


def rotate_rows(shape, x, pos):
    """Rotate-half pairs (i, i + dh/2) of x [n][heads][dh] by pos * inv_freq_i."""
    x = np.asarray(x, np.float64)
    half = shape.head_dim // 2
    angle = np.asarray(pos, np.float64)[:, None] * rope_inv_freq(shape.head_dim, shape.rope_theta, shape.rope_scaling)[None]
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def block_exponent(bound):
    """The least e with bound <= 448 * 2^(e - 127) in [E_MIN, E_MAX]; 0 for bound 0."""
    if not bound > 0:
        return 0
    m, p = np.frexp(bound / 448.0)   # bound / 448 = m 2^p, m in [0.5, 1)
    return int(np.clip((p - 1 if m == 0.5 else p) + 127, E_MIN, E_MAX))


def append_blocks(codes, exps, block, seq_len, start, x, bound):
    """Writes the rows' values x [n][Hkv][dh] (bound [n][Hkv]: what a block's
    exponent has to hold of each row) into copies of codes and exps.  Returns
    (codes, exps, exact): exact [B][cap][Hkv][dh] holds, where a row was written,
    the value before rounding."""
    codes, exps = codes.copy(), exps.copy()
    exact = np.full(codes.shape, np.nan)
    for b in range(len(seq_len)):
        n = start[b + 1] - start[b]
        for g in range(codes.shape[2]):
            slot, end = seq_len[b], seq_len[b] + n
            while slot < end:
                j = slot // block
                stop = min(end, (j + 1) * block)
                rows = start[b] + np.arange(slot, stop) - seq_len[b]
                held = slice(j * block, slot)
                e_old = int(exps[b, j, g]) if slot > j * block else 0
                e = max(block_exponent(bound[rows, g].max()), e_old) or E_ONE
                if slot > j * block and e > e_old:
                    v = e4m3_decode(codes[b, held, g]) * 2.0 ** (e_old - e)
                    codes[b, held, g] = e4m3_encode(v)
                y = np.where(np.isinf(x[rows, g]), np.nan, x[rows, g])
                exact[b, slot:stop, g] = y
                codes[b, slot:stop, g] = e4m3_encode(y * 2.0 ** (127 - e))
                exps[b, j, g] = e
                slot = stop
    return codes, exps, exact


def k_bound(k):
    """Bound of each row's rotated pairs per head, as the format defines it."""
    a = np.where(np.isfinite(k), np.abs(k), 0.0)
    half = a.shape[-1] // 2
    lo, hi = np.minimum(a[..., :half], a[..., half:]), np.maximum(a[..., :half], a[..., half:])
    return (hi + lo / 2).astype(np.float32).astype(np.float64).max(-1)   # (an fp32 sum)


def v_bound(v):
    return np.where(np.isfinite(v), np.abs(v), 0.0).max(-1)


def attend_rows(q, k, v, seq_len, start, memory_only=False):
    """q [n][Hq][dh] over values k, v [B][cap][Hkv][dh].  Returns out, lse and
    spread [n][Hq][dh] = sum_j p_j |V_j| (what rounding of p is relative to)."""
    q = np.asarray(q, np.float64)
    n, hq, dh = q.shape
    g = hq // k.shape[2]
    out, spread, lse = np.zeros_like(q), np.zeros_like(q), np.full((n, hq), -np.inf)
    for b in range(len(seq_len)):
        for r in range(start[b], start[b + 1]):
            end = seq_len[b] if memory_only else seq_len[b] + r - start[b] + 1
            if end == 0:
                continue
            for h in range(hq):
                s = k[b, :end, h // g] @ q[r, h] / np.sqrt(dh)
                m = s.max()
                p = np.exp(s - m)
                out[r, h] = p @ v[b, :end, h // g] / p.sum()
                spread[r, h] = p @ np.abs(v[b, :end, h // g]) / p.sum()
                lse[r, h] = m + np.log(p.sum())
    return out, lse, spread


def token_logprobs(z, targets, top):
    """Log-probabilities of targets, entropies, top ids and their
    log-probabilities of logits z [n][vocab] without NaN or +inf."""
    z = np.asarray(z, np.float64)
    lp, ent = np.empty(len(z)), np.empty(len(z))
    ids, tlp = np.empty((len(z), top), np.int32), np.empty((len(z), top))
    for r, row in enumerate(z):
        m = row.max()
        log_p = row - m - np.log(np.exp(row - m).sum())
        p = np.exp(log_p)
        lp[r] = log_p[targets[r]]
        ent[r] = -(p[p > 0] * log_p[p > 0]).sum()
        order = np.lexsort((np.arange(len(row)), -row))[:top]
        ids[r], tlp[r] = order, log_p[order]
    return lp, ent, ids, tlp


def received(q, k, lse, seq_len, start, memory_only=False):
    """The attention that each slot of values k [B][cap][Hkv][dh] receives from the rows:
    sum over rows and heads of exp(score - lse) where a row sees the slot; lse [n][Hq],
    rows and heads where it is not finite add nothing.  Returns (sums, slack), both
    [B][cap]: slack = sum of the same terms, each times sum_i |q_i K_i| / sqrt(dh) (what
    rounding of a product's sum is relative to) + |score| + |lse|."""
    q, lse = np.asarray(q, np.float64), np.asarray(lse, np.float64)
    n, hq, dh = q.shape
    g = hq // k.shape[2]
    out, slack = np.zeros(k.shape[:2]), np.zeros(k.shape[:2])
    for b in range(len(seq_len)):
        for r in range(start[b], start[b + 1]):
            end = seq_len[b] if memory_only else seq_len[b] + r - start[b] + 1
            for h in range(hq):
                if end == 0 or not np.isfinite(lse[r, h]):
                    continue
                x = k[b, :end, h // g]
                s = x @ q[r, h] / np.sqrt(dh)
                w = np.exp(s - lse[r, h])
                out[b, :end] += w
                slack[b, :end] += w * (np.abs(x) @ np.abs(q[r, h]) / np.sqrt(dh) + np.abs(s) + abs(lse[r, h]))
    return out, slack


def compact_blocks(codes, exps, block, keep):
    """The kept slots keep[b] (ascending) of codes [B][cap][Hkv][dh] moved down, in copies
    of codes and exps: a block's exponent is the largest of its slots' old ones but 255,
    and codes are rounded to it; slots of exponent 255 become NaN codes, unless the block
    holds nothing else."""
    old_codes, old_exps = codes, exps
    codes, exps = codes.copy(), exps.copy()
    for b, idx in enumerate(keep):
        for j in range(0, len(idx), block):
            src = np.asarray(idx[j:j + block], int)
            for g in range(codes.shape[2]):
                e = old_exps[b, src // block, g].astype(int)
                numbers = e[e != 255]
                top = numbers.max() if len(numbers) else 255
                exps[b, j // block, g] = top
                for i, (s, es) in enumerate(zip(src, e)):
                    c = old_codes[b, s, g]
                    if es == 255 and top != 255:
                        c = np.full_like(c, 0x7F)
                    elif es != top:   # (a scale of 0: zeros, but for codes that are no numbers)
                        c = e4m3_encode(e4m3_decode(c) * (2.0 ** (es - top) if es else 0.0))
                    codes[b, j + i, g] = c
    return codes, exps


def join_parts(parts, lses):
    """Attention over disjoint slots joined: parts [P][n][Hq][dh], lses [P][n][Hq]."""
    parts, lses = np.asarray(parts, np.float64), np.asarray(lses, np.float64)
    out, lse = np.zeros(parts.shape[1:]), np.full(lses.shape[1:], -np.inf)
    for r in range(lses.shape[1]):
        for h in range(lses.shape[2]):
            s = lses[:, r, h]
            if (np.isnan(s) | (s == np.inf)).any():
                lse[r, h] = np.nan
                continue
            live = [i for i in range(len(s)) if s[i] > -np.inf]
            if live:
                m = s[live].max()
                w = np.exp(s[live] - m)
                out[r, h] = sum(wi * parts[i, r, h] for wi, i in zip(w, live)) / w.sum()
                lse[r, h] = m + np.log(w.sum())
    return out, lse
