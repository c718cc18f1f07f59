"""References of the paged operators in 64 bits (NumPy), and the inputs of their tests."""
import numpy as np
import torch

MAX = {torch.float16: 65504.0, torch.float8_e4m3fn: 448.0}
#: Half of a type's smallest step (its subnormal numbers), where relative rounding ends.
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float8_e4m3fn: 2.0 ** -10, torch.float32: 2.0 ** -150}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------ page map
def page_map(lens, rows, table, ring, queue, page, max_rows):
    """The step, sequence by sequence.  Returns (table, ring, lens, queue, row_start, row_seq, row_pos, slots) or None if it is refused."""
    table, ring, (head, count) = table.copy(), ring.copy(), [int(x) for x in queue]
    out_len, start, seq, pos, slots = [], [0], [], [], []
    give = []
    taken = 0
    for i, (n, r) in enumerate(zip(map(int, lens), map(int, rows))):
        had = -(-n // page)
        if r == -1:
            give += list(table[i, :had])
            out_len.append(0)
            start.append(start[-1])
            continue
        has = -(-(n + r) // page)
        if has > table.shape[1]:
            return None
        for b in range(had, has):
            if taken >= count:
                return None
            table[i, b] = ring[(head + taken) % len(ring)]
            taken += 1
        for p in range(n, n + r):
            seq.append(i)
            pos.append(p)
            slots.append(int(table[i, p // page]) * page + p % page)
        out_len.append(n + r)
        start.append(start[-1] + r)
    if len(seq) > max_rows or len(give) > len(ring) - count:
        return None
    for t, p in enumerate(give):
        ring[(head + count + t) % len(ring)] = p
    pad = [-1] * (max_rows - len(seq))
    return (table, ring, np.array(out_len), np.array([(head + taken) % len(ring), count - taken + len(give)]), np.array(start),
            np.array(seq + pad), np.array(pos + pad), np.array(slots + pad))


# ------------------------------------------------------------------ attention
def attend(q, k_pages, v_pages, table, lens, row_start, scale, p_eps, k_scale=None, v_scale=None):
    """(out, lse, tolerance of out, of lse) of every row, None for rows of no sequence.  q [n, Hq, hd] and pages [pages, Hkv, page, hd] in
    float64.  The tolerance, without the output's own rounding: with A = sum p |v|, a softmax weight is off by p_eps (its rounding)
    and 2 d, d the error of a score: fp32 sums of hd products (and 2^-20 for exp2 and the logarithm); the sums over n positions by n fp32 roundings."""
    n, Hq, hd = q.shape
    pages, Hkv, P, _ = k_pages.shape
    g = Hq // Hkv
    out, lse, tol, ltol = [None] * n, [None] * n, [None] * n, [None] * n
    for i, length in enumerate(lens):
        rows = range(row_start[i], row_start[i + 1])
        length = min(int(length), table.shape[1] * P)
        R = len(rows)
        for j, r in enumerate(rows):
            m = min(length, int(lens[i]) - R + 1 + j)
            where = [(int(table[i, p // P]), p % P) for p in range(max(m, 0)) if 0 <= table[i, p // P] < pages]
            o, le, to, lt = np.zeros((Hq, hd)), np.full(Hq, -np.inf), np.zeros((Hq, hd)), np.zeros(Hq)
            if where:
                pg, off = np.array(where).T
                for hk in range(Hkv):
                    k, v = k_pages[pg, hk, off], v_pages[pg, hk, off]
                    if k_scale is not None:
                        k, v = k * k_scale[hk], v * v_scale[hk]
                    qs = q[r, hk * g:(hk + 1) * g]
                    s = scale * qs @ k.T
                    top = s.max(1, keepdims=True)
                    w = np.exp(s - top)
                    total = w.sum(1, keepdims=True)
                    h = slice(hk * g, (hk + 1) * g)
                    o[h] = w @ v / total
                    le[h] = (top + np.log(total))[:, 0]
                    d = scale * (np.abs(qs) @ np.abs(k).T).max() * (hd + 8) * 2.0 ** -24 + 2.0 ** -20
                    to[h] = (w @ np.abs(v) / total) * (p_eps + 2 * d + (len(where) + 64) * 2.0 ** -24)
                    lt[h] = d + (len(where) + 64) * 2.0 ** -24 + 2.0 ** -22 * np.abs(le[h])
            out[r], lse[r], tol[r], ltol[r] = o, le, to, lt
    return out, lse, tol, ltol


# ------------------------------------------------------------------ sampling
def sample(z, lo, hi, temperature, top_k, top_p, min_p, u):
    """(token, log probability) of one row, from the definition in 64 bits."""
    z = np.asarray(z, np.float64)
    ids = np.array([i for i in range(max(lo, 0), min(hi, len(z))) if not np.isnan(z[i]) and z[i] != -np.inf], np.int64)
    if len(ids) == 0:
        return -1, -np.inf
    order = ids[np.argsort(-z[ids], kind="stable")]
    top = z[order[0]]
    T = float(temperature)
    greedy = not T > 0
    with np.errstate(invalid="ignore"):
        d = np.where(z[order] == top, 0.0, (z[order] - top) / (1.0 if greedy else T))
    w = np.exp(d)
    total = w.sum()
    if greedy:
        return int(order[0]), float(d[0] - np.log(total))
    n = len(order) if top_k <= 0 else min(top_k, len(order))
    mass = np.cumsum(w)
    if top_p < 1:
        n = min(n, int(np.searchsorted(mass[:n], top_p * mass[n - 1])) + 1)
    if min_p > 0:
        n = min(n, max(1, int((w >= min_p).sum())))
    n = max(1, min(n, int((w > 0).sum())))
    j = min(int(np.searchsorted(mass[:n], u * mass[n - 1], side="right")), n - 1)
    return int(order[j]), float(d[j] - np.log(total))
