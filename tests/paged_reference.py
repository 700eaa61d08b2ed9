"""Plain 64-bit forms of the paged-cache operators for the tests: loops over sequences and tokens, numpy only."""
import numpy as np


def pages_of(tokens, page):
    return -(-tokens // page)


def append(len_new, kv_len, page, table, free, n_free, total):
    """Returns kv_len, table, n_free, cu_q, pos, slot_map after the call."""
    table, stack = table.copy(), list(free[:n_free])
    pos, slot = [], []
    for s, (kv, add) in enumerate(zip(kv_len, len_new)):
        for j in range(pages_of(kv, page), pages_of(kv + add, page)):
            table[s, j] = stack.pop()
        for t in range(kv, kv + add):
            pos.append(t)
            slot.append(table[s, t // page] * page + t % page)
    pad = total - len(pos)
    cu = np.concatenate([[0], np.cumsum(len_new)]).astype(np.int64)
    return kv_len + len_new, table, len(stack), cu, np.array(pos + [0] * pad), np.array(slot + [-1] * pad)


def release(keep, kv_len, page, shared, table, free, n_free):
    """Returns kv_len, table, free, n_free after the call."""
    free = free.copy()
    rows, lens = np.full_like(table, -1), np.zeros_like(kv_len)
    for s in range(len(kv_len)):
        if s not in set(keep):
            for j in range(shared, pages_of(kv_len[s], page)):
                free[n_free] = table[s, j]
                n_free += 1
    for i, s in enumerate(keep):
        have = pages_of(kv_len[s], page)
        rows[i, :have] = table[s, :have]
        lens[i] = kv_len[s]
    return lens, rows, free, n_free


def norm_rope(x, pos, gain, eps, theta):
    """x [rows, heads, dh] fp64; gain None: no norm.  Returns the rotated heads and |a| + |b| of every pair (what a rounding
    inside the rotation is relative to), both [rows, heads, dh]."""
    dh = x.shape[-1]
    if gain is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * gain
    ang = np.asarray(pos, np.float64)[:, None] * theta ** (-2.0 * np.arange(dh // 2) / dh)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :dh // 2], x[..., dh // 2:]
    size = np.abs(a) + np.abs(b)
    return np.concatenate([a * c - b * s, b * c + a * s], -1), np.concatenate([size, size], -1)


def attention(q, k, v, table, cu, kv_len, causal):
    """q [rows, hq, dh], caches [pages, hkv, page, dh], all fp64.  Returns the output, the same average of |v|, and for every
    (row, head) the largest sum_d |q_d k_d| / sqrt(dh) over its visible keys (what the rounding of a score is relative to)."""
    rows, hq, dh = q.shape
    hkv, page = k.shape[1], k.shape[2]
    g = hq // hkv
    out, avg, size = np.zeros_like(q), np.zeros_like(q), np.zeros((rows, hq))
    for s in range(len(kv_len)):
        n = int(kv_len[s])
        ids = table[s, :pages_of(n, page)]
        ks = k[ids].transpose(1, 0, 2, 3).reshape(hkv, -1, dh)[:, :n]
        vs = v[ids].transpose(1, 0, 2, 3).reshape(hkv, -1, dh)[:, :n]
        lq = int(cu[s + 1] - cu[s])
        for i in range(lq):
            r = int(cu[s]) + i
            seen = min(n, n - lq + i + 1) if causal else n
            if seen <= 0:
                continue
            qr = q[r].reshape(hkv, g, dh)
            sc = np.einsum("hgd,hkd->hgk", qr, ks[:, :seen]) / np.sqrt(dh)
            p = np.exp(sc - sc.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[r] = np.einsum("hgk,hkd->hgd", p, vs[:, :seen]).reshape(hq, dh)
            avg[r] = np.einsum("hgk,hkd->hgd", p, np.abs(vs[:, :seen])).reshape(hq, dh)
            size[r] = (np.einsum("hgd,hkd->hgk", np.abs(qr), np.abs(ks[:, :seen])).max(-1) / np.sqrt(dh)).reshape(hq)
    return out, avg, size


def attention_tolerance(out, avg, size, dh, n_keys, bf16):
    """Bound on |computed - out|, element by element.

    A score is a sum of dh products held in fp32 (tensor cores may truncate: one whole step, 2^-23, an addition), scaled
    and put through exp2: the exponent is off by at most e = (dh + 4) 2^-23 size (in units of the natural exponent, |score| <=
    size), the exponential itself by 2^-21 relative (special-function unit, its argument rounded once more: 2^-23 size).
    Weights with relative errors up to d move a weighted average by at most 2 d avg.  Summing n products and n weights in
    fp32 adds 2 n 2^-23 avg; joining pieces or the parts of a block 2^-20 avg.  In bf16 the weights of the numerator are
    rounded (2^-8 each, hence 2^-8 avg), and the result is rounded once: 2^-8 |out| (fp32: 2^-24 |out|)."""
    d = ((dh + 5) * 2.0 ** -23 * size + 2.0 ** -21)[..., None]
    tol = avg * (2 * d + 2 * n_keys * 2.0 ** -23 + 2.0 ** -20)
    if bf16:
        tol = tol + 2.0 ** -8 * avg
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    return tol + half * (np.abs(out) + tol) + 1e-30
