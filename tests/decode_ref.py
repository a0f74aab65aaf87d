"""Plain 64-bit forms of the decoding operators, a cache maker, and the bounds that the GPU tests hold results to.

Bounds, counted in roundings (u = 2^-24, half a step of fp32; 2^-8 half a step of bf16):
  score     a sum of 128 products and a scaling: off by at most 132 u S, S = scale * sum |q| |k|; the running maximum and the
            exponent add 4 roundings of a number no larger than S + 16
  exp, sum  a term is off by twice that (exponent and normaliser) and a few u; a sum of n terms by n u more
  out       probabilities are two bf16 parts: the first is off by at most 2^-8 p, the second rounds that rest, 2^-8 of it, so 2^-16 p
            are left; with more than 64 query rows per KV head they are the first part alone, 2^-8 p off.  out is a sum of p v, so off
            by that share of sum p |v|, and rounded to bf16 once, 2^-8 |out|
"""
import numpy as np

U = 2.0 ** -24


def bf16(rng, *size, scale=1.0):
    from workloads import f32_to_bf16_bits
    return f32_to_bf16_bits((scale * rng.standard_normal(size)).astype(np.float32))


def f64(bits):
    from workloads import bf16_bits_to_f64
    return bf16_bits_to_f64(bits)


def dev_i32(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def dev_f32(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()


def to_pages(rng, dense, caps, page, spare=2, fill=0x7FC0):
    """dense [nl, T, h, d] bits -> (pool [nl, pages, page, h, d] bits, table [n_seq, most]); unowned rows are NaN, unused entries -1."""
    nl, _, h, d = dense.shape
    per = [-(-c // page) for c in caps]
    n = sum(per) + spare
    order = rng.permutation(n)
    table = np.full((len(caps), max(per) + 1), -1, np.int32)
    pool = np.full((nl, n, page, h, d), fill, np.uint16)
    at = used = 0
    for s, c in enumerate(caps):
        for p in range(per[s]):
            table[s, p] = order[used]
            m = min(page, c - p * page)
            pool[:, order[used], :m] = dense[:, at + p * page:at + p * page + m]
            used += 1
        at += c
    return pool, table


def from_pages(pool, table, caps, page):
    out = []
    for s, c in enumerate(caps):
        j = np.arange(c)
        out.append(pool[:, table[s, j // page], j % page])
    return np.concatenate(out, axis=1)


def attend_ref(q, k, v, see, scale):
    """One (layer, sequence, KV head): q [rows, d], k, v [n, d] float64, see [rows, n] bool.  (out, lse, weights of the rows, bounds)"""
    rows, n = see.shape
    out, lse = np.zeros((rows, v.shape[1])), np.full(rows, -np.inf)
    w, tol_out, tol_lse, tol_w = np.zeros(n), np.zeros_like(out), np.zeros(rows), np.zeros(n)
    for r in range(rows):
        idx = np.nonzero(see[r])[0]
        if not idx.size:
            continue
        x = scale * (k[idx] @ q[r])
        S = (scale * (np.abs(k[idx]) @ np.abs(q[r]))).max()
        m = x.max()
        e = np.exp(x - m)
        lse[r] = m + np.log(e.sum())
        p = e / e.sum()
        out[r] = p @ v[idx]
        w[idx] += p
        score = 132 * U * S + 4 * U * (S + 16)
        term = 2 * score + (idx.size + 400) * U
        part = 2.0 ** -16 if rows <= 64 else 2.0 ** -8
        tol_out[r] = 2.0 ** -8 * np.abs(out[r]) + (part + term) * (p @ np.abs(v[idx])) + 1e-38
        tol_lse[r] = score + (idx.size + 400) * U + 4 * U * abs(lse[r])
        tol_w[idx] += term * p + 1e-37  # (exp flushes what is below 2^-126)
    return out, lse, w, tol_out, tol_lse, tol_w


def visible(mode, n, n_q, group, seen=None):
    """[n_q * group rows, n] bool: rows are (token, head of the group)."""
    see = np.ones((n_q, n), bool)
    j = np.arange(n)
    for i in range(n_q):
        if mode == "causal":
            see[i] = j < n - n_q + i + 1
        elif mode == "tree":
            t = j - (n - n_q)
            bits = np.array([(int(seen[i, x // 32]) >> (x % 32)) & 1 for x in range(n_q)], bool)
            see[i] = (t < 0) | bits[np.clip(t, 0, n_q - 1)]
    return np.repeat(see, group, axis=0)


def random_tree(rng, n_q):
    """seen [n_q, words] uint32 of a random tree: each node its ancestors and itself."""
    words = -(-n_q // 32)
    seen = np.zeros((n_q, words), np.uint32)
    for i in range(n_q):
        parent = int(rng.integers(max(-1, i - 5), i)) if i else -1
        if parent >= 0:
            seen[i] = seen[parent]
        seen[i, i // 32] |= np.uint32(1 << (i % 32))
    return seen


def evict_order(w, pos, n, B, first, last):
    """Kept rows, ascending: the B heaviest of the first n, lower rows first among equals, protected positions before all."""
    newest = int(pos[:n].max()) if n else 0
    rows = sorted(range(n), key=lambda j: (not (pos[j] < first or pos[j] > newest - last), -float(w[j]), j))
    return np.array(sorted(rows[:B]), dtype=np.int64)


def lightest(w, pos, n, token, first, last):
    rows = sorted(range(n), key=lambda j: (pos[j] < first or pos[j] > token - last, float(w[j]), j))
    return rows[0]
