"""Plain 64-bit definitions of the operators on a filled pool (attention, eviction).

Shares no code with the library: a pool is a numpy array of its logical shape, a token is
looked up through its block table one at a time.
"""
from __future__ import annotations

import numpy as np

BLOCK_MAJOR = 0


def token_rows(pool, layout, block, layer, kv, head, tbl, n):
    """[n, dim] rows of one head, tokens 0..n-1 of the sequence with block ids ``tbl``."""
    out = np.zeros((n, pool.shape[-1]))
    for t in range(n):
        b, tt = int(tbl[t // block]), t % block
        out[t] = pool[b, layer, kv, tt, head] if layout == BLOCK_MAJOR else pool[layer, kv, b, head, tt]
    return out


def attend(pool, layout, block, layer, seqs, lens, q, num_kv_heads, scale):
    """Returns out, lse, weights (per sequence: [KV head, row, own token]) and the error scale of
    each row: sum of weight * |v| per dim, largest |scale| * sum |q||k| and largest |logit| over visible tokens with a finite logit.
    ``pool``: float64 array of the logical shape; ``q``: [n, Q, Hq, D] float64."""
    n, Q, Hq, D = q.shape
    G = Hq // num_kv_heads
    out, lse = np.zeros(q.shape), np.full((n, Q, Hq), -np.inf)
    mag = np.zeros(q.shape)
    dot_mag, z_mag, seen_n, v_mag = (np.zeros((n, Q, Hq)) for _ in range(4))
    weights = []
    for r in range(n):
        own = int(lens[r])
        weights.append(np.zeros((num_kv_heads, Q * G, own)))
        tbl = seqs.tbl[seqs.tbl_off[r]:seqs.tbl_off[r + 1]]
        p = int(seqs.seq_prefix[r]) if seqs.seq_prefix is not None and seqs.prefix_len is not None else -1
        for h in range(num_kv_heads):
            k = token_rows(pool, layout, block, layer, 0, h, tbl, own)
            v = token_rows(pool, layout, block, layer, 1, h, tbl, own)
            first = 0
            if p >= 0:
                first = int(seqs.prefix_len[p])
                ptbl = seqs.prefix_tbl[seqs.prefix_tbl_off[p]:seqs.prefix_tbl_off[p + 1]]
                k = np.concatenate([token_rows(pool, layout, block, layer, 0, h, ptbl, first), k])
                v = np.concatenate([token_rows(pool, layout, block, layer, 1, h, ptbl, first), v])
            for i in range(Q):
                sees = first + max(0, own - (Q - 1 - i))
                if sees == 0:
                    continue
                for g in range(G):
                    x = q[r, i, h * G + g]
                    z = scale * (k[:sees] @ x)
                    top = z.max()
                    if top == -np.inf:
                        continue
                    w = np.exp(z - top)
                    total = w.sum()
                    w /= total
                    out[r, i, h * G + g] = w @ v[:sees]
                    lse[r, i, h * G + g] = top + np.log(total)
                    mag[r, i, h * G + g] = w @ np.abs(v[:sees])
                    fin = np.isfinite(z)
                    dot_mag[r, i, h * G + g] = abs(scale) * (np.abs(k[:sees][fin]) @ np.abs(x)).max()
                    z_mag[r, i, h * G + g] = np.abs(z[fin]).max()
                    v_mag[r, i, h * G + g] = np.abs(v[:sees]).max()
                    seen_n[r, i, h * G + g] = sees
                    weights[r][h, i * G + g, :max(0, sees - first)] = w[first:]
    return out, lse, weights, dict(mag=mag, dot=dot_mag, z=z_mag, n=seen_n, v=v_mag)


def select(scores, budget, sink, recent):
    """Indices kept of one row of scores, ascending."""
    n = len(scores)
    if n <= budget:
        return np.arange(n)
    middle = [(-np.inf if np.isnan(s) else float(s), not np.isnan(s), -t) for t, s in enumerate(scores)]
    order = sorted(range(sink, n - recent), key=lambda t: (middle[t][1], middle[t][0], middle[t][2]), reverse=True)
    keep = order[:budget - sink - recent]
    return np.array(sorted(list(range(sink)) + keep + list(range(n - recent, n))), np.int64)


def move(src, src_layout, src_block, src_tbl, dst, dst_layout, dst_block, dst_tbl, layer, head, kept):
    """Copies the kept tokens' K and V rows to slots 0.. (``src`` must not be ``dst``)."""
    for j, t in enumerate(kept):
        a, b = int(src_tbl[t // src_block]), int(dst_tbl[j // dst_block])
        for kv in (0, 1):
            row = src[a, layer, kv, t % src_block, head] if src_layout == BLOCK_MAJOR else src[layer, kv, a, head, t % src_block]
            if dst_layout == BLOCK_MAJOR:
                dst[b, layer, kv, j % dst_block, head] = row
            else:
                dst[layer, kv, b, head, j % dst_block] = row
