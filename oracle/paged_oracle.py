"""fp64 oracle of the paged cache (include/qp_paged.h), written from the definitions, sequence by sequence.

A pool is a dict of numpy arrays k, v [pages][H_kv][P][d], pos, weight [pages][H_kv][P]; a batch is table [S][pages], lens [S],
row_start [S + 1]. Nothing here shares code with the kernels.
"""
import numpy as np


def places(table, length, page_tokens, n_pages):
    """Entry numbers of a sequence that are there, with their pages and slots."""
    j = np.arange(max(0, min(length, len(table) * page_tokens)))
    page = np.asarray(table)[j // page_tokens]
    here = (page >= 0) & (page < n_pages)
    return j[here], page[here], (j % page_tokens)[here]


def _sequences(batch, n_rows):
    for s, length in enumerate(batch["lens"]):
        begin = min(max(batch["row_start"][s], 0), n_rows)
        end = min(max(batch["row_start"][s + 1], begin), n_rows)
        yield s, length, begin, end - begin


def attend(q, pool, batch, scale):
    """out [rows][H_q][d] and lse [H_q][rows] (NaN where a row belongs to nobody), and per output the softmax mean of |v| and per row the largest |logit| and
    the largest sum |q||k|, which error bounds need."""
    n_rows, h_q, d = q.shape
    n_pages, h_kv, p, _ = pool["k"].shape
    r = h_q // h_kv
    out, absv = np.full((n_rows, h_q, d), np.nan), np.zeros((n_rows, h_q, d))
    lse, size = np.full((h_q, n_rows), np.nan), np.zeros((h_q, n_rows))
    for s, length, begin, n in _sequences(batch, n_rows):
        j, page, slot = places(batch["table"][s], length, p, n_pages)
        base = min(length, len(batch["table"][s]) * p) - n
        for qh in range(h_q):
            k, v = pool["k"][page, qh // r, slot], pool["v"][page, qh // r, slot]
            for i in range(n):
                see = j <= base + i
                row = begin + i
                if not see.any():
                    out[row, qh], lse[qh, row] = 0, -np.inf
                    continue
                x = scale * (k[see] @ q[row, qh])
                m = x.max()
                w = np.exp(x - m)
                w /= w.sum()
                out[row, qh] = w @ v[see]
                absv[row, qh] = w @ np.abs(v[see])
                lse[qh, row] = m + np.log(np.exp(x - m).sum())
                size[qh, row] = scale * (np.abs(k[see]) @ np.abs(q[row, qh])).max() + np.abs(x).max()
    return out, lse, absv, size


def weigh(q, lse, pool, batch, scale, accumulate):
    """The pool's weights after the call, and what was added (for error bounds)."""
    n_rows, h_q, d = q.shape
    n_pages, h_kv, p, _ = pool["k"].shape
    r = h_q // h_kv
    weight, added = pool["weight"].copy(), np.zeros_like(pool["weight"])
    for s, length, begin, n in _sequences(batch, n_rows):
        j, page, slot = places(batch["table"][s], length, p, n_pages)
        base = min(length, len(batch["table"][s]) * p) - n
        for h in range(h_kv):
            k = pool["k"][page, h, slot]
            got = np.zeros(len(j))
            for i in range(n):
                see = j <= base + i
                for qh in range(h * r, (h + 1) * r):
                    z = lse[qh, begin + i]
                    if z != -np.inf:
                        got[see] += np.exp(scale * (k[see] @ q[begin + i, qh]) - z)
            added[page, h, slot] = got
            weight[page, h, slot] = got + (weight[page, h, slot] if accumulate else 0)
    return weight, added


def append(k, v, pos, pool, batch):
    """The pool after the new rows were stored: k, v [rows][H_kv][d] as the pool holds them, pos [rows][H_kv]."""
    pool = {name: x.copy() for name, x in pool.items()}
    n_pages, h_kv, p, _ = pool["k"].shape
    for s, length, begin, n in _sequences(batch, len(k)):
        length = max(0, min(length, len(batch["table"][s]) * p))
        for i in range(n):
            j = length - n + i
            if j < 0:
                continue
            page = batch["table"][s][j // p]
            if 0 <= page < n_pages:
                pool["k"][page, :, j % p], pool["v"][page, :, j % p] = k[begin + i], v[begin + i]
                pool["pos"][page, :, j % p], pool["weight"][page, :, j % p] = pos[begin + i], 0
    return pool


def evict(pool, table, lens, keep, n_first, n_last):
    """Old entry numbers kept per (sequence, head), ascending."""
    n_pages, h_kv, p, _ = pool["k"].shape
    kept = []
    for s, length in enumerate(lens):
        j, page, slot = places(table[s], length, p, n_pages)
        length = max(0, min(length, len(table[s]) * p))
        for h in range(h_kv):
            w = pool["weight"][page, h, slot].astype(np.float64) + 0.0
            stays = (j < n_first) | (j >= length - n_last)
            # largest first, what stays before all others, equal ones in ascending order
            order = sorted(range(len(j)), key=lambda x: (not stays[x], -w[x], j[x]))
            kept.append(np.sort(j[order[:keep]]))
    return kept
