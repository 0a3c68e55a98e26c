"""fp64 oracle of the paged cache (include/qp_paged.h), written from the definitions, sequence by sequence.

A pool is a dict of numpy arrays k, v [pages][H_kv][P][d], pos, weight [pages][H_kv][P]; a batch is table [S][pages], lens [S],
row_start [S + 1]. A pool with scales has codes in k and v and k_scale, v_scale [pages][H_kv][P / 16]. Nothing here shares code with the kernels.
"""
import numpy as np

from oracle.qp_oracle import fp8_e4m3_round


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


def dequantised(pool):
    """A pool with scales as one of the values that its codes stand for."""
    wide = lambda x: np.repeat(x, 16, axis=2)[..., None]
    return dict(pool, k=pool["k"] * wide(pool["k_scale"]), v=pool["v"] * wide(pool["v_scale"]))


def attend(q, pool, batch, scale, window=None, n_sink=0):
    """A row that is entry p sees j <= p, with a window those with j > p - window or j < n_sink. out [rows][H_q][d] and lse [H_q][rows] (NaN where a row belongs to nobody), and per output the softmax mean of |v| and per row the largest |logit| and
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
                if window is not None:
                    see &= (j > base + i - window) | (j < n_sink)
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


def turn(x, axes, theta, section):
    """x [rows][heads][d], pairs (i, i + d / 2) turned by axes[axis(i)][row] * theta^(-2 i / d)."""
    half = x.shape[-1] // 2
    axis = np.repeat(np.arange(3), section)
    angle = np.asarray(axes, np.float64)[axis].T * np.float64(theta) ** (-np.arange(half) / half)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def block_exponent(x, largest):
    """The least e from -117 to 120 with |x| <= largest * 2^e for the finite ones of x."""
    most = max([0.0] + [abs(float(v)) for v in np.ravel(x) if np.isfinite(v)])
    e = -117
    while e < 120 and most > largest * 2.0 ** e:
        e += 1
    return e


def codes_that_fit(x, e):
    """Scaled values as far as codes can hold them: at a scale of 2^120 those beyond 240 would stand for more than f32 holds."""
    return np.clip(x, -240.0, 240.0) if e == 120 else x


def append_scaled(k, v, k_size, pos, pool, batch, k_largest, store=fp8_e4m3_round):
    """The pool with scales after the new rows: entry by entry, which gives a block the same scale as all at once, and its earlier entries'
    codes as if the block's scale had been known (one rescaling of what was there before the call). k_size: rows whose magnitudes the keys' scales
    hold, up to k_largest; store: codes of scaled values."""
    pool = {name: x.copy() for name, x in pool.items()}
    n_pages, h_kv, p, _ = pool["k"].shape
    for s, length, begin, n in _sequences(batch, len(k)):
        length = max(0, min(length, len(batch["table"][s]) * p))
        first = length - n
        for block in range(max(first, 0) // 16, -(-length // 16)):
            page, at = batch["table"][s][block * 16 // p], block * 16 % p
            if not 0 <= page < n_pages or n == 0:
                continue
            new = [j for j in range(block * 16, min(length, block * 16 + 16)) if j >= first]
            old = [j for j in range(block * 16, min(first, block * 16 + 16))]
            rows = [begin + j - first for j in new]
            for h in range(h_kv):
                for x, size, name, largest in ((k, k_size, "k", k_largest), (v, v, "v", 448.0)):
                    e = block_exponent(size[rows, h], largest)
                    scale = pool[name + "_scale"]
                    if old:
                        was = int(np.log2(scale[page, h, at // 16]))
                        e = max(e, was)
                        slots = [j % p for j in old]
                        pool[name][page, h, slots] = fp8_e4m3_round(pool[name][page, h, slots] * 2.0 ** (was - e))
                    scale[page, h, at // 16] = 2.0 ** e
                    pool[name][page, h, [j % p for j in new]] = store(codes_that_fit(x[rows, h] * 2.0 ** -e, e))
            for j, row in zip(new, rows):
                pool["pos"][page, :, j % p], pool["weight"][page, :, j % p] = pos[row], 0
    return pool


def move_scaled(pool, table, kept, to_table):
    """The pool with scales after the entries kept[s][h] of every sequence and head were moved to the pages of to_table: a block of them gets the
    largest of their scales."""
    pool = {name: x.copy() for name, x in pool.items()}
    p = pool["k"].shape[2]
    for s, heads in enumerate(kept):
        for h, entries in enumerate(heads):
            for block in range(-(-len(entries) // 16)):
                old = entries[16 * block:16 * block + 16]
                page, slot = np.asarray(table[s])[old // p], old % p
                to, at = to_table[s][16 * block // p], 16 * block % p
                for name in ("k", "v"):
                    scales = pool[name + "_scale"][page, h, slot // 16]
                    pool[name + "_scale"][to, h, at // 16] = scales.max()
                    pool[name][to, h, at:at + len(old)] = fp8_e4m3_round(pool[name][page, h, slot] * (scales / scales.max())[:, None])
                for name in ("pos", "weight"):
                    pool[name][to, h, at:at + len(old)] = pool[name][page, h, slot]
    return pool
