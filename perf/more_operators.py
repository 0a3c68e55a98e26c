"""Performance cases of the paged cache's operators for rotated keys, 8-bit pools with scales and sliding windows:

  store    new tokens' keys turned by their rotary angles (three position axes) on their way into the sequences' pages, with
           their values; the queries of the same rows turned in the same call. Pools of the layout's type, of plain 8-bit
           codes, and of 8-bit codes with a power of two for every block of 16 entries and head
  scaled   attention of each sequence's new tokens over an 8-bit pool with such scales
  window   attention in which a token sees the last `window` entries up to itself and the sequence's first `sinks` ones

With `own` the calls are the library's; without, the same results from elementary torch operations in 32 bits (angles in
64). `exact()` has them in 64 bits, sequence by sequence, from the definitions. An 8-bit pool is returned as its codes'
values and the scales that they stand for multiples of.
"""
import math
import random

import torch

own = False

# (query heads, KV heads, head_dim, dtype, frequencies per position axis): a tiny f32 layout for the smallest calls, and those of
# the 7B and 72B models
LAYOUTS = {"tiny": (4, 2, 64, "f32", (8, 12, 12)), "7b": (28, 4, 128, "bf16", (16, 24, 24)), "72b": (64, 8, 128, "bf16", (16, 24, 24))}
THETA = 1e6
MAX_PAIRS = 9e8            # (row, entry) pairs over all query heads of a batch: no more than the largest listed chunk has
MAX_ENTRIES = 1.2e6        # entries times KV heads of a batch
BLOCK = 16                 # entries that share a scale
E_MIN, E_MAX = -117, 120   # its exponents


def _case(name, op, layout, seqs, new, entries, ragged, page, fmt="same", **more):
    return dict(name=name, op=op, layout=layout, seqs=seqs, new=new, entries=entries, ragged=ragged, page=page, fmt=fmt, **more)


def listed():
    return [
        # the smallest call: one token of one answer in f32; launches and waits are what it costs
        _case("store_reply_f32", "store", "tiny", 1, 1, 333, 1.0, 16, queries=True),
        # a decoding step of 32 answers behind a plain projection: queries and keys turned, keys and values stored
        _case("store_replies_7b", "store", "7b", 32, 1, 2000, 0.1, 64, queries=True),
        # up to four drafted tokens of 16 answers into blocks that are partly full: their scales may grow
        _case("store_drafts_72b_scaled", "store", "72b", 16, 4, 1500, 0.3, 32, "scaled", queries=True),
        # a group of a video (64 frames of 121 tokens), three position axes
        _case("store_group_7b", "store", "7b", 1, 7744, 20000, 1.0, 64, queries=True),
        # what an hour-long video left, kept with unturned keys, into an 8-bit pool with scales
        _case("store_video_72b_scaled", "store", "72b", 1, 46125, 46125, 1.0, 64, "scaled", queries=False),
        # one answer's token over the hour-long video's cache: few rows, a long axis
        _case("scaled_reply_7b", "scaled", "7b", 1, 1, 46125, 1.0, 64, "scaled", holes=False),
        # the large model's caches, up to four drafted tokens per answer; freed pages in the middle
        _case("scaled_drafts_72b", "scaled", "72b", 16, 4, 32768, 0.3, 32, "scaled", holes=True),
        # four questions of up to 300 tokens over hour-long caches: the matrix products count
        _case("scaled_questions_7b", "scaled", "7b", 4, 300, 46125, 0.3, 128, "scaled", holes=False),
        # one token of one answer in f32 that sees its last 256 entries and the first 4
        _case("window_reply_f32", "window", "tiny", 1, 1, 5000, 1.0, 16, window=256, sinks=4, freed=False),
        # a decoding step of 32 answers that see 4096 entries of caches many times as long, whose pages behind were given back
        _case("window_replies_7b", "window", "7b", 32, 1, 46125, 0.1, 64, window=4096, sinks=64, freed=True),
        # drafted tokens of the large model over an 8-bit pool with scales, a window that no page ends with
        _case("window_drafts_72b_scaled", "window", "72b", 16, 4, 16000, 0.3, 32, "scaled", window=2000, sinks=16, freed=False),
        # four questions of up to 300 tokens, each token with a window of its own
        _case("window_questions_7b", "window", "7b", 4, 300, 46125, 0.3, 128, window=8192, sinks=100, freed=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "scaled", "window"])
    layout = rng.choice(["7b", "72b"]) if op == "scaled" else rng.choice(["tiny", "7b", "7b", "72b"])
    h_q, h_kv, d, dtype, _ = LAYOUTS[layout]
    most = 5000 if dtype == "f32" else 46125
    fmt = "scaled" if op == "scaled" else "same" if dtype == "f32" else rng.choice(["same", "same", "fp8", "scaled"])
    page = rng.choice([16, 32, 64, 128, 256])
    entries = _log(rng, 1, most)
    seqs = min(_log(rng, 1, 64), max(1, int(MAX_ENTRIES / (h_kv * entries))))
    new = _log(rng, 1, 8) if rng.random() < 0.6 else _log(rng, 8, 600 if dtype == "bf16" else 64)
    new = max(1, min(new, entries, int(MAX_PAIRS / (seqs * h_q * entries))))
    ragged = rng.choice([0.05, 0.3, 0.7, 1.0])
    if op == "store":
        queries = rng.random() < 0.6
        if rng.random() < 0.4:                            # a whole group, or what a video left
            new = min(entries, 8000) if queries else entries
            seqs = max(1, min(seqs, 2, int(6e5 / (h_kv * new))))
        return _draw(op, layout, seqs, new, entries, ragged, page, fmt, queries=queries)
    if op == "scaled":
        return _draw(op, layout, seqs, new, entries, ragged, page, fmt, holes=rng.random() < 0.25)
    return _draw(op, layout, seqs, new, entries, ragged, page, fmt, window=_log(rng, 1, 10000), sinks=rng.choice([0, 1, 4, 16, 64, 100]),
                 freed=rng.random() < 0.4)


def _draw(*a, **more):
    c = _case("", *a, **more)
    del c["name"]
    return c


def _lengths(case):
    """Entries and new rows of each sequence: the first has the most, the others spread down to `ragged` of it."""
    spread = [1.0 if i == 0 else case["ragged"] + (1 - case["ragged"]) * ((i * 0.6180339887) % 1.0) for i in range(case["seqs"])]
    lens = [max(1, int(case["entries"] * f)) for f in spread]
    new = [min(n, max(1, int(math.ceil(case["new"] * (1.5 * f - 0.5 if f > 0.5 else f))))) for n, f in zip(lens, spread)]
    return lens, new


def _missing(case, s, n_pages, length, n):
    """Pages of sequence s that were given back: one in the middle, or (windows) all that none of its new rows sees."""
    if case.get("holes"):
        return [n_pages // 3] if s % 2 == 0 and n_pages >= 4 else []
    if case.get("freed"):
        p, low = case["page"], length - n + 1 - case["window"]     # the first row's first entry
        return [b for b in range(n_pages) if b * p >= case["sinks"] and (b + 1) * p <= low]
    return []


def work(case):
    h_q, h_kv, d, dtype, _ = LAYOUTS[case["layout"]]
    lens, new = _lengths(case)
    act = 4 if dtype == "f32" else 2                      # bytes of an activation
    ele = act if case["fmt"] == "same" else 1             # and of a cached element
    scales = 8 / BLOCK if case["fmt"] == "scaled" else 0  # K's and V's, per entry
    rows = sum(new)
    if case["op"] == "store":
        turned = h_kv + (h_q if case["queries"] else 0)
        return {"bytes": rows * (h_kv * (2 * d * (act + ele) + 8 + scales) + (2 * h_q * d * act if case["queries"] else 0) + 16),
                "flops": rows * turned * 3 * d}
    pairs = entries = 0
    for s, (length, n) in enumerate(zip(lens, new)):
        gone = len(_missing(case, s, -(-length // case["page"]), length, n))
        if case["op"] == "scaled":
            length -= gone * case["page"]
            entries += length
            pairs += length * n - n * (n - 1) // 2
            continue
        w, k = case["window"], case["sinks"]
        low = length - n + 1 - w                           # what the first row sees begins here; sinks are 0 .. k - 1
        entries += length if low <= k else length - low + k
        pairs += sum(p + 1 if p - w < k else w + k for p in range(length - n, length))
    return {"bytes": h_kv * entries * (2 * d * ele + scales) + rows * h_q * (2 * d * act + 4), "flops": 4 * d * pairs * h_q}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _pow2(e):
    """2 ** e of whole numbers in -126 .. 127, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _code(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn)


def _random_pool(case, n_pages, h_kv, d, dt, g, lean):
    """Keys of very different norms, a few that most queries look at, and channels with large offsets, as trained models have;
    values of ordinary size."""
    shape = (n_pages, h_kv, case["page"], d)
    k = torch.randn(shape, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(*shape[:3], 1, generator=g, device="cuda"))
    k += lean * (torch.rand(*shape[:3], 1, generator=g, device="cuda") < 0.02)
    v = torch.randn(shape, generator=g, device="cuda")
    if case["fmt"] != "scaled":
        return [_code(x.to(dt).float()) if case["fmt"] == "fp8" else x.to(dt) for x in (k, v)] + [None, None]
    k[..., 5] += 600.0                                     # more than plain codes hold; the same for all keys, so no row minds
    codes, scales = [], []
    for x in (k, v):
        blocks = x.to(dt).float().view(n_pages, h_kv, -1, BLOCK, d)
        e = torch.frexp(blocks.abs().amax((3, 4)) / 448)[1].clamp(E_MIN, E_MAX)
        codes.append(_code(blocks * _pow2(-e)[..., None, None]).view(shape))
        scales.append(_pow2(e))
    return codes + scales


def prepare(case, seed):
    h_q, h_kv, d, dtype, section = LAYOUTS[case["layout"]]
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    page = case["page"]
    lens, new = _lengths(case)
    need = [-(-n // page) for n in lens]
    gone = [_missing(case, s, need[s], lens[s], new[s]) for s in range(len(lens))]
    n_pages = sum(need) - sum(len(x) for x in gone) + 3
    at = rng.sample(range(n_pages), n_pages)               # a pool that has been in use for a while
    table = torch.full((case["seqs"], max(need)), -1, dtype=torch.int32)
    for s, n in enumerate(need):
        for b in sorted(set(range(n)) - set(gone[s])):
            table[s, b] = at.pop()
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    rows = starts[-1]
    st = dict(case=case, h_q=h_q, h_kv=h_kv, d=d, page=page, fmt=case["fmt"], dt=dt, section=section, max_len=max(lens), max_new=max(new),
              scale=1 / math.sqrt(d))
    st["table"] = table.cuda()
    st["len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    st["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    lean = torch.randn(h_kv, 1, d, generator=g, device="cuda") * 0.6
    st["k"], st["v"], st["k_scale"], st["v_scale"] = _random_pool(case, n_pages, h_kv, d, dt, g, lean)
    st["pos"] = torch.randint(0, 460800, (n_pages, h_kv, page), generator=g, device="cuda", dtype=torch.int32)
    st["weight"] = torch.exp(1.5 * torch.randn(n_pages, h_kv, page, generator=g, device="cuda"))
    if case["op"] == "store":
        x = torch.randn(rows, h_q + 2 * h_kv, d, generator=g, device="cuda")               # the rows of a projection
        x[:, h_q:] *= torch.exp(0.5 * torch.randn(rows, 2 * h_kv, 1, generator=g, device="cuda"))
        if case["fmt"] == "scaled":
            x[:, h_q:h_q + h_kv, 5] += 600.0
        st["x"] = x.to(dt)
        st["new_pos"] = torch.randint(0, 460800, (rows,), generator=g, device="cuda", dtype=torch.int32)
        if case["new"] > 600:                              # a video's: frames of 11 x 11
            r, first = torch.arange(rows, device="cuda"), rng.randrange(400000)
            st["axes"] = (first + torch.stack([r // 121, r % 121 // 11, r % 11])).int().contiguous()
        else:                                              # text: the same on all axes
            st["axes"] = torch.randint(0, 460800, (rows,), generator=g, device="cuda", dtype=torch.int32).expand(3, rows).contiguous()
        st["q_out"] = torch.zeros(rows, h_q, d, dtype=dt, device="cuda") if case["queries"] else None
    else:
        q = torch.randn(rows, h_kv, h_q // h_kv, d, generator=g, device="cuda") + lean.view(1, h_kv, 1, d)
        st["q"] = q.view(rows, h_q, d).to(dt).contiguous()
        st["out"] = torch.zeros(rows, h_q, d, dtype=dt, device="cuda")
        st["lse"] = torch.zeros(h_q, rows, dtype=torch.float32, device="cuda")
    if own:
        from paper_2505_16175_amd import binding as B
        st["layout"] = B.make_layout(h_q, h_kv, d, dt)
        fmt = {"same": B.QP_CACHE_SAME, "fp8": B.QP_CACHE_FP8_E4M3, "scaled": B.QP_CACHE_FP8_E4M3_SCALED}[case["fmt"]]
        st["cache"] = B.PagedCache(st["layout"], n_pages, page, fmt=fmt, k=st["k"], v=st["v"], pos=st["pos"], weight=st["weight"],
                                   k_scale=st["k_scale"], v_scale=st["v_scale"])
        st["batch"] = B.PagedBatch(st["table"], st["len"], st["row_start"], n_rows=rows, max_new=st["max_new"], max_len=st["max_len"])
        st["ws"] = B.make_paged_workspace(st["layout"], st["batch"])
        if case["op"] == "store":
            st["rope"] = B.PagedRope(st["layout"], st["axes"], THETA, section)
    return st


# ---- the operators ------------------------------------------------------------------------------------------------

def run(st):
    case = st["case"]
    if own:
        from paper_2505_16175_amd import binding as B
        if case["op"] == "store":
            q, k, v = st["x"].split((st["h_q"], st["h_kv"], st["h_kv"]), 1)
            B.paged_append_rope(st["layout"], st["cache"], st["batch"], k, v, st["new_pos"], st["rope"],
                                q if case["queries"] else None, st["q_out"])
        elif case["op"] == "window":
            B.paged_attend_window(st["layout"], st["cache"], st["batch"], case["window"], case["sinks"], st["q"], st["out"], st["lse"],
                                  st["ws"])
        else:
            B.paged_attend(st["layout"], st["cache"], st["batch"], st["q"], st["out"], st["lse"], st["ws"])
    elif case["op"] == "store":
        _store(st)
    else:
        _attend(st)
    if case["op"] != "store":
        return {"out": st["out"], "lse": st["lse"]}
    return {name: st[name] for name in ("k", "v", "k_scale", "v_scale", "pos", "weight", "q_out")}


def _places(st, j):
    """Page and slot of entries j [S, n] of the sequences, and whether the table has a page there."""
    index = (j // st["page"]).clamp(0, st["table"].shape[1] - 1).long()
    page = torch.gather(st["table"], 1, index).long()
    return page.clamp(min=0), (j % st["page"]).long(), (page >= 0) & (page < st["k"].shape[0])


def _new_rows(st):
    """Row numbers [S, N] of every sequence's new tokens, and which there are."""
    n = st["row_start"][1:] - st["row_start"][:-1]
    i = torch.arange(st["max_new"], device="cuda").expand(n.shape[0], -1)
    ok = i < n[:, None]
    return torch.where(ok, st["row_start"][:-1, None] + i, 0).long(), ok, i, n


def _gather(pool, scale, page, slot):
    """Entries [S, H, L, d] of the pool in 32 bits."""
    raw = pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool
    got = raw.permute(0, 2, 1, 3)[page, slot]
    got = (got.view(torch.float8_e4m3fn) if pool.dtype == torch.float8_e4m3fn else got).float()
    if scale is not None:
        got = got * scale.transpose(1, 2)[page, slot // BLOCK][..., None]
    return got.transpose(1, 2)


def _attend(st):
    j = torch.arange(st["max_len"], device="cuda").expand(st["len"].shape[0], -1)
    page, slot, here = _places(st, j)
    here = here & (j < st["len"][:, None])
    row, ok, i, n = _new_rows(st)
    S, N, h_kv, r, d = row.shape[0], row.shape[1], st["h_kv"], st["h_q"] // st["h_kv"], st["d"]
    q = st["q"].float()[row].view(S, N, h_kv, r, d).transpose(1, 2).reshape(S, h_kv, N * r, d)
    s = torch.matmul(q, _gather(st["k"], st["k_scale"], page, slot).transpose(2, 3)).view(S, h_kv, N, r, -1) * st["scale"]
    at = ((st["len"] - n)[:, None] + i)[:, :, None]                                        # the row's own entry
    j = j[:, None, :]
    seen = here[:, None, :] & (j <= at) & ok[:, :, None]
    if st["case"]["op"] == "window":
        seen = seen & ((j < st["case"]["sinks"]) | (j > at - st["case"]["window"]))
    s = s.masked_fill(~seen[:, None, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - m)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(S, h_kv, N * r, -1), _gather(st["v"], st["v_scale"], page, slot)).view(S, h_kv, N, r, d)
    o = torch.where(total > 0, o / total, 0)
    st["out"][row[ok]] = o.permute(0, 2, 1, 3, 4).reshape(S, N, st["h_q"], d)[ok].to(st["out"].dtype)
    lse = torch.where(total > 0, m + torch.log(total), -math.inf)[..., 0]
    st["lse"][:, row[ok]] = lse.permute(0, 2, 1, 3).reshape(S, N, st["h_q"])[ok].t()


def _turn(st, x):
    """x [rows, heads, d] in 32 bits, pairs (i, i + d / 2) turned by their rows' angles, which are taken in 64 bits."""
    half = st["d"] // 2
    freq = THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    t, h, w = st["axes"].double()[:, :, None] * freq
    angle = torch.cat([part[:, a:b] for part, a, b in zip((t, h, w), (0, st["section"][0], half - st["section"][2]),
                                                          (st["section"][0], half - st["section"][2], half))], 1)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    lo, hi = x[..., :half], x[..., half:]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)


def _exponents(x, largest):
    """The least e with |x| <= largest * 2 ** e for the finite values of the last dimension. `largest` is its mantissa, times 2 ** 9."""
    size = x.abs()
    m, e = torch.frexp(torch.where(size < math.inf, size, 0).amax(-1))
    return torch.where(m > 0, e - 9 + (m > largest).int(), E_MIN).clamp(E_MIN, E_MAX)


def _store(st):
    q, k, v = st["x"].float().split((st["h_q"], st["h_kv"], st["h_kv"]), 1)
    if st["q_out"] is not None:
        st["q_out"].copy_(_turn(st, q))
    turned = _turn(st, k)
    # whole blocks of entries around the new ones: [S, blocks, BLOCK]
    n = (st["row_start"][1:] - st["row_start"][:-1])[:, None]
    begin = st["len"][:, None] - n
    j = begin // BLOCK * BLOCK + torch.arange((st["max_new"] + 2 * BLOCK - 2) // BLOCK * BLOCK, device="cuda")
    page, slot, here = _places(st, j)
    is_new = here & (j >= begin) & (j < st["len"][:, None])
    row = torch.where(is_new, st["row_start"][:-1, None] + j - begin, 0).long()
    new_page, new_slot, new_row = page[is_new], slot[is_new], row[is_new]
    st["pos"].transpose(1, 2)[new_page, new_slot] = st["new_pos"][new_row][:, None].expand(-1, st["h_kv"])
    st["weight"].transpose(1, 2)[new_page, new_slot] = 0
    if st["fmt"] != "scaled":
        for pool, x in ((st["k"], turned), (st["v"], v)):
            x = _code(x).view(torch.uint8) if st["fmt"] == "fp8" else x.to(st["dt"])
            pool.view(x.dtype).transpose(1, 2)[new_page, new_slot] = x[new_row]
        return
    S, h_kv = j.shape[0], st["h_kv"]
    first = here & (j < begin)                                                             # earlier entries of the first block
    old_page, old_slot = page[first], slot[first]
    block_page, block = (x.view(S, -1, BLOCK)[..., 0] for x in (page, slot // BLOCK))
    written = is_new.view(S, -1, BLOCK).any(-1)
    # turned keys are at most sqrt(2) times as large as before: 316 = 0.6171875 * 2 ** 9 of them for 448 = 0.875 * 2 ** 9
    for pool, scale, x, size, largest in ((st["k"], st["k_scale"], turned, k, 0.6171875), (st["v"], st["v_scale"], v, v, 0.875)):
        e = torch.where(is_new[..., None], _exponents(size, largest)[row], E_MIN).view(S, -1, BLOCK, h_kv).amax(2)
        before = scale.transpose(1, 2)[block_page, block]                                   # [S, blocks, H]
        before_e = torch.where(first.view(S, -1, BLOCK).any(-1)[..., None], (before.view(torch.int32) >> 23) - 127, E_MIN)
        e = torch.maximum(e, before_e).clamp(E_MIN, E_MAX)
        wide = e.repeat_interleave(BLOCK, 1)
        raw = pool.view(torch.uint8).transpose(1, 2)
        was = raw[old_page, old_slot].view(torch.float8_e4m3fn).float()
        raw[old_page, old_slot] = _code(was * _pow2((before_e.repeat_interleave(BLOCK, 1)[first] - wide[first]).clamp(min=-126))[..., None]).view(torch.uint8)
        raw[new_page, new_slot] = _code(x[new_row] * _pow2(-wide[is_new])[..., None]).view(torch.uint8)
        scale.transpose(1, 2)[block_page[written], block[written]] = _pow2(e[written])


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return _exact_store(st, case) if case["op"] == "store" else _exact_attend(st, case)


def _exact_store(st, case):
    lens, new = _lengths(case)
    d, h_q, h_kv, page = st["d"], st["h_q"], st["h_kv"], case["page"]
    axis = [a for a in range(3) for _ in range(st["section"][a])]
    angle = torch.stack([st["axes"][a].double() * math.exp(-2 * i / d * math.log(THETA)) for i, a in enumerate(axis)], 1)
    z = torch.polar(torch.ones_like(angle), angle)[:, None]
    x = st["x"].double()

    def turned(y):
        y = torch.complex(y[..., : d // 2], y[..., d // 2:]) * z
        return torch.cat([y.real, y.imag], -1)

    rows = {"k": turned(x[:, h_q:h_q + h_kv]), "v": x[:, h_q + h_kv:]}
    limit = {"k": 316.0, "v": 448.0}
    got = {"k": st["k"].to(torch.float64), "v": st["v"].to(torch.float64), "k_scale": None, "v_scale": None, "pos": None, "weight": None,
           "q_out": turned(x[:, :h_q]) if case["queries"] else None}
    scaled = case["fmt"] == "scaled"
    if scaled:
        got.update(k_scale=st["k_scale"].double(), v_scale=st["v_scale"].double())
    first_row = 0
    for s, (length, n) in enumerate(zip(lens, new)):
        pages = st["table"][s].tolist()
        for name in ("k", "v"):
            pool, to = got[name], rows[name]
            j = torch.arange(length - n, length, device="cuda")
            p = torch.tensor(pages, device="cuda")[j // page]
            y = to[first_row:first_row + n]
            if not scaled:
                pool[p, :, j % page] = y.clamp(-448, 448) if case["fmt"] == "fp8" else y
                continue
            source = x[first_row:first_row + n, h_q:h_q + h_kv] if name == "k" else y
            size = source.abs().amax(-1)                                                   # [n, H]
            block = j // BLOCK - (length - n) // BLOCK
            most = torch.zeros(int(block[-1]) + 1, h_kv, dtype=torch.float64, device="cuda")
            most.scatter_reduce_(0, block[:, None].expand(-1, h_kv), size, "amax")
            e = torch.ceil(torch.log2((most / limit[name]).clamp(min=2.0 ** E_MIN)) - 1e-13).clamp(E_MIN, E_MAX)
            scales = got[name + "_scale"]
            old = (length - n) % BLOCK
            if old:
                q, b = pages[(length - n) // page], (length - n) % page // BLOCK
                was = torch.log2(scales[q, :, b])
                e[0] = torch.maximum(e[0], was)
                pool[q, :, b * BLOCK:b * BLOCK + old] *= torch.exp2(was - e[0])[:, None, None]
            pool[p, :, j % page] = (y * torch.exp2(-e[block])[..., None]).clamp(-448, 448)
            scales[p, :, j % page // BLOCK] = torch.exp2(e[block])
        first_row += n
    return got


def _exact_attend(st, case):
    lens, new = _lengths(case)
    r, page, rows = st["h_q"] // st["h_kv"], case["page"], sum(new)
    out = torch.zeros(rows, st["h_q"], st["d"], dtype=torch.float64, device="cuda")
    lse = torch.full((st["h_q"], rows), -math.inf, dtype=torch.float64, device="cuda")
    begin = 0
    for s, (length, n) in enumerate(zip(lens, new)):
        pages = st["table"][s, : -(-length // page)].tolist()
        number = torch.cat([torch.arange(b * page, min(length, (b + 1) * page)) for b, p in enumerate(pages) if p >= 0]).cuda()
        at = torch.cat([torch.arange(p * page, p * page + min(page, length - b * page)) for b, p in enumerate(pages) if p >= 0]).cuda()
        limit = (length - n + torch.arange(n, device="cuda")).repeat_interleave(r)
        for h in range(st["h_kv"]):
            k, v = (st[name][at // page, h, at % page] if case["fmt"] == "same" else
                    st[name].view(torch.uint8)[at // page, h, at % page].view(torch.float8_e4m3fn) for name in ("k", "v"))
            k, v = k.double(), v.double()
            if case["fmt"] == "scaled":
                k = k * st["k_scale"][at // page, h, at % page // BLOCK].double()[:, None]
                v = v * st["v_scale"][at // page, h, at % page // BLOCK].double()[:, None]
            q = st["q"][begin:begin + n, h * r:(h + 1) * r].reshape(n * r, -1).double()
            for a in range(0, n * r, 1024):
                last = limit[a:a + 1024, None]
                hidden = number[None, :] > last
                if case["op"] == "window":
                    hidden |= (number[None, :] <= last - case["window"]) & (number[None, :] >= case["sinks"])
                x = (q[a:a + 1024] @ k.t()) / math.sqrt(st["d"])
                x[hidden] = -math.inf
                z = torch.logsumexp(x, -1)
                o = torch.softmax(x, -1) @ v
                o[z == -math.inf] = 0
                row = torch.arange(a, a + len(x), device="cuda")
                out[begin + row // r, h * r + row % r] = o
                lse[h * r + row % r, begin + row // r] = z
        begin += n
    return {"out": out, "lse": lse}
