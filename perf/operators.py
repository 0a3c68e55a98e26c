"""Performance cases of the paged cache: many sequences over one pool of pages, as answers to questions about videos are
served. Its four operators, each over the range of sizes that it meets:

  append   new keys and values (a decoding step's, or the pruned entries that a video left) stored in the sequences' pages
  attend   attention of each sequence's new tokens over its entries, with the rows' log-sum-exps
  weigh    the attention weight that each entry received from those rows, taken anew or added to what it had
  evict    the entries of most weight, with the first and the last ones, moved to other pages

With `own` the calls are the library's; without, the same results from elementary torch operations in 32 bits. `exact()`
has them in 64 bits, sequence by sequence, from the definitions.
"""
import math
import random

import torch

own = False

# (query heads, KV heads, head_dim, dtype): a tiny f32 layout for the smallest calls, and those of the 7B and 72B models
LAYOUTS = {"tiny": (4, 2, 64, "f32"), "7b": (28, 4, 128, "bf16"), "72b": (64, 8, 128, "bf16")}
MAX_PAIRS = 1.5e9          # (row, entry) pairs over all query heads of a batch: what the largest listed chunk has
MAX_ENTRIES = 1.2e6        # entries times KV heads of a batch


def _case(name, op, layout, seqs, new, entries, ragged, page, fp8=False, holes=False, **more):
    return dict(name=name, op=op, layout=layout, seqs=seqs, new=new, entries=entries, ragged=ragged, page=page, fp8=fp8,
                holes=holes, **more)


def listed():
    return [
        # the smallest call: one token of one answer over a tiny cache in f32; launches and waits are what it costs
        _case("attend_reply_f32", "attend", "tiny", 1, 1, 333, 1.0, 16),
        # one answer's token over the hour-long video's cache: few rows, a long axis
        _case("attend_reply_7b", "attend", "7b", 1, 1, 46125, 1.0, 64),
        # a decoding step of 32 answers over caches of very different lengths
        _case("attend_replies_7b", "attend", "7b", 32, 1, 9840, 0.1, 64),
        # the large model's 8-bit caches, up to four drafted tokens per answer; freed pages in the middle
        _case("attend_drafts_72b_fp8", "attend", "72b", 16, 4, 32768, 0.3, 32, fp8=True, holes=True),
        # four questions of up to 300 tokens over hour-long caches: the matrix products count
        _case("attend_questions_7b", "attend", "7b", 4, 300, 46125, 0.3, 128),
        # a decoding step's keys and values of 32 answers
        _case("append_replies_7b", "append", "7b", 32, 1, 9840, 0.1, 64),
        # what an hour-long video left, moved from the flat pruned cache into 8-bit pages
        _case("append_video_72b_fp8", "append", "72b", 1, 46125, 46125, 1.0, 64, fp8=True),
        # the weights of a decoding step added to those of 32 answers' entries
        _case("weigh_replies_7b", "weigh", "7b", 32, 1, 9840, 0.1, 64, accumulate=True),
        # what a question of 500 tokens looks at in an hour-long video
        _case("weigh_question_7b", "weigh", "7b", 1, 500, 46125, 1.0, 64, accumulate=False),
        # two short questions over 8-bit caches of the large model
        _case("weigh_questions_72b_fp8", "weigh", "72b", 2, 77, 20000, 0.5, 32, fp8=True, accumulate=True),
        # one long cache cut to its budget
        _case("evict_hour_7b", "evict", "7b", 1, 0, 46125, 1.0, 64, keep=16384, first=4, last=64),
        # sixteen answers of the large model back to theirs
        _case("evict_replies_72b", "evict", "72b", 16, 0, 8300, 0.4, 32, keep=4096, first=4, last=256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "weigh", "evict"])
    layout = rng.choice(["tiny", "7b", "7b", "72b"])
    h_q, h_kv, d, dtype = LAYOUTS[layout]
    most = 5000 if dtype == "f32" else 46125
    fp8 = dtype == "bf16" and rng.random() < 0.3
    page = rng.choice([16, 32, 64, 128, 256])
    entries = _log(rng, 1, most)
    seqs = min(_log(rng, 1, 64), max(1, int(MAX_ENTRIES / (h_kv * entries))))
    new = _log(rng, 1, 8) if rng.random() < 0.6 else _log(rng, 8, 600 if dtype == "bf16" else 64)
    new = max(1, min(new, entries, int(MAX_PAIRS / (seqs * h_q * entries))))
    ragged = rng.choice([0.05, 0.3, 0.7, 1.0])
    holes = rng.random() < 0.25
    if op == "append":
        new = entries if rng.random() < 0.4 else new
        return _draw(op, layout, seqs, new, entries, ragged, page, fp8, False)
    if op == "evict":
        keep = max(1, int(entries * rng.uniform(0.1, 0.9)))
        first = min(rng.choice([0, 1, 4]), keep)
        return _draw(op, layout, seqs, 0, entries, ragged, page, fp8, holes, keep=keep, first=first,
                     last=min(rng.choice([0, 16, 256]), keep - first))
    if op == "weigh":
        return _draw(op, layout, seqs, new, entries, ragged, page, fp8, holes, accumulate=rng.random() < 0.5)
    return _draw(op, layout, seqs, new, entries, ragged, page, fp8, holes)


def _draw(*a, **more):
    c = _case("", *a, **more)
    del c["name"]
    return c


def _lengths(case):
    """Entries and new rows of each sequence: the first has the most, the others spread down to `ragged` of it."""
    spread = [1.0 if i == 0 else case["ragged"] + (1 - case["ragged"]) * ((i * 0.6180339887) % 1.0) for i in range(case["seqs"])]
    lens = [max(1, int(case["entries"] * f)) for f in spread]
    new = [min(n, max(1, int(math.ceil(case["new"] * (1.5 * f - 0.5 if f > 0.5 else f))))) if case["new"] else 0
           for n, f in zip(lens, spread)]
    return lens, new


def _hole(case, s, n_pages):
    """A page of sequence s that was given back (a window slid on), or none: never one of the last two."""
    return n_pages // 3 if case["holes"] and s % 2 == 0 and n_pages >= 4 else None


def _present(case):
    """Entries of each sequence that are in the pool."""
    lens, _ = _lengths(case)
    return [n - (case["page"] if _hole(case, s, -(-n // case["page"])) is not None else 0) for s, n in enumerate(lens)]


def work(case):
    h_q, h_kv, d, dtype = LAYOUTS[case["layout"]]
    lens, new = _lengths(case)
    here = _present(case)
    act = 4 if dtype == "f32" else 2                     # bytes of an activation
    ele = 1 if case["fp8"] else act                      # and of a cached element
    rows = sum(new)
    if case["op"] == "append":
        return {"bytes": rows * h_kv * (2 * d * (act + ele) + 8) + 4 * rows, "flops": 0}
    if case["op"] == "evict":
        kept = sum(min(n, case["keep"]) for n in here)
        return {"bytes": h_kv * (4 * sum(here) + kept * (2 * (2 * d * ele) + 4 + 8)), "flops": 0}
    # pairs that are seen: a row i of n sees the first L - n + i + 1 entries
    pairs = sum(h * n - n * (n - 1) // 2 for h, n in zip(here, new)) * h_q
    if case["op"] == "weigh":
        known = 8 if case["accumulate"] else 4
        return {"bytes": h_kv * sum(here) * (d * ele + known) + rows * h_q * (d * act + 4), "flops": 2 * d * pairs}
    return {"bytes": h_kv * sum(here) * 2 * d * ele + rows * h_q * (2 * d * act + 4), "flops": 4 * d * pairs}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _to_pool(x, fp8):
    return x.to(torch.float8_e4m3fn) if fp8 else x


def prepare(case, seed):
    h_q, h_kv, d, dtype = LAYOUTS[case["layout"]]
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(seed)
    page, fp8 = case["page"], case["fp8"]
    lens, new = _lengths(case)
    need = [-(-n // page) for n in lens]
    keep_pages = -(-case["keep"] // page) if case["op"] == "evict" else 0
    n_pages = sum(need) + keep_pages * case["seqs"] + 3
    at = random.Random(seed).sample(range(n_pages), n_pages)      # a pool that has been in use for a while
    table = torch.full((case["seqs"], max(need)), -1, dtype=torch.int32)
    for s, n in enumerate(need):
        table[s, :n] = torch.tensor([at.pop() for _ in range(n)], dtype=torch.int32)
        hole = _hole(case, s, n)
        if hole is not None:
            table[s, hole] = -1
    st = dict(case=case, h_q=h_q, h_kv=h_kv, d=d, page=page, fp8=fp8, max_len=max(lens), max_new=max(new), scale=1 / math.sqrt(d))
    st["table"] = table.cuda()
    st["len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    rows = starts[-1]
    st["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")

    # keys of very different norms and a few that most queries look at, as in trained models
    lean = torch.randn(h_kv, 1, d, generator=g, device="cuda") * 0.6
    if case["op"] == "append":
        pool_k = torch.zeros(n_pages, h_kv, page, d, dtype=torch.float8_e4m3fn if fp8 else dt, device="cuda")
        pool_v = torch.zeros_like(pool_k)
        if case["new"] == case["entries"] and case["new"] > 1:    # entries of a flat pruned cache: heads first
            src = lambda: torch.randn(h_kv, rows, d, generator=g, device="cuda").to(dt).transpose(0, 1)
            st["new_pos"] = torch.sort(torch.randint(0, 460800, (h_kv, rows), generator=g, device="cuda", dtype=torch.int32))[0].t()
        else:
            src = lambda: torch.randn(rows, h_kv, d, generator=g, device="cuda").to(dt)
            st["new_pos"] = torch.randint(0, 460800, (rows,), generator=g, device="cuda", dtype=torch.int32)
        st["new_k"], st["new_v"] = src(), src()
    else:
        pool_k = torch.randn(n_pages, h_kv, page, d, generator=g, device="cuda")
        pool_k *= torch.exp(0.5 * torch.randn(n_pages, h_kv, page, 1, generator=g, device="cuda"))
        pool_k += lean * (torch.rand(n_pages, h_kv, page, 1, generator=g, device="cuda") < 0.02)
        pool_k = _to_pool(pool_k.to(dt), fp8)
        pool_v = _to_pool(torch.randn(n_pages, h_kv, page, d, generator=g, device="cuda").to(dt), fp8)
    pos = torch.randint(0, 460800, (n_pages, h_kv, page), generator=g, device="cuda", dtype=torch.int32)
    weight = torch.exp(1.5 * torch.randn(n_pages, h_kv, page, generator=g, device="cuda"))
    weight[torch.rand(n_pages, h_kv, page, generator=g, device="cuda") < 0.05] = 0.25       # equal weights happen
    st.update(k=pool_k, v=pool_v, pos=pos, weight=weight)
    if rows and case["op"] != "append":
        q = torch.randn(rows, h_kv, h_q // h_kv, d, generator=g, device="cuda") + lean.view(1, h_kv, 1, d)
        st["q"] = q.view(rows, h_q, d).to(dt).contiguous()
    if case["op"] == "attend":
        st["out"] = torch.zeros(rows, h_q, d, dtype=dt, device="cuda")
        st["lse"] = torch.zeros(h_q, rows, dtype=torch.float32, device="cuda")
    if case["op"] == "weigh":                                     # what attention of these rows returned
        s, seen, _, row, ok = _scores(st)
        lse = torch.logsumexp(s.masked_fill(~seen, -math.inf), -1)
        st["lse"] = torch.zeros(h_q, rows, dtype=torch.float32, device="cuda")
        _put_lse(st, lse, row, ok)
        del s, seen
    if case["op"] == "evict":
        to = torch.tensor([[at.pop() for _ in range(keep_pages)] for _ in range(case["seqs"])], dtype=torch.int32)
        st["to_table"] = to.cuda()
        st["to_len"] = torch.zeros(case["seqs"], dtype=torch.int32, device="cuda")
        st["kept"] = torch.full((case["seqs"], h_kv, case["keep"]), -1, dtype=torch.int32, device="cuda")
    if own:
        from paper_2505_16175_amd import binding as B
        st["layout"] = B.make_layout(h_q, h_kv, d, dt)
        st["cache"] = B.PagedCache(st["layout"], n_pages, page, k=st["k"], v=st["v"], pos=pos, weight=weight)
        st["batch"] = B.PagedBatch(st["table"], st["len"], st["row_start"], n_rows=rows, max_new=st["max_new"], max_len=st["max_len"])
        st["ws"] = B.make_paged_workspace(st["layout"], st["batch"], case.get("keep", 0))
    return st


# ---- the operators ------------------------------------------------------------------------------------------------

def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2505_16175_amd import binding as B
        if op == "append":
            B.paged_append(st["layout"], st["cache"], st["batch"], st["new_k"], st["new_v"], st["new_pos"])
        elif op == "attend":
            B.paged_attend(st["layout"], st["cache"], st["batch"], st["q"], st["out"], st["lse"], st["ws"])
        elif op == "weigh":
            B.paged_weigh(st["layout"], st["cache"], st["batch"], st["q"], st["lse"], st["case"]["accumulate"], st["ws"])
        else:
            B.paged_evict(st["layout"], st["cache"], st["batch"], st["case"]["keep"], st["case"]["first"], st["case"]["last"],
                          st["to_table"], st["to_len"], st["kept"], st["ws"])
    else:
        {"append": _append, "attend": _attend, "weigh": _weigh, "evict": _evict}[op](st)
    if op == "append":
        return {"k": st["k"], "v": st["v"], "pos": st["pos"], "weight": st["weight"]}
    if op == "attend":
        return {"out": st["out"], "lse": st["lse"]}
    if op == "weigh":
        return {"weight": st["weight"]}
    return {"k": st["k"], "v": st["v"], "pos": st["pos"], "weight": st["weight"], "len": st["to_len"], "kept": st["kept"]}


def _places(st, table, j):
    """Page and slot of entries j [S, n] (any shape behind S), and whether the table has a page there."""
    index = (j // st["page"]).clamp(0, table.shape[1] - 1).long()
    page = torch.gather(table, 1, index).long()
    return page.clamp(min=0), (j % st["page"]).long(), (page >= 0) & (page < st["k"].shape[0])


def _entries(st):
    """Entry numbers [S, L] of every sequence, their places, and which of them there are."""
    j = torch.arange(st["max_len"], device="cuda").expand(st["len"].shape[0], -1)
    page, slot, here = _places(st, st["table"], j)
    return j, page, slot, here & (j < st["len"][:, None])


def _gather(pool, page, slot):
    """Entries [S, H, L, d] of the pool in 32 bits."""
    raw = pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool
    got = raw.permute(0, 2, 1, 3)[page, slot]
    return (got.view(torch.float8_e4m3fn) if pool.dtype == torch.float8_e4m3fn else got).float().transpose(1, 2)


def _new_rows(st):
    """Row numbers [S, N] of every sequence's new tokens, and which there are."""
    n = st["row_start"][1:] - st["row_start"][:-1]
    i = torch.arange(st["max_new"], device="cuda").expand(n.shape[0], -1)
    ok = i < n[:, None]
    return torch.where(ok, st["row_start"][:-1, None] + i, 0).long(), ok, i, n


def _scores(st):
    """Scaled products [S, H_kv, N, R, L] and what each row sees of them, the values' places, the rows."""
    j, page, slot, here = _entries(st)
    row, ok, i, n = _new_rows(st)
    S, N, h_kv, r, d = row.shape[0], row.shape[1], st["h_kv"], st["h_q"] // st["h_kv"], st["d"]
    q = st["q"].float()[row].view(S, N, h_kv, r, d).transpose(1, 2).reshape(S, h_kv, N * r, d)
    s = torch.matmul(q, _gather(st["k"], page, slot).transpose(2, 3)).view(S, h_kv, N, r, -1) * st["scale"]
    last = (st["len"] - n)[:, None] + i
    seen = here[:, None, :] & (j[:, None, :] <= last[:, :, None]) & ok[:, :, None]
    return s, seen[:, None, :, None, :], (page, slot), row, ok


def _put_lse(st, lse, row, ok):
    """lse [S, H_kv, N, R] to its rows."""
    st["lse"][:, row[ok]] = lse.permute(0, 2, 1, 3).reshape(*row.shape, st["h_q"])[ok].t()


def _attend(st):
    s, seen, (page, slot), row, ok = _scores(st)
    s = s.masked_fill(~seen, -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - m)
    total = p.sum(-1, keepdim=True)
    S, h_kv, N, r, L = p.shape
    o = torch.matmul(p.view(S, h_kv, N * r, L), _gather(st["v"], page, slot)).view(S, h_kv, N, r, -1)
    o = torch.where(total > 0, o / total, 0)
    st["out"][row[ok]] = o.permute(0, 2, 1, 3, 4).reshape(S, N, st["h_q"], -1)[ok].to(st["out"].dtype)
    _put_lse(st, torch.where(total > 0, m + torch.log(total), -math.inf)[..., 0], row, ok)


def _weigh(st):
    s, seen, (page, slot), row, ok = _scores(st)
    S, h_kv, N, r, L = s.shape
    lse = st["lse"].t()[row].view(S, N, h_kv, r).transpose(1, 2)[..., None]
    got = torch.where(seen & (lse > -math.inf), torch.exp(s - lse), 0).sum((2, 3))       # [S, H_kv, L]
    here = _entries(st)[3]
    old = st["weight"].transpose(1, 2)[page, slot] if st["case"]["accumulate"] else 0
    st["weight"].transpose(1, 2)[page[here], slot[here]] = (old + got.transpose(1, 2))[here]


def _append(st):
    row, ok, i, n = _new_rows(st)
    page, slot, here = _places(st, st["table"], (st["len"] - n)[:, None] + i)
    here = here & ok
    page, slot, row = page[here], slot[here], row[here]
    k, v = st["new_k"][row], st["new_v"][row]
    if st["fp8"]:                                                  # values beyond the largest one saturate
        k, v = (x.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x in (k, v))
    byte = torch.uint8 if st["fp8"] else st["k"].dtype
    st["k"].view(byte).transpose(1, 2)[page, slot] = k
    st["v"].view(byte).transpose(1, 2)[page, slot] = v
    pos = st["new_pos"][row]
    st["pos"].transpose(1, 2)[page, slot] = pos if pos.dim() == 2 else pos[:, None].expand(-1, st["h_kv"])
    st["weight"].transpose(1, 2)[page, slot] = 0


def _evict(st):
    keep, first, last = (st["case"][n] for n in ("keep", "first", "last"))
    j, page, slot, here = _entries(st)
    w = st["weight"].transpose(1, 2)[page, slot].transpose(1, 2)                           # [S, H, L]
    stays = (j < first) | (j >= st["len"][:, None] - last)
    w = torch.where(stays[:, None], math.inf, w).masked_fill(~here[:, None], -math.inf)
    order = torch.argsort(w, dim=-1, descending=True, stable=True)[..., :keep]
    count = here.sum(-1).clamp(max=keep)
    past = torch.arange(order.shape[-1], device="cuda") >= count[:, None]
    kept = torch.sort(order.masked_fill(past[:, None], st["max_len"]))[0]                  # ascending, what is not there last
    st["to_len"].copy_(count)
    st["kept"].fill_(-1)
    st["kept"][..., : kept.shape[-1]] = torch.where(past[:, None], -1, kept).int()
    S, H, n = kept.shape
    ok = ~past[:, None].expand(S, H, n)
    head = torch.arange(H, device="cuda")[None, :, None].expand(S, H, n)[ok]
    src = kept.clamp(max=st["max_len"] - 1).view(S, H * n)
    sp, sl = (x.view(S, H, n)[ok] for x in (torch.gather(page, 1, src), torch.gather(slot, 1, src)))
    dst = torch.arange(n, device="cuda").expand(S, H, n).reshape(S, H * n)
    dp, dl = (x.view(S, H, n)[ok] for x in _places(st, st["to_table"], dst)[:2])
    byte = torch.uint8 if st["fp8"] else st["k"].dtype
    st["k"].view(byte)[dp, head, dl] = st["k"].view(byte)[sp, head, sl]
    st["v"].view(byte)[dp, head, dl] = st["v"].view(byte)[sp, head, sl]
    st["pos"][dp, head, dl] = st["pos"][sp, head, sl]
    st["weight"][dp, head, dl] = st["weight"][sp, head, sl]


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] in ("append", "evict"):
        return None                                                # nothing is computed: values are moved
    st = prepare(case, seed)
    lens, new = _lengths(case)
    r, page = st["h_q"] // st["h_kv"], case["page"]
    out = torch.zeros(sum(new), st["h_q"], st["d"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["h_q"], sum(new), dtype=torch.float64, device="cuda")
    weight = st["weight"].double()
    begin = 0
    for s, (length, n) in enumerate(zip(lens, new)):
        pages = st["table"][s, : -(-length // page)].tolist()
        number = torch.cat([torch.arange(b * page, min(length, (b + 1) * page)) for b, p in enumerate(pages) if p >= 0]).cuda()
        at = torch.cat([torch.arange(p * page, p * page + min(page, length - b * page)) for b, p in enumerate(pages) if p >= 0]).cuda()
        limit = (length - n + torch.arange(n, device="cuda")).repeat_interleave(r)
        for h in range(st["h_kv"]):
            k = st["k"][:, h].reshape(-1, st["d"]).view(torch.uint8 if st["fp8"] else st["k"].dtype)[at]
            v = st["v"][:, h].reshape(-1, st["d"]).view(torch.uint8 if st["fp8"] else st["v"].dtype)[at]
            if st["fp8"]:
                k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
            k, v = k.double(), v.double()
            q = st["q"][begin:begin + n, h * r:(h + 1) * r].reshape(n * r, -1).double()
            added = torch.zeros(len(at), dtype=torch.float64, device="cuda")
            for a in range(0, n * r, 1024):
                x = (q[a:a + 1024] @ k.t()) / math.sqrt(st["d"])
                x[number[None, :] > limit[a:a + 1024, None]] = -math.inf
                if case["op"] == "attend":
                    z = torch.logsumexp(x, -1)
                    o = torch.softmax(x, -1) @ v
                    o[z == -math.inf] = 0
                    row = torch.arange(a, a + len(x), device="cuda")
                    out[begin + row // r, h * r + row % r] = o
                    lse[h * r + row % r, begin + row // r] = z
                else:
                    z = st["lse"][h * r:(h + 1) * r, begin:begin + n].t().reshape(-1)[a:a + 1024].double()
                    x = torch.exp(x - z[:, None])
                    x[z == -math.inf] = 0
                    added += x.sum(0)
            if case["op"] == "weigh":
                old = weight[at // page, h, at % page] if case["accumulate"] else 0
                weight[at // page, h, at % page] = old + added
        begin += n
    return {"out": out, "lse": lse} if case["op"] == "attend" else {"weight": weight}
