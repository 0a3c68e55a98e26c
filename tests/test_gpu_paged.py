"""GPU parity of the paged cache's calls (include/qp_paged.h) against their fp64 oracle.

Tolerances count roundings. u = 2^-24 is half a step of f32, h half a step of the output's type (2^-8 for bf16). A logit is a
sum of d exact (bf16) or once-rounded (f32) products scaled once, off by at most (d + 2) u scale sum |q||k|, and its distance from a
row's reference or lse, in f32 and base 2, by a few u of its size: `size` = the largest of both sums, so an exponential's relative error
is at most e = (d + 16) u size + 2^-22 (its own). A result sum p v / sum p is off by e twice, by the numerators' rounding n (two bf16
terms 2^-16; f32: none), by the sums' roundings (in parts of a few hundred terms, merged: 2^-15 covers the longest here), all relative to
the mean of |v| under the softmax, and by its own rounding."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paper_2505_16175_amd import binding as B
from paper_2505_16175_amd.workload import to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TINY, F32, BF64, L7, L72, ODD, WIDE = ((4, 2, 64, "f32"), (6, 3, 128, "f32"), (10, 2, 64, "bf16"), (28, 4, 128, "bf16"), (64, 8, 128, "bf16"),
                                  (15, 5, 128, "bf16"), (40, 1, 128, "bf16"))


class Scene:
    """A pool in use, sequences over pages of it in random order, and their new rows; what nobody may look at holds NaN."""

    def __init__(self, layout, page, lens, new, seed=0, fp8=False, missing=(), spare_rows=(2, 3), spare_pages=3, scale=0.0, sharp=1.0,
                 table_extra=0):
        h_q, h_kv, d, dtype = layout
        self.layout = B.make_layout(*layout, softmax_scale=scale)
        self.scale, self.h_q, self.h_kv, self.d, self.page = scale or 1 / math.sqrt(d), h_q, h_kv, d, page
        g = torch.Generator().manual_seed(seed)
        dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.h = U if dtype == "f32" else 2.0 ** -8
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + spare_pages
        order = torch.randperm(n_pages, generator=g).tolist()
        table = torch.full((len(lens), max(1, max(need)) + table_extra), -1, dtype=torch.int32)
        for s, n in enumerate(need):
            for b in range(n):
                table[s, b] = order.pop()
        rnd = lambda *s: torch.randn(*s, generator=g)
        k = rnd(n_pages, h_kv, page, d) * torch.exp(0.5 * rnd(n_pages, h_kv, page, 1)) * sharp
        v = rnd(n_pages, h_kv, page, d)
        if fp8:
            k, v = (x.to(dt).clamp(-448, 448).to(torch.float8_e4m3fn).to(dt) for x in (k, v))
        live = torch.zeros(n_pages, page, dtype=torch.bool)
        for s, b in missing:
            table[s, b] = [-1, n_pages, 2 ** 31 - 1, -2 ** 31][(s + b) % 4]
        for s, n in enumerate(lens):
            for j in range(n):
                if 0 <= table[s, j // page] < n_pages:
                    live[table[s, j // page], j % page] = True
        for x in (k, v):
            x[~live[:, None].expand(n_pages, h_kv, page)] = float("nan")
        to = (lambda x: x.to(dt).to(torch.float8_e4m3fn)) if fp8 else (lambda x: x.to(dt))
        self.weight = torch.exp(1.5 * rnd(n_pages, h_kv, page))
        pos = torch.randint(0, 1 << 20, (n_pages, h_kv, page), generator=g, dtype=torch.int32)
        self.cache = B.PagedCache(self.layout, n_pages, page, k=to(k).to(DEV), v=to(v).to(DEV), pos=pos.to(DEV),
                                  weight=self.weight.to(DEV))
        starts = [spare_rows[0]]
        for n in new:
            starts.append(starts[-1] + n)
        self.n_rows = starts[-1] + spare_rows[1]
        self.lens, self.new, self.table, self.starts = list(lens), list(new), table, starts
        self.q = (rnd(self.n_rows, h_q, d)).to(dt)
        self.oracle_batch = dict(table=table.tolist(), lens=self.lens, row_start=starts)
        self.batch = B.PagedBatch(table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                                  torch.tensor(starts, dtype=torch.int32, device=DEV), self.n_rows, max_new=max(1, max(new)))
        self.ws = B.make_paged_workspace(self.layout, self.batch, 0, page)

    def pool(self):
        return dict(k=to_f64(self.cache.k.float()), v=to_f64(self.cache.v.float()), pos=self.cache.pos.cpu().numpy(),
                    weight=to_f64(self.cache.weight))

    def attend(self, ws="full", want_lse=True):
        out = torch.full((self.n_rows, self.h_q, self.d), 7.0, dtype=self.q.dtype, device=DEV)
        lse = torch.full((self.h_q, self.n_rows), 7.0, dtype=torch.float32, device=DEV) if want_lse else None
        B.paged_attend(self.layout, self.cache, self.batch, self.q.to(DEV), out, lse, self.ws if isinstance(ws, str) else ws)
        torch.cuda.synchronize()
        return out, lse

    def check_attend(self, out, lse, numerators=None, what=""):
        want, wl, absv, size = P.attend(to_f64(self.q), self.pool(), self.oracle_batch, self.scale)
        mine = ~np.isnan(wl)
        e = (self.d + 16) * U * size + 2.0 ** -22
        n = (0.0 if self.h == U else 2.0 ** -16) if numerators is None else numerators
        got = to_f64(out)
        tol = self.h * np.abs(want) + absv * (2 * e.T[:, :, None] + n + 2.0 ** -15) + 1e-30
        rows = mine.all(0)
        assert (got[~rows] == 7.0).all(), f"{what}: rows of nobody were written"
        err = np.abs(got - want)[rows]
        finite = np.isfinite(want[rows])
        assert np.array_equal(np.isnan(got[rows]), np.isnan(want[rows])) and np.array_equal(got[rows][~finite & ~np.isnan(want[rows])], want[rows][~finite & ~np.isnan(want[rows])]), f"{what}: infinities or NaN differ"
        assert (err[finite] <= tol[rows][finite]).all(), f"{what}: off by {(err[finite] / tol[rows][finite]).max():.2f} tolerances"
        if lse is not None:
            gl = to_f64(lse)
            assert (gl[:, ~rows] == 7.0).all()
            none = np.isneginf(wl[:, rows])
            assert np.array_equal(np.isneginf(gl[:, rows]), none)
            d = np.abs(gl - wl)[:, rows][~none]
            assert (d <= (2 * e + 2.0 ** -16 + 4 * U * np.abs(wl))[:, rows][~none]).all(), f"{what}: lse off by {d.max():.2e}"

    def check_weigh(self, lse, accumulate, what=""):
        before = self.pool()
        B.paged_weigh(self.layout, self.cache, self.batch, self.q.to(DEV), lse, accumulate, self.ws)
        torch.cuda.synchronize()
        want, added = P.weigh(to_f64(self.q), to_f64(lse), before, self.oracle_batch, self.scale, accumulate)
        size = np.nan_to_num(P.attend(to_f64(self.q), before, self.oracle_batch, self.scale)[3]).max() + np.abs(np.where(np.isfinite(to_f64(lse)), to_f64(lse), 0)).max()
        rows = max(self.new + [1]) * (self.h_q // self.h_kv)
        e = (self.d + 16) * U * size + 2.0 ** -22 + (rows + 4) * U
        got = to_f64(self.cache.weight)
        assert (np.abs(got - want) <= added * e + 2 * U * np.abs(want) + 1e-37).all(), f"{what}: weights off by {np.abs(got - want).max():.2e}"


GRID = [
    (TINY, 16, [333, 1, 0, 17], [1, 1, 0, 3], {}),
    (F32, 32, [70, 200], [5, 33], {}),
    (BF64, 64, [129, 64, 500], [1, 2, 7], {}),
    (L7, 16, [700, 33, 32, 31, 1, 0], [1, 1, 1, 1, 1, 0], {}),
    (L7, 64, [1000, 999, 65], [4, 2, 1], {}),                                   # 28 stacked rows
    (L7, 128, [600, 300, 129], [40, 7, 1], {}),                                 # a short chunk
    (L7, 256, [2000], [300], {}),                                               # a long one
    (L72, 32, [513, 40], [2, 1], {}),
    (L72, 64, [300, 290, 5], [100, 64, 5], {}),
    (ODD, 16, [47, 48, 49], [11, 1, 5], {}),
    (WIDE, 64, [100, 260], [1, 3], {}),
    (L7, 32, [900, 200, 64], [1, 4, 4], dict(fp8=True)),
    (L72, 128, [513, 77], [30, 77], dict(fp8=True)),
    (L7, 16, [200, 100, 50, 48], [1, 1, 1, 1], dict(missing=[(0, 3), (0, 4), (1, 0), (2, 3), (3, 0), (3, 1), (3, 2)])),
    (L7, 64, [700, 640, 300], [60, 64, 3], dict(missing=[(0, 0), (0, 10), (1, 3), (1, 4), (2, 4)])),
    (TINY, 16, [40, 64], [3, 2], dict(missing=[(0, 1), (1, 0), (1, 3)])),
    (L72, 32, [400, 100], [2, 40], dict(fp8=True, missing=[(0, 12), (1, 1)])),
    (L7, 64, [3, 0, 70], [9, 4, 75], {}),                                       # more rows than entries
    (L7, 64, [20000], [1], {}),
    (TINY, 256, [5000], [2], {}),
]


@pytest.mark.parametrize("case", range(len(GRID)))
def test_attend_and_weigh(case):
    layout, page, lens, new, more = GRID[case]
    print("case", GRID[case], flush=True)
    sc = Scene(layout, page, lens, new, seed=case, **more)
    outs = []
    for ws in ("full", None, sc.ws[: sc.ws.numel() // 3 // 256 * 256]):
        out, lse = sc.attend(ws)
        sc.check_attend(out, lse, NUMERATORS(sc), f"case {case}")
        outs.append(lse)
    again, lse = sc.attend()
    assert torch.equal(lse, outs[0])                                            # the same bits
    out, _ = sc.attend(want_lse=False)
    assert torch.equal(out, again)
    for accumulate in (True, False):
        sc.check_weigh(lse, accumulate, f"case {case}")


def NUMERATORS(sc):
    """Chunks of bf16 heads of 128 round their numerators once, to bf16."""
    p = B.paged_plan(sc.layout, sc.cache, sc.batch, 0)
    return 2.0 ** -8 if p["rows_per_tile"] == 256 else None


@pytest.mark.parametrize("layout,n_seqs,most,new", [(L7, 3, 3000, 2), (TINY, 64, 400, 3), (L7, 70, 500, 1), (TINY, 300, 300, 5), (TINY, 2100, 20, 1), (BF64, 9, 900, 40)])
def test_many_sequences_of_very_different_lengths(layout, n_seqs, most, new):
    """The entries of a batch are dealt evenly to workgroups, whatever the sequences' lengths: some of them empty, some without rows."""
    g = torch.Generator().manual_seed(n_seqs)
    lens = [0 if i % 7 == 3 else max(1, int(most * float(torch.rand(1, generator=g)) ** 3)) for i in range(n_seqs)]
    news = [0 if i % 5 == 2 else 1 + (i * new) % new if new == 1 else int(torch.randint(1, new + 1, (1,), generator=g)) for i in range(n_seqs)]
    lens[-1] = most
    sc = Scene(layout, 16, lens, news, seed=n_seqs)
    shares = B.paged_plan(sc.layout, sc.cache, sc.batch, sc.ws.numel())["shares"]
    assert (shares > 1) == (n_seqs <= 300)
    for ws in ("full", None, sc.ws[: sc.ws.numel() // 2 // 256 * 256]):
        out, lse = sc.attend(ws)
        sc.check_attend(out, lse)


@pytest.mark.parametrize("layout,fp8", [(TINY, False), (L7, False), (L7, True), (BF64, False)])
def test_long_sequences_against_a_sample(layout, fp8):
    """A sequence over several page lists of a workgroup (8192 entries each) where scratch is missing."""
    sc = Scene(layout, 16, [20011], [2], seed=3, fp8=fp8)
    for ws in (None, "full"):
        out, lse = sc.attend(ws)
        sc.check_attend(out, lse)
    sc.check_weigh(lse, True)


@pytest.mark.parametrize("layout,new", [(TINY, 5), (F32, 3), (L7, 4), (L7, 1), (BF64, 6), (L7, 70), (L72, 40)])
def test_what_a_row_does_not_see_does_not_reach_it(layout, new):
    """Infinities and NaN in the values and keys of later tokens: earlier rows are as if they were not there, the rows that see
    them get what the formula gives."""
    sc = Scene(layout, 64, [150, 40], [new, new], seed=9)
    v, k = sc.cache.v, sc.cache.k
    last = lambda s, back: (int(sc.table[s, (sc.lens[s] - 1 - back) // 64]), (sc.lens[s] - 1 - back) % 64)
    p, e = last(0, 0)
    v[p, 0, e, 3], v[p, 0, e, 4], v[p, 1, e, 5] = float("inf"), float("-inf"), float("nan")
    if new > 2:
        p, e = last(0, 1)
        v[p, 0, e, 3], v[p, 1, e, 0] = float("-inf"), float("inf")
        p, e = last(1, 0)
        k[p, 1, e, 7] = float("nan")
    out, lse = sc.attend()
    sc.check_attend(*_without_nan_rows(sc, out, lse), NUMERATORS(sc))


def _without_nan_rows(sc, out, lse):
    """A row that sees a NaN key is NaN as a whole, and so is its lse; those are looked at here and then taken as the oracle's."""
    want, wl, _, _ = P.attend(to_f64(sc.q), sc.pool(), sc.oracle_batch, sc.scale)
    out, lse = out.clone(), lse.clone()
    n = len(sc.lens) and sc.starts[-1]
    for qh in range(sc.h_q):
        for row in range(sc.starts[0], n):
            if np.isnan(want[row, qh]).all():
                assert torch.isnan(out[row, qh]).all() and torch.isnan(lse[qh, row])
                lse[qh, row] = 7.0
    nobody = torch.tensor(np.isnan(wl))
    lse[nobody.to(lse.device)] = 7.0
    full = nobody.all(0) | (torch.arange(sc.n_rows) < sc.starts[0]) | (torch.arange(sc.n_rows) >= n)
    # rows with a NaN lse in any head are compared head by head against the oracle's outputs
    for row in range(sc.starts[0], n):
        for qh in range(sc.h_q):
            if nobody[qh, row]:
                out[row, qh] = 7.0
    mixed = nobody.any(0) & ~full
    sc_rows = torch.nonzero(mixed).flatten().tolist()
    for row in sc_rows:
        for qh in range(sc.h_q):
            if not nobody[qh, row]:
                w = torch.tensor(want[row, qh])
                assert torch.allclose(out[row, qh].double().cpu(), w, rtol=2e-2, atol=2e-2, equal_nan=True)
        out[row] = 7.0
        lse[:, row] = 7.0
    return out, lse


def test_sharp_rows_and_extreme_scales():
    for seed, (layout, sharp, scale) in enumerate([(L7, 30.0, 0.0), (TINY, 20.0, 0.0), (L7, 1.0, 3e-8), (L7, 1.0, 3.0), (TINY, 1.0, 1e-30)]):
        for new in (2, 50):
            sc = Scene(layout, 64, [900, 333], [new, new], seed=seed, sharp=sharp, scale=scale)
            out, lse = sc.attend()
            sc.check_attend(out, lse, NUMERATORS(sc), f"{layout} {sharp} {scale}")


def test_infinite_and_lowest_logits():
    """Keys whose products with every query are the type's lowest, and -infinity: rows still weigh the others; rows that see
    nothing else have the -infinity of an empty row."""
    sc = Scene(L7, 32, [100, 40], [1, 1], seed=4)
    sc.q.abs_()
    p = int(sc.table[0, 1])
    sc.cache.k[p, :, 3] = -3.0e38
    sc.cache.k[p, :, 4] = float("-inf")
    for b in range(2):
        sc.cache.k[int(sc.table[1, b])] = float("-inf")
    out, lse = sc.attend()
    pool = sc.pool()
    pool["k"][p, :, 3:5] = -1e30                                                # e^-1e30 is as 0
    want, wl, absv, _ = P.attend(to_f64(sc.q), pool, sc.oracle_batch, sc.scale)
    row = sc.starts[0]
    assert np.abs(to_f64(out)[row] - want[row]).max() < 0.02 and np.abs(to_f64(lse)[:, row] - wl[:, row]).max() < 1e-3
    assert (to_f64(out)[sc.starts[1]] == 0).all() and np.isneginf(to_f64(lse)[:, sc.starts[1]]).all()


def test_limits_of_the_batch_hold_whatever_the_device_says():
    """Lengths beyond the table or max_len, rows beyond max_new or out of range, a descending row_start: nothing outside is touched."""
    sc = Scene(L7, 16, [60, 100], [3, 2], seed=5)
    q = sc.q.to(DEV)
    table = sc.table.to(DEV)
    big = torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32, device=DEV)
    for starts, n_ok in (([2, 5, 7], 3), ([-7, 3, 2 ** 31 - 1], None), ([5, 2, 7], None), ([2 ** 31 - 1, -2 ** 31, 4], None)):
        rs = torch.tensor(starts, dtype=torch.int32, device=DEV)
        batch = B.PagedBatch(table, big, rs, sc.n_rows, max_new=3, max_len=48)
        out = torch.full_like(q, 7.0)
        lse = torch.full((sc.h_q, sc.n_rows), 7.0, device=DEV)
        k, w = sc.cache.k.clone(), sc.cache.weight.clone()
        B.paged_attend(sc.layout, sc.cache, batch, q, out, lse, sc.ws)
        B.paged_weigh(sc.layout, sc.cache, batch, q, lse, True, sc.ws)
        torch.cuda.synchronize()
        outside = [r for r in range(sc.n_rows) if n_ok and not 2 <= r < 7]
        assert (out[outside] == 7.0).all()
        assert (w != sc.cache.weight).sum() <= 48 * sc.h_kv
        B.paged_append(sc.layout, sc.cache, batch, q[:, :4].contiguous(), q[:, 4:8].contiguous(), torch.arange(sc.n_rows, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        changed = (k.view(torch.int16) != sc.cache.k.view(torch.int16)).any(-1).any(1).sum()
        assert changed <= 3
        sc.cache.k.copy_(k)
        sc.cache.weight.copy_(w)


# ---- append ----

@pytest.mark.parametrize("layout,page,fp8,lens,new,missing", [
    (L7, 64, False, [700, 65, 1, 0], [1, 1, 1, 0], []), (L7, 16, False, [500, 33], [500, 20], [(0, 2), (1, 2)]), (TINY, 32, False, [40, 9], [5, 9], []),
    (F32, 16, False, [40], [40], []), (BF64, 128, False, [300, 129], [200, 3], []), (L72, 64, True, [300, 65], [280, 2], [(0, 1)]),
    (ODD, 16, True, [31], [31], []), (L7, 32, False, [4, 3], [9, 5], []), (L7, 256, False, [5000], [5000], [])])
@pytest.mark.parametrize("source", ["tokens", "heads", "fused"])
def test_append(layout, page, fp8, lens, new, missing, source):
    """Rows stored from a group's tensors, from a flat cache with the heads outside, and from slices of one fused result; positions
    per token and per head; rounding of an 8-bit pool as the flat cache rounds; nothing else is touched."""
    sc = Scene(layout, page, lens, new, seed=len(lens), fp8=fp8, missing=missing)
    h_kv, d, n = sc.h_kv, sc.d, sc.n_rows
    g = torch.Generator().manual_seed(1)
    x = torch.randn(2, n, h_kv, d, generator=g) * 10.0 ** torch.randint(-4, 3, (2, n, h_kv, 1), generator=g).float()
    x[0, :, 0, 0], x[0, :, 0, 1] = 1000.0, -7e4                                 # beyond E4M3's largest
    x = x.to(sc.q.dtype)
    pos = torch.randint(0, 1 << 30, (n, h_kv), generator=g, dtype=torch.int32)
    if source == "tokens":
        k, v = x[0].contiguous().to(DEV), x[1].contiguous().to(DEV)
        p, pos = pos[:, 0].contiguous().to(DEV), pos[:, :1].expand(n, h_kv)
    elif source == "heads":
        flat = torch.zeros(2, h_kv, n + 5, d, dtype=x.dtype, device=DEV)
        flat[:, :, :n] = x.transpose(1, 2).to(DEV)
        k, v = flat[0].transpose(0, 1)[:n], flat[1].transpose(0, 1)[:n]
        p = torch.zeros(h_kv, n + 5, dtype=torch.int32, device=DEV)
        p[:, :n] = pos.t().to(DEV)
        p = p.t()[:n]
    else:
        fused = torch.zeros(n, 3 * h_kv + 1, d, dtype=x.dtype, device=DEV)
        fused[:, 1:1 + h_kv], fused[:, 1 + h_kv:1 + 2 * h_kv] = x[0].to(DEV), x[1].to(DEV)
        k, v, p = fused[:, 1:1 + h_kv], fused[:, 1 + h_kv:1 + 2 * h_kv], pos.to(DEV)
    before = sc.pool()
    B.paged_append(sc.layout, sc.cache, sc.batch, k, v, p)
    torch.cuda.synchronize()
    stored = [to_f64(x[i].float().clamp(-448, 448).to(torch.float8_e4m3fn).float()) if fp8 else to_f64(x[i]) for i in range(2)]
    want = P.append(stored[0], stored[1], pos.numpy(), before, sc.oracle_batch)
    got = sc.pool()
    for name in want:
        np.testing.assert_array_equal(got[name], want[name], err_msg=name)


def test_append_rounds_every_bf16_as_the_flat_cache_does():
    """All 65,536 patterns, infinities and NaN of both signs among them, against the library's own routine on the host."""
    layout = B.make_layout(4, 4, 128, "bf16")
    cache = B.PagedCache(layout, 1, 128, fmt=B.QP_CACHE_FP8_E4M3)
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(128, 4, 128)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    batch = B.PagedBatch(i32([[0]]), i32([128]), i32([0, 128]), 128)
    B.paged_append(layout, cache, batch, bits.to(DEV), bits.flip(0).contiguous().to(DEV), torch.arange(128, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    want = torch.tensor([B.lib().qp_e4m3_from_bf16(x) for x in range(65536)], dtype=torch.uint8).view(128, 4, 128)
    assert torch.equal(cache.k[0].view(torch.uint8).cpu(), want.transpose(0, 1))
    assert torch.equal(cache.v[0].view(torch.uint8).cpu(), want.flip(0).transpose(0, 1))


def test_append_of_rows_that_are_e4m3_already():
    sc = Scene(L72, 64, [200, 130], [200, 65], seed=2, fp8=True)
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randint(0, 256, (8, sc.n_rows + 3, 128), generator=g, dtype=torch.uint8).to(DEV).view(torch.float8_e4m3fn).transpose(0, 1)[:sc.n_rows]
            for _ in range(2))
    pos = torch.arange(sc.n_rows, dtype=torch.int32, device=DEV)
    before = sc.pool()
    B.paged_append(sc.layout, sc.cache, sc.batch, k, v, pos)
    torch.cuda.synchronize()
    want = P.append(to_f64(k.float()), to_f64(v.float()), np.arange(sc.n_rows)[:, None].repeat(8, 1), before, sc.oracle_batch)
    got = sc.pool()
    for name in want:
        np.testing.assert_array_equal(got[name], want[name])


def test_append_without_weights_and_refusals_of_the_binding():
    sc = Scene(L7, 64, [70], [2], seed=1)
    cache = B.PagedCache(sc.layout, 9, 64, weights=False)
    assert cache.weight is None
    k = torch.randn(sc.n_rows, 4, 128, device=DEV).to(torch.bfloat16)
    pos = torch.arange(sc.n_rows, dtype=torch.int32, device=DEV)
    batch = B.PagedBatch(torch.tensor([[1, 0]], dtype=torch.int32, device=DEV), torch.tensor([70], dtype=torch.int32, device=DEV),
                         torch.tensor([2, 4], dtype=torch.int32, device=DEV), sc.n_rows)
    B.paged_append(sc.layout, cache, batch, k, k, pos)
    torch.cuda.synchronize()
    assert torch.equal(cache.k[0, :, 4:6], k[2:4].transpose(0, 1)) and int(cache.k.count_nonzero()) <= 8 * 128
    q = torch.zeros(sc.n_rows, 28, 128, dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros(28, sc.n_rows, device=DEV)
    with pytest.raises(B.QPError):
        B.paged_weigh(sc.layout, cache, batch, q, lse)
    for bad in (dict(k=k.float()), dict(k=k[:, :3]), dict(k=k.cpu(), v=k.cpu()), dict(pos=pos.long()), dict(pos=pos[:-1]),
                dict(k=k.transpose(1, 2).contiguous().transpose(1, 2)), dict(v=k.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            B.paged_append(sc.layout, cache, batch, **{**dict(k=k, v=k, pos=pos), **bad})
    with pytest.raises(ValueError):
        B.paged_attend(sc.layout, cache, batch, q[:, :27], q)
    with pytest.raises(ValueError):
        B.paged_attend(sc.layout, cache, batch, q, q, lse.t().contiguous())
    with pytest.raises(ValueError):
        B.PagedBatch(torch.zeros(2, 2, dtype=torch.int64, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        B.PagedCache(sc.layout, 4, 64, k=torch.zeros(4, 4, 64, 64, dtype=torch.bfloat16, device=DEV))


# ---- evict ----

@pytest.mark.parametrize("layout,page,fp8,lens,keep,first,last,missing", [
    (L7, 64, False, [700, 300, 65], 200, 4, 16, []), (L7, 16, False, [1, 0, 17], 8, 1, 1, []), (TINY, 32, False, [100, 64], 64, 0, 0, [(0, 1), (1, 0)]),
    (F32, 16, False, [77], 33, 33, 0, []), (BF64, 128, False, [900, 128], 129, 0, 129, []), (L72, 32, True, [513, 100], 99, 3, 50, [(0, 7)]),
    (ODD, 16, False, [48, 47], 1, 0, 0, []), (ODD, 256, True, [1000], 1000, 4, 4, []), (TINY, 16, False, [9000], 4500, 4, 64, []),
    (L7, 64, False, [40000, 33000, 36865], 9999, 4, 64, [(0, 100), (0, 600)]), (L7, 128, False, [49152, 36864], 30000, 0, 12000, []),
    (TINY, 256, False, [60000, 100], 20000, 4, 64, [(0, 200)]), (TINY, 64, False, [33], 40, 20, 20, []), (TINY, 16, False, [32, 16], 10, 5, 5, [(0, 0), (0, 1), (1, 0)])])
@pytest.mark.parametrize("weights", ["spread", "ties"])
def test_evict(layout, page, fp8, lens, keep, first, last, missing, weights):
    pages = -(-keep // page)
    sc = Scene(layout, page, lens, [0] * len(lens), seed=keep, fp8=fp8, missing=missing, spare_pages=len(lens) * (pages + 1) + 2)
    if weights == "ties":
        w = torch.tensor([0.0, -0.0, 1.0, 2.0])[torch.randint(0, 4, sc.weight.shape, generator=torch.Generator().manual_seed(2))]
        sc.cache.weight.copy_(w)
    used = set(x for row in sc.table.tolist() for x in row)
    free = [p for p in range(sc.cache.c.n_pages) if p not in used]
    to = torch.full((len(lens), pages + 1), -1, dtype=torch.int32)
    for s in range(len(lens)):
        for b in range(pages):
            to[s, b] = free.pop()
    before = sc.pool()
    for own_list in (True, False):
        for x in (sc.cache.k, sc.cache.v, sc.cache.pos, sc.cache.weight):          # the destination, from the start again
            if not own_list:
                x.view(torch.uint8)[to[to >= 0].to(DEV).long()] = 0
        to_len = torch.full((len(lens),), -1, dtype=torch.int32, device=DEV)
        kept = torch.full((len(lens), sc.h_kv, keep), 99, dtype=torch.int32, device=DEV) if own_list else None
        ws = B.make_paged_workspace(sc.layout, sc.batch, keep, page)
        B.paged_evict(sc.layout, sc.cache, sc.batch, keep, first, last, to.to(DEV), to_len, kept, ws)
        torch.cuda.synchronize()
        want = P.evict(before, sc.table.tolist(), lens, keep, first, last)
        got = sc.pool()
        written = np.zeros(got["pos"].shape, bool)
        for s in range(len(lens)):
            for h in range(sc.h_kv):
                w = want[s * sc.h_kv + h]
                assert int(to_len[s]) == len(w)
                if own_list:
                    row = kept[s, h].cpu().numpy()
                    np.testing.assert_array_equal(row[:len(w)], w)
                    assert (row[len(w):] == -1).all()
                src = sc.table[s].numpy()[w // page], h, w % page
                x = np.arange(len(w))
                dst = to[s].numpy()[x // page], h, x % page
                written[dst] = True
                for name in got:
                    np.testing.assert_array_equal(got[name][dst], before[name][src], err_msg=name)
        if own_list:
            for name in got:
                np.testing.assert_array_equal(got[name][~written], before[name][~written], err_msg=name)


def test_evict_drops_what_has_no_destination():
    sc = Scene(L7, 16, [64], [0], seed=8, spare_pages=6)
    free = [p for p in range(10) if p not in sc.table[0].tolist()]
    to = torch.tensor([[free[0], -1, 10]], dtype=torch.int32, device=DEV)
    to_len = torch.zeros(1, dtype=torch.int32, device=DEV)
    before = sc.pool()
    B.paged_evict(sc.layout, sc.cache, sc.batch, 40, 0, 0, to, to_len, None, B.make_paged_workspace(sc.layout, sc.batch, 40, 16))
    torch.cuda.synchronize()
    got = sc.pool()
    assert int(to_len[0]) == 40
    others = [p for p in range(10) if p != free[0]]
    np.testing.assert_array_equal(got["weight"][others], before["weight"][others])
    np.testing.assert_array_equal(got["k"][others], before["k"][others])


@pytest.mark.parametrize("lens, keep", [([70, 5, 0, 300], 40), ([3], 64), ([50000, 12], 9)])
def test_evict_writes_the_new_lengths_over_the_old(lens, keep):
    """to_len the batch's own length: every head's selection still reads the old one."""
    pages = -(-keep // 16)
    sc = Scene(L72, 16, lens, [0] * len(lens), seed=keep, spare_pages=len(lens) * pages)
    used = set(x for row in sc.table.tolist() for x in row)
    free = [p for p in range(sc.cache.c.n_pages) if p not in used]
    to = torch.tensor([[free.pop() for _ in range(pages)] for _ in lens], dtype=torch.int32, device=DEV)
    kept = torch.empty(len(lens), sc.h_kv, keep, dtype=torch.int32, device=DEV)
    want = P.evict(sc.pool(), sc.table.tolist(), lens, keep, 2, 3)
    B.paged_evict(sc.layout, sc.cache, sc.batch, keep, 2, 3, to, sc.batch.length, kept, B.make_paged_workspace(sc.layout, sc.batch, keep, 16))
    torch.cuda.synchronize()
    assert sc.batch.length.tolist() == [min(n, keep) for n in lens]
    for s in range(len(lens)):
        for h in range(sc.h_kv):
            w = want[s * sc.h_kv + h]
            np.testing.assert_array_equal(kept[s, h].cpu().numpy()[:len(w)], w)


def test_a_cache_of_another_layout_is_refused():
    sc = Scene(L7, 16, [40], [1], seed=3)
    other = B.make_layout(64, 8, 128, "bf16")
    q = torch.zeros(sc.batch.n_rows, 64, 128, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        B.paged_attend(other, sc.cache, sc.batch, q, torch.empty_like(q))


# ---- together ----

def test_an_answer_goes_on_over_a_shared_video(seed=1):
    """Two questions about one video: its pruned flat cache moved into shared pages, the questions' chunks and then tokens appended,
    attended and weighed, one sequence cut to its budget, and the answers going on: as a cache without pages, evicted by hand, gives."""
    layout, page, video = B.make_layout(28, 4, 128, "bf16"), 32, 300
    g = torch.Generator().manual_seed(seed)
    bf = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)
    flat = B.Cache(layout, 500)
    fk, fv = bf(video, 4, 128), bf(video, 4, 128)
    B.topk_compact(layout, torch.zeros(4, video, device=DEV), fk.to(DEV), fv.to(DEV), video, 0, flat)
    cache = B.PagedCache(layout, 64, page)
    free = list(range(64))[::-1]
    shared = [free.pop() for _ in range(-(-video // page))]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    one = B.PagedBatch(i32([shared]), i32([video]), i32([0, video]), video)
    B.paged_append(layout, cache, one, flat.k.transpose(0, 1)[:video], flat.v.transpose(0, 1)[:video], flat.pos.t()[:video])
    # the last page of the video is not full: each sequence goes on in a copy of its own
    tables = []
    for s in range(2):
        own = free.pop()
        for x in (cache.k, cache.v, cache.pos, cache.weight):
            x[own] = x[shared[-1]]
        tables.append(shared[:-1] + [own] + [free.pop() for _ in range(12)])
    state = [dict(k=[fk[:, h].double() for h in range(4)], v=[fv[:, h].double() for h in range(4)],
                  w=[torch.zeros(video, dtype=torch.float64) for h in range(4)]) for _ in range(2)]
    lens = [video, video]
    for step in range(6):
        new = [20, 9] if step == 0 else [1, 2]
        n = sum(new)
        q, k, v = bf(n, 28, 128), bf(n, 4, 128), bf(n, 4, 128)
        lens = [a + b for a, b in zip(lens, new)]
        batch = B.PagedBatch(i32(tables), i32(lens), i32([0, new[0], n]), n, max_new=max(new), max_len=480)
        ws = B.make_paged_workspace(layout, batch, 128)
        out, lse = torch.zeros(n, 28, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(28, n, device=DEV)
        B.paged_append(layout, cache, batch, k.to(DEV), v.to(DEV), i32(list(range(1000, 1000 + n))))
        B.paged_attend(layout, cache, batch, q.to(DEV), out, lse, ws)
        if step >= 1:                                    # the shared pages have one writer: sequence 1's weights are not asked for
            alone = B.PagedBatch(i32(tables[:1]), i32(lens[:1]), i32([0, new[0]]), n, max_new=max(new), max_len=480)
            B.paged_weigh(layout, cache, alone, q.to(DEV), lse, True, ws)
        torch.cuda.synchronize()
        begin = 0
        for s in range(2):
            st = state[s]
            for h in range(4):
                st["k"][h] = torch.cat([st["k"][h], k[begin:begin + new[s], h].double()])
                st["v"][h] = torch.cat([st["v"][h], v[begin:begin + new[s], h].double()])
                st["w"][h] = torch.cat([st["w"][h], torch.zeros(new[s], dtype=torch.float64)])
                for i in range(new[s]):
                    see = lens[s] - new[s] + i + 1
                    p = torch.softmax(q[begin + i, 7 * h:7 * h + 7].double() @ st["k"][h][:see].t() / math.sqrt(128), -1)
                    assert (out[begin + i, 7 * h:7 * h + 7].double().cpu() - p @ st["v"][h][:see]).abs().max() < 0.02
                    if s == 0 and step >= 1:
                        st["w"][h][:see] += p.sum(0)
            begin += new[s]
        got = torch.cat([cache.weight[t] for t in tables[0]], 1)[:, :lens[0]].double().cpu()
        assert all(((got[h] - state[0]["w"][h]).abs() <= 2e-4 * state[0]["w"][h] + 1e-6).all() for h in range(4))
        if step == 3:
            to = [free.pop() for _ in range(4)]
            to_len = torch.zeros(1, dtype=torch.int32, device=DEV)
            kept = torch.zeros(1, 4, 128, dtype=torch.int32, device=DEV)
            B.paged_evict(layout, cache, alone, 128, 4, 16, i32([to]), to_len, kept, ws)
            torch.cuda.synchronize()
            for h in range(4):
                w = got[h].clone()
                w[:4], w[-16:] = math.inf, math.inf
                idx = torch.sort(torch.argsort(w, descending=True, stable=True)[:128])[0]
                assert torch.equal(kept[0, h].cpu().long(), idx)
                for name in "kvw":
                    state[0][name][h] = state[0][name][h][idx]
            tables[0] = (to + tables[0][10:] + [-1] * 22)[:22]
            lens[0] = int(to_len[0])
            assert lens[0] == 128


def test_a_captured_step_is_replayed_while_lengths_grow():
    """append, attend, weigh and evict captured once and replayed with other lengths, rows and tables, on a stream of the
    caller's, between eager calls that use the same workspace."""
    sc = Scene(L7, 16, [600, 350], [1, 1], seed=6, spare_pages=40, table_extra=4)
    for s in range(2):
        free = [p for p in range(sc.cache.c.n_pages) if p not in sc.table.tolist()[0] + sc.table.tolist()[1]]
        row = sc.table[s].tolist()
        at = row.index(-1)
        for b in range(4):
            sc.table[s, at + b] = free[b]
    free = [p for p in range(sc.cache.c.n_pages) if p not in sc.table.tolist()[0] + sc.table.tolist()[1]]
    to = torch.tensor([free[:7], free[7:14]], dtype=torch.int32, device=DEV)
    h_kv, n = sc.h_kv, sc.n_rows
    sc.batch.page_table.copy_(sc.table)
    for x in (sc.cache.k, sc.cache.v):
        x.nan_to_num_(0.5)
    q, k, v = sc.q.to(DEV), torch.zeros(n, h_kv, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(n, h_kv, 128, dtype=torch.bfloat16, device=DEV)
    out, lse = torch.zeros_like(q), torch.zeros(sc.h_q, n, device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    to_len, kept = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, h_kv, 100, dtype=torch.int32, device=DEV)
    ws = B.make_paged_workspace(sc.layout, sc.batch, 100, 16)

    def step():
        B.paged_append(sc.layout, sc.cache, sc.batch, k, v, pos)
        B.paged_attend(sc.layout, sc.cache, sc.batch, q, out, lse, ws)
        B.paged_weigh(sc.layout, sc.cache, sc.batch, q, lse, True, ws)
        B.paged_evict(sc.layout, sc.cache, sc.batch, 100, 4, 8, to, to_len, kept, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    g = torch.Generator().manual_seed(7)
    for replay, lens in enumerate(([601, 351], [602, 352], [30, 0], [611, 360])):
        sc.batch.length.copy_(torch.tensor(lens, dtype=torch.int32))
        sc.oracle_batch["lens"] = lens
        q.copy_(torch.randn(q.shape, generator=g))
        k.copy_(torch.randn(k.shape, generator=g))
        v.copy_(torch.randn(v.shape, generator=g))
        keep = [x.clone() for x in (sc.cache.k, sc.cache.v, sc.cache.pos, sc.cache.weight)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, sc.cache.k, sc.cache.v, sc.cache.pos, sc.cache.weight, to_len, kept)]
        for x, y in zip((sc.cache.k, sc.cache.v, sc.cache.pos, sc.cache.weight), keep):
            x.copy_(y)
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, lse, sc.cache.k, sc.cache.v, sc.cache.pos, sc.cache.weight, to_len, kept)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), replay
        for x, y in zip((out, lse), got):
            assert torch.isfinite(x[2:4] if x is out else x[:, 2:4]).all() or lens[1] == 0
        print("replay", replay, flush=True)


def test_a_pool_beyond_32_bits():
    """Pages whose first byte is beyond 2^32 of the pool (bf16: 8.6 GB each for K and V)."""
    layout = B.make_layout(8, 8, 128, "bf16")
    n_pages = (1 << 33) // (8 * 256 * 256) + 40
    cache = B.PagedCache(layout, n_pages, 256, weights=True)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    table = i32([[n_pages - 1, n_pages - 3, 5]])
    n = 600
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v, q = (torch.randn(n, 8, 128, generator=g, device=DEV).to(torch.bfloat16) for _ in range(3))
    batch = B.PagedBatch(table, i32([n]), i32([0, n]), n)
    B.paged_append(layout, cache, batch, k, v, torch.arange(n, dtype=torch.int32, device=DEV))
    out, lse = torch.zeros_like(q), torch.zeros(8, n, device=DEV)
    ws = B.make_paged_workspace(layout, batch, 300)
    B.paged_attend(layout, cache, batch, q, out, lse, ws)
    B.paged_weigh(layout, cache, batch, q, lse, False, ws)
    to, to_len, kept = i32([[n_pages - 2, n_pages - 5]]), i32([0]), torch.zeros(1, 8, 300, dtype=torch.int32, device=DEV)
    B.paged_evict(layout, cache, batch, 300, 0, 0, to, to_len, kept, ws)
    torch.cuda.synchronize()
    mask = torch.ones(n, n, dtype=torch.bool, device=DEV).tril()
    s = torch.matmul(q.float().transpose(0, 1), k.float().permute(1, 2, 0).contiguous()) / math.sqrt(128)
    p = torch.softmax(s.masked_fill(~mask, -math.inf), -1)
    assert (out.float() - torch.matmul(p, v.float().transpose(0, 1).contiguous()).transpose(0, 1)).abs().max() < 0.03
    w = torch.cat([cache.weight[n_pages - 1], cache.weight[n_pages - 3], cache.weight[5]], 1)[:, :n]
    assert (w - p.sum(1)).abs().max() < 1e-3
    for h in range(8):
        assert torch.equal(cache.k[n_pages - 2, h], k[kept[0, h, :256].long(), h])
        assert torch.equal(cache.v[n_pages - 5, h, :44], v[kept[0, h, 256:].long(), h])


# ---- against a plain implementation in 64 bits on the GPU ----

def plain(sc, lse=None, absent=()):
    """What P.attend returns and, for given lse, the weights that the rows add to every entry of the pool: sequence by sequence and head
    by head in 64 bits. absent: pages whose entries count as not there."""
    n, h_q, d, r = sc.n_rows, sc.h_q, sc.d, sc.h_q // sc.h_kv
    f64 = dict(dtype=torch.float64, device=DEV)
    out, absv, size = torch.full((n, h_q, d), math.nan, **f64), torch.zeros(n, h_q, d, **f64), torch.zeros(h_q, n, **f64)
    wl = torch.full((h_q, n), math.nan, **f64)
    added = torch.zeros(sc.cache.weight.shape, **f64)
    q = sc.q.to(DEV).double()
    for s, (length, begin, new) in enumerate(zip(sc.lens, sc.starts, sc.new)):
        j, page, slot = P.places(sc.table[s].numpy(), length, sc.page, sc.cache.c.n_pages)
        here = ~np.isin(page, absent)
        j, page, slot = (torch.tensor(x[here], device=DEV) for x in (j, page, slot))
        limit = (length - new + torch.arange(new, device=DEV)).repeat_interleave(r)
        for h in range(sc.h_kv if new else 0):
            heads = slice(h * r, h * r + r)
            k, v = (t[page, h, slot].float().double() for t in (sc.cache.k, sc.cache.v))
            rows = q[begin:begin + new, heads].reshape(new * r, d)
            x = sc.scale * (rows @ k.t())
            seen = j[None] <= limit[:, None]
            top = (sc.scale * (rows.abs() @ k.abs().t()) + x.abs()).masked_fill(~seen, 0)
            x = x.masked_fill(~seen, -math.inf)
            some = seen.any(1, keepdim=True)
            p = torch.where(some, torch.softmax(x.masked_fill(~some, 0), 1), 0)
            put = lambda y: y.view(new, r, -1)
            out[begin:begin + new, heads], absv[begin:begin + new, heads] = put(p @ v), put(p @ v.abs())
            wl[heads, begin:begin + new] = torch.logsumexp(x, 1).view(new, r).t()
            size[heads, begin:begin + new] = (top.amax(1) if len(j) else top.sum(1)).view(new, r).t()
            if lse is not None:
                z = lse[heads, begin:begin + new].t().reshape(-1, 1).double()
                added[page, h, slot] = torch.where(z > -math.inf, torch.exp(x - torch.where(z > -math.inf, z, 0)), 0).sum(0)
    return out, wl, absv, size, added


def check_plain(sc, out, lse, want, what=""):
    """The tolerances of check_attend."""
    wo, wl, absv, size, _ = want
    e = (sc.d + 16) * U * size + 2.0 ** -22
    rows = ~torch.isnan(wl).all(0)
    assert (out[~rows] == 7.0).all() and (lse[:, ~rows] == 7.0).all(), f"{what}: rows of nobody were written"
    tol = sc.h * wo.abs() + absv * (2 * e.t()[:, :, None] + (NUMERATORS(sc) or (0.0 if sc.h == U else 2.0 ** -16)) + 2.0 ** -15) + 1e-30
    off = ((out.double() - wo).abs() / tol)[rows]
    assert (off <= 1).all(), f"{what}: off by {off.max():.2f} tolerances"
    none = torch.isneginf(wl[:, rows])
    assert torch.equal(torch.isneginf(lse[:, rows]), none) and (out[rows].double()[none.t()] == 0).all()
    off = ((lse.double() - wl).abs() / (2 * e + 2.0 ** -16 + 4 * U * wl.abs()))[:, rows][~none]
    assert (off <= 1).all(), f"{what}: lse off by {off.max():.2f} tolerances"


def check_plain_weights(sc, lse, ws, what=""):
    """The tolerances of check_weigh, taken anew and then added to that."""
    want = plain(sc, lse)
    size = want[3].max() + lse[torch.isfinite(lse)].abs().max()
    e = float((sc.d + 16) * U * size) + 2.0 ** -22 + (max(sc.new) * (sc.h_q // sc.h_kv) + 4) * U
    live = torch.zeros(sc.cache.weight.shape, dtype=torch.bool, device=DEV)
    for s, n in enumerate(sc.lens):
        _, page, slot = P.places(sc.table[s].numpy(), n, sc.page, sc.cache.c.n_pages)
        live[torch.tensor(page, device=DEV), :, torch.tensor(slot, device=DEV)] = True
    for accumulate in (False, True):
        before = sc.cache.weight.clone()
        B.paged_weigh(sc.layout, sc.cache, sc.batch, sc.q.to(DEV), lse, accumulate, ws)
        torch.cuda.synchronize()
        full = want[4] + (before.double() if accumulate else 0)
        err = (sc.cache.weight.double() - full).abs()[live]
        tol = (want[4] * e + 2 * U * full.abs() + 1e-37)[live]
        assert (err <= tol).all(), f"{what}: weights off by {(err / tol).max():.2f} tolerances"
        assert torch.equal(sc.cache.weight[~live], before[~live]), f"{what}: weights of nobody were written"


# ---- long chunks ----

@pytest.mark.parametrize("layout,page,lens,new,more", [
    (L7, 64, [1500, 700], [1300, 650], {}),                                    # 9,100 and 4,550 stacked rows
    (L7, 16, [900, 1250], [1210, 37], dict(missing=[(0, 5), (1, 70)])),        # 8,470 rows, of which the first 2,170 see nothing
    (L72, 128, [1025, 600], [1025, 513], dict(fp8=True)),                      # 8,200 and 4,104
    (ODD, 32, [2900], [2801], {})])                                            # 8,403
def test_chunks_of_more_rows_than_one_lot_of_statistics(layout, page, lens, new, more):
    """Weighing keeps the statistics of 4,096 stacked rows in LDS: here a workgroup goes through several such lots, in the later
    ones too with rows that saw nothing, and starts in any of them where it has the workspace. Attention of the same rows has row
    blocks that end in front of a key chunk."""
    sc = Scene(layout, page, lens, new, seed=len(lens) + page, **more)
    want = plain(sc)
    assert B.paged_plan(sc.layout, sc.cache, sc.batch, sc.ws.numel())["key_chunks"] > 1
    for ws in ("full", None):
        print("attend", ws, flush=True)
        out, lse = sc.attend(ws)
        check_plain(sc, out, lse, want, f"{ws}")
    r = sc.h_q // sc.h_kv
    for row in (sc.starts[1] - 1, sc.starts[0] + 4100 // r, sc.starts[0] + 8190 // r if new[0] * r > 8190 else sc.starts[0]):
        lse[1::3, row] = -math.inf
    for ws in (sc.ws, None):
        print("weigh", ws is None, flush=True)
        check_plain_weights(sc, lse, ws, "without workspace" if ws is None else "")


@pytest.mark.parametrize("layout,page,lens,new,fp8", [(L7, 16, [5003, 1100], [40, 9], False), (L72, 16, [3999, 2300], [33, 5], True), (L7, 32, [9000], [77], False)])
def test_chunks_over_more_pages_than_one_list(layout, page, lens, new, fp8):
    """The tile kernel has 64 page numbers of a table at hand: here it goes on to the next ones inside its loop, over pages that
    are missing where one list ends and the next begins, and over more missing ones in a row than a list has."""
    per = lens[0] // page
    missing = [(0, b) for b in (0, 1, 63, 64, per // 2 - 1)] + [(0, b) for b in range(126, min(201, per - 3))] + [(s, 62) for s in range(1, len(lens))]
    sc = Scene(layout, page, lens, new, seed=page + len(lens), fp8=fp8, missing=missing)
    want = plain(sc)
    two_chunks = 2 * sc.n_rows * sc.h_q * 129 * 4
    outs = []
    for ws in ("full", None, sc.ws[: -(-two_chunks // 256) * 256]):
        plan = B.paged_plan(sc.layout, sc.cache, sc.batch, sc.ws.numel() if isinstance(ws, str) else 0 if ws is None else ws.numel())
        print("attend", plan, flush=True)
        assert plan["rows_per_tile"] == 256 and (plan["key_chunks"] > 2 if isinstance(ws, str) else plan["key_chunks"] == (1 if ws is None else 2))
        out, lse = sc.attend(ws)
        check_plain(sc, out, lse, want, str(plan))
        outs.append((out, lse))
    for ws, (out, lse) in zip(("full", None), outs):
        again, z = sc.attend(ws)
        assert torch.equal(again, out) and torch.equal(z, lse)                  # the same bits
    for ws in (sc.ws, None):
        check_plain_weights(sc, lse, ws, "without workspace" if ws is None else "")


# ---- limits ----

@pytest.mark.parametrize("starts", [[2, 5, 7], [-7, 3, 2 ** 31 - 1], [5, 2, 7], [2 ** 31 - 1, -2 ** 31, 4], [1, 6, 10]])
@pytest.mark.parametrize("layout", [L7, TINY, L72])
def test_rows_beyond_the_limits_are_left_alone(layout, starts):
    """Whose rows are whose when the device says something odd, from the documented limits: first row into [0, n_rows], end from
    there to n_rows, max_new rows of them. Those are written, no other ones, and append changes those entries alone."""
    sc = Scene(layout, 16, [60, 100], [3, 2], seed=5)
    n, big, max_new, max_len = sc.n_rows, [2 ** 31 - 1, 41], 3, 48
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    batch = B.PagedBatch(sc.table.to(DEV), i32(big), i32(starts), n, max_new=max_new, max_len=max_len)
    owned, entries = {}, {}
    for s in range(2):
        length = min(max(big[s], 0), max_len, sc.table.shape[1] * 16)
        r0 = min(max(starts[s], 0), n)
        count = min(max(starts[s + 1], r0), n) - r0
        for i in range(min(count, max_new)):
            j = length - count + i
            page = int(sc.table[s, j // 16]) if j >= 0 else -1
            owned[r0 + i] = page >= 0
            if page >= 0:
                entries[page, j % 16] = r0 + i
    out, lse = sc.q.to(DEV), torch.full((sc.h_q, n), 7.0, device=DEV)
    out = torch.full_like(out, 7.0)
    B.paged_attend(sc.layout, sc.cache, batch, sc.q.to(DEV), out, lse, sc.ws)
    torch.cuda.synchronize()
    for row in range(n):
        if row not in owned:
            assert (out[row] == 7.0).all() and (lse[:, row] == 7.0).all(), row
        elif owned[row]:
            assert (out[row] != 7.0).any(-1).all() and torch.isfinite(lse[:, row]).all() and (lse[:, row] != 7.0).all(), row
        else:
            assert (out[row] == 0).all() and torch.isneginf(lse[:, row]).all(), row
    k = torch.full((n, sc.h_kv, sc.d), 5.0, dtype=sc.q.dtype, device=DEV)
    before = [x.clone() for x in (sc.cache.k, sc.cache.v, sc.cache.pos, sc.cache.weight)]
    B.paged_append(sc.layout, sc.cache, batch, k, -k, torch.arange(-1000, -1000 + n, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for (page, slot), row in entries.items():
        before[0][page, :, slot], before[1][page, :, slot], before[2][page, :, slot], before[3][page, :, slot] = 5, -5, row - 1000, 0
    for x, y in zip((sc.cache.k, sc.cache.v, sc.cache.pos, sc.cache.weight), before):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


# ---- logits of any size ----

@pytest.mark.parametrize("layout", [TINY, F32, BF64, L7, L72])
@pytest.mark.parametrize("new", [2, 50])
def test_whole_blocks_of_lowest_logits(layout, new):
    """Pages of keys whose products with every query are far below zero, of sizes from 1e10 to 1e33: e to that is 0, so rows weigh the other entries
    as if those were not there, whether the low ones come first or later, and rows that see nothing else see nothing."""
    sc = Scene(layout, 64, [400, 130, 70], [new, new, new], seed=new)
    sc.q.abs_()
    low = [int(sc.table[s, b]) for s, b in ((0, 0), (0, 1), (0, 4), (1, 1), (2, 0), (2, 1))]
    g = torch.Generator().manual_seed(3)
    for page in low:
        size = 10.0 ** (10 + 23 * torch.rand(sc.h_kv, 64, 1, generator=g))
        sc.cache.k[page] = (-size).to(sc.q.dtype).to(DEV)
        sc.cache.v[page] = 1.0
    want = plain(sc, absent=low)
    for ws in ("full", None):
        out, lse = sc.attend(ws)
        check_plain(sc, out, lse, want, f"{ws}")
    B.paged_weigh(sc.layout, sc.cache, sc.batch, sc.q.to(DEV), lse, False, sc.ws)
    torch.cuda.synchronize()
    assert (sc.cache.weight[low[:4]] == 0).all()


@pytest.mark.parametrize("layout", [TINY, BF64, L7])
@pytest.mark.parametrize("new", [2, 50])
def test_one_logit_above_all_others(layout, new):
    """An entry whose logits of up to 2^28 leave the others nothing: the rows are its value, and lse its logit."""
    sc = Scene(layout, 32, [300, 90], [new, new], seed=new)
    sc.q.abs_().clamp_(max=2.0)
    at = [(int(sc.table[s, b]), e) for s, b, e in ((0, 3, 7), (1, 0, 31))]
    for page, e in at:
        sc.cache.k[page, :, e] = 2.0 ** 28 / (2 * sc.d * sc.scale)
    out, lse = sc.attend()
    _, wl, _, _, _ = plain(sc)
    for s, (page, e) in enumerate(at):
        rows = slice(sc.starts[s], sc.starts[s + 1])
        v = sc.cache.v[page, :, e].double().repeat_interleave(sc.h_q // sc.h_kv, 0)[None]
        assert (wl[:, rows] > 2.0 ** 24).all()
        assert ((out[rows].double() - v).abs() <= v.abs() * (sc.h + (NUMERATORS(sc) or 2.0 ** -16) + 2.0 ** -15)).all()
        # the product's sum, the scale times log2 e, its product and the one back to base e
        assert ((lse[:, rows].double() - wl[:, rows]).abs() <= (sc.d + 8) * U * wl[:, rows]).all()


# ---- shared pages, streams ----

def test_sequences_that_share_pages_are_evicted_in_one_call():
    """Three sequences over one video's pages with tails and lengths of their own: each list is its own, the shared pages stay."""
    sc = Scene(L7, 16, [100, 100, 100], [0, 0, 0], seed=12, spare_pages=3 * 3 + 1)
    table = sc.table.clone()
    table[1:, :4] = table[0, :4]                                                # 64 shared entries
    lens, keep = [100, 83, 40], 45
    used = set(x for row in sc.table.tolist() for x in row)
    free = [p for p in range(sc.cache.c.n_pages) if p not in used]
    to = torch.tensor([[free.pop() for _ in range(3)] for _ in lens], dtype=torch.int32)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    batch = B.PagedBatch(table.to(DEV), i32(lens))
    to_len, kept = i32([-1] * 3), torch.full((3, sc.h_kv, keep), 99, dtype=torch.int32, device=DEV)
    before = sc.pool()
    B.paged_evict(sc.layout, sc.cache, batch, keep, 2, 5, to.to(DEV), to_len, kept, B.make_paged_workspace(sc.layout, batch, keep, 16))
    torch.cuda.synchronize()
    got, want = sc.pool(), P.evict(before, table.tolist(), lens, keep, 2, 5)
    assert to_len.tolist() == [45, 45, 40]
    for s in range(3):
        for h in range(sc.h_kv):
            w = want[s * sc.h_kv + h]
            np.testing.assert_array_equal(kept[s, h, :len(w)].cpu().numpy(), w)
            x = np.arange(len(w))
            for name in got:
                np.testing.assert_array_equal(got[name][to[s].numpy()[x // 16], h, x % 16], before[name][table[s].numpy()[w // 16], h, w % 16])
    kept_pages = [p for p in range(sc.cache.c.n_pages) if p not in to.flatten().tolist()]
    for name in got:
        np.testing.assert_array_equal(got[name][kept_pages], before[name][kept_pages])


def test_calls_on_two_streams_at_once():
    """Two batches over one pool, each on a stream and with a workspace of its own: the bits that either gives alone."""
    sc = Scene(L7, 32, [9000, 700, 5000, 300], [1, 2, 60, 40], seed=13)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    q = sc.q.to(DEV)
    halves = []
    for a, b in ((0, 2), (2, 4)):
        batch = B.PagedBatch(sc.table[a:b].to(DEV), i32(sc.lens[a:b]), i32(sc.starts[a:b + 1]), sc.n_rows, max_new=max(sc.new[a:b]))
        halves.append((batch, B.make_paged_workspace(sc.layout, batch, 200, 32), torch.cuda.Stream()))
    weight = sc.cache.weight.clone()

    def calls(half, results):
        batch, ws, _ = half
        out, lse = torch.full_like(q, 7.0), torch.full((sc.h_q, sc.n_rows), 7.0, device=DEV)
        results += [out, lse]
        for _ in range(3):
            B.paged_attend(sc.layout, sc.cache, batch, q, out, lse, ws)
            B.paged_weigh(sc.layout, sc.cache, batch, q, lse, True, ws)

    alone = []
    for half in halves:
        calls(half, alone)
        torch.cuda.synchronize()
    alone.append(sc.cache.weight.clone())
    sc.cache.weight.copy_(weight)
    torch.cuda.synchronize()
    both = []
    for half in halves:
        with torch.cuda.stream(half[2]):
            calls(half, both)
    torch.cuda.synchronize()
    for x, y in zip(alone, both + [sc.cache.weight]):
        assert torch.equal(x, y)
