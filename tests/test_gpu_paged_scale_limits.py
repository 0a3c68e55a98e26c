"""The ends of the scales' range over the paged cache (include/qp_paged.h), and windows within the limits that a batch states.

At a scale of 2^120 codes beyond 240 would stand for more than f32 and bf16 hold: appends saturate there, and such codes, where a
caller's pool has them, are infinities like those of a bf16 pool. Tolerances are those of test_gpu_paged.py and
test_gpu_paged_rope_window.py."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paper_2505_16175_amd import binding as B
from paper_2505_16175_amd.workload import to_f64
from test_gpu_paged import DEV, L7, L72, TINY, U, Scene, check_plain
from test_gpu_paged_rope_window import SCALED, SECTION, attend, i32, plain, scaled_pool

pytestmark = pytest.mark.gpu
TOP = 240 * 2.0 ** 120                                            # 1.875 * 2^127


def pool_of(sc):
    return dict(sc.pool(), k_scale=to_f64(sc.cache.k_scale), v_scale=to_f64(sc.cache.v_scale))


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("layout,lens,new", [(L7, [70, 16], [3, 16]), (L72, [100, 300], [37, 1])])
def test_the_largest_values_are_stored_finite(layout, lens, new, rope):
    """bf16's largest, some that just do and just do not fit, infinities and NaN, in blocks of their own and behind entries of ordinary size."""
    sc = scaled_pool(Scene(layout, 16, lens, new, seed=sum(lens)), seed=1, spread=2)
    g = torch.Generator().manual_seed(2)
    kv = torch.randn(2, sc.n_rows, sc.h_kv, sc.d, generator=g)
    kv[:, :, 0] *= 2.0 ** 126
    kv = kv.to(torch.bfloat16)
    most = torch.finfo(torch.bfloat16).max
    for c, x in enumerate((most, -most, 1.75 * 2.0 ** 127, 1.7578125 * 2.0 ** 127, -1.875 * 2.0 ** 127, 1.9375 * 2.0 ** 127, -1.9453125 * 2.0 ** 127,
                           float("inf"), float("-inf"), float("nan"))):
        kv[:, sc.starts[0]::2, 1, 3 * c] = x
        kv[:, sc.starts[0]::2, 1, 64 + 3 * c] = x if c % 2 else -x  # where both turn by 45 degrees the sum is sqrt(2) times as large
    k, v = kv.to(DEV)
    pos = torch.arange(sc.n_rows, dtype=torch.int32)
    before = pool_of(sc)
    axes = torch.randint(0, 1000, (3, sc.n_rows), generator=g, dtype=torch.int32)
    turned = to_f64(k)
    if rope:
        with np.errstate(invalid="ignore"):
            turned = P.turn(turned, axes.numpy(), 1e6, SECTION[128])
        B.paged_append_rope(sc.layout, sc.cache, sc.batch, k, v, pos.to(DEV), B.PagedRope(sc.layout, axes.to(DEV), 1e6, SECTION[128]))
    else:
        B.paged_append(sc.layout, sc.cache, sc.batch, k, v, pos.to(DEV))
    torch.cuda.synchronize()
    want = P.append_scaled(turned, to_f64(v), to_f64(k), pos[:, None].expand(-1, sc.h_kv).numpy(), before, sc.oracle_batch, 316.0 if rope else 448.0)
    got = pool_of(sc)
    live = torch.zeros(sc.cache.c.n_pages, 16, dtype=torch.bool)
    for s in range(len(lens)):
        j = torch.arange(lens[s])
        live[sc.table[s].long()[j // 16], j % 16] = True
    live = live[:, None].expand(-1, sc.h_kv, -1).numpy()
    for name in ("k", "v"):
        assert (want[name + "_scale"] == 2.0 ** 120).any()
        np.testing.assert_array_equal(got[name + "_scale"], want[name + "_scale"], err_msg=name)
        with np.errstate(invalid="ignore"):
            size = np.abs(P.dequantised(got)[name])[live]
        assert (size[~np.isnan(size)] <= TOP).all(), f"{name}: codes that stand for infinities"
        if name == "v" or not rope:
            np.testing.assert_array_equal(got[name], want[name], err_msg=name)
    if rope:                                                      # one code apart where a turned value lies next to the middle between two
        finite = np.isfinite(turned).all()
        assert not finite                                         # the planted ones
        new_here = np.zeros_like(live)
        for s in range(len(lens)):
            j = np.arange(lens[s] - new[s], lens[s])
            new_here[sc.table[s].numpy()[j // 16], :, j % 16] = True
        assert np.array_equal(np.isnan(got["k"][new_here]), np.isnan(want["k"][new_here]))
        off = np.abs(got["k"] - want["k"])[new_here]
        step = np.maximum(2.0 ** -3 * np.abs(want["k"][new_here]), 2.0 ** -9)
        assert (off[~np.isnan(off)] <= step[~np.isnan(off)]).all()


@pytest.mark.parametrize("made_by", ["append", "caller"])
@pytest.mark.parametrize("new,window", [(1, None), (4, None), (4, (40, 3)), (40, None), (40, (64, 5))])
def test_the_largest_values_do_not_reach_rows_that_do_not_see_them(new, window, made_by):
    """A sequence's last entry holds bf16's largest values, stored by an append, or codes of 448 at the largest scale, which are infinities:
    the rows before it are as if it was not there."""
    lens = [230, 97]                                              # last entries at 5 and 0 of their blocks: with others, and alone
    sc = scaled_pool(Scene(L7, 16, lens, [new, new], seed=new), seed=3, spread=0)
    huge = []
    for s, n in enumerate(lens):
        page, block = int(sc.table[s, (n - 1) // 16]), (n - 1) // 16 * 16
        for h in (0, 2):
            if made_by == "append":
                rows = torch.zeros(n - block, 1, 128, dtype=torch.bfloat16)
                rows[-1, 0, 3], rows[-1, 0, 70] = torch.finfo(torch.bfloat16).max, -torch.finfo(torch.bfloat16).max
                one = B.make_layout(1, 1, 128, "bf16")
                pool = B.PagedCache(one, 1, 16, fmt=SCALED)
                B.paged_append(one, pool, B.PagedBatch(i32([[0]]), i32([n - block]), i32([0, n - block]), n - block), rows.to(DEV), rows.to(DEV),
                               torch.zeros(n - block, dtype=torch.int32, device=DEV))
                torch.cuda.synchronize()
                assert pool.v_scale.item() == 2.0 ** 120
                sc.cache.v.view(torch.uint8)[page, h] = pool.v.view(torch.uint8)[0, 0]
            else:
                sc.cache.v.view(torch.uint8)[page, h] = 0
                sc.cache.v.view(torch.uint8)[page, h, (n - 1) % 16, 3], sc.cache.v.view(torch.uint8)[page, h, (n - 1) % 16, 70] = 0x7e, 0xfe
            sc.cache.v_scale[page, h] = 2.0 ** 120
            huge.append((s, h))
    want = plain(sc, *(window or (None,)))
    for ws in ("full", None):
        out, lse = attend(sc, *(window or (None,)), ws=ws)
        for s, h in huge:
            row, heads = sc.starts[s] + new - 1, slice(7 * h, 7 * h + 7)
            seen = out[row, heads][:, [3, 70]]
            if made_by == "caller":
                assert not torch.isfinite(seen).any()
            out[row, heads] = want[0][row, heads].to(out.dtype)   # the row that sees it: what a sum of them holds is not looked at here
        check_plain(sc, out, lse, want, f"{new} {window} {made_by}")


def test_a_row_that_sees_the_largest_value_has_it():
    """One entry and its row, one value in the middle of zeros: the softmax's only weight is 1."""
    L = B.make_layout(4, 2, 128, "bf16")
    for rows, n in ((1, 1), (20, 20)):                            # few rows, and a tile (40 stacked rows)
        cache = B.PagedCache(L, 4, 16, fmt=SCALED)
        batch = B.PagedBatch(i32([[2, 0]]), i32([n]), i32([0, rows]), rows)
        v = torch.zeros(rows, 2, 128, dtype=torch.bfloat16, device=DEV)
        v[0, :, 5], v[0, :, 6] = torch.finfo(torch.bfloat16).max, -1.75 * 2.0 ** 127
        q = torch.zeros(rows, 4, 128, dtype=torch.bfloat16, device=DEV)
        B.paged_append(L, cache, batch, torch.zeros_like(v), v, torch.zeros(rows, dtype=torch.int32, device=DEV))
        out = torch.zeros_like(q)
        B.paged_attend(L, cache, batch, q, out)
        torch.cuda.synchronize()
        assert (out[0, :, 5].double() == TOP).all() and (out[0, :, 6].double() == -1.75 * 2.0 ** 127).all() and (out[0, :, :5] == 0).all()
        count = torch.arange(1, rows + 1, device=DEV, dtype=torch.float64)[:, None]
        for c, x in ((5, TOP), (6, -1.75 * 2.0 ** 127)):          # the mean over the entries so far: the value over their number
            assert ((out[:, :, c].double() - x / count).abs() <= (2.0 ** -8 + 2.0 ** -14) * abs(x) / count).all()


@pytest.mark.parametrize("layout,lens,new", [(L7, [200, 90], 1), (L7, [200, 90], 4), (L7, [200, 90], 40), ((1030, 1030, 128, "bf16"), [50], 33)])
def test_weigh_with_small_scales_and_large_queries(layout, lens, new):
    """Codes' own products with such queries exceed what f32 holds; the keys' do not."""
    sc = Scene(layout, 16, lens, [new] * len(lens), seed=new, fp8=True)
    shape = (sc.cache.c.n_pages, sc.h_kv, 1)
    g = torch.Generator().manual_seed(7)
    sc.cache.k.copy_((sc.cache.k.float() * 100).clamp(-448, 448).to(torch.float8_e4m3fn))
    sc.cache = B.PagedCache(sc.layout, shape[0], 16, fmt=SCALED, k=sc.cache.k, v=sc.cache.v, pos=sc.cache.pos, weight=sc.cache.weight,
                            k_scale=torch.exp2(-117 + torch.randint(0, 2, shape, generator=g).float()).to(DEV), v_scale=torch.ones(shape, device=DEV))
    q = sc.q.float() * 2.0 ** 120
    q[:, :, ::2] *= 2.0 ** -12
    q[:, ::3] *= 2.0 ** -4                                        # logits of size 100 and 1,000
    sc.q = q.to(torch.bfloat16)
    codes = torch.nan_to_num(sc.cache.k.float()).abs().amax().item()
    assert float(sc.q.float().abs().max()) * codes > 2.0 ** 128
    values_pool = P.dequantised(pool_of(sc))
    _, wl, _, size = P.attend(to_f64(sc.q), values_pool, sc.oracle_batch, sc.scale)
    if layout is L7:
        _, lse = attend(sc)
        assert torch.isfinite(lse[:, sc.starts[0]:sc.starts[-1]]).all()
    else:                                                         # more heads than the tiles of weighing take
        lse = torch.tensor(np.nan_to_num(wl), dtype=torch.float32, device=DEV)
    tol = (sc.d + 16) * U * (np.nan_to_num(size).max() + np.abs(to_f64(lse)).max()) + 2.0 ** -22 + (new * sc.h_q // sc.h_kv + 4) * U
    for accumulate in (True, False):
        for ws in (sc.ws, None):
            before = dict(values_pool, weight=to_f64(sc.cache.weight))
            B.paged_weigh(sc.layout, sc.cache, sc.batch, sc.q.to(DEV), lse, accumulate, ws)
            torch.cuda.synchronize()
            want, added = P.weigh(to_f64(sc.q), to_f64(lse), before, sc.oracle_batch, sc.scale, accumulate)
            got = to_f64(sc.cache.weight)
            assert np.isfinite(got).all()
            assert (np.abs(got - want) <= added * np.expm1(tol) + 2 * U * np.abs(want) + 1e-37).all()


@pytest.mark.parametrize("layout,fmt", [(L7, "same"), (TINY, "same"), (L7, "scaled")])
def test_windowed_rows_within_the_limits_are_right(layout, fmt):
    """Lengths and rows that the device states wrongly: the rows that the batch's limits leave see the entries that they leave, and the others
    stay as they were."""
    sc = Scene(layout, 16, [60, 100], [3, 2], seed=5)
    if fmt == "scaled":
        scaled_pool(sc)
    q, r = sc.q.to(DEV), sc.h_q // sc.h_kv
    pool = pool_of(sc) if fmt == "scaled" else sc.pool()
    if fmt == "scaled":
        with np.errstate(invalid="ignore"):
            pool = P.dequantised(pool)
    q64 = to_f64(sc.q)
    for starts in ([2, 5, 7], [-7, 3, 2 ** 31 - 1], [5, 2, 7], [2 ** 31 - 1, -2 ** 31, 4]):
        for lens in ([2 ** 31 - 1, -5], [-2 ** 31, 47], [49, 48]):
            batch = B.PagedBatch(sc.table.to(DEV), i32(lens), i32(starts), sc.n_rows, max_new=3, max_len=48)
            for window, n_sink in ((5, 2), (2 ** 31 - 1, 0), (1, 2 ** 31 - 1), (20, 0)):
                for ws in (sc.ws, None):
                    out, lse = torch.full_like(q, 7.0), torch.full((sc.h_q, sc.n_rows), 7.0, device=DEV)
                    B.paged_attend_window(sc.layout, sc.cache, batch, window, n_sink, q, out, lse, ws)
                    torch.cuda.synchronize()
                    got, gl, owned = to_f64(out), to_f64(lse), set()
                    for s in range(2):
                        length = min(max(lens[s], 0), 48)
                        r0 = min(max(starts[s], 0), sc.n_rows)
                        count = min(max(starts[s + 1], r0), sc.n_rows) - r0
                        for i in range(min(count, 3)):
                            owned.add(r0 + i)
                            p = length - count + i
                            j = np.arange(max(p + 1, 0))
                            j = j[(j > p - window) | (j < n_sink)]
                            page, slot = sc.table[s].numpy()[j // 16], j % 16
                            for qh in range(sc.h_q):
                                if len(j) == 0:
                                    assert (got[r0 + i, qh] == 0).all() and np.isneginf(gl[qh, r0 + i])
                                    continue
                                k, v = pool["k"][page, qh // r, slot], pool["v"][page, qh // r, slot]
                                x = sc.scale * (k @ q64[r0 + i, qh])
                                w = np.exp(x - x.max())
                                z = x.max() + np.log(w.sum())
                                w /= w.sum()
                                size = sc.scale * (np.abs(k) @ np.abs(q64[r0 + i, qh])).max() + np.abs(x).max()
                                e = (sc.d + 16) * U * size + 2.0 ** -22
                                tol = sc.h * np.abs(w @ v) + (w @ np.abs(v)) * (2 * e + (0 if sc.h == U else 2.0 ** -16) + 2.0 ** -15) + 1e-30
                                assert (np.abs(got[r0 + i, qh] - w @ v) <= tol).all(), (starts, lens, window, r0 + i, qh)
                                assert abs(gl[qh, r0 + i] - z) <= 2 * e + 2.0 ** -16 + 4 * U * abs(z)
                    rest = [row for row in range(sc.n_rows) if row not in owned]
                    assert (got[rest] == 7.0).all() and (gl[:, rest] == 7.0).all()


def test_numbers_beyond_32_bits_are_refused():
    """Their lower bits alone would be a window, a count of first entries or a section of another size."""
    sc = Scene(TINY, 16, [60], [2], seed=1)
    q, out = sc.q.to(DEV), torch.full((sc.n_rows, sc.h_q, sc.d), 7.0, device=DEV)
    for window, n_sink in (((1 << 32) + 5, 2), (5, 1 << 32), (5 - (1 << 32), 0), (5, 1 << 31), (1 << 40, 0)):
        with pytest.raises(ValueError):
            B.paged_attend_window(sc.layout, sc.cache, sc.batch, window, n_sink, q, out)
    with pytest.raises(ValueError):
        B.PagedRope(sc.layout, torch.zeros(5, dtype=torch.int32, device=DEV), section=((1 << 32) + 8, 12, 12))
    assert (out == 7.0).all()
    B.paged_attend_window(sc.layout, sc.cache, sc.batch, 2 ** 31 - 1, 2 ** 31 - 1, q, out)
    assert not (out[sc.starts[0]:sc.starts[1]] == 7.0).any()


@pytest.mark.parametrize("layout,keep,more", [(L7, 75, 5), (L72, 33, 40), (L7, 16, 17)])
def test_an_evicted_cache_with_scales_goes_on(layout, keep, more):
    """Entries stored, attended, weighed and cut to a budget that ends inside a block, and the next tokens stored behind them: the block that
    the move began takes them, its scale grows from what the move gave it. Lengths stay on the device."""
    h_q, h_kv, d, _ = layout
    L, g, page, lens = B.make_layout(*layout), torch.Generator().manual_seed(keep), 32, [230, 41]
    cache = B.PagedCache(L, 30, page, fmt=SCALED)
    order = torch.randperm(30, generator=g)
    table, to = order[:16].view(2, 8).int(), order[16:].view(2, 7).int()
    made = lambda n, size: (size * torch.randn(n, h_kv, d, generator=g)).to(torch.bfloat16)
    pool = lambda: dict(k=to_f64(cache.k.float()), v=to_f64(cache.v.float()), pos=cache.pos.cpu().numpy(), weight=to_f64(cache.weight),
                        k_scale=to_f64(cache.k_scale), v_scale=to_f64(cache.v_scale))

    def append(t, length, lens, starts, size):
        n, before = starts[-1], pool()
        k, v, pos = made(n, size), made(n, 1 / size), torch.arange(n, dtype=torch.int32)
        B.paged_append(L, cache, B.PagedBatch(t.to(DEV), length, i32(starts), n), k.to(DEV), v.to(DEV), pos.to(DEV))
        torch.cuda.synchronize()
        want = P.append_scaled(to_f64(k), to_f64(v), to_f64(k), pos[:, None].expand(-1, h_kv).numpy(), before,
                               dict(table=t.tolist(), lens=lens, row_start=starts), 448.0)
        got = pool()
        for name in want:
            np.testing.assert_array_equal(got[name], want[name], err_msg=name)

    append(table, i32(lens), lens, [0, lens[0], sum(lens)], 1.0)
    length, rows = i32(lens), 2
    q = torch.randn(2 * rows, h_q, d, generator=g).to(torch.bfloat16).to(DEV)
    batch = B.PagedBatch(table.to(DEV), length, i32([0, rows, 2 * rows]), 2 * rows, max_new=rows)
    ws = B.make_paged_workspace(L, batch, keep, page)
    out, lse = torch.empty_like(q), torch.empty(h_q, 2 * rows, device=DEV)
    B.paged_attend(L, cache, batch, q, out, lse, ws)
    B.paged_weigh(L, cache, batch, q, lse, True, ws)
    torch.cuda.synchronize()
    before = pool()
    lists = P.evict(before, table.tolist(), lens, keep, 4, 8)
    lists = [lists[:h_kv], lists[h_kv:]]
    B.paged_evict(L, cache, batch, keep, 4, 8, to.to(DEV), length, None, ws)
    want = P.move_scaled(before, table.tolist(), lists, to.tolist())
    torch.cuda.synchronize()
    got = pool()
    for name in want:
        np.testing.assert_array_equal(got[name], want[name], err_msg=name)
    lens = [min(keep, n) for n in lens]
    assert length.tolist() == lens
    for size in (30.0, 1e-3):
        length.add_(more)
        lens = [n + more for n in lens]
        append(to, length, lens, [0, more, 2 * more], size)
    now = P.dequantised(pool())
    q = torch.randn(2 * more, h_q, d, generator=g).to(torch.bfloat16)
    batch = B.PagedBatch(to.to(DEV), length, i32([0, more, 2 * more]), 2 * more, max_new=more)
    numerators = 2.0 ** -8 if B.paged_plan(L, cache, batch, 0)["rows_per_tile"] == 256 else 2.0 ** -16
    for window, n_sink in ((1 << 20, 0), (20, 3)):
        out, lse = torch.empty(2 * more, h_q, d, dtype=torch.bfloat16, device=DEV), torch.empty(h_q, 2 * more, device=DEV)
        B.paged_attend_window(L, cache, batch, window, n_sink, q.to(DEV), out, lse, B.make_paged_workspace(L, batch, 0, page))
        torch.cuda.synchronize()
        want, wl, absv, size = P.attend(to_f64(q), now, dict(table=to.tolist(), lens=lens, row_start=[0, more, 2 * more]), 128 ** -0.5, window, n_sink)
        e = (d + 16) * U * size + 2.0 ** -22
        assert (np.abs(to_f64(out) - want) <= 2.0 ** -8 * np.abs(want) + absv * (2 * e.T[:, :, None] + numerators + 2.0 ** -15) + 1e-30).all()
        assert (np.abs(to_f64(lse) - wl) <= 2 * e + 2.0 ** -16 + 4 * U * np.abs(wl)).all()
