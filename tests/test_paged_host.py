"""The paged cache without a GPU: its oracle on hand cases, the arithmetic behind its kernels' bounds, refusals, sizes."""
import ctypes
import os
import subprocess
import types

import numpy as np
import pytest
import torch

from conftest import ROOT
from oracle import paged_oracle as P
from paper_2505_16175_amd import binding as B
from paper_2505_16175_amd import build as qp_build

FAKE = 1 << 20


def test_device_values_are_brought_into_the_batchs_limits(tmp_path):
    exe = str(tmp_path / "paged_host")
    built = subprocess.run(["hipcc", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                            "-packed-fp32-ops", "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I",
                            qp_build.CSRC, "-x", "hip", os.path.join(ROOT, "tests", "paged_host.cpp"), "-o", exe],
                           capture_output=True, text=True)
    assert built.returncode == 0, built.stderr[-2000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0 and "ALL OK" in run.stdout, run.stdout


def _call(**change):
    """A valid call of every entry point over made-up addresses, with some of its values changed: the statuses."""
    L = B.make_layout(8, 2, change.pop("d", 128), change.pop("dtype", "bf16"), change.pop("scale", 0.0))
    v = dict(k=FAKE, v=FAKE, pos=FAKE, weight=FAKE, n_pages=8, page_tokens=64, format=0, table=FAKE, len=FAKE, row_start=FAKE,
             n_seqs=2, table_pages=4, n_rows=6, max_new=4, max_len=200, q=FAKE, out=FAKE, lse=FAKE, ws=FAKE, wb=1 << 40,
             token_stride=256, head_stride=128, pos_stride=1, source=0, keep=50, first=4, last=4, to=FAKE, to_pages=4, to_len=FAKE,
             kept=None)
    assert set(change) <= set(v)
    v.update(change)
    c = B.qp_paged_cache(v["k"], v["v"], v["pos"], v["weight"], v["n_pages"], v["page_tokens"], v["format"])
    b = B.qp_paged_batch(v["table"], v["len"], v["row_start"], v["n_seqs"], v["table_pages"], v["n_rows"], v["max_new"], v["max_len"])
    L, c, b, lib = ctypes.byref(L), ctypes.byref(c), ctypes.byref(b), B.lib()
    return dict(append=lib.qp_paged_append(L, c, b, v["q"], v["out"], v["token_stride"], v["head_stride"], v["pos"],
                                           v["pos_stride"], 0, v["source"], None),
                attend=lib.qp_paged_attend(L, c, b, v["q"], v["out"], v["lse"], v["ws"], v["wb"], None),
                weigh=lib.qp_paged_weigh(L, c, b, v["q"], v["lse"], 1, v["ws"], v["wb"], None),
                evict=lib.qp_paged_evict(L, c, b, v["keep"], v["first"], v["last"], v["to"], v["to_pages"], v["to_len"], v["kept"],
                                         v["ws"], v["wb"], None))


INV, UNS, CAP = B.QP_ERR_INVALID_ARG, B.QP_ERR_UNSUPPORTED, B.QP_ERR_CAPACITY
ALL = ("append", "attend", "weigh", "evict")
ROWS = ("append", "attend", "weigh")


@pytest.mark.parametrize("change,status,calls", [
    (dict(k=None), INV, ALL), (dict(v=FAKE + 8), INV, ALL), (dict(pos=FAKE + 2), INV, ALL), (dict(weight=FAKE + 4), INV, ALL),
    (dict(weight=None), INV, ("weigh", "evict")), (dict(n_pages=0), INV, ALL), (dict(page_tokens=0), INV, ALL),
    (dict(page_tokens=48), UNS, ALL), (dict(page_tokens=512), UNS, ALL), (dict(page_tokens=8), UNS, ALL),
    (dict(format=2), INV, ALL), (dict(format=1, dtype="f32"), UNS, ALL), (dict(format=1, d=64), UNS, ALL), (dict(d=96), UNS, ALL),
    (dict(scale=-1.0), INV, ALL), (dict(scale=float("inf")), INV, ALL), (dict(scale=float("nan")), INV, ALL),
    (dict(table=None), INV, ALL), (dict(table=FAKE + 2), INV, ALL), (dict(len=None), INV, ALL), (dict(row_start=None), INV, ROWS),
    (dict(n_seqs=0), INV, ALL), (dict(n_seqs=-1), INV, ALL), (dict(n_seqs=(1 << 20) + 1), UNS, ALL), (dict(table_pages=0), INV, ALL),
    (dict(n_rows=0), INV, ROWS), (dict(n_rows=-5), INV, ROWS), (dict(n_rows=(1 << 30) + 1), UNS, ROWS),
    (dict(max_new=0), INV, ROWS), (dict(max_new=-1), INV, ROWS), (dict(max_len=0), INV, ALL), (dict(max_len=(1 << 30) + 1), UNS, ALL),
    (dict(q=None), INV, ROWS), (dict(q=FAKE + 8), INV, ROWS), (dict(out=None), INV, ("append", "attend")),
    (dict(lse=None), INV, ("weigh",)), (dict(lse=FAKE + 2), INV, ("attend", "weigh")), (dict(ws=FAKE + 128), INV, ("attend", "weigh", "evict")),
    (dict(token_stride=-128), INV, ("append",)), (dict(token_stride=132), INV, ("append",)), (dict(head_stride=4), INV, ("append",)),
    (dict(pos_stride=-1), INV, ("append",)), (dict(source=3), INV, ("append",)), (dict(source=1), UNS, ("append",)),
    (dict(token_stride=1 << 50), UNS, ("append",)),
    (dict(keep=0), INV, ("evict",)), (dict(keep=7), INV, ("evict",)), (dict(first=-1), INV, ("evict",)), (dict(last=-1), INV, ("evict",)),
    (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), INV, ("evict",)), (dict(to=None), INV, ("evict",)), (dict(to_len=None), INV, ("evict",)),
    (dict(to_pages=0), INV, ("evict",)), (dict(kept=FAKE + 2), INV, ("evict",)), (dict(keep=257), CAP, ("evict",)),
    (dict(ws=None), CAP, ("evict",)), (dict(wb=100), CAP, ("evict",)),
    # more workgroups than one launch takes
    (dict(n_seqs=1 << 20, max_len=1 << 30, ws=None, max_new=1 << 30, n_rows=1 << 30), UNS, ROWS),
])
def test_refusals(change, status, calls):
    if torch.cuda.is_available():
        pytest.skip("calls that are not refused would run over made-up addresses")
    got = _call(**change)
    for name in calls:
        assert got[name] == status, (name, change)


def test_a_valid_call_reaches_the_launch():
    if torch.cuda.is_available():
        pytest.skip("would run over made-up addresses")
    assert set(_call().values()) == {B.QP_ERR_HIP}                # no GPU here: the launch itself fails, after all checks
    assert set(_call(format=1).values()) == {B.QP_ERR_HIP}
    assert _call(row_start=None, n_rows=0, max_new=0)["evict"] == B.QP_ERR_HIP


@pytest.mark.parametrize("layout", [(28, 4, 128, "bf16"), (64, 8, 128, "bf16"), (4, 2, 64, "f32"), (5, 1, 64, "bf16")])
def test_plans_cover_the_entries_and_fit_what_is_offered(layout):
    L = B.make_layout(*layout)
    for n_seqs in (1, 3, 64, 5000):
        for max_new in (1, 2, 4, 33, 700):
            for max_len in (1, 31, 257, 9840, 46125, 1 << 24):
                for n_rows in (n_seqs, n_seqs * max_new):
                    ws = B.paged_workspace_bytes(L, n_seqs, n_rows, max_new, max_len, 0)
                    assert 0 < ws <= (129 << 20)
                    c = B.qp_paged_cache(FAKE, FAKE, FAKE, None, 8, 64, 0)
                    b = B.qp_paged_batch(FAKE, FAKE, FAKE, n_seqs, 1 << 20, n_rows, max_new, max_len)
                    for offered in (0, 4096, ws // 3, ws, 1 << 40):
                        p = B.qp_paged_plan_info()
                        assert B.lib().qp_paged_plan(ctypes.byref(L), ctypes.byref(c), ctypes.byref(b), offered, ctypes.byref(p)) == B.QP_OK
                        assert p.key_chunks >= 1 and p.scratch_bytes <= min(offered, ws)
                        assert (p.key_chunks - 1) * p.chunk_entries < max_len <= p.key_chunks * p.chunk_entries
                        assert p.key_chunks == 1 or p.chunk_entries % 64 == 0
                        assert p.shares == 0 or p.rows_per_tile < 256 and p.key_chunks == 1 and p.workgroups == p.shares * layout[1]
                        assert (p.scratch_bytes > 0) == (p.shares > 0 or p.key_chunks > 1)
    assert B.lib().qp_paged_plan(ctypes.byref(L), ctypes.byref(c), ctypes.byref(b), 0, None) == INV
    assert B.paged_workspace_bytes(L, 0, 1, 1, 1) == 0 and B.paged_workspace_bytes(L, 1, 1, 1, 0) == 0
    assert B.paged_workspace_bytes(L, 1, 1, 1, 1, -1) == 0
    assert B.paged_workspace_bytes(L, 3, 0, 0, 60000, 1000) >= 4 * 3 * layout[1] * 60000 > B.paged_workspace_bytes(L, 3, 0, 0, 60000, 0)


class _Tensor:
    """What the binding looks at of a tensor on the GPU."""

    def __init__(self, *shape, dtype=torch.int32):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return FAKE


def test_a_batch_without_max_len_is_as_long_as_each_pools_pages_whoever_else_uses_it():
    """Two threads may use one batch over pools of different pages: what one call was handed does not change under it."""
    batch = B.PagedBatch(_Tensor(2, 5), _Tensor(2), _Tensor(3), n_rows=7)
    small, large = (types.SimpleNamespace(c=B.qp_paged_cache(page_tokens=p)) for p in (16, 128))
    read = lambda ref: ctypes.cast(ref, ctypes.POINTER(B.qp_paged_batch)).contents
    first = batch.of(small)
    second = batch.of(large)
    assert read(first).max_len == 80 and read(second).max_len == 640
    assert read(batch.of(small)).max_len == 80
    for b in (read(first), read(second)):
        assert (b.page_table, b.len, b.row_start, b.n_seqs, b.table_pages, b.n_rows, b.max_new) == (FAKE, FAKE, FAKE, 2, 5, 7, 7)
    stated = B.PagedBatch(_Tensor(2, 5), _Tensor(2), _Tensor(3), n_rows=7, max_new=3, max_len=33)
    assert read(stated.of(small)).max_len == read(stated.of(large)).max_len == 33 and read(stated.of(small)).max_new == 3
    huge = B.PagedBatch(_Tensor(1, 1 << 28), _Tensor(1))
    assert read(huge.of(large)).max_len == 1 << 30


# ---- the oracle, by hand ----

def _pool(entries, weight=None):
    """One head of one element per entry, in pages of 2."""
    n = len(entries)
    x = np.asarray(entries, float).reshape(n // 2, 1, 2, 1)
    w = np.zeros((n // 2, 1, 2)) if weight is None else np.asarray(weight, float).reshape(n // 2, 1, 2)
    return dict(k=x.copy(), v=x.copy(), pos=np.arange(n).reshape(n // 2, 1, 2), weight=w)


def test_oracle_attend_follows_the_table_the_causal_limit_and_missing_pages():
    pool = _pool([0, np.log(2), np.log(3), np.log(4), 9, 9])
    batch = dict(table=[[1, 0, -1], [0, 7, 2]], lens=[3, 0], row_start=[1, 3, 4])
    q = np.ones((5, 1, 1))
    out, lse, _, _ = P.attend(q, pool, batch, 1.0)
    # sequence 0: entries log 3, log 4, 0; its two rows are the last two
    np.testing.assert_allclose(lse[0, 1:3], [np.log(7), np.log(8)])
    np.testing.assert_allclose(out[2, 0], (3 * np.log(3) + 4 * np.log(4)) / 8)
    assert out[3, 0] == 0 and lse[0, 3] == -np.inf                  # an empty sequence's row
    assert np.isnan(out[[0, 4]]).all()                              # nobody's rows
    batch = dict(table=[[9, 2]], lens=[4], row_start=[0, 1])        # the first page is missing
    assert P.attend(q[:1], pool, batch, 1.0)[0][0, 0] == 9
    batch = dict(table=[[0]], lens=[1], row_start=[0, 3])           # more rows than entries: the first two see nothing
    out, lse, _, _ = P.attend(q[:3], pool, batch, 1.0)
    assert list(lse[0]) == [-np.inf, -np.inf, 0.0]


def test_oracle_weights_of_a_row_sum_to_one():
    pool = _pool([0.3, -1, 2, 0.5, 1, 1], [1] * 6)
    batch = dict(table=[[2, 0, 1]], lens=[5], row_start=[0, 2])
    q = np.array([[[0.7]], [[-0.2]]])
    lse = P.attend(q, pool, batch, 1.0)[1]
    w, added = P.weigh(q, lse, pool, batch, 1.0, True)
    np.testing.assert_allclose(added.sum(), 2)
    np.testing.assert_allclose(w - 1, added)
    assert added[1, 0, 1] == 0 and added[1, 0, 0] > 0               # past the end; the last entry, seen by the last row only


def test_oracle_evict_keeps_ends_large_weights_and_low_ties():
    pool = _pool([0] * 8, [1, 5, 2, 2, 2, 7, 0, 1])
    assert P.evict(pool, [[0, 1, 2, 3]], [8], 4, 1, 1)[0].tolist() == [0, 1, 5, 7]
    assert P.evict(pool, [[0, 1, 2, 3]], [8], 4, 0, 0)[0].tolist() == [1, 2, 3, 5]
    assert P.evict(pool, [[0, -1, 2, 3]], [8], 4, 0, 3)[0].tolist() == [1, 5, 6, 7]
    assert P.evict(pool, [[0, -1]], [4], 4, 1, 1)[0].tolist() == [0, 1]


def test_oracle_append_stores_the_last_rows_where_the_table_says():
    pool = _pool([0] * 6, [3] * 6)
    new = np.arange(1.0, 4.0).reshape(3, 1, 1)
    got = P.append(new, -new, np.array([[10], [11], [12]]), pool, dict(table=[[2, 0], [1, -1]], lens=[3, 4], row_start=[0, 2, 3]))
    assert got["k"].ravel().tolist() == [2, 0, 0, 0, 0, 1] and got["v"][0, 0, 0, 0] == -2
    assert got["pos"][2, 0, 1] == 10 and got["weight"].ravel().tolist() == [0, 3, 3, 3, 3, 0]
