"""Rotated appends, pools with scales and windows over the paged cache without a GPU: the arithmetic of the windows, refusals, the oracle by hand."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from conftest import ROOT
from oracle import paged_oracle as P
from paper_2505_16175_amd import binding as B
from paper_2505_16175_amd import build as qp_build

FAKE = 1 << 20


def test_a_row_tile_meets_what_its_windows_see_and_little_more(tmp_path):
    exe = str(tmp_path / "paged_window_host")
    built = subprocess.run(["hipcc", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                            "-packed-fp32-ops", "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I",
                            qp_build.CSRC, "-x", "hip", os.path.join(ROOT, "tests", "paged_window_host.cpp"), "-o", exe],
                           capture_output=True, text=True)
    assert built.returncode == 0, built.stderr[-2000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0 and "ALL OK" in run.stdout, run.stdout


def _call(**change):
    """Valid calls over made-up addresses, with some of their values changed: the statuses."""
    L = B.make_layout(8, 2, change.pop("d", 128), change.pop("dtype", "bf16"))
    v = dict(k=FAKE, v=FAKE, pos=FAKE, weight=FAKE, n_pages=8, page_tokens=64, format=2, k_scale=FAKE, v_scale=FAKE, table=FAKE, len=FAKE,
             row_start=FAKE, n_seqs=2, table_pages=4, n_rows=6, max_new=4, max_len=200, q=FAKE, out=FAKE, lse=FAKE, ws=FAKE, wb=1 << 40,
             q_token_stride=1024, q_head_stride=128, token_stride=256, head_stride=128, new_pos=FAKE, pos_token_stride=1, pos_head_stride=0,
             source=0, axes=FAKE, axis_stride=6, theta=1e6, section=(16, 24, 24), rope=True, window=50, n_sink=4)
    assert set(change) <= set(v)
    v.update(change)
    c = B.qp_paged_cache(v["k"], v["v"], v["pos"], v["weight"], v["n_pages"], v["page_tokens"], v["format"], v["k_scale"], v["v_scale"])
    b = B.qp_paged_batch(v["table"], v["len"], v["row_start"], v["n_seqs"], v["table_pages"], v["n_rows"], v["max_new"], v["max_len"])
    r = B.qp_paged_rope(v["axes"], v["axis_stride"], v["theta"], (ctypes.c_int32 * 3)(*v["section"]))
    L, c, b, lib = ctypes.byref(L), ctypes.byref(c), ctypes.byref(b), B.lib()
    return dict(append=lib.qp_paged_append(L, c, b, v["q"], v["q"], v["token_stride"], v["head_stride"], v["new_pos"], v["pos_token_stride"],
                                           v["pos_head_stride"], v["source"], None),
                rope=lib.qp_paged_append_rope(L, c, b, ctypes.byref(r) if v["rope"] else None, v["q"], v["q_token_stride"], v["q_head_stride"], v["k"],
                                              v["v"], v["token_stride"], v["head_stride"], v["new_pos"], v["pos_token_stride"], v["pos_head_stride"],
                                              v["out"], None),
                attend=lib.qp_paged_attend(L, c, b, v["q"], v["out"], v["lse"], v["ws"], v["wb"], None),
                window=lib.qp_paged_attend_window(L, c, b, v["window"], v["n_sink"], v["q"], v["out"], v["lse"], v["ws"], v["wb"], None),
                weigh=lib.qp_paged_weigh(L, c, b, v["q"], v["lse"], 1, v["ws"], v["wb"], None),
                evict=lib.qp_paged_evict(L, c, b, 50, 4, 4, FAKE, 4, FAKE, None, v["ws"], v["wb"], None))


INV, UNS = B.QP_ERR_INVALID_ARG, B.QP_ERR_UNSUPPORTED
ALL = ("append", "rope", "attend", "window", "weigh", "evict")
NEW = ("append", "rope", "attend", "window")


@pytest.mark.parametrize("change,status,calls", [
    (dict(k_scale=None), INV, ALL), (dict(v_scale=None), INV, ALL), (dict(k_scale=FAKE + 2), INV, ALL), (dict(v_scale=FAKE + 1), INV, ALL),
    (dict(format=3), INV, ALL), (dict(format=-1), INV, ALL), (dict(dtype="f32"), UNS, ALL), (dict(d=64, section=(8, 12, 12)), UNS, ALL),
    (dict(source=1), UNS, ("append",)),
    (dict(page_tokens=8), UNS, NEW), (dict(n_rows=0), INV, NEW), (dict(max_new=0), INV, NEW), (dict(row_start=None), INV, NEW),
    (dict(len=None), INV, NEW), (dict(n_seqs=0), INV, NEW), (dict(max_len=(1 << 30) + 1), UNS, NEW),
    (dict(rope=False), INV, ("rope",)), (dict(axes=None), INV, ("rope",)), (dict(axes=FAKE + 2), INV, ("rope",)), (dict(axis_stride=-1), INV, ("rope",)),
    (dict(axis_stride=1 << 50), UNS, ("rope",)), (dict(theta=0.0), INV, ("rope",)), (dict(theta=-1e6), INV, ("rope",)),
    (dict(theta=float("nan")), INV, ("rope",)), (dict(theta=float("inf")), INV, ("rope",)), (dict(section=(16, 24, 23)), INV, ("rope",)),
    (dict(section=(-1, 41, 24)), INV, ("rope",)), (dict(section=(2 ** 31 - 1, 2 ** 31 - 1, 66)), INV, ("rope",)), (dict(section=(8, 12, 12)), INV, ("rope",)),
    (dict(q=None), INV, ("rope", "window")), (dict(out=None), INV, ("rope", "window")), (dict(q=FAKE + 8), INV, ("rope", "window")),
    (dict(out=FAKE + 8), INV, ("rope", "window")), (dict(new_pos=None), INV, ("append", "rope")), (dict(new_pos=FAKE + 2), INV, ("append", "rope")),
    (dict(k=None), INV, ("rope",)), (dict(v=FAKE + 8), INV, ("rope",)),
    (dict(token_stride=-128), INV, ("append", "rope")), (dict(token_stride=132), INV, ("append", "rope")), (dict(head_stride=4), INV, ("append", "rope")),
    (dict(head_stride=1 << 50), UNS, ("append", "rope")), (dict(q_token_stride=-8), INV, ("rope",)), (dict(q_token_stride=1 << 50), UNS, ("rope",)),
    (dict(q_head_stride=12), INV, ("rope",)), (dict(pos_token_stride=-1), INV, ("append", "rope")), (dict(pos_head_stride=1 << 50), UNS, ("append", "rope")),
    (dict(window=0), INV, ("window",)), (dict(window=-5), INV, ("window",)), (dict(n_sink=-1), INV, ("window",)), (dict(lse=FAKE + 2), INV, ("window",)),
    (dict(ws=FAKE + 128), INV, ("window",)),
    # more workgroups than one launch takes
    (dict(n_seqs=1 << 20, max_len=1 << 30, ws=None, max_new=1 << 30, n_rows=1 << 30), UNS, NEW),
])
def test_refusals(change, status, calls):
    if torch.cuda.is_available():
        pytest.skip("calls that are not refused would run over made-up addresses")
    got = _call(**change)
    for name in calls:
        assert got[name] == status, (name, change)


def test_valid_calls_reach_the_launch():
    if torch.cuda.is_available():
        pytest.skip("would run over made-up addresses")
    hip = B.QP_ERR_HIP                                            # no GPU here: the launch itself fails, after all checks
    for change in ({}, dict(format=0), dict(format=1), dict(format=0, dtype="f32"), dict(format=0, d=64, section=(8, 12, 12)),
                   dict(format=0, dtype="f32", d=64, section=(32, 0, 0), axis_stride=0), dict(window=2 ** 31 - 1, n_sink=2 ** 31 - 1), dict(weight=None),
                   dict(max_new=300, n_rows=900, n_seqs=3)):
        got = _call(**change)
        assert {got[name] for name in (NEW if change.get("weight", 1) is None else ALL)} == {hip}, change
    assert _call(q=None, out=None)["rope"] == hip                 # keys and values only
    assert _call(format=0, k_scale=None, v_scale=None)["attend"] == hip


def test_a_flat_cache_takes_no_scales():
    """QP_CACHE_FP8_E4M3_SCALED is a format of paged pools."""
    L = B.make_layout(8, 2, 128, "bf16")
    c = B.qp_cache(FAKE, FAKE, FAKE, 100, 10, 2)
    assert B.lib().qp_group_attend(ctypes.byref(L), FAKE, FAKE, FAKE, 4, ctypes.byref(c), FAKE, None, None, 0, None) == INV
    assert B.lib().qp_topk_compact(ctypes.byref(L), FAKE, FAKE, FAKE, 4, 2, 0, ctypes.byref(c), None, None, 0, None) == INV


# ---- the oracle, by hand ----

def test_oracle_windows():
    x = np.zeros((2, 1, 16, 1))
    pool = dict(k=x.copy(), v=np.arange(32.0).reshape(2, 1, 16, 1), pos=np.zeros((2, 1, 16), int), weight=np.zeros((2, 1, 16)))
    batch = dict(table=[[0, 1]], lens=[20], row_start=[0, 2])
    q = np.ones((2, 1, 1))
    out, lse, _, _ = P.attend(q, pool, batch, 1.0, window=3, n_sink=2)
    np.testing.assert_allclose(lse[0], np.log([5, 5]))
    np.testing.assert_allclose(out[:, 0, 0], [(0 + 1 + 16 + 17 + 18) / 5, (0 + 1 + 17 + 18 + 19) / 5])
    assert P.attend(q, pool, batch, 1.0, window=1)[0][:, 0, 0].tolist() == [18, 19]
    np.testing.assert_array_equal(P.attend(q, pool, batch, 1.0, window=20)[0], P.attend(q, pool, batch, 1.0)[0])


def test_oracle_exponents_of_blocks():
    assert P.block_exponent(np.array([448.0, -1.0]), 448.0) == 0 and P.block_exponent(np.array([449.0]), 448.0) == 1
    assert P.block_exponent(np.array([224.0]), 448.0) == -1 and P.block_exponent(np.array([0.0]), 448.0) == -117
    assert P.block_exponent(np.array([316.0, np.inf, np.nan]), 316.0) == 0 and P.block_exponent(np.array([3.4e38]), 448.0) == 120


def test_oracle_scaled_append_grows_a_blocks_scale_and_its_codes_with_it():
    p = dict(k=np.zeros((1, 1, 16, 2)), v=np.zeros((1, 1, 16, 2)), pos=np.zeros((1, 1, 16), int), weight=np.ones((1, 1, 16)),
             k_scale=np.ones((1, 1, 1)), v_scale=np.ones((1, 1, 1)))
    batch = lambda n: dict(table=[[0]], lens=[n], row_start=[0, 1])
    one = np.array([[[448.0, 2.0 ** -9]]])
    p = P.append_scaled(one, one, one, np.array([[7]]), p, batch(1), 448.0)
    assert p["k_scale"].item() == 1.0 and p["k"][0, 0, 0].tolist() == [448.0, 2.0 ** -9]
    two = np.array([[[900.0, 3.0]]])
    p = P.append_scaled(two, two, two, np.array([[8]]), p, batch(2), 448.0)
    # 900 / 4 = 225 -> 224; 448 -> 112; 2^-9 -> 2^-11 rounds to 0
    assert p["k_scale"].item() == 4.0 and p["k"][0, 0, 0].tolist() == [112.0, 0.0] and p["k"][0, 0, 1].tolist() == [224.0, 0.75]
    p = P.append_scaled(one / 64, one / 64, one / 64, np.array([[9]]), p, batch(3), 448.0)
    assert p["k_scale"].item() == 4.0 and p["pos"][0, 0, :3].tolist() == [7, 8, 9] and p["weight"][0, 0, :4].tolist() == [0, 0, 0, 1]


def test_oracle_turns_pairs_by_their_axis():
    x = np.array([[[1.0, 0, 2, 0, 0, 0]]])                        # pairs (0, 3), (1, 4), (2, 5)
    axes = np.array([[1], [5], [2]])
    got = P.turn(x, axes, 100.0, (1, 1, 1))[0, 0]
    a = 2 * 100 ** (-4 / 6)
    np.testing.assert_allclose(got, [np.cos(1), 0, 2 * np.cos(a), np.sin(1), 0, 2 * np.sin(a)])


def test_oracle_moves_entries_of_different_scales_into_one_block():
    k = np.zeros((3, 1, 16, 1))
    k[0, 0, :2, 0], k[1, 0, 0, 0] = [448.0, 2.0 ** -9], 3.0
    scale = np.array([1.0, 8.0, 64.0]).reshape(3, 1, 1)
    pool = dict(k=k, v=k.copy(), pos=np.arange(48).reshape(3, 1, 16), weight=np.ones((3, 1, 16)), k_scale=scale, v_scale=scale.copy())
    got = P.move_scaled(pool, [[0, 1]], [[np.array([0, 1, 16])]], [[2]])
    assert got["k_scale"][2, 0, 0] == 8.0 and got["k"][2, 0, :3, 0].tolist() == [56.0, 0.0, 3.0] and got["pos"][2, 0, :3].tolist() == [0, 1, 16]
