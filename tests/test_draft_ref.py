"""The references of the calls around a step with drafted tokens, and what needs no GPU of the calls themselves."""
import ctypes

import numpy as np
import pytest

from paper_2609_13285_b200 import binding as gb
from paper_2609_13285_b200 import build as gbuild
from tests import draft_ref as ref


@pytest.fixture(scope="module")
def lib():
    gbuild.build()
    return gb.load()


def test_ancestors_are_the_closure_of_the_parents():
    rng = np.random.default_rng(1)
    for n in (1, 2, 7, 40):
        parents = [-1] + [int(rng.integers(-1, i)) for i in range(1, n)]
        see = ref.ancestors(parents)
        step = np.eye(n, dtype=bool)
        for i, p in enumerate(parents):
            if p >= 0:
                step[i, p] = True
        power = np.linalg.matrix_power(step.astype(np.int64).astype(object), n) if n > 1 else step
        assert np.array_equal(see, power > 0)
    words = ref.mask_words(ref.ancestors([-1, 0, 1]), 2)
    assert words.tolist() == [[1, 0], [3, 0], [7, 0]]


def test_commit_takes_the_first_child_that_was_chosen():
    #        0 -> 1, 2, 3;  2 -> 4;  3 -> 5
    assert ref.commit([-1, 0, 0, 0, 2, 3], [9, 5, 6, 6, 7, 7], [6, 0, 7, 7, 8, 8]) == ([0, 2, 4], 8)
    assert ref.commit([-1, -1], [1, 2], [2, 3]) == ([0], 2)      # another first token is no child
    assert ref.commit([], [], []) == ([], -1)


def test_pages_are_kept_count_of():
    rng = np.random.default_rng(2)
    P, N, B, most = 32, 40, 6, 9
    used, pages = [0] * B, [0] * B
    table, ring, free = np.full((B, most), -1), rng.permutation(N), (11, N)
    for step in range(200):
        want = [int(rng.integers(0, most * P)) if rng.random() < 0.3 else u for u in used]
        r = ref.assign_pages(used, want, pages, table, P, N, ring, free, 300)
        used, pages, table, ring, free = r["lens"], r["pages"], r["table"], r["ring"], r["free"]
        held = [table[b, j] for b in range(B) for j in range(pages[b])]
        kept = [ring[(free[0] + i) % N] for i in range(free[1])]
        assert sorted(held + kept) == list(range(N))
        assert r["cu"][-1] == len(r["pos"]) == len(r["slots"]) <= 300


@pytest.mark.parametrize("d", [4, 8, 24, 64, 128])
def test_frequencies(lib, d):
    for kw in ({}, {"scaling": "linear", "factor": 4.0}, {"scaling": "base", "factor": 8.0}, {"scaling": "parts", "factor": 8.0, "low": 1.0, "high": 4.0, "original_len": 8192},
               {"scaling": "parts", "factor": 2.5, "low": 0.0, "high": 0.5, "original_len": 33, "base": 500.0}):
        kind = {"plain": 0, "linear": 1, "base": 2, "parts": 3}[kw.get("scaling", "plain")]
        rope = gb.make_rope(d_rot=d, **{**kw, "scaling": kind})
        # a power has a few roundings of 2^-53, a sum of two positive parts one more
        assert np.allclose(gb.gva_rope_frequencies(rope), ref.frequencies(d, **kw), rtol=1e-14, atol=0)
    f = gb.gva_rope_frequencies(gb.make_rope(d_rot=d, scaling=gb.GVA_ROPE_BASE, factor=16.0))
    plain = gb.gva_rope_frequencies(gb.make_rope(d_rot=d))
    assert f[0] == plain[0] == 1.0 and abs(f[-1] * 16 / plain[-1] - 1) < 1e-13         # the fastest as it was, the slowest by 1 / factor


BAD_ROPES = [dict(d_rot=0), dict(d_rot=7), dict(d_rot=-2), dict(d_rot=8, layout=2), dict(d_rot=8, layout=-1), dict(d_rot=8, scaling=4), dict(d_rot=8, base=1.0), dict(d_rot=8, base=float("nan")),
             dict(d_rot=8, base=float("inf")), dict(d_rot=8, magnitude=0.0), dict(d_rot=8, magnitude=float("nan")), dict(d_rot=8, scaling=1, factor=0.5), dict(d_rot=8, scaling=1, factor=float("inf")),
             dict(d_rot=2, scaling=2, factor=2.0), dict(d_rot=8, scaling=3, factor=2.0, low=1.0, high=1.0, original_len=10), dict(d_rot=8, scaling=3, factor=2.0, low=0.0, high=1.0, original_len=0),
             dict(d_rot=8, scaling=3, factor=2.0, low=-1.0, high=1.0, original_len=10), dict(d_rot=8, scaling=3, factor=2.0, low=1.0, high=float("inf"), original_len=10)]


@pytest.mark.parametrize("kw", BAD_ROPES, ids=str)
def test_bad_rotations_are_refused(lib, kw):
    out = (ctypes.c_double * 64)()
    assert lib.gva_rope_frequencies(ctypes.byref(gb.make_rope(**kw)), out) == gb.GVA_ERR_INVALID_ARG


def test_calls_without_a_handle_are_refused(lib):
    rope = gb.make_rope(d_rot=8)
    assert lib.gva_rope_frequencies(None, None) == gb.GVA_ERR_INVALID_ARG
    assert lib.gva_rope_frequencies(ctypes.byref(rope), None) == gb.GVA_ERR_INVALID_ARG
    assert lib.gva_set_rope(None, ctypes.byref(rope)) == lib.gqa_set_rope(None, ctypes.byref(rope)) == gb.GVA_ERR_INVALID_ARG
    n = None
    assert lib.gva_assign_pages(n, n, n, n, n, n, 1, 1, n, n, n, n, n, n, n, 0, 1, n, n) == gb.GVA_ERR_INVALID_ARG
    assert lib.gva_tree_masks(n, n, n, n, n, 1, n, 1, 1, n, n) == gb.GVA_ERR_INVALID_ARG
    assert lib.gqa_append(n, n, n, 0, n, 0, n, 0, n, n, n, 1, n, n) == gb.GVA_ERR_INVALID_ARG
    assert lib.gva_append_rows(n, n, n, n, n, n, 1, n, n) == gb.GVA_ERR_INVALID_ARG
    assert lib.gva_decode_tree_workspace_bytes(n, 1, 1, 1, 1, 0) == 0
    assert lib.gva_decode_tree(n, n, n, n, 1, n, n, n, n, n, 0, 1, 1, 1, 1, 0, n, n) == gb.GVA_ERR_INVALID_ARG
    assert lib.gva_tree_commit(n, n, n, n, n, n, n, n, n, n, 1, 1, n, n) == gb.GVA_ERR_INVALID_ARG
    assert "room" in gb.status_string(gb.GVA_ERR_NO_ROOM) or "free pages" in gb.status_string(gb.GVA_ERR_NO_ROOM)
    assert "parent" in gb.status_string(gb.GVA_ERR_TREE)
