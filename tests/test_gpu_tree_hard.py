"""GPU tests of tree attention where its kernel is hardest: softmax references that move from tile to tile, elements that are not
numbers, pages that are none, more sequences than anything else holds -- over every width, page size and strip size, with the 64-bit
reference and the tolerances of tests/test_gpu_draft.py (a score e = (d + 4) 2^-23 sum |q k| scale, an output
2 e A + (T + 16) 2^-24 A + 2^-8 A + 2^-8 |out|, A = sum of weight * |value|; over f32 caches without the last two)."""
import numpy as np
import pytest
import torch

from paper_2609_13285_b200 import binding as gb
from paper_2609_13285_b200 import workloads as wl
from tests import draft_ref as ref
from tests.test_gpu_compact import DTYPE, G1, Handle, dev, ints
from tests.test_gpu_draft import check_tree, tree, tree_case

pytestmark = pytest.mark.gpu
KINDS = [("bf16", 64), ("bf16", 32), ("bf16", 96), ("f32", 32), ("fp8", 64)]
SHAPES = [wl.SHAPE_A, wl.SHAPE_B, wl.SHAPE_C, wl.SHAPE_A0, wl.SHAPE_B0]
WIDE1 = wl.HeadShape(H=4, G=1, d_v=128, d_c=128, d_r=32)
CAST = {"bf16": wl.f32_to_bf16_bits, "fp8": wl.f32_to_e4m3_bits, "f32": lambda a: a}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from tests import gpu_util
    gpu_util.ensure_built()


def served(shape, kind):
    if kind == "fp8" and shape.d_r == 24:
        pytest.skip("no such cache")


def put(c, pool, b, t, at, value):
    """Element `at` (a group and an index, or an index) of token t of sequence b becomes value (a NaN in 8 bits)."""
    x = np.uint8(0x7F) if c.kind == "fp8" else CAST[c.kind](np.full(1, value, dtype=np.float32))[0]
    page, slot = c.ids[b, t // c.page], t % c.page
    if pool == 0:
        c.pools[0][page, at[0], slot, at[1]] = x
    else:
        c.pools[1][page, slot, at] = x


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind,page", KINDS)
@pytest.mark.parametrize("n", [1, 12, 20, 40])
def test_references_move_from_tile_to_tile(shape, kind, page, n):
    """Values that grow by half every 64 tokens and long queries: a row's maximum grows by more than 2^8 again and again, over up to
    sixteen tiles, which every group of softmax warps has in its turn."""
    served(shape, kind)
    ctx, sizes = [900, 0, 333], [n, n, n]
    with Handle(shape, page=page, dtype=DTYPE[kind]) as h:
        c, q, see = tree_case(shape, ctx, sizes, page, kind, seed=n, gain=30.0)
        for b, T in enumerate(c.lens):
            for t in range(T):
                row = c.pools[0][c.ids[b, t // page], :, t % page]
                c.pools[0][c.ids[b, t // page], :, t % page] = CAST[kind]((wl.pool_to_f64(row) * 0.02 * 1.5 ** (t // 64)).astype(np.float32))
        c.upload()
        for num_splits in (0, 1, 4):
            check_tree(h, c, q, see, ctx, sizes, num_splits)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind,page", KINDS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_no_row_sees_may_hold_anything(shape, kind, page, bad):
    """Elements that are not numbers in nodes of large and small trees, before, across and behind the halves of a tile, in either half of a
    wide row: rows that do not see them keep their bits."""
    served(shape, kind)
    if kind == "fp8" and not np.isnan(bad):
        pytest.skip("the type has no infinities")
    ctx, sizes, where = [70, 0, 120, 61, 30, 200], [40, 6, 12, 33, 16, 17], [5, 3, 9, 20, 1, 16]
    dims, s = [17, shape.d_v - 1, 0, shape.d_v // 2 + 3, shape.d_v - 5, shape.d_v // 2 - 1], shape
    first = np.concatenate([[0], np.cumsum(sizes)])
    with Handle(shape, page=page, dtype=DTYPE[kind]) as h:
        c, q, see = tree_case(shape, ctx, sizes, page, kind, seed=page)
        splits = (0, 1, 3)
        clean = [check_tree(h, c, q, see, ctx, sizes, k) for k in splits]
        kept = [p.copy() for p in c.pools]
        for pool in (0, 1) if s.d_r else (0,):
            c.pools = [p.copy() for p in kept]
            hit, element = np.zeros((first[-1], s.H), dtype=bool), np.zeros(first[-1], dtype=int)
            for b, j in enumerate(where):
                g = (s.G - 1 - b) % s.G
                put(c, pool, b, ctx[b] + j, (g, dims[b]) if pool == 0 else b % s.d_r, bad)
                heads = slice(g * s.H // s.G, (g + 1) * s.H // s.G) if pool == 0 else slice(0, s.H)
                hit[first[b]:first[b + 1], heads] = see[b][:, j][:, None]
                element[first[b]:first[b + 1]] = dims[b]
            c.upload()
            for k, (o, l) in zip(splits, clean):
                out, lse, status = tree(h, c, q, see, ctx, sizes, k)
                assert status == 0
                assert np.array_equal(out[~hit], o[~hit]) and np.array_equal(lse[~hit], l[~hit])
                if pool == 0:
                    row, head = np.nonzero(hit)
                    assert np.isnan(out[row, head, element[row]]).all()
                elif np.isnan(bad):
                    assert np.isnan(out[hit]).all() and np.isnan(lse[hit]).all()


def near(shape, kind, out, lse, q, v, kr, see, ctx, scale):
    """check_tree's comparison for one sequence whose tokens are v and kr."""
    o, l, size, terms = ref.tree_attention(q, v, kr, see, ctx, scale, shape.G)
    e, T, step = (shape.d_v + shape.d_r + 4) * 2.0 ** -23 * terms, len(v), 0.0 if kind == "f32" else 2.0 ** -8
    assert (np.abs(out - o) <= (2 * e + (T + 16) * 2.0 ** -24 + step) * size + step * np.abs(o) + 1e-30).all()
    live = np.isfinite(l)
    assert np.array_equal(lse[~live], l[~live])
    assert (np.abs(lse[live] - l[live]) <= e + 2.0 ** -22 * (8 + np.abs(l[live])) + (T + 16) * 2.0 ** -24).all()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind,page", KINDS)
def test_tokens_of_pages_that_are_none_count_as_absent(shape, kind, page):
    """A bad page in the context, at its end, at its start, under the nodes themselves, and under a whole sequence."""
    served(shape, kind)
    ctx, sizes, s = [100, 300, 64, 200, 150, 90, 0, 500], [5, 9, 3, 33, 4, 2, 12, 40], shape
    first = np.concatenate([[0], np.cumsum(sizes)])
    with Handle(shape, page=page, dtype=DTYPE[kind]) as h:
        c, q, see = tree_case(shape, ctx, sizes, page, kind, seed=8)
        clean = {k: tree(h, c, q, see, ctx, sizes, k) for k in (0, 1, 2)}
        table = c.table.copy()
        wrong = {1: [150 // page], 3: [0, 199 // page], 4: [150 // page], 5: list(range(table.shape[1])), 7: [1, 2, 520 // page]}
        for i, (b, pages) in enumerate(wrong.items()):
            table[b, pages] = [c.num_pages, -1, 2 ** 31 - 1, -2 ** 31, c.num_pages + 7][i]
        c.d_table = ints(table)
        c.c = gb.make_cache(c.d[0], c.d[1] if s.d_r else None, c.d_table, c.num_pages, c.max_pages)
        qf = q.float().cpu().numpy().astype(np.float64)
        for k in (0, 1, 2):
            out, lse, status = tree(h, c, q, see, ctx, sizes, k)
            assert status & 0xff == gb.GVA_ERR_BAD_PAGE and status >> 8 in wrong
            for b, n in enumerate(sizes):
                rows = slice(first[b], first[b + 1])
                if b not in wrong:
                    assert np.array_equal(out[rows], clean[k][0][rows]) and np.array_equal(lse[rows], clean[k][1][rows])
                    continue
                T = ctx[b] + n
                keep = ~np.isin(np.arange(T) // page, wrong[b])
                v, kr = c.values(b, T)
                near(s, kind, out[rows], lse[rows], qf[rows], v[keep], kr[keep], see[b][:, keep[ctx[b]:]], int(keep[:ctx[b]].sum()), h.scale)
            assert (out[first[5]:first[6]] == 0).all() and np.isneginf(lse[first[5]:first[6]]).all()


@pytest.mark.parametrize("shape", [WIDE1, G1], ids=str)
def test_as_many_sequences_as_a_call_takes(shape):
    """8192 of them: their offsets beside the ring of tiles fill a block's shared memory to within a few kilobytes for wide heads."""
    B = 8192
    with Handle(shape, page=32) as h:
        ctx, sizes = [(7 * i) % 30 for i in range(B)], [1 + i % 2 for i in range(B)]
        c, q, see = tree_case(shape, ctx, sizes, page=32, seed=1)
        check_tree(h, c, q, see, ctx, sizes)
