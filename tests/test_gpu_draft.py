"""GPU tests of the calls around a step with drafted tokens, against the 64-bit references of tests/draft_ref.py, which read the
identical cached values.

Tolerances.  Whole numbers and moved rows are exact.  A rotated element x c - x' s has the error of its sine and cosine (the
fraction of a half-turn rounded to f32: pi 2^-25, two units in the last place of the function: 2^-22) and three roundings of
2^-24: in all below 6e-7 (|x| + |x'|); rounding it to a cache type adds half a step (bf16 2^-8, e4m3 2^-4 of the value).  Attention: a
score is a sum of d products in f32, off by e = (d + 4) 2^-23 sum |q k| scale at most (2^-23 a step: the accumulator of the tensor
cores truncates), which is the relative error of a weight and the absolute one of the lse; an output is off by 2 e A and the
sums' (T + 16) 2^-24 A with A = sum of weight * |value|, and over 16-bit operands by 2^-8 A for the weights and 2^-8 |out| for itself."""
import numpy as np
import pytest
import torch

from paper_2609_13285_b200 import binding as gb
from paper_2609_13285_b200 import workloads as wl
from tests import draft_ref as ref
from tests.test_gpu_compact import DTYPE, G1, G2W, G3, G8, SHAPES, Cache, Handle, dev, ints

pytestmark = pytest.mark.gpu
TURN = 6e-7
HALF = {"f32": 0.0, "bf16": 2.0 ** -8, "fp8": 2.0 ** -4}
LEAST = {"f32": 1e-38, "bf16": 1e-38, "fp8": 2.0 ** -10}          # half of the smallest step of a type


@pytest.fixture(scope="module", autouse=True)
def _built():
    from tests import gpu_util
    gpu_util.ensure_built()


def zeros(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device="cuda")


def code(status):
    return int(status.item()) & 0xff, int(status.item()) >> 8


# ---- pages ---------------------------------------------------------------------------------------------------
class Pages:
    """A random but sound state of B sequences."""

    def __init__(self, B, P, most, seed, spare=20, held=None, ahead=0.2):
        rng = np.random.default_rng(seed)
        self.B, self.P, self.most = B, P, most
        self.used = [int(rng.integers(0, most * P * 0.7)) for _ in range(B)] if held is None else list(held)
        self.pages = [min(most, -(-u // P) + int(rng.random() < ahead)) for u in self.used]
        self.N = sum(self.pages) + spare
        ids = rng.permutation(self.N)
        self.table = np.full((B, most), -5, dtype=np.int64)
        at = 0
        for b, n in enumerate(self.pages):
            self.table[b, :n] = ids[at:at + n]
            at += n
        first = int(rng.integers(self.N))
        self.ring = np.full(self.N, -9, dtype=np.int64)
        self.ring[(first + np.arange(spare)) % self.N] = ids[at:]
        self.free = (first, spare)


def assign(handle, s, want, max_rows, alias=False):
    used, pages, table, ring, free = ints(s.used), ints(s.pages), ints(s.table), ints(s.ring), ints(s.free)
    lens, out_pages, free_out = (used, pages, free) if alias else (zeros(s.B) - 3, zeros(s.B) - 3, zeros(2) - 3)
    cu, pos, slots, status = zeros(s.B + 1) - 3, zeros(max_rows + 4) - 7, zeros(max_rows + 4) - 7, zeros(1)
    gb.gva_assign_pages(handle.h, used, ints(want), pages, out_pages, table, s.most, s.N, ring, free, free_out, lens, cu, pos, slots, max_rows, s.B, status)
    get = lambda t: t.cpu().numpy().tolist()  # noqa: E731
    n = get(cu)[-1]
    assert get(pos)[n:] == [-7] * (max_rows + 4 - n) and get(slots)[n:] == [-7] * (max_rows + 4 - n)
    return {"pages": get(out_pages), "lens": get(lens), "cu": get(cu), "pos": get(pos)[:n], "slots": get(slots)[:n], "table": get(table), "ring": get(ring), "free": get(free_out)}, code(status)[0]


def check_assign(handle, s, want, max_rows, alias=False):
    r = ref.assign_pages(s.used, want, s.pages, s.table, s.P, s.N, s.ring, s.free, max_rows)
    got, status = assign(handle, s, want, max_rows, alias)
    for k in got:
        assert got[k] == np.asarray(r[k]).tolist(), k
    assert (status == 0) == (r["code"] == 0)
    return r


@pytest.mark.parametrize("B,most,new", [(1, 3, 1), (4, 40, 1), (31, 9, 64), (33, 20, 200), (300, 12, 5), (1025, 5, 40), (2500, 4, 1), (8192, 3, 2), (7, 300, 9000)])
@pytest.mark.parametrize("alias", [False, True])
def test_pages_slots_and_rows(B, most, new, alias):
    for P in (32, 64, 96):
        with Handle(wl.SHAPE_A, page=P) as h:
            s = Pages(B, P, most, seed=B + P, spare=B * (new // P + 2) + 3)
            rng = np.random.default_rng(B)
            want = [min(most * P, u + int(rng.integers(0, new + 1))) if rng.random() < 0.8 else int(rng.integers(0, u + 1)) for u in s.used]
            r = check_assign(h, s, want, sum(max(0, w - u) for w, u in zip(want, s.used)), alias)
            assert r["code"] == 0


@pytest.mark.parametrize("B", [1, 2, 40, 3000])
def test_too_few_pages_or_rows(B):
    with Handle(wl.SHAPE_A) as h:
        rng = np.random.default_rng(B)
        for spare, share in ((0, 1.0), (B // 2 + 1, 1.0), (4 * B, 0.4), (4 * B, 0.0), (B // 3, 0.5)):
            s = Pages(B, 64, 8, seed=B, spare=spare)
            want = [min(8 * 64, u + int(rng.integers(0, 150))) if rng.random() < 0.9 else 0 for u in s.used]
            rows = sum(max(0, w - u) for w, u in zip(want, s.used))
            check_assign(h, s, want, int(rows * share))


def test_bad_lengths_pages_and_rings():
    with Handle(wl.SHAPE_A) as h:
        held = [10, 100, 64, 65, 0, 0, 200, 300]
        for b, change in enumerate([{"used": -1}, {"want": -1}, {"pages": 0}, {"pages": 9}, {"pages": -1}, {"want": 8 * 64 + 1}, {"want": 2 ** 31 - 1}, {"used": 2 ** 31 - 1}]):
            s = Pages(8, 64, 8, seed=5, held=held, ahead=0)
            want = [u + 70 for u in s.used]
            if "want" in change:
                want[b] = change["want"]
            for k in ("used", "pages"):
                if k in change:
                    getattr(s, k)[b] = change[k]
            r = check_assign(h, s, want, 700)
            assert r["code"] == gb.GVA_ERR_SEQ_LEN
        for free in ((-1, 5), (0, -1), (10 ** 6, 3), (0, 10 ** 6)):
            s = Pages(8, 64, 8, seed=6, held=held)
            s.free = free
            r = check_assign(h, s, [u + 70 if i % 2 else 0 for i, u in enumerate(s.used)], 700)
            assert r["code"] == gb.GVA_ERR_BAD_PAGE and r["lens"] == s.used and r["cu"][-1] == 0
        s = Pages(8, 64, 8, seed=7, held=held)                    # a ring that says it is full, and pages that come back
        s.free = (3, s.N)
        assert check_assign(h, s, [0] * 8, 10)["code"] == gb.GVA_ERR_BAD_PAGE
        s = Pages(8, 64, 8, seed=8, held=held)                    # a bad page in the table under new rows: no slot
        s.table[7, s.used[7] // 64] = s.N
        got, _ = assign(h, s, [u + 3 for u in s.used], 100)
        assert got["slots"][-3:] == [-1] * 3


def test_no_sequences_and_no_rows():
    with Handle(wl.SHAPE_A) as h:
        ring, free, cu, free_out, status = ints([3, 1, 2]), ints([1, 2]), zeros(1) - 3, zeros(2) - 3, zeros(1)
        gb.gva_assign_pages(h.h, None, None, None, None, None, 4, 3, ring, free, free_out, None, cu, None, None, 0, 0, status)
        assert cu.tolist() == [0] and free_out.tolist() == [1, 2]
        s = Pages(5, 64, 4, seed=1, held=[0] * 5, ahead=0)
        for rows in (0, 20_000):
            check_assign(h, s, [0] * 5, rows)


def test_a_captured_step_goes_on_in_place():
    with Handle(wl.SHAPE_A) as h:
        s = Pages(50, 64, 30, seed=9, spare=400)
        used, pages, table, ring, free = ints(s.used), ints(s.pages), ints(s.table), ints(s.ring), ints(s.free)
        want, cu, pos, slots, status = zeros(50), zeros(51), zeros(4000), zeros(4000), zeros(1)
        call = lambda: gb.gva_assign_pages(h.h, used, want, pages, pages, table, s.most, s.N, ring, free, free, used, cu, pos, slots, 4000, 50, status)  # noqa: E731
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                call()
        rng = np.random.default_rng(3)
        for step in range(6):
            new = [int(rng.integers(0, 30)) if rng.random() < 0.9 else -u for u in s.used]
            w = [max(0, min(30 * 64, u + d)) for u, d in zip(s.used, new)]
            want.copy_(ints(w))
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            r = ref.assign_pages(s.used, w, s.pages, s.table, 64, s.N, s.ring, s.free, 4000)
            n = r["cu"][-1]
            for have, k in ((used, "lens"), (pages, "pages"), (table, "table"), (ring, "ring"), (free, "free"), (cu, "cu"), (pos[:n], "pos"), (slots[:n], "slots")):
                assert have.cpu().numpy().tolist() == np.asarray(r[k]).tolist(), (step, k)
            s.used, s.pages, s.table, s.ring, s.free = r["lens"], r["pages"], r["table"], r["ring"], r["free"]
        assert int(status.item()) == 0
        del g


# ---- trees ---------------------------------------------------------------------------------------------------
def random_parents(n, seed, roots=0.0, chain=0.0):
    rng = np.random.default_rng(seed)
    return [-1 if i == 0 or rng.random() < roots else i - 1 if rng.random() < chain else int(rng.integers(0, i)) for i in range(n)]


@pytest.mark.parametrize("sizes", [[1], [0, 3, 0], [5, 1, 32, 33, 64, 0, 2], [256, 255, 1, 100], [7] * 900])
def test_masks_and_positions(sizes):
    with Handle(wl.SHAPE_A) as h:
        trees = [random_parents(n, i, roots=0.1, chain=1.0 if i % 3 == 0 else 0.3) for i, n in enumerate(sizes)]
        most = max(max(sizes), 1)
        words, n = (most + 31) // 32 + (1 if most <= 224 else 0), sum(sizes)
        ctx = [13 * i for i in range(len(sizes))]
        cu = np.concatenate([[0], np.cumsum(sizes)])
        mask, pos, status = zeros(n + 2, words) - 3, zeros(n + 2) - 3, zeros(1)
        parents = ints(np.concatenate([np.asarray(t, dtype=np.int32) for t in trees] + [np.zeros(0, np.int32)]) if n else [0])
        gb.gva_tree_masks(h.h, parents, ints(cu), ints(ctx), mask, words, pos, len(sizes), most, status)
        assert int(status.item()) == 0
        got, at = mask.cpu().numpy().view(np.uint32), pos.cpu().numpy()
        for b, t in enumerate(trees):
            if t:
                see = ref.ancestors(t)
                assert np.array_equal(got[cu[b]:cu[b + 1]], ref.mask_words(see, words))
                assert np.array_equal(at[cu[b]:cu[b + 1]], ctx[b] + see.sum(1) - 1)
        assert (mask[n:] == -3).all() and (pos[n:] == -3).all()


def test_bad_trees_are_left_out():
    with Handle(wl.SHAPE_A) as h:
        trees = [[-1, 0, 1], [-1, 1], [0], [-1, -2], [-1] * 9, [-1, 0]]
        cu = np.concatenate([[0], np.cumsum([len(t) for t in trees])])
        mask, status = zeros(int(cu[-1]), 1) - 3, zeros(1)
        gb.gva_tree_masks(h.h, ints(sum(trees, [])), ints(cu), None, mask, 1, None, len(trees), 8, status)
        got = mask.cpu().numpy().view(np.uint32)[:, 0].tolist()
        assert got[:3] == [1, 3, 7] and got[-2:] == [1, 3] and set(got[3:-2]) == {2 ** 32 - 3}
        assert code(status)[0] == gb.GVA_ERR_TREE and 1 <= code(status)[1] <= 4


# ---- rows by slot map ------------------------------------------------------------------------------------------
def value(bits_tensor, kind):
    return wl.pool_to_f64(bits_tensor)


@pytest.mark.parametrize("shape", SHAPES + [G1, G3, G8, G2W], ids=str)
@pytest.mark.parametrize("kind,page", [("bf16", 32), ("bf16", 192), ("f32", 32), ("fp8", 64)])
def test_rows_are_what_append_cache_at_writes(shape, kind, page):
    if kind == "fp8" and shape.d_r == 24:
        pytest.skip("no such cache")
    for n in (1, 7, 700):
        with Handle(shape, page=page, dtype=DTYPE[kind]) as h:
            a = Cache(shape, [n + 60], page=page, kind=kind, seed=n)
            rng = np.random.default_rng(n)
            places = rng.permutation(n + 60)[:n]
            slots = a.ids[0, places // page] * page + places % page
            pos = rng.integers(0, 100_000, n)
            v, kr = (rng.standard_normal((n, shape.G, shape.d_v)) * 3).astype(np.float32), rng.standard_normal((n, shape.d_r)).astype(np.float32)
            b = Cache(shape, [n + 60], page=page, kind=kind, seed=n)
            status = zeros(1)
            gb.gva_append_rows(h.h, a.c, dev(v), dev(kr) if shape.d_r else None, ints(pos), ints(slots), n, status)
            for i in range(min(n, 40)):
                k = i if n <= 40 else i * (n // 40)
                gb.gva_append_cache_at(h.h, b.c, dev(v[k:k + 1]), dev(kr[k:k + 1]) if shape.d_r else None, ints(places[k:k + 1]), ints(pos[k:k + 1]), 1, status)
            assert int(status.item()) == 0
            got, want = a.download(), b.download()
            every = [i if n <= 40 else i * (n // 40) for i in range(min(n, 40))]
            for x, y in zip(got, want):
                for i in every:
                    assert np.array_equal(ref_row(x, slots[i], page), ref_row(y, slots[i], page))
            touched = np.zeros((a.num_pages, page), dtype=bool)
            touched[slots // page, slots % page] = True
            for x, y in zip(got, a.pools):                        # nothing else changes
                keep = np.broadcast_to(~touched[:, None], x.shape[:-1]) if x.ndim == 4 else ~touched
                assert np.array_equal(x[keep].view(np.uint8), y[keep].view(np.uint8))


def ref_row(pool, slot, page):
    return pool[slot // page, ..., slot % page, :].view(np.uint8)


def test_rows_with_an_odd_address():
    with Handle(wl.SHAPE_A) as h:
        a, b = (Cache(wl.SHAPE_A, [64], kind="bf16", seed=4) for _ in range(2))
        v = torch.randn(9 * 4 * 64 + 1, device="cuda")
        kr, pos, slots = torch.randn(9, 16, device="cuda"), ints(np.arange(9)), ints(np.arange(9) + a.ids[0, 0] * 64)
        gb.gva_append_rows(h.h, a.c, v[1:], kr, pos, slots, 9)
        gb.gva_append_rows(h.h, b.c, v[1:].clone(), kr, pos, slots, 9)
        for x, y in zip(a.download(), b.download()):
            assert np.array_equal(x, y)


SPECS = [("pairs", None, "plain", {}), ("halves", None, "plain", {}), ("pairs", 0.5, "linear", {"factor": 4.0}), ("halves", 0.5, "base", {"factor": 3.0}), ("halves", 24, "parts", None),
         ("pairs", 8, "parts", None), ("pairs", 40, "plain", {}), ("halves", 8, "plain", {})]
PARTS = {"factor": 8.0, "low": 1.0, "high": 4.0, "original_len": 4096}


@pytest.mark.parametrize("shape", [wl.SHAPE_A, wl.SHAPE_B0, G1, G3], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("spec", SPECS, ids=lambda s: "-".join(map(str, s[:3])))
def test_gqa_append(shape, kind, spec):
    layout, part, scaling, kw = spec
    if kind == "fp8" and shape.d_r == 24:
        pytest.skip("no such cache")
    kw, d, H, G, page = PARTS if kw is None else kw, shape.d_v, shape.H, shape.G, 64
    d_rot = d if part is None else int(d * part) if isinstance(part, float) else part
    m = 1.25 if scaling == "parts" else 1.0
    rope = gb.make_rope(layout=gb.GVA_ROPE_HALVES if layout == "halves" else gb.GVA_ROPE_PAIRS, d_rot=d_rot, magnitude=m,
                        scaling=["plain", "linear", "base", "parts"].index(scaling), **kw)
    f = ref.frequencies(d_rot, scaling=scaling, **kw)
    for n in (1, 6, 2500):
        rng = np.random.default_rng(n)
        pages = n // page + 3
        qkv = rng.standard_normal((n, H + 2 * G, d)).astype(np.float32)
        pos = rng.integers(0, 200_000, n)
        slots = rng.permutation(pages * page)[:n]
        slots[n // 2:n // 2 + 1] = -1 if n > 1 else slots[0]
        np_type = {"bf16": np.uint16, "f32": np.float32, "fp8": np.uint8}[kind]
        pools = [np.full((pages, G, page, d), 3, dtype=np_type) for _ in range(2)]
        k_pool, v_pool = (dev(p.view(np.int16)) if kind == "bf16" else dev(p) for p in pools)
        x = dev(qkv)
        out = torch.full((n, H, d), float("nan"), device="cuda")
        status, row = zeros(1), (H + 2 * G) * d
        with Handle(shape, page=page, dtype=DTYPE[kind]) as h:
            gb.gqa_set_rope(h.h, rope)
            gb.gqa_append(h.h, gb.make_gqa_cache(k_pool, v_pool, None, pages, 1), x, row, x[:, H:], row, x[:, H + G:], row, ints(pos), ints(slots), out, n, status)
        assert int(status.item()) == 0
        want = ref.rotate(qkv[:, :H + G], pos, f, layout == "halves", m)
        size = np.abs(qkv[:, :H + G].astype(np.float64))
        both = ref.rotate(size, np.zeros(n), f, layout == "halves")
        other = both.copy()                                       # |x| + |x'| of the element's pair
        lo, hi = (slice(0, d_rot // 2), slice(d_rot // 2, d_rot)) if layout == "halves" else (slice(0, d_rot, 2), slice(1, d_rot, 2))
        other[..., lo] = other[..., hi] = both[..., lo] + both[..., hi]
        tol = m * TURN * other
        tol[..., d_rot:] = 0
        assert (np.abs(out.cpu().numpy() - want[:, :H]) <= tol[:, :H]).all()
        put = np.nonzero(slots >= 0)[0]
        for pool, old, w, t in ((k_pool, pools[0], want[:, H:], tol[:, H:]), (v_pool, pools[1], qkv[:, H + G:].astype(np.float64), 0 * tol[:, H:])):
            got = pool.cpu().numpy().view(np_type)
            rows = wl.pool_to_f64(got[slots[put] // page, :, slots[put] % page])
            assert (np.abs(rows - w[put]) <= HALF[kind] * np.abs(w[put]) + t[put] * (1 + HALF[kind]) + LEAST[kind]).all()
            rest = np.ones((pages, page), dtype=bool)
            rest[slots[put] // page, slots[put] % page] = False
            keep = np.broadcast_to(rest[:, None], got.shape[:-1])
            assert np.array_equal(got[keep], old[keep])


def test_gqa_append_in_place_without_queries_and_with_bad_rows():
    H, G, d, n, page, pages = 16, 4, 64, 9, 64, 2
    rng = np.random.default_rng(0)
    q, k, v = (rng.standard_normal((n, x, d)).astype(np.float32) for x in (H, G, G))
    pos, slots = np.arange(n) * 7, np.arange(n) * 5
    pos[3], slots[4], slots[5], pos[6], slots[6] = -1, pages * page, 2 ** 31 - 1, -4, -2
    pools = [torch.full((pages, G, page, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    with Handle(wl.SHAPE_A) as h:
        x, out, status = dev(q), torch.empty(n, H, d, device="cuda"), zeros(1)
        gb.gqa_append(h.h, gb.make_gqa_cache(pools[0], pools[1], None, pages, 1), x, H * d, dev(k), G * d, dev(v), G * d, ints(pos), ints(slots), out, n, status)
        assert code(status)[0] in (gb.GVA_ERR_BAD_PAGE, gb.GVA_ERR_SEQ_LEN) and code(status)[1] in (3, 4, 5)
        gb.gqa_append(h.h, gb.make_gqa_cache(pools[2], pools[3], None, pages, 1), None, 0, dev(k), G * d, dev(v), G * d, ints(pos), ints(slots), None, n, None)
        assert all(torch.equal(a, b) for a, b in zip(pools[:2], pools[2:]))
        gb.gqa_append(h.h, gb.make_gqa_cache(pools[2], pools[3], None, pages, 1), x, H * d, dev(k), G * d, dev(v), G * d, ints(pos), ints(slots), x, n, None)
        assert torch.equal(x, out)
    kept = pools[0].permute(0, 2, 1, 3).reshape(pages * page, -1)
    written = [i * 5 for i in range(n) if i not in (3, 4, 5, 6)]
    assert ((kept != 7).any(dim=1).nonzero()[:, 0].cpu().numpy() == written).all()


def test_a_scaled_rotation_reaches_every_call_of_the_handle():
    shape, n = wl.SHAPE_A, 40
    rope = gb.make_rope(d_rot=16, scaling=gb.GVA_ROPE_PARTS, **PARTS)
    f = ref.frequencies(16, scaling="parts", **PARTS)
    rng = np.random.default_rng(1)
    v, kr, pos = rng.standard_normal((n, 4, 64)).astype(np.float32), rng.standard_normal((n, 16)).astype(np.float32), rng.integers(0, 60_000, n)
    with Handle(shape, dtype=gb.GVA_F32) as h:
        c = Cache(shape, [n], kind="f32", seed=1)
        gb.gva_set_rope(h.h, rope)
        slots = c.ids[0, np.arange(n) // 64] * 64 + np.arange(n) % 64
        gb.gva_append_rows(h.h, c.c, dev(v), dev(kr), ints(pos), ints(slots), n)
        got = c.values(0, n, c.download())[1]
        want = ref.rotate(kr[:, None], pos, f, False)[:, 0]
        assert np.abs(got - want).max() <= 2.0 ** -24 * 8 + 1e-9    # rotated in fp64, rounded once (|element| < 8); angles of 6e4 to 1e-11
        q_c, q_r, M = rng.standard_normal((n, 16, 64)).astype(np.float32), rng.standard_normal((n, 16, 16)).astype(np.float32), rng.standard_normal((16, 64, 64)).astype(np.float32)
        out = torch.empty(n, 16, 80, device="cuda")
        Md = dev(M)
        torch.cuda.synchronize()
        gb.gva_absorb_query(h.h, dev(q_c), dev(q_r), Md, ints(pos), out, n)
        assert np.abs(out.cpu().numpy()[..., 64:] - ref.rotate(q_r, pos, f, False)).max() <= 2.0 ** -24 * 8 + 1e-9


# ---- attention -------------------------------------------------------------------------------------------------
def tree_case(shape, ctx, sizes, page=64, kind="bf16", seed=0, gain=1.5, see=None, **kw):
    """A cache with its trees: (cache, queries as the call gets them, what each node sees)."""
    c = Cache(shape, [t + n for t, n in zip(ctx, sizes)], page=page, kind=kind, seed=seed, **kw)
    q = (np.random.default_rng(seed + 1).standard_normal((sum(sizes), shape.H, shape.d_v + shape.d_r)) * gain).astype(np.float32)
    q = dev(q) if kind == "f32" else dev(q).bfloat16()
    if see is None:
        see = [ref.ancestors(random_parents(n, seed + i, roots=0.05, chain=0.3)) for i, n in enumerate(sizes)]
    return c, q, see


def tree(handle, c, q, see, ctx, sizes, num_splits=0, words=None, max_len=None, most=None, cu=None):
    s, B, n = c.shape, len(ctx), sum(sizes)
    most = max(sizes + [1]) if most is None else most
    words = (most + 31) // 32 if words is None else words
    max_len = max(max(a + b for a, b in zip(ctx, sizes)), 1) if max_len is None else max_len
    bits = np.concatenate([ref.mask_words(x, words) for x in see if len(x)] + [np.zeros((1, words), np.uint32)])
    out = torch.full((n + 2, s.H, s.d_v), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((n + 2, s.H), 7.0, device="cuda")
    ws = torch.full((gb.gva_decode_tree_workspace_bytes(handle.h, B, n, most, max_len, num_splits),), 0xFF, dtype=torch.uint8, device="cuda")
    status = zeros(1)
    cu = np.concatenate([[0], np.cumsum(sizes)]) if cu is None else cu
    gb.gva_decode_tree(handle.h, c.c, q, dev(bits.view(np.int32)), words, ints(cu), ints(ctx), out, lse, ws, B, n, most, max_len, num_splits, status)
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    return out[:n].float().cpu().numpy().astype(np.float64), lse[:n].cpu().numpy().astype(np.float64), int(status.item())


def check_tree(handle, c, q, see, ctx, sizes, num_splits=0, **kw):
    out, lse, status = tree(handle, c, q, see, ctx, sizes, num_splits, **kw)
    assert status == 0
    s, at, qf = c.shape, 0, q.float().cpu().numpy().astype(np.float64)
    step = 0.0 if c.kind == "f32" else 2.0 ** -8
    for b, n in enumerate(sizes):
        T = ctx[b] + n
        v, kr = c.values(b, T)
        o, l, size, terms = ref.tree_attention(qf[at:at + n], v, kr, see[b], ctx[b], handle.scale, s.G)
        e = (s.d_v + s.d_r + 4) * 2.0 ** -23 * terms
        tol = (2 * e + (T + 16) * 2.0 ** -24 + step) * size + step * np.abs(o) + 1e-30
        assert (np.abs(out[at:at + n] - o) <= tol).all(), (b, np.abs(out[at:at + n] - o).max())
        live = np.isfinite(l)
        assert np.array_equal(lse[at:at + n][~live], l[~live])
        assert (np.abs(lse[at:at + n][live] - l[live]) <= e + 2.0 ** -22 * (8 + np.abs(l[live])) + (T + 16) * 2.0 ** -24).all()
        if n:                                                      # the mean error is a rounding's, not a bound's
            rel = np.linalg.norm(out[at:at + n] - o) / max(np.linalg.norm(o), 1e-30)
            assert rel <= (2.0 ** -8 if step else 2e-5)
        at += n
    return out, lse


KINDS = [("bf16", 64), ("bf16", 32), ("bf16", 96), ("f32", 32), ("fp8", 64)]
CTX = [0, 1, 31, 63, 64, 65, 127, 500, 1000]
SIZES = [3, 1, 33, 2, 64, 0, 9, 40, 17]


@pytest.mark.parametrize("shape", SHAPES + [G1, G3, G8, G2W], ids=str)
@pytest.mark.parametrize("kind,page", KINDS)
@pytest.mark.parametrize("num_splits", [0, 1, 3])
def test_trees_over_ragged_sequences(shape, kind, page, num_splits):
    if kind == "fp8" and shape.d_r == 24:
        pytest.skip("no such cache")
    with Handle(shape, page=page, dtype=DTYPE[kind]) as h:
        c, q, see = tree_case(shape, CTX, SIZES, page, kind, seed=page)
        check_tree(h, c, q, see, CTX, SIZES, num_splits)


@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 65, 100, 255, 256])
def test_every_size_of_tree(n):
    with Handle(wl.SHAPE_A) as h:
        for ctx in ([0], [60, 200]):
            sizes = [n] * len(ctx)
            c, q, see = tree_case(wl.SHAPE_A, ctx, sizes, seed=n, paged=ctx != [0])
            check_tree(h, c, q, see, ctx, sizes)


@pytest.mark.parametrize("shape", [wl.SHAPE_A, wl.SHAPE_B], ids=str)
@pytest.mark.parametrize("B,T,n", [(1, 20_000, 5), (3, 9_000, 32), (40, 700, 16), (300, 100, 3), (2000, 3, 2)])
def test_long_and_many(shape, B, T, n):
    with Handle(shape) as h:
        ctx, sizes = [T - 7 * (i % 11) if T > 100 else i % (T + 1) for i in range(B)], [1 + (n - 1 + i) % n for i in range(B)]
        c, q, see = tree_case(shape, ctx, sizes, seed=T)
        check_tree(h, c, q, see, ctx, sizes)
        if B <= 3:
            check_tree(h, c, q, see, ctx, sizes, num_splits=64)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_masks_of_any_kind(kind):
    """Rows that see nothing, every node, later nodes, no context; words and bounds larger than needed."""
    rng = np.random.default_rng(5)
    with Handle(wl.SHAPE_A, dtype=DTYPE[kind]) as h:
        ctx, sizes = [0, 0, 100, 64, 0], [40, 5, 33, 64, 1]
        see = [rng.random((n, n)) < p for n, p in zip(sizes, (0.3, 0.0, 0.5, 1.0, 1.0))]
        see[0][7] = False
        c, q, _ = tree_case(wl.SHAPE_A, ctx, sizes, kind=kind, seed=1, room=64)
        for num_splits in (0, 2):
            out, lse = check_tree(h, c, q, see, ctx, sizes, num_splits, words=5, most=130, max_len=6000)
            assert (out[7] == 0).all() and np.isneginf(lse[7]).all() and (out[40:45] == 0).all()
        wide = [np.concatenate([x, np.ones((len(x), 96 - x.shape[1]), dtype=bool)], axis=1) for x in see]      # bits behind the tree say nothing
        check_tree(h, c, q, wide, ctx, sizes, words=3, most=64)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_is_out_of_sight_may_hold_anything(kind, bad):
    shape, ctx, sizes = wl.SHAPE_A, [70, 0], [40, 6]
    with Handle(shape, dtype=DTYPE[kind]) as h:
        c, q, see = tree_case(shape, ctx, sizes, kind=kind, seed=3)
        without = {k: check_tree(h, c, q, see, ctx, sizes, k) for k in (0, 2)}
        slot = lambda b, t: (c.ids[b, t // 64], t % 64)  # noqa: E731
        pg, at = slot(0, 70 + 5)
        c.d[0][pg, 2, at, 17] = dev(np.array([wl.f32_to_bf16_bits(np.float32([bad]))[0]]).view(np.int16))[0] if kind == "bf16" else bad
        pg, at = slot(1, 3)
        c.d[1][pg, at, 4] = dev(np.array([wl.f32_to_bf16_bits(np.float32([bad]))[0]]).view(np.int16))[0] if kind == "bf16" else bad
        for num_splits in (0, 2):
            out, lse, status = tree(h, c, q, see, ctx, sizes, num_splits)
            clean, clean_lse = without[num_splits]
            assert status == 0
            hit = np.zeros(out.shape[:2], dtype=bool)
            hit[:40, 8:12] = see[0][:, 5][:, None]
            hit[40:] = see[1][:, 3][:, None]
            assert np.array_equal(out[~hit], clean[~hit]) and np.array_equal(lse[~hit], clean_lse[~hit])
            if np.isnan(bad):
                assert np.isnan(out[hit]).all()
            else:
                value_hit = hit.copy()
                value_hit[40:] = False
                assert not np.isfinite(out[value_hit]).all(axis=-1).any()


def test_bad_lengths_and_pages_stay_with_their_sequence():
    shape, ctx, sizes = wl.SHAPE_A, [100, 300, 64, 200, 150, 90], [5, 9, 3, 33, 4, 2]
    for kind in ("bf16", "f32"):
        with Handle(shape, dtype=DTYPE[kind]) as h:
            c, q, see = tree_case(shape, ctx, sizes, kind=kind, seed=8)
            clean, clean_lse, _ = tree(h, c, q, see, ctx, sizes, num_splits=1)
            cu = np.concatenate([[0], np.cumsum(sizes)])
            for b, (wrong, most) in enumerate([(-1, 33), (10 ** 6, 33), (2 ** 31 - 1, 33), (200, 32)]):
                at = list(ctx)
                at[b] = wrong
                out, lse, status = tree(h, c, q, see, at, sizes, num_splits=1, most=most, max_len=400, words=2)
                assert status & 0xff == gb.GVA_ERR_SEQ_LEN and status >> 8 == b
                other = np.ones(len(out), dtype=bool)
                other[cu[b]:cu[b + 1]] = False
                assert np.array_equal(out[other], clean[other]) and (out[~other] == 7).all() and (lse[~other] == 7).all()
            table = c.table.copy()
            table[1, 2], table[3, 0] = c.num_pages, -1
            c.d_table = ints(table)
            c.c = gb.make_cache(c.d[0], c.d[1], c.d_table, c.num_pages, c.max_pages)
            out, lse, status = tree(h, c, q, see, ctx, sizes, num_splits=1)
            assert status & 0xff == gb.GVA_ERR_BAD_PAGE and status >> 8 in (1, 3)
            other = np.ones(len(out), dtype=bool)
            other[cu[1]:cu[2]] = other[cu[3]:cu[4]] = False
            assert np.array_equal(out[other], clean[other])
            # the tokens of that page count as absent
            v, kr = c.values(1, 309)
            keep = np.ones(309, dtype=bool)
            keep[128:192] = False
            o, l, size, _ = ref.tree_attention(q.float().cpu().numpy().astype(np.float64)[5:14], v[keep], kr[keep], see[1], 300 - 64, h.scale, shape.G)
            assert (np.abs(out[5:14] - o) <= 2.0 ** -7 * size + 1e-6).all() and np.abs(lse[5:14] - l).max() <= 1e-4


def test_rows_beyond_what_the_call_allows_for_are_not_written():
    shape, ctx, sizes = wl.SHAPE_A, [30, 40, 500], [4, 5, 6]
    for kind in ("bf16", "f32"):
        with Handle(shape, dtype=DTYPE[kind]) as h:
            c, q, see = tree_case(shape, ctx, sizes, kind=kind, seed=9)
            clean, clean_lse, _ = tree(h, c, q, see, ctx, sizes, num_splits=2)
            mask = dev(np.concatenate([ref.mask_words(x, 1) for x in see]).view(np.int32))
            out, lse, status = torch.full((15, 16, 64), 7.0, dtype=q.dtype, device="cuda"), torch.full((15, 16), 7.0, device="cuda"), zeros(1)
            ws = torch.empty(gb.gva_decode_tree_workspace_bytes(h.h, 3, 14, 6, 506, 2), dtype=torch.uint8, device="cuda")
            gb.gva_decode_tree(h.h, c.c, q, mask, 1, ints([0, 4, 9, 15]), ints(ctx), out, lse, ws, 3, 14, 6, 506, 2, status)
            assert code(status) == (gb.GVA_ERR_SEQ_LEN, 2) and (out[9:] == 7).all() and (lse[9:] == 7).all()
            assert np.array_equal(out[:9].float().cpu().numpy(), clean[:9]) and np.array_equal(lse[:9].cpu().numpy(), clean_lse[:9])


def test_large_scores_and_moving_maxima():
    """Queries 30 times as long, and values that grow along the sequence: the softmax's reference moves again and again."""
    shape, ctx, sizes = wl.SHAPE_A, [900], [20]
    with Handle(shape) as h:
        c, q, see = tree_case(shape, ctx, sizes, seed=2, gain=30.0)
        check_tree(h, c, q, see, ctx, sizes)
        c2 = Cache(shape, [920], kind="bf16", seed=2)
        x = wl.bf16_bits_to_f32(c2.pools[0])
        for j in range(15):
            x[c2.ids[0, j]] *= 0.02 * 1.5 ** j
        c2.pools[0] = wl.f32_to_bf16_bits(np.nan_to_num(x))
        c2.upload()
        for num_splits in (0, 1, 4):
            check_tree(h, c2, q, see, ctx, sizes, num_splits)


def test_twice_the_same_bits_on_two_streams_and_in_a_graph():
    shape, ctx, sizes = wl.SHAPE_A, [3000, 100, 777], [16, 3, 40]
    with Handle(shape) as h:
        c, q, see = tree_case(shape, ctx, sizes, seed=4)
        first = tree(h, c, q, see, ctx, sizes)
        again = tree(h, c, q, see, ctx, sizes)
        assert all(np.array_equal(a, b) for a, b in zip(first[:2], again[:2]))
        bits = np.concatenate([ref.mask_words(x, 2) for x in see])
        n = sum(sizes)
        args = [dev(bits.view(np.int32)), ints(np.concatenate([[0], np.cumsum(sizes)])), ints(ctx)]
        size = gb.gva_decode_tree_workspace_bytes(h.h, 3, n, 40, 3016)
        streams, got, graphs, keep = [torch.cuda.Stream() for _ in range(2)], [], [], []
        torch.cuda.synchronize()
        for st in streams:
            out, lse = torch.zeros(n, 16, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 16, device="cuda")
            ws = torch.empty(size, dtype=torch.uint8, device="cuda")
            keep.append((out, lse, ws))
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                gb.gva_decode_tree(h.h, c.c, q, args[0], 2, args[1], args[2], out, lse, ws, 3, n, 40, 3016)
            graphs.append(g)
        for _ in range(3):
            for st, g in zip(streams, graphs):
                with torch.cuda.stream(st):
                    g.replay()
        torch.cuda.synchronize()
        for out, lse, _ in keep:
            assert np.array_equal(out.float().cpu().numpy(), first[0]) and np.array_equal(lse.cpu().numpy(), first[1])
        del graphs


def test_a_chain_is_what_decode_tokens_computes():
    shape, ctx, n = wl.SHAPE_A, [500, 1234], 4
    with Handle(shape) as h:
        see = [np.tril(np.ones((n, n), dtype=bool))] * 2
        c, q, _ = tree_case(shape, ctx, [n] * 2, seed=6, see=see)
        out, lse = check_tree(h, c, q, see, ctx, [n] * 2)
        o, l = torch.empty(2 * n, 16, 64, device="cuda"), torch.empty(2 * n, 16, device="cuda")
        ws = torch.empty(gb.gva_decode_tokens_workspace_bytes(h.h, 2, n, 1238), dtype=torch.uint8, device="cuda")
        gb.gva_decode_tokens(h.h, c.c, q.float(), ints([t + n for t in ctx]), o, l, ws, 2, n, 1238)
        # that call rounds its weights to bf16 too, this one its output besides
        assert np.abs(out - o.cpu().numpy()).max() <= 2e-2 and np.abs(lse - l.cpu().numpy()).max() <= 1e-4


# ---- commit ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", SHAPES + [G1, G3, G8, G2W], ids=str)
@pytest.mark.parametrize("kind,page", KINDS)
@pytest.mark.parametrize("agree", [0.0, 0.9])
def test_commit_moves_the_rows_that_stay(shape, kind, page, agree):
    if kind == "fp8" and shape.d_r == 24:
        pytest.skip("no such cache")
    ctx, sizes = [0, 1, 31, 60, 64, 500, 90, 95], [3, 1, 33, 8, 64, 0, 256, 40]
    with Handle(shape, page=page, dtype=DTYPE[kind]) as h:
        c = Cache(shape, [t + n for t, n in zip(ctx, sizes)], page=page, kind=kind, seed=page)
        rng = np.random.default_rng(page)
        trees = [random_parents(n, i, chain=0.5) for i, n in enumerate(sizes)]
        tokens = [rng.integers(0, 4, n) for n in sizes]              # few tokens: siblings that say the same
        chosen = [rng.integers(0, 4, n) for n in sizes]
        for b, n in enumerate(sizes):                                # deep paths: what is chosen was drafted
            for i in range(1, n):
                if rng.random() < agree:
                    chosen[b][trees[b][i]] = tokens[b][i]
        path, last, status = zeros(sum(sizes) + 2) - 5, zeros(len(ctx)), zeros(1)
        lens = ints(ctx)
        gb.gva_tree_commit(h.h, c.c, ints(sum(trees, [])), ints(np.concatenate(tokens)), ints(np.concatenate(chosen)), ints(np.concatenate([[0], np.cumsum(sizes)])), lens, path, lens, last,
                           len(ctx), 256, status)
        assert int(status.item()) == 0
        want, at = [p.copy() for p in c.pools], 0
        got_path = path.cpu().numpy().tolist()
        for b, n in enumerate(sizes):
            p, end = ref.commit(trees[b], tokens[b], chosen[b])
            assert got_path[at:at + n] == p + [-1] * (n - len(p)) and int(lens[b]) == ctx[b] + len(p) and int(last[b]) == end
            place = lambda t: (c.ids[b, t // page], t % page)  # noqa: E731
            for w, old in zip(want, c.pools):
                for i, node in enumerate(p):
                    (dp, ds), (sp, ss) = place(ctx[b] + i), place(ctx[b] + node)
                    w[dp, ..., ds, :] = old[sp, ..., ss, :]
            at += n
        assert got_path[at:] == [-5, -5]
        for w, g in zip(want, c.download()):
            assert np.array_equal(w.view(np.uint8), g.view(np.uint8))


@pytest.mark.parametrize("kind,page", KINDS)
def test_commit_of_a_long_path(kind, page):
    """A comb: nodes 0, 1, 2, 4, 6, .. 82 stay, the odd ones between them go; 43 rows, more than a batch and than a page of 32."""
    shape, n = wl.SHAPE_B if kind == "fp8" else wl.SHAPE_A, 84
    parents = [-1, 0, 1] + [i - 1 if i % 2 else i - 2 for i in range(3, n)]
    tokens = [100 + i if i < 2 or i % 2 == 0 else 7 for i in range(n)]
    chosen = [101, 102] + [102 + i for i in range(2, n)]
    want = [0, 1] + list(range(2, n, 2))
    assert ref.commit(parents, tokens, chosen) == (want, chosen[want[-1]])
    with Handle(shape, page=page, dtype=DTYPE[kind]) as h:
        c = Cache(shape, [50 + n], page=page, kind=kind, seed=2)
        path, lens, last = zeros(n), zeros(1), zeros(1)
        gb.gva_tree_commit(h.h, c.c, ints(parents), ints(tokens), ints(chosen), ints([0, n]), ints([50]), path, lens, last, 1, 96)
        assert path.cpu().tolist() == want + [-1] * (n - len(want)) and int(lens) == 50 + len(want)
        place = lambda t: (c.ids[0, t // page], t % page)  # noqa: E731
        for old, g in zip(c.pools, c.download()):
            w = old.copy()
            for i, node in enumerate(want):
                (dp, ds), (sp, ss) = place(50 + i), place(50 + node)
                w[dp, ..., ds, :] = old[sp, ..., ss, :]
            assert np.array_equal(w.view(np.uint8), g.view(np.uint8))


def test_commit_leaves_bad_sequences_alone():
    shape, ctx, sizes = wl.SHAPE_A, [60, 60, 60, -1, 10 ** 6, 60], [6, 6, 6, 6, 6, 6]
    with Handle(shape) as h:
        c = Cache(shape, [66] * 6, kind="bf16", seed=1)
        trees = [[-1, 0, 0, 2, 2, 4]] * 6
        trees[1] = [-1, 0, 3, 2, 2, 4]
        tokens, chosen = [[0, 1, 2, 3, 4, 5]] * 6, [[2, 9, 4, 9, 5, 8]] * 6      # path 0, 2, 4, 5
        table = c.table.copy()
        table[2, 1] = -7
        c.d_table = ints(table)
        c.c = gb.make_cache(c.d[0], c.d[1], c.d_table, c.num_pages, c.max_pages)
        path, lens, last, status = zeros(36) - 5, zeros(6), zeros(6), zeros(1)
        gb.gva_tree_commit(h.h, c.c, ints(sum(trees, [])), ints(sum(tokens, [])), ints(sum(chosen, [])), ints(np.arange(7) * 6), ints(ctx), path, lens, last, 6, 8, status)
        assert code(status)[0] in (gb.GVA_ERR_TREE, gb.GVA_ERR_SEQ_LEN, gb.GVA_ERR_BAD_PAGE) and code(status)[1] in (1, 2, 3, 4)
        good = [0, 2, 4, 5, -1, -1]
        assert path.cpu().numpy().reshape(6, 6).tolist() == [good] + [[-1] * 6] * 4 + [good]
        assert lens.cpu().numpy().tolist() == [64, 60, 60, -1, 10 ** 6, 64] and last.cpu().numpy().tolist() == [8, -1, -1, -1, -1, 8]
        got = c.download()
        for b in range(6):
            for w, g in zip(c.pools, got):
                for t in range(66):
                    src = 60 + good[t - 60] if b in (0, 5) and 60 <= t < 64 else t
                    assert np.array_equal(g[c.ids[b, t // 64], ..., t % 64, :], w[c.ids[b, src // 64], ..., src % 64, :])


# ---- refusals --------------------------------------------------------------------------------------------------
def refused(handle, name, good, **changes):
    """The status of a call with some of its arguments changed; it launches nothing."""
    args = dict(good)
    args.update(changes)
    return getattr(gb, name)(handle.h, *args.values(), check=False)


def test_refusals():
    shape, t = wl.SHAPE_A, zeros(4096)
    c = Cache(shape, [200], kind="bf16", seed=1)
    x = torch.zeros(64 * 1024, device="cuda")
    odd = x.view(torch.uint8)[1:]
    U, I, W = gb.GVA_ERR_UNSUPPORTED, gb.GVA_ERR_INVALID_ARG, gb.GVA_ERR_WORKSPACE
    with Handle(shape) as h:
        a = dict(used=t, want=t, pages_in=t, pages_out=t, table=t, most=4, pages=9, ring=t, free_in=t, free_out=t, lens=t, cu=t, pos=t, slots=t, rows=5, B=3)
        for k in ("used", "want", "pages_in", "pages_out", "table", "ring", "free_in", "free_out", "lens", "cu", "pos", "slots"):
            assert refused(h, "gva_assign_pages", a, **{k: None}) == I
            assert refused(h, "gva_assign_pages", a, **{k: odd}) == I
        for k in ("most", "pages", "rows", "B"):
            assert refused(h, "gva_assign_pages", a, **{k: -1}) == I
        assert refused(h, "gva_assign_pages", a, B=8193) == U and refused(h, "gva_assign_pages", a, pages=2 ** 25) == U
        a = dict(parents=t, cu=t, ctx=t, mask=t, words=1, pos=t, B=2, most=32)
        for k in ("parents", "cu", "mask"):
            assert refused(h, "gva_tree_masks", a, **{k: None}) == I and refused(h, "gva_tree_masks", a, **{k: odd}) == I
        assert refused(h, "gva_tree_masks", a, ctx=None) == I and refused(h, "gva_tree_masks", a, most=33) == I and refused(h, "gva_tree_masks", a, B=-1) == I
        assert refused(h, "gva_tree_masks", a, most=257, words=9) == U and refused(h, "gva_tree_masks", a, words=9) == U and refused(h, "gva_tree_masks", a, B=8193) == U
        cache = gb.make_gqa_cache(c.d[0], c.d[0], None, 4, 1)
        a = dict(cache=cache, q=x, qs=1024, k=x, ks=256, v=x, vs=256, pos=t, slots=t, out=x, n=3)
        for k in ("k", "v", "pos", "slots", "out", "q"):
            assert refused(h, "gqa_append", a, **{k: None}) == I and refused(h, "gqa_append", a, **{k: odd}) == I
        for k in ("qs", "ks", "vs"):
            assert refused(h, "gqa_append", a, **{k: a[k] - 4}) == I and refused(h, "gqa_append", a, **{k: a[k] + 2}) == I
        assert refused(h, "gqa_append", a, qs=2048) == I and refused(h, "gqa_append", a, n=-1) == I
        assert refused(h, "gqa_append", a, cache=gb.make_gqa_cache(None, c.d[0], None, 4, 1)) == I
        assert refused(h, "gqa_append", a, cache=gb.make_gqa_cache(c.d[0], c.d[0], None, 2 ** 25, 1)) == U
        a = dict(cache=c.c, v=x, kr=x, pos=t, slots=t, n=3)
        for k in ("v", "kr", "pos", "slots"):
            assert refused(h, "gva_append_rows", a, **{k: None}) == I and refused(h, "gva_append_rows", a, **{k: odd}) == I
        assert refused(h, "gva_append_rows", a, n=-1) == I
        q, ws = torch.zeros(8, 16, 80, dtype=torch.bfloat16, device="cuda"), torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
        a = dict(cache=c.c, q=q, mask=t, words=1, cu=t, ctx=t, out=q, lse=x, ws=ws, B=2, n=8, most=4, max_len=200, splits=0)
        for k in ("q", "mask", "cu", "ctx", "out"):
            assert refused(h, "gva_decode_tree", a, **{k: None}) == I and refused(h, "gva_decode_tree", a, **{k: odd}) == I
        assert refused(h, "gva_decode_tree", a, lse=odd) == I and refused(h, "gva_decode_tree", a, words=0) == I
        assert refused(h, "gva_decode_tree", a, ws=None) == W and refused(h, "gva_decode_tree", a, ws=ws[:64]) == W and refused(h, "gva_decode_tree", a, ws=ws[16:]) == I
        for k in ("B", "n", "most", "max_len", "splits"):
            assert refused(h, "gva_decode_tree", a, **{k: -1}) == I
        assert refused(h, "gva_decode_tree", a, most=257, words=9) == U and refused(h, "gva_decode_tree", a, B=8193) == U and refused(h, "gva_decode_tree", a, splits=65) == U
        assert refused(h, "gva_decode_tree", a, B=8192, most=256, words=8, max_len=2 ** 31 - 1) == U and refused(h, "gva_decode_tree", a, max_len=2 ** 30 + 1) == U
        assert gb.gva_decode_tree_workspace_bytes(h.h, 8193, 1, 1, 1) == 0 and gb.gva_decode_tree_workspace_bytes(h.h, 1, 1, 257, 1) == 0
        a = dict(cache=c.c, parents=t, tokens=t, chosen=t, cu=t, ctx=t, path=t, lens=t, last=t, B=2, most=8)
        for k in ("parents", "tokens", "chosen", "cu", "ctx", "path", "lens", "last"):
            assert refused(h, "gva_tree_commit", a, **{k: None}) == I and refused(h, "gva_tree_commit", a, **{k: odd}) == I
        assert refused(h, "gva_tree_commit", a, B=-1) == I and refused(h, "gva_tree_commit", a, most=257) == U and refused(h, "gva_tree_commit", a, B=8193) == U
        for kw in (dict(d_rot=12), dict(d_rot=72), dict(d_rot=128)):
            with pytest.raises(gb.GvaError) as e:
                gb.gqa_set_rope(h.h, gb.make_rope(**kw))
            assert e.value.status == U
        for kw in (dict(d_rot=8), dict(d_rot=16, layout=gb.GVA_ROPE_HALVES), dict(d_rot=16, magnitude=1.5)):
            with pytest.raises(gb.GvaError) as e:
                gb.gva_set_rope(h.h, gb.make_rope(**kw))
            assert e.value.status == U
        torch.cuda.synchronize()
        assert (t == 0).all()


# ---- together --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape,kind", [(wl.SHAPE_A, "bf16"), (wl.SHAPE_B, "bf16"), (wl.SHAPE_C, "f32"), (wl.SHAPE_A, "fp8")], ids=str)
def test_steps_with_trees_end_where_single_tokens_do(shape, kind):
    """Four steps of drafting over three sequences.  The model's choice is a function of the tokens so far, so the accepted tokens
    are known; after every commit the cache is what single tokens would have left, and the last accepted node's output is what
    attention over that cache gives."""
    B, P, most, N = 3, 64, 6, 18
    rng = np.random.default_rng(7)
    s, table_v, table_k = shape, rng.standard_normal((50, shape.G, shape.d_v)).astype(np.float32), rng.standard_normal((50, shape.d_r)).astype(np.float32)
    # a token's rows in the cache follow from it, its query too; what comes after a token is (3 t + 1) % 50
    table_q = rng.standard_normal((50, s.H, s.d_c)).astype(np.float32)
    table_qr = rng.standard_normal((50, s.H, s.d_r)).astype(np.float32)
    M = (rng.standard_normal((s.H, s.d_v, s.d_c)) / 8).astype(np.float32)
    said = lambda t: (3 * t + 1) % 50  # noqa: E731
    with Handle(s, page=P, dtype=DTYPE[kind]) as h:
        c = Cache(s, [0] * B, page=P, kind=kind, seed=0, paged=False, spare=N, room=1)
        v_pool, kr_pool = c.d
        pages = v_pool.shape[0]
        d_table, ring, free = zeros(B, most) - 1, ints(rng.permutation(pages)), ints([4, pages])
        cache = gb.make_cache(v_pool, kr_pool, d_table, pages, most)
        used, held, status, Md = zeros(B), zeros(B), zeros(1), dev(M)
        texts, roots = [[5], [17], [30]], [5, 17, 30]
        for step in range(4):
            sizes = [(9, 1, 20), (3, 33, 2), (16, 40, 0), (5, 5, 5)][step]
            parents, tokens = [], []
            for b, n in enumerate(sizes):
                par = random_parents(n, 10 * step + b, chain=0.4)
                tok = [roots[b]] + [said(0)] * (n - 1)
                for i in range(1, n):
                    tok[i] = said(tok[par[i]]) if rng.random() < 0.6 else int(rng.integers(0, 50))
                parents.append(par), tokens.append(tok[:n])
            n, top = sum(sizes), max(sizes)
            words = (top + 31) // 32
            flat = np.concatenate([np.asarray(t, dtype=np.int64) for t in tokens])
            ctx = used.clone()
            want = used + ints(sizes)
            cu, pos, slots, mask, tree_pos = zeros(B + 1), zeros(n), zeros(n), zeros(n, words), zeros(n)
            gb.gva_assign_pages(h.h, used, want, held, held, d_table, most, pages, ring, free, free, used, cu, pos, slots, n, B, status)
            gb.gva_tree_masks(h.h, ints(sum(parents, [])), cu, ctx, mask, words, tree_pos, B, top, status)
            q_abs = torch.empty(n, s.H, s.d_v + s.d_r, device="cuda")
            gb.gva_absorb_query(h.h, dev(table_q[flat]), dev(table_qr[flat]) if s.d_r else None, Md, tree_pos, q_abs, n)
            gb.gva_append_rows(h.h, cache, dev(table_v[flat]), dev(table_k[flat]) if s.d_r else None, tree_pos, slots, n, status)
            q = q_abs if kind == "f32" else q_abs.bfloat16()
            out, lse = torch.empty(n, s.H, s.d_v, dtype=q.dtype, device="cuda"), torch.empty(n, s.H, device="cuda")
            ws = torch.empty(gb.gva_decode_tree_workspace_bytes(h.h, B, n, top, most * P), dtype=torch.uint8, device="cuda")
            gb.gva_decode_tree(h.h, cache, q, mask, words, cu, ctx, out, lse, ws, B, n, top, most * P, 0, status)
            path, last = zeros(n), zeros(B)
            gb.gva_tree_commit(h.h, cache, ints(sum(parents, [])), ints(flat), ints([said(t) for t in flat]), cu, ctx, path, used, last, B, top, status)
            assert int(status.item()) == 0
            at = 0
            for b, m in enumerate(sizes):
                p, end = ref.commit(parents[b], tokens[b], [said(t) for t in tokens[b]])
                assert path[at:at + m].cpu().tolist() == p + [-1] * (m - len(p))
                if m:
                    texts[b] += [tokens[b][i] for i in p[1:]] + [end]
                    roots[b] = end
                assert int(used[b]) == len(texts[b]) - 1 and (not m or int(last[b]) == roots[b])
                assert all(said(a) == x for a, x in zip(texts[b], texts[b][1:]))
                at += m
            # the cache holds the texts (all but the newest token), as single appends would have left them
            lens = [len(t) - 1 for t in texts]
            alone = Cache(s, [most * P] * B, page=P, kind=kind, seed=1, paged=False)
            for b, t in enumerate(texts):
                k = np.asarray(t[:-1], dtype=np.int64)
                if len(k):
                    sl = alone.ids[b, np.arange(len(k)) // P] * P + np.arange(len(k)) % P
                    gb.gva_append_rows(h.h, alone.c, dev(table_v[k]), dev(table_k[k]) if s.d_r else None, ints(np.arange(len(k))), ints(sl), len(k), status)
            full = d_table.cpu().numpy()
            for got, w in zip([v_pool, kr_pool], alone.download()):
                got = got.cpu().numpy().view(w.dtype)
                for b in range(B):
                    for t in range(lens[b]):
                        assert np.array_equal(got[full[b, t // P], ..., t % P, :], w[alone.ids[b, t // P], ..., t % P, :])
            # ... and the last node that stayed saw exactly that
            o = torch.empty(B, s.H, s.d_v, device="cuda")
            l = torch.empty(B, s.H, device="cuda")
            rows = [sum(sizes[:b]) + ref.commit(parents[b], tokens[b], [said(t) for t in tokens[b]])[0][-1] if sizes[b] else 0 for b in range(B)]
            ws = torch.empty(gb.gva_decode_workspace_bytes(h.h, B, most * P), dtype=torch.uint8, device="cuda")
            gb.gva_decode(h.h, cache, q.float()[rows].contiguous(), used, o, l, ws, B, most * P, 0, status)
            for b in range(B):
                if sizes[b]:
                    assert (out[rows[b]].float() - o[b]).abs().max() <= (2e-5 if kind == "f32" else 2e-2) and (lse[rows[b]] - l[b]).abs().max() <= 1e-4
        # done: all pages come back
        gb.gva_assign_pages(h.h, used, zeros(B), held, held, d_table, most, pages, ring, free, free, used, cu, pos, slots, 1, B, status)
        f = free.cpu().tolist()
        assert f[1] == pages and sorted(ring.cpu().tolist()) == list(range(pages)) and int(status.item()) == 0


def test_a_whole_step_captured_and_replayed():
    """Pages, masks, rows, attention and commit in one graph, in place, against the same calls made one by one on a copy of the state."""
    shape, B, n, P, most = wl.SHAPE_A, 5, 7, 64, 8
    with Handle(shape, page=P) as h:
        def state():
            c = Cache(shape, [most * P] * B, page=P, kind="bf16", seed=3, paged=False, spare=0)
            x = {"v": c.d[0], "kr": c.d[1], "table": zeros(B, most) - 1, "ring": ints(np.random.default_rng(1).permutation(c.num_pages)), "free": ints([2, c.num_pages])}
            x.update({k: zeros(*v) for k, v in {"used": [B], "held": [B], "want": [B], "cu": [B + 1], "pos": [B * n], "slots": [B * n], "mask": [B * n, 1], "at": [B * n], "ctx": [B],
                                                "path": [B * n], "last": [B], "status": [1]}.items()})
            x["out"], x["lse"] = torch.zeros(B * n, 16, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(B * n, 16, device="cuda")
            x["ws"] = torch.zeros(gb.gva_decode_tree_workspace_bytes(h.h, B, B * n, n, most * P), dtype=torch.uint8, device="cuda")
            x["cache"] = gb.make_cache(x["v"], x["kr"], x["table"], c.num_pages, most)
            x["pages"] = c.num_pages
            return x

        rng = np.random.default_rng(4)
        inputs = {"parents": zeros(B * n), "tokens": zeros(B * n), "chosen": zeros(B * n), "v_new": torch.zeros(B * n, 4, 64, device="cuda"), "kr_new": torch.zeros(B * n, 16, device="cuda"),
                  "q": torch.zeros(B * n, 16, 80, dtype=torch.bfloat16, device="cuda")}

        def step(x):
            i = inputs
            x["ctx"].copy_(x["used"])
            torch.add(x["used"], n, out=x["want"])
            gb.gva_assign_pages(h.h, x["used"], x["want"], x["held"], x["held"], x["table"], most, x["pages"], x["ring"], x["free"], x["free"], x["used"], x["cu"], x["pos"], x["slots"], B * n, B,
                                x["status"])
            gb.gva_tree_masks(h.h, i["parents"], x["cu"], x["ctx"], x["mask"], 1, x["at"], B, n, x["status"])
            gb.gva_append_rows(h.h, x["cache"], i["v_new"], i["kr_new"], x["at"], x["slots"], B * n, x["status"])
            gb.gva_decode_tree(h.h, x["cache"], i["q"], x["mask"], 1, x["cu"], x["ctx"], x["out"], x["lse"], x["ws"], B, B * n, n, most * P, 0, x["status"])
            gb.gva_tree_commit(h.h, x["cache"], i["parents"], i["tokens"], i["chosen"], x["cu"], x["ctx"], x["path"], x["used"], x["last"], B, n, x["status"])

        one, two = state(), state()
        torch.cuda.synchronize()
        g, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g, stream=stream):
            step(one)
        for k in range(25):
            trees = [random_parents(n, 100 * k + b, chain=0.5) for b in range(B)]
            tokens, chosen = rng.integers(0, 3, (B, n)), rng.integers(0, 3, (B, n))
            for name, x in (("parents", ints(sum(trees, []))), ("tokens", ints(tokens.ravel())), ("chosen", ints(chosen.ravel())), ("v_new", torch.randn(B * n, 4, 64, device="cuda")),
                            ("kr_new", torch.randn(B * n, 16, device="cuda")), ("q", torch.randn(B * n, 16, 80, device="cuda").bfloat16())):
                inputs[name].copy_(x)
            torch.cuda.synchronize()
            g.replay()
            step(two)
            torch.cuda.synchronize()
            assert int(one["status"]) == int(two["status"]) == 0
            for name in ("v", "kr", "table", "ring", "free", "used", "held", "cu", "pos", "slots", "mask", "at", "path", "last", "out", "lse"):
                a, b = one[name], two[name]
                assert torch.equal(a.view(torch.int16) if a.dtype == torch.bfloat16 else a, b.view(torch.int16) if b.dtype == torch.bfloat16 else b), (k, name)
            paths = [ref.commit(t, a, b)[0] for t, a, b in zip(trees, tokens, chosen)]
            assert (one["used"] - one["ctx"]).tolist() == [len(x) for x in paths] and torch.isfinite(one["lse"]).all()
        del g


def test_commit_over_contiguous_pages():
    shape = wl.SHAPE_A
    with Handle(shape) as h:
        c = Cache(shape, [70, 70], kind="bf16", seed=5, paged=False)
        path, lens, last = zeros(8), zeros(2), zeros(2)
        gb.gva_tree_commit(h.h, c.c, ints([-1, 0, 0, 2] * 2), ints([1, 2, 3, 4] * 2), ints([3, 9, 4, 7] * 2), ints([0, 4, 8]), ints([62, 63]), path, lens, last, 2, 4)
        assert path.tolist() == [0, 2, 3, -1] * 2 and lens.tolist() == [65, 66] and last.tolist() == [7, 7]
        for w, g in zip(c.pools, c.download()):
            for b, ctx in ((0, 62), (1, 63)):
                for i, node in enumerate([0, 2, 3]):
                    d, s = ctx + i, ctx + node
                    assert np.array_equal(g[c.ids[b, d // 64], ..., d % 64, :], w[c.ids[b, s // 64], ..., s % 64, :])


def test_queries_and_keys_by_slot_map_feed_gqa_decode():
    H, G, d, P, lens = 16, 4, 64, 64, [130, 1, 64]
    rng = np.random.default_rng(3)
    n, pages = sum(lens), 8
    rope = dict(layout=gb.GVA_ROPE_HALVES, d_rot=32)
    with Handle(wl.SHAPE_A, page=P) as h:
        gb.gqa_set_rope(h.h, gb.make_rope(**rope))
        k_pool, v_pool = (torch.zeros(pages, G, P, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        table, ring, free = zeros(3, 3) - 1, ints(rng.permutation(pages)), ints([6, pages])
        used, held, cu, pos, slots, status = zeros(3), zeros(3), zeros(4), zeros(n), zeros(n), zeros(1)
        gb.gva_assign_pages(h.h, used, ints(lens), held, held, table, 3, pages, ring, free, free, used, cu, pos, slots, n, 3, status)
        qkv = rng.standard_normal((n, H + 2 * G, d)).astype(np.float32)
        x, q = dev(qkv), torch.empty(n, H, d, device="cuda")
        cache, row = gb.make_gqa_cache(k_pool, v_pool, table, pages, 3), (H + 2 * G) * d
        gb.gqa_append(h.h, cache, x, row, x[:, H:], row, x[:, H + G:], row, pos, slots, q, n, status)
        rows = np.cumsum(lens) - 1
        out, lse = torch.empty(3, H, d, device="cuda"), torch.empty(3, H, device="cuda")
        ws = torch.empty(gb.gva_decode_workspace_bytes(h.h, 3, 130), dtype=torch.uint8, device="cuda")
        gb.gqa_decode(h.h, cache, q[dev(rows)].contiguous(), used, out, lse, ws, 3, 130, 0, status)
        assert int(status.item()) == 0
        kq = ref.rotate(qkv[:, :H + G], np.concatenate([np.arange(t) for t in lens]), ref.frequencies(32), True)
        at = 0
        for b, t in enumerate(lens):
            bf = lambda a: wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(a.astype(np.float32))).astype(np.float64)  # noqa: E731
            kb, vb = bf(kq[at:at + t, H:]), bf(qkv[at:at + t, H + G:])
            for hh in range(H):
                s = kb[:, hh // 4] @ kq[at + t - 1, hh] / np.sqrt(d)
                p = np.exp(s - s.max())
                # keys next to a rounding border may lie a step of 2^-8 apart: a score off by 2^-8 |q| |k| scale / few elements, 1e-3 here
                assert np.abs(out[b, hh].cpu().numpy() - p @ vb[:, hh // 4] / p.sum()).max() <= 5e-3
            at += t
