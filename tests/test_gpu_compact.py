"""GPU parity of the 4-bit cache, the gathered attention weights and the eviction against the 64-bit references of
tests/compact_ref.py, which read the identical cached values.

Tolerances: codes, steps, moved rows and everything an eviction decides are exact.  Decode and weights are f32 arithmetic on
exact cached values, so the gates of the other decode tests apply: a score is a sum of d_v + d_r <= 160 products accumulated in f32
(relative error about sqrt(160) 2^-24 of the sum of magnitudes, which is some 6 after the softmax scale for unit rows:
5e-6 absolute), and a relative error of that size per weight is averaged over the tokens in the output: max-abs 2e-5,
relative L2 1e-5."""
import numpy as np
import pytest
import torch

from paper_2609_13285_b200 import binding as gb
from paper_2609_13285_b200 import workloads as wl
from tests import compact_ref as ref

pytestmark = pytest.mark.gpu

TOL_MAX, TOL_REL = 2e-5, 1e-5
EDGE = [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 640, 641, 1000]
SHAPES = [wl.SHAPE_A, wl.SHAPE_B, wl.SHAPE_C, wl.SHAPE_A0, wl.SHAPE_B0]
G1 = wl.HeadShape(H=4, G=1, d_v=64, d_c=64, d_r=16)
G1R = wl.HeadShape(H=4, G=1, d_v=64, d_c=64, d_r=24)
G3 = wl.HeadShape(H=12, G=3, d_v=64, d_c=64, d_r=24)
G8 = wl.HeadShape(H=32, G=8, d_v=64, d_c=64, d_r=16)
G2W = wl.HeadShape(H=8, G=2, d_v=128, d_c=128, d_r=32)


@pytest.fixture(scope="module", autouse=True)
def _built():
    from tests import gpu_util
    gpu_util.ensure_built()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ints(a):
    return dev(np.asarray(a, dtype=np.int32))


def bf16_values(bits):
    return wl.bf16_bits_to_f32(bits).astype(np.float64)


class Handle:
    def __init__(self, shape, page=64, dtype=gb.GVA_BF16):
        self.h = gb.gva_create(H=shape.H, G=shape.G, d_v=shape.d_v, d_c=shape.d_c, d_r=shape.d_r, page_size=page, cache_dtype=dtype)
        self.scale = (shape.d_c + shape.d_r) ** -0.5

    def __enter__(self):
        return self

    def __exit__(self, *a):
        torch.cuda.synchronize()
        gb.gva_destroy(self.h)


class Cache:
    """A cache of `lens` random tokens per sequence, in numpy and on the device.  Everything no live token occupies is poison."""

    def __init__(self, shape, lens, page=64, kind="q4", seed=0, paged=True, spare=2, gain=1.0, room=0):
        rng = np.random.default_rng(seed)
        s, self.shape, self.lens, self.page, self.kind = shape, shape, list(lens), page, kind
        B = len(lens)
        self.max_pages = max(1, max((n + room + page - 1) // page for n in lens))
        self.num_pages = B * self.max_pages + spare
        self.table = rng.permutation(self.num_pages)[: B * self.max_pages].reshape(B, self.max_pages).astype(np.int32) if paged else None
        full = self.table if paged else np.arange(B * self.max_pages, dtype=np.int32).reshape(B, self.max_pages)
        x = (rng.standard_normal((self.num_pages, s.G, page, s.d_v)) * gain).astype(np.float32)
        k = rng.standard_normal((self.num_pages, page, s.d_r)).astype(np.float32)
        self.ids = full
        live = np.zeros((self.num_pages, page), dtype=bool)
        for b, n in enumerate(lens):
            t = np.arange(n)
            live[full[b, t // page], t % page] = True
        dead = ~live
        if kind == "q4":
            c, st, z = ref.quantise(x)
            v = ref.pack(c)
            sz = np.stack([st, z], axis=-1)
            v[np.broadcast_to(dead[:, None], v.shape[:-1])] = 0xA5
            sz[np.broadcast_to(dead[:, None], sz.shape[:-1])] = np.nan
            kr = wl.f32_to_bf16_bits(k)
            kr[dead] = wl.BF16_NAN_BITS
            self.pools = [v, sz, kr]
        else:
            cast = {"bf16": wl.f32_to_bf16_bits, "fp8": wl.f32_to_e4m3_bits, "f32": lambda a: a.copy()}[kind]
            nan = {"bf16": wl.BF16_NAN_BITS, "fp8": np.uint8(0x7F), "f32": np.float32(np.nan)}[kind]
            v, kr = cast(x), cast(k)
            v[np.broadcast_to(dead[:, None], v.shape[:-1])] = nan
            kr[dead] = nan
            self.pools = [v, kr]
        self.upload()

    def upload(self):
        self.d = [dev(p.view(np.int16)) if p.dtype == np.uint16 else dev(p) for p in self.pools]
        self.d_table = None if self.table is None else dev(self.table)
        kr = self.d[-1] if self.shape.d_r else None
        if self.kind == "q4":
            self.c = gb.make_q4_cache(self.d[0], self.d[1], kr, self.d_table, self.num_pages, self.max_pages)
        else:
            self.c = gb.make_cache(self.d[0], kr, self.d_table, self.num_pages, self.max_pages)

    def download(self):
        return [t.cpu().numpy().view(p.dtype) for t, p in zip(self.d, self.pools)]

    def values(self, b, n, pools=None):
        """Values [n][G][d_v] and positional keys [n][d_r] of sequence b in 64 bits."""
        pools = self.pools if pools is None else pools
        r = [ref.rows_of(p, self.ids, b, n, self.page) for p in pools]
        if self.kind == "q4":
            return ref.widen(ref.unpack(r[0]), r[1][..., 0], r[1][..., 1]), bf16_values(r[2])
        return wl.pool_to_f64(r[0]), wl.pool_to_f64(r[1])


DTYPE = {"q4": gb.GVA_BF16, "bf16": gb.GVA_BF16, "fp8": gb.GVA_E4M3, "f32": gb.GVA_F32}


def queries(shape, rows, seed, gain=1.0):
    return (np.random.default_rng(seed).standard_normal((rows, shape.H, shape.d_v + shape.d_r)) * gain).astype(np.float32)


def decode(handle, cache, q, lens=None, num_splits=0, max_len=None):
    B = len(cache.lens)
    lens = cache.lens if lens is None else lens
    max_len = max(max(lens), 1) if max_len is None else max_len
    s = cache.shape
    out = torch.full((B, s.H, s.d_v), float("nan"), device="cuda")
    lse = torch.full((B, s.H), float("nan"), device="cuda")
    ws = torch.full((gb.gva_q4_decode_workspace_bytes(handle.h, B, max_len, num_splits),), 0xFF, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gb.gva_q4_decode(handle.h, cache.c, dev(q), ints(lens), out, lse, ws, B, max_len, num_splits, status)
    return out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64), int(status.item())


def check_decode(handle, cache, q, num_splits=0, lens=None, max_len=None, tol=TOL_MAX, rel=TOL_REL):
    lens = cache.lens if lens is None else lens
    out, lse, status = decode(handle, cache, q, lens, num_splits, max_len)
    assert status == 0
    want = [ref.attend(q[b].astype(np.float64), *cache.values(b, n), handle.scale) for b, n in enumerate(lens)]
    o, l = np.stack([w[0] for w in want]), np.stack([w[1] for w in want])
    assert np.isfinite(out).all()
    assert np.max(np.abs(out - o)) <= tol, np.max(np.abs(out - o))
    assert np.linalg.norm(out - o) <= rel * max(np.linalg.norm(o), 1e-30)
    live = np.isfinite(l)
    assert np.array_equal(np.isneginf(lse), ~live)
    assert np.max(np.abs(lse[live] - l[live]), initial=0) <= 1e-5 * max(1.0, np.max(np.abs(l[live]), initial=0))
    return out, lse


# ---- append ----------------------------------------------------------------------------------------------------------
def odd_rows(shape, n, seed):
    """Rows of many kinds: ordinary, tiny, huge, far from zero, of one value, on the borders between codes, with specials."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, shape.G, shape.d_v)).astype(np.float32)
    for i in range(n):
        kind = i % 12
        if kind == 1: x[i] *= np.float32(1e-5)
        if kind == 2: x[i] *= np.float32(1e5)
        if kind == 3: x[i] = 500 + 0.03 * x[i]
        if kind == 4: x[i] = np.float32(-1.37)
        if kind == 5: x[i] = 0
        if kind == 6: x[i] = rng.integers(0, 31, x[i].shape) * np.float32(0.5) - 3          # borders: ties
        if kind == 7: x[i, :, 3] = np.inf
        if kind == 8: x[i, :, 5], x[i, :, 6] = -np.inf, 7e4
        if kind == 9: x[i, -1, 0] = np.nan
        if kind == 10: x[i] = np.float32(1e-30) * x[i]
        if kind == 11: x[i, :, 1:] = -0.0
    return x


def expect_rows(cache, x, kr, places, pos):
    """What the pools hold once row i of x / kr has gone to (b, slot) = places[i] (None: nowhere)."""
    v, sz, k = [p.copy() for p in cache.pools]
    c, st, z = ref.quantise(x)
    rot = wl.f32_to_bf16_bits(np.zeros(kr.shape, np.float32)) if kr.shape[-1] == 0 else None
    for i, place in enumerate(places):
        if place is None:
            continue
        b, t = place
        pg, sl = cache.ids[b, t // cache.page], t % cache.page
        v[pg, :, sl] = ref.pack(c[i])
        sz[pg, :, sl, 0], sz[pg, :, sl, 1] = st[i], z[i]
        if rot is None:
            y = ref.rotate(kr[i], pos[i])
            k[pg, sl] = torch.from_numpy(y).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    return [v, sz, k]


def same_pools(got, want):
    for g, w in zip(got, want):
        if g.dtype == np.float16:
            both = np.isnan(g) & np.isnan(w)
            assert np.array_equal(np.where(both, 0, g.view(np.uint16)), np.where(both, 0, w.view(np.uint16)))
        else:
            assert np.array_equal(g, w)


@pytest.mark.parametrize("shape", SHAPES + [G1, G3, G8])
@pytest.mark.parametrize("offset", [0, 1])
def test_append_writes_the_nearest_codes_and_nothing_else(shape, offset):
    B = 24
    cache = Cache(shape, [100] * B, page=32, seed=1, room=40)
    x = odd_rows(shape, B, 2)
    kr = np.random.default_rng(3).standard_normal((B, shape.d_r)).astype(np.float32)
    slots = (np.arange(B) * 5) % 140
    pos = slots + 1000 * np.arange(B)
    with Handle(shape, 32) as h:
        xs = torch.zeros(x.size + 1, device="cuda")
        xs[offset:offset + x.size] = dev(x).reshape(-1)                 # offset 1: no 16-byte alignment
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        gb.gva_q4_append(h.h, cache.c, xs[offset:], dev(kr) if shape.d_r else None, ints(slots), ints(pos), B, status)
        assert int(status.item()) == 0
        same_pools(cache.download(), expect_rows(cache, x, kr, [(b, int(slots[b])) for b in range(B)], pos))


@pytest.mark.parametrize("shape", SHAPES + [G3])
def test_append_chunk_of_ragged_prompts(shape):
    q_lens, ctx = [0, 17, 1, 0, 70, 8, 0], [5, 60, 0, 3, 31, 64, 1]
    cache = Cache(shape, [c + q for c, q in zip(ctx, q_lens)], page=32, seed=4)
    n = sum(q_lens)
    x = odd_rows(shape, n + 5, 5)                                        # five rows behind the last sequence
    x[n:] = np.nan
    kr = np.random.default_rng(6).standard_normal((n + 5, shape.d_r)).astype(np.float32)
    cu = np.concatenate([[0], np.cumsum(q_lens)])
    for first in (None, [7 + 100 * b for b in range(len(ctx))]):
        cache.upload()
        places, pos = [], []
        for b in range(len(ctx)):
            places += [(b, ctx[b] + i) for i in range(q_lens[b])]
            pos += [(ctx[b] if first is None else first[b]) + i for i in range(q_lens[b])]
        with Handle(shape, 32) as h:
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            gb.gva_q4_append_chunk(h.h, cache.c, dev(x), dev(kr) if shape.d_r else None, ints(cu), ints(ctx), None if first is None else ints(first),
                                   len(ctx), n + 5, status)
            assert int(status.item()) == 0
            same_pools(cache.download(), expect_rows(cache, x, kr, places, pos))


def check_chunk(shape, rows, seed, B=37, page=32, offset=0):
    """A chunk large enough for `rows` input rows per block (a block takes n_q / (4 SMs), as many as its threads have shares
    for at most), over ragged sequences whose borders lie inside blocks, empty ones among them, the last block cut short
    by cu_q[B] < n_q."""
    rng = np.random.default_rng(seed)
    n_q = rows * 4 * torch.cuda.get_device_properties(0).multi_processor_count + 7
    share = rng.random(B) * (rng.random(B) < 0.8)
    q_lens = np.floor(share / share.sum() * (n_q - 5)).astype(np.int64)
    q_lens[int(np.argmax(q_lens))] += n_q - 5 - q_lens.sum()
    ctx = rng.integers(0, 100, B)
    cache = Cache(shape, list(ctx + q_lens), page=page, seed=seed + 1)
    n = int(q_lens.sum())
    x = odd_rows(shape, n_q, seed + 2)
    x[n:] = np.nan
    kr = rng.standard_normal((n_q, shape.d_r)).astype(np.float32)
    first = rng.integers(0, 100000, B)
    cu = np.concatenate([[0], np.cumsum(q_lens)])
    b = np.repeat(np.arange(B), q_lens)
    i = np.arange(n) - cu[b]
    pg, sl = cache.ids[b, (ctx[b] + i) // page], (ctx[b] + i) % page
    want = [p.copy() for p in cache.pools]
    c, st, z = ref.quantise(x[:n])
    want[0][pg, :, sl] = ref.pack(c)
    want[1][pg, :, sl] = np.stack([st, z], axis=-1)
    if shape.d_r:
        want[2][pg, sl] = ref.to_bf16_bits(ref.rotate(kr[:n], first[b] + i))
    with Handle(shape, page) as h:
        xs = torch.zeros(x.size + 1, device="cuda")
        xs[offset:offset + x.size] = dev(x).reshape(-1)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        gb.gva_q4_append_chunk(h.h, cache.c, xs[offset:], dev(kr) if shape.d_r else None, ints(cu), ints(ctx), ints(first), B, n_q, status)
        assert int(status.item()) == 0
        same_pools(cache.download(), want)


@pytest.mark.parametrize("rows", [85, 86, 127, 128, 130])
def test_append_chunk_of_one_group_with_the_widest_positional_slice(rows):
    # up to 128 rows to a block, 12 positional pairs to a row: 1020 pairs with 85 rows, 1032 with 86, 1536 at most
    check_chunk(G1R, rows, 300 + rows)


@pytest.mark.parametrize("rows,offset", [(2, 0), (5, 1), (1000, 0)])
@pytest.mark.parametrize("shape", [wl.SHAPE_A, wl.SHAPE_C, G1, G3])
def test_append_chunk_of_several_rows_per_block(shape, rows, offset):
    # 1000: as many rows as a block takes, one more block than that needs
    check_chunk(shape, min(rows, 8192 // (shape.G * shape.d_v) + 1), 400 + rows, offset=offset)


@pytest.mark.parametrize("rows", [2, 1000])
@pytest.mark.parametrize("shape", [wl.SHAPE_B, wl.SHAPE_A0, wl.SHAPE_B0, G8, G2W])
def test_append_chunk_of_several_rows_per_block_on_the_other_shapes(shape, rows):
    check_chunk(shape, min(rows, 8192 // (shape.G * shape.d_v) + 1), 500 + rows, B=19, page=64, offset=1 if rows == 2 else 0)


def test_append_reports_what_has_no_place_and_writes_the_rest():
    shape = wl.SHAPE_A
    cache = Cache(shape, [64] * 5, seed=7, room=64)
    cache.ids = cache.table.copy()
    cache.table[3, 0] = cache.num_pages                                  # a page that is not there
    cache.upload()
    x, kr = odd_rows(shape, 5, 8)[[0, 0, 0, 0, 0]], np.ones((5, 16), dtype=np.float32)
    slots, pos = [3, -1, 128, 9, 10], [3, 4, 5, 6, -2]
    with Handle(shape) as h:
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        gb.gva_q4_append(h.h, cache.c, dev(x), dev(kr), ints(slots), ints(pos), 5, status)
        got = int(status.item())
        assert (got & 0xFF, got >> 8) in {(gb.GVA_ERR_SEQ_LEN, 1), (gb.GVA_ERR_SEQ_LEN, 2), (gb.GVA_ERR_BAD_PAGE, 3), (gb.GVA_ERR_SEQ_LEN, 4)}
        same_pools(cache.download(), expect_rows(cache, x, kr, [(0, 3), None, None, None, None], pos))


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_append_at_is_append_where_slot_and_position_agree_and_turns_by_position_elsewhere(kind):
    shape = wl.SHAPE_A
    rng = np.random.default_rng(9)
    x, kr = rng.standard_normal((3, shape.G, shape.d_v)).astype(np.float32), rng.standard_normal((3, shape.d_r)).astype(np.float32)
    with Handle(shape, dtype=DTYPE[kind]) as h:
        a, b = Cache(shape, [70] * 3, kind=kind, seed=10), Cache(shape, [70] * 3, kind=kind, seed=10)
        gb.gva_append_cache(h.h, a.c, dev(x), dev(kr), ints([3, 69, 64]), 3)
        gb.gva_append_cache_at(h.h, b.c, dev(x), dev(kr), ints([3, 69, 64]), ints([3, 69, 64]), 3)
        assert all(np.array_equal(p.view(np.uint8), q.view(np.uint8)) for p, q in zip(a.download(), b.download()))
        # key turned to position 500, stored in slot 3: what append writes at 500, found at 3
        far = Cache(shape, [501] * 3, kind=kind, seed=11)
        gb.gva_append_cache(h.h, far.c, dev(x), dev(kr), ints([500] * 3), 3)
        gb.gva_append_cache_at(h.h, b.c, dev(x), dev(kr), ints([3] * 3), ints([500] * 3), 3)
        torch.cuda.synchronize()
        for i in range(3):
            for p, q in zip(b.download(), far.download()):
                assert np.array_equal(ref.rows_of(p, b.ids, i, 4, 64)[3].view(np.uint8), ref.rows_of(q, far.ids, i, 501, 64)[500].view(np.uint8))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        before = b.download()
        gb.gva_append_cache_at(h.h, b.c, dev(x), dev(kr), ints([4, 4000, -1]), ints([-1, 3, 3]), 3, status)
        assert int(status.item()) & 0xFF == gb.GVA_ERR_SEQ_LEN
        assert all(np.array_equal(p.view(np.uint8), q.view(np.uint8)) for p, q in zip(before, b.download()))


@pytest.mark.parametrize("kind,shape", [(k, s) for k in ("bf16", "fp8", "f32") for s in SHAPES + [G3] if not (k == "fp8" and s.d_r == 24)])
def test_append_at_on_every_head_shape(kind, shape):
    # the row that append writes at its position, in any slot, and nothing else
    rng = np.random.default_rng(110)
    B, slots, pos = 5, [0, 63, 64, 130, 7], [500, 0, 77, 130, 400]
    x, kr = rng.standard_normal((B, shape.G, shape.d_v)).astype(np.float32), rng.standard_normal((B, shape.d_r)).astype(np.float32)
    with Handle(shape, dtype=DTYPE[kind]) as h:
        near, far = Cache(shape, [140] * B, kind=kind, seed=111), Cache(shape, [501] * B, kind=kind, seed=112)
        keys = dev(kr) if shape.d_r else None
        gb.gva_append_cache(h.h, far.c, dev(x), keys, ints(pos), B)
        gb.gva_append_cache_at(h.h, near.c, dev(x), keys, ints(slots), ints(pos), B)
        got, at, want = near.download(), far.download(), [p.copy() for p in near.pools]
        for b in range(B):
            for w, f in zip(want, at):
                row = ref.rows_of(f, far.ids, b, 501, 64)[pos[b]]
                pg, sl = near.ids[b, slots[b] // 64], slots[b] % 64
                if w.ndim == 4: w[pg, :, sl] = row
                else: w[pg, sl] = row
        assert all(np.array_equal(g.view(np.uint8), w.view(np.uint8)) for g, w in zip(got, want))


# ---- widen -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape,page,paged", [(wl.SHAPE_A, 64, True), (wl.SHAPE_B, 32, True), (wl.SHAPE_C, 96, False), (wl.SHAPE_B0, 128, True), (G3, 64, True)])
def test_widen_rounds_each_value_once_and_leaves_the_rest(shape, page, paged):
    lens, starts = [0, 1, 33, 64, 200, 150, 7], [0, 0, 32, 0, 65, 150, 9]
    cache = Cache(shape, lens, page=page, seed=12, paged=paged, gain=3.0)
    wide = Cache(shape, lens, page=page, kind="bf16", seed=13, paged=True)
    with Handle(shape, page) as h:
        for st in (None, starts):
            wide.upload()
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            gb.gva_q4_widen(h.h, cache.c, wide.c, None if st is None else ints(st), ints(lens), len(lens), 100, status)     # a bound too low: still whole
            assert int(status.item()) == 0
            v, k = [p.copy() for p in wide.pools]
            for b, n in enumerate(lens):
                lo = st[b] if st else 0
                if lo >= n:
                    continue
                t = np.arange(lo, n)
                val, _ = cache.values(b, n)
                # z + s c in f32 (one rounding), then to bf16
                v[wide.ids[b, t // page], :, t % page] = wl.f32_to_bf16_bits(val[lo:].astype(np.float32))
                k[wide.ids[b, t // page], t % page] = ref.rows_of(cache.pools[2], cache.ids, b, n, page)[lo:]
            got = wide.download()
            assert np.array_equal(got[0], v) and np.array_equal(got[1], k)


@pytest.mark.parametrize("wide_pages", [4, 3])
def test_widen_of_lengths_beyond_the_block_tables_stops_at_their_end(wide_pages):
    shape, page = wl.SHAPE_A, 64
    cache = Cache(shape, [200, 256, 256, 64, 256], seed=160)
    wide = Cache(shape, [64 * wide_pages] * 5, kind="bf16", seed=161)
    lens = [200, 2 ** 31 - 1, 257, 64, 2 ** 31 - 1]
    starts = [0, 70, 0, 3, 2 ** 31 - 5]
    with Handle(shape) as h:
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        gb.gva_q4_widen(h.h, cache.c, wide.c, ints(starts), ints(lens), 5, 256, status)
        code = int(status.item())
        assert code & 0xFF == gb.GVA_ERR_SEQ_LEN and code >> 8 in ((1, 2, 4) if wide_pages == 4 else (0, 1, 2, 4))
        v, k = [p.copy() for p in wide.pools]
        for b in range(5):
            n = min(lens[b], page * wide_pages)
            if starts[b] >= n:
                continue
            t = np.arange(starts[b], n)
            val, _ = cache.values(b, n)
            v[wide.ids[b, t // page], :, t % page] = wl.f32_to_bf16_bits(val[t].astype(np.float32))
            k[wide.ids[b, t // page], t % page] = ref.rows_of(cache.pools[2], cache.ids, b, n, page)[t]
        got = wide.download()
        assert np.array_equal(got[0], v) and np.array_equal(got[1], k)


# ---- decode ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("num_splits", [0, 1, 5, 40])
def test_decode_ragged_edge_lengths(shape, num_splits):
    cache = Cache(shape, EDGE, seed=20)
    with Handle(shape) as h:
        check_decode(h, cache, queries(shape, len(EDGE), 21), num_splits)


@pytest.mark.parametrize("shape", [G1, G2W, G3, G8])
@pytest.mark.parametrize("page,paged", [(32, True), (64, False), (96, True), (256, True)])
def test_decode_group_counts_and_page_sizes(shape, page, paged):
    lens = [5, 64, 700, 2049, 0, 333]
    cache = Cache(shape, lens, page=page, seed=22, paged=paged)
    with Handle(shape, page) as h:
        for num_splits in (0, 3):
            check_decode(h, cache, queries(shape, len(lens), 23), num_splits)


@pytest.mark.parametrize("B,T", [(1, 1), (1, 97), (1, 20000), (3, 7000), (40, 300), (600, 70)])
def test_decode_batches_and_lengths(B, T):
    shape = wl.SHAPE_A
    cache = Cache(shape, [max(1, T - 3 * (b % 7)) for b in range(B)], seed=24)
    with Handle(shape) as h:
        check_decode(h, cache, queries(shape, B, 25))


@pytest.mark.parametrize("gain", [1e-4, 1.0, 300.0])
@pytest.mark.parametrize("shape", [wl.SHAPE_A, wl.SHAPE_B])
def test_decode_keeps_its_precision_at_any_size_of_the_values(gain, shape):
    # values scaled by `gain`, queries by 1 / gain: the same softmax, outputs scaled; the gates scale along
    lens = [300, 64, 1025]
    cache = Cache(shape, lens, seed=26, gain=gain)
    q = queries(shape, len(lens), 27)
    q[..., :shape.d_v] /= np.float32(gain)
    with Handle(shape) as h:
        check_decode(h, cache, q, tol=TOL_MAX * gain)


def test_decode_of_rows_of_very_different_steps():
    # tokens whose values are a thousand times smaller than their neighbours' keep theirs; rows of one value (step 0) among them
    shape = wl.SHAPE_A
    cache = Cache(shape, [512, 130], seed=28)
    v, sz, kr = cache.pools
    for b in range(2):
        for t in range(cache.lens[b]):
            pg, sl = cache.ids[b, t // 64], t % 64
            if t % 3 == 1: sz[pg, :, sl] *= np.float16(1e-3)
            if t % 3 == 2: sz[pg, :, sl, 0] = 0
    cache.upload()
    with Handle(shape) as h:
        check_decode(h, cache, queries(shape, 2, 29))


def test_decode_peaked_and_flat():
    shape, lens = wl.SHAPE_A, [500, 2049, 64]
    cache = Cache(shape, lens, seed=30)
    with Handle(shape) as h:
        check_decode(h, cache, queries(shape, 3, 31, gain=0.0))
        # scores thirty times larger carry thirty times the absolute error into the exponent
        check_decode(h, cache, queries(shape, 3, 31, gain=30.0), tol=30 * TOL_MAX, rel=30 * TOL_REL)


@pytest.mark.parametrize("shape", [wl.SHAPE_A, wl.SHAPE_B, wl.SHAPE_C])
def test_decode_every_dim_and_slot_lands_where_it_should(shape):
    T = 128
    cache = Cache(shape, [T] * shape.d_v, seed=32)
    v, sz, kr = cache.pools
    v[:], sz[..., 0], sz[..., 1], kr[:] = 0, 1, 0, 0
    for b in range(shape.d_v):
        t, g = (37 * b + 5) % T, b % shape.G
        v[cache.ids[b, t // 64], g, t % 64, b // 2] = 9 << (4 * (b % 2))
    cache.upload()
    with Handle(shape) as h:
        out, _, _ = decode(h, cache, queries(shape, shape.d_v, 33, gain=0.0))
        want = np.zeros_like(out)
        for b in range(shape.d_v):
            want[b, 4 * (b % shape.G):4 * (b % shape.G) + 4, b] = 9 / T
        assert np.max(np.abs(out - want)) <= 1e-6
    # and the score side: a query along one dim picks the token that has it (positional dims included)
    dims = shape.d_v + shape.d_r
    cache = Cache(shape, [64] * dims, seed=34)
    v, sz, kr = cache.pools
    v[:], sz[..., 0], sz[..., 1], kr[:] = 0, 1, 0, 0
    for d in range(dims):
        t = (7 * d + 3) % 64
        pg = cache.ids[d, 0]
        if d < shape.d_v: v[pg, :, t, d // 2] |= 15 << (4 * (d % 2))
        else: kr[pg, t, d - shape.d_v] = wl.f32_to_bf16_bits(np.array([15.0], np.float32))[0]
        mark = (d + 9) % shape.d_v
        v[pg, :, t, mark // 2] |= 1 << (4 * (mark % 2))
    cache.upload()
    q = np.zeros((dims, shape.H, dims), dtype=np.float32)
    for d in range(dims):
        q[d, :, d] = 60.0
    with Handle(shape) as h:
        out, _, _ = decode(h, cache, q)
        for d in range(dims):
            assert np.all(np.abs(out[d, :, (d + 9) % shape.d_v] - 1) < 1e-3), d


def test_decode_rows_with_nan_stay_with_their_head_and_sequence():
    shape = wl.SHAPE_A
    cache = Cache(shape, [200, 200], seed=35)
    cache.pools[1][cache.ids[0, 1], 2, 3, 1] = np.nan                    # sequence 0, group 2
    cache.upload()
    with Handle(shape) as h:
        out, lse, _ = decode(h, cache, queries(shape, 2, 36))
        assert np.isnan(out[0, 8:12]).all() and np.isnan(lse[0, 8:12]).all()
        assert np.isfinite(out[1]).all() and np.isfinite(np.delete(out[0], range(8, 12), axis=0)).all()


@pytest.mark.parametrize("num_splits", [0, 1, 3, 40])
@pytest.mark.parametrize("shape", [wl.SHAPE_A, wl.SHAPE_B])
def test_decode_nan_is_carried_however_the_sequences_are_split(shape, num_splits):
    # fifteen tiles each: a range of them holds nothing but what is NaN (a head's whole query, a row alone in the last tile, a
    # group's whole sequence), and a NaN is not an empty range
    lens = [900, 897, 900, 333]
    cache = Cache(shape, lens, seed=130)
    step = cache.pools[1]
    step[cache.ids[1, 896 // 64], 2, 896 % 64, 1] = np.nan
    step[cache.ids[2], 0, :, 1] = np.nan
    cache.upload()
    q = queries(shape, len(lens), 131)
    q[0, 5, 7], q[0, 6, 3], q[0, 7, -1] = np.nan, np.inf, np.nan
    nan = np.zeros((len(lens), shape.H), dtype=bool)
    nan[0, 5:8], nan[1, 8:12], nan[2, 0:4] = True, True, True
    with Handle(shape) as h:
        out, lse, status = decode(h, cache, q, num_splits=num_splits)
        assert status == 0
        assert np.array_equal(np.isnan(lse), nan) and np.array_equal(np.isnan(out), np.broadcast_to(nan[..., None], out.shape))
        for b, n in enumerate(lens):
            o, l = ref.attend(np.nan_to_num(q[b].astype(np.float64), nan=0, posinf=0), *cache.values(b, n), h.scale)
            live = ~nan[b]
            assert np.max(np.abs(out[b, live] - o[live])) <= TOL_MAX
            assert np.max(np.abs(lse[b, live] - l[live])) <= 1e-5 * np.max(np.abs(l[live]))


def test_decode_pages_beyond_four_gigabytes():
    shape, page = wl.SHAPE_A, 64
    pages = (5 << 30) // (shape.G * page * shape.d_v // 2)
    cache = Cache(shape, [130, 64], seed=37)
    far = np.array([[pages - 1, 3, pages - 7], [pages // 2, 0, 1]], dtype=np.int32)
    v = torch.zeros(pages, shape.G, page, shape.d_v // 2, dtype=torch.uint8, device="cuda")
    sz = torch.zeros(pages, shape.G, page, 2, dtype=torch.float16, device="cuda")
    kr = torch.zeros(pages, page, shape.d_r, dtype=torch.int16, device="cuda")
    for b in range(2):
        for j in range((cache.lens[b] + 63) // 64):
            for to, p in zip((v, sz, kr), cache.d):
                to[int(far[b, j])] = p[int(cache.ids[b, j])]
    table = dev(far)
    cache.c = gb.make_q4_cache(v, sz, kr, table, pages, 3)
    with Handle(shape) as h:
        check_decode(h, cache, queries(shape, 2, 38))


def test_three_thousand_sequences():
    shape, B = G1, 3000
    lens = [b % 71 for b in range(B)]
    cache = Cache(shape, lens, page=32, seed=46)
    with Handle(shape, 32) as h:
        check_decode(h, cache, queries(shape, B, 47))
        check_decode(h, cache, queries(shape, B, 47), num_splits=2)
    check_weights(shape, lens, "q4", [1 + b % 3 for b in range(B)], page=32)
    check_evict(shape, lens, [40] * B, page=32)


def test_decode_same_bits_every_time_and_on_a_side_stream():
    shape = wl.SHAPE_A
    cache = Cache(shape, [5000, 64, 1, 777], seed=39)
    q = queries(shape, 4, 40)
    with Handle(shape) as h:
        first = decode(h, cache, q)
        for _ in range(3):
            again = decode(h, cache, q)
            assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            again = decode(h, cache, q)
        assert np.array_equal(first[0], again[0])


def test_two_decodes_at_once_on_two_streams_of_one_handle():
    shape = wl.SHAPE_A
    caches = [Cache(shape, [3000, 64, 900], seed=41), Cache(shape, [64, 2500, 1], seed=42)]
    q = [queries(shape, 3, 43 + i) for i in range(2)]
    with Handle(shape) as h:
        alone = [decode(h, c, x, max_len=3000)[0] for c, x in zip(caches, q)]        # the same arguments as below
        streams = [torch.cuda.Stream() for _ in range(2)]
        lens, qs = [ints(c.lens) for c in caches], [dev(x) for x in q]
        outs = [torch.zeros(3, shape.H, shape.d_v, device="cuda") for _ in range(2)]
        ws = [torch.empty(gb.gva_q4_decode_workspace_bytes(h.h, 3, 3000), dtype=torch.uint8, device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(20):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    gb.gva_q4_decode(h.h, caches[i].c, qs[i], lens[i], outs[i], None, ws[i], 3, 3000)
        torch.cuda.synchronize()
        for i in range(2):
            assert np.array_equal(outs[i].cpu().numpy().astype(np.float64), alone[i])


def test_bad_lengths_and_pages_are_reported_and_the_rest_is_right():
    shape = wl.SHAPE_A
    cache = Cache(shape, [200, 300, 100, 64], seed=44)
    q = queries(shape, 4, 45)
    with Handle(shape) as h:
        out, lse, status = decode(h, cache, q, lens=[200, -5, cache.max_pages * 64 + 1, 64])
        assert status & 0xFF == gb.GVA_ERR_SEQ_LEN and status >> 8 in (1, 2)
        assert np.all(out[1:3] == 0) and np.isneginf(lse[1:3]).all()
        for b in (0, 3):
            o, _ = ref.attend(q[b].astype(np.float64), *cache.values(b, cache.lens[b]), h.scale)
            assert np.max(np.abs(out[b] - o)) <= TOL_MAX
        for page in (-1, cache.num_pages, 2 ** 31 - 1):
            table = cache.table.copy()
            cache.table[1, 2] = page
            cache.upload()
            out, lse, status = decode(h, cache, q)
            assert status == gb.GVA_ERR_BAD_PAGE | (1 << 8)
            for b in (0, 2, 3):
                o, _ = ref.attend(q[b].astype(np.float64), *cache.values(b, cache.lens[b]), h.scale)
                assert np.max(np.abs(out[b] - o)) <= TOL_MAX
            cache.table = table
    torch.cuda.synchronize()


# ---- gathered weights --------------------------------------------------------------------------------------------------
def check_weights(shape, lens, kind, rows, page=64, paged=True, seed=50, decay=0.5, alias=False, cu=True, gain=1.5, most=None):
    cache = Cache(shape, lens, page=page, kind=kind, seed=seed, paged=paged)
    rng = np.random.default_rng(seed + 1)
    B, n = len(lens), sum(rows)
    q = queries(shape, n, seed + 2, gain)
    cu_q = np.concatenate([[0], np.cumsum(rows)])
    stride = max(max(lens), 1) + 3
    before = rng.random((B, stride)).astype(np.float32)
    with Handle(shape, page, DTYPE[kind]) as h:
        lse, want = np.full((n, shape.H), -np.inf, dtype=np.float32), before.astype(np.float64).copy() if alias else np.full((B, stride), 7.0)
        for b in range(B):
            v, kr = cache.values(b, lens[b])
            R = rows[b]
            for i in range(R):
                m = lens[b] - (R - 1 - i)
                if m > 0:
                    lse[cu_q[b] + i] = ref.attend(q[cu_q[b] + i].astype(np.float64), v[:m], kr[:m], h.scale)[1]
            counted = lse[cu_q[b]:cu_q[b + 1]].astype(np.float64)
            if most is not None:
                counted[most:] = -np.inf                                     # rows that max_q_len cuts off add nothing
            want[b, :lens[b]] = ref.gathered(q[cu_q[b]:cu_q[b + 1]].astype(np.float64), counted, v, kr, h.scale, before[b, :lens[b]], decay)
        w_in = dev(before)
        w_out = w_in if alias else torch.full((B, stride), 7.0, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        call = gb.gva_q4_attention_weights if kind == "q4" else gb.gva_attention_weights
        call(h.h, cache.c, dev(q), dev(lse), ints(cu_q) if cu else None, ints(lens), decay, w_in, w_out, stride, B, max(max(rows), 1) if most is None else most, max(max(lens), 1), status)
        got = w_out.cpu().numpy().astype(np.float64)
        assert int(status.item()) == 0
        # a weight is exp of a difference that is off by 5e-6 (see above) plus the rounding of lse to f32 (2^-24 of some 8)
        assert np.max(np.abs(got - want) / np.maximum(np.abs(want), 1e-3)) <= 4e-5, np.max(np.abs(got - want) / np.maximum(np.abs(want), 1e-3))
        assert np.linalg.norm(got - want) <= TOL_REL * np.linalg.norm(want)
        return got


@pytest.mark.parametrize("kind,shape", [(k, s) for k in ("q4", "bf16", "fp8", "f32") for s in SHAPES if not (k == "fp8" and s is wl.SHAPE_C)])
def test_weights_of_one_row_at_edge_lengths(kind, shape):
    check_weights(shape, EDGE, kind, [1] * len(EDGE))
    check_weights(shape, EDGE, kind, [1] * len(EDGE), cu=False, alias=True)


@pytest.mark.parametrize("kind", ["q4", "bf16", "fp8", "f32"])
@pytest.mark.parametrize("shape", [wl.SHAPE_A, wl.SHAPE_B, G1, G8])
def test_weights_of_several_rows(kind, shape):
    check_weights(shape, [1, 3, 64, 200, 0, 129, 700], kind, [3, 5, 2, 33, 2, 0, 9], decay=0.0)


@pytest.mark.parametrize("page,paged", [(32, True), (64, False), (96, True), (256, True)])
@pytest.mark.parametrize("kind", ["q4", "bf16"])
def test_weights_page_sizes(page, paged, kind):
    check_weights(G3 if kind == "q4" else wl.SHAPE_C, [5, 64, 700, 0, 333], kind, [1, 2, 4, 1, 3], page=page, paged=paged)


def test_weights_of_one_long_sequence_and_of_many_short_ones():
    check_weights(wl.SHAPE_A, [20001], "q4", [2])
    check_weights(wl.SHAPE_A, [40 + b % 60 for b in range(400)], "q4", [1] * 400)


@pytest.mark.parametrize("kind", ["q4", "bf16", "f32"])
@pytest.mark.parametrize("most", [1, 2, 3])
def test_weights_count_the_first_rows_where_there_are_more(kind, most):
    check_weights(wl.SHAPE_A, [200, 64, 3], kind, [5, 1, 4], most=most)


@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 2, 5]])
@pytest.mark.parametrize("kind", ["q4", "bf16", "fp8", "f32"])
@pytest.mark.parametrize("shape", [wl.SHAPE_A, wl.SHAPE_B])
def test_weights_of_a_row_without_lse_add_nothing_whatever_its_query_holds(shape, kind, rows):
    # lse = -inf marks a (row, head) that attended to nothing: its query may be what the buffer held before
    lens = [200, 129, 77]
    cache = Cache(shape, lens, kind=kind, seed=150)
    rng = np.random.default_rng(151)
    cu_q = np.concatenate([[0], np.cumsum(rows)])
    n, stride = int(cu_q[-1]), 210
    q, before = queries(shape, n, 152), rng.random((3, stride)).astype(np.float32)
    with Handle(shape, dtype=DTYPE[kind]) as h:
        lse, want = np.full((n, shape.H), -np.inf, dtype=np.float32), before.astype(np.float64)
        dead = rng.random((n, shape.H)) < 0.3
        dead[cu_q[0]:cu_q[1]] = True                                     # sequence 0: nothing at all is added
        for b in range(3):
            v, kr = cache.values(b, lens[b])
            for i in range(rows[b]):
                m = lens[b] - (rows[b] - 1 - i)
                lse[cu_q[b] + i] = ref.attend(q[cu_q[b] + i].astype(np.float64), v[:m], kr[:m], h.scale)[1]
        lse[dead] = -np.inf
        for b in range(3):
            v, kr = cache.values(b, lens[b])
            at = slice(cu_q[b], cu_q[b + 1])
            want[b, :lens[b]] = ref.gathered(q[at].astype(np.float64), lse[at].astype(np.float64), v, kr, h.scale, before[b, :lens[b]], 0.5)
        q[dead] = rng.choice(np.array([np.nan, np.inf, 3e38], dtype=np.float32), (int(dead.sum()), 1))
        w_out = torch.full((3, stride), 7.0, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        call = gb.gva_q4_attention_weights if kind == "q4" else gb.gva_attention_weights
        call(h.h, cache.c, dev(q), dev(lse), ints(cu_q), ints(lens), 0.5, dev(before), w_out, stride, 3, max(rows), 200, status)
        assert int(status.item()) == 0
        got = w_out.cpu().numpy().astype(np.float64)
        assert np.array_equal(got[0, :200], before[0, :200].astype(np.float64) / 2)
        for b in range(3):
            assert np.max(np.abs(got[b, :lens[b]] - want[b, :lens[b]]) / np.maximum(want[b, :lens[b]], 1e-3)) <= 4e-5
            assert np.all(got[b, lens[b]:] == 7)


def test_weights_of_one_row_sum_to_the_number_of_heads():
    got = check_weights(wl.SHAPE_A, [3000], "q4", [1], decay=0.0, gain=3.0)
    assert abs(got[0, :3000].sum() - 16) <= 1e-4


def test_weights_report_bad_lengths_and_pages():
    shape = wl.SHAPE_A
    cache = Cache(shape, [200, 300, 100], seed=55)
    cache.table[1, 2] = -1
    cache.upload()
    q = queries(shape, 3, 56)
    with Handle(shape) as h:
        lse = torch.zeros(3, shape.H, device="cuda")
        w = torch.full((3, 310), 3.0, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        gb.gva_q4_attention_weights(h.h, cache.c, dev(q), lse, None, ints([200, 300, 311]), 0.5, w, w, 310, 3, 1, 310, status)
        code = int(status.item())
        assert (code & 0xFF, code >> 8) in {(gb.GVA_ERR_BAD_PAGE, 1), (gb.GVA_ERR_SEQ_LEN, 2)}
        got = w.cpu().numpy()
        assert np.all(got[2] == 3) and np.all(got[1, 128:192] == 1.5) and np.all(got[1, :128] > 1.5) and np.all(got[1, 192:300] > 1.5)


@pytest.mark.parametrize("rows", [1, 5])
@pytest.mark.parametrize("kind", ["q4", "bf16", "fp8", "f32"])
@pytest.mark.parametrize("shape", [wl.SHAPE_A, wl.SHAPE_B, wl.SHAPE_B0])
def test_every_bit_of_a_query_counts(shape, kind, rows):
    """Cached dims alternate between 1 and -1 and a query holds two numbers near 2^12 on a pair of them (a positional pair in every
    other head), so that a score is what their last bits leave.

    A score is then off by A = 2^12 softmax_scale times: 2 * 2^-24 for the product of both numbers with the scale, their two
    roundings to the operands (2^-22 each in two f16 parts, 2^-24 in f32 or three bf16 parts), and 2^-23 for each of the four
    additions that meet them (an accumulator that truncates).  Two bf16 parts would be off by up to 2 * 2^-18 A."""
    lens = [100, 64]
    cache = Cache(shape, lens, kind=kind, seed=120)
    plus = np.where(np.arange(shape.d_v) % 2 == 0, 1.0, -1.0).astype(np.float32)
    plus_r = np.where(np.arange(shape.d_r) % 2 == 0, 1.0, -1.0).astype(np.float32)
    cast = {"q4": wl.f32_to_bf16_bits, "bf16": wl.f32_to_bf16_bits, "fp8": wl.f32_to_e4m3_bits, "f32": lambda a: a}[kind]
    if kind == "q4":
        cache.pools[0][:] = 0x02                                           # value = -1 + 1 * (2 or 0)
        cache.pools[1][..., 0], cache.pools[1][..., 1] = 1, -1
    else:
        cache.pools[0][:] = cast(plus)
    cache.pools[-1][:] = cast(plus_r)
    cache.upload()
    rng, n = np.random.default_rng(121), 2 * rows
    q = np.zeros((n, shape.H, shape.d_v + shape.d_r), dtype=np.float32)
    for r in range(n):
        for h in range(shape.H):
            first, width = (shape.d_v, shape.d_r) if shape.d_r and h % 2 else (0, shape.d_v)
            i, j = 2 * rng.integers(0, width // 2), 2 * rng.integers(0, width // 2) + 1
            q[r, h, first + i] = 4096 * (1 + rng.random() / 64)
            q[r, h, first + j] = q[r, h, first + i] + np.float32(rng.standard_normal())
    cu_q = [0, rows, n]
    with Handle(shape, dtype=DTYPE[kind]) as h:
        off = 4200 * h.scale * (2 * 2.0 ** -24 + 2 * (2.0 ** -22 if kind in ("q4", "fp8") else 2.0 ** -24) + 4 * 2.0 ** -23)
        lse, want = np.zeros((n, shape.H), dtype=np.float32), []
        for b in range(2):
            v, kr = cache.values(b, lens[b])
            at = slice(cu_q[b], cu_q[b + 1])
            want.append(ref.gathered(q[at].astype(np.float64), lse[at].astype(np.float64), v, kr, h.scale, np.zeros(lens[b]), 0.0))
        w = torch.zeros(2, 100, device="cuda")
        call = gb.gva_q4_attention_weights if kind == "q4" else gb.gva_attention_weights
        call(h.h, cache.c, dev(q), dev(lse), ints(cu_q), ints(lens), 0.0, None, w, 100, 2, rows, 100)
        got = w.cpu().numpy().astype(np.float64)
        for b in range(2):
            assert np.max(np.abs(got[b, :lens[b]] / want[b] - 1)) <= off
        if kind == "q4" and rows == 1:                                     # the decode kernel's scores, by its lse
            for splits in (1, 2):
                _, got, _ = decode(h, cache, q, num_splits=splits)
                for b in range(2):
                    _, l = ref.attend(q[b].astype(np.float64), *cache.values(b, lens[b]), h.scale)
                    assert np.max(np.abs(got[b] - l)) <= off + 2.0 ** -22 * np.max(np.abs(l))


# ---- eviction ----------------------------------------------------------------------------------------------------------
def check_evict(shape, lens, keep, kind="q4", page=64, paged=True, sinks=2, recent=5, weights=None, positions=True, alias=True, seed=60, max_len=None):
    cache = Cache(shape, lens, page=page, kind=kind, seed=seed, paged=paged)
    rng = np.random.default_rng(seed + 1)
    B = len(lens)
    max_len = max(max(lens), 1) if max_len is None else max_len
    stride = max_len + 4
    w = (rng.random((B, stride)) if weights is None else weights((B, stride), rng)).astype(np.float32)
    pos = np.stack([rng.permutation(stride) * 2 for _ in range(B)]).astype(np.int32) if positions else np.broadcast_to(np.arange(stride, dtype=np.int32), (B, stride)).copy()
    nxt = np.array([pos[b, :n].max() + 1 if n else 0 for b, n in enumerate(lens)], dtype=np.int32)
    want_w, want_p = (w.copy(), pos.copy()) if alias else (np.full((B, stride), 9, np.float32), np.full((B, stride), 9, np.int32))
    if alias and not positions:
        want_p = np.full((B, stride), 9, np.int32)
    pools = [p.copy() for p in cache.pools]
    for b, n in enumerate(lens):
        moves, want_w[b, :n], want_p[b, :n] = ref.evict(w[b, :n], pos[b, :n], keep[b], int(nxt[b]), sinks, recent)
        for to, t in moves:
            for p, old in zip(pools, cache.pools):
                a, c = cache.ids[b, to // page], cache.ids[b, t // page]
                if p.ndim == 4: p[a, :, to % page] = old[c, :, t % page]
                else: p[a, to % page] = old[c, t % page]
    with Handle(shape, page, DTYPE[kind]) as h:
        w_in, p_in = dev(w), dev(pos)
        w_out = w_in if alias else torch.full((B, stride), 9.0, device="cuda")
        p_out = p_in if alias and positions else torch.full((B, stride), 9, dtype=torch.int32, device="cuda")
        seq = ints(lens)
        new = seq if alias else torch.full((B,), -7, dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.full((gb.gva_evict_workspace_bytes(h.h, B, max_len),), 0xFF, dtype=torch.uint8, device="cuda")
        call = gb.gva_q4_evict if kind == "q4" else gb.gva_evict
        call(h.h, cache.c, w_in, p_in if positions else None, seq, ints(keep), dev(nxt) if recent else None, sinks, recent, w_out, p_out, new, stride, ws, B, max_len, status)
        assert int(status.item()) == 0
        assert new.cpu().tolist() == [min(k, n) for k, n in zip(keep, lens)]
        assert np.array_equal(p_out.cpu().numpy(), want_p)
        assert np.array_equal(w_out.cpu().numpy(), want_w, equal_nan=True)
        for g, p in zip(cache.download(), pools):
            assert np.array_equal(g.view(np.uint8), p.view(np.uint8))


@pytest.mark.parametrize("kind,shape", [(k, s) for k in ("q4", "bf16", "fp8", "f32") for s in SHAPES if not (k == "fp8" and s is wl.SHAPE_C)])
def test_evict_edge_lengths(kind, shape):
    lens = EDGE
    check_evict(shape, lens, [max(0, n // 2) for n in lens], kind)
    check_evict(shape, lens, [max(0, n - 1) for n in lens], kind, alias=False, positions=False)


@pytest.mark.parametrize("keep", [0, 1, 63, 64, 299, 300, 301, 10 ** 9])
def test_evict_budgets(keep):
    check_evict(wl.SHAPE_A, [300, 300, 1, 0], [keep] * 4)
    check_evict(wl.SHAPE_A, [300, 300, 1, 0], [keep] * 4, alias=False, recent=0, sinks=0)


WEIGHTS = {
    "equal": lambda shape, rng: np.full(shape, 0.25),
    "few values": lambda shape, rng: rng.integers(0, 3, shape),
    "wide": lambda shape, rng: np.exp(8 * rng.standard_normal(shape)),
    "signs": lambda shape, rng: rng.standard_normal(shape) * (rng.random(shape) < 0.7) * np.where(rng.random(shape) < 0.5, -1.0, 1.0),
    "specials": lambda shape, rng: np.where(rng.random(shape) < 0.1, np.nan, np.where(rng.random(shape) < 0.1, np.inf, np.where(rng.random(shape) < 0.1, -np.inf, rng.random(shape)))),
    "neighbours": lambda shape, rng: (np.float32(1.0).view(np.uint32) + rng.integers(0, 40, shape).astype(np.uint32)).astype(np.uint32).view(np.float32),
}


@pytest.mark.parametrize("name", list(WEIGHTS))
@pytest.mark.parametrize("alias", [True, False])
def test_evict_ties_and_special_weights(name, alias):
    check_evict(wl.SHAPE_A, [2500, 1024, 77, 5000], [1200, 1000, 30, 4000], weights=WEIGHTS[name], alias=alias)


@pytest.mark.parametrize("sinks,recent", [(0, 0), (3, 0), (0, 50), (200, 200), (10 ** 6, 0)])
def test_evict_protects_the_first_and_the_last_positions(sinks, recent):
    check_evict(wl.SHAPE_A, [400, 90], [100, 80], sinks=sinks, recent=recent)


@pytest.mark.parametrize("page,paged", [(32, True), (64, False), (96, True), (256, False)])
def test_evict_page_sizes(page, paged):
    check_evict(G3, [700, 33], [300, 20], page=page, paged=paged)


@pytest.mark.parametrize("B,T", [(1, 70000), (1, 300000), (9, 9000), (200, 150)])
def test_evict_batches_and_lengths(B, T):
    # one sequence over several blocks, one beyond what they hold in shared memory, one block per sequence
    check_evict(G1, [T - 11 * (b % 5) for b in range(B)], [T // 3] * B, weights=WEIGHTS["few values"] if B == 9 else None)


def test_evict_leaves_bad_sequences_alone():
    shape = wl.SHAPE_A
    cache = Cache(shape, [200] * 5, seed=70)
    cache.table[1, 3] = cache.num_pages
    cache.upload()
    with Handle(shape) as h:
        w = torch.rand(5, 200, device="cuda")
        p = torch.arange(200, dtype=torch.int32, device="cuda").repeat(5, 1)
        lens, new = ints([200, 200, 201, 200, -1]), ints([0] * 5)
        w0, p0 = w.clone(), p.clone()
        ws = torch.empty(gb.gva_evict_workspace_bytes(h.h, 5, 200), dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        gb.gva_q4_evict(h.h, cache.c, w, p, lens, ints([100, 100, 100, -1, 100]), None, 0, 0, w, p, new, 200, ws, 5, 200, status)
        code = int(status.item())
        assert (code & 0xFF, code >> 8) in {(gb.GVA_ERR_BAD_PAGE, 1), (gb.GVA_ERR_SEQ_LEN, 2), (gb.GVA_ERR_SEQ_LEN, 3), (gb.GVA_ERR_SEQ_LEN, 4)}
        assert new.cpu().tolist() == [100, 200, 201, 200, -1]
        assert torch.equal(w[1:], w0[1:]) and torch.equal(p[1:], p0[1:]) and not torch.equal(w[0], w0[0])
        got = cache.download()
        for b in range(1, 5):
            for j in range(4):
                if b == 1 and j == 3:
                    continue
                assert all(np.array_equal(a[cache.table[b, j]].view(np.uint8), c[cache.table[b, j]].view(np.uint8)) for a, c in zip(got, cache.pools))


@pytest.mark.parametrize("kind", ["q4", "bf16"])
@pytest.mark.parametrize("T", [200, 20000])
def test_evict_with_a_negative_budget_hands_weights_and_positions_on(kind, T):
    # the sequence stays as it is, and so the outputs say, when they are other buffers than the inputs
    shape = wl.SHAPE_A
    cache = Cache(shape, [T, T - 7, 5], kind=kind, seed=140)
    with Handle(shape) as h:
        w, p = torch.rand(3, T, device="cuda"), torch.randint(0, 10 ** 6, (3, T), dtype=torch.int32, device="cuda")
        w2, p2, new = torch.full_like(w, 9.0), torch.full_like(p, 9), ints([0, 0, 0])
        ws = torch.empty(gb.gva_evict_workspace_bytes(h.h, 3, T), dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        call = gb.gva_q4_evict if kind == "q4" else gb.gva_evict
        call(h.h, cache.c, w, p, ints([T, T - 7, 5]), ints([T, -3, -2 ** 31]), None, 0, 0, w2, p2, new, T, ws, 3, T, status)
        code = int(status.item())
        assert code & 0xFF == gb.GVA_ERR_SEQ_LEN and code >> 8 in (1, 2)
        assert new.cpu().tolist() == [T, T - 7, 5]
        for b, n in enumerate([T, T - 7, 5]):
            assert torch.equal(w2[b, :n], w[b, :n]) and torch.equal(p2[b, :n], p[b, :n])
            assert torch.all(w2[b, n:] == 9) and torch.all(p2[b, n:] == 9)
        assert all(np.array_equal(g.view(np.uint8), q.view(np.uint8)) for g, q in zip(cache.download(), cache.pools))


def test_bounds_up_to_the_largest_number():
    """max_seq_len is a bound: one that nobody made an effort for gives what a close one gives."""
    shape, most = wl.SHAPE_A, 2 ** 31 - 1
    lens = [200, 70]
    cache, wide = Cache(shape, lens, seed=170), [Cache(shape, lens, kind="bf16", seed=171) for _ in range(2)]
    q = queries(shape, 2, 172)
    with Handle(shape) as h:
        check_decode(h, cache, q, max_len=most)
        for w, bound in zip(wide, (most, 200)):
            gb.gva_q4_widen(h.h, cache.c, w.c, None, ints(lens), 2, bound)
        assert all(np.array_equal(a, b) for a, b in zip(wide[0].download(), wide[1].download()))
        for bound in (2 ** 30 + 1, most):
            assert gb.gva_evict_workspace_bytes(h.h, 1, bound) == 0
            w, i, ws = torch.zeros(1, 200, device="cuda"), ints([200]), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
            assert gb.gva_q4_evict(h.h, cache.c, w, None, i, i, None, 0, 0, w, i, i, bound, ws, 1, bound, check=False) == gb.GVA_ERR_UNSUPPORTED
    row = torch.empty(most, device="cuda")
    for kind in ("q4", "f32"):
        one = Cache(shape, [200], kind=kind, seed=173)
        with Handle(shape, dtype=DTYPE[kind]) as h:
            call = gb.gva_q4_attention_weights if kind == "q4" else gb.gva_attention_weights
            near, lse = torch.zeros(200, device="cuda"), torch.full((1, shape.H), 5.0, device="cuda")
            call(h.h, one.c, dev(q[:1]), lse, None, ints([200]), 0.0, None, near, 200, 1, 1, 200)
            call(h.h, one.c, dev(q[:1]), lse, None, ints([200]), 0.0, None, row, most, 1, 1, most)
            assert torch.equal(row[:200], near) and float(near.sum()) > 0


# ---- refusals ----------------------------------------------------------------------------------------------------------
def test_refusals():
    shape = wl.SHAPE_A
    cache, wide = Cache(shape, [100, 50], seed=80), Cache(shape, [100, 50], kind="bf16", seed=81)
    x, kr, q = torch.zeros(2, 4, 64, device="cuda"), torch.zeros(2, 16, device="cuda"), torch.zeros(2, 16, 80, device="cuda")
    i, out, lse, w = ints([3, 4]), torch.zeros(2, 16, 64, device="cuda"), torch.zeros(2, 16, device="cuda"), torch.zeros(2, 100, device="cuda")
    p = torch.zeros(2, 100, dtype=torch.int32, device="cuda")
    INV, UNS, WS = gb.GVA_ERR_INVALID_ARG, gb.GVA_ERR_UNSUPPORTED, gb.GVA_ERR_WORKSPACE
    no = dict(check=False)
    with Handle(shape) as h, Handle(shape, dtype=gb.GVA_F32) as f32:
        ws = torch.empty(max(gb.gva_q4_decode_workspace_bytes(h.h, 2, 100), gb.gva_evict_workspace_bytes(h.h, 2, 100)), dtype=torch.uint8, device="cuda")
        c = cache.c
        # a handle of another cache type
        assert gb.gva_q4_append(f32.h, c, x, kr, i, i, 2, **no) == UNS
        assert gb.gva_q4_append_chunk(f32.h, c, x, kr, i, i, None, 1, 2, **no) == UNS
        assert gb.gva_q4_widen(f32.h, c, wide.c, None, i, 2, 100, **no) == UNS
        assert gb.gva_q4_decode(f32.h, c, q, i, out, lse, ws, 2, 100, **no) == UNS
        assert gb.gva_q4_attention_weights(f32.h, c, q, lse, None, i, 1.0, w, w, 100, 2, 1, 100, **no) == UNS
        assert gb.gva_q4_evict(f32.h, c, w, p, i, i, None, 0, 0, w, p, i, 100, ws, 2, 100, **no) == UNS
        # missing and misaligned pointers
        for bad in (gb.make_q4_cache(None, cache.d[1], cache.d[2], None, 9, 2), gb.make_q4_cache(cache.d[0], None, cache.d[2], None, 9, 2),
                    gb.make_q4_cache(cache.d[0], cache.d[1], None, None, 9, 2), gb.make_q4_cache(cache.d[0].view(-1)[8:], cache.d[1], cache.d[2], None, 9, 2),
                    gb.make_q4_cache(cache.d[0], cache.d[1].view(-1)[2:], cache.d[2], None, 9, 2), gb.make_q4_cache(cache.d[0], cache.d[1], cache.d[2], None, 0, 2),
                    gb.make_q4_cache(cache.d[0], cache.d[1], cache.d[2], None, 9, 0)):
            assert gb.gva_q4_append(h.h, bad, x, kr, i, i, 2, **no) == INV
            assert gb.gva_q4_decode(h.h, bad, q, i, out, lse, ws, 2, 100, **no) == INV
            assert gb.gva_q4_evict(h.h, bad, w, p, i, i, None, 0, 0, w, p, i, 100, ws, 2, 100, **no) == INV
        assert gb.gva_q4_append(h.h, c, None, kr, i, i, 2, **no) == INV
        assert gb.gva_q4_append(h.h, c, x, None, i, i, 2, **no) == INV
        assert gb.gva_q4_append(h.h, c, x, kr, None, i, 2, **no) == INV
        assert gb.gva_q4_append(h.h, c, x, kr, i, i, -1, **no) == INV
        assert gb.gva_append_cache_at(h.h, wide.c, x, kr, i, None, 2, **no) == INV
        assert gb.gva_q4_append_chunk(h.h, c, x, kr, None, i, None, 1, 2, **no) == INV
        assert gb.gva_q4_append_chunk(h.h, c, x, kr, i, i, None, 1, -2, **no) == INV
        assert gb.gva_q4_widen(h.h, c, gb.make_cache(None, wide.d[1], None, 9, 2), None, i, 2, 100, **no) == INV
        assert gb.gva_q4_widen(h.h, c, wide.c, None, None, 2, 100, **no) == INV
        assert gb.gva_q4_decode(h.h, c, q, i, None, lse, ws, 2, 100, **no) == INV
        assert gb.gva_q4_decode(h.h, c, q.view(-1)[1:], i, out, lse, ws, 2, 100, **no) == INV
        assert gb.gva_q4_decode(h.h, c, q, i, out, lse, ws, 2, 100, num_splits=-1, **no) == INV
        assert gb.gva_q4_decode(h.h, c, q, i, out, lse, ws[:64], 2, 100, num_splits=3, **no) == WS
        assert gb.gva_q4_decode(h.h, c, q, i, out, lse, None, 2, 100, num_splits=3, **no) == WS
        assert gb.gva_q4_decode(h.h, c, q, i, out, lse, ws, 9000, 100, **no) == UNS
        for decay in (-0.5, float("inf"), float("nan")):
            assert gb.gva_q4_attention_weights(h.h, c, q, lse, None, i, decay, w, w, 100, 2, 1, 100, **no) == INV
        assert gb.gva_q4_attention_weights(h.h, c, q, lse, None, i, 1.0, w, w, 99, 2, 1, 100, **no) == INV
        assert gb.gva_q4_attention_weights(h.h, c, q, None, None, i, 1.0, w, w, 100, 2, 1, 100, **no) == INV
        assert gb.gva_attention_weights(h.h, wide.c, q, lse, None, i, 1.0, w, None, 100, 2, 1, 100, **no) == INV
        assert gb.gva_q4_evict(h.h, c, w, p, i, i, None, 0, 5, w, p, i, 100, ws, 2, 100, **no) == INV         # recent without next_pos
        assert gb.gva_q4_evict(h.h, c, w, p, i, i, None, -1, 0, w, p, i, 100, ws, 2, 100, **no) == INV
        assert gb.gva_q4_evict(h.h, c, w, p, i, None, None, 0, 0, w, p, i, 100, ws, 2, 100, **no) == INV
        assert gb.gva_q4_evict(h.h, c, w, p, i, i, None, 0, 0, w, p, i, 99, ws, 2, 100, **no) == INV
        assert gb.gva_q4_evict(h.h, c, w, p, i, i, None, 0, 0, w, p, i, 100, ws[:128], 2, 100, **no) == WS
        assert gb.gva_evict(h.h, wide.c, w, p, i, i, None, 0, 0, w, p, i, 100, ws[128:], 2, 100, workspace_bytes=1 << 20, **no) == INV
        # nothing to do
        assert gb.gva_q4_decode(h.h, c, None, None, None, None, None, 0, 100) == 0
        assert gb.gva_q4_append(h.h, c, None, None, None, None, 0) == 0
        assert gb.gva_q4_evict(h.h, c, None, None, None, None, None, 0, 0, None, None, None, 0, None, 0, 0) == 0
        torch.cuda.synchronize()
        same_pools(cache.download(), cache.pools)


# ---- a run of them together --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind,shape", [("q4", wl.SHAPE_A), ("q4", wl.SHAPE_B), ("bf16", wl.SHAPE_A), ("fp8", wl.SHAPE_A)])
def test_serving_loop_with_a_budget(kind, shape):
    """Prompts enter the cache, tokens are decoded, weights gathered every step, and whenever a sequence is over its
    budget the least attended tokens leave; a plain simulation in 64 bits goes along."""
    rng = np.random.default_rng(90)
    page, budget, over, steps, B = 64, 150, 8, 24, 3
    prompt = [140, 155, 97]
    cache = Cache(shape, [0] * B, page=page, kind=kind, seed=91, room=256)
    stride = cache.max_pages * page
    with Handle(shape, page, DTYPE[kind]) as h:
        lens, pos = list(prompt), list(prompt)
        w, p = torch.zeros(B, stride, device="cuda"), torch.full((B, stride), -1, dtype=torch.int32, device="cuda")
        sim_p = [np.arange(n, dtype=np.int32) for n in prompt]
        sim_w = [np.zeros(n) for n in prompt]
        for b in range(B):
            p[b, :prompt[b]] = torch.arange(prompt[b], device="cuda")
        n = sum(prompt)
        x, kr = rng.standard_normal((n, shape.G, shape.d_v)).astype(np.float32), rng.standard_normal((n, shape.d_r)).astype(np.float32)
        cu = np.concatenate([[0], np.cumsum(prompt)])
        if kind == "q4":
            gb.gva_q4_append_chunk(h.h, cache.c, dev(x), dev(kr), ints(cu), ints([0] * B), None, B, n)
        else:
            gb.gva_append_chunk(h.h, cache.c, dev(x), dev(kr), ints(cu), ints([0] * B), B, n)
        out, lse = torch.zeros(B, shape.H, shape.d_v, device="cuda"), torch.zeros(B, shape.H, device="cuda")
        bytes_of = gb.gva_q4_decode_workspace_bytes if kind == "q4" else gb.gva_decode_workspace_bytes
        ws = torch.empty(bytes_of(h.h, B, stride), dtype=torch.uint8, device="cuda")
        ews = torch.empty(gb.gva_evict_workspace_bytes(h.h, B, stride), dtype=torch.uint8, device="cuda")
        rows = [[ref.rows_of(a, cache.ids, b, lens[b], page) for a in cache.download()] for b in range(B)]
        evictions = 0
        for step in range(steps):
            x, kr = rng.standard_normal((B, shape.G, shape.d_v)).astype(np.float32), rng.standard_normal((B, shape.d_r)).astype(np.float32)
            q = queries(shape, B, 1000 + step, 2.0)
            append = gb.gva_q4_append if kind == "q4" else gb.gva_append_cache_at
            append(h.h, cache.c, dev(x), dev(kr), ints(lens), ints(pos), B)
            for b in range(B):
                p[b, lens[b]] = pos[b]
                sim_p[b], sim_w[b] = np.append(sim_p[b], np.int32(pos[b])), np.append(sim_w[b], 0.0)
                lens[b] += 1
                pos[b] += 1
            seq = ints(lens)
            if kind == "q4":
                gb.gva_q4_decode(h.h, cache.c, dev(q), seq, out, lse, ws, B, stride)
                gb.gva_q4_attention_weights(h.h, cache.c, dev(q), lse, None, seq, 0.9, w, w, stride, B, 1, stride)
            else:
                gb.gva_decode(h.h, cache.c, dev(q), seq, out, lse, ws, B, stride)
                gb.gva_attention_weights(h.h, cache.c, dev(q), lse, None, seq, 0.9, w, w, stride, B, 1, stride)
            got = cache.download()
            for b in range(B):
                rows[b] = [np.concatenate([a, ref.rows_of(g, cache.ids, b, lens[b], page)[-1:]]) for a, g in zip(rows[b], got)]
                if kind == "q4":
                    v, k = ref.widen(ref.unpack(rows[b][0]), rows[b][1][..., 0], rows[b][1][..., 1]), bf16_values(rows[b][2])
                else:
                    v, k = wl.pool_to_f64(rows[b][0]), wl.pool_to_f64(rows[b][1])
                o, l = ref.attend(q[b].astype(np.float64), v, k, h.scale)
                assert np.max(np.abs(out[b].cpu().numpy() - o)) <= 2 * TOL_MAX
                sim_w[b] = ref.gathered(q[b:b + 1].astype(np.float64), l[None], v, k, h.scale, sim_w[b], 0.9)
                # each step within the gate, and the decay bounds their sum to ten of them
                assert np.max(np.abs(w[b, :lens[b]].cpu().numpy() - sim_w[b])) <= 4e-5 * max(1.0, sim_w[b].max()) * 10
            if max(lens) > budget + over:
                evictions += 1
                w_now = w.cpu().numpy()
                keep = [budget] * B
                call = gb.gva_q4_evict if kind == "q4" else gb.gva_evict
                call(h.h, cache.c, w, p, seq, ints(keep), ints(pos), 4, 16, w, p, seq, stride, ews, B, stride)
                for b in range(B):
                    moves, new_w, new_p = ref.evict(w_now[b, :lens[b]], sim_p[b], keep[b], pos[b], 4, 16)
                    for to, t in moves:
                        for a in rows[b]:
                            a[to] = a[t]
                        sim_w[b][to] = sim_w[b][t]
                    lens[b] = min(keep[b], lens[b])
                    rows[b] = [a[:lens[b]] for a in rows[b]]
                    sim_p[b], sim_w[b] = new_p[:lens[b]], sim_w[b][:lens[b]]
                    assert np.array_equal(p[b, :lens[b]].cpu().numpy(), sim_p[b])
                assert seq.cpu().tolist() == lens
        assert evictions >= 2


def test_a_chunk_prefilled_over_a_widened_context():
    """A second chunk of a prompt whose first part is held in 4 bits: widen, append the chunk to the bf16 pages, prefill,
    and put the chunk into the 4-bit cache."""
    shape, page, ctx, q_len = wl.SHAPE_A, 64, [200, 63], [40, 70]
    rng = np.random.default_rng(95)
    cache = Cache(shape, ctx, seed=96, room=100)
    wide = Cache(shape, [0, 0], kind="bf16", seed=97, room=300)
    n = sum(q_len)
    cu = ints([0, q_len[0], n])
    x, kr = rng.standard_normal((n, shape.G, shape.d_v)).astype(np.float32), rng.standard_normal((n, shape.d_r)).astype(np.float32)
    q = queries(shape, n, 98)
    with Handle(shape) as h:
        out, lse = torch.zeros(n, shape.H, shape.d_v, device="cuda"), torch.zeros(n, shape.H, device="cuda")
        gb.gva_q4_widen(h.h, cache.c, wide.c, None, ints(ctx), 2, 200)
        gb.gva_append_chunk(h.h, wide.c, dev(x), dev(kr), cu, ints(ctx), 2, n)
        gb.gva_prefill(h.h, wide.c, dev(q), cu, ints(ctx), out, lse, 2, max(q_len))
        gb.gva_q4_append_chunk(h.h, cache.c, dev(x), dev(kr), cu, ints(ctx), None, 2, n)
        got = wide.download()
        row = 0
        for b in range(2):
            v, k = wide.values(b, ctx[b] + q_len[b], got)
            exact, _ = cache.values(b, ctx[b])
            assert np.max(np.abs(v[:ctx[b]] - exact)) <= np.max(np.abs(exact)) * 2.0 ** -8
            for i in range(q_len[b]):
                o, _ = ref.attend(q[row].astype(np.float64), v[:ctx[b] + i + 1], k[:ctx[b] + i + 1], h.scale)
                assert np.max(np.abs(out[row].cpu().numpy() - o)) <= 2e-2           # the prefill kernel's contract
                row += 1
        # the 4-bit cache has gone on: decode over context and chunk
        lens = [c + m for c, m in zip(ctx, q_len)]
        cache.pools, cache.lens = cache.download(), lens
        check_decode(h, cache, queries(shape, 2, 99))


@pytest.mark.parametrize("kind", ["q4", "bf16"])
def test_a_captured_step_replays_on_new_lengths(kind):
    """append, decode, gather and evict captured once; replayed after the inputs in the same buffers have changed."""
    shape, page = wl.SHAPE_A, 64
    with Handle(shape, page, DTYPE[kind]) as h:
        cache = Cache(shape, [900, 200], kind=kind, seed=100, room=64)
        B, stride = 2, cache.max_pages * page
        x, kr, q = torch.zeros(B, 4, 64, device="cuda"), torch.zeros(B, 16, device="cuda"), torch.zeros(B, 16, 80, device="cuda")
        slots, pos, seq, keep, new = ints([0, 0]), ints([0, 0]), ints([1, 1]), ints([100, 100]), ints([0, 0])
        out, lse = torch.zeros(B, 16, 64, device="cuda"), torch.zeros(B, 16, device="cuda")
        w, w2 = torch.zeros(B, stride, device="cuda"), torch.zeros(B, stride, device="cuda")
        p2 = torch.zeros(B, stride, dtype=torch.int32, device="cuda")
        bytes_of = gb.gva_q4_decode_workspace_bytes if kind == "q4" else gb.gva_decode_workspace_bytes
        ws = torch.empty(bytes_of(h.h, B, stride), dtype=torch.uint8, device="cuda")
        ews = torch.empty(gb.gva_evict_workspace_bytes(h.h, B, stride), dtype=torch.uint8, device="cuda")

        def step():
            if kind == "q4":
                gb.gva_q4_append(h.h, cache.c, x, kr, slots, pos, B)
                gb.gva_q4_decode(h.h, cache.c, q, seq, out, lse, ws, B, stride)
                gb.gva_q4_attention_weights(h.h, cache.c, q, lse, None, seq, 0.0, None, w, stride, B, 1, stride)
                gb.gva_q4_evict(h.h, cache.c, w, None, seq, keep, pos, 1, 3, w2, p2, new, stride, ews, B, stride)
            else:
                gb.gva_append_cache_at(h.h, cache.c, x, kr, slots, pos, B)
                gb.gva_decode(h.h, cache.c, q, seq, out, lse, ws, B, stride)
                gb.gva_attention_weights(h.h, cache.c, q, lse, None, seq, 0.0, None, w, stride, B, 1, stride)
                gb.gva_evict(h.h, cache.c, w, None, seq, keep, pos, 1, 3, w2, p2, new, stride, ews, B, stride)

        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for n in ([900, 200], [64, 1], [333, 129]):
            results = []
            for replay in (False, True):
                for t, a in zip(cache.d, cache.pools):
                    t.copy_(torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a))
                rng = np.random.default_rng(sum(n))
                x.copy_(dev(rng.standard_normal((B, 4, 64)).astype(np.float32)))
                kr.copy_(dev(rng.standard_normal((B, 16)).astype(np.float32)))
                q.copy_(dev(rng.standard_normal((B, 16, 80)).astype(np.float32)))
                slots.copy_(ints([m - 1 for m in n]))
                pos.copy_(ints([m + 40 for m in n]))
                seq.copy_(ints(n))
                w.zero_(); w2.zero_(); p2.zero_()
                torch.cuda.synchronize()
                if replay: graph.replay()
                else: step()
                torch.cuda.synchronize()
                results.append([t.clone() for t in (out, lse, w, w2, p2, new, *cache.d)])
            for a, b in zip(*results):
                assert torch.equal(torch.nan_to_num(a.float(), nan=-77.0), torch.nan_to_num(b.float(), nan=-77.0))
        del graph


def test_two_chains_at_once_on_two_streams_of_one_handle():
    """append, decode, gather (one row and several), evict, widen: two batches on two streams, nothing shared but the handle; what
    each leaves is what it leaves alone, bit for bit."""
    shape, page, steps = wl.SHAPE_A, 64, 6
    with Handle(shape, page) as h:
        def batch(i):
            B, T = (3, 1500) if i == 0 else (40, 260)
            rng = np.random.default_rng(180 + i)
            cache = Cache(shape, [T - 9 * (b % 5) for b in range(B)], seed=182 + i, room=64)
            wide = Cache(shape, [1] * B, kind="bf16", seed=184 + i, room=cache.max_pages * page - 1)
            stride = cache.max_pages * page
            x = [dev(rng.standard_normal((B, 4, 64)).astype(np.float32)) for _ in range(steps)]
            kr, q = dev(rng.standard_normal((B, 16)).astype(np.float32)), dev(queries(shape, 2 * B, 186 + i))
            seq, pos, keep = ints(cache.lens), ints(np.array(cache.lens) + 100), ints([T // 2 + 3 * b for b in range(B)])
            cu = ints(2 * np.arange(B + 1))
            out, lse, lse2 = torch.zeros(B, 16, 64, device="cuda"), torch.zeros(B, 16, device="cuda"), torch.full((2 * B, 16), 6.0, device="cuda")
            w, p = torch.zeros(B, stride, device="cuda"), torch.zeros(B, stride, dtype=torch.int32, device="cuda")
            ws = torch.zeros(gb.gva_q4_decode_workspace_bytes(h.h, B, stride), dtype=torch.uint8, device="cuda")
            ews = torch.zeros(gb.gva_evict_workspace_bytes(h.h, B, stride), dtype=torch.uint8, device="cuda")

            def step(k):
                gb.gva_q4_append(h.h, cache.c, x[k], kr, seq, pos, B)
                seq.add_(1)
                pos.add_(1)
                gb.gva_q4_decode(h.h, cache.c, q, seq, out, lse, ws, B, stride)
                gb.gva_q4_attention_weights(h.h, cache.c, q, lse, None, seq, 0.5, w, w, stride, B, 1, stride)
                gb.gva_q4_attention_weights(h.h, cache.c, q, lse2, cu, seq, 1.0, w, w, stride, B, 2, stride)
                if k % 2:
                    gb.gva_q4_evict(h.h, cache.c, w, p, seq, keep, pos, 1, 3, w, p, seq, stride, ews, B, stride)
                gb.gva_q4_widen(h.h, cache.c, wide.c, None, seq, B, stride)

            def left():
                return [t.clone() for t in (out, lse, w, p, seq, *cache.d, *wide.d)]
            return step, left

        alone = []
        for i in range(2):
            step, left = batch(i)
            for k in range(steps):
                step(k)
            torch.cuda.synchronize()
            alone.append(left())
        both = [batch(i) for i in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for k in range(steps):
            for (step, _), s in zip(both, streams):
                with torch.cuda.stream(s):
                    step(k)
        torch.cuda.synchronize()
        for want, (_, left) in zip(alone, both):
            for a, b in zip(want, left()):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
