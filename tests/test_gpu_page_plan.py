"""GPU tests of what gva_assign_pages says of bad sequences, pages and rings, and of what becomes of bad pages.  All whole numbers: exact."""
import numpy as np
import pytest
import torch

from paper_2609_13285_b200 import binding as gb
from paper_2609_13285_b200 import workloads as wl
from tests import draft_ref as ref
from tests.test_gpu_compact import Handle, ints
from tests.test_gpu_draft import Pages, code, zeros

pytestmark = pytest.mark.gpu
ROWS = [500, 9000]             # rows allowed for: by the kernel of the plan itself, by one of their own


@pytest.fixture(scope="module", autouse=True)
def _built():
    from tests import gpu_util
    gpu_util.ensure_built()


def plan(handle, s, want, max_rows):
    """The call in place on a state of tests.test_gpu_draft.Pages, which it moves on: rows, (error, index)."""
    used, pages, table, ring, free = ints(s.used), ints(s.pages), ints(s.table), ints(s.ring), ints(s.free)
    cu, pos, slots, status = zeros(s.B + 1), zeros(max_rows), zeros(max_rows), zeros(1)
    gb.gva_assign_pages(handle.h, used, ints(want), pages, pages, table, s.most, s.N, ring, free, free, used, cu, pos, slots, max_rows, s.B, status)
    n = int(cu[-1])
    s.used, s.pages, s.free = used.tolist(), pages.tolist(), tuple(free.tolist())
    s.table, s.ring = table.cpu().numpy().astype(np.int64), ring.cpu().numpy().astype(np.int64)
    return {"cu": cu.tolist(), "pos": pos[:n].tolist(), "slots": slots[:n].tolist()}, code(status)


def expected(s, want, max_rows):
    """What the call is to leave where pages that come back may be bad: the reference's, but for those, which are dropped.  (What ring
    entries hold beside the free pages is nobody's business.)"""
    r = ref.assign_pages(s.used, want, s.pages, s.table, s.P, s.N, s.ring, s.free, max_rows)
    first, count = s.free
    back = [(b, int(s.table[b, j])) for b in range(s.B) for j in range(r["pages"][b], s.pages[b])]
    taken = sum(max(0, r["pages"][b] - s.pages[b]) for b in range(s.B))
    good = [p for _, p in back if 0 <= p < s.N]
    ring = s.ring.copy()
    for i, p in enumerate(good[: s.N - count]):
        ring[(first + count + i) % s.N] = p
    r["ring"], r["free"] = ring, ((first + taken) % s.N, count - taken + min(len(good), s.N - count))
    return r, sorted({b for b, p in back if not 0 <= p < s.N})


def check(handle, s, want, max_rows, errors=()):
    """errors: the (error, index) pairs of which the call has to say one; none: all is well."""
    r, dropped = expected(s, want, max_rows)
    got, said = plan(handle, s, want, max_rows)
    errors = set(errors) | {(gb.GVA_ERR_BAD_PAGE, b) for b in dropped}
    assert said in errors if errors else said == (0, 0), (said, errors)
    for k in ("cu", "pos", "slots"):
        assert got[k] == [int(x) for x in r[k]], k
    assert s.used == [int(x) for x in r["lens"]] and s.pages == [int(x) for x in r["pages"]] and s.free == tuple(r["free"])
    assert np.array_equal(s.table, r["table"]) and np.array_equal(free_pages(s, s.ring), free_pages(s, r["ring"]))
    return r


def free_pages(s, ring):
    return ring[(s.free[0] + np.arange(s.free[1])) % s.N]


@pytest.mark.parametrize("rows", ROWS)
def test_a_bad_page_that_comes_back_goes_to_nobody(rows):
    with Handle(wl.SHAPE_A) as h:
        s = Pages(3, 64, 8, seed=1, held=[300, 100, 64], ahead=0, spare=2)
        s.table[0, 2], s.table[0, 4] = s.N, -3
        check(h, s, [0, 101, 64], rows)                             # sequence 0 is done: five pages, two of them bad
        assert s.free[1] == 5 and len(set(s.ring[(s.free[0] + np.arange(5)) % s.N])) == 5
        check(h, s, [8 * 64, 101, 64], rows, [(gb.GVA_ERR_NO_ROOM, 0)])
        r = check(h, s, [5 * 64, 101, 64], rows)                    # what is left of the ring serves: every row has a slot
        assert min(r["slots"]) >= 0 and s.free[1] == 0


@pytest.mark.parametrize("B,most", [(40, 9), (1025, 6), (3000, 5), (8192, 3), (2, 3000)])
@pytest.mark.parametrize("rows", ROWS)
def test_bad_pages_among_many_that_come_back(B, most, rows):
    """Scattered, first and last, all of a sequence's; of sequences that shrink, end, and grow within pages they hold too many of."""
    with Handle(wl.SHAPE_A) as h:
        for share in (0.001, 0.1, 1.0):
            s = Pages(B, 64, most, seed=B, spare=7 * B // 2, ahead=0.5)
            rng = np.random.default_rng(B)
            room = rows
            want = []
            for b, u in enumerate(s.used):
                x = rng.random()
                new = int(rng.integers(1, 6)) if x < 0.3 and room > 6 else 0
                want.append(min(u + new, most * 64) if new else 0 if x < 0.6 else int(rng.integers(0, u + 1)))
                room -= max(0, want[-1] - u)
            keep = [-(-w // 64) for w in want]
            for b in range(B):
                for j in range(keep[b], s.pages[b]):
                    if rng.random() < share:
                        s.table[b, j] = rng.choice([-1, s.N, s.N + 5, 2 ** 31 - 1, -2 ** 31])
            for b in (0, B - 1):
                if s.pages[b] > keep[b]:
                    s.table[b, keep[b]] = s.N
            check(h, s, want, rows)
            for step in range(2):                                   # ... and the ring that is left serves the next steps
                check(h, s, [min(most * 64, u + 1 + b % 2) if b < rows // 2 else u for b, u in enumerate(s.used)], rows)


def test_more_bad_pages_than_a_full_ring_has_room_for():
    with Handle(wl.SHAPE_A) as h:
        s = Pages(4, 64, 8, seed=3, held=[300, 300, 300, 300], ahead=0, spare=2)
        s.free = (s.free[0], s.N - 3)                               # a ring that says it holds nearly all
        s.table[1, 1] = -1
        r, _ = expected(s, [300, 0, 300, 0], 10)
        got, said = plan(h, s, [300, 0, 300, 0], 10)
        assert said in {(gb.GVA_ERR_BAD_PAGE, 0), (gb.GVA_ERR_BAD_PAGE, 1)}
        assert s.free == tuple(r["free"]) and np.array_equal(free_pages(s, s.ring), free_pages(s, r["ring"])) and s.free[1] == s.N


@pytest.mark.parametrize("rows", ROWS)
def test_new_rows_on_a_bad_page_are_reported(rows):
    bad = lambda b: {(gb.GVA_ERR_BAD_PAGE, b)}  # noqa: E731
    with Handle(wl.SHAPE_A) as h:
        s = Pages(8, 64, 8, seed=8, held=[10, 100, 64, 65, 0, 0, 200, 300], ahead=0)
        s.table[7, 300 // 64] = s.N                                 # under the sequence's next rows
        r = check(h, s, [u + 3 for u in s.used], rows, bad(7))
        assert r["slots"][-3:] == [-1] * 3 and min(r["slots"][:-3]) >= 0
        s.table[7, 0] = -1                                          # under rows that it has had: nothing is asked of it
        check(h, s, [u + 3 for u in s.used[:7]] + [s.used[7]], rows)
        for value in (s.N, -1, 2 ** 31 - 1, -2 ** 31):              # among the free pages: with who takes it
            s = Pages(5, 64, 8, seed=9, held=[64, 64, 10, 64, 128], ahead=0, spare=6)
            s.ring[(s.free[0] + 1) % s.N] = value
            r = check(h, s, [65, 64, 20, 70, 129], rows, bad(3))
            assert [x < 0 for x in r["slots"]] == [False] * 11 + [True] * 6 + [False]


@pytest.mark.parametrize("P,pages", [(32, 2 ** 26 - 1), (2 ** 20, 2 ** 11 - 1)])
def test_as_many_rows_as_slots_have_numbers(P, pages):
    """One prompt over the whole pool (17 GB of positions and slots), and one of nearly nothing behind it."""
    n = pages * P
    with Handle(wl.SHAPE_A, page=P) as h:
        ring = torch.randperm(pages, dtype=torch.int32, device="cuda")
        table, held, lens, cu, status = torch.full((2, pages), -1, dtype=torch.int32, device="cuda"), zeros(2), zeros(2), zeros(3), zeros(1)
        pos, slots = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
        free = ints([pages // 3, pages])
        order = torch.roll(ring, -(pages // 3))
        gb.gva_assign_pages(h.h, zeros(2), ints([n - P, 1]), held, held, table, pages, pages, ring, free, free, lens, cu, pos, slots, n, 2, status)
        assert int(status) == 0 and cu.tolist() == [0, n - P, n - P + 1] and lens.tolist() == [n - P, 1] and free.tolist()[1] == 0
        assert torch.equal(table[0, :-1], order[:-1]) and int(table[1, 0]) == int(order[-1])
        step = P * max(1, 2 ** 26 // P)
        for at in range(0, n - P, step):
            t = torch.arange(at, min(at + step, n - P), device="cuda")
            assert torch.equal(pos[at:at + len(t)], t.int())
            assert torch.equal(slots[at:at + len(t)].long(), order[t // P].long() * P + t % P)
        assert pos[n - P:].tolist()[:2] == [0, -7] and int(slots[n - P]) == int(order[-1]) * P and (slots[n - P + 1:] == -7).all()


@pytest.mark.parametrize("rows", ROWS)
def test_every_error_names_its_sequence(rows):
    L, N, F = gb.GVA_ERR_SEQ_LEN, gb.GVA_ERR_NO_ROOM, gb.GVA_ERR_BAD_PAGE
    held = [10, 100, 64, 65, 0, 0, 200, 300]
    with Handle(wl.SHAPE_A) as h:
        for b, change in enumerate([{"used": -1}, {"want": -1}, {"pages": 0}, {"pages": 9}, {"pages": -1}, {"want": 8 * 64 + 1}, {"want": 2 ** 31 - 1}, {"used": 2 ** 31 - 1}]):
            s = Pages(8, 64, 8, seed=5, held=held, ahead=0)
            want = [u + 50 for u in s.used]
            if "want" in change:
                want[b] = change["want"]
            for k in ("used", "pages"):
                if k in change:
                    getattr(s, k)[b] = change[k]
            check(h, s, want, rows, {(L, b)})
        for first, count in ((-1, 5), (None, -1), (10 ** 6, 3), (None, 10 ** 6)):
            s = Pages(8, 64, 8, seed=6, held=held)
            s.free = (s.free[0] if first is None else first, count)
            before = (list(s.used), list(s.pages), s.free)
            got, said = plan(h, s, [u + 70 if i % 2 else 0 for i, u in enumerate(s.used)], rows)
            assert said == (F, 0) and got["cu"] == [0] * 9 and (s.used, s.pages, s.free) == before
        s = Pages(8, 64, 8, seed=7, held=held, ahead=0, spare=3)     # pages for the first three that need one
        check(h, s, [u + 64 for u in held], rows, {(N, b) for b in range(3, 8)})
        s = Pages(8, 64, 8, seed=7, held=held, ahead=0, spare=40)    # rows for the first three
        check(h, s, [u + 150 for u in held], 3 * 150 + 5 if rows < 8192 else rows, {(N, b) for b in range(3, 8)} if rows < 8192 else ())
        s = Pages(8, 64, 8, seed=7, held=held, ahead=0)              # a ring that is full, and pages that come back
        s.free = (3, s.N)
        check(h, s, [0] * 8, rows, {(F, 0)})
