"""Pages that sequences share, on the GPU against the integer / float64 oracles: tables, counts and stored bytes exactly, attention within what its roundings add up to."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as po
from oracle.pages_shared_oracle import Tables
from paper_2507_20030_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def ints(x):
    return dev(np.asarray(x, np.int32))


def f64(t):
    return t.detach().cpu().double().numpy()


class Both:
    """Tables of the oracle and the library's, changed side by side and compared after every change."""

    def __init__(self, batch, W, n_pages, P, rng):
        self.o = Tables(batch, W, n_pages, P, rng.permutation(n_pages))
        self.P, self.rng = P, rng
        self.table, self.lens, self.free, self.refs = (dev(x) for x in self.o.arrays().values())

    def same(self, **more):
        o = self.o
        assert np.array_equal(self.lens.cpu().numpy(), o.lens) and np.array_equal(self.refs.cpu().numpy(), o.refs)
        n = int(o.free[0]) + 1
        assert np.array_equal(self.free.cpu().numpy()[:n], o.free[:n])
        table = self.table.cpu().numpy()
        for b in range(len(o.lens)):
            assert np.array_equal(table[b, :len(o.pages(b))], o.pages(b)), b
        for name, (got, ref) in more.items():
            assert np.array_equal(got.cpu().numpy(), ref), name
        assert o.consistent()

    def fork(self, parent, keep=None, **kw):
        self.o.fork(parent, keep)
        B.iwdft_pages_fork(ints(parent), None if keep is None else ints(keep), self.table, self.lens, self.free, self.refs, self.P, **kw)
        self.same()

    def resize(self, want, n_slots):
        batch = len(self.o.lens)
        starts, slots, copies = (torch.full(s, 77, dtype=torch.int32, device=DEV) for s in ((batch + 1,), (n_slots,), (batch, 2)))
        ref = self.o.resize(want, n_slots)
        B.iwdft_pages_resize_shared(ints(want), self.table, self.lens, self.free, self.refs, starts, slots, copies, self.P)
        self.same(starts=(starts, ref[0]), slots=(slots, ref[1]), copies=(copies, ref[2]))
        return ref

    def compact(self, n_moves):
        moves = torch.full((n_moves, 2), 77, dtype=torch.int32, device=DEV)
        ref = self.o.compact(n_moves)
        B.iwdft_pages_compact(self.table, self.lens, self.free, self.refs, moves, self.P)
        self.same(moves=(moves, ref))
        return ref


@pytest.mark.parametrize("batch,W,P,n_pages,n_slots,most", [
    (1, 4, 16, 5, 64, 60), (3, 6, 32, 12, 200, 150), (16, 20, 16, 150, 300, 300), (16, 600, 16, 2500, 9000, 3000), (65, 150, 32, 1500, 2500, 900), (256, 40, 16, 900, 4000, 400),
    (300, 30, 128, 900, 30000, 2000), (1024, 9, 16, 2000, 3000, 100), (40, 1, 16, 33, 300, 16), (5, 3, 16, 9, 0, 40),
])
def test_tables(batch, W, P, n_pages, n_slots, most):
    """Forks of whole sequences and beginnings, rows that change places, growth into shared pages, pools and slots that run out, compaction; small and large tables."""
    rng = np.random.default_rng(batch * W + P)
    t = Both(batch, W, n_pages, P, rng)
    t.resize(rng.integers(0, most + 1, size=batch) * (rng.random(batch) < 0.3), n_slots)
    copied = refused = moved = 0
    for r in range(8):
        if r % 4 == 3:
            moved += int((t.compact([n_pages // 2, 3][r % 2] if r > 3 else 2)[:, 0] >= 0).sum())
        parent = np.where(rng.random(batch) < 0.4, np.arange(batch), rng.integers(-1, batch + 1, size=batch))
        keep = np.where(rng.random(batch) < 0.7, -1, rng.integers(0, most + 1, size=batch))
        t.fork(parent, None if r % 3 == 1 else keep)
        lens = t.o.lens.copy()
        want = np.where(rng.random(batch) < 0.7, lens + rng.integers(0, 4, size=batch), rng.integers(0, most + 1, size=batch))
        want = np.where(rng.random(batch) < 0.1, -1, np.where(rng.random(batch) < 0.1, W * P + 1, want))
        copies = t.resize(want, n_slots)[2]
        copied += int((copies[:, 0] >= 0).sum())
        refused += int(((want > t.o.lens) & (want <= W * P)).sum())
    assert n_slots == 0 or batch == 1 or copied > 0
    assert n_pages < 100 or moved > 0  # small pools are full


def test_all_samples_of_a_prompt_leave_its_last_page_but_one():
    t = Both(6, 8, 30, 16, np.random.default_rng(0))
    t.resize([40, 0, 0, 0, 0, 0], 40)
    t.fork([0, 0, 0, 0, 0, 5])
    assert t.o.refs.max() == 5 and t.o.free[0] == 27
    copies = t.resize([41, 41, 60, 41, 41, 3], 60)[2]
    assert (copies[:4, 0] >= 0).all() and copies[4, 0] == -1 and len(set(copies[:4, 0])) == 1
    t.fork([0] * 6)
    assert (t.resize([-1, 42, -1, 45, 50, 0], 60)[2][[1, 3, 4], 0] >= 0).all()   # two stay where they are: all who grow leave


def test_who_stays_is_held_to_the_pages_that_are_left():
    """Two samples share a page and one page is free; a page needed before them leaves none: neither grows, not even the one that needs none of its own."""
    for spare in (0, 1):
        t = Both(3, 4, 3 + spare, 16, np.random.default_rng(1))
        t.resize([16, 20, 0], 40)
        t.fork([0, 1, 1])
        t.resize([17, 21, 21], 40)
        assert list(t.o.lens) == ([17, 21, 21] if spare > 1 else [17, 20, 20] if spare else [16, 20, 20])


def test_without_shared_pages_as_resize():
    """The same tables, stack, starts and slots as iwdft_pages_resize; a call that undoes another one leaves the stack as it was."""
    rng = np.random.default_rng(4)
    for batch in (9, 200, 700):
        plain, shared = (B.PagedCache(1, 4000, 1, 1, 128, torch.float32, batch, 2000, 16, DEV) for _ in range(2))
        refs, copies = torch.zeros(4000, dtype=torch.int32, device=DEV), torch.empty((batch, 2), dtype=torch.int32, device=DEV)
        for r in range(5):
            want = ints(rng.integers(0, 3000 // batch, size=batch) if r != 3 else rng.integers(0, 120, size=batch))
            starts, slots = plain.resize(want, 9000)
            s2, l2 = torch.empty_like(starts), torch.empty_like(slots)
            B.iwdft_pages_resize_shared(want, shared.table, shared.lens, shared.free, refs, s2, l2, copies, 16)
            n = int(plain.free[0])
            assert torch.equal(starts, s2) and torch.equal(slots, l2) and torch.equal(plain.lens, shared.lens) and (copies == -1).all()
            assert torch.equal(plain.free[:n + 1], shared.free[:n + 1]) and int((refs > 0).sum()) == 4000 - n


def test_tables_no_sequences_and_damaged_arrays():
    """batch 0; lengths, counts, tables, parents and page ids that nothing valid has: no slot or page outside of the pool comes out."""
    e = torch.empty(0, dtype=torch.int32, device=DEV)
    none, starts, slots = torch.empty((0, 4), dtype=torch.int32, device=DEV), ints([5]), ints([5] * 7)
    B.iwdft_pages_resize_shared(e, none, e, ints(range(5)), ints([0] * 4), starts, slots, torch.empty((0, 2), dtype=torch.int32, device=DEV), 16)
    assert starts.tolist() == [0] and slots.tolist() == [-1] * 7
    B.iwdft_pages_fork(e, None, none, e, ints(range(5)), ints([0] * 4), 16)
    free, refs = ints([2, 9, 9, 9, 9]), ints([0, 1, 0, 0])
    B.iwdft_pages_compact(none, e, free, refs, torch.empty((2, 2), dtype=torch.int32, device=DEV), 16)
    assert refs.tolist() == [1, 0, 0, 0] and free.tolist() == [3, 3, 2, 1, 9]
    for W, n_slots in ((4, 400), (3000, 3000)):
        for seed in range(3):
            rng = np.random.default_rng(seed)
            wild = lambda *s: ints(rng.choice([-2 ** 31, -7, -1, 0, 1, 2, 3, 4, 9999, 2 ** 31 - 1], size=s))  # noqa: E731
            table, lens, free, refs, copies = wild(3, W), wild(3), wild(5), wild(4), wild(3, 2)
            starts, slots, moves = wild(4), wild(n_slots), wild(4, 2)
            for _ in range(2):
                B.iwdft_pages_fork(wild(3), wild(3), table, lens, free, refs, 16)
                B.iwdft_pages_resize_shared(wild(3), table, lens, free, refs, starts, slots, copies, 16)
                s = slots.cpu().numpy()
                assert ((s >= -1) & (s < 4 * 16)).all() and 0 <= int(free[0]) <= 4
                B.iwdft_pages_compact(table, lens, free, refs, moves, 16)
                m = moves.cpu().numpy()
                assert ((m >= -1) & (m < 4)).all() and 0 <= int(free[0]) <= 4


# ------------------------------------------------------------------------------------------------------------------ copying
@pytest.mark.parametrize("P,heads,layers", [(16, 1, 1), (32, 3, 4), (64, 8, 2), (128, 5, 1)])
def test_copy(P, heads, layers):
    rng = np.random.default_rng(P)
    for n_to in (None, 9, 40):
        values = torch.randint(0, 256, (layers, 30, heads, 2, P * 128), dtype=torch.uint8, device=DEV)
        exponents = torch.randint(-100, 100, (layers, 30, heads, 2), dtype=torch.int32, device=DEV)
        other = (values, exponents) if n_to is None else (torch.full((layers, n_to, heads, 2, P * 128), 7, dtype=torch.uint8, device=DEV),
                                                          torch.full((layers, n_to, heads, 2), 7, dtype=torch.int32, device=DEV))
        to = rng.permutation(30 if n_to is None else n_to)
        pairs = [(int(a), int(b)) for a, b in zip(rng.integers(20, 30, size=len(to)), to) if n_to is not None or b < 20]
        pairs[2:2] = [(-1, -1), (0, 10 ** 6), (-5, 3), (30, 2)]  # left out
        first, n = (1, layers - 1) if layers > 1 else (0, None)
        ref = other[0].clone(), other[1].clone()
        for a, b in pairs:
            if 0 <= a < 30 and 0 <= b < ref[0].shape[1]:
                ref[0][first:, b], ref[1][first:, b] = values[first:, a], exponents[first:, a]
        B.iwdft_pages_copy(ints(pairs), values, exponents, *([] if n_to is None else other), layer=first, n_layers=n)
        assert torch.equal(other[0], ref[0]) and torch.equal(other[1], ref[1])


def test_copy_far_into_a_long_pool():
    """Offsets beyond 32 bits."""
    n_pages, P = 160_000, 128
    values, exponents = torch.zeros((1, n_pages, 1, 2, P * 128), dtype=torch.uint8, device=DEV), torch.zeros((1, n_pages, 1, 2), dtype=torch.int32, device=DEV)
    values[0, 159_999], exponents[0, 159_999] = 3, 4
    B.iwdft_pages_copy(ints([[159_999, 140_000], [159_999, 2]]), values, exponents)
    assert (values[0, [2, 140_000]] == 3).all() and (exponents[0, [2, 140_000]] == 4).all() and int((values.view(-1)[:: 1 << 13] != 0).sum()) == 3 * 4
