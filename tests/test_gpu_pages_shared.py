"""Pages that sequences share, on the GPU against the integer / float64 oracles: tables, counts and stored bytes exactly, attention within what its roundings add up to."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as po
from oracle.pages_shared_oracle import Tables
from paper_2507_20030_amd import binding as B
from test_gpu_pages import near

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


def test_many_pages_at_once():
    """More pages given up than one turn of the workgroup takes, by holders alone and together; more slots than fit the first launch; a wide table that is hardly used."""
    rng = np.random.default_rng(8)
    t = Both(5, 9000, 30000, 16, rng)
    t.resize([140_000, 30, 0, 90_000, 0], 300_000)
    t.fork([0, 1, 0, 3, 3], [-1, -1, 139_000, -1, 50_001])
    t.resize([139_990, 31, 139_001, 90_001, 50_002], 100)
    t.resize([100, 31, 0, 80_000, 20], 100)                      # 16 thousand entries at a time, most of them held twice
    t.fork([0, 3, 2, 4, 4])
    t.resize([0, 0, 0, 0, 0], 0)
    assert t.o.free[0] == 30000


def test_a_pool_of_more_pages_than_bits_in_lds():
    rng = np.random.default_rng(9)
    t = Both(3, 3000, 140_001, 16, rng)
    t.resize([40_000, 100, 20_000], 70_000)
    t.fork([0, 0, 2], [-1, 30_000, -1])
    assert (t.compact(70)[:, 0] >= 0).all()                     # some of what would have to move
    t.resize([41_000, -1, 0], 2_000)
    t.compact(20)


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


# ------------------------------------------------------------------------------------------------------------------ attention
class Pool:
    """Sequences (parent or -1, tokens shared with it, length) over a pool full of tokens; pages in random order."""

    def __init__(self, rng, forest, P, heads=2, layers=1):
        rows = []
        n = 0
        for parent, keep, length in forest:
            row = rows[parent][:keep // P] if parent >= 0 else []
            fresh = -(-length // P) - len(row)
            rows.append(row + list(range(n, n + fresh)))
            n += fresh
        self.P, self.n_pages = P, n + 3
        order = rng.permutation(self.n_pages)
        self.lens = np.array([length for _, _, length in forest], np.int32)
        self.table = np.full((len(forest), max(1, max(map(len, rows))) + 1), -1, np.int32)
        for b, row in enumerate(rows):
            self.table[b, :len(row)] = order[row]
        self.store = po.Store(layers, self.n_pages, heads, P)
        full = rng.normal(size=(layers, self.n_pages * P, heads, 128)) * 10.0 ** rng.uniform(-1, 1, size=128)
        self.store.write(full, rng.normal(size=full.shape) * 10.0 ** rng.uniform(-2, 2, size=(1, full.shape[1], 1, 1)), np.arange(self.n_pages * P))
        self.upload()

    def upload(self):
        self.values, self.exponents, self.d_table, self.d_lens = (dev(x) for x in (self.store.packed(), self.store.exponents, self.table, self.lens))


def plan_of(pool, starts, n, G, dtype, layers=1, **kw):
    return B.iwdft_pages_plan(ints(starts), pool.d_table, pool.d_lens, n, pool.n_pages, pool.store.raw.shape[2], pool.store.raw.shape[2] * G, pool.P, DT[dtype],
                              n_layers=layers, **kw)


def attend(pool, rng, news, G, dtype, layer=0, layers=1, pad=0, scale=None, q=None, **kw):
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    n = int(starts[-1]) + pad
    q = dev(rng.normal(size=(layers, n, pool.store.raw.shape[2] * G, 128))).to(DT[dtype]) if q is None else q
    out = torch.full_like(q, 7.0)
    plan = plan_of(pool, starts, n, G, dtype, layers, **kw)
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan, pool.d_table, out, layer, scale=scale or 0.0)
    ref, *rest = pool.store.attend(f64(q), starts, pool.table, pool.lens, layer, scale=scale, **kw)
    if pad:
        assert (out[:, starts[-1]:] == 7.0).all()
        ref, out = ref[:, :starts[-1]], out[:, :starts[-1]]
        rest = [r[:, :starts[-1]] for r in rest]
    near(out, ref, *rest, dtype)
    return out


def forest_of(rng, kind, batch, prompt, tail):
    got = [(-1, 0, prompt + int(rng.integers(1, tail + 1)))]
    for b in range(1, batch):
        own = int(rng.integers(1, tail + 1))
        if kind == "samples":
            got.append((0, prompt, prompt + own))
        elif kind == "nested":
            parent = int(rng.integers(b))
            keep = int(rng.integers(0, got[parent][2] + 1))
            got.append((parent, keep, keep + own))
        elif kind == "chain":  # each begins with all of the one before
            got.append((b - 1, got[-1][2], got[-1][2] + own))
        elif kind == "cut":  # nothing of their own: shorter and shorter beginnings
            got.append((0, prompt * (batch - b) // batch, prompt * (batch - b) // batch))
        else:
            got.append((-1, 0, int(rng.integers(0, prompt + own))))
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("kind", ["samples", "nested", "chain", "cut", "alone"])
def test_attention_of_who_shares_what(kind, P, dtype):
    rng = np.random.default_rng(P + len(kind))
    forest = forest_of(rng, kind, 7, 300, 90)
    attend(Pool(rng, forest, P), rng, [1 if n else 0 for _, _, n in forest], 4, dtype, pad=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,G,heads", [(1, 1, 1), (3, 5, 1), (4, 4, 1), (5, 7, 1), (8, 4, 2), (17, 8, 1), (9, 16, 1), (33, 8, 1), (70, 2, 2), (300, 1, 1)])
def test_attention_rows(batch, G, heads, dtype):
    """From one row to blocks of rows in each of the kernels, several sequences to a row of LDS."""
    rng = np.random.default_rng(batch + G)
    forest = forest_of(rng, "samples", batch, 120, 20 if batch > 40 else 200)
    attend(Pool(rng, forest, 32, heads=heads), rng, [1] * batch, G, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,news,G", [("samples", [1, 5, 1, 3], 4), ("nested", [9, 0, 1, 40, 2, 7], 2), ("chain", [0, 70, 1, 1], 3), ("cut", [1, 130, 0, 2], 8), ("samples", [400, 1, 1], 1)])
def test_attention_drafts_and_prompts(kind, news, G, dtype):
    """New tokens that see each other, more of them than the sequence is long, rows behind the last one."""
    rng = np.random.default_rng(sum(news))
    attend(Pool(rng, forest_of(rng, kind, len(news), 310, 50), 16), rng, news, G, dtype, pad=3, scale=0.1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sink,recent", [(0, 1), (0, 40), (10, 50), (33, 64), (1, 1), (64, 1000), (500, 3), (0, 2 ** 31 - 1), (2 ** 31 - 1, 5)])
def test_attention_windows(sink, recent, dtype):
    rng = np.random.default_rng(sink % 1000 + recent % 1000)
    forest = forest_of(rng, "samples", 6, 400, 150) + [(-1, 0, 12), (2, 390, 391), (0, 64, 64), (0, 0, 0)]
    attend(Pool(rng, forest, 16), rng, [1, 7, 12, 1, 1, 2, 12, 1, 1, 0], 2, dtype, n_sink=sink, n_recent=recent)
    attend(Pool(rng, forest_of(rng, "nested", 40, 200, 60), 32, heads=1), rng, [1] * 40, 4, dtype, n_sink=sink, n_recent=recent)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_layers(dtype):
    rng = np.random.default_rng(3)
    pool = Pool(rng, forest_of(rng, "samples", 12, 200, 40), 32, heads=3, layers=4)
    attend(pool, rng, [1] * 12, 4, dtype, layer=1, layers=2)
    attend(pool, rng, [1] * 12, 4, dtype, layer=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,W,n_pages", [(5, 9, 4), (40, 30, 3), (70, 12, 50), (3, 200, 2)])
def test_attention_any_table(batch, W, n_pages, dtype):
    """Pages at several places, sets that change at every place and come together again, pages that are not there: more changes than a plan holds, too."""
    rng = np.random.default_rng(batch)
    pool = Pool(rng, [(-1, 0, 16 * n_pages)], 16)
    pool.table = rng.integers(-1, n_pages + 4, size=(batch, W)).astype(np.int32)
    pool.table[batch // 2:, : W // 2] = pool.table[0, : W // 2]
    pool.lens = rng.integers(0, W * 16 + 1, size=batch).astype(np.int32)
    pool.upload()
    attend(pool, rng, rng.integers(0, 3, size=batch), 2, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_does_not_see_what_is_masked(dtype):
    """NaN and the largest values behind the sequences' ends, in pages of nobody, and in shared tokens that only some of the rows see."""
    rng = np.random.default_rng(9)
    for batch, G in ((3, 2), (20, 4)):
        forest = [(-1, 0, 100)] + [(0, 100, 100 + 3 * b) for b in range(1, batch)]
        pool = Pool(rng, forest, 32)
        raw = pool.store.raw
        held = set()
        for b in range(batch):
            n = int(pool.lens[b])
            raw[0, pool.table[b, (n - 1) // 32], :, :, n % 32 or 32:] = 0x7f
            held.update(pool.table[b, :-(-n // 32)].tolist())
        for p in set(range(pool.n_pages)) - held:
            raw[0, p] = 0xff
        raw[0, pool.table[0, 1], 1, 1, 8, 40] = 0x7f      # V, token 40, channel 40: within the window of the first sequence only
        pool.upload()
        out = attend(pool, rng, [1] * batch, G, dtype, n_sink=2, n_recent=60)
        nan = torch.isnan(out.float())
        assert nan[0, 0, G:, 40].all() and int(nan.sum()) == G
        out = attend(pool, rng, [1] * batch, G, dtype)
        assert int(torch.isnan(out.float()).sum()) == G * batch


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_queries_that_are_not_finite_stay_in_their_row(dtype):
    rng = np.random.default_rng(10)
    for batch in (3, 20):
        pool = Pool(rng, forest_of(rng, "samples", batch, 200, 30), 32)
        q = torch.randn((1, batch, 8, 128), device=DEV).to(DT[dtype])
        q[0, 1, 2, 5], q[0, 1, 3, 7] = float("nan"), float("inf")
        starts = ints(range(batch + 1))
        out, plain = torch.zeros_like(q), torch.zeros_like(q)
        B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan_of(pool, range(batch + 1), batch, 4, dtype), pool.d_table, out)
        B.iwdft_pages_attn(pool.values, pool.exponents, q, starts, pool.d_table, pool.d_lens, plain)
        bad = torch.isnan(out.float()).any(-1)
        assert torch.equal(bad, torch.isnan(plain.float()).any(-1)) and not bad[0, 0].any() and not bad[0, 2:].any() and bad[0, 1, 2]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_pages_far_apart(dtype):
    """Pages of V whose scales are up to 2^120 apart, within runs and between them; K's scales apart as far as scores stay small."""
    rng = np.random.default_rng(14)
    for batch, G in ((3, 4), (24, 4)):
        pool = Pool(rng, forest_of(rng, "nested", batch, 150, 60), 16)
        e = pool.store.exponents
        e[..., 0] -= rng.integers(2, 12, size=e.shape[:3]).astype(np.int32)
        e[..., 1] += rng.integers(-60, 60, size=e.shape[:3]).astype(np.int32)
        pool.upload()
        attend(pool, rng, [1] * batch, G, dtype)


def test_attention_far_into_a_long_pool_and_over_long_sequences():
    """Offsets beyond 32 bits; half a million tokens shared by two sequences: against iwdft_pages_attn."""
    g = torch.Generator(device=DEV).manual_seed(3)
    n_pages, P = 160_000, 128
    values, exponents = torch.zeros((1, n_pages, 1, 2, P * 128), dtype=torch.uint8, device=DEV), torch.full((1, n_pages, 1, 2), -7, dtype=torch.int32, device=DEV)
    assert values.numel() > 1 << 32
    values[:, 155_000:] = torch.randint(0, 120, (1, 5000, 1, 2, P * 128), dtype=torch.uint8, device=DEV, generator=g)
    shared = torch.arange(n_pages - 1, n_pages - 1 - 4000, -1, dtype=torch.int32, device=DEV)
    table = torch.full((3, 4100), -1, dtype=torch.int32, device=DEV)
    table[:2, :4000] = shared
    table[2, :1500] = shared[:1500]
    table[1, 4000:4003], table[0, 4000], table[2, 1500] = torch.arange(155_500, 155_503, device=DEV), 155_400, 155_401
    lens, starts = ints([4000 * P + 77, 4002 * P + 1, 1500 * P + 128]), ints([0, 1, 2, 4])
    for dtype in ("f32", "bf16"):
        q = (torch.randn((1, 4, 2, 128), device=DEV, generator=g) * 0.05).to(DT[dtype])
        out, ref = torch.zeros_like(q), torch.zeros_like(q)
        B.iwdft_pages_attn(values, exponents, q, starts, table, lens, ref)
        plan = B.iwdft_pages_plan(starts, table, lens, 4, n_pages, 1, 2, P, DT[dtype])
        B.iwdft_pages_attn_shared(values, exponents, q, plan, table, out)
        err = float((out.double() - ref.double()).norm() / ref.double().norm())
        # two roundings of the result; fp32: sums of 16000 tiles, 2^-24 each, of both calls (at random 2^-16, all one way 2^-9), far from each other's
        assert err < (2.0 ** -7 if dtype == "bf16" else 2.0 ** -9), err


def test_attention_of_short_sequences_in_a_wide_table():
    rng = np.random.default_rng(15)
    pool = Pool(rng, forest_of(rng, "samples", 5, 50, 20), 16)
    wide = np.full((5, 70_000), -1, np.int32)
    wide[:, :pool.table.shape[1]] = pool.table
    pool.table = wide
    pool.upload()
    attend(pool, rng, [1] * 5, 2, "f32")


def test_attention_one_sequence_for_each_row_of_a_large_table():
    rng = np.random.default_rng(2)
    forest = forest_of(rng, "nested", 1024, 40, 5)
    attend(Pool(rng, forest, 16, heads=1), rng, [1 if n else 0 for _, _, n in forest], 1, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_long_and_as_page_attention(dtype):
    """Thousands of tokens, many parts: against iwdft_pages_attn, which is within its roundings of the definition."""
    for batch, prompt, G, H, window in ((16, 9000, 4, 8, {}), (2, 30000, 8, 2, {}), (64, 5000, 2, 4, dict(n_sink=5, n_recent=3000)), (3, 40, 1, 1, {})):
        g = torch.Generator(device=DEV).manual_seed(batch)
        P, rng = 64, np.random.default_rng(batch)
        forest = forest_of(rng, "nested" if batch == 64 else "samples", batch, prompt, 700)
        t = Both(batch, 200 if batch == 64 else 600, 9000, P, rng)
        t.resize([forest[0][2]] + [0] * (batch - 1), 100_000)
        for b, (parent, keep, length) in enumerate(forest[1:], 1):
            ids, keeps = np.arange(batch), np.full(batch, -1)
            ids[b], keeps[b] = parent, keep
            t.o.fork(ids, keeps)
            want = np.full(batch, -1)
            want[b] = length
            t.o.resize(want, 100_000)
        table, lens = ints(t.o.table), ints(t.o.lens)
        values = torch.randint(0, 127, (1, 9000, H, 2, P * 128), dtype=torch.uint8, device=DEV, generator=g) ^ (torch.randint(0, 2, (1, 9000, H, 2, P * 128), dtype=torch.uint8, device=DEV, generator=g) << 7)
        exponents = torch.randint(-8, -4, (1, 9000, H, 2), dtype=torch.int32, device=DEV, generator=g)
        q = torch.randn((1, batch, G * H, 128), device=DEV, generator=g).to(DT[dtype]) * 0.02
        starts = ints(range(batch + 1))
        ref, out = torch.zeros_like(q), torch.zeros_like(q)
        B.iwdft_pages_attn(values, exponents, q, starts, table, lens, ref, **window)
        plan = B.iwdft_pages_plan(starts, table, lens, batch, 9000, H, G * H, P, DT[dtype], **window)
        B.iwdft_pages_attn_shared(values, exponents, q, plan, table, out)
        err = float((out.double() - ref.double()).norm() / ref.double().norm())
        assert err < (2.0 ** -7 if dtype == "bf16" else 2.0 ** -17), err  # two roundings of the result; fp32: 22 bits of both calls, sums of 1000 tiles at random: 2 sqrt(1000) 2^-24 = 2^-18
        again = torch.zeros_like(q)
        B.iwdft_pages_attn_shared(values, exponents, q, plan, table, again)
        assert torch.equal(out, again)


def test_plans_that_do_not_fit():
    """Another plan's sizes, starts that overlap: out stays; the binding refuses what it can see."""
    rng = np.random.default_rng(1)
    pool = Pool(rng, forest_of(rng, "samples", 4, 100, 20), 16)
    q = torch.randn((1, 4, 4, 128), device=DEV)
    out = torch.full_like(q, 7.0)
    starts = ints([0, 3, 1, 4, 4])
    plan = B.iwdft_pages_plan(starts, pool.d_table, pool.d_lens, 4, pool.n_pages, 2, 4, 16, torch.float32)
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan, pool.d_table, out)
    assert (out == 7.0).all()
    good = B.iwdft_pages_plan(ints(range(5)), pool.d_table, pool.d_lens, 4, pool.n_pages, 2, 4, 16, torch.float32, plan=plan)
    assert good is plan
    plan.n_recent = 5                                           # not what the buffer holds
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan, pool.d_table, out)
    assert (out == 7.0).all()
    plan.n_recent = 0
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan, pool.d_table, out)
    assert not (out == 7.0).all(dim=-1).any()
    for bad in (dict(q=q[:, :3].contiguous()), dict(q=q.bfloat16()), dict(table=pool.d_table[:3]), dict(out=out[:, :, :2]), dict(values=pool.values[:, :-1].contiguous(), exponents=pool.exponents[:, :-1].contiguous())):
        args = {**dict(values=pool.values, exponents=pool.exponents, q=q, plan=plan, table=pool.d_table, out=out), **bad}
        with pytest.raises(ValueError):
            B.iwdft_pages_attn_shared(**args)
    with pytest.raises(ValueError):
        B.iwdft_pages_plan(ints(range(5)), pool.d_table, pool.d_lens, 4, pool.n_pages, 2, 4, 16, torch.float32, n_recent=9, plan=plan)


# ------------------------------------------------------------------------------------------------------------------ together
class Served:
    """A shared PagedCache and the oracles of its tables and of its pool, through the same steps."""

    def __init__(self, rng, batch, W, n_pages, P, heads, G, layers, dtype):
        self.c = B.PagedCache(layers, n_pages, heads, heads * G, 128, DT[dtype], batch, W * P, P, DEV, shared=True)
        self.t, self.store, self.rng, self.dtype, self.G = Tables(batch, W, n_pages, P), po.Store(layers, n_pages, heads, P), rng, dtype, G

    def tokens(self, n, heads):
        L = self.store.raw.shape[0]
        return dev(self.rng.normal(size=(L, n, heads, 128)) * 2.0 ** self.rng.integers(-2, 3, size=(1, n, 1, 1))).to(DT[self.dtype])

    def fork(self, parent, keep=None):
        self.t.fork(parent, keep)
        self.c.fork(ints(parent), None if keep is None else ints(keep))

    def step(self, want, shared=True, **windows):
        layers, _, heads = self.store.raw.shape[:3]
        n = int(sum(max(0, w - h) for w, h in zip(want, self.t.lens))) + 2
        starts, slots, copies = self.t.resize(want, n)
        for a, b in copies[copies[:, 0] >= 0]:
            self.store.raw[:, b], self.store.exponents[:, b] = self.store.raw[:, a], self.store.exponents[:, a]
        k, v, q = self.tokens(n, heads), self.tokens(n, heads), self.tokens(n, heads * self.G)
        self.store.write(f64(k), f64(v), list(slots))
        d_starts, d_slots = self.c.resize(ints(want), n)
        assert np.array_equal(d_starts.cpu().numpy(), starts) and np.array_equal(d_slots.cpu().numpy(), slots)
        plan = self.c.plan(d_starts, n, **windows) if shared else None
        outs = []
        for layer in range(layers):
            self.c.write(k[layer:layer + 1], v[layer:layer + 1], d_slots, layer)
            outs.append(self.c.attend(q[layer:layer + 1], d_starts, layer, plan=plan, **({} if shared else windows)))
        out = torch.cat(outs)
        ref, *rest = self.store.attend(f64(q), starts, self.t.table, self.t.lens, **windows)
        m = int(starts[-1])
        near(out[:, :m], ref[:, :m], *(r[:, :m] for r in rest), self.dtype)
        assert not out[:, m:].any()

    def same_pool(self):
        held = np.flatnonzero(self.t.refs > 0)
        assert np.array_equal(self.c.refs.cpu().numpy()[held], self.t.refs[held]) and np.array_equal(self.c.lens.cpu().numpy(), self.t.lens)
        assert np.array_equal(self.c.values[:, held].cpu().numpy(), self.store.packed()[:, held])
        assert np.array_equal(self.c.exponents[:, held].cpu().numpy(), self.store.exponents[:, held])


@pytest.mark.parametrize("dtype,P,G,windows", [("bf16", 32, 4, {}), ("f32", 16, 2, {}), ("bf16", 16, 8, dict(n_sink=3, n_recent=60))])
def test_beams_from_a_prompt_to_an_answer(dtype, P, G, windows):
    """A prompt, its samples, steps of beam search that drop and double beams, a second prompt, drafts taken back, pages moved together, another pool."""
    rng = np.random.default_rng(P + G)
    s = Served(rng, 8, 12, 90, P, 2, G, 2, dtype)
    s.step([5 * P + 3, 0, 0, 0, 0, 0, 0, 0], **windows)
    s.fork([0] * 6 + [6, 7])
    s.same_pool()
    for r in range(6):
        s.step([n + 1 if n and b != 3 else -1 for b, n in enumerate(s.t.lens)], shared=r != 2, **windows)
        s.same_pool()
        if r == 1:
            s.step([-1] * 6 + [3 * P, 40], **windows)
        s.fork(rng.choice(6, size=6).tolist() + [6, 7 if r < 4 else 6], None if r % 2 else [-1] * 7 + [2 * P + 5])
    s.step([int(n) + 3 for n in s.t.lens], **windows)                      # drafts
    s.step([max(0, int(n) - 2) for n in s.t.lens], **windows)              # two of three are taken back
    for n_moves in (3, 45):
        for a, b in s.t.compact(n_moves):
            if a >= 0:
                s.store.raw[:, b], s.store.exponents[:, b] = s.store.raw[:, a], s.store.exponents[:, a]
        s.c.compact(n_moves)
        s.same_pool()
    held = int((s.t.refs > 0).sum())
    before = s.c.read(40)
    with pytest.raises(ValueError):
        s.c.repool(held - 1)
    for n_pages in (held + 40, held):
        s.c.repool(n_pages)
        assert s.c.values.shape[1] == n_pages and int(s.c.free[0]) == n_pages - held and all(torch.equal(x, y) for x, y in zip(before, s.c.read(40)))
        assert s.c.free[1:1 + n_pages - held].tolist() == list(range(n_pages - 1, held - 1, -1))
    s.c.fork(ints(range(8)), ints([0] * 8))
    assert int(s.c.free[0]) == held and not s.c.refs.any() and not s.c.lens.any()


def test_a_pool_is_given_back_when_its_last_read_is_done():
    """repool on a stream of its own: once it returns, nobody reads the old pool, whose memory the next allocation may get."""
    rng = np.random.default_rng(21)
    c = B.PagedCache(2, 400, 2, 4, 128, torch.bfloat16, 2, 4000, 16, DEV, shared=True)
    x = dev(rng.normal(size=(2, 2, 3000, 2, 128))).bfloat16()
    _, slots = c.resize(ints([3000, 0]), 3000)
    c.write(x[0], x[1], slots)
    c.fork(ints([0, 0]))
    before, side = c.read(3000), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for given, n_pages in ((side, 300), (side.cuda_stream, 200)):
        c.repool(n_pages, stream=given)
        assert side.query() and c.values.shape[1] == n_pages
    assert all(torch.equal(a, b) for a, b in zip(before, c.read(3000)))


def test_a_shared_beginning_is_compressed():
    """Two requests with one beginning, handed to the frequency domain together: as from pages of their own."""
    rng = np.random.default_rng(7)
    c = B.PagedCache(1, 60, 2, 4, 128, torch.bfloat16, 3, 400, 16, DEV, shared=True)
    x = dev(rng.normal(size=(2, 1, 300, 2, 128))).bfloat16()
    _, slots = c.resize(ints([300, 0, 0]), 300)
    c.write(x[0], x[1], slots)
    c.fork(ints([0, 0, 2]), ints([-1, 272, -1]))
    K, V = c.read(272)
    assert torch.equal(K[:, 0], K[:, 1]) and torch.equal(V[:, 0], V[:, 1])
    frozen = B.Cache(1, 2, 2, 4, 128, torch.bfloat16, 256, [np.arange(32, dtype=np.int32)], n_sink=4, n_recent=12, device=DEV)
    assert c.compress(frozen, sequences=[1, 0]) == [0, 28]
    a, b = frozen.export_coeffs(0)
    assert torch.equal(a[0], a[1]) and torch.equal(b[0], b[1])
    frozen.close()


def test_a_captured_step_replayed():
    """Fork, growth with copies on write, writing, the plan and attention of two layers in a graph: every replay as the same step issued call by call, with eager work in between."""
    rng = np.random.default_rng(11)
    P, batch, H, G, n = 16, 6, 2, 4, 12

    def cache():
        return B.PagedCache(2, 80, H, H * G, 128, torch.bfloat16, batch, 20 * P, P, DEV, shared=True)

    first = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((2, 2, 100, H, 128), device=DEV, generator=first).bfloat16()
    caches = [cache(), cache()]
    for c in caches:
        _, slots = c.resize(ints([100, 0, 0, 0, 0, 0]), 100)
        c.write(x[0], x[1], slots)
    parent, want = ints([0] * 6), ints([-1] * 6)
    k, v = (torch.zeros((2, n, H, 128), device=DEV, dtype=torch.bfloat16) for _ in range(2))
    q, out = (torch.zeros((2, n, H * G, 128), device=DEV, dtype=torch.bfloat16) for _ in range(2))

    def step(c, out):
        c.fork(parent)
        starts, slots = c.resize(want, n)
        plan = c.plan(starts, n)
        for layer in range(2):
            c.write(k[layer:layer + 1], v[layer:layer + 1], slots, layer)
            c.attend(q[layer:layer + 1], starts, layer, out=out[layer:layer + 1], plan=plan)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(cache(), torch.zeros_like(out))  # before the capture: everything loaded
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], out)
    for r in range(6):
        parent.copy_(ints(rng.integers(0, 6, size=6) if r else [0] * 6))
        lens = caches[1].lens[parent.long()]
        want.copy_(lens + ints(rng.integers(0, 3, size=6)))
        for y in (k, v, q):
            y.normal_()
        graph.replay()
        other = torch.zeros_like(out)
        step(caches[1], other)
        torch.cuda.synchronize()
        m = int((caches[1].lens - lens).sum())
        assert torch.equal(out[:, :m], other[:, :m]) and m > 0
        assert torch.equal(caches[0].refs, caches[1].refs) and torch.equal(caches[0].lens, caches[1].lens)
        held = caches[0].refs > 0
        assert torch.equal(caches[0].values[:, held], caches[1].values[:, held])


def test_two_graphs_and_another_stream():
    """Two captured attentions on one plan, replayed at once on two streams, and calls on a stream of their own."""
    rng = np.random.default_rng(12)
    pool = Pool(rng, forest_of(rng, "samples", 24, 900, 300), 32, heads=4)
    q = [torch.randn((1, 24, 16, 128), device=DEV).bfloat16() for _ in range(2)]
    plan = plan_of(pool, range(25), 24, 4, "bf16")
    ref = [torch.zeros_like(x) for x in q]
    for x, o in zip(q, ref):
        B.iwdft_pages_attn_shared(pool.values, pool.exponents, x, plan, pool.d_table, o)
    out, graphs, streams = [torch.zeros_like(x) for x in q], [], [torch.cuda.Stream() for _ in q]
    torch.cuda.synchronize()
    for x, o in zip(q, out):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(4):
                B.iwdft_pages_attn_shared(pool.values, pool.exponents, x, plan, pool.d_table, o)
        graphs.append(g)
    for _ in range(5):
        for o in out:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
    side = torch.cuda.Stream()
    o = torch.zeros_like(ref[0])
    side.wait_stream(torch.cuda.current_stream())
    starts = ints(range(25))
    torch.cuda.synchronize()
    p = B.iwdft_pages_plan(starts, pool.d_table, pool.d_lens, 24, pool.n_pages, 4, 16, 32, torch.bfloat16, stream=side)
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q[0], p, pool.d_table, o, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(o, ref[0])


def test_a_plan_is_dropped_while_another_stream_reads_it():
    """Made on one stream, read on another that is still at work when the plan goes: its memory is not handed out before."""
    rng = np.random.default_rng(22)
    pool = Pool(rng, forest_of(rng, "samples", 24, 900, 300), 32, heads=4)
    starts, q = ints(range(25)), torch.randn((1, 24, 16, 128), device=DEV).bfloat16()
    ref, out = torch.zeros_like(q), torch.zeros_like(q)
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan_of(pool, range(25), 24, 4, "bf16"), pool.d_table, ref)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for drop_on, read_on in ((side, torch.cuda.current_stream()), (torch.cuda.current_stream(), side)):
        with torch.cuda.stream(drop_on):
            plan = B.iwdft_pages_plan(starts, pool.d_table, pool.d_lens, 24, pool.n_pages, 4, 16, 32, torch.bfloat16)
            drop_on.synchronize()
            size, at = plan.buffer.nbytes, plan.buffer.data_ptr()
        with torch.cuda.stream(read_on):
            out.zero_()
            torch.cuda._sleep(20_000_000)
            B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan, pool.d_table, out)
        del plan
        with torch.cuda.stream(drop_on):
            others = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(4)]
            assert all(t.data_ptr() != at for t in others) or read_on.query()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


def test_calls_without_rows_or_sequences():
    """No new tokens, no sequences, sequences that bring nothing: nothing is written where nothing is to be."""
    rng = np.random.default_rng(13)
    pool = Pool(rng, forest_of(rng, "samples", 3, 60, 10), 16)
    none = torch.empty((1, 0, 4, 128), device=DEV)
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, none, plan_of(pool, [0] * 4, 0, 2, "f32"), pool.d_table, torch.empty_like(none))
    q = torch.randn((1, 5, 4, 128), device=DEV)
    out = torch.full_like(q, 7.0)
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan_of(pool, [0] * 4, 5, 2, "f32"), pool.d_table, out)
    assert (out == 7.0).all()
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan_of(pool, [2, 2, 4, 4], 5, 2, "f32"), pool.d_table, out)
    assert (out[:, [0, 1, 4]] == 7.0).all() and not (out[:, 2:4] == 7.0).any()
    table, lens = torch.empty((0, 4), dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    plan = B.iwdft_pages_plan(ints([0]), table, lens, 5, pool.n_pages, 2, 4, 16, torch.float32)
    out.fill_(7.0)
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan, table, out)
    assert (out == 7.0).all()
    zero = Pool(rng, [(-1, 0, 40), (0, 0, 0), (0, 40, 40)], 16)
    attend(zero, rng, [1, 2, 3], 2, "f32")                      # a sequence without tokens whose rows see nothing
    B.iwdft_pages_copy(torch.empty((0, 2), dtype=torch.int32, device=DEV), pool.values, pool.exponents)
    with pytest.raises(ValueError, match="shared"):
        B.PagedCache(1, 4, 1, 1, 128, torch.float32, 2, 64, 16, DEV).fork(ints([0, 0]))
    with pytest.raises(B.IwdftError):
        B.PagedCache(1, 4, 1, 1, 128, torch.float32, 1025, 64, 16, DEV, shared=True)


def test_copy_of_more_than_the_caches_hold():
    """Over 256 MB of pages go another way."""
    g = torch.Generator(device=DEV).manual_seed(1)
    values = torch.randint(0, 256, (2, 300, 9, 2, 128 * 128), dtype=torch.uint8, device=DEV, generator=g)
    exponents = torch.randint(-100, 100, (2, 300, 9, 2), dtype=torch.int32, device=DEV, generator=g)
    other = torch.zeros((2, 520, 9, 2, 128 * 128), dtype=torch.uint8, device=DEV), torch.zeros((2, 520, 9, 2), dtype=torch.int32, device=DEV)
    to = torch.randperm(520, device=DEV, generator=g)[:500].to(torch.int32)
    source = torch.randint(-1, 300, (500,), dtype=torch.int32, device=DEV, generator=g)
    B.iwdft_pages_copy(torch.stack([source, to], 1).contiguous(), values, exponents, *other)
    there = source >= 0
    assert int(there.sum()) > 400 and torch.equal(other[0][:, to[there].long()], values[:, source[there].long()])
    assert torch.equal(other[1][:, to[there].long()], exponents[:, source[there].long()])
    rest = torch.ones(520, dtype=torch.bool, device=DEV)
    rest[to[there].long()] = False
    assert not other[0][:, rest].any() and not other[1][:, rest].any()


def test_copy_of_a_list_longer_than_a_launch():
    """More than 2^24 workgroups, most of them of pairs that are not there: pages at both ends of the list and at the borders between launches, each layer a launch of its own."""
    values = torch.randint(0, 256, (2, 40, 8, 2, 128 * 128), dtype=torch.uint8, device=DEV)
    exponents = torch.randint(-100, 100, (2, 40, 8, 2), dtype=torch.int32, device=DEV)
    n = 300_000
    pairs, ref = torch.full((n, 2), -1, dtype=torch.int32), (values.clone(), exponents.clone())
    for i, at in enumerate((0, 1, 262_142, 262_143, 262_144, n - 1)):
        pairs[at] = torch.tensor([i, 39 - i])
        ref[0][:, 39 - i], ref[1][:, 39 - i] = values[:, i], exponents[:, i]
    B.iwdft_pages_copy(pairs.to(DEV), values, exponents)
    assert torch.equal(values, ref[0]) and torch.equal(exponents, ref[1])


def test_a_pool_of_most_of_the_memory():
    """130 GiB: a resize, pages moved together, 66 GiB of them into another pool."""
    L, H, P, n_pages, held = 32, 8, 32, 66_560, 33_900
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 220 << 30:
        pytest.skip("less than 220 GiB are free")
    c = B.PagedCache(L, n_pages, H, H, 128, torch.bfloat16, 3, held * P, P, DEV, shared=True)
    c.resize(ints([100 * P, (held - 2) * P, 0]), (held + 100) * P)
    c.fork(ints([0, 1, 1]))
    c.resize(ints([0, -1, (held - 2) * P + 1]), 1)
    for b in (1, 2):
        for place in (0, 77, held - 3, held - 2)[:2 + b]:
            page = int(c.table[b, place])
            c.values[:, page] = 16 * b + place % 16 + 1
            c.exponents[:, page] = b + place
    before = [[(c.values[:, p].clone(), c.exponents[:, p].clone()) for p in c.table[b, [0, 77, held - 3]].tolist()] for b in (1, 2)]
    last = int(c.table[2, held - 2])
    last = c.values[:, last].clone(), c.exponents[:, last].clone()

    def same():
        for b in (1, 2):
            for p, (v, e) in zip(c.table[b, [0, 77, held - 3]].tolist(), before[b - 1]):
                assert torch.equal(c.values[:, p], v) and torch.equal(c.exponents[:, p], e)
        p = int(c.table[2, held - 2])
        assert torch.equal(c.values[:, p], last[0]) and torch.equal(c.exponents[:, p], last[1]) and bool((last[0] > 32).all())

    n = n_pages - int(c.free[0])
    assert n == held - 1
    assert int((c.compact()[:, 0] >= 0).sum()) > 0 and int(c.table[1:].max()) == n - 1
    same()
    c.repool(n + 3)
    same()
    del c
    torch.cuda.empty_cache()


@pytest.mark.parametrize("batch,starts", [
    (3, [0, 4, 2, 6]), (3, [0, 2, 0, 1]), (4, [5, 8, 0, 6, 6]), (3, [4, 6, -3, 5]), (4, [0, 20, 3, 3, 5]), (70, [0] + [3, 2] * 35), (300, list(range(0, 299)) + [297, 299]),
])
def test_starts_that_overlap_are_found_whatever_they_add_up_to(batch, starts):
    """Fewer new tokens than there are rows, and a row of two sequences all the same: out stays."""
    rng = np.random.default_rng(batch)
    pool = Pool(rng, [(-1, 0, 50)] + [(0, 48, 50 + b % 7) for b in range(1, batch)], 16, heads=1)
    n = 400
    q = torch.randn((1, n, 2, 128), device=DEV)
    out = torch.full_like(q, 7.0)
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan_of(pool, starts, n, 2, "f32"), pool.d_table, out)
    assert (out == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch", [5, 69, 299])
def test_starts_that_go_back_and_do_not_overlap(batch, dtype):
    """Sequences whose rows lie in the other order, one without new tokens between every two of them."""
    rng = np.random.default_rng(batch)
    pool = Pool(rng, [(-1, 0, 50)] + [(0, 48, 50 + b % 7) for b in range(1, batch)], 16, heads=1)
    n = 2 * batch + 3
    starts = np.array([n - 2 * b + x for b in range(1, batch // 2 + 2) for x in (0, 2)], np.int32)[:batch + 1]
    q = dev(rng.normal(size=(1, n, 2, 128))).to(DT[dtype])
    out = torch.full_like(q, 7.0)
    B.iwdft_pages_attn_shared(pool.values, pool.exponents, q, plan_of(pool, starts, n, 2, dtype), pool.d_table, out)
    ref, *rest = pool.store.attend(f64(q), starts, pool.table, pool.lens)
    rows = ~np.isnan(ref).all(axis=(0, 2, 3))
    assert rows.sum() == 2 * ((batch + 1) // 2) and (out[:, ~rows] == 7.0).all()
    near(out[:, rows], ref[:, rows], *(r[:, rows] for r in rest), dtype)


def events_of(table, lens, news, n_pages, P):
    """What a plan counts: places where the set that a sequence names -- the first of those that hold the same page there -- begins, ends or changes; ends of rows do not count."""
    pages = [-(-int(n) // P) if m else 0 for n, m in zip(lens, news)]
    count, prev = 0, [-2] * len(lens)
    for c in range(max(pages, default=0)):
        first, cur = {}, []
        for b, row in enumerate(table):
            there = c < pages[b]
            cur.append(first.setdefault(int(row[c]), b) if there and 0 <= row[c] < n_pages else b if there else -1)
        changed = {x for pair in zip(cur, prev) if pair[0] != pair[1] for x in pair if x >= 0}
        count += sum(1 for b in changed if cur[b] == b or prev[b] == b and cur[b] >= 0)
        prev = cur
    return count


def head_of(plan):
    """Runs; whether the plan gave up on sharing."""
    head = plan.buffer[:64].view(torch.int32).tolist()
    return head[11], head[15]


@pytest.mark.parametrize("windows", [{}, dict(n_sink=5, n_recent=90)])
@pytest.mark.parametrize("kind,batch", [("samples", 7), ("samples", 70), ("samples", 300), ("nested", 7), ("nested", 100), ("chain", 7), ("chain", 30), ("cut", 7), ("alone", 12)])
def test_a_plan_shares_what_there_is(kind, batch, windows):
    """As many runs as sets and no more: not sequence by sequence, which gives the same results."""
    rng = np.random.default_rng(batch)
    for P in (16, 64):
        pool = Pool(rng, forest_of(rng, kind, batch, 320, 90), P, heads=1)
        for news in ([1 if n else 0 for n in pool.lens], [min(int(n), b % 4) for b, n in enumerate(pool.lens)]):
            starts = np.concatenate([[0], np.cumsum(news)])
            runs, unshared = head_of(plan_of(pool, starts, int(starts[-1]), 2, "bf16", **windows))
            count = events_of(pool.table, pool.lens, news, pool.n_pages, P)
            assert not unshared and runs == count <= 3 * batch
            if kind == "samples" and all(news):
                assert runs == 1 + batch                       # the prompt, and what each has of its own
            if kind == "alone" and all(news):
                assert runs == batch


@pytest.mark.parametrize("batch,W,n_pages", [(5, 9, 4), (40, 30, 3), (70, 12, 50), (3, 200, 2)])
def test_a_plan_gives_up_where_there_is_no_order(batch, W, n_pages):
    """More changes than a plan holds, and as many as it does."""
    rng = np.random.default_rng(batch)
    pool = Pool(rng, [(-1, 0, 16 * n_pages)], 16)
    pool.table = rng.integers(-1, n_pages + 4, size=(batch, W)).astype(np.int32)
    pool.lens = np.full(batch, W * 16, np.int32)
    given_up = 0
    for ordered in range(W, -1, -1):                            # so many places that all share
        pool.table[:, :ordered] = pool.table[0, :ordered] = 0
        pool.upload()
        runs, unshared = head_of(plan_of(pool, range(batch + 1), batch, 2, "f32"))
        count = events_of(pool.table, pool.lens, [1] * batch, pool.n_pages, 16)
        assert unshared == (count > 3 * batch) and runs == (batch if unshared else count)
        given_up += unshared
        pool.table = rng.integers(-1, n_pages + 4, size=(batch, W)).astype(np.int32)
    assert 0 < given_up <= W


def test_all_who_share_a_page_grow_and_the_last_of_them_stays():
    """With a page for whoever needs one; and with one too few, where a place before them takes it."""
    for spare, lens in ((2, [17, 21, 21]), (3, [17, 21, 21]), (1, [17, 20, 20])):
        t = Both(3, 4, 3 + spare, 16, np.random.default_rng(1))
        t.resize([16, 20, 0], 40)
        t.fork([0, 1, 1])
        copies = t.resize([17, 21, 21], 40)[2]
        assert list(t.o.lens) == lens and (copies[[0, 2]] == -1).all() and (copies[1, 0] >= 0) == (spare > 1)
