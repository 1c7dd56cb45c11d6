"""The 8-bit paged cache on the GPU against the integer / float64 oracle: whole numbers and stored bytes exactly, attention within what its roundings add up to."""
import numpy as np
import pytest
import torch

from oracle import iwdft_oracle as orc
from oracle import pages_oracle as po
from paper_2507_20030_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def f64(t):
    return t.detach().cpu().double().numpy()


class Pool:
    """Sequences of the given lengths with pages in random order, filled through the oracle; the same on the GPU."""

    def __init__(self, rng, lens, P, heads=2, layers=1, n_pages=None, scale=None, stale=True):
        used = sum(-(-n // P) for n in lens)
        n_pages = used + 3 if n_pages is None else n_pages
        self.store, self.P = po.Store(layers, n_pages, heads, P), P
        self.lens = np.array(lens, np.int32)
        self.table = np.full((len(lens), max(1, max(-(-n // P) for n in lens)) + 1), -1, np.int32)
        order = list(rng.permutation(n_pages))
        for b, n in enumerate(lens):
            for j in range(-(-n // P)):
                self.table[b, j] = order.pop()
        full = rng.normal(size=(layers, n_pages * P, heads, 128)) * (10.0 ** rng.uniform(-1, 1, size=128) if scale is None else scale)
        if stale:
            self.store.write(full, rng.normal(size=full.shape) * 10.0 ** rng.uniform(-2, 2, size=(1, full.shape[1], 1, 1)), np.arange(n_pages * P))
        self.upload()

    def upload(self):
        self.values, self.exponents = dev(self.store.packed()), dev(self.store.exponents)
        self.d_table, self.d_lens = dev(self.table), dev(self.lens)


# ------------------------------------------------------------------------------------------------------------------ tables
def check_resize(rng, B_, W, P, n_pages, n_slots, rounds, most):
    table, lens = np.full((B_, W), -1, np.int32), np.zeros(B_, np.int32)
    free = np.concatenate([[n_pages], rng.permutation(n_pages)]).astype(np.int32)
    d_table, d_lens, d_free = dev(table), dev(lens), dev(free)
    refused = 0
    for r in range(rounds):
        want = rng.integers(0, most + 1, size=B_)
        want = np.where(rng.random(B_) < 0.3, lens + rng.integers(0, 3, size=B_), want)
        want = np.where(rng.random(B_) < 0.1, -1, np.where(rng.random(B_) < 0.15, 0, want))
        if r % 3 == 2:
            want[rng.integers(B_)] = W * P + 1
        want = want.astype(np.int32)
        d_starts, d_slots = (torch.full((n,), 77, dtype=torch.int32, device=DEV) for n in (B_ + 1, n_slots))
        B.iwdft_pages_resize(dev(want), d_table, d_lens, d_free, d_starts, d_slots, P)
        starts, slots = po.resize(want, table, lens, free, n_slots, P)
        for name, got, ref in (("table", d_table, table), ("lens", d_lens, lens), ("free", d_free, free), ("starts", d_starts, starts), ("slots", d_slots, slots)):
            assert np.array_equal(got.cpu().numpy(), ref), (name, r)
        refused += int(((want > lens) & (want >= 0)).sum())
    return refused


@pytest.mark.parametrize("batch,W,P,n_pages,n_slots,most", [
    (1, 4, 16, 5, 64, 60), (3, 6, 32, 12, 200, 150), (16, 20, 16, 200, 300, 300), (64, 9, 128, 300, 2048, 1000), (1024, 3, 16, 900, 1500, 40),
    (1, 300, 16, 310, 5000, 4700), (40, 40, 32, 900, 30000, 1200), (1025, 4, 16, 2000, 700, 50), (2500, 5, 64, 6000, 100000, 300), (5, 3, 16, 9, 0, 40),
])
def test_tables_and_slots(batch, W, P, n_pages, n_slots, most):
    """Pools and slot maps that run out, lengths beyond the table, idle and finished sequences; one launch and two."""
    refused = check_resize(np.random.default_rng(batch * W + P), batch, W, P, n_pages, n_slots, 7, most)
    assert refused > 0


def test_a_call_that_undoes_another_leaves_the_stack():
    for batch, new in ((9, 40), (9, 900)):
        rng = np.random.default_rng(new)
        base = rng.integers(0, 500, size=batch).astype(np.int32)
        c = B.PagedCache(1, 700, 1, 1, 128, torch.float32, batch, 2000, 16, DEV)
        c.resize(dev(base), 5000)
        free, table = c.free.clone(), c.table.clone()
        s1 = c.resize(dev(base + new), batch * new)
        c.resize(dev(base), batch * new)
        assert torch.equal(c.free[:1 + int(free[0])], free[:1 + int(free[0])]) and torch.equal(c.free[0], free[0])
        s2 = c.resize(dev(base + new), batch * new)
        assert torch.equal(s1[0], s2[0]) and torch.equal(s1[1], s2[1]) and int(c.lens.sum()) == int(base.sum()) + batch * new
        held = table >= 0
        assert torch.equal(c.table[held], table[held])


def test_no_sequences_and_damaged_arrays():
    """batch 0; lengths, counts, tables and page ids that nothing valid has: no slot outside of the pool comes out."""
    starts, slots = torch.full((1,), 5, dtype=torch.int32, device=DEV), torch.full((7,), 5, dtype=torch.int32, device=DEV)
    e = torch.empty(0, dtype=torch.int32, device=DEV)
    B.iwdft_pages_resize(e, torch.empty((0, 4), dtype=torch.int32, device=DEV), e, dev(np.arange(5, dtype=np.int32)), starts, slots, 16)
    assert starts.tolist() == [0] and slots.tolist() == [-1] * 7
    for n_slots in (400, 3000):
        table = dev(np.array([[9999, -5, 2, 3], [1, 1, 1, 1], [0, 0, 0, 0]], np.int32))
        lens = dev(np.array([10 ** 9, -7, 33], np.int32))
        free = dev(np.array([2 ** 30, 77777, -3, 5, 6], np.int32))
        starts, slots = torch.empty(4, dtype=torch.int32, device=DEV), torch.empty(n_slots, dtype=torch.int32, device=DEV)
        B.iwdft_pages_resize(dev(np.array([3, 64, 64], np.int32)), table, lens, free, starts, slots, 16)
        B.iwdft_pages_resize(dev(np.array([64, 0, 1], np.int32)), table, lens, free, starts, slots, 16)
        s = slots.cpu().numpy()
        assert ((s >= -1) & (s < 4 * 16)).all() and 0 <= int(free[0]) <= 4


# ------------------------------------------------------------------------------------------------------------------ writing
def run_write(pool, k, v, slots, layer, dtype):
    dk, dv = dev(k).to(dtype), dev(v).to(dtype)
    B.iwdft_pages_write(pool.values, pool.exponents, dk, dv, dev(np.asarray(slots, np.int32)), layer)
    pool.store.write(f64(dk), f64(dv), list(slots), layer)


def same_pool(pool):
    got, ref = pool.values.cpu().numpy(), pool.store.packed()
    nan = (ref & 127) == 127
    assert np.array_equal(pool.exponents.cpu().numpy(), pool.store.exponents)
    assert np.array_equal(nan, (got & 127) == 127) and np.array_equal(got[~nan], ref[~nan])


def slots_of(pool, runs):
    """runs: (sequence, first position, tokens)."""
    return [int(pool.table[b, p // pool.P]) * pool.P + p % pool.P for b, first, n in runs for p in range(first, first + n)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_write_prompts_and_single_tokens(P, dtype):
    rng = np.random.default_rng(P)
    pool = Pool(rng, [3 * P + 5, 1, 2 * P, 7, 130], P, heads=3, layers=3)
    runs = [(0, 0, 3 * P + 5), (1, 0, 1), (2, P - 3, P + 3), (3, 6, 1), (4, 100, 30)]
    slots = slots_of(pool, runs)
    cut = len(slots) // 2
    slots[cut:cut] = [-1, -1]                                   # rows of nothing in between
    slots += [-1, 10 ** 6, -5]
    k, v = (rng.normal(size=(2, len(slots), 3, 128)) * 2.0 ** rng.integers(-3, 6, size=(1, len(slots), 1, 1)) for _ in range(2))
    run_write(pool, k, v, slots, 1, DT[dtype])
    same_pool(pool)
    for step in range(4):                                       # decode: one token each, louder and quieter
        lens = [3 * P + step - 8, step, P + step + 3]
        slots = slots_of(pool, [(0, lens[0], 1), (2, lens[2], 1), (4, 97 + step, 1)])
        k, v = (rng.normal(size=(3, 3, 3, 128)) * 8.0 ** rng.integers(-3, 4, size=(1, 3, 3, 1)) for _ in range(2))
        run_write(pool, k, v, slots, 0, DT[dtype])
        same_pool(pool)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_write_extreme_values(dtype):
    """Zeros, values next to the border of a scale, ties, the type's largest and smallest, infinities and NaN."""
    rng = np.random.default_rng(5)
    pool = Pool(rng, [40, 64], 32, heads=1)
    n = 40
    x = rng.normal(size=(1, n, 1, 128)).astype(np.float32)
    x[0, 0] = 0
    x[0, 1, 0, :8] = [448, -448, 449, 447.9, 1.75, 1.7500001, 2.0 ** -9, 2.0 ** -10]
    x[0, 2, 0, :6] = [np.inf, -np.inf, np.nan, -0.0, 3 * 2.0 ** -10, 5 * 2.0 ** -10]
    x[0, 3] = po.TABLE[rng.integers(0, 126, size=128)] + po.TABLE[rng.integers(0, 126, size=128)]
    x[0, 33, 0, 5] = np.nan
    x[0, 34:] *= 2.0 ** -20
    y = x.copy()
    y[0, 36, 0, 7] = 3.3e38 if dtype == "f32" else 3.3e38
    run_write(pool, x, y, slots_of(pool, [(0, 0, n)]), 0, DT[dtype])
    same_pool(pool)
    tiny = np.full((1, 20, 1, 128), 2.0 ** -120)
    run_write(pool, tiny, np.zeros_like(tiny), slots_of(pool, [(1, 0, 20)]), 0, DT[dtype])
    same_pool(pool)
    for scale in (2.0 ** -130, 2.0 ** -90, 1.0, 2.0 ** 100):    # a page whose exponent passes through the whole range
        x = rng.normal(size=(1, 1, 1, 128)) * scale
        at = 20 + [2.0 ** -130, 2.0 ** -90, 1.0, 2.0 ** 100].index(scale)
        run_write(pool, x, x, slots_of(pool, [(1, at, 1)]), 0, DT[dtype])
        same_pool(pool)


def test_write_far_into_a_long_pool():
    """Offsets beyond 32 bits: 5 GB of values, the pages at both ends; neighbours stay."""
    n_pages, P = 160_000, 128
    values, exponents = torch.zeros((1, n_pages, 1, 2, P * 128), dtype=torch.uint8, device=DEV), torch.zeros((1, n_pages, 1, 2), dtype=torch.int32, device=DEV)
    assert values.numel() > 1 << 32
    rng = np.random.default_rng(3)
    k, v = (dev(rng.normal(size=(1, 200, 1, 128))).float() for _ in range(2))
    pages = [n_pages - 1, 140_001]
    slots = np.array([pages[j // P] * P + j % P for j in range(200)], np.int32)
    B.iwdft_pages_write(values, exponents, k, v, dev(slots))
    small = po.Store(1, 2, 1, P)
    small.write(f64(k), f64(v), list(range(200)))
    got = values[:, pages].cpu().numpy()
    ref = small.packed()
    assert np.array_equal(got, ref) and np.array_equal(exponents[:, pages].cpu().numpy(), small.exponents)
    assert int((values.view(-1)[:: 1 << 20] != 0).sum()) <= 1 and not values[0, 140_002].any() and not values[0, 0].any()
    table, lens = dev(np.array([pages], np.int32)), dev(np.array([200], np.int32))
    K, V = (torch.empty((1, 1, 1, 200, 128), device=DEV) for _ in range(2))
    B.iwdft_pages_read(values, exponents, table, lens, K, V)
    rk, rv = small.read(np.array([[0, 1]]), [200], 200, 0, 1)
    assert np.array_equal(f64(K), rk) and np.array_equal(f64(V), rv)
    q, out = torch.randn((1, 1, 2, 128), device=DEV), torch.empty((1, 1, 2, 128), device=DEV)
    B.iwdft_pages_attn(values, exponents, q, dev(np.array([0, 1], np.int32)), table, lens, out)
    ref, *rest = small.attend(f64(q), [0, 1], np.array([[0, 1]]), [200])
    near(out, ref, *rest, "f32")


# ------------------------------------------------------------------------------------------------------------------ reading
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P,n", [(16, 1), (16, 43), (32, 70), (64, 64), (128, 137)])
def test_read(P, n, dtype):
    rng = np.random.default_rng(P + n)
    pool = Pool(rng, [n, 0, n // 2, n + 40, 3], P, heads=2, layers=3)
    pool.table[3, 1] = -1                                       # a page that is not there: its tokens are 0
    pool.upload()
    K, V = (torch.full((2, 5, 2, n, 128), float("nan"), device=DEV, dtype=DT[dtype]) for _ in range(2))
    B.iwdft_pages_read(pool.values, pool.exponents, pool.d_table, pool.d_lens, K, V, 1)
    ref = pool.store.read(pool.table, pool.lens, n, 1, 2)
    assert np.array_equal(f64(K), ref[0]) and np.array_equal(f64(V), ref[1])
    K2 = torch.full_like(K, float("nan"))
    B.iwdft_pages_read(pool.values, pool.exponents, pool.d_table, pool.d_lens, K2, None, 1)
    assert torch.equal(K, K2)


# ------------------------------------------------------------------------------------------------------------------ attention
def near(out, ref, weight, reach, seen, floor, dtype):
    """|out - ref| <= half a step of the result + A * (weights + scores + sums), A = sum p |v|:
    weights to 11 bits (bf16) or 22, the exponential one step of 2^-23 and its argument; a score errs by 2^-22 (fp32 query in two parts) and by the sums of 128
    products, 2^-24 each, of sum |q k|, twice (the denominator has it too); the sums over the tokens by 2^-24 for each of the tiles, parts and rescalings.
    And fp16 ends at 2^-25: a weight 2^lift P_j (lift 6, fp32 15) is off by that much, whatever its size.  With V_j = v_j 2^-e_j as stored, the result is
    sum P_j V_j / sum P_j 2^-e_j, and the largest P_j, j = *, is at least 1: the denominator at least 2^-e*, the error at most
    2^(-25 - lift) sum |V_j| / 2^-e*.  (Where the heaviest tokens store zeros in a channel, as small channels of a page do, nothing else is left.)"""
    got = f64(out)
    rows = ~np.isnan(ref).all(axis=(0, 2, 3)) if not np.isnan(weight).any() else np.ones(ref.shape[1], bool)
    got, ref, weight, reach, seen, floor = (x[:, rows] for x in (got, ref, weight, reach, seen, floor))
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    step, bits = (2.0 ** -8, 2.0 ** -11) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -22)
    # 1.45: log2 e, in which scores are taken
    score = (2.0 ** -22 + 140 * 2.0 ** -24) * reach * 1.45 + 2.0 ** -22
    rel = bits + 2 * score + (seen / 32 + 100) * 2.0 ** -24
    bound = step * np.abs(ref) + (rel[..., None] * weight + 2.0 ** (-25 - (6 if dtype == "bf16" else 15)) * floor) * (1 + step) + 1e-30
    err = np.abs(got - ref)
    ok = ~(err > bound) | np.isnan(ref)
    assert ok.all(), (float(np.nanmax(err / bound)), np.argwhere(~ok)[:5].tolist())


def attend(pool, rng, news, G, dtype, layer=0, layers=1, pad=0, q_scale=1.0, q=None, **kw):
    heads = pool.store.raw.shape[2]
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    n = int(starts[-1]) + pad
    q = dev(rng.normal(size=(layers, n, heads * G, 128)) * q_scale).to(DT[dtype]) if q is None else q
    out = torch.full_like(q, 7.0)
    B.iwdft_pages_attn(pool.values, pool.exponents, q, dev(starts), pool.d_table, pool.d_lens, out, layer, **kw)
    args = {k: v for k, v in kw.items() if k in ("n_sink", "n_recent")}
    ref, *rest = pool.store.attend(f64(q), starts, pool.table, pool.lens, layer, scale=kw.get("scale") or None, **args)
    if pad:
        assert (out[:, starts[-1]:] == 7.0).all()
        ref, out = ref[:, :starts[-1]], out[:, :starts[-1]]
        rest = [r[:, :starts[-1]] for r in rest]
    near(out, ref, *rest, dtype)
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("lens", [[1], [31, 32, 33], [0, 200, 5, 127, 128, 129], [700]])
def test_attention_single_tokens(lens, P, dtype):
    rng = np.random.default_rng(sum(lens) + P)
    attend(Pool(rng, lens, P), rng, [1 if n else 0 for n in lens], 4, dtype, pad=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G,heads", [(1, 1), (2, 3), (3, 2), (8, 1), (16, 1), (20, 1), (64, 1)])
def test_attention_heads(G, heads, dtype):
    rng = np.random.default_rng(G)
    attend(Pool(rng, [150, 40], 32, heads=heads, layers=2), rng, [2, 1], G, dtype, layer=1)
    attend(Pool(rng, [70], 16, heads=heads, layers=3), rng, [1], G, dtype, layer=1, layers=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,news,G", [
    ([5, 64, 33], [5, 64, 33], 4), ([300, 80, 0, 9], [37, 1, 0, 9], 3), ([200], [200], 1), ([190], [190], 8), ([513, 260], [129, 1], 4), ([90, 90], [17, 70], 2), ([40] * 70, [1] * 69 + [40], 2),
])
def test_attention_drafts_and_prompts(lens, news, G, dtype):
    rng = np.random.default_rng(len(lens) + G)
    attend(Pool(rng, lens, 16 if G % 2 else 64, heads=2), rng, news, G, dtype, pad=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sink,recent", [(0, 1), (0, 40), (10, 50), (33, 64), (1, 1), (64, 1000), (500, 3), (0, 2 ** 31 - 1), (2 ** 31 - 1, 5)])
def test_attention_windows(sink, recent, dtype):
    rng = np.random.default_rng(sink % 1000 + recent % 1000)
    attend(Pool(rng, [400, 61, 12, 300], 32), rng, [1, 7, 12, 90], 2, dtype, n_sink=sink, n_recent=recent)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_rows_before_the_first_token(dtype):
    """More new tokens than the sequence is long: the first ones see nothing and are 0; scale and padding rows."""
    rng = np.random.default_rng(8)
    pool = Pool(rng, [3, 0, 40], 16)
    out = attend(pool, rng, [8, 4, 1], 2, dtype, pad=3, scale=0.3)
    assert not out[:, :5].any() and not out[:, 8:12].any() and out[:, 5:8].all(dim=-1).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_does_not_see_what_is_masked(dtype):
    """NaN and the largest values behind a sequence's end, outside the window, in pages of nobody and in tokens that only later rows see; NaN that
    a row sees is its own."""
    rng = np.random.default_rng(9)
    for news, kw in (([1, 1], {}), ([6, 40], {}), ([6, 40], dict(n_sink=5, n_recent=20)), ([1, 1], dict(n_sink=3, n_recent=20)), ([60, 110], dict(n_sink=0, n_recent=40))):
        pool = Pool(rng, [75, 110], 32, heads=2)
        hidden = rng.integers(0, 2, size=pool.store.raw.shape[1:3])
        raw = pool.store.raw
        for b in (0, 1):
            n = int(pool.lens[b])
            raw[0, pool.table[b, (n - 1) // 32], :, :, n % 32 or 32:] = 0x7f                       # behind the end
            if kw.get("n_recent") == 20:
                raw[0, pool.table[b, 0], :, :, kw["n_sink"]:30] = 0xff                                   # between sinks and window of every row
        raw[0, pool.table[1, 109 // 32], 1, 1, 109 % 32, 40] = 0x7f                                     # V, the last token: the last row sees it
        raw[0, pool.table[0, 72 // 32], 0, 0, 72 % 32, 3] = 0x7f                                        # K, token 72
        del hidden
        pool.upload()
        out = attend(pool, rng, news, 2, dtype, **kw)
        nan = torch.isnan(out.float())
        last = sum(news) - 1
        assert nan[0, last, 2:4, 40].all() and int(nan[0, last].sum()) == 2  # heads 2, 3 read KV head 1
        assert nan[0, news[0] - 1, :2].all() and not nan[0, news[0] - 1, 2:].any()
        if news[0] == 6:
            assert not nan[0, :3].any() and nan[0, 3:6, :2].all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_queries_that_are_not_finite_stay_in_their_row(dtype):
    rng = np.random.default_rng(10)
    pool = Pool(rng, [100], 32, heads=1)
    q = torch.randn((1, 5, 2, 128), device=DEV).to(DT[dtype])
    q[0, 1, 0, 7], q[0, 3, 1, 0] = float("nan"), float("inf")
    out, ref = torch.empty_like(q), torch.empty_like(q)
    starts = dev(np.array([0, 5], np.int32))
    B.iwdft_pages_attn(pool.values, pool.exponents, q, starts, pool.d_table, pool.d_lens, out)
    q2 = torch.nan_to_num(q, nan=0.0, posinf=0.0)
    B.iwdft_pages_attn(pool.values, pool.exponents, q2, starts, pool.d_table, pool.d_lens, ref)
    bad = torch.isnan(out.float()).any(-1)
    assert bad.nonzero().tolist() == [[0, 1, 0], [0, 3, 1]] and torch.equal(out[~bad], ref[~bad])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_far_apart_scales(dtype):
    """Pages whose K or V are 2^40 times as large as others', queries from 2^-60 to 2^30: no weight overflows, none of the small pages' bits are lost."""
    rng = np.random.default_rng(11)
    P, n = 16, 160
    pool = Pool(rng, [n], P, heads=1, stale=False)
    for j in range(n // P):
        k = rng.normal(size=(1, P, 1, 128)) * (2.0 ** -30 if j % 3 == 1 else 1.0)
        v = rng.normal(size=(1, P, 1, 128)) * 2.0 ** ((-90, 0, 40, -40)[j % 4])
        pool.store.write(k, v, [int(pool.table[0, j]) * P + i for i in range(P)])
    pool.upload()
    for scale in (1.0, 2.0 ** -60, 30.0, 2.0 ** 30):
        attend(pool, rng, [3], 3, dtype, q_scale=scale)
    # one page only, of tiny values: the result is tiny and as exact as any
    pool.lens[0] = P
    pool.upload()
    out = attend(pool, rng, [3], 3, dtype)
    assert 0 < float(out.abs().max()) < 2.0 ** -80


def test_attention_of_pages_that_are_not_there():
    """Table entries outside the pool hold no tokens; a sequence of none but these is 0."""
    rng = np.random.default_rng(12)
    pool = Pool(rng, [100, 40, 200], 16)
    pool.table[0, 1], pool.table[0, 4], pool.table[2, 12] = -1, 10 ** 6, pool.store.raw.shape[1]
    pool.table[1] = -3
    pool.upload()
    out = attend(pool, rng, [2, 1, 9], 2, "bf16")
    assert not out[:, 2].any()


def test_attention_of_damaged_lengths_and_starts():
    """Nothing that they say reaches memory outside the arrays; rows of no sequence stay."""
    rng = np.random.default_rng(13)
    pool = Pool(rng, [100, 40, 64], 16)
    q, out = (torch.full((1, 6, 4, 128), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.iwdft_pages_attn(pool.values, pool.exponents, q, dev(np.array([5, 2, 2, 900], np.int32)), pool.d_table, dev(np.array([50, -9, 10 ** 9], np.int32)), out)
    assert (out[:, :2] == 3.0).all() and torch.isfinite(out.float()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,news,G,P", [([5000], [1], 4, 16), ([20000, 3], [3, 1], 1, 128), ([9000], [90], 2, 32), ([6000, 800], [1, 300], 2, 64)])
def test_attention_of_long_sequences_in_parts(lens, news, G, P, dtype):
    rng = np.random.default_rng(sum(lens))
    attend(Pool(rng, lens, P, heads=1), rng, news, G, dtype)
    if lens[0] < 9000:
        attend(Pool(rng, lens, P, heads=1), rng, news, G, dtype, n_sink=40, n_recent=2500)


# ------------------------------------------------------------------------------------------------------------------ together
def test_a_served_batch_from_prompt_to_frequency_domain():
    """Prompts, drafts that are partly taken back, single tokens, a request that ends and one that takes its pages, and the hand-over to iwdft_prefill."""
    rng = np.random.default_rng(14)
    L, H, G, P, n, NB = 2, 2, 2, 32, 3, 26
    c = B.PagedCache(L, NB, H, H * G, 128, torch.bfloat16, n, 400, P, DEV)
    store, table, lens = po.Store(L, NB, H, P), np.full((n, c.table.shape[1]), -1, np.int32), np.zeros(n, np.int32)
    free = np.concatenate([[NB], np.arange(NB)]).astype(np.int32)
    steps = [[70, 130, 0], [73, 134, 5], [71, 134, 6], [72, 135, 7], [0, 136, 8], [300, 137, 9], [301, 138, 10], [302, 300, 300], [256 + 9, 256 + 9, 256 + 9]]
    for i, want in enumerate(steps):
        want = np.array(want, np.int32)
        starts, slots = c.resize(dev(want), 700)
        r_starts, r_slots = po.resize(want, table, lens, free, 700, P)
        assert np.array_equal(starts.cpu().numpy(), r_starts) and np.array_equal(slots.cpu().numpy(), r_slots) and np.array_equal(c.lens.cpu().numpy(), lens)
        m = int(r_starts[-1]) + 2
        k, v = (torch.randn((L, m, H, 128), device=DEV, dtype=torch.bfloat16) for _ in range(2))
        q = torch.randn((L, m, H * G, 128), device=DEV, dtype=torch.bfloat16)
        for layer in range(L):  # as a model goes through them
            c.write(k[layer:layer + 1], v[layer:layer + 1], slots[:m].contiguous(), layer)
            out = c.attend(q[layer:layer + 1], starts, layer)
            store.write(f64(k[layer:layer + 1]), f64(v[layer:layer + 1]), list(r_slots[:m]), layer)
            ref, *rest = store.attend(f64(q[layer:layer + 1]), r_starts, table, lens, layer)
            near(out[:, :-2], ref[:, :-2], *[x[:, :-2] for x in rest], "bf16")
            assert not out[:, -2:].any()
    bins = [np.arange(40, dtype=np.int32)] * L
    cache = B.Cache(L, n, H, H * G, 128, torch.bfloat16, 256, bins, device=DEV, n_sink=4, n_recent=5)
    c.compress(cache)
    K, V = store.read(table, lens, 265, 0, L)
    for layer in range(L):
        SK, SV = cache.export_coeffs(layer)
        for b in range(n):
            for h in range(H):
                for got, x in ((SK, K), (SV, V)):
                    want = orc.prefill(x[layer, b, h, 4:260], bins[layer])
                    assert np.linalg.norm(got[b, h].cpu().numpy() - want) <= 1e-4 * np.linalg.norm(want)
    q = torch.randn((L, n, H * G, 128), device=DEV, dtype=torch.bfloat16)
    assert torch.isfinite(cache.attend(q).float()).all()
    with pytest.raises(ValueError):
        c.compress(B.Cache(L, 1, H, H * G, 128, torch.bfloat16, 256, bins, device=DEV))
    cache.close()


def test_a_step_in_a_captured_graph():
    """Tables, writing and attention of a decode step captured once and replayed, every replay against eager calls on a copy, with eager work between."""
    H, G, P, n, L = 2, 4, 16, 5, 2
    mk = lambda: B.PagedCache(L, 700, H, H * G, 128, torch.bfloat16, n, 2100, P, DEV)  # noqa: E731
    a, b = mk(), mk()
    gen = torch.Generator(DEV).manual_seed(4)
    rnd = lambda *s: torch.randn(s, generator=gen, device=DEV).to(torch.bfloat16)  # noqa: E731
    first = dev(np.array([2000, 1, 17, 0, 900], np.int32))
    k, v = rnd(L, 2918, H, 128), rnd(L, 2918, H, 128)
    for c in (a, b):
        _, slots = c.resize(first, 2918)
        c.write(k, v, slots)
    want, k1, v1, q1 = first.clone(), rnd(L, n, H, 128), rnd(L, n, H, 128), rnd(L, n, H * G, 128)
    out = torch.zeros_like(q1)

    def step(c, out):
        starts, slots = c.resize(want, n)
        c.write(k1, v1, slots)
        c.attend(q1, starts, out=out)
    step(a, out), step(b, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a, out)
    for i in range(6):
        want.copy_(torch.where(torch.arange(n, device=DEV) == i % n, want, want + 1))
        if i == 4:
            want[1] = 0
        for x in (k1, v1, q1):
            x.copy_(rnd(*x.shape))
        ref = torch.zeros_like(q1)
        step(b, ref)
        torch.cuda.synchronize()
        out.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        for x, y in ((out, ref), (a.values, b.values), (a.exponents, b.exponents), (a.table, b.table), (a.lens, b.lens), (a.free, b.free)):
            assert torch.equal(x, y), i


def test_two_calls_at_once_and_a_workspace_of_the_caller():
    rng = np.random.default_rng(15)
    pools = [Pool(rng, [3000], 32, heads=1) for _ in range(2)]
    qs = [torch.randn((1, 2, 8, 128), device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    starts = dev(np.array([0, 2], np.int32))
    call = lambda i, out, **kw: B.iwdft_pages_attn(pools[i].values, pools[i].exponents, qs[i], starts, pools[i].d_table, pools[i].d_lens, out, **kw)  # noqa: E731
    refs = [torch.empty_like(q) for q in qs]
    call(0, refs[0]), call(1, refs[1])
    need = B.iwdft_pages_attn_bytes(B.pages_desc(1, pools[0].values.shape[1], 1, 8, 128, 32, pools[0].table.shape[1]), 1, 1, 2)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(qs[0])
    call(0, out, workspace=ws)
    assert torch.equal(out, refs[0])
    with pytest.raises(B.IwdftError) as e:
        call(0, out, workspace=ws[:need - 256])
    assert e.value.code == B.IWDFT_ERR_SIZE
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[torch.zeros_like(qs[i]) for _ in range(20)] for i in range(2)]
    torch.cuda.synchronize()
    for r in range(20):
        for i in range(2):
            call(i, outs[i][r], stream=streams[i] if r % 2 else streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert torch.equal(o, refs[i])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("news", [[3, 1], [120, 1], [40, 100]])
@pytest.mark.parametrize("apart", [(-100, -6), (-30, 0), (-14, 2), (-6, 0), (-90, 30)])
def test_attention_over_pages_of_small_or_no_values(apart, news, dtype):
    """Pages of V that hold zeros or much smaller values than others have their full share of the weights: in front of the others, behind them, in turn."""
    rng = np.random.default_rng(news[0] - apart[0])
    P = 32 if apart[0] == -30 else 16
    for small in (lambda j: j < 4, lambda j: j >= 4, lambda j: j % 2 == 0):
        pool = Pool(rng, [150, 100], P, heads=1, stale=False)
        for b in (0, 1):
            for j in range(-(-int(pool.lens[b]) // P)):
                k, v = (rng.normal(size=(1, P, 1, 128)) for _ in range(2))
                v = v * 0.0 if small(j) and apart[0] == -100 else v * 2.0 ** apart[0 if small(j) else 1]
                pool.store.write(k, v, [int(pool.table[b, j]) * P + i for i in range(P)])
        pool.upload()
        attend(pool, rng, news, 3, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("news", [[2], [70]])
def test_attention_of_queries_of_all_sizes(news, dtype):
    """Channels of q from 2^-30 of the largest one on, rows of zeros, and the largest channel over a column of K that is zero.  Beside what `near` allows, a
    score errs by 2^-22 of the row's largest |q| (fp32, two fp16 parts: 2^-39) times sum |k|: added to `reach` in units of its factor."""
    rng = np.random.default_rng(21)
    heads, G = 2, 2
    pool = Pool(rng, [130], 32, heads=heads, scale=1.0)
    pool.store.raw[:, :, :, 0, :, 5] = 0
    pool.upload()
    q = rng.normal(size=(1, news[0], heads * G, 128)) * 2.0 ** -rng.uniform(0, 30, size=(1, news[0], heads * G, 128))
    q[0, 1] = 0.0
    q[0, 0, :, 5] = 2.0 ** 6
    q = dev(q).to(DT[dtype])
    starts, out = np.array([0, news[0]], np.int32), torch.empty_like(q)
    B.iwdft_pages_attn(pool.values, pool.exponents, q, dev(starts), pool.d_table, pool.d_lens, out)
    ref, weight, reach, seen, floor = pool.store.attend(f64(q), starts, pool.table, pool.lens)
    sums = np.array([np.abs(pool.store.sequence(0, h // G, 0, pool.table[0], 130)).sum(1).max() for h in range(heads * G)])
    err = 2.0 ** (-22 if dtype == "bf16" else -39) * np.abs(f64(q)).max(-1) * sums / np.sqrt(128.0)
    near(out, ref, weight, reach + err / (2.0 ** -22 + 140 * 2.0 ** -24), seen, floor, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,news,G,kw", [
    ([3000] + [20] * 70 + [1500], [1] * 72, 2, {}),                                   # more sequences than lanes, two of them cut
    ([20] * 66 + [1500, 900], [1] * 66 + [70, 90], 2, {}),                             # ... beside prompts
    ([2500, 700], [2, 1], 20, {}), ([3000], [1], 64, {}),                              # 33 to 64 rows
    ([1500], [75], 7, dict(n_sink=3, n_recent=1300)),                                  # 525 rows of 8 layers and heads: the other way of joining
    ([700, 40, 1300], [130, 1, 60], 3, {}),
])
def test_attention_schedules(lens, news, G, kw, dtype):
    rng = np.random.default_rng(sum(lens) + G)
    heads, layers = (2, 4) if lens == [1500] else (1, 2)
    pool = Pool(rng, lens, 16 if G % 2 else 64, heads=heads, layers=layers + 1)
    attend(pool, rng, news, G, dtype, layer=1, layers=layers, pad=2, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [16, 64])
def test_attention_with_pages_missing_everywhere(P, dtype):
    rng = np.random.default_rng(P + 1)
    pool = Pool(rng, [900, 300, 130, 64], P)
    for b, n in enumerate(pool.lens):
        gone = rng.random(-(-int(n) // P)) < 0.4
        gone[0] = b == 0
        pool.table[b, :len(gone)][gone] = rng.choice([-1, -2 ** 31, 2 ** 31 - 1, pool.store.raw.shape[1]], size=int(gone.sum()))
    pool.table[3] = -1
    pool.upload()
    for kw in ({}, dict(n_sink=20, n_recent=100)):
        attend(pool, rng, [90, 1, 70, 33], 2, dtype, pad=1, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_write_past_rows_of_nothing(dtype):
    """Pages' new tokens with any number of rows without a slot between them, in front and behind; runs that end with a segment of the slots."""
    rng = np.random.default_rng(23)
    for P, gaps in ((16, (1, 2, 600)), (128, (1, 63, 64, 65, 511, 512, 513, 1100))):
        pool = Pool(rng, [5 * P, 3 * P], P, heads=2)
        parts = [slots_of(pool, [(0, 3, 2 * P)]), slots_of(pool, [(0, 2 * P + 3, 1)]), slots_of(pool, [(0, 2 * P + 4, P)]), slots_of(pool, [(1, P - 1, 1)]),
                 slots_of(pool, [(1, P, P)]), slots_of(pool, [(0, 3 * P + 4, 7)])]
        for gap, those in [(gap, those) for gap in gaps for those in (parts[:-1], parts[-1:])]:  # the last part continues a page that others follow: a call of its own
            slots = []
            for part in those:
                cut = int(rng.integers(0, len(part) + 1))
                slots += part[:cut] + [-1] * gap + part[cut:]
            n = len(slots)
            k, v = (rng.normal(size=(1, n, 2, 128)) * 2.0 ** rng.integers(-3, 6, size=(1, n, 1, 1)) for _ in range(2))
            dk, dv = dev(k).to(DT[dtype]), dev(v).to(DT[dtype])
            B.iwdft_pages_write(pool.values, pool.exponents, dk, dv, dev(np.asarray(slots, np.int32)))
            # the oracle takes a page's runs one after the other; each call here continues what the last one left
            keep = [i for i, s in enumerate(slots) if s >= 0]
            runs, at = [], 0
            while at < len(keep):
                end = at + 1
                while end < len(keep) and keep[end] == keep[end - 1] + 1:
                    end += 1
                runs.append(keep[at:end])
                at = end
            for run in runs:
                pool.store.write(f64(dk)[:, run], f64(dv)[:, run], [slots[i] for i in run])
            same_pool(pool)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_beside_single_tokens_in_a_captured_graph(dtype):
    """Lengths and starts change between replays; the workspace is the graph's own; eager work between."""
    rng = np.random.default_rng(24)
    pool = Pool(rng, [1400, 900, 30], 32, heads=2)
    q = torch.randn((1, 160, 4, 128), device=DEV).to(DT[dtype])
    starts, lens = dev(np.array([0, 120, 121, 122], np.int32)), pool.d_lens.clone()
    out, ref = torch.zeros_like(q), torch.zeros_like(q)
    call = lambda o: B.iwdft_pages_attn(pool.values, pool.exponents, q, starts, pool.d_table, lens, o, n_sink=4, n_recent=1000)  # noqa: E731
    call(ref)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out)
    for new_lens, new_starts in (([1400, 900, 30], [0, 120, 121, 122]), ([130, 900, 5], [0, 1, 120, 125]), ([0, 0, 0], [0, 0, 0, 0]), ([1400, 900, 30], [0, 7, 107, 137])):
        lens.copy_(dev(np.array(new_lens, np.int32))), starts.copy_(dev(np.array(new_starts, np.int32)))
        q.normal_()
        ref.fill_(3.0)
        call(ref)
        out.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and (out[:, new_starts[-1]:] == 3.0).all()
        assert torch.isfinite(out.float()).all() and (out[:, :new_starts[-1]] != 3.0).any() == (new_starts[-1] > 0)


def test_calls_on_another_stream():
    """Everything on a stream of the caller's, given as such or as a number; arrays that are allocated for the call follow it."""
    rng = np.random.default_rng(25)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c, d = (B.PagedCache(1, 300, 2, 4, 128, torch.bfloat16, 2, 4000, 32, DEV) for _ in range(2))
    want = dev(np.array([3000, 50], np.int32))
    k, v, q = (torch.randn((1, 3050, h, 128), device=DEV).to(torch.bfloat16) for h in (2, 2, 4))
    K, V = (torch.empty((1, 2, 2, 100, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    torch.cuda.synchronize()
    starts, slots = c.resize(want, 3050, stream=side)
    c.write(k, v, slots, stream=side.cuda_stream)
    out = c.attend(q, starts, stream=side)
    got = c.read(100, stream=side.cuda_stream)
    s2, sl2 = d.resize(want, 3050)
    d.write(k, v, sl2)
    ref = d.attend(q, s2)
    K, V = d.read(100)
    torch.cuda.synchronize()
    assert torch.equal(out, ref) and torch.equal(got[0], K) and torch.equal(got[1], V) and torch.equal(c.values, d.values) and torch.equal(slots, sl2)
    del rng


def test_the_binding_refuses_what_does_not_fit_on_the_gpu():
    z = lambda *s, dtype=torch.int32, device=DEV: torch.zeros(s, dtype=dtype, device=device)  # noqa: E731
    f = torch.float32
    values, exponents = z(2, 4, 2, 2, 32 * 128, dtype=torch.uint8), z(2, 4, 2, 2)
    k, q, table, lens, starts, slots = z(1, 3, 2, 128, dtype=f), z(1, 3, 4, 128, dtype=f), z(2, 4), z(2), z(3), z(3)
    kv = z(1, 2, 2, 5, 128, dtype=f)
    calls = {
        "write": (B.iwdft_pages_write, dict(values=values, exponents=exponents, k=k, v=k.clone(), slots=slots - 1)),
        "attn": (B.iwdft_pages_attn, dict(values=values, exponents=exponents, q=q, starts=starts, table=table, lens=lens, out=q.clone())),
        "read": (B.iwdft_pages_read, dict(values=values, exponents=exponents, table=table, lens=lens, K=kv, V=kv.clone())),
        "resize": (B.iwdft_pages_resize, dict(want=lens.clone(), table=table, lens=lens, free=z(5), starts=starts, slots=slots, page_tokens=32)),
    }
    for name, (call, good) in calls.items():
        call(**good)
        for arg, t in good.items():
            if not isinstance(t, torch.Tensor):
                continue
            bad = [t.cpu(), t.to(torch.float64) if t.dtype != torch.uint8 else t.to(torch.int8), t[..., :-1], t.unsqueeze(0)]
            if t.numel() > 1 and t.dim() == 1:
                bad.append(torch.stack([t, t], 1)[:, 0])
            if t.dim() > 1:
                bad.append(t.transpose(0, 1).contiguous().transpose(0, 1) if t.shape[0] > 1 and t.shape[1] > 1 else torch.stack([t, t], -1)[..., 0])
            for x in bad:
                if name == "resize" and arg in ("free", "slots") and x.dim() == 1 and x.is_contiguous() and x.dtype == torch.int32 and x.is_cuda:
                    continue  # any length will do
                with pytest.raises((ValueError, B.IwdftError)):
                    call(**{**good, arg: x})
    for name in ("write", "attn", "read"):
        call, good = calls[name]
        for layer in (-1, 2, 2 ** 31 - 1):
            with pytest.raises(B.IwdftError):
                call(**good, layer=layer)
    with pytest.raises(ValueError):
        B.iwdft_pages_attn(**calls["attn"][1], workspace=torch.empty(10, dtype=torch.uint8))
    with pytest.raises(B.IwdftError):
        B.iwdft_pages_attn(**{**calls["attn"][1], "out": q})  # in place
    with pytest.raises(B.IwdftError):
        B.iwdft_pages_attn(**calls["attn"][1], n_sink=2)
    torch.cuda.synchronize()


@pytest.mark.parametrize("batch", [65, 256, 257, 1024])
@pytest.mark.parametrize("n_slots", [900, 2049])
def test_tables_of_every_kind_of_launch(batch, n_slots):
    """Sequences by one wave, 256 and 1024 threads, in one launch and two; a call that takes what it gives back."""
    check_resize(np.random.default_rng(batch + n_slots), batch, 6, 16, 2 * batch, n_slots, 5, 60)
    rng = np.random.default_rng(batch)
    table, lens = np.full((batch, 6), -1, np.int32), np.zeros(batch, np.int32)
    free = np.concatenate([[batch], rng.permutation(batch)]).astype(np.int32)
    arrays = [dev(x) for x in (table, lens, free)]
    for want in (np.where(np.arange(batch) % 2, 32, 0), np.where(np.arange(batch) % 2, 0, 32), np.full(batch, 16)):
        want = np.where(np.cumsum(want) <= n_slots, want, 0).astype(np.int32)
        d_starts, d_slots = (torch.full((n,), 77, dtype=torch.int32, device=DEV) for n in (batch + 1, n_slots))
        B.iwdft_pages_resize(dev(want), *arrays, d_starts, d_slots, 16)
        starts, slots = po.resize(want, table, lens, free, n_slots, 16)
        for got, ref in zip(arrays + [d_starts, d_slots], (table, lens, free, starts, slots)):
            assert np.array_equal(got.cpu().numpy(), ref)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("news", [[3, 1], [120, 1], [40, 100]])
@pytest.mark.parametrize("apart", [(-100, 60), (-95, 60), (-90, 112), (-100, 100), (-60, 112), (-30, 112)])
def test_attention_over_pages_very_far_apart(apart, news, dtype):
    """Pages of V whose sizes are 2^140 to 2^212 apart, more than fp32 holds: the small ones (-100: zeros) have their share of the weights all the same."""
    rng = np.random.default_rng(news[0] + apart[1] - apart[0])
    for small in (lambda j: j < 4, lambda j: j >= 4, lambda j: j % 2 == 0):
        pool = Pool(rng, [150, 100], 16, heads=1, stale=False)
        for b in (0, 1):
            for j in range(-(-int(pool.lens[b]) // 16)):
                k, v = (rng.normal(size=(1, 16, 1, 128)) for _ in range(2))
                v = v * 0.0 if small(j) and apart[0] == -100 else v * 2.0 ** apart[0 if small(j) else 1]
                pool.store.write(k, v, [int(pool.table[b, j]) * 16 + i for i in range(16)])
        pool.upload()
        for q_scale in (1.0, 8.0):
            attend(pool, rng, news, 3, dtype, q_scale=q_scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size,last", [(0.0, 1.0), (2.0 ** -92, 2.0 ** -92), (2.0 ** 110, 2.0 ** -80)])
@pytest.mark.parametrize("G", [3, 80])
def test_attention_over_many_pages_of_one_size(G, size, last, dtype):
    """65536 tokens whose values are zeros, tiny or huge, 40 others behind them: the denominator neither overflows nor vanishes, in a part's sums and in their join."""
    rng = np.random.default_rng(G)
    P, n = 128, 65536 + 40
    pool = Pool(rng, [n], P, heads=1, stale=False)
    store, pages = pool.store, pool.table[0, :n // P]
    k, v = (rng.normal(size=(1, 4 * P, 1, 128)) for _ in range(2))
    store.write(k, v * size, [int(p) * P + i for p in pages[:4] for i in range(P)])
    for j, page in enumerate(pages[4:]):
        store.raw[:, page], store.exponents[:, page] = store.raw[:, pages[j % 4]], store.exponents[:, pages[j % 4]]
    k, v = (rng.normal(size=(1, 40, 1, 128)) for _ in range(2))
    store.write(k, v * last, [int(pool.table[0, n // P]) * P + i for i in range(40)])
    pool.upload()
    attend(pool, rng, [1], G, dtype)


def filled(lens, max_tokens=400, L=2, H=2, G=2, P=32, dtype=torch.bfloat16):
    """A paged cache with sequences of these lengths and what the oracle reads from it."""
    c = B.PagedCache(L, 60, H, H * G, 128, dtype, len(lens), max_tokens, P, DEV)
    _, slots = c.resize(dev(np.array(lens, np.int32)), sum(lens))
    k, v = (torch.randn((L, sum(lens), H, 128), device=DEV).to(dtype) for _ in range(2))
    c.write(k, v, slots)
    store = po.Store(L, 60, H, P)
    store.unpack(c.values.cpu().numpy(), c.exponents.cpu().numpy())
    return c, store.read(c.table.cpu().numpy(), c.lens.cpu().numpy(), max(lens), 0, L)


def frequency_cache(batch, M=256, L=2, H=2, G=2, device=DEV, dtype=torch.bfloat16):
    return B.Cache(L, batch, H, H * G, 128, dtype, M, [np.arange(40, dtype=np.int32)] * L, device=device, n_sink=4, n_recent=5)


def same_coefficients(cache, tokens, rows):
    for layer in range(2):
        for got, x in zip(cache.export_coeffs(layer), tokens):
            for i, b in enumerate(rows):
                for h in range(2):
                    want = orc.prefill(x[layer, b, h, 4:260], np.arange(40))
                    assert np.linalg.norm(got[i, h].cpu().numpy() - want) <= 1e-4 * np.linalg.norm(want)


def test_compressing_sequences_that_are_too_short():
    """Zeros for tokens that never were would have weight: given ones are refused and nothing is written; of the whole batch a warning and the counts tell which they are."""
    for lens, short in (([265, 264], [1]), ([0, 300], [0]), ([20, 100], [0, 1])):
        c, tokens = filled(lens)
        cache = frequency_cache(2)
        before = cache.T
        with pytest.raises(ValueError, match=str(short[0])):
            c.compress(cache, sequences=[0, 1])
        assert cache.T == before
        with pytest.warns(UserWarning, match=str(short[-1])):
            assert c.compress(cache) == [n - 265 for n in lens]
        cache.close()


def test_compressing_some_sequences():
    """Those that are long enough, in the order given; what they have behind the prompt is told and stays in the pages."""
    c, tokens = filled([268, 20, 0, 265, 300])
    for rows, left in (([0], [3]), ([3, 0], [0, 3]), ([4, 3], [35, 0])):
        cache = frequency_cache(len(rows))
        assert c.compress(cache, sequences=rows) == left
        same_coefficients(cache, tokens, rows)
        with pytest.raises(ValueError):
            c.compress(cache, sequences=rows * 2)  # a batch of another size
        cache.close()
    for bad in ([5], [-1], [1]):
        cache = frequency_cache(1)
        with pytest.raises(ValueError):
            c.compress(cache, sequences=bad)
        cache.close()
    whole, tokens = filled([265, 270])
    cache, side = frequency_cache(2), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert whole.compress(cache, side) == [0, 5]
    side.synchronize()
    same_coefficients(cache, tokens, [0, 1])


def test_compressing_in_a_captured_graph():
    """Lengths may change before a replay: one that is too short then gives NaN, not a result with zeros for tokens."""
    c, tokens = filled([268, 270, 20])
    cache = frequency_cache(2)
    c.compress(cache, sequences=[0, 1])
    q = torch.randn((2, 2, 4, 128), device=DEV).to(torch.bfloat16)
    ref = cache.attend(q).clone()
    torch.cuda.synchronize()
    g, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(g):
        assert c.compress(cache, sequences=[0, 1]) is None
        cache.attend(q, out)
    for lens, ok in (([268, 270], [True, True]), ([268, 264], [True, False]), ([265, 270], [True, True]), ([0, 265], [False, True])):
        c.lens[:2].copy_(dev(np.array(lens, np.int32)))
        out.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        for b in (0, 1):
            assert torch.equal(out[:, b], ref[:, b]) if ok[b] else torch.isnan(out[:, b].float()).all(), lens


@pytest.mark.parametrize("names", [("cuda", "cuda:0"), ("cuda:0", "cuda"), ("cuda", "cuda")])
def test_one_device_under_two_names(names):
    """A cache made on "cuda" is on the same GPU as one made on "cuda:0"."""
    c = B.PagedCache(2, 20, 2, 4, 128, torch.bfloat16, 1, 400, 32, names[0])
    starts, slots = c.resize(dev(np.array([265], np.int32)), 265)
    k, v = (torch.randn((2, 265, 2, 128), device=DEV).to(torch.bfloat16) for _ in range(2))
    c.write(k, v, slots)
    cache = frequency_cache(1, device=names[1])
    assert c.compress(cache) == [0]
    assert torch.isfinite(cache.attend(torch.randn((2, 1, 4, 128), device=DEV).to(torch.bfloat16)).float()).all()
    cache.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,news,G", [([6, 20, 40], [1, 1, 3], 4), ([30, 8], [2, 8], 17), ([300], [1], 3), ([40, 12], [40, 12], 8), ([90], [70], 1)])
@pytest.mark.parametrize("channels", [(0, 1), (3, 40), (17, 127)])
def test_attention_of_products_that_cancel(channels, lens, news, G, dtype):
    """Two channels whose products are hundreds of times as large as the others' and cancel: a score is a sum in fp32, so the small ones keep their bits.  `near`
    allows for 140 * 2^-24 of the sum of all |products|."""
    rng = np.random.default_rng(channels[0] + len(lens) + G)
    for size in (50.0, 400.0):
        pool = Pool(rng, lens, 16, heads=2, scale=1.0)
        raw = pool.store.raw
        raw[:, :, :, 0, :, :] = po.to_e4m3(rng.normal(size=raw.shape[:3] + raw.shape[4:]))
        raw[:, :, :, 0, :, channels[0]] = po.to_e4m3(size * rng.uniform(0.5, 1.0, size=raw.shape[:3] + raw.shape[4:5]))
        raw[:, :, :, 0, :, channels[1]] = raw[:, :, :, 0, :, channels[0]] ^ 128
        pool.store.exponents[..., 0] = 0
        pool.upload()
        q = dev(rng.normal(size=(1, sum(news), 2 * G, 128))).to(DT[dtype])
        q[..., channels[0]] = q[..., channels[1]] = 8.0 * (1.0 + torch.rand(q.shape[:3], device=DEV)).to(DT[dtype])
        attend(pool, rng, news, G, dtype, q=q)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,news,G", [([32], [17], 17), ([27], [6], 12), ([0, 27, 20], [0, 25, 20], 8), ([2, 3, 1], [1, 1, 1], 33), ([324, 158], [12, 12], 8)])
def test_attention_of_large_scores(lens, news, G, dtype):
    rng = np.random.default_rng(G + sum(lens))
    for P in (16, 128):
        attend(Pool(rng, lens, P, heads=2), rng, news, G, dtype, q_scale=20.0)
