"""Pages that sequences share, without a GPU: the oracle's own pins, and what the library and the binding refuse before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pages_oracle as po
from oracle.pages_shared_oracle import Tables
from paper_2507_20030_amd import binding as B


# ------------------------------------------------------------------------------------------------------------------ oracle
def test_the_oracle_by_hand():
    t = Tables(4, 4, 8, 16)
    starts, slots, copies = t.resize([20, 0, 16, 0], 40)
    assert t.pages(0) == [7, 6] and t.pages(2) == [5] and list(starts) == [0, 20, 20, 36, 36] and (copies == -1).all()
    t.fork([0, 0, 2, 2], [-1, 20, -1, 9])                    # 1 begins as 0, 3 with nine tokens of 2
    assert t.pages(1) == [7, 6] and t.pages(3) == [5] and list(t.lens) == [20, 20, 16, 9] and list(t.refs) == [0, 0, 0, 0, 0, 2, 2, 2]
    starts, slots, copies = t.resize([21, 21, 17, 10], 40)   # 0 leaves page 6 to 1, which stays; 2 begins a page; 3 leaves page 5
    assert copies.tolist() == [[6, 4], [-1, -1], [-1, -1], [5, 2]] and t.pages(0) == [7, 4] and t.pages(1) == [7, 6] and t.pages(2) == [5, 3] and t.pages(3) == [2]
    assert slots[:4].tolist() == [4 * 16 + 4, 6 * 16 + 4, 3 * 16, 2 * 16 + 9] and t.free[0] == 2 and t.consistent()
    t.fork([1, 0, 2, 3], [0, -1, -1, -1])                    # 1 becomes 0, 0 is given up
    assert t.pages(1) == [7, 4] and t.pages(0) == [] and list(t.free[:4]) == [3, 0, 1, 6] and t.consistent()
    moves = t.compact(1)
    assert moves.tolist() == [[7, 0]] and t.pages(1) == [0, 4] and list(t.free[:4]) == [3, 7, 6, 1] and t.consistent()
    assert t.compact(4).tolist() == [[5, 1], [-1, -1], [-1, -1], [-1, -1]] and t.pages(2) == [1, 3] and list(t.free[:4]) == [3, 7, 6, 5]


@pytest.mark.parametrize("seed", range(4))
def test_the_oracle_keeps_its_books(seed):
    rng = np.random.default_rng(seed)
    t = Tables(9, 12, 60, 16, rng.permutation(60))
    for _ in range(40):
        t.fork(np.where(rng.random(9) < 0.5, np.arange(9), rng.integers(0, 9, size=9)), rng.integers(-1, 150, size=9))
        assert t.consistent()
        lens = t.lens.copy()
        _, slots, copies = t.resize(np.where(rng.random(9) < 0.6, lens + rng.integers(0, 30, size=9), rng.integers(-1, 200, size=9)), 300)
        assert t.consistent() and len(set(slots[slots >= 0])) == (slots >= 0).sum()
        assert not set(copies[copies[:, 0] >= 0, 0]) & set(copies[copies[:, 0] >= 0, 1])
        written = {int(s) // 16 for s in slots if s >= 0}
        assert all(t.refs[p] == 1 for p in written)          # nobody writes to what others hold
        if rng.random() < 0.3:
            t.compact(int(rng.integers(0, 30)))
            assert t.consistent()


def test_without_shared_pages_the_oracle_is_the_other_one():
    rng = np.random.default_rng(5)
    t = Tables(7, 9, 40, 16)
    table, lens, free = np.full((7, 9), -1, np.int32), np.zeros(7, np.int32), t.free.copy()
    for _ in range(30):
        want, n = rng.integers(-1, 160, size=7), int(rng.integers(0, 200))
        starts, slots, copies = t.resize(want, n)
        s2, l2 = po.resize(want, table, lens, free, n, 16)
        assert np.array_equal(starts, s2) and np.array_equal(slots, l2) and np.array_equal(lens, t.lens) and (copies == -1).all()
        assert np.array_equal(free[:1 + free[0]], t.free[:1 + t.free[0]])


# ---------------------------------------------------------------------------------------------------------------- refusals
FAKE = 1 << 20  # an address that nothing reads: every one of these calls is refused before a launch


def c_desc(**kw):
    args = dict(n_layers=2, n_pages=10, n_kv_heads=2, n_q_heads=4, head_dim=128, page_tokens=32, max_pages=4, dtype=torch.bfloat16)
    args.update(kw)
    return B.pages_desc(**args)


TABLES = (dict(P=24), B.IWDFT_ERR_UNSUPPORTED), (dict(n_pages=0), B.IWDFT_ERR_ARG), (dict(max_pages=-1), B.IWDFT_ERR_ARG), (dict(batch=-1), B.IWDFT_ERR_ARG), (
    dict(batch=1025), B.IWDFT_ERR_UNSUPPORTED), (dict(batch=1024, max_pages=1 << 21), B.IWDFT_ERR_ARG), (dict(table=None), B.IWDFT_ERR_ARG), (
    dict(lens=None), B.IWDFT_ERR_ARG), (dict(free=None), B.IWDFT_ERR_ARG), (dict(refs=None), B.IWDFT_ERR_ARG), (dict(lens=FAKE + 2), B.IWDFT_ERR_ARG), (
    dict(refs=FAKE + 1), B.IWDFT_ERR_ARG)


def refused(call, good, changes):
    for change, code in changes:
        assert call(*{**good, **change}.values(), None) == code, change
        assert B.iwdft_last_error()


def test_fork_refuses():
    lib = B.load_library()
    good = dict(P=32, n_pages=10, max_pages=4, parent=FAKE, keep=None, batch=2, table=FAKE, lens=FAKE, free=FAKE, refs=FAKE, ws=None, ws_bytes=0)
    refused(lib.iwdft_pages_fork, good, (*TABLES, (dict(parent=None), B.IWDFT_ERR_ARG), (dict(keep=FAKE + 2), B.IWDFT_ERR_ARG), (dict(max_pages=5000), B.IWDFT_ERR_SIZE),
                                         (dict(max_pages=5000, ws=FAKE, ws_bytes=100), B.IWDFT_ERR_SIZE), (dict(max_pages=5000, ws=FAKE + 4, ws_bytes=1 << 20), B.IWDFT_ERR_ARG)))
    assert lib.iwdft_pages_fork(*{**good, "batch": 0, "table": None}.values(), None) == B.IWDFT_OK
    assert B.iwdft_pages_fork_bytes(8, 1024) == 0 and B.iwdft_pages_fork_bytes(8, 1025) > 4 * 8 * 1025
    n = ctypes.c_size_t()
    for batch, pages in ((-1, 4), (1025, 4), (4, 0), (1024, 1 << 21)):
        assert lib.iwdft_pages_fork_bytes(batch, pages, ctypes.byref(n)) != B.IWDFT_OK
    assert lib.iwdft_pages_fork_bytes(4, 4, None) == B.IWDFT_ERR_ARG


def test_resize_shared_refuses():
    good = dict(P=32, n_pages=10, max_pages=4, want=FAKE, batch=2, table=FAKE, lens=FAKE, free=FAKE, refs=FAKE, starts=FAKE, slots=FAKE, n_slots=4, copies=FAKE)
    refused(B.load_library().iwdft_pages_resize_shared, good,
            (*TABLES, (dict(want=None), B.IWDFT_ERR_ARG), (dict(starts=None), B.IWDFT_ERR_ARG), (dict(slots=None), B.IWDFT_ERR_ARG), (dict(copies=None), B.IWDFT_ERR_ARG),
             (dict(copies=FAKE + 4), B.IWDFT_ERR_ARG), (dict(n_slots=-1), B.IWDFT_ERR_ARG), (dict(n_slots=2 ** 30 + 1), B.IWDFT_ERR_ARG)))


def test_copy_refuses():
    lib = B.load_library()
    good = dict(desc=ctypes.byref(c_desc()), layer=0, n_layers=1, copies=FAKE, n=3, values=FAKE, exponents=FAKE, to_pages=10, to_values=FAKE, to_exponents=FAKE)
    refused(lib.iwdft_pages_copy, good,
            [(c, B.IWDFT_ERR_ARG) for c in (dict(desc=None), dict(layer=-1), dict(layer=2), dict(n_layers=3), dict(n_layers=0), dict(n=-1), dict(n=2 ** 30), dict(copies=None),
                                            dict(values=None), dict(exponents=None), dict(to_values=None), dict(to_exponents=None), dict(to_pages=0), dict(to_pages=1 << 27),
                                            dict(values=FAKE + 8), dict(to_values=FAKE + 4), dict(copies=FAKE + 4), dict(exponents=FAKE + 4), dict(to_exponents=FAKE + 4))])
    assert lib.iwdft_pages_copy(*{**good, "n": 0, "copies": None}.values(), None) == B.IWDFT_OK


def test_compact_refuses():
    lib = B.load_library()
    good = dict(P=32, n_pages=10, max_pages=4, batch=2, table=FAKE, lens=FAKE, free=FAKE, refs=FAKE, moves=FAKE, n_moves=3, ws=FAKE, ws_bytes=1 << 20)
    refused(lib.iwdft_pages_compact, good, (*TABLES, (dict(n_moves=-1), B.IWDFT_ERR_ARG), (dict(moves=None), B.IWDFT_ERR_ARG), (dict(moves=FAKE + 4), B.IWDFT_ERR_ARG),
                                            (dict(ws=None), B.IWDFT_ERR_SIZE), (dict(ws_bytes=20), B.IWDFT_ERR_SIZE), (dict(ws=FAKE + 4), B.IWDFT_ERR_ARG)))
    n = ctypes.c_size_t()
    assert lib.iwdft_pages_compact_bytes(0, ctypes.byref(n)) == B.IWDFT_ERR_ARG and lib.iwdft_pages_compact_bytes(5, None) == B.IWDFT_ERR_ARG
    assert B.iwdft_pages_compact_bytes(1000) >= 4 * 1000


def test_plan_and_attention_refuse():
    lib, n = B.load_library(), ctypes.c_size_t()
    d = c_desc()
    plan, ws = B.iwdft_pages_plan_bytes(d, 1, 2, 3), B.iwdft_pages_attn_shared_bytes(d, 1, 2, 3)
    assert plan > 0 and ws > 0
    both = [(dict(desc=None), B.IWDFT_ERR_ARG), (dict(n_layers=0), B.IWDFT_ERR_ARG), (dict(n_layers=3), B.IWDFT_ERR_ARG), (dict(n=-1), B.IWDFT_ERR_ARG), (dict(n=2 ** 27 + 1), B.IWDFT_ERR_ARG),
            (dict(batch=-1), B.IWDFT_ERR_ARG), (dict(batch=1025), B.IWDFT_ERR_UNSUPPORTED), (dict(table=None), B.IWDFT_ERR_ARG), (dict(table=FAKE + 2), B.IWDFT_ERR_ARG),
            (dict(sink=-1), B.IWDFT_ERR_ARG), (dict(recent=-1), B.IWDFT_ERR_ARG), (dict(sink=4), B.IWDFT_ERR_ARG), (dict(plan=None), B.IWDFT_ERR_SIZE),
            (dict(plan_bytes=plan - 1), B.IWDFT_ERR_SIZE), (dict(plan=FAKE + 64), B.IWDFT_ERR_ARG)]
    good = dict(desc=ctypes.byref(d), n_layers=1, starts=FAKE, n=3, table=FAKE, lens=FAKE, batch=2, sink=0, recent=0, plan=FAKE, plan_bytes=plan)
    refused(lib.iwdft_pages_plan, good, [*both, (dict(starts=None), B.IWDFT_ERR_ARG), (dict(lens=None), B.IWDFT_ERR_ARG)])
    assert lib.iwdft_pages_plan(*{**good, "n": 0, "plan": None}.values(), None) == lib.iwdft_pages_plan(*{**good, "batch": 0}.values(), None) == B.IWDFT_OK
    good = dict(desc=ctypes.byref(d), layer=0, n_layers=1, q=FAKE, n=3, plan=FAKE, plan_bytes=plan, table=FAKE, batch=2, values=FAKE, exponents=FAKE, out=2 * FAKE, sink=0,
                recent=0, scale=0.0, ws=FAKE, ws_bytes=ws)
    refused(lib.iwdft_pages_attn_shared, good,
            [*both, *[(c, B.IWDFT_ERR_ARG) for c in (dict(layer=2), dict(q=None), dict(values=None), dict(exponents=None), dict(out=None), dict(out=FAKE), dict(out=FAKE + 256),
                                                     dict(q=FAKE + 4), dict(out=2 * FAKE + 8), dict(scale=float("nan")), dict(ws=FAKE + 16))],
             (dict(ws=None), B.IWDFT_ERR_SIZE), (dict(ws_bytes=ws - 1), B.IWDFT_ERR_SIZE)])
    assert lib.iwdft_pages_attn_shared(*{**good, "n": 0, "q": None}.values(), None) == lib.iwdft_pages_attn_shared(*{**good, "batch": 0}.values(), None) == B.IWDFT_OK
    for call in (lib.iwdft_pages_plan_bytes, lib.iwdft_pages_attn_shared_bytes):
        assert call(ctypes.byref(d), 1, 2, 3, None) == B.IWDFT_ERR_ARG and call(ctypes.byref(d), 1, 1025, 3, ctypes.byref(n)) == B.IWDFT_ERR_UNSUPPORTED
        assert call(ctypes.byref(d), 1, 0, 3, ctypes.byref(n)) == B.IWDFT_OK and n.value == 0


def test_binding_refuses_tensors_that_do_not_fit():
    z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype)  # noqa: E731
    table, lens, free, refs = z(2, 4), z(2), z(6), z(5)
    for call, args in ((B.iwdft_pages_fork, (z(2), None, table, lens, free, refs, 16)), (B.iwdft_pages_resize_shared, (z(2), table, lens, free, refs, z(3), z(4), z(2, 2), 16)),
                       (B.iwdft_pages_compact, (table, lens, free, refs, z(3, 2), 16)), (B.iwdft_pages_plan, (z(3), table, lens, 4, 5, 1, 1, 16, torch.float32))):
        with pytest.raises(ValueError, match="device"):  # nothing here is on a GPU
            call(*args)
    values, exponents = z(1, 4, 2, 2, 32 * 128, dtype=torch.uint8), z(1, 4, 2, 2)
    with pytest.raises(ValueError, match="device"):
        B.iwdft_pages_copy(z(3, 2), values, exponents)
    with pytest.raises(ValueError, match="refs"):
        B._expect("refs", z(4), torch.int32, (5,), torch.device("cpu"))
    with pytest.raises(ValueError, match="shared"):
        B.PagedCache._shares(type("cache", (), dict(refs=None)))


def test_a_large_calls_plan_and_workspace_serve_no_other_by_size():
    """Bytes grow with each of the sizes."""
    for f in (B.iwdft_pages_plan_bytes, B.iwdft_pages_attn_shared_bytes):
        for dtype in (torch.float32, torch.bfloat16):
            d = c_desc(n_layers=8, n_kv_heads=4, n_q_heads=32, max_pages=300, dtype=dtype)
            for a, b in (((1, 1, 1), (1, 1, 2)), ((1, 4, 9), (1, 5, 9)), ((1, 64, 64), (4, 64, 64)), ((2, 1024, 1024), (2, 1024, 5000))):
                assert 0 < f(d, *a) <= f(d, *b)


@pytest.mark.parametrize("layers,heads,P,pages", [(32, 8, 32, 66_560), (80, 8, 32, 27_000), (64, 32, 128, 2_100), (32, 8, 32, 143_000), (1, 1, 16, (1 << 27) - 1)])
def test_no_list_of_a_caches_own_is_too_long_to_copy(layers, heads, P, pages):
    """Lists that come with tables that have changed already: of a resize (1024 sequences), of a compaction, of all pages; pools of 130 GB and more.  Only the pointers are refused."""
    lib, d = B.load_library(), ctypes.byref(c_desc(n_layers=layers, n_pages=pages, n_kv_heads=heads, n_q_heads=heads, page_tokens=P))
    for n in (1024, pages // 2, pages):
        assert lib.iwdft_pages_copy(d, 0, layers, None, n, None, None, pages, None, None, None) == B.IWDFT_ERR_ARG
        assert "NULL" in B.iwdft_last_error(), (n, B.iwdft_last_error())


def test_compact_copies_no_more_than_can_move(monkeypatch):
    """A list longer than half of the pool, of which the rest is never anything."""
    lengths = []
    monkeypatch.setattr(B, "iwdft_pages_compact", lambda table, lens, free, refs, moves, *a: lengths.append(len(moves)))
    monkeypatch.setattr(B, "iwdft_pages_copy", lambda moves, *a, **kw: lengths.append(len(moves)))
    cache = type("cache", (), dict(refs=torch.zeros(9), table=None, lens=None, free=None, page_tokens=16, device=torch.device("cpu"), values=torch.zeros(1, 9), exponents=None,
                                   _shares=lambda self: None))()
    assert [len(B.PagedCache.compact(cache, n)) for n in (None, 3, 50)] == [4, 3, 50] and lengths == [4, 4, 3, 3, 50, 4]
