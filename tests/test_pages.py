"""The 8-bit paged cache without a GPU: the oracle's own pins, and what the library and the binding refuse before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pages_oracle as po
from paper_2507_20030_amd import binding as B


# ------------------------------------------------------------------------------------------------------------------ oracle
def test_e4m3_of_the_oracle_is_torchs():
    x = np.concatenate([po.TABLE[:127], (po.TABLE[:126] + po.TABLE[1:127]) / 2, np.random.default_rng(0).normal(size=4000) * 20,
                        np.random.default_rng(1).normal(size=4000) * 2.0 ** -8])
    x = np.concatenate([x, -x]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(po.to_e4m3(x), want)
    assert list(po.to_e4m3(np.array([1e9, -np.inf, np.nan]))) == [126, 254, 127]
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(np.nan_to_num(po.TABLE, nan=-1.0), np.nan_to_num(every, nan=-1.0))


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.0001, 1), (449.0, 1), (224.0, -1), (1.75, -8), (1.76, -7), (0.0, -100), (2.0 ** -140, -100), (3.4e38, 120)])
def test_exponent_of_the_oracle(top, e):
    assert po.exponent(np.array([0.5 * top, -top, np.nan, np.inf])) == e


def test_resize_of_the_oracle_by_hand():
    table, lens = np.full((3, 4), -1, np.int32), np.zeros(3, np.int32)
    free = np.array([8, 0, 1, 2, 3, 4, 5, 6, 7], np.int32)
    starts, slots = po.resize([17, 0, 33], table, lens, free, 60, 16)
    assert list(table[0]) == [7, 6, -1, -1] and list(table[2]) == [5, 4, 3, -1] and free[0] == 3
    assert list(starts) == [0, 17, 17, 50] and slots[0] == 112 and slots[16] == 96 and slots[17] == 80 and slots[49] == 48 and set(slots[50:]) == {-1}
    before = free.copy(), table.copy()
    po.resize([17, 20, 48], table, lens, free, 60, 16)                   # two more pages
    assert list(lens) == [17, 20, 48] and list(table[1]) == [2, 1, -1, -1] and free[0] == 1
    po.resize([17, 0, 33], table, lens, free, 0, 16)                     # and back
    assert np.array_equal(free, before[0]) and np.array_equal(table[[0, 2]], before[1][[0, 2]])
    starts, slots = po.resize([0, 65, 49], table, lens, free, 60, 16)    # too long for the table; a page from those given back
    assert list(lens) == [0, 0, 49] and list(starts) == [0, 0, 0, 16] and free[0] == 4 and table[2, 3] == 7
    assert list(free[1:5]) == [0, 1, 2, 6]


# ---------------------------------------------------------------------------------------------------------------- refusals
def c_desc(**kw):
    args = dict(n_layers=2, n_pages=10, n_kv_heads=2, n_q_heads=4, head_dim=128, page_tokens=32, max_pages=4, dtype=torch.bfloat16)
    args.update(kw)
    return B.pages_desc(**args)


@pytest.mark.parametrize("kw,code", [
    (dict(n_layers=0), B.IWDFT_ERR_ARG), (dict(n_pages=0), B.IWDFT_ERR_ARG), (dict(n_kv_heads=0), B.IWDFT_ERR_ARG), (dict(n_q_heads=3), B.IWDFT_ERR_ARG),
    (dict(n_q_heads=0), B.IWDFT_ERR_ARG), (dict(max_pages=0), B.IWDFT_ERR_ARG), (dict(n_pages=1 << 26), B.IWDFT_ERR_ARG),
    (dict(max_pages=(1 << 25) + 1), B.IWDFT_ERR_ARG), (dict(head_dim=64), B.IWDFT_ERR_UNSUPPORTED), (dict(page_tokens=8), B.IWDFT_ERR_UNSUPPORTED),
    (dict(page_tokens=48), B.IWDFT_ERR_UNSUPPORTED), (dict(page_tokens=0), B.IWDFT_ERR_UNSUPPORTED),
])
def test_bad_page_descriptors_are_refused(kw, code):
    with pytest.raises(B.IwdftError) as e:
        B.iwdft_pages_query_bytes(c_desc(**kw))
    assert e.value.code == code and B.iwdft_last_error()


def test_page_bytes():
    assert B.iwdft_pages_query_bytes(c_desc()) == (2 * 10 * 2 * 2 * 32 * 128, 2 * 10 * 2 * 2 * 4)
    lib, n = B.load_library(), ctypes.c_size_t()
    assert lib.iwdft_pages_query_bytes(None, ctypes.byref(n), ctypes.byref(n)) == B.IWDFT_ERR_ARG
    assert lib.iwdft_pages_query_bytes(ctypes.byref(c_desc()), None, ctypes.byref(n)) == B.IWDFT_ERR_ARG
    d = c_desc()
    d = B.iwdft_pages_desc(*[getattr(d, f) for f, _ in d._fields_])
    d.kv_dtype = 5
    assert lib.iwdft_pages_query_bytes(ctypes.byref(d), ctypes.byref(n), ctypes.byref(n)) == B.IWDFT_ERR_ARG


def test_resize_workspace_by_rule():
    assert B.iwdft_pages_resize_bytes(1024, 2048) == 0
    assert B.iwdft_pages_resize_bytes(1025, 1) == 4 * (4 + 3 * 1025) and B.iwdft_pages_resize_bytes(0, 2049) == 16
    for batch, slots in ((-1, 0), (0, -1)):
        with pytest.raises(B.IwdftError):
            B.iwdft_pages_resize_bytes(batch, slots)


def test_attention_workspace_by_rule():
    """None where no sequence can be longer than a part of it is at least."""
    assert B.iwdft_pages_attn_bytes(c_desc(page_tokens=16, max_pages=6), 1, 3, 3) == 0
    assert B.iwdft_pages_attn_bytes(c_desc(max_pages=4096), 1, 3, 3) > 0
    assert B.iwdft_pages_attn_bytes(c_desc(max_pages=4096), 1, 0, 3) == B.iwdft_pages_attn_bytes(c_desc(max_pages=4096), 1, 3, 0) == 0
    for kw in (dict(batch=-1), dict(n_tokens=-1), dict(n_layers=3), dict(n_layers=0)):
        with pytest.raises(B.IwdftError) as e:
            B.iwdft_pages_attn_bytes(**{**dict(desc=c_desc(), n_layers=1, batch=1, n_tokens=1), **kw})
        assert e.value.code == B.IWDFT_ERR_ARG


FAKE = 1 << 20  # an address that nothing reads: every one of these calls is refused before a launch


def test_resize_refuses():
    lib = B.load_library()
    good = dict(P=32, n_pages=10, max_pages=4, want=FAKE, batch=2, table=FAKE, lens=FAKE, free=FAKE, starts=FAKE, slots=FAKE, n_slots=4, ws=None, ws_bytes=0)
    for change, code in ((dict(P=24), B.IWDFT_ERR_UNSUPPORTED), (dict(n_pages=0), B.IWDFT_ERR_ARG), (dict(max_pages=-1), B.IWDFT_ERR_ARG),
                         (dict(batch=-1), B.IWDFT_ERR_ARG), (dict(n_slots=-1), B.IWDFT_ERR_ARG), (dict(want=None), B.IWDFT_ERR_ARG),
                         (dict(table=None), B.IWDFT_ERR_ARG), (dict(lens=None), B.IWDFT_ERR_ARG), (dict(free=None), B.IWDFT_ERR_ARG),
                         (dict(starts=None), B.IWDFT_ERR_ARG), (dict(slots=None), B.IWDFT_ERR_ARG), (dict(lens=FAKE + 2), B.IWDFT_ERR_ARG),
                         (dict(n_slots=5000), B.IWDFT_ERR_SIZE), (dict(n_slots=5000, ws=FAKE, ws_bytes=20), B.IWDFT_ERR_SIZE)):
        assert lib.iwdft_pages_resize(*{**good, **change}.values(), None) == code, change


def test_write_refuses():
    lib = B.load_library()
    good = dict(desc=ctypes.byref(c_desc()), layer=0, n_layers=1, k=FAKE, v=FAKE, slots=FAKE, n=3, values=FAKE, exponents=FAKE)
    for change in (dict(desc=None), dict(layer=-1), dict(layer=2), dict(n_layers=3), dict(n_layers=0), dict(layer=1, n_layers=2), dict(layer=2 ** 31 - 1), dict(n=-1), dict(n=2 ** 30 + 1),
                   dict(k=None), dict(v=None), dict(slots=None), dict(values=None), dict(exponents=None), dict(k=FAKE + 8), dict(values=FAKE + 4),
                   dict(exponents=FAKE + 4), dict(slots=FAKE + 1)):
        assert lib.iwdft_pages_write(*{**good, **change}.values(), None) == B.IWDFT_ERR_ARG, change
    assert lib.iwdft_pages_write(*{**good, "n": 0, "k": None}.values(), None) == B.IWDFT_OK


def test_attention_refuses():
    lib = B.load_library()
    good = dict(desc=ctypes.byref(c_desc()), layer=0, n_layers=1, q=FAKE, starts=FAKE, n=3, table=FAKE, lens=FAKE, batch=2, values=FAKE, exponents=FAKE,
                out=2 * FAKE, sink=0, recent=0, scale=0.0, ws=None, ws_bytes=0)
    for change in (dict(desc=None), dict(layer=2), dict(n_layers=0), dict(n=-1), dict(n=2 ** 30), dict(batch=-2), dict(q=None), dict(starts=None), dict(table=None),
                   dict(lens=None), dict(values=None), dict(exponents=None), dict(out=None), dict(out=FAKE), dict(out=FAKE + 256), dict(q=FAKE + 4),
                   dict(out=2 * FAKE + 8), dict(sink=-1), dict(recent=-1), dict(sink=4), dict(scale=float("nan"))):
        got = lib.iwdft_pages_attn(*{**good, **change}.values(), None)
        assert got == B.IWDFT_ERR_ARG, change
    long = ctypes.byref(c_desc(max_pages=4096))
    assert lib.iwdft_pages_attn(*{**good, "desc": long}.values(), None) == B.IWDFT_ERR_SIZE
    assert lib.iwdft_pages_attn(*{**good, "desc": long, "ws": FAKE, "ws_bytes": 1000}.values(), None) == B.IWDFT_ERR_SIZE
    assert lib.iwdft_pages_attn(*{**good, "desc": long, "ws": FAKE + 16, "ws_bytes": 1 << 30}.values(), None) == B.IWDFT_ERR_ARG
    assert lib.iwdft_pages_attn(*{**good, "n": 0}.values(), None) == lib.iwdft_pages_attn(*{**good, "batch": 0}.values(), None) == B.IWDFT_OK


def test_read_refuses():
    lib = B.load_library()
    good = dict(desc=ctypes.byref(c_desc()), layer=0, n_layers=1, table=FAKE, lens=FAKE, batch=2, n=3, values=FAKE, exponents=FAKE, K=FAKE, V=FAKE)
    for change in (dict(desc=None), dict(layer=-1), dict(n_layers=5), dict(batch=-1), dict(n=-1), dict(n=2 ** 30), dict(table=None), dict(lens=None), dict(values=None),
                   dict(exponents=None), dict(K=FAKE + 4), dict(V=FAKE + 2)):
        assert lib.iwdft_pages_read(*{**good, **change}.values(), None) == B.IWDFT_ERR_ARG, change
    for change in (dict(n=0), dict(batch=0), dict(K=None, V=None)):
        assert lib.iwdft_pages_read(*{**good, **change}.values(), None) == B.IWDFT_OK


def test_binding_refuses_tensors_that_do_not_fit():
    z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype)  # noqa: E731
    values, exponents = z(1, 4, 2, 2, 32 * 128, dtype=torch.uint8), z(1, 4, 2, 2)
    with pytest.raises(ValueError, match="device"):  # nothing here is on a GPU
        B.iwdft_pages_write(values, exponents, z(1, 3, 2, 128, dtype=torch.float32), z(1, 3, 2, 128, dtype=torch.float32), z(3))
    with pytest.raises(ValueError, match="device"):
        B.iwdft_pages_resize(z(2), z(2, 4), z(2), z(5), z(3), z(2), 32)
    with pytest.raises(ValueError, match="shape"):
        B.iwdft_pages_read(values[0], exponents, z(1, 4), z(1), z(1, 1, 2, 5, 128, dtype=torch.float32), None)
    dev = torch.device("cpu")
    for bad in (z(3), z(2, 2), z(2, dtype=torch.int64), z(4)[::2]):
        with pytest.raises(ValueError):
            B._expect("x", bad, torch.int32, (2,), dev)
    with pytest.raises(ValueError):
        B._expect("x", z(2), torch.int32, (2,), torch.device("meta"))
    with pytest.raises(ValueError):
        B._kv_dtype("q", z(2, dtype=torch.float16))
    with pytest.raises(ValueError):
        B.PagedCache(1, 4, 2, 2, 128, torch.float16, 1, 64)
    with pytest.raises(B.IwdftError):
        B.PagedCache(1, 4, 2, 3, 128, torch.float32, 1, 64)


def test_sizes_whose_counts_would_not_fit():
    """Products of sizes that pass 64 bits, launches of 2^32 threads and more, counts that pass 32 bits."""
    lib, n = B.load_library(), ctypes.c_size_t()
    huge = dict(n_layers=2 ** 31 - 1, n_pages=2 ** 24, n_kv_heads=2 ** 30, n_q_heads=2 ** 30, page_tokens=64)
    with pytest.raises(B.IwdftError) as e:
        B.iwdft_pages_query_bytes(c_desc(**huge))
    assert e.value.code == B.IWDFT_ERR_ARG
    wide = ctypes.byref(c_desc(n_layers=2 ** 20, n_kv_heads=2 ** 14, n_q_heads=2 ** 30, page_tokens=16, n_pages=1))
    for call, args in ((lib.iwdft_pages_attn_bytes, (wide, 2 ** 20, 1, 2 ** 30, ctypes.byref(n))), (lib.iwdft_pages_attn_bytes, (wide, 1, 2 ** 30 + 1, 1, ctypes.byref(n))),
                       (lib.iwdft_pages_resize_bytes, (2 ** 30 + 1, 1, ctypes.byref(n))), (lib.iwdft_pages_resize_bytes, (1, 2 ** 30 + 1, ctypes.byref(n))),
                       (lib.iwdft_pages_write, (wide, 0, 2 ** 20, FAKE, FAKE, FAKE, 2 ** 30, FAKE, FAKE, None)),
                       (lib.iwdft_pages_write, (wide, 0, 2 ** 12, FAKE, FAKE, FAKE, 1, FAKE, FAKE, None)),                       # 2^27 waves
                       (lib.iwdft_pages_write, (ctypes.byref(c_desc(page_tokens=16)), 0, 1, FAKE, FAKE, FAKE, 2 ** 29, FAKE, FAKE, None)),
                       (lib.iwdft_pages_read, (wide, 0, 2 ** 20, FAKE, FAKE, 2 ** 30, 2 ** 30, FAKE, FAKE, FAKE, FAKE, None)),
                       (lib.iwdft_pages_read, (ctypes.byref(c_desc()), 0, 2, FAKE, FAKE, 2 ** 25, 1, FAKE, FAKE, FAKE, FAKE, None))):  # 2^27 waves of one token
        assert call(*args) == B.IWDFT_ERR_ARG, args


def test_descriptors_are_the_callers_own():
    """Changing the one that was handed out changes neither the next one nor what the calls take for the same sizes."""
    sizes = dict(n_layers=1, n_pages=700, n_kv_heads=2, n_q_heads=4, head_dim=128, page_tokens=16, max_pages=512, dtype=torch.float32)
    d = B.pages_desc(**sizes)
    d.max_pages = 3
    assert B.pages_desc(**sizes).max_pages == 512
    ref = B._pages_ref(*sizes.values())
    assert ref._obj.max_pages == 512 and B._attn_sizes(1, 1, 1, *sizes.values())[0]._obj.max_pages == 512
    B.pages_desc(**sizes).kv_dtype = B.IWDFT_BF16
    assert B._pages_ref(*sizes.values())._obj.kv_dtype == B.IWDFT_F32


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.uint8])
def test_descriptors_of_other_types_are_refused(dtype):
    with pytest.raises(ValueError):
        B.pages_desc(1, 4, 2, dtype=dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 16, 17, 33, 40, 64, 71])
def test_attention_workspace_serves_smaller_calls(G, dtype):
    """What is asked for the largest call never falls with its sizes and is enough for every smaller one: these get past the check of the workspace to the one
    of its alignment."""
    d = c_desc(n_kv_heads=8, n_q_heads=8 * G, max_pages=512, dtype=dtype)
    lib, ref = B.load_library(), ctypes.byref(d)
    tokens, batches = (1, 2, 3, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 128, 129, 1000, 4096), (1, 2, 3, 4, 8, 16, 32, 33, 64, 256)
    need = {(n, b): B.iwdft_pages_attn_bytes(d, 1, b, n) for n in tokens for b in batches}
    for i, n in enumerate(tokens):
        for j, b in enumerate(batches):
            assert need[n, b] >= max(need[tokens[max(i - 1, 0)], b], need[n, batches[max(j - 1, 0)]])
            for limit in (need[n, b], need[tokens[-1], batches[-1]]):
                assert lib.iwdft_pages_attn(ref, 0, 1, FAKE, FAKE, n, FAKE, FAKE, b, FAKE, FAKE, 1 << 36, 0, 0, 0.0, FAKE + 16, limit, None) == B.IWDFT_ERR_ARG
                assert "256-byte" in B.iwdft_last_error()
