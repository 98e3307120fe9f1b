"""The block-cache calls without a GPU: every refusal (arguments are checked
before the context), and where rows of well-formed and malformed windows lie
(the kernels' own lookup, run on host memory)."""
import ctypes

import numpy as np
import pytest

from tests.block_util import REQ, Window

A = 1 << 20  # an aligned address that no call here reads


@pytest.fixture(scope="module")
def lib():
    import paper_2609_33224_amd as ps
    return ps.load_library()


def _cache(**kw):
    from paper_2609_33224_amd.binding import PsKvCache
    d = dict(k=A, v=A, k_exp=A, v_exp=A, n_pages=10, page_stride=2 * 16 * 64, exp_page_stride=32, n_kv_heads=2,
             head_dim=64, block_tokens=16, dtype=2)
    d.update(kw)
    return PsKvCache(**d)


def _window(**kw):
    from paper_2609_33224_amd.binding import PsKvWindow
    d = dict(pages=A, reqs=A, ctx_tok=A, row_off=A, pages_len=10, n_pages=10, n_req=2, n_rows=4)
    d.update(kw)
    return PsKvWindow(**d)


def _rows(**kw):
    from paper_2609_33224_amd.binding import PsRows
    d = dict(data=A, row_stride=128, head_stride=64, dtype=0)
    d.update(kw)
    return PsRows(**d)


def _ref(x):
    return ctypes.byref(x) if x is not None else None


def _err(lib):
    return lib.ps_last_error(None).decode()


BAD_CACHE = [
    (dict(k=None), -1, "NULL"), (dict(v=None), -1, "NULL"), (dict(k=A + 8), -1, "aligned"),
    (dict(v=A + 4), -1, "aligned"), (dict(k_exp=None), -1, "exponent"), (dict(v_exp=None), -1, "exponent"),
    (dict(n_pages=-1), -5, "n_pages"), (dict(n_pages=1 << 31), -5, "n_pages"),
    (dict(page_stride=2 * 16 * 64 - 16), -1, "page_stride"), (dict(page_stride=2 * 16 * 64 + 8), -1, "page_stride"),
    (dict(exp_page_stride=31), -1, "exp_page_stride"), (dict(n_kv_heads=0), -5, "n_kv_heads"),
    (dict(n_kv_heads=129), -5, "n_kv_heads"), (dict(head_dim=72), -5, "head_dim"), (dict(head_dim=0), -5, "head_dim"),
    (dict(head_dim=272), -5, "head_dim"), (dict(block_tokens=0), -5, "block_tokens"),
    (dict(block_tokens=1025), -5, "block_tokens"), (dict(dtype=3), -1, "type"), (dict(dtype=-1), -1, "type"),
]
BAD_WINDOW = [
    (dict(pages=None), -1, "NULL"), (dict(reqs=None), -1, "NULL"), (dict(ctx_tok=None), -1, "NULL"),
    (dict(row_off=None), -1, "NULL"), (dict(n_req=-1), -1, "negative"), (dict(pages_len=-1), -1, "negative"),
    (dict(n_rows=-1), -5, "n_rows"), (dict(n_rows=(1 << 20) + 1), -5, "n_rows"), (dict(n_pages=-1), -5, "n_pages"),
]
BAD_ROWS = [
    (dict(data=None), -1, "NULL"), (dict(data=A + 2), -1, "aligned"), (dict(row_stride=129), -1, "strides"),
    (dict(head_stride=60), -1, "strides"), (dict(row_stride=-128), -1, "strides"), (dict(dtype=2), -1, "16-bit"),
]


@pytest.mark.parametrize("call", ["ps_kv_write_dev", "ps_kv_read_dev"])
def test_cache_calls_refuse(lib, call):
    f = getattr(lib, call)

    def go(cache=_cache(), window=_window(), k=_rows(), v=_rows()):
        return f(None, _ref(cache), _ref(window), _ref(k), _ref(v), None)

    assert go() == -1 and "ctx is NULL" in _err(lib)
    assert go(cache=None) == -1 and "cache is NULL" in _err(lib)
    assert go(window=None) == -1 and "window is NULL" in _err(lib)
    assert go(k=None) == -1 and "k is NULL" in _err(lib)
    for kw, code, text in BAD_CACHE:
        assert go(cache=_cache(**kw)) == code and text in _err(lib), (kw, _err(lib))
    for kw, code, text in BAD_WINDOW:
        assert go(window=_window(**kw)) == code and text in _err(lib), (kw, _err(lib))
    for kw, code, text in BAD_ROWS:
        assert go(k=_rows(**kw)) == code and text in _err(lib), (kw, _err(lib))
        assert go(v=_rows(**kw)) == code and text in _err(lib), (kw, _err(lib))
    assert go(window=_window(n_pages=11)) == -1 and "more pages" in _err(lib)
    assert go(v=_rows(dtype=1)) == -1 and "differ in type" in _err(lib)
    assert go(cache=_cache(dtype=1, k_exp=None, v_exp=None)) == -1 and "differ in type" in _err(lib)
    # rows that are written may not lie on each other; rows that are read may
    for kw in (dict(row_stride=0), dict(head_stride=0)):
        assert go(k=_rows(**kw)) == -1
        assert ("overlap" if call == "ps_kv_read_dev" else "ctx is NULL") in _err(lib)
    # a window without requests or rows is checked no further
    for kw in (dict(n_req=0, reqs=None, ctx_tok=None, row_off=None, pages=None), dict(n_rows=0)):
        assert go(window=_window(**kw), k=None, v=None) == -1 and "ctx is NULL" in _err(lib)


def test_plan_calls_refuse(lib):
    out = ctypes.c_void_p()

    def create(heads=8, kv=2, dim=64, bt=16, req=4, rows=4, to=ctypes.byref(out)):
        return lib.ps_attend_plan_create(None, heads, kv, dim, bt, req, rows, to)

    assert create() == -1 and "ctx is NULL" in _err(lib)
    assert create(to=None) == -1 and "out is NULL" in _err(lib)
    for kw, text in ((dict(heads=7), "n_heads"), (dict(heads=0), "n_heads"), (dict(heads=1026), "n_heads"),
                     (dict(kv=0), "n_kv_heads"), (dict(kv=130, heads=260), "n_kv_heads"), (dict(dim=24), "head_dim"),
                     (dict(dim=512), "head_dim"), (dict(bt=0), "block_tokens"), (dict(bt=2000), "block_tokens"),
                     (dict(req=-1), "max_req"), (dict(req=8193), "max_req"), (dict(rows=-1), "max_rows"),
                     (dict(rows=(1 << 20) + 1), "max_rows")):
        assert create(**kw) == -5 and text in _err(lib), kw
    assert lib.ps_attend_plan_destroy(None) == 0
    assert lib.ps_attend_plan_dev(None, _ref(_window()), None, None) == -1 and "plan is NULL" in _err(lib)
    assert lib.ps_attend_plan_dev(None, None, None, None) == -1 and "window is NULL" in _err(lib)
    for kw, code, text in BAD_WINDOW:
        assert lib.ps_attend_plan_dev(None, _ref(_window(**kw)), None, None) == code and text in _err(lib)


def test_attention_refuses(lib):
    def go(cache=_cache(), q=_rows(), out=_rows(), scale=1.0):
        return lib.ps_attend_window_dev(None, _ref(cache), _ref(q), _ref(out), None, scale, None)

    assert go() == -1 and "plan is NULL" in _err(lib)
    for kw, code, text in BAD_CACHE:
        assert go(cache=_cache(**kw)) == code and text in _err(lib), kw
    for kw, code, text in BAD_ROWS:
        assert go(q=_rows(**kw)) == code and text in _err(lib), kw
        assert go(out=_rows(**kw)) == code and text in _err(lib), kw
    assert go(out=_rows(row_stride=0)) == -1 and "overlap" in _err(lib)
    assert go(out=_rows(dtype=1)) == -1 and "differ in type" in _err(lib)
    assert go(cache=_cache(dtype=1, k_exp=None, v_exp=None)) == -1 and "differ in type" in _err(lib)
    for s in (float("inf"), float("nan")):
        assert go(scale=s) == -1 and "scale" in _err(lib)


def _locate(lib, w, row, **kw):
    f = lib.ps_test_block_locate
    f.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
    f.restype = ctypes.c_int32
    keep = [np.ascontiguousarray(a) for a in (w.pages, w.reqs, w.ctx, w.row_off)]
    win = _window(**{**dict(pages=keep[0].ctypes.data, reqs=keep[1].ctypes.data, ctx_tok=keep[2].ctypes.data,
                            row_off=keep[3].ctypes.data, pages_len=len(w.pages), n_pages=w.n_pages, n_req=w.n_req,
                            n_rows=w.n_rows), **kw})
    page, slot = ctypes.c_int64(-7), ctypes.c_int32(-7)
    got = f(ctypes.byref(win), w.bt, row, ctypes.byref(page), ctypes.byref(slot))
    return (got, page.value, slot.value) if got == 2 else (got,)


@pytest.mark.parametrize("bt", [1, 5, 16, 64])
@pytest.mark.parametrize("pad", [0, 3])
def test_rows_lie_where_the_chain_says(lib, bt, pad):
    w = Window([0, 3, 1], [(0, 1, 1), (1, 3 * bt + 2, 2), (2, 0, 0), (2, 4, 7), (1, 2 * bt, 1), (0, 0, 2), (0, 9, 9)],
               bt, seed=bt, spare=1, pad=pad)
    seen = set()
    for r in range(w.n_req):
        ch = w.chain(r)
        for row, pos in w.rows(r):
            seen.add(row)
            assert _locate(lib, w, row) == ((2, ch[pos // bt], pos % bt) if pos >= 0 else (1,)), (r, row)
    for row in set(range(w.n_rows)) - seen:
        assert _locate(lib, w, row) == (0,)


def test_malformed_windows_have_no_place(lib):
    base = lambda: Window([2], [(0, 40, 2), (0, 37, 3)], 16)  # noqa: E731
    edits = [("pre_off", -1), ("pre_off", 1 << 62), ("pre_off", -(1 << 63)), ("tail_off", 5), ("pre_len", -1),
             ("pre_len", 1 << 30), ("tail_len", (1 << 31) - 1), ("tail_len", 0), ("tail_len", -3),
             ("tail_off", (1 << 63) - 1)]
    for field, v in edits:
        w = base()
        w.reqs[1][field] = v
        assert [_locate(lib, w, i)[0] for i in range(5)] == [2, 2, 1, 1, 1], (field, v)
    for ctx in (-1, 49, (1 << 31) - 1, -(1 << 31)):
        w = base()
        w.ctx[1] = ctx
        assert [_locate(lib, w, i)[0] for i in range(5)] == [2, 2, 1, 1, 1], ctx
    for page in (-1, 1 << 30, -(1 << 31)):
        w = base()
        w.pages[w.reqs[1]["tail_off"]] = page
        assert [_locate(lib, w, i)[0] for i in range(5)] == [2, 2, 1, 1, 1], page
    # a window that names fewer pages than it uses
    w = base()
    assert all(_locate(lib, w, i, n_pages=0)[0] == 1 for i in range(5))
    # whatever row_off holds, a row found lies inside its request's range and its chain
    rng = np.random.default_rng(0)
    for _ in range(300):
        w = base()
        w.row_off = rng.choice([-(1 << 31), -1, 0, 1, 2, 3, 5, 9, (1 << 31) - 1], 3).astype(np.int32)
        for row in range(5):
            got = _locate(lib, w, row)
            if got[0] == 2:
                assert got[1] in w.pages and 0 <= got[2] < 16


def test_quantiser_of_the_tests():
    """The 64-bit quantiser that the GPU tests compare with, on values that can be read off."""
    from tests.block_util import quantise
    x = np.array([[448.0, 1.0625, 1.1875, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, -3.3, np.inf],
                  [449.0, 0, 0, 0, 0, 0, np.nan, -np.inf], [0] * 8])
    y, e = quantise(x)
    assert list(e) == [127, 128, 1]
    assert list(y[0]) == [448, 1.0, 1.25, 2.0 ** -9, 0, 2.0 ** -8, -3.25, 448]
    assert y[1][0] == 224 and np.isnan(y[1][6]) and y[1][7] == -448
    assert REQ.itemsize == 24


def test_scales_that_overflow_are_refused(lib):
    q, cache = _rows(), _cache()

    def go(scale):
        return lib.ps_attend_window_dev(None, _ref(cache), _ref(q), _ref(q), None, scale, None)

    for s in (3.0e38, -2.4e38):
        assert go(s) == -1 and "scale" in _err(lib)
    for s in (2.3e38, -2.3e38, 0.0, 1e-45):
        assert go(s) == -1 and "plan is NULL" in _err(lib)


def test_rows_that_would_be_written_over_each_other(lib):
    """Against every pair of rows and heads; and the read call refuses what the check finds."""
    f = lib.ps_test_rows_overlap
    f.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32]
    f.restype = ctypes.c_int32
    rng = np.random.default_rng(0)
    found = [0, 0]
    for _ in range(4000):
        n, heads, dim = int(rng.integers(1, 7)), int(rng.integers(1, 6)), 16 * int(rng.integers(1, 4))
        rs, hs = (8 * int(x) for x in rng.integers(0, 40, 2))
        at = np.sort((np.arange(n)[:, None] * rs + np.arange(heads)[None] * hs).reshape(-1))
        want = bool((np.diff(at) < dim).any())
        assert bool(f(ctypes.byref(_rows(row_stride=rs, head_stride=hs)), n, heads, dim)) == want, (n, heads, dim, rs, hs)
        found[want] += 1
    assert min(found) > 500
    # (1 << 20) rows of 128 heads
    big = lambda rs, hs, n=1 << 20, h=128: f(ctypes.byref(_rows(row_stride=rs, head_stride=hs)), n, h, 128)  # noqa: E731
    assert not big(128 * 128, 128) and not big(128, 128 << 20) and big(128 * 127, 128) and big(128, (128 << 20) - 8)

    def read(**kw):
        k = _rows(**kw)
        code = lib.ps_kv_read_dev(None, _ref(_cache()), _ref(_window(n_rows=4)), _ref(k), _ref(_rows()), None)
        return code, _err(lib)

    assert read(row_stride=64, head_stride=64)[0] == -1 and "overlap" in read(row_stride=64, head_stride=64)[1]
    for kw in (dict(row_stride=128, head_stride=64), dict(row_stride=64, head_stride=256),
               dict(row_stride=64 * 3, head_stride=64 * 2)):
        assert "ctx is NULL" in read(**kw)[1], kw
