"""The block cache on the GPU: rows written, quantised and read back, and the
attention of windows over it, against the same written out in 64 bits
(tests/block_util.py); needs an MI355X."""
import numpy as np
import pytest
import torch

from tests.block_util import Window, check_attention, quantise

pytestmark = pytest.mark.gpu

BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ps():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_33224_amd as ps
    return ps


@pytest.fixture(scope="module")
def sc(ps):
    s = ps.Scorer(0)
    yield s
    s.close()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _cache(ps, w, heads, dim, dtype, seed=0, fill=True):
    c = ps.KvCache.empty(w.n_pages, heads, w.bt, dim, dtype)
    if fill:
        g = _gen(seed)
        for t, x in zip(c.tensors[:2], c.tensors[2:]):
            v = _randn(g, *t.shape)
            if dtype == E4M3:
                t.view(torch.uint8).copy_((v * 60).to(E4M3).view(torch.uint8))
                x.copy_(torch.randint(119, 123, x.shape, generator=g, device="cuda"))
            else:
                t.copy_(v)
    return c


# sessions (blocks of their prefix) and requests (session, context, rows): single tokens,
# chunks, contexts of 0 and 1, more rows than tokens, contexts inside the shared prefix
def _mixed(bt):
    return [0, 4, 2, 7], [(0, 1, 1), (1, 4 * bt + 3, 1), (1, 4 * bt + 2 * bt, 2), (0, 0, 1), (2, 2 * bt + 1, 1),
                          (1, 5 * bt, 1), (3, 7 * bt + 9, 9), (2, 2 * bt + 33, 4), (0, 3, 6), (1, bt + 1, 1),
                          (3, 7 * bt + 1, 1), (2, 2 * bt, 1), (0, 70, 70), (0, 5, 0)]


# ------------------------------------------------------------------ rows
@pytest.mark.parametrize("heads,dim,bt", [(1, 16, 1), (2, 64, 16), (3, 96, 5), (8, 128, 16), (1, 256, 64), (5, 208, 7)])
@pytest.mark.parametrize("dtype,typ", [(BF16, BF16), (F16, F16), (E4M3, BF16), (E4M3, F16)])
def test_write_and_read(ps, sc, heads, dim, bt, dtype, typ):
    w = Window(*_mixed(bt), bt, seed=dim, pad=2)
    win = w.dev()
    # every request writes its own tail; rows in a prefix several share hold the same values
    g = _gen(heads)
    token = _randn(g, w.n_pages, bt, 2, heads, dim) * torch.exp2(8 * _randn(g, w.n_pages, bt, 2, 1, 1))
    k, v = (torch.zeros(w.n_rows, heads, dim, dtype=typ, device="cuda") for _ in range(2))
    for r in range(w.n_req):
        ch = w.chain(r)
        for row, pos in w.rows(r):
            if pos >= 0:
                k[row], v[row] = token[int(ch[pos // bt]), pos % bt].to(typ)
    c = _cache(ps, w, heads, dim, dtype, fill=True)
    before = [t.clone() if t is not None else None for t in c.tensors]
    sc.kv_write_dev(c, win, k, v)
    want = [t.clone() if t is not None else None for t in before]
    for r in range(w.n_req):
        ch = w.chain(r)
        for row, pos in w.rows(r):
            if pos < 0:
                continue
            at = (int(ch[pos // bt]), slice(None), pos % bt)
            for n, x in enumerate((k, v)):
                if dtype == E4M3:
                    code, e = quantise(x[row].double().cpu().numpy())
                    want[n].view(torch.uint8)[at] = torch.from_numpy(code).to(E4M3).view(torch.uint8).cuda()
                    want[2 + n][at] = torch.from_numpy(e).cuda()
                else:
                    want[n][at] = x[row]
    for got, ref in zip(c.tensors, want):  # untouched slots too, bit for bit (but for -0)
        if ref is not None:
            assert torch.equal(got.float(), ref.float())
    ok, ov = (torch.full_like(k, 7.0) for _ in range(2))
    sc.kv_read_dev(c, win, ok, ov)
    for n, got in enumerate((ok, ov)):
        ref = torch.full_like(got, 7.0)
        for r in range(w.n_req):
            ch = w.chain(r)
            for row, pos in w.rows(r):
                ref[row] = 0
                if pos >= 0:
                    at = (int(ch[pos // bt]), slice(None), pos % bt)
                    x = want[n][at].double()
                    if dtype == E4M3:
                        x = x * torch.exp2(want[2 + n][at].double() - 127)[:, None]
                    ref[row] = x.to(typ)
        assert torch.equal(got, ref)


@pytest.mark.parametrize("typ", [BF16, F16])
def test_every_16_bit_value_quantises_to_the_nearest(ps, sc, typ):
    """All 65,536 patterns, under row maxima that put them anywhere on the e4m3 grid."""
    dim, bt = 256, 16
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(typ).cuda()
    x = torch.cat([bits.view(-1, dim)] * 4)
    n = x.shape[0]
    tops = torch.tensor([float("nan"), 448.0, 1e-3, 3e4], device="cuda").repeat_interleave(n // 4).to(typ)
    whole = torch.isnan(tops)[:, None]  # rows as they are; the others hold what is below their top
    x = torch.where(whole | (x.abs() <= tops[:, None]), x, torch.zeros_like(x))
    x[:, 0] = torch.where(torch.isnan(tops), x[:, 0], tops)
    w = Window([0], [(0, n, n)], bt)
    c = ps.KvCache.empty(w.n_pages, 1, bt, dim)
    sc.kv_write_dev(c, w.dev(), x[:, None].contiguous(), x.flip(1)[:, None].contiguous())
    ch = torch.from_numpy(w.chain(0).astype(np.int64)).cuda()
    t = torch.arange(n, device="cuda")
    code, e = quantise(x.double().cpu().numpy())
    for buf, ex, want in ((c.tensors[0], c.tensors[2], code), (c.tensors[1], c.tensors[3], code[:, ::-1])):
        got = buf.view(torch.uint8)[ch[t // bt], 0, t % bt].view(E4M3).double().cpu().numpy()
        assert np.array_equal(got, want, equal_nan=True)
        assert np.array_equal(ex[ch[t // bt], 0, t % bt].cpu().numpy(), e)


def test_strided_rows_and_pages(ps, sc):
    """Rows with the heads outermost, pages with K and V side by side."""
    heads, dim, bt = 4, 64, 16
    w = Window([2], [(0, 50, 18), (0, 45, 1)], bt)
    win, g = w.dev(), _gen(1)
    both = torch.zeros(w.n_pages, 2, heads, bt, dim, dtype=F16, device="cuda")
    c = ps.KvCache(both[:, 0], both[:, 1])
    plain = ps.KvCache.empty(w.n_pages, heads, bt, dim, F16)
    k = _randn(g, heads, w.n_rows, dim).half().transpose(0, 1)
    v = _randn(g, w.n_rows, 2 * heads, dim).half()[:, ::2]
    sc.kv_write_dev(c, win, k, v)
    sc.kv_write_dev(plain, win, k.contiguous(), v.contiguous())
    assert torch.equal(both[:, 0], plain.tensors[0]) and torch.equal(both[:, 1], plain.tensors[1])
    ok = torch.zeros(heads, w.n_rows, dim, dtype=F16, device="cuda").transpose(0, 1)
    ov = torch.zeros(w.n_rows, 2 * heads, dim, dtype=F16, device="cuda")[:, ::2]
    sc.kv_read_dev(c, win, ok, ov)
    assert torch.equal(ok, k) and torch.equal(ov, v)
    # attention with q and out in such layouts
    q = _randn(g, 3 * heads, w.n_rows, dim).half().transpose(0, 1)
    out = torch.zeros(3 * heads, w.n_rows, dim, dtype=F16, device="cuda").transpose(0, 1)
    p = sc.attend_plan(3 * heads, heads, dim, bt, w.n_req, w.n_rows)
    p.build_dev(win)
    p.attend_dev(c, q, out)
    check_attention(w, c.tensors, q, out, None, dim ** -0.5)


def test_bad_pages_and_requests_are_skipped(ps, sc):
    heads, dim, bt = 2, 32, 8
    w = Window([3, 3], [(0, 40, 3), (1, 30, 2), (0, 33, 1), (1, 41, 5), (0, 26, 2), (1, 27, 1)], bt, pad=1)
    good = w.dev()
    c = _cache(ps, w, heads, dim, E4M3)
    g = _gen(2)
    k, v = (_randn(g, w.n_rows, heads, dim).bfloat16() for _ in range(2))
    sc.kv_write_dev(c, good, k, v)
    q = _randn(g, w.n_rows, 4, dim).bfloat16()
    p = sc.attend_plan(4, heads, dim, bt, w.n_req, w.n_rows)
    p.build_dev(good)
    ref = torch.zeros_like(q)
    p.attend_dev(c, q, ref)
    bad = {1, 2, 3, 4}
    w.pages[w.reqs[1]["tail_off"]] = w.n_pages  # the page of its rows
    w.reqs[2]["tail_off"] = len(w.pages)
    w.ctx[3] = 1 << 30
    w.reqs[4]["pre_len"] = -1
    win = w.dev()
    flags = torch.full((w.n_req,), 9, dtype=torch.int32, device="cuda")
    p.build_dev(win, d_flags=flags)
    assert flags.tolist() == [8 if r in bad else 0 for r in range(w.n_req)]
    out, lse = torch.full_like(q, 5.0), torch.full((w.n_rows, 4), 5.0, device="cuda")
    p.attend_dev(c, q, out, lse)
    before = [t.clone() for t in c.tensors]
    sc.kv_write_dev(c, win, k, v)  # the good rows hold what they write
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, c.tensors))
    rk, rv = torch.full_like(k, 5.0), torch.full_like(v, 5.0)
    sc.kv_read_dev(c, win, rk, rv)
    lo = w.row_off
    for r in range(w.n_req):
        rows = slice(lo[r], lo[r + 1])
        if r in bad:
            assert (out[rows] == 0).all() and (lse[rows] == -np.inf).all()
            assert (rk[rows] == 0).all() and (rv[rows] == 0).all()
        else:
            assert torch.equal(out[rows], ref[rows])
            assert (rk[rows] != 5).all()
    for t in (out, lse, rk, rv):  # rows of no request
        assert (t[0] == 5).all() and (t[-1] == 5).all()
    # row offsets that do not ascend: nothing is written
    w.row_off[2], w.row_off[3] = w.row_off[3], w.row_off[2]
    p.build_dev(w.dev(), d_flags=flags)
    assert (flags == 8).all()
    out.fill_(5.0)
    p.attend_dev(c, q, out)
    assert (out == 5).all()


def test_offsets_past_32_bits(ps, sc):
    """Pages 2^31 + 4096 elements apart: the last begins past 2^32."""
    heads, dim, bt, n_pages = 1, 64, 16, 3
    stride = (1 << 31) + 4096
    raw = [torch.empty((n_pages - 1) * stride + heads * bt * dim, dtype=torch.uint8, device="cuda") for _ in range(2)]
    k, v = (torch.as_strided(t, (n_pages, heads, bt, dim), (stride, bt * dim, dim, 1)) for t in raw)
    x = [torch.ones(n_pages, heads, bt, dtype=torch.uint8, device="cuda") for _ in range(2)]
    c = ps.KvCache(k.view(E4M3), v.view(E4M3), *x)
    w = Window([0], [(0, 40, 40)], bt)
    w.n_pages, w.pages = n_pages, np.array([2, 0, 1], np.int32)
    g, win = _gen(3), w.dev()
    kr, vr = (_randn(g, 40, heads, dim).bfloat16() for _ in range(2))
    sc.kv_write_dev(c, win, kr, vr)
    q = _randn(g, 40, 4, dim).bfloat16()
    out = torch.zeros_like(q)
    p = sc.attend_plan(4, heads, dim, bt, 1, 40)
    p.build_dev(win)
    p.attend_dev(c, q, out)
    near = ps.KvCache(k.contiguous().view(E4M3), v.contiguous().view(E4M3), *x)
    check_attention(w, near.tensors, q, out, None, dim ** -0.5)
    ref = torch.zeros_like(q)
    p.attend_dev(near, q, ref)
    assert torch.equal(out, ref)


# ------------------------------------------------------------------ attention
SHAPES = [(4, 1, 64, 16), (8, 8, 128, 16), (12, 2, 128, 5), (16, 1, 96, 32), (15, 3, 256, 16), (40, 2, 16, 1),
          (32, 4, 208, 64), (64, 1, 128, 16)]


@pytest.mark.parametrize("heads,kv,dim,bt", SHAPES)
@pytest.mark.parametrize("dtype,typ", [(BF16, BF16), (F16, F16), (E4M3, BF16), (E4M3, F16)])
def test_attention_of_mixed_windows(ps, sc, heads, kv, dim, bt, dtype, typ):
    w = Window(*_mixed(bt), bt, seed=heads, pad=3, spare=1)
    c = _cache(ps, w, kv, dim, dtype)
    q = _randn(_gen(dim), w.n_rows, heads, dim).to(typ)
    out, lse = torch.full_like(q, 3.0), torch.full((w.n_rows, heads), 3.0, device="cuda")
    p = sc.attend_plan(heads, kv, dim, bt, w.n_req, w.n_rows)
    p.build_dev(w.dev())
    p.attend_dev(c, q, out, lse)
    check_attention(w, c.tensors, q, out, lse, dim ** -0.5)
    for t in (out, lse):
        assert (t[:3] == 3).all() and (t[-3:] == 3).all()


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 511, 513, 2049, 5000])
@pytest.mark.parametrize("dtype,typ", [(BF16, BF16), (E4M3, F16)])
def test_lengths(ps, sc, n, dtype, typ):
    heads, kv, dim, bt = 8, 2, 128, 16
    w = Window([0], [(0, n, 1)], bt, seed=n)
    c = _cache(ps, w, kv, dim, dtype)
    q = 2 * _randn(_gen(n), 1, heads, dim).to(typ)
    out, lse = torch.zeros_like(q), torch.zeros(1, heads, device="cuda")
    p = sc.attend_plan(heads, kv, dim, bt, 1, 1)
    p.build_dev(w.dev())
    p.attend_dev(c, q, out, lse)
    check_attention(w, c.tensors, q, out, lse, dim ** -0.5)


@pytest.mark.parametrize("members,pre,rows", [(2, 5, 1), (16, 9, 1), (33, 4, 1), (70, 40, 1), (9, 12, 5), (3, 20, 40),
                                              (130, 3, 2)])
@pytest.mark.parametrize("heads,kv,dim,dtype,typ", [(8, 2, 128, E4M3, BF16), (6, 2, 64, F16, F16),
                                                    (5, 1, 256, BF16, BF16)])
def test_shared_prefixes(ps, sc, members, pre, rows, heads, kv, dim, dtype, typ):
    bt = 16
    rng = np.random.default_rng(members)
    reqs = [(0, pre * bt + int(rng.integers(0, 50)), rows) for _ in range(members)]
    reqs += [(1, 3 * bt + 1, 1), (0, pre * bt + rows, rows), (1, 7 * bt, 2)]
    w = Window([pre, 3], reqs, bt, seed=members)
    c = _cache(ps, w, kv, dim, dtype)
    q = _randn(_gen(rows), w.n_rows, heads, dim).to(typ)
    out, lse = torch.zeros_like(q), torch.zeros(w.n_rows, heads, device="cuda")
    p = sc.attend_plan(heads, kv, dim, bt, w.n_req, w.n_rows)
    p.build_dev(w.dev())
    p.attend_dev(c, q, out, lse)
    check_attention(w, c.tensors, q, out, lse, dim ** -0.5)


@pytest.mark.parametrize("heads,kv,dim,bt,n,ctx", [(4, 1, 128, 16, 300, 300), (8, 8, 64, 16, 129, 700),
                                                   (2, 1, 256, 16, 200, 1000), (6, 2, 96, 7, 161, 500)])
@pytest.mark.parametrize("dtype,typ", [(BF16, BF16), (E4M3, F16)])
def test_prefill_chunks(ps, sc, heads, kv, dim, bt, n, ctx, dtype, typ):
    w = Window([2], [(0, ctx, n), (0, ctx // 2, n // 3), (0, n // 2, n)], bt, seed=n)
    c = _cache(ps, w, kv, dim, dtype)
    q = _randn(_gen(n), w.n_rows, heads, dim).to(typ)
    out, lse = torch.zeros_like(q), torch.zeros(w.n_rows, heads, device="cuda")
    p = sc.attend_plan(heads, kv, dim, bt, w.n_req, w.n_rows)
    p.build_dev(w.dev())
    p.attend_dev(c, q, out, lse)
    check_attention(w, c.tensors, q, out, lse, dim ** -0.5)


@pytest.mark.parametrize("dtype,typ", [(BF16, BF16), (F16, F16), (E4M3, BF16)])
@pytest.mark.parametrize("heads", [4, 40])
def test_what_lies_behind_a_row_does_not_reach_it(ps, sc, dtype, typ, heads):
    """NaN and infinities in later tokens of the chunk, in the rest of the last page and in unused pages: the
    rows before them keep their bits."""
    kv, dim, bt = 1, 64, 16
    w = Window([3], [(0, 70, 70), (0, 3 * bt + 21, 5), (0, 3 * bt + 5, 1), (0, 3 * bt, 3)], bt, spare=2)
    c = _cache(ps, w, kv, dim, dtype)
    q = _randn(_gen(5), w.n_rows, heads, dim).to(typ)
    p = sc.attend_plan(heads, kv, dim, bt, w.n_req, w.n_rows)
    p.build_dev(w.dev())
    ref, out = torch.zeros_like(q), torch.zeros_like(q)
    lref, lse = torch.zeros(w.n_rows, heads, device="cuda"), torch.zeros(w.n_rows, heads, device="cuda")
    p.attend_dev(c, q, ref, lref)
    check_attention(w, c.tensors, q, ref, lref, dim ** -0.5)
    junk = torch.tensor([float("nan"), float("inf"), -float("inf"), 3.0], device="cuda").repeat(dim // 4)
    if dtype == E4M3:
        junk = torch.tensor([0x7F, 0xFF, 0x7E, 0x80], dtype=torch.uint8, device="cuda").repeat(dim // 4)

    def spoil(page, slot):
        for t in c.tensors[:2]:
            if dtype == E4M3:
                t.view(torch.uint8)[page, :, slot] = junk
            else:
                t[page, :, slot] = junk.to(dtype)

    used = {(int(w.chain(r)[t // bt]), t % bt) for r in range(w.n_req) for t in range(w.ctx[r])}
    for page in range(w.n_pages):
        for slot in range(bt):
            if (page, slot) not in used:
                spoil(page, slot)
    first = 55  # tokens from here on of the first request's own part, and its later rows, are spoiled
    ch = w.chain(0)
    for t in range(first, 70):
        spoil(int(ch[t // bt]), t % bt)
    p.attend_dev(c, q, out, lse)
    same = torch.ones(w.n_rows, dtype=torch.bool)
    same[first:70] = False
    assert torch.equal(out[same], ref[same]) and torch.equal(lse[same], lref[same])
    assert torch.isnan(out[first:70]).any()


def test_large_scores_and_equal_ones(ps, sc):
    """Scores of many hundreds (one weight takes all) and all alike (the mean of v)."""
    heads, kv, dim, bt = 4, 2, 64, 16
    w = Window([4], [(0, 4 * bt + 40, 3), (0, 4 * bt + 7, 1)], bt)
    c = _cache(ps, w, kv, dim, BF16)
    q = 60 * _randn(_gen(1), w.n_rows, heads, dim).bfloat16()
    q[0] = 0
    out, lse = torch.zeros_like(q), torch.zeros(w.n_rows, heads, device="cuda")
    p = sc.attend_plan(heads, kv, dim, bt, w.n_req, w.n_rows)
    p.build_dev(w.dev())
    p.attend_dev(c, q, out, lse)
    check_attention(w, c.tensors, q, out, lse, dim ** -0.5)
    p.attend_dev(c, q, out, lse, scale=0.0)
    check_attention(w, c.tensors, q, out, lse, 0.0)


def test_layers_of_a_step(ps, sc):
    """Plan once; per layer write the new rows, attend, read back."""
    heads, kv, dim, bt = 8, 2, 128, 16
    w = Window([6, 9], [(0, 6 * bt + 5, 1), (1, 9 * bt + 20, 2), (0, 6 * bt + 30, 1), (1, 9 * bt + 1, 1), (0, 100, 4)],
               bt)
    win, g = w.dev(), _gen(7)
    p = sc.attend_plan(heads, kv, dim, bt, w.n_req, w.n_rows)
    p.build_dev(win)
    for layer, dtype in enumerate((E4M3, BF16, E4M3)):
        c = _cache(ps, w, kv, dim, dtype, seed=layer)
        k, v = (_randn(g, w.n_rows, kv, dim).bfloat16() for _ in range(2))
        q = _randn(g, w.n_rows, heads, dim).bfloat16()
        out, lse = torch.zeros_like(q), torch.zeros(w.n_rows, heads, device="cuda")
        sc.kv_write_dev(c, win, k, v)
        p.attend_dev(c, q, out, lse)
        rk, rv = torch.zeros_like(k), torch.zeros_like(v)
        sc.kv_read_dev(c, win, rk, rv)
        # half a step of e4m3 relative, or of its smallest step under the row's maximum
        for a, b in ((rk, k), (rv, v)):
            a, b = a.double(), b.double()
            top = b.abs().amax(-1, keepdim=True)
            assert ((a - b).abs() <= (0 if dtype == BF16 else torch.maximum(b.abs() / 16, top / 224 * 2.0 ** -10))).all()
        check_attention(w, c.tensors, q, out, lse, dim ** -0.5)


def test_same_bits_every_time_and_on_other_streams(ps, sc):
    heads, kv, dim, bt = 16, 2, 128, 16
    rng = np.random.default_rng(3)
    w = Window([30, 11, 0], [(int(s), 30 * bt + int(rng.integers(1, 300)), int(rng.integers(1, 4)))
                             for s in rng.integers(0, 3, 60)], bt)
    win = w.dev()
    c = _cache(ps, w, kv, dim, E4M3)
    q = _randn(_gen(1), w.n_rows, heads, dim).bfloat16()
    ref = torch.zeros_like(q)
    p = sc.attend_plan(heads, kv, dim, bt, w.n_req, w.n_rows)
    p.build_dev(win)
    p.attend_dev(c, q, ref)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for k in range(6):
        other = sc.attend_plan(heads, kv, dim, bt, w.n_req + k, w.n_rows + 5 * k)
        out = torch.zeros_like(q)
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream if k % 2 else torch.cuda.current_stream()):
            other.build_dev(win)
            other.attend_dev(c, q, out)
        torch.cuda.synchronize()
        assert torch.equal(out, ref), k
        other.close()


def test_graphs_replay_with_new_windows(ps, sc):
    """Plan, write, attend and read captured once; replays take what the buffers then hold.  Two graphs with a plan
    each, replayed in turn, with eager work between."""
    heads, kv, dim, bt, n = 8, 2, 64, 16, 6

    def window(seed):
        rng = np.random.default_rng(seed)
        return Window([5, 2], [(int(s), (5, 2)[s] * bt + int(rng.integers(1, 33)), 1)
                               for s in rng.integers(0, 2, n)], bt, seed=seed)

    class Graph:
        def __init__(self):
            g = _gen(1)
            self.pages = torch.zeros(7 + 3 * n, dtype=torch.int32, device="cuda")
            self.reqs = torch.zeros(n * 24, dtype=torch.uint8, device="cuda")
            self.ctx = torch.zeros(n, dtype=torch.int32, device="cuda")
            self.off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
            self.cache = ps.KvCache.empty(40, kv, bt, dim)
            self.k, self.v = (_randn(g, n, kv, dim).bfloat16() for _ in range(2))
            self.q = _randn(g, n, heads, dim).bfloat16()
            self.out, self.lse = torch.zeros_like(self.q), torch.zeros(n, heads, device="cuda")
            self.win = ps.KvWindow(self.pages, self.reqs, self.ctx, self.off, n, n, 40)
            self.plan = sc.attend_plan(heads, kv, dim, bt, n, n)
            self.flags = torch.zeros(n, dtype=torch.int32, device="cuda")
            self.graph = torch.cuda.CUDAGraph()
            self.load(window(0))
            torch.cuda.synchronize()
            with torch.cuda.graph(self.graph):
                self.calls()

        def calls(self):
            self.plan.build_dev(self.win, d_flags=self.flags)
            sc.kv_write_dev(self.cache, self.win, self.k, self.v)
            self.plan.attend_dev(self.cache, self.q, self.out, self.lse)

        def load(self, w):
            self.w = w
            w.n_pages = 40
            self.pages[:len(w.pages)] = torch.from_numpy(w.pages).cuda()
            self.reqs.copy_(torch.from_numpy(w.reqs.view(np.uint8).reshape(-1).copy()))
            self.ctx.copy_(torch.from_numpy(w.ctx))

    a, b = Graph(), Graph()
    for turn in range(8):
        for gr in (a, b):
            gr.load(window(10 * turn + (gr is a)))
            gr.out.fill_(9.0)
            gr.graph.replay()
        torch.cuda.synchronize()
        for gr in (a, b):
            assert (gr.flags == 0).all()
            check_attention(gr.w, gr.cache.tensors, gr.q, gr.out, gr.lse, dim ** -0.5)
            got = gr.out.clone()
            gr.calls()
            assert torch.equal(gr.out, got)


def test_limits_and_states(ps, sc):
    heads, kv, dim, bt = 4, 2, 64, 16
    w = Window([2], [(0, 40, 2), (0, 50, 1)], bt)
    win, c = w.dev(), None
    c = _cache(ps, w, kv, dim, BF16)
    q = torch.zeros(3, heads, dim, dtype=BF16, device="cuda")
    p = sc.attend_plan(heads, kv, dim, bt, 2, 3)
    with pytest.raises(ps.PackServeError) as e:
        p.attend_dev(c, q, torch.zeros_like(q))
    assert e.value.code == ps.binding.PS_E_STATE
    for small in (sc.attend_plan(heads, kv, dim, bt, 1, 3), sc.attend_plan(heads, kv, dim, bt, 2, 2)):
        with pytest.raises(ps.PackServeError) as e:
            small.build_dev(win)
        assert e.value.code == ps.binding.PS_E_RANGE
    p.build_dev(win)
    for other in (_cache(ps, w, 1, dim, BF16), _cache(ps, w, kv, 32, BF16),
                  ps.KvCache.empty(w.n_pages, kv, 8, dim, BF16)):
        with pytest.raises((ps.PackServeError, ValueError)):
            p.attend_dev(other, q, torch.zeros_like(q))
    short = ps.KvCache.empty(w.n_pages - 1, kv, bt, dim, BF16)
    for call in (lambda: p.attend_dev(short, q, torch.zeros_like(q)),
                 lambda: sc.kv_read_dev(short, win, q[:, :kv].contiguous(), q[:, :kv].contiguous())):
        with pytest.raises(ps.PackServeError) as e:
            call()
        assert "more pages" in str(e.value)
    with pytest.raises(ValueError):
        p.attend_dev(c, q[:2], torch.zeros_like(q))
    with pytest.raises(ValueError):
        p.attend_dev(c, q.cpu(), torch.zeros_like(q))
    with pytest.raises(ValueError):
        p.attend_dev(c, q, torch.zeros_like(q), lse=torch.zeros(3, heads + 1, device="cuda"))
    # an empty window, and a plan of nothing
    empty = Window([0], [], bt)
    p.build_dev(empty.dev())
    p.attend_dev(c, q, torch.zeros_like(q))
    sc.attend_plan(heads, kv, dim, bt, 0, 0).build_dev(empty.dev())
    p.close()
    with pytest.raises(ValueError):
        p.attend_dev(c, q, torch.zeros_like(q))


def test_plans_go_with_their_context(ps):
    from tests.gpu_util import limit_memory
    s = ps.Scorer(0)
    held = limit_memory(s, 0)
    p = s.attend_plan(8, 2, 128, 16, 64, 512)
    assert limit_memory(s, 0) > held
    limit_memory(s, limit_memory(s, 0) + 1024)
    with pytest.raises(ps.PackServeError) as e:
        s.attend_plan(8, 2, 128, 16, 64, 512)
    assert e.value.code == ps.binding.PS_E_NOMEM
    limit_memory(s, 0)
    q = s.attend_plan(8, 2, 128, 16, 64, 512)
    p.close()
    s.close()
    q.close()  # freed with the context
    with pytest.raises(ValueError):
        q.build_dev(Window([0], [], 16).dev())


def _attend(ps, sc, w, heads, kv, dim, dtype, typ, seed=1, amp=1.0, check=True, plan=None):
    c = _cache(ps, w, kv, dim, dtype, seed=seed)
    q = amp * _randn(_gen(seed), w.n_rows, heads, dim).to(typ)
    out, lse = torch.full_like(q, 3.0), torch.full((w.n_rows, heads), 3.0, device="cuda")
    p = plan or sc.attend_plan(heads, kv, dim, w.bt, w.n_req, w.n_rows)
    p.build_dev(w.dev())
    p.attend_dev(c, q, out, lse)
    if check:
        check_attention(w, c.tensors, q, out, lse, dim ** -0.5)
    return c, q, out, lse, p


# windows with many rows a request: tiles of 256 rows; the last has one that decodes beside them
TALL = [(64, 1, 128, 16, [3], [(0, 700, 150), (0, 3 * 16 + 90, 90)]),
        (96, 1, 96, 7, [9], [(0, 201, 120), (0, 64, 1)]),
        (64, 2, 112, 16, [0], [(0, 65, 65), (0, 257, 257), (0, 129, 129)]),
        (16, 1, 80, 5, [0, 4], [(0, 640, 600), (1, 300, 1)])]


@pytest.mark.parametrize("heads,kv,dim,bt,sessions,reqs", TALL)
@pytest.mark.parametrize("dtype,typ", [(BF16, BF16), (F16, F16), (E4M3, BF16), (E4M3, F16)])
def test_tall_tiles(ps, sc, heads, kv, dim, bt, sessions, reqs, dtype, typ):
    w = Window(sessions, reqs, bt, seed=dim, pad=1)
    _, _, out, lse, _ = _attend(ps, sc, w, heads, kv, dim, dtype, typ)
    for t in (out, lse):
        assert (t[:1] == 3).all() and (t[-1:] == 3).all()


@pytest.mark.parametrize("n", [64, 65, 127, 128, 129, 191, 192, 193, 320])
def test_tall_tiles_of_few_steps(ps, sc, n):
    """Contexts about as long as the steps that are staged ahead."""
    w = Window([0], [(0, n, 64)], 16, seed=n)
    _attend(ps, sc, w, 64, 1, 128, E4M3, BF16, amp=2.0)


@pytest.mark.parametrize("dtype,typ", [(BF16, BF16), (E4M3, F16)])
def test_what_lies_behind_a_row_does_not_reach_it_in_tall_tiles(ps, sc, dtype, typ):
    heads, kv, dim, bt, n, first = 64, 1, 128, 16, 150, 101
    w = Window([0], [(0, 200, n)], bt)
    c, q, ref, lref, p = _attend(ps, sc, w, heads, kv, dim, dtype, typ)
    ch = w.chain(0)
    junk = torch.tensor([float("nan"), float("inf"), -float("inf"), 3.0], device="cuda").repeat(dim // 4)
    if dtype == E4M3:
        junk = torch.tensor([0x7F, 0xFF, 0x7E, 0x80], dtype=torch.uint8, device="cuda").repeat(dim // 4)
    for t in range(50 + first, -(-200 // bt) * bt):
        for x in c.tensors[:2]:
            if dtype == E4M3:
                x.view(torch.uint8)[int(ch[t // bt]), :, t % bt] = junk
            else:
                x[int(ch[t // bt]), :, t % bt] = junk.to(dtype)
    out, lse = torch.zeros_like(q), torch.zeros_like(lref)
    p.attend_dev(c, q, out, lse)
    assert torch.equal(out[:first], ref[:first]) and torch.equal(lse[:first], lref[:first])
    assert torch.isnan(out[first:]).any(-1).all()


def test_growing_scores(ps, sc):
    """Maxima that grow slowly, at once and not at all, so that rows follow them at different steps."""
    heads, kv, dim, bt = 64, 1, 128, 16
    for n in (64, 1):
        w = Window([0], [(0, 600, n)], bt)
        c = _cache(ps, w, kv, dim, BF16)
        ch = torch.from_numpy(w.chain(0).astype(np.int64)).cuda()
        t = torch.arange(600, device="cuda")
        c.tensors[0][ch[t // bt], 0, t % bt, 0] = (t / 8).bfloat16()
        q = _randn(_gen(2), n, heads, dim).bfloat16()
        q[:, :, 0] = torch.linspace(-6, 6, heads, device="cuda").bfloat16()
        out, lse = torch.zeros_like(q), torch.zeros(n, heads, device="cuda")
        p = sc.attend_plan(heads, kv, dim, bt, 1, n)
        p.build_dev(w.dev())
        for scale in (dim ** -0.5, 1.0):
            p.attend_dev(c, q, out, lse, scale=scale)
            check_attention(w, c.tensors, q, out, lse, scale)


@pytest.mark.parametrize("heads,kv,dim,n_req,most", [(2, 1, 16, 1500, 40), (1, 1, 16, 8192, 9), (64, 1, 16, 1100, 20),
                                                     (64, 8, 64, 150, 90)])
def test_windows_of_many_requests(ps, sc, heads, kv, dim, n_req, most):
    """More requests than the plan's tables in shared memory hold, or more tiles than workgroups; contexts of 0 too."""
    bt = 4
    rng = np.random.default_rng(n_req)
    sessions = [0, 2, 30, 17]
    reqs = []
    for s in rng.integers(0, 4, n_req):
        ctx = int(rng.integers(0, most))
        reqs.append((int(s), ctx + (sessions[s] * bt if rng.random() < 0.8 else 0), 1))
    w = Window(sessions, reqs, bt, seed=n_req)
    _attend(ps, sc, w, heads, kv, dim, E4M3, BF16)


@pytest.mark.parametrize("heads,kv,dim", [(300, 1, 32), (128, 128, 16), (1024, 4, 64)])
def test_many_heads(ps, sc, heads, kv, dim):
    w = Window([9, 0], [(0, 150, 1), (0, 9 * 16 + 1, 1), (1, 70, 2), (0, 9 * 16, 1)], 16)
    _attend(ps, sc, w, heads, kv, dim, F16, F16)


def test_a_negative_scale_turns_q(ps, sc):
    for heads, kv, n in ((4, 2, 1), (8, 1, 20), (64, 1, 70)):
        w = Window([2], [(0, 90, n)], 16)
        c, q, _, _, p = _attend(ps, sc, w, heads, kv, 128, E4M3, BF16)
        a, b = torch.zeros_like(q), torch.zeros_like(q)
        p.attend_dev(c, q, a, scale=-0.1)
        p.attend_dev(c, -q, b, scale=0.1)
        assert torch.equal(a, b)


def test_a_page_twice_in_a_chain(ps, sc):
    w = Window([4], [(0, 150, 3), (0, 100, 1)], 16)
    w.pages[1] = w.pages[0]
    d = w.reqs[0]
    w.pages[d["tail_off"]:d["tail_off"] + 3] = w.pages[3]
    _attend(ps, sc, w, 8, 2, 64, BF16, BF16)


def test_padding_requests_and_a_plan_for_more(ps, sc):
    """Requests of no rows and no blocks behind the last; one plan for large and small windows in turn."""
    heads, kv, dim, bt = 64, 1, 128, 16
    p = sc.attend_plan(heads, kv, dim, bt, 1200, 400)
    big = [(0, 48 + 5 * k, 1) for k in range(9)]
    for reqs in (big + [(1, 0, 0)] * 7, [(1, 130, 130)], [(1, 0, 0)] * 3, big, [(1, 300, 200), (0, 50, 1)]):
        w = Window([3, 0], reqs, bt, pad=2)
        _, _, out, _, _ = _attend(ps, sc, w, heads, kv, dim, E4M3, BF16, plan=p)
        assert (out[:2] == 3).all() and (out[-2:] == 3).all()


def test_two_streams_at_once(ps, sc):
    """Two plans at work at the same time, each on its own stream."""
    rng = np.random.default_rng(1)
    work = []
    for k, (heads, kv, dim) in enumerate(((16, 2, 128), (64, 1, 128))):
        w = Window([40], [(0, 640 + int(rng.integers(1, 300)), 1 if k == 0 else 100) for _ in range(8 if k == 0 else 1)], 16)
        c, q, ref, _, _ = _attend(ps, sc, w, heads, kv, dim, E4M3, BF16)
        p = sc.attend_plan(heads, kv, dim, 16, w.n_req, w.n_rows)
        work.append((p, w.dev(), c, q, ref, [torch.zeros_like(q) for _ in range(5)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(5):
        for p, win, c, q, _, outs, stream in work:
            with torch.cuda.stream(stream):
                p.build_dev(win)
                p.attend_dev(c, q, outs[i])
    torch.cuda.synchronize()
    for _, _, _, _, ref, outs, _ in work:
        assert all(torch.equal(o, ref) for o in outs)


def test_flags_of_a_window_without_rows(ps, sc):
    w = Window([2], [(0, 40, 0), (0, 0, 0), (0, 35, 0)], 16)
    w.reqs[2]["pre_off"] = 1 << 40
    flags = torch.full((3,), 9, dtype=torch.int32, device="cuda")
    p = sc.attend_plan(4, 2, 64, 16, 3, 0)
    p.build_dev(w.dev(), d_flags=flags)
    assert w.n_rows == 0 and flags.tolist() == [0, 0, 8]
    c = _cache(ps, w, 2, 64, E4M3)
    q = torch.ones(1, 4, 64, dtype=BF16, device="cuda")
    p.attend_dev(c, q, q)
    assert (q == 1).all()


def test_pages_over_each_other_and_other_devices_are_refused(ps, sc):
    w = Window([0], [(0, 20, 2)], 16)
    win, rows = w.dev(), torch.zeros(2, 1, 64, dtype=BF16, device="cuda")
    one = ps.KvCache.empty(1, 1, 16, 64)
    k, v, kx, vx = one.tensors
    n = w.n_pages
    for c in (ps.KvCache(k.expand(n, -1, -1, -1), v.expand(n, -1, -1, -1), *(x.repeat(n, 1, 1) for x in (kx, vx))),
              ps.KvCache(k.repeat(n, 1, 1, 1), v.repeat(n, 1, 1, 1), *(x.expand(n, -1, -1) for x in (kx, vx)))):
        for call in (sc.kv_write_dev, sc.kv_read_dev):
            with pytest.raises(ps.PackServeError) as e:
                call(c, win, rows, rows)
            assert e.value.code == ps.binding.PS_E_INVAL and "stride" in str(e.value)
    c = ps.KvCache.empty(n, 1, 16, 64)
    p = sc.attend_plan(1, 1, 64, 16, 1, 2)
    sc.device_index += 1
    try:
        for call in (lambda: sc.kv_write_dev(c, win, rows, rows), lambda: sc.kv_read_dev(c, win, rows, rows),
                     lambda: p.build_dev(win)):
            with pytest.raises(ValueError):
                call()
    finally:
        sc.device_index -= 1


def test_growing_scores_in_half_precision(ps, sc):
    """Weights are taken from a maximum that may lie 2^8 below the row's: they must stay in the type's range."""
    heads, kv, dim, bt = 64, 1, 128, 16
    for n in (64, 1):
        w = Window([0], [(0, 600, n)], bt)
        c = _cache(ps, w, kv, dim, F16)
        ch = torch.from_numpy(w.chain(0).astype(np.int64)).cuda()
        t = torch.arange(600, device="cuda")
        c.tensors[0][ch[t // bt], 0, t % bt, 0] = ((t * 37) % 600 / 8).half()
        q = _randn(_gen(2), n, heads, dim).half()
        q[:, :, 0] = torch.linspace(-6, 6, heads, device="cuda").half()
        out, lse = torch.zeros_like(q), torch.zeros(n, heads, device="cuda")
        p = sc.attend_plan(heads, kv, dim, bt, 1, n)
        p.build_dev(w.dev())
        for scale in (dim ** -0.5, 1.0):
            p.attend_dev(c, q, out, lse, scale=scale)
            check_attention(w, c.tensors, q, out, lse, scale)


@pytest.mark.parametrize("heads,n", [(4, 1), (4, 30), (64, 64)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_an_infinity_that_is_seen(ps, sc, heads, n, dtype):
    """Of one sign: every row that sees it is infinite in that element, the rows before it keep their bits."""
    kv, dim, bt, ctx = 1, 128, 16, 64
    w = Window([0], [(0, ctx, n)], bt)
    c, q, ref, lref, p = _attend(ps, sc, w, heads, kv, dim, dtype, dtype)
    at = ctx - 1 - n // 2
    c.tensors[1][int(w.chain(0)[at // bt]), 0, at % bt, 5] = float("inf")
    out, lse = torch.zeros_like(q), torch.zeros_like(lref)
    p.attend_dev(c, q, out, lse)
    sees = torch.arange(ctx - n, ctx, device="cuda") >= at
    assert torch.equal(lse, lref) and torch.equal(out[~sees], ref[~sees])
    rest = torch.arange(dim, device="cuda") != 5
    assert (out[sees][:, :, 5] == float("inf")).all() and torch.equal(out[:, :, rest], ref[:, :, rest])


def test_attention_captured_without_its_plan(ps, sc):
    """Another window planned in between, cut for other workgroups: nothing is written; the first one again: its
    results."""
    heads, kv, dim, bt = 63, 7, 128, 16
    w = Window([2], [(0, 32 + 9 * k, 1) for k in range(12)], bt)
    big = Window([0], [(0, 200, 190)], bt)
    p = sc.attend_plan(heads, kv, dim, bt, 12, 190)
    c, q, ref, _, _ = _attend(ps, sc, w, heads, kv, dim, E4M3, BF16, plan=p)
    win, many = w.dev(), big.dev()
    out = torch.full_like(q, 3.0)
    p.build_dev(win)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.attend_dev(c, q, out)
    for _ in range(3):
        out.fill_(3.0)
        p.build_dev(many)
        graph.replay()
        torch.cuda.synchronize()
        assert (out == 3).all()
        p.build_dev(win)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
