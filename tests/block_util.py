"""Windows over a block cache for the tests, and the cache calls and the
attention written out in 64 bits on the CPU."""
import numpy as np
import torch

REQ = np.dtype([("pre_off", "<i8"), ("tail_off", "<i8"), ("pre_len", "<i4"), ("tail_len", "<i4")])
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # half a step, relative


class Window:
    """n_pages pages in a shuffled order.  reqs: (session, tokens of the context, rows);
    sessions: blocks of each session's shared prefix.  A request's chain holds its
    context and `spare` blocks more.  `pad` rows lie before the first request and
    behind the last."""

    def __init__(self, sessions, reqs, bt, seed=0, spare=0, pad=0):
        rng = np.random.default_rng(seed)
        self.bt, self.n_req = bt, len(reqs)
        pre_at = np.concatenate([[0], np.cumsum(sessions)]).astype(int)
        self.reqs = np.zeros(len(reqs), REQ)
        at = pre_at[-1]
        for r, (s, ctx, rows) in enumerate(reqs):
            pre = sessions[s]
            tail = max(0, -(-ctx // bt) - pre) + spare
            self.reqs[r] = (pre_at[s], at, pre, tail)
            at += tail
        self.n_pages = at + 2
        self.pages = rng.permutation(self.n_pages)[:at].astype(np.int32)
        self.ctx = np.array([c for _, c, _ in reqs], np.int32)
        self.row_off = (pad + np.concatenate([[0], np.cumsum([n for _, _, n in reqs])])).astype(np.int32)
        self.n_rows = int(self.row_off[-1]) + pad

    def chain(self, r):
        d = self.reqs[r]
        return np.concatenate([self.pages[d["pre_off"]:d["pre_off"] + d["pre_len"]],
                               self.pages[d["tail_off"]:d["tail_off"] + d["tail_len"]]])

    def rows(self, r):
        """(row, position) of every row of request r."""
        lo, hi = self.row_off[r], self.row_off[r + 1]
        return [(i, int(self.ctx[r]) - (hi - lo) + (i - lo)) for i in range(lo, hi)]

    def dev(self):
        import paper_2609_33224_amd as ps
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        return ps.KvWindow(up(self.pages), up(self.reqs.view(np.uint8).reshape(-1).copy()), up(self.ctx),
                           up(self.row_off), self.n_req, self.n_rows, self.n_pages)


def quantise(x):
    """(codes as float64, exponents + 127) of rows x (float64): the least e in [-126, 127] with
    max finite |x| <= 448 * 2^e; round to nearest even on the e4m3 grid."""
    big = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    m, e = np.frexp(big)
    e = np.where(big == 0, -126, e - 9 + (m > 0.875)).clip(-126, 127)
    y = np.clip(x * np.exp2(-e.astype(float))[..., None], -448, 448)  # (NaN stays)
    a = np.maximum(np.abs(y), 2.0 ** -60)
    step = np.exp2(np.maximum(np.floor(np.log2(a)), -6.0) - 3)
    return np.round(y / step) * step, (e + 127).astype(np.uint8)


def values(cache):
    """(k, v) of a cache (tensors) in float64."""
    k, v, kx, vx = [t.cpu() if t is not None else None for t in cache]
    if kx is None:
        return k.double().numpy(), v.double().numpy()
    return tuple(t.double().numpy() * np.exp2(x.double().numpy() - 127.0)[..., None] for t, x in ((k, kx), (v, vx)))


def attend(w, kval, vval, q, scale, typ, skip=()):
    """(out, sum of p |v|, lse, largest sum of |q k| scale) per row and head; rows of no request are NaN
    in out.  skip: malformed requests, whose rows come out empty."""
    rows, heads, dim = q.shape
    ratio = heads // kval.shape[1]
    out, mag = np.full((rows, heads, dim), np.nan), np.zeros((rows, heads, dim))
    lse, big = np.full((rows, heads), np.nan), np.zeros((rows, heads))
    for r in range(w.n_req):
        for i, pos in w.rows(r):
            out[i], lse[i] = 0.0, -np.inf
            if pos < 0 or r in skip:
                continue
            t = np.arange(pos + 1)
            ch = w.chain(r)
            k, v = (x[ch[t // w.bt], :, t % w.bt] for x in (kval, vval))  # (token, KV head, element)
            for h in range(heads):
                kk, vv = k[:, h // ratio], v[:, h // ratio]
                s = kk @ q[i, h] * scale
                big[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
                top = s.max()
                p = np.exp(s - top)
                lse[i, h] = top + np.log(p.sum())
                p /= p.sum()
                out[i, h], mag[i, h] = p @ vv, p @ np.abs(vv)
    return out, mag, lse, big


def check_attention(w, cache, q, out, lse, scale, skip=()):
    """Against the bound of one rounding of the weights and one of the result.

    With h half a step of the type: each weight is off by h (rounding) and by the error of
    its exponent, at most dim * 2^-24 of the sum of |q k| scale (fp32 sums of dim products,
    whatever their order) plus 2^-20 (scaling, exponential); numerator and denominator both.
    Sums over T tokens in fp32, in blocks of 16 at least: (T / 16 + 16) 2^-24.  A weight below
    the smallest normal fp16 number is off by 2^-25 instead."""
    typ = q.dtype
    kval, vval = values(cache)
    want, mag, want_lse, big = attend(w, kval, vval, q.double().cpu().numpy(), scale, typ, skip)
    h, dim, T = HALF[typ], q.shape[2], max(1, int(w.ctx.max()) if w.n_req else 1)
    err = dim * 2.0 ** -24 * big + 2.0 ** -20 + (T / 16 + 16) * 2.0 ** -24
    tol = h * np.abs(want) + (h + 2 * err[..., None]) * (1 + h) * mag
    if typ == torch.float16:
        tol = tol + T * 2.0 ** -25 * np.abs(vval[np.isfinite(vval)]).max() + 2.0 ** -25
    got = out.double().cpu().numpy()
    mine = ~np.isnan(want)
    off = np.abs(got - want)[mine]
    worst = (off / (tol[mine] + 1e-300)).max() if mine.any() else 0.0
    assert (off <= tol[mine] + 1e-300).all(), f"off by {worst:.2f} times the bound"
    if lse is not None:
        g = lse.double().cpu().numpy()
        m = ~np.isnan(want_lse)
        empty = np.isneginf(want_lse) & m
        assert (g[empty] == -np.inf).all()
        m &= ~empty
        ltol = err + 2.0 ** -22 * np.abs(np.where(m, want_lse, 0)) + 2.0 ** -22
        assert (np.abs(g[m] - want_lse[m]) <= ltol[m]).all(), np.abs(g[m] - want_lse[m]).max()
    return worst
