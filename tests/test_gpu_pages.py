"""A paged 4-bit KV cache on the GPU: rows in and out, attention over it, and
its page tables, against plain definitions in 64 bits (oracle/pages.py).

Tolerances.  An fp16 result is off by at most half a step, 2^-11 of its value
(2^-25 below 2^-14).  Whole numbers and what rows stand for in the cache are
equal.  Attention adds, per weight, one more rounding to fp16 where a sequence
has many queries (2^-11 of the weight, against values of at most max|V|), and
what the fp32 sums of q . code leave: codes are held as 16 + c or 256 + c, so a
sum over a group of 64 runs up to 272 sum|q|, is rounded about 66 times by up to
2^-25 of that (root 66 = 8 together) and multiplied by a scale; that error of a
score, four times over for the sum of two groups and its largest of many, is a
relative error of a weight."""
import ctypes

import numpy as np
import pytest

from oracle import pages as O
from paper_2504_03664_amd import binding as B
from paper_2504_03664_amd.binding import DeviceBuffer as DB

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -11


def dev(a, dtype=None):
    return DB.from_array(np.ascontiguousarray(a, dtype))


class Cache:
    """Sequences of given lengths on pages in random order; the pool starts out
    as bytes of `fill` (255: every scale and min a NaN)."""

    def __init__(self, lens, Hkv, D, ps, rng, extra=3, layers=1, fill=255, width=0):
        self.lens, self.Hkv, self.D, self.ps, self.layers = list(lens), Hkv, D, ps, layers
        need = [-(-n // ps) for n in lens]
        self.n_pages = sum(need) + extra
        self.width = max(need + [1]) + width
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(lens), self.width), -1, np.int32)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.page = B.pipo_kv_page_bytes(ps, Hkv, D)
        self.pool = dev(np.full(layers * self.n_pages * self.page, fill, np.uint8))
        self.d_table = dev(self.table)

    def c(self):
        return B.PipoKvPages(self.pool.ptr, self.n_pages * self.page, self.d_table.ptr, self.width,
                             self.layers, self.n_pages, self.ps, self.Hkv, self.D, len(self.lens))

    def set_table(self, t):
        self.table = np.ascontiguousarray(t, np.int32)
        self.d_table = dev(self.table)

    def fill(self, k, v, layer=0):
        """k, v: per sequence [len][Hkv * D] fp16; returns the float64 values"""
        seq = np.concatenate([np.full(len(x), i) for i, x in enumerate(k)] or [[]])
        pos = np.concatenate([np.arange(len(x)) for x in k] or [[]])
        self.append(seq, pos, np.concatenate(k), np.concatenate(v), layer)
        return [O.page_rows(x).reshape(-1, self.Hkv, self.D) for x in k], [
            O.page_rows(x).reshape(-1, self.Hkv, self.D) for x in v]

    def append(self, seq, pos, k, v, layer=0, shift=0, pad=0):
        M, w = len(seq), self.Hkv * self.D
        rows = [np.zeros((M, w + pad), np.float16) for _ in "kv"]
        for r, x in zip(rows, (k, v)):
            r[:, :w] = x
        dk, dv = (dev(np.concatenate([np.zeros(shift, np.float16), r.reshape(-1)])) for r in rows)
        ds, dp = dev(seq, np.int32), dev(pos, np.int32)
        B.pipo_op_kv_pages_append(self.c(), layer, ds.ptr, dp.ptr, dk.ptr + 2 * shift, w + pad,
                                  dv.ptr + 2 * shift, w + pad, M)
        B.pipo_dev_synchronize()

    def read(self, seq, pos, layer=0, shift=0, pad=0, fill=7.0):
        M, w = len(seq), self.Hkv * self.D
        bufs = [dev(np.full(shift + M * (w + pad), fill, np.float16)) for _ in "kv"]
        ds, dp = dev(seq, np.int32), dev(pos, np.int32)
        B.pipo_op_kv_pages_read(self.c(), layer, ds.ptr, dp.ptr, bufs[0].ptr + 2 * shift, w + pad,
                                bufs[1].ptr + 2 * shift, w + pad, M)
        B.pipo_dev_synchronize()
        out = [b.to_array(np.float16, (shift + M * (w + pad),)) for b in bufs]
        for x in out:
            assert (x[:shift] == fill).all() and (x[shift:].reshape(M, -1)[:, w:] == fill).all()
        return [x[shift:].reshape(M, -1)[:, :w] for x in out]

    def bytes(self):
        return self.pool.to_array(np.uint8, (self.layers, self.n_pages, self.page))


def attend(c, q, rows, n_heads, lens=None, layer=0, split=True, shift=0, pad=0, max_q=None,
           max_len=None, behind=2, starts=None):
    """q [M][H * D] -> o [M + behind][H * D]; the rows behind keep 9"""
    M, w = q.shape[0], n_heads * c.D
    lens = c.lens if lens is None else lens
    starts = np.concatenate([[0], np.cumsum(rows)]) if starts is None else starts
    total = M + behind
    full = np.full((total, w + pad), 5, np.float16)
    full[:M, :w] = q
    z = np.zeros(shift, np.float16)
    dq = dev(np.concatenate([z, full.reshape(-1)]))
    do = dev(np.full(shift + total * (w + pad), 9, np.float16))
    ds, dl = dev(starts, np.int32), dev(lens, np.int32)
    max_q = max(rows) if max_q is None else max_q
    max_len = max(max(lens), 0) if max_len is None else max_len
    n = B.pipo_op_attn_pages_workspace_bytes(c.c(), n_heads, total, max_q, max_len) if split else 0
    ws = dev(np.full(max(n // 4, 1), np.nan, np.float32))
    B.pipo_op_attn_pages(c.c(), layer, dq.ptr + 2 * shift, w + pad, ds.ptr, dl.ptr, do.ptr + 2 * shift,
                         w + pad, n_heads, total, max_q, max_len, ws.ptr if n else None, n)
    B.pipo_dev_synchronize()
    out = do.to_array(np.float16, (shift + total * (w + pad),))
    assert (out[:shift] == 9).all()
    out = out[shift:].reshape(total, w + pad)
    assert (out[:, w:] == 9).all()
    return out[:, :w]


def want_attention(q, k, v, rows, lens, H, D):
    """(values, tolerance) of every row"""
    out, tol, at = [], [], 0
    for kk, vv, r, n in zip(k, v, rows, lens):
        if r == 0:
            continue
        x = q[at:at + r].reshape(r, H, D)
        n = min(n, len(kk))
        last = n - r + np.arange(r)
        seen = np.arange(n)[None] <= last[:, None]
        o = O.page_attention(x, kk[:n], vv[:n], seen)
        big = np.abs(vv[:n]).max() if n else 0.0
        step = 0.0
        if n:
            g = kk[:n].reshape(n, kk.shape[1], D // 64, 64)
            scale = (g.max(-1) - g.min(-1)).max() / 15
            qsum = np.abs(x.astype(np.float64)).reshape(r, H, D // 64, 64).sum(-1).max()
            step = 4 * 8 * 2.0 ** -25 * 272 * qsum * scale
        out.append(o.reshape(r, -1))
        tol.append(HALF * np.abs(o.reshape(r, -1)) + (HALF + step) * big + 2.0 ** -25)
        at += r
    return np.concatenate(out), np.concatenate(tol)


def check(got, want, tol, what):
    bad = ~(np.abs(got.astype(np.float64) - want) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])


def draw_rows(lens, width, rng, std=1.0):
    return [(rng.standard_normal((n, width)) * std).astype(np.float16) for n in lens]


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("M,H,Hkv,D,shift,pad", [
    (1, 1, 1, 128, 0, 0), (3, 6, 2, 64, 0, 8), (17, 5, 5, 128, 1, 3), (40, 8, 1, 64, 0, 0),
    (33, 32, 8, 128, 0, 16), (700, 40, 8, 128, 0, 0), (900, 12, 12, 64, 3, 1),
    (3700, 28, 8, 128, 0, 8), (7300, 30, 6, 64, 0, 0)])  # past the L2
@pytest.mark.parametrize("norm", [True, False])
def test_norm_rope(M, H, Hkv, D, shift, pad, norm):
    print(f"norm_rope M={M} H={H}/{Hkv} D={D} shift={shift} pad={pad} norm={norm}", flush=True)
    rng = np.random.default_rng(M + H)
    n_pos, eps, scale = 50, 1e-5, D ** -0.5
    ang = np.arange(n_pos)[:, None] * 10000.0 ** (-2 * np.arange(D // 2) / D)
    cs = np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)
    width = (H + 2 * Hkv) * D + pad
    x = (rng.standard_normal((M, width)) * 2).astype(np.float16)
    x[0] = 0                                          # a head of zeros stays zero
    gq, gk = (1 + 0.3 * rng.standard_normal((2, D))).astype(np.float16)
    pos = rng.integers(0, n_pos, M).astype(np.int32)
    if M > 4:
        pos[[1, 3, 4]] = -1, n_pos, np.iinfo(np.int32).max      # padding
    dx = dev(np.concatenate([np.zeros(shift, np.float16), x.reshape(-1)]))
    do = [dev(np.full(shift + M * (n * D + pad), 9, np.float16)) for n in (H, Hkv)]
    keep = dev(gq), dev(gk), dev(cs), dev(pos)
    q0 = dx.ptr + 2 * shift
    B.pipo_op_qk_norm_rope(q0, width, q0 + 2 * H * D, width, keep[0].ptr if norm else None,
                           keep[1].ptr if norm else None, keep[2].ptr, n_pos, keep[3].ptr,
                           do[0].ptr + 2 * shift, H * D + pad, do[1].ptr + 2 * shift, Hkv * D + pad, M,
                           H, Hkv, D, eps, scale)
    B.pipo_dev_synchronize()
    ok = (pos >= 0) & (pos < n_pos)
    outs = []
    for n, g, at, sc, buf in ((H, gq, 0, scale, do[0]), (Hkv, gk, H * D, 1.0, do[1])):
        got = buf.to_array(np.float16, (shift + M * (n * D + pad),))
        assert (got[:shift] == 9).all()
        got = got[shift:].reshape(M, n * D + pad)
        assert (got[:, n * D:] == 9).all() and (got[~ok] == 9).all()
        got = got[:, :n * D].reshape(M, n, D)[ok]
        src = x[ok, at:at + n * D].reshape(-1, n, D)
        want = O.norm_rope(src, g if norm else None, cs[pos[ok]], eps, sc)
        # fp32: the norm and the two products are within 16 steps of 2^-24 of |a| + |b|
        y = O.norm_rope(src, g if norm else None, np.stack([np.ones((ok.sum(), D // 2)),
                                                           np.zeros((ok.sum(), D // 2))], -1), eps, sc)
        y = np.abs(y).reshape(-1, n, 2, D // 2).sum(2, keepdims=True).repeat(2, 2).reshape(want.shape)
        check(got, want, HALF * np.abs(want) + 2.0 ** -20 * y + 2.0 ** -25, "norm_rope")
        outs.append(got)
    # in place over the fused rows: the same bits, v and padding rows untouched
    B.pipo_op_qk_norm_rope(q0, width, q0 + 2 * H * D, width, keep[0].ptr if norm else None,
                           keep[1].ptr if norm else None, keep[2].ptr, n_pos, keep[3].ptr, q0, width,
                           q0 + 2 * H * D, width, M, H, Hkv, D, eps, scale)
    B.pipo_dev_synchronize()
    y = dx.to_array(np.float16, (shift + M * width,))[shift:].reshape(M, width)
    assert np.array_equal(y[ok, :H * D].reshape(-1, H, D).view(np.uint16), outs[0].view(np.uint16))
    assert np.array_equal(y[ok, H * D:(H + Hkv) * D].reshape(-1, Hkv, D).view(np.uint16),
                          outs[1].view(np.uint16))
    assert np.array_equal(y[:, (H + Hkv) * D:], x[:, (H + Hkv) * D:])
    assert np.array_equal(y[~ok].view(np.uint16), x[~ok].view(np.uint16))


def test_norm_rope_one_norm_and_one_bad_head():
    """gamma of one of the two alone; a NaN stays in its head."""
    rng = np.random.default_rng(5)
    M, H, Hkv, D = 4, 3, 2, 128
    q, k = (rng.standard_normal((M, n, D)).astype(np.float16) for n in (H, Hkv))
    q[2, 1, 5] = np.nan
    g = (1 + 0.3 * rng.standard_normal(D)).astype(np.float16)
    cs = np.stack([np.cos(np.ones((1, D // 2))), np.sin(np.ones((1, D // 2)))], -1).astype(np.float32)
    bufs = dev(q), dev(k), dev(g), dev(cs), dev(np.zeros(M, np.int32)), DB(q.nbytes), DB(k.nbytes)
    p = [b.ptr for b in bufs]
    B.pipo_op_qk_norm_rope(p[0], H * D, p[1], Hkv * D, None, p[2], p[3], 1, p[4], p[5], H * D, p[6],
                           Hkv * D, M, H, Hkv, D, 1e-6, 1.0)
    B.pipo_dev_synchronize()
    cs = np.repeat(cs, M, 0)
    for x, gamma, buf in ((q, None, bufs[5]), (k, g, bufs[6])):
        got, want = buf.to_array(np.float16, x.shape), O.norm_rope(x, gamma, cs, 1e-6, 1.0)
        nan = np.isnan(x).any(-1)
        assert np.isfinite(got[~nan]).all()
        check(got[~nan], want[~nan], HALF * np.abs(want[~nan]) + 2.0 ** -19 * 8, "one norm")


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("lens,Hkv,D,ps,shift,pad", [
    ([1], 1, 64, 16, 0, 0), ([5, 0, 17], 3, 128, 16, 0, 8), ([33, 64, 1, 100], 8, 128, 64, 0, 0),
    ([40, 3], 2, 64, 32, 1, 3), ([300], 5, 128, 256, 0, 0), ([129, 128, 127], 1, 128, 128, 5, 0),
    ([2500, 101, 7], 51, 64, 64, 0, 0), ([5050, 51], 13, 128, 32, 0, 8), ([2700], 51, 64, 16, 3, 1)])
def test_append_and_read(lens, Hkv, D, ps, shift, pad):
    print(f"append lens={lens} Hkv={Hkv} D={D} ps={ps} shift={shift} pad={pad}", flush=True)
    rng = np.random.default_rng(sum(lens) + ps)
    c = Cache(lens, Hkv, D, ps, rng, layers=2, fill=0xA5)
    seq = np.concatenate([np.full(n, i) for i, n in enumerate(lens)])
    pos = np.concatenate([np.arange(n) for n in lens])
    k, v = (rng.standard_normal((len(seq), Hkv * D)) * 3).astype(np.float16), rng.standard_normal(
        (len(seq), Hkv * D)).astype(np.float16)
    k[0, :64] = 1.5                                     # a group of one value: scale 0
    v[0] = 0
    k[-1, 3], k[-1, 64 * (Hkv * D // 64) - 1], v[-1, 7], v[-1, 9] = np.inf, -np.inf, np.nan, 65504
    order = rng.permutation(len(seq))                   # any order of rows
    if len(seq) > 1000:                                 # and, of a prompt, their own
        order = np.arange(len(seq))
    half = len(order) // 2
    for part in (order[:half], order[half:]):           # two calls: neighbours in a byte's word
        c.append(seq[part], pos[part], k[part], v[part], layer=1, shift=shift, pad=pad)
    got = c.read(seq, pos, layer=1, shift=shift, pad=pad)
    for x, y in zip((k, v), got):
        want = O.page_rows(x).astype(np.float32).astype(np.float16)
        assert np.array_equal(want, y)
    # nothing else was written: the other layer, unused pages, unused positions
    b = c.bytes()
    assert (b[0] == 0xA5).all()
    used = {int(p) for row, n in zip(c.table, lens) for p in row[:-(-n // ps)]}
    assert all((b[1, p] == 0xA5).all() for p in range(c.n_pages) if p not in used)
    written = (b[1] != 0xA5).sum()
    assert written <= len(seq) * Hkv * 2 * 9 * D // 16


def test_append_skips_rows_without_a_slot():
    rng = np.random.default_rng(2)
    c = Cache([40, 20], 2, 128, 16, rng, fill=0xA5)
    c.set_table(np.array([[c.table[0, 0], -1, c.n_pages], [c.table[1, 0], 1 << 30, -(1 << 31)]], np.int32))
    c.width = 3
    rows = [(-1, 0), (2, 0), (1 << 30, 3), (0, -1), (0, 16), (0, 47), (0, 48), (1, 1 << 30), (1, 17), (1, 33),
            (0, 2 ** 31 - 1), (-(2 ** 31), -(2 ** 31))]
    seq, pos = np.array(rows + [(0, 3)]).T
    x = rng.standard_normal((len(seq), 256)).astype(np.float16)
    c.append(seq, pos, x, x)
    assert 0 < (c.bytes() != 0xA5).sum() <= 2 * 2 * 72
    k, v = c.read(seq, pos)
    assert (k[:-1] == 7).all() and (v[:-1] == 7).all()
    want = O.page_rows(x[-1:]).astype(np.float32).astype(np.float16)
    assert np.array_equal(k[-1:], want) and np.array_equal(v[-1:], want)


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("lens,rows,H,Hkv,D,ps", [
    ([1], [1], 1, 1, 64, 16), ([1, 15, 16, 17], [1] * 4, 4, 4, 128, 16),
    ([31, 32, 33, 0, 100], [1] * 5, 8, 2, 128, 32), ([130, 7], [1, 1], 6, 2, 64, 64),
    ([257, 255, 256], [1] * 3, 10, 2, 128, 256), ([40, 90], [1, 1], 7, 1, 128, 128),
    ([65, 20], [1, 1], 32, 2, 64, 16), ([50, 300], [1, 1], 71, 1, 64, 64),
    ([20, 33, 64], [2, 0, 3], 8, 2, 128, 32), ([70, 16, 5], [5, 16, 5], 12, 4, 128, 16),
    ([200, 100], [17, 100], 4, 4, 64, 64), ([150, 330, 40], [130, 1, 40], 8, 2, 128, 64),
    ([700, 600], [300, 257], 4, 1, 128, 32), ([333], [333], 3, 3, 64, 16),
    ([530, 90, 260, 33], [1, 90, 129, 2], 10, 2, 128, 64)])
@pytest.mark.parametrize("shift,pad", [(0, 0), (1, 3)])
def test_attention(lens, rows, H, Hkv, D, ps, shift, pad):
    print(f"attn lens={lens} rows={rows} H={H}/{Hkv} D={D} ps={ps} shift={shift}", flush=True)
    rng = np.random.default_rng(sum(lens) + H)
    c = Cache(lens, Hkv, D, ps, rng, layers=2)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng), layer=1)
    q = (rng.standard_normal((sum(rows), H * D)) * 1.5 * D ** -0.5).astype(np.float16)
    got = attend(c, q, rows, H, layer=1, shift=shift, pad=pad)
    want, tol = want_attention(q, k, v, rows, lens, H, D)
    check(got[:len(q)], want, tol, "attention")
    assert (got[len(q):] == 9).all()
    if want.size > 500:
        # all in all: the last rounding (rms 2^-11 / root 3) and one of the weights
        err = np.linalg.norm(got[:len(q)].astype(np.float64) - want) / np.linalg.norm(want)
        assert err <= np.sqrt(2 / 3) * HALF * 1.1, err


@pytest.mark.parametrize("n", [64, 65, 200])
def test_attention_of_many_sequences(n):
    """Prompts' pieces among single rows, over the counts at which workgroups find
    their sequence in another way; columns at 64, 65, 128 and 129."""
    print(f"attn sequences n={n}", flush=True)
    rng = np.random.default_rng(n)
    H, Hkv, D = 4, 2, 64
    rows = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 32, 33, 64, 65, 90], n)]
    lens = [r + int(x) for r, x in zip(rows, rng.integers(0, 60, n))]
    c = Cache(lens, Hkv, D, 16, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((sum(rows), H * D)) * 1.5 * D ** -0.5).astype(np.float16)
    got = attend(c, q, rows, H)
    want, tol = want_attention(q, k, v, rows, lens, H, D)
    check(got[:len(q)], want, tol, "many sequences")
    assert (got[len(q):] == 9).all()


def test_attention_of_many_column_tiles():
    """More column tiles than three a CU: one team a workgroup."""
    rng = np.random.default_rng(14)
    n, H, Hkv, D = 12, 64, 8, 64
    rows = [130] * (n - 1) + [129]
    lens = [r + int(x) for r, x in zip(rows, rng.integers(0, 90, n))]
    c = Cache(lens, Hkv, D, 32, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((sum(rows), H * D)) * 1.5 * D ** -0.5).astype(np.float16)
    got = attend(c, q, rows, H)
    want, tol = want_attention(q, k, v, rows, lens, H, D)
    check(got[:len(q)], want, tol, "many tiles")


@pytest.mark.parametrize("lens,rows,H,Hkv,split", [
    ([9000], [1], 2, 1, False),              # eight waves
    ([4500] + [1] * 511, [1] * 512, 2, 1, True),    # four waves
    ([1500] + [1] * 1100, [1] * 1101, 2, 1, True),  # two
    ([300] + [2] * 1100, [1] * 1101, 2, 1, True),
    ([1500, 1100, 1061, 1089], [2, 4, 1, 3], 2, 1, False), ([2200, 1], [1, 1], 8, 1, False),
    ([9000], [40], 4, 1, False), ([40000], [17], 8, 1, False), ([40000], [1], 2, 1, True)])
def test_attention_past_a_waves_page_indices(lens, rows, H, Hkv, split):
    """Waves hold the pages of 32 (64) of their blocks at a time."""
    print(f"attn long lens={lens[:2]} rows={rows[:2]} split={split}", flush=True)
    rng = np.random.default_rng(lens[0])
    D = 64
    c = Cache(lens, Hkv, D, 16, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((sum(rows), H * D)) * 2 * D ** -0.5).astype(np.float16)
    got = attend(c, q, rows, H, split=split)
    want, tol = want_attention(q, k, v, rows, lens, H, D)
    check(got[:len(q)], want, tol, "long")
    err = np.linalg.norm(got[:len(q)].astype(np.float64) - want) / np.linalg.norm(want)
    assert err <= np.sqrt(2 / 3) * HALF * 1.1, err


@pytest.mark.parametrize("rows", [1, 4, 60])
def test_attention_with_holes_in_a_long_row(rows):
    """Table entries that are no pages here and there in 1500 keys."""
    rng = np.random.default_rng(15)
    lens, H, Hkv, D, ps = [1500], 2, 1, 128, 16
    c = Cache(lens, Hkv, D, ps, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((rows, H * D)) * 0.1).astype(np.float16)
    holes = [0, 7, 8, 33, 34, 35, 36, 61, 92]
    t = c.table.copy()
    t[0, holes] = [-1, c.n_pages, 1 << 30, -5, -1, -1, c.n_pages + 7, -(1 << 31), -1]
    c.set_table(t)
    seen = np.arange(1500)[None] <= (1500 - rows + np.arange(rows))[:, None]
    for i in holes:
        seen[:, i * ps:(i + 1) * ps] = False
    o = O.page_attention(q.reshape(rows, H, D), k[0], v[0], seen).reshape(rows, -1)
    for split in (False, True):
        got = attend(c, q, [rows], H, split=split)[:rows]
        check(got, o, HALF * np.abs(o) + 2 * HALF * np.abs(v[0]).max(), "holes")


@pytest.mark.parametrize("lens,rows,H,Hkv,D,split", [
    ([400, 30, 1, 90], [150, 1, 1, 3], 8, 2, 128, True),      # both kinds in one launch
    ([400, 30, 1, 90], [150, 1, 1, 3], 8, 2, 64, False),
    ([1600, 1300, 2], [80, 1, 2], 8, 2, 128, True),           # both in parts
    ([900, 30], [300, 1], 8, 1, 128, True),                   # one after the other
    ([900, 30], [300, 1], 8, 1, 64, False),
    ([1500] + [3, 1100] * 64, [70] + [1] * 128, 2, 2, 128, True),   # 64 keys at a time
    ([1500] + [3, 1100] * 64, [70] + [1, 4] * 64, 4, 2, 64, True),
    ([700] * 25 + [40] * 7, [600] * 25 + [2] * 7, 32, 8, 64, True)])  # tiles for all CUs
def test_attention_of_many_and_few_rows(lens, rows, H, Hkv, D, split):
    print(f"attn both lens={lens[:4]} rows={rows[:4]} D={D} split={split}", flush=True)
    rng = np.random.default_rng(sum(lens) + D)
    c = Cache(lens, Hkv, D, 16, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((sum(rows), H * D)) * 2 * D ** -0.5).astype(np.float16)
    got = attend(c, q, rows, H, split=split, behind=3)
    want, tol = want_attention(q, k, v, rows, lens, H, D)
    check(got[:len(q)], want, tol, "both")
    assert (got[len(q):] == 9).all()


def test_attention_of_equal_shares_that_are_not():
    """As many rows as sequences times max_q, and sequences of fewer rows behind
    which some belong to none."""
    rng = np.random.default_rng(13)
    H, Hkv, D, rows, lens = 8, 2, 128, [40, 1, 0, 12], [100, 300, 20, 12]
    c = Cache(lens, Hkv, D, 32, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((sum(rows), H * D)) * 0.1).astype(np.float16)
    got = attend(c, q, rows, H, behind=4 * 40 - sum(rows))
    want, tol = want_attention(q, k, v, rows, lens, H, D)
    check(got[:len(q)], want, tol, "shares")
    assert (got[len(q):] == 9).all()


@pytest.mark.parametrize("lens,rows,H,Hkv,D,ps", [
    ([4000], [1], 8, 2, 128, 64), ([3001, 1, 0, 2600], [1, 1, 1, 1], 4, 4, 64, 16),
    ([2100, 5000], [3, 1], 8, 1, 128, 128), ([3000, 700], [100, 1], 4, 1, 128, 32),
    ([2500], [2500], 2, 1, 64, 64)])
def test_attention_splits(lens, rows, H, Hkv, D, ps):
    """Few sequences over many keys: with and without the workspace."""
    print(f"attn splits lens={lens} rows={rows} H={H}/{Hkv} D={D}", flush=True)
    rng = np.random.default_rng(sum(lens))
    c = Cache(lens, Hkv, D, ps, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((sum(rows), H * D)) * 2 * D ** -0.5).astype(np.float16)
    want, tol = want_attention(q, k, v, rows, lens, H, D)
    for split in (True, False):
        got = attend(c, q, rows, H, split=split)
        check(got[:len(q)], want, tol, "splits")
        assert (got[len(q):] == 9).all()
        assert np.array_equal(attend(c, q, rows, H, split=split), got)      # the same bits again


def test_attention_of_no_keys_is_zero():
    rng = np.random.default_rng(3)
    lens, rows, H, Hkv, D = [0, 3, 2, 40], [2, 5, 2, 100], 8, 2, 128
    c = Cache(lens, Hkv, D, 16, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((sum(rows), H * D)) * 0.2).astype(np.float16)
    got = attend(c, q, rows, H)
    want, tol = want_attention(q, k, v, rows, lens, H, D)
    assert (want[:4] == 0).all() and (want[9:69] == 0).all()      # rows before the first key
    check(got[:len(q)], want, tol, "no keys")
    assert (got[:4] == 0).all() and (got[9:69] == 0).all()


@pytest.mark.parametrize("rows", [[1, 1, 1], [60, 1, 70]])
def test_attention_with_wrong_lengths_starts_and_pages(rows):
    """Lengths above max_len count as max_len, negative ones as 0; keys on an
    entry that is no page are not seen; starts are kept inside the rows."""
    print(f"attn wrong rows={rows}", flush=True)
    rng = np.random.default_rng(4)
    lens, H, Hkv, D, ps = [100, 90, 80], 8, 2, 64, 16
    c = Cache(lens, Hkv, D, ps, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((sum(rows), H * D)) * 0.2).astype(np.float16)
    got = attend(c, q, rows, H, lens=[1 << 30, -5, 80], max_len=96)
    want, tol = want_attention(q, k, v, rows, [96, 0, 80], H, D)
    check(got[:len(q)], want, tol, "lengths")
    t = c.table.copy()
    t[0, 1], t[0, 3], t[2] = -1, c.n_pages, 1 << 30
    c.set_table(t)
    got = attend(c, q, rows, H)
    at = 0
    for i, r in enumerate(rows):
        seen = np.arange(lens[i])[None] <= (lens[i] - r + np.arange(r))[:, None]
        if i == 0:
            seen[:, 16:32] = seen[:, 48:64] = False
        if i == 2:
            seen[:] = False
        o = O.page_attention(q[at:at + r].reshape(r, H, D), k[i], v[i], seen).reshape(r, -1)
        check(got[at:at + r], o, HALF * np.abs(o) + 2 * HALF * np.abs(v[i]).max(), "pages")
        at += r
    for most in (1, 17, 65):          # rows past the max_q-th of a sequence are left
        got, at = attend(c, q, rows, H, max_q=most), 0
        for r in rows:
            assert (got[at + most:at + r] == 9).all() and (got[at:at + min(r, most)] != 9).any()
            at += r
    total = sum(rows)
    for starts in ([-7, rows[0], total, 1 << 30], [0, 5, 3, total], [1 << 30] * 4):
        got = attend(c, q, rows, H, starts=starts, max_q=max(rows))
        assert np.isfinite(got).all()


@pytest.mark.parametrize("rows", [[1], [80]])
@pytest.mark.parametrize("gap", [14, 20, 23.5])
def test_attention_small_probabilities(rows, gap):
    """A key of value 0 in every 32 and a long tail `gap` below its score, of
    value 1000 or 50000: the output is the tail's alone.  Each of its weights
    has 11 bits, those of the output, even there (its own half 2^-11); exp2 of
    an argument of 35 in fp32 adds 2^-19, the sums of 4096 keys 2^-12 of the
    biased codes' 2^-24 * 16 / c, well under 2^-19."""
    print(f"attn tail rows={rows} gap={gap}", flush=True)
    rng = np.random.default_rng(6)
    T, H, Hkv, D = 4096, 8, 2, 128
    c = Cache([T], Hkv, D, 64, rng)
    k, v = np.zeros((T, Hkv * D), np.float16), np.zeros((T, Hkv * D), np.float16)
    k[:, ::D] = -gap
    k[::32, ::D] = 0
    v[:] = 1000 if gap < 20 else 50000
    v[::32] = 0
    k, v = c.fill([k], [v])
    q = np.zeros((rows[0], H * D), np.float16)
    q[:, ::D] = 1
    for split in (True, False):
        got = attend(c, q, rows, H, split=split)[:rows[0]].astype(np.float64)
        want, _ = want_attention(q, k, v, rows, [T], H, D)
        assert want.min() > 2.0 ** -14
        assert np.abs(got / want - 1).max() <= 2 * HALF + 2 * 2.0 ** -19


@pytest.mark.parametrize("rows", [1, 90])
@pytest.mark.parametrize("size", [2.0 ** -20, 1e-4, 1.0, 300.0, 65504.0])
def test_attention_values_of_every_size(rows, size):
    """Values from subnormal halves to the largest, next to keys of their own
    scale; mixed sizes in one cache."""
    print(f"attn size={size} rows={rows}", flush=True)
    rng = np.random.default_rng(7)
    lens, H, Hkv, D = [150, 97], 4, 2, 64
    c = Cache(lens, Hkv, D, 32, rng)
    vals = [np.clip(x.astype(np.float64) / 3 * size, -65504, 65504).astype(np.float16)
            for x in draw_rows(lens, Hkv * D, rng)]
    vals[1][:50] = draw_rows([50], Hkv * D, rng)[0]         # other sizes before these
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), vals)
    q = (rng.standard_normal((2 * rows, H * D)) * 0.2).astype(np.float16)
    got = attend(c, q, [rows, rows], H)[:2 * rows]
    want, tol = want_attention(q, k, v, [rows, rows], lens, H, D)
    check(got, want, tol, "sizes")
    assert np.isfinite(got).all()


@pytest.mark.parametrize("rows", [1, 70])
def test_attention_large_scores(rows):
    """Scores of hundreds: one key takes all the weight."""
    rng = np.random.default_rng(8)
    lens, H, Hkv, D = [200], 4, 2, 128
    c = Cache(lens, Hkv, D, 64, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng, 8), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((rows, H * D)) * 4).astype(np.float16)
    got = attend(c, q, [rows], H)[:rows]
    want, tol = want_attention(q, k, v, [rows], lens, H, D)
    check(got, want, tol, "large scores")


@pytest.mark.parametrize("rows", [1, 70])
def test_attention_keeps_a_bad_query_to_itself(rows):
    rng = np.random.default_rng(9)
    lens, H, Hkv, D = [120], 4, 1, 128
    c = Cache(lens, Hkv, D, 64, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((rows, H * D)) * 0.1).astype(np.float16)
    bad = q.copy()
    bad[0, 5], bad[-1, D + 1] = np.nan, np.inf
    a, b = attend(c, q, [rows], H)[:rows], attend(c, bad, [rows], H)[:rows]
    hit = np.zeros((rows, H), bool)
    hit[0, 0] = hit[-1, 1] = True
    hit = hit.repeat(D, 1)
    assert np.array_equal(a[~hit], b[~hit]) and np.isnan(b[0, :D]).all()


# ---------------------------------------------------------------------------
def tables(rng, n, width, ps, n_pages, share=True):
    """A table over distinct pages, some rows sharing a prefix"""
    order, at = rng.permutation(n_pages), 0
    t, lens = rng.integers(-3, n_pages + 3, (n, width)).astype(np.int32), np.zeros(n, np.int32)
    for i in range(n):
        lens[i] = rng.integers(0, width * ps + 1) if rng.random() < 0.8 else 0
        need = -(-int(lens[i]) // ps)
        if at + need > n_pages:
            lens[i] = need = 0
        t[i, :need] = order[at:at + need]
        at += need
        if share and i and lens[i] >= ps and lens[i - 1] >= ps and rng.random() < 0.3:
            t[i, 0] = t[i - 1, 0]
    return t, lens


SHAPES = [(1, 1, 16, 1), (3, 4, 16, 9), (20, 7, 64, 100), (100, 30, 32, 1500), (17, 200, 256, 4001),
          (2048, 3, 16, 5000), (40, 900, 128, 40000)]


@pytest.mark.parametrize("n,width,ps,n_pages", SHAPES)
@pytest.mark.parametrize("inplace", [False, True])
def test_resize(n, width, ps, n_pages, inplace):
    print(f"resize n={n} width={width} ps={ps} pages={n_pages}", flush=True)
    rng = np.random.default_rng(n + width)
    t, lens = tables(rng, n, width, ps, n_pages)
    kinds = [("grow", np.minimum(lens + 1, width * ps)), ("keep", np.full(n, -1)), ("free", np.zeros(n)),
             ("mixed", np.where(rng.random(n) < 0.4, rng.integers(-2, width * ps // 2 + 1, n), -1)),
             ("all", np.full(n, width * ps)), ("past", np.where(np.arange(n) == n - 1, width * ps + 1, -1)),
             ("far", np.full(n, 2 ** 31 - 1))]
    for what, want in kinds:
        want = want.astype(np.int32)
        a, b, lack = O.resize(t, lens.tolist(), want.tolist(), n_pages, ps)
        dt, dl, dw, dm = dev(t), dev(lens), dev(want), dev(np.full(1, 77, np.int32))
        ot, ol = (dt, dl) if inplace else (DB(t.nbytes), DB(lens.nbytes))
        B.pipo_op_kv_pages_resize(dt.ptr, dl.ptr, dw.ptr, ot.ptr, ol.ptr, width, n, n_pages, ps, dm.ptr)
        B.pipo_dev_synchronize()
        if what != "far":         # (there the count of pages lacking is only known to be positive)
            assert dm.to_array(np.int32, (1,))[0] == lack, what
        assert (dm.to_array(np.int32, (1,))[0] > 0) == (lack > 0)
        assert np.array_equal(ol.to_array(np.int32, (n,)), b), what
        got = ot.to_array(np.int32, t.shape)
        held = np.arange(width)[None] < -(-b // ps)[:, None]
        assert np.array_equal(np.where(held, got, -1), a), what
        assert (got[~held] == -1).all(), what


@pytest.mark.parametrize("n,width,ps,n_pages", SHAPES)
def test_fork(n, width, ps, n_pages):
    print(f"fork n={n} width={width} ps={ps} pages={n_pages}", flush=True)
    rng = np.random.default_rng(n + width + 1)
    t, lens = tables(rng, n, width, ps, n_pages // 2 + 1)
    for n_out in (1, n, min(2 * n, 2048)):
        for parent in (rng.integers(0, n, n_out), rng.integers(-2, n + 2, n_out), np.full(n_out, -1),
                       np.zeros(n_out), np.arange(n_out) // 2):
            parent = parent.astype(np.int32)
            a, b, pairs, lack = O.fork(t, lens.tolist(), parent.tolist(), n_pages, ps)
            dt, dl, dp = dev(t), dev(lens), dev(parent)
            ot, ol = dev(np.full((n_out, width), 55, np.int32)), dev(np.full(n_out, 55, np.int32))
            opairs, cnt = dev(np.full((n_out, 2), 55, np.int32)), dev(np.full(2, 55, np.int32))
            B.pipo_op_kv_pages_fork(dt.ptr, dl.ptr, n, dp.ptr, ot.ptr, ol.ptr, n_out, width, n_pages, ps,
                                    opairs.ptr, cnt.ptr, cnt.ptr + 4)
            B.pipo_dev_synchronize()
            assert cnt.to_array(np.int32, (2,)).tolist() == [len(pairs), lack]
            got = opairs.to_array(np.int32, (n_out, 2))
            assert [tuple(x) for x in got[:len(pairs)]] == pairs and (got[len(pairs):] == 55).all()
            gt, gl = ot.to_array(np.int32, (n_out, width)), ol.to_array(np.int32, (n_out,))
            if lack:
                assert (gt == 55).all() and (gl == 55).all()
            else:
                assert np.array_equal(gt, a) and np.array_equal(gl, b)


@pytest.mark.parametrize("n,width,ps,n_pages", SHAPES)
@pytest.mark.parametrize("inplace", [False, True])
def test_compact(n, width, ps, n_pages, inplace):
    print(f"compact n={n} width={width} ps={ps} pages={n_pages}", flush=True)
    rng = np.random.default_rng(n + width + 2)
    t, lens = tables(rng, n, width, ps, n_pages)
    for keep in (1.0, 0.5, 0.0):
        ln = np.where(rng.random(n) <= keep, lens, 0).astype(np.int32)
        a, pairs = O.compact(t, ln.tolist(), n_pages, ps)
        dt, dl = dev(t), dev(ln)
        ot = dt if inplace else DB(t.nbytes)
        opairs, cnt = dev(np.full((n_pages // 2 + 1, 2), 55, np.int32)), dev(np.full(1, 55, np.int32))
        B.pipo_op_kv_pages_compact(dt.ptr, dl.ptr, ot.ptr, width, n, n_pages, ps, opairs.ptr, cnt.ptr)
        B.pipo_dev_synchronize()
        assert cnt.to_array(np.int32, (1,))[0] == len(pairs) <= n_pages // 2
        got = opairs.to_array(np.int32, (n_pages // 2 + 1, 2))
        assert [tuple(x) for x in got[:len(pairs)]] == pairs and (got[len(pairs):] == 55).all()
        assert np.array_equal(ot.to_array(np.int32, t.shape), a)


@pytest.mark.parametrize("n_pages", [(1 << 20) - 1, 1 << 20])
def test_tables_of_the_largest_pool(n_pages):
    """Pages at the end of the largest pool; resize finds the few free ones."""
    rng = np.random.default_rng(1)
    width, ps = 1 << 10, 16
    n = n_pages // width
    t = rng.permutation(n_pages)[:n * width].reshape(n, width).astype(np.int32)
    lens = np.full(n, width * ps, np.int32)
    lens[5] = 0
    dt, dl = dev(t), dev(lens)
    ot, ol, m = DB(t.nbytes), DB(lens.nbytes), dev(np.zeros(1, np.int32))
    want = np.full(n, -1, np.int32)
    want[5] = 3 * ps
    dw = dev(want)
    B.pipo_op_kv_pages_resize(dt.ptr, dl.ptr, dw.ptr, ot.ptr, ol.ptr, width, n, n_pages, ps, m.ptr)
    B.pipo_dev_synchronize()
    a, b, lack = O.resize(t, lens.tolist(), want.tolist(), n_pages, ps)
    assert np.array_equal(ot.to_array(np.int32, t.shape), a) and lack == 0
    opairs, cnt = DB(n_pages * 4), dev(np.zeros(1, np.int32))
    B.pipo_op_kv_pages_compact(ot.ptr, ol.ptr, ot.ptr, width, n, n_pages, ps, opairs.ptr, cnt.ptr)
    B.pipo_dev_synchronize()
    c, pairs = O.compact(a, b.tolist(), n_pages, ps)
    assert cnt.to_array(np.int32, (1,))[0] == len(pairs)
    assert np.array_equal(ot.to_array(np.int32, t.shape), c)


@pytest.mark.parametrize("Hkv,D,ps,layers", [(1, 64, 16, 1), (3, 128, 32, 3), (8, 128, 64, 2)])
def test_copy(Hkv, D, ps, layers):
    rng = np.random.default_rng(Hkv)
    c = Cache([ps] * 8, Hkv, D, ps, rng, layers=layers, extra=13)
    x = rng.integers(0, 256, (layers, c.n_pages, c.page)).astype(np.uint8)
    c.pool = dev(x)
    pairs = np.array([(3, 5), (3, 6), (-1, 7), (4, -1), (c.n_pages, 8), (9, 1 << 30), (10, 10), (11, 12)],
                     np.int32)
    dp = dev(pairs)
    for count, most in ((0, 8), (-3, 8), (2, 8), (8, 8), (1 << 30, 8), (8, 1)):
        c.pool = dev(x)
        n = dev(np.array([count], np.int32))
        B.pipo_op_kv_pages_copy(c.c(), dp.ptr, n.ptr, most)
        B.pipo_dev_synchronize()
        want = x.copy()
        for a, b in pairs[:min(max(count, 0), most)]:
            if 0 <= a < c.n_pages and 0 <= b < c.n_pages:
                want[:, b] = x[:, a]
        assert np.array_equal(c.bytes(), want), (count, most)


# ---------------------------------------------------------------------------
def test_a_batch_from_prompts_through_beams():
    """The calls as a serving loop makes them: prompts of different lengths in
    two pieces, tokens one by one, beams forked, sequences freed, the pool
    compacted, and on; every step's attention against 64 bits."""
    rng = np.random.default_rng(11)
    L, H, Hkv, D, ps, n, width, n_pages = 2, 8, 2, 128, 16, 6, 12, 64
    page = B.pipo_kv_page_bytes(ps, Hkv, D)
    pool = dev(np.full(L * n_pages * page, 255, np.uint8))
    table, lens = dev(np.full((n, width), -1, np.int32)), dev(np.zeros(n, np.int32))
    table2, lens2 = DB(n * width * 4), DB(n * 4)
    cnt, pairs = dev(np.zeros(4, np.int32)), DB(max(n, n_pages // 2) * 8)
    ang = np.arange(width * ps)[:, None] * 10000.0 ** (-2 * np.arange(D // 2) / D)
    cs = np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)
    dcs = dev(cs)
    gq, gk = (1 + 0.2 * rng.standard_normal((2, D))).astype(np.float16)
    dgq, dgk = dev(gq), dev(gk)
    ref = [[[], []] for _ in range(n)]      # values [layer] -> (k, v) rows of each sequence
    ref = [[([], []) for _ in range(L)] for _ in range(n)]
    length = [0] * n

    def cache():
        return B.PipoKvPages(pool.ptr, n_pages * page, table.ptr, width, L, n_pages, ps, Hkv, D, n)

    def step(rows):
        want = np.array([length[i] + r if r else -1 for i, r in enumerate(rows)], np.int32)
        dw = dev(want)
        B.pipo_op_kv_pages_resize(table.ptr, lens.ptr, dw.ptr, table.ptr, lens.ptr, width, n, n_pages, ps,
                                  cnt.ptr)
        B.pipo_dev_synchronize()
        assert cnt.to_array(np.int32, (4,))[0] == 0
        seq = np.repeat(np.arange(n), rows).astype(np.int32)
        pos = np.concatenate([length[i] + np.arange(r) for i, r in enumerate(rows)]).astype(np.int32)
        M = len(seq)
        for i, r in enumerate(rows):
            length[i] += r
        assert lens.to_array(np.int32, (n,)).tolist() == length
        dseq, dpos, dstart = dev(seq), dev(pos), dev(np.concatenate([[0], np.cumsum(rows)]), np.int32)
        for layer in range(L):
            qkv = rng.standard_normal((M, (H + 2 * Hkv) * D)).astype(np.float16)
            x, ld = dev(qkv), (H + 2 * Hkv) * D
            k, v = x.ptr + 2 * H * D, x.ptr + 2 * (H + Hkv) * D
            B.pipo_op_qk_norm_rope(x.ptr, ld, k, ld, dgq.ptr, dgk.ptr, dcs.ptr, width * ps, dpos.ptr,
                                   x.ptr, ld, k, ld, M, H, Hkv, D, 1e-5, D ** -0.5)
            B.pipo_op_kv_pages_append(cache(), layer, dseq.ptr, dpos.ptr, k, ld, v, ld, M)
            o = dev(np.zeros((M, H * D), np.float16))
            nb = B.pipo_op_attn_pages_workspace_bytes(cache(), H, M, max(rows), max(length))
            ws = DB(nb)
            B.pipo_op_attn_pages(cache(), layer, x.ptr, ld, dstart.ptr, lens.ptr, o.ptr, H * D, H, M,
                                 max(rows), max(length), ws.ptr, nb)
            B.pipo_dev_synchronize()
            y = x.to_array(np.float16, qkv.shape)
            for a, b, g, sc, heads in ((0, H, gq, D ** -0.5, H), (H, H + Hkv, gk, 1.0, Hkv)):
                w = O.norm_rope(qkv[:, a * D:b * D].reshape(M, heads, D), g, cs[pos], 1e-5, sc)
                check(y[:, a * D:b * D].reshape(w.shape), w, HALF * np.abs(w) + 2.0 ** -18, "norm")
            got, at = o.to_array(np.float16, (M, H * D)), 0
            for i, r in enumerate(rows):
                if not r:
                    continue
                for c, base in ((0, H), (1, H + Hkv)):
                    new = y[at:at + r, base * D:(base + Hkv) * D]
                    ref[i][layer][c].extend(O.page_rows(new).reshape(r, Hkv, D))
                kk, vv = (np.array(t) for t in ref[i][layer])
                want_o, tol = want_attention(y[at:at + r, :H * D], [kk], [vv], [r], [length[i]], H, D)
                check(got[at:at + r], want_o, tol, (i, layer))
                at += r

    step([40, 0, 17, 1, 33, 16])
    step([25, 5, 0, 30, 1, 1])
    for _ in range(3):
        step([1] * n)
    parent = [0, 0, 2, 2, 0, 5]
    dp = dev(parent, np.int32)
    B.pipo_op_kv_pages_fork(table.ptr, lens.ptr, n, dp.ptr, table2.ptr, lens2.ptr, n, width, n_pages, ps,
                            pairs.ptr, cnt.ptr + 4, cnt.ptr + 8)
    table, table2, lens, lens2 = table2, table, lens2, lens
    B.pipo_op_kv_pages_copy(cache(), pairs.ptr, cnt.ptr + 4, n)
    ref = [[(list(a), list(b)) for a, b in ref[p]] for p in parent]
    length = [length[p] for p in parent]
    for _ in range(2):
        step([1, 1, 0, 2, 1, 3])
    free = dev([0, -1, -1, 0, -1, -1], np.int32)
    B.pipo_op_kv_pages_resize(table.ptr, lens.ptr, free.ptr, table.ptr, lens.ptr, width, n, n_pages, ps,
                              cnt.ptr)
    for i in (0, 3):
        ref[i], length[i] = [([], []) for _ in range(L)], 0
    B.pipo_op_kv_pages_compact(table.ptr, lens.ptr, table.ptr, width, n, n_pages, ps, pairs.ptr,
                               cnt.ptr + 4)
    B.pipo_op_kv_pages_copy(cache(), pairs.ptr, cnt.ptr + 4, n_pages // 2)
    B.pipo_dev_synchronize()
    t = table.to_array(np.int32, (n, width))
    used = {int(p) for i in range(n) for p in t[i, :-(-length[i] // ps)]}
    assert used == set(range(len(used)))
    step([20, 1, 1, 0, 1, 70])
    step([1] * n)


class Hip:
    """The HIP runtime that the library itself runs on, for streams and graphs."""

    def __init__(self):
        B.lib()
        path = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line)
        self.lib = ctypes.CDLL(path)

    def __call__(self, name, *args):
        assert getattr(self.lib, name)(*args) == 0, name

    def stream(self):
        s = ctypes.c_void_p()
        self("hipStreamCreate", ctypes.byref(s))
        return s

    def capture(self, stream, work):
        g, e = ctypes.c_void_p(), ctypes.c_void_p()
        self("hipStreamBeginCapture", stream, 0)
        work()
        self("hipStreamEndCapture", stream, ctypes.byref(g))
        self("hipGraphInstantiate", ctypes.byref(e), g, None, None, ctypes.c_size_t(0))
        return e


def test_streams_and_graphs():
    """Two decode steps captured into graphs on a stream of their own, each with
    a workspace, replayed in turn with other rows and lengths; each replay
    against 64 bits and against the same attention called eagerly."""
    hip = Hip()
    rng = np.random.default_rng(12)
    n, H, Hkv, D, ps, top = 3, 8, 2, 128, 32, 2000
    length = [1500, 3, 700]
    width = top // ps + 1
    n_pages = n * width
    page = B.pipo_kv_page_bytes(ps, Hkv, D)
    pool = dev(np.full(n_pages * page, 255, np.uint8))
    table, lens = dev(np.full((n, width), -1, np.int32)), dev(np.zeros(n, np.int32))
    cnt, start, seq = dev(np.zeros(1, np.int32)), dev(np.arange(n + 1, dtype=np.int32)), dev(
        np.arange(n, dtype=np.int32))
    c = B.PipoKvPages(pool.ptr, n_pages * page, table.ptr, width, 1, n_pages, ps, Hkv, D, n)
    nb = B.pipo_op_attn_pages_workspace_bytes(c, H, n, 1, top)
    assert nb > 0
    cs = np.zeros((top, D // 2, 2), np.float32)
    cs[..., 0] = 1
    dcs = dev(cs)
    stream = hip.stream()

    def resize(want, s):
        B.pipo_op_kv_pages_resize(table.ptr, lens.ptr, want.ptr, table.ptr, lens.ptr, width, n, n_pages,
                                  ps, cnt.ptr, s)

    class Step:
        def __init__(self):
            self.q, self.k, self.v, self.o = (DB(n * w * D * 2) for w in (H, Hkv, Hkv, H))
            self.qr, self.kr = DB(n * H * D * 2), DB(n * Hkv * D * 2)
            self.ws, self.want, self.pos = DB(nb), DB(n * 4), DB(n * 4)

        def attend(self, o, s):
            B.pipo_op_attn_pages(c, 0, self.qr.ptr, H * D, start.ptr, lens.ptr, o.ptr, H * D, H, n, 1, top,
                                 self.ws.ptr, nb, s)

        def run(self, s):
            resize(self.want, s)
            B.pipo_op_qk_norm_rope(self.q.ptr, H * D, self.k.ptr, Hkv * D, None, None, dcs.ptr, top,
                                   self.pos.ptr, self.qr.ptr, H * D, self.kr.ptr, Hkv * D, n, H, Hkv, D,
                                   1e-5, 1.0, s)
            B.pipo_op_kv_pages_append(c, 0, seq.ptr, self.pos.ptr, self.kr.ptr, Hkv * D, self.v.ptr,
                                      Hkv * D, n, s)
            self.attend(self.o, s)

    def put(buf, a):
        B._check(B.lib().pipo_copy_h2d(buf.ptr, a.ctypes.data, a.nbytes), "pipo_copy_h2d")

    steps = [Step(), Step()]
    graphs = [hip.capture(stream, lambda s=s: s.run(stream)) for s in steps]
    assert lens.to_array(np.int32, (n,)).tolist() == [0] * n        # captured, not run
    resize(dev(np.array(length, np.int32)), stream)                 # the prompts, eagerly
    k, v = draw_rows(length, Hkv * D, rng), draw_rows(length, Hkv * D, rng)
    pseq, ppos = dev(np.repeat(np.arange(n), length), np.int32), dev(
        np.concatenate([np.arange(x) for x in length]), np.int32)
    pk, pv = dev(np.concatenate(k)), dev(np.concatenate(v))
    B.pipo_op_kv_pages_append(c, 0, pseq.ptr, ppos.ptr, pk.ptr, Hkv * D, pv.ptr, Hkv * D, sum(length),
                              stream)
    hip("hipStreamSynchronize", stream)
    refs = [[list(O.page_rows(x).reshape(-1, Hkv, D)) for x in y] for y in (k, v)]
    for it in range(6):
        s, g = steps[it % 2], graphs[it % 2]
        new = [(rng.standard_normal((n, w * D)) * sc).astype(np.float16)
               for w, sc in ((H, 0.1), (Hkv, 1), (Hkv, 1))]
        for buf, x in zip((s.q, s.k, s.v), new):
            put(buf, x)
        put(s.pos, np.array(length, np.int32))
        length = [x + 1 for x in length]
        put(s.want, np.array(length, np.int32))
        hip("hipGraphLaunch", g, stream)
        hip("hipStreamSynchronize", stream)
        for i in range(n):
            for r, x in zip(refs, new[1:]):
                r[i].extend(O.page_rows(x[i:i + 1]).reshape(1, Hkv, D))
        assert lens.to_array(np.int32, (n,)).tolist() == length
        assert cnt.to_array(np.int32, (1,))[0] == 0
        want, tol = want_attention(new[0], [np.array(x) for x in refs[0]], [np.array(x) for x in refs[1]],
                                   [1] * n, length, H, D)
        got = s.o.to_array(np.float16, (n, H * D))
        check(got, want, tol, it)
        o = dev(np.zeros((n, H * D), np.float16))
        s.attend(o, stream)
        hip("hipStreamSynchronize", stream)
        assert np.array_equal(o.to_array(np.float16, (n, H * D)), got)


def test_a_graph_of_prompts_and_single_tokens():
    """One captured call whose rows are shared out anew before each replay: prompts
    beside single tokens, single tokens alone, a prompt alone."""
    hip = Hip()
    rng = np.random.default_rng(21)
    lens, H, Hkv, D = [900, 40, 300, 1, 1300], 8, 2, 128
    n, M, top, max_q = len(lens), 160, 1300, 150
    c = Cache(lens, Hkv, D, 32, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((M, H * D)) * 0.2).astype(np.float16)
    nb = B.pipo_op_attn_pages_workspace_bytes(c.c(), H, M, max_q, top)
    dq, do, ws = dev(q), DB(M * H * D * 2), DB(max(nb, 16))
    start, length = DB((n + 1) * 4), dev(np.array(lens, np.int32))
    stream = hip.stream()

    def put(buf, a):
        B._check(B.lib().pipo_copy_h2d(buf.ptr, a.ctypes.data, a.nbytes), "pipo_copy_h2d")

    def run(s):
        B.pipo_op_attn_pages(c.c(), 0, dq.ptr, H * D, start.ptr, length.ptr, do.ptr, H * D, H, M, max_q,
                             top, ws.ptr, nb, s)

    graph = hip.capture(stream, lambda: run(stream))
    for rows in ([150, 1, 1, 1, 1], [1] * 5, [0, 0, 0, 0, 150], [30, 40, 3, 0, 80], [150, 1, 1, 1, 1]):
        put(start, np.concatenate([[0], np.cumsum(rows)]).astype(np.int32))
        put(do, np.full((M, H * D), 9, np.float16))
        hip("hipGraphLaunch", graph, stream)
        hip("hipStreamSynchronize", stream)
        got = do.to_array(np.float16, (M, H * D))
        want, tol = want_attention(q, k, v, rows, lens, H, D)
        check(got[:sum(rows)], want, tol, rows)
        assert (got[sum(rows):] == 9).all()
        put(do, np.full((M, H * D), 9, np.float16))
        run(stream)
        hip("hipStreamSynchronize", stream)
        assert np.array_equal(do.to_array(np.float16, (M, H * D)), got)
