"""A paged 8-bit KV cache on the GPU: rows in and out, and attention with capped and
biased scores, windows and prefixes, against plain definitions in 64 bits
(oracle/pages8.py).

Tolerances.  What the cache holds and gives back is equal.  An fp16 output is off by at
most half a step, 2^-11 of its value (2^-25 below 2^-14), and by what its weights are
off, against values of at most max|V|.  A score is a sum of D products in fp32, each
addition rounded by up to 2^-24 of sum|q k|: D 2^-24 sum|q k| at most; a tanh written
with exp and a reciprocal adds up to 2^-21 of the cap (each of four steps 2^-23 of a
number up to 2), biases, the factor log2(e) and the largest score's subtraction 2^-22 of
the largest score and bias.  An error of a score is a relative error of its
weight, and of the sum that divides it.  Where a sequence has more than 64 columns (rows
times heads of a key/value head) weights are rounded to halves: 2^-11 more."""
import numpy as np
import pytest

from oracle import pages8 as O
from oracle.sample import sample
from paper_2504_03664_amd import binding as B
from paper_2504_03664_amd.binding import DeviceBuffer as DB
from test_gpu_pages import Hip

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -11
FMT = {"e4m3": B.PIPO_KV8_E4M3, "int8": B.PIPO_KV8_INT8}
BOTH = pytest.mark.parametrize("fmt", ["e4m3", "int8"])


def dev(a, dtype=None):
    return DB.from_array(np.ascontiguousarray(a, dtype))


class Cache:
    """Sequences of given lengths on pages in random order, beside what their blocks
    hold by definition; the pool starts out as bytes of `fill` (255: NaNs)."""

    def __init__(self, lens, Hkv, D, ps, fmt, rng, extra=3, layers=1, fill=255, width=0):
        self.lens, self.Hkv, self.D, self.ps, self.layers = list(lens), Hkv, D, ps, layers
        self.fmt = fmt
        need = [-(-n // ps) for n in lens]
        self.n_pages = sum(need) + extra
        self.width = max(need + [1]) + width
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(lens), self.width), -1, np.int32)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.page = B.pipo_kv8_page_bytes(ps, Hkv, D)
        self.pool = dev(np.full(layers * self.n_pages * self.page, fill, np.uint8))
        self.d_table = dev(self.table)
        self.k, self.v = ([O.Blocks(Hkv, D, fmt) for _ in lens] for _ in "kv")

    def c(self):
        return B.PipoKv8Pages(self.pool.ptr, self.n_pages * self.page, self.d_table.ptr, self.width,
                              self.layers, self.n_pages, self.ps, self.Hkv, self.D, len(self.lens),
                              FMT[self.fmt])

    def set_table(self, t):
        self.table = np.ascontiguousarray(t, np.int32)
        self.width = self.table.shape[1]
        self.d_table = dev(self.table)

    def call(self, rows, lens, k, v, layer=0, shift=0, pad=0, starts=None, stream=None):
        M, w = len(k), self.Hkv * self.D
        bufs = []
        for x in (k, v):
            full = np.zeros((M, w + pad), np.float16)
            full[:, :w] = x.reshape(M, w)
            bufs.append(dev(np.concatenate([np.zeros(shift, np.float16), full.reshape(-1)])))
        starts = np.concatenate([[0], np.cumsum(rows)]) if starts is None else starts
        ds, dl = dev(starts, np.int32), dev(lens, np.int32)
        B.pipo_op_kv8_pages_append(self.c(), layer, ds.ptr, dl.ptr, bufs[0].ptr + 2 * shift, w + pad,
                                   bufs[1].ptr + 2 * shift, w + pad, M, stream)
        B.pipo_dev_synchronize()

    def append(self, k, v, lens=None, **kw):
        """k, v: per sequence [rows][Hkv * D]; they end at lens"""
        lens = [len(b.units) + len(x) for b, x in zip(self.k, k)] if lens is None else lens
        for i, n in enumerate(lens):
            for blocks, x in ((self.k[i], k[i]), (self.v[i], v[i])):
                if len(x):
                    blocks.append(x.reshape(len(x), self.Hkv, self.D), n)
        self.call([len(x) for x in k], lens, np.concatenate(k), np.concatenate(v), **kw)

    def fill(self, rng, std=1.0, **kw):
        draw = lambda: [(rng.standard_normal((n, self.Hkv * self.D)) * std).astype(np.float16)  # noqa: E731
                        for n in self.lens]
        self.append(draw(), draw(), **kw)

    def read(self, seq, pos, layer=0, shift=0, pad=0, fill=7.0):
        M, w = len(seq), self.Hkv * self.D
        bufs = [dev(np.full(shift + M * (w + pad), fill, np.float16)) for _ in "kv"]
        ds, dp = dev(seq, np.int32), dev(pos, np.int32)
        B.pipo_op_kv8_pages_read(self.c(), layer, ds.ptr, dp.ptr, bufs[0].ptr + 2 * shift, w + pad,
                                 bufs[1].ptr + 2 * shift, w + pad, M)
        B.pipo_dev_synchronize()
        out = [b.to_array(np.float16, (shift + M * (w + pad),)) for b in bufs]
        for x in out:
            assert (x[:shift] == fill).all() and (x[shift:].reshape(M, -1)[:, w:] == fill).all()
        return [x[shift:].reshape(M, -1)[:, :w] for x in out]

    def check_all(self, **kw):
        seq = np.concatenate([np.full(len(b.units), i) for i, b in enumerate(self.k)])
        pos = np.concatenate([np.arange(len(b.units)) for b in self.k])
        got = self.read(seq, pos, **kw)
        for y, blocks in zip(got, (self.k, self.v)):
            want = np.concatenate([b.values() for b in blocks]).reshape(len(seq), -1)
            bad = y.astype(np.float64) != want
            assert not bad.any(), (np.argwhere(bad)[:4], seq[bad.any(1)][:4], pos[bad.any(1)][:4],
                                   y[bad][:4], want[bad][:4])

    def bytes(self):
        return self.pool.to_array(np.uint8, (self.layers, self.n_pages, self.page))


def attend(c, q, rows, n_heads, lens=None, layer=0, split=True, shift=0, pad=0, max_q=None,
           max_len=None, behind=2, starts=None, cap=0.0, slopes=None, window=0, prefix=None,
           max_prefix=None, stream=None):
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
    keep = [dev(slopes, np.float32) if slopes is not None else None,
            dev(prefix, np.int32) if prefix is not None else None]
    if prefix is not None and max_prefix is None:
        max_prefix = max(max(prefix), 0)
    f = B.PipoAttnScores(cap, window, *(x.ptr if x else None for x in keep), max_prefix or 0)
    if not cap and slopes is None and not window and prefix is None:
        f = None
    n = B.pipo_op_attn_kv8_pages_workspace_bytes(c.c(), f, n_heads, total, max_q, max_len) if split else 0
    ws = dev(np.full(max(n // 4, 1), np.nan, np.float32))
    B.pipo_op_attn_kv8_pages(c.c(), layer, f, dq.ptr + 2 * shift, w + pad, ds.ptr, dl.ptr,
                             do.ptr + 2 * shift, w + pad, n_heads, total, max_q, max_len,
                             ws.ptr if n else None, n, stream)
    B.pipo_dev_synchronize()
    out = do.to_array(np.float16, (shift + total * (w + pad),))
    assert (out[:shift] == 9).all()
    out = out[shift:].reshape(total, w + pad)
    assert (out[:, w:] == 9).all()
    return out[:, :w]


def want_attention(c, q, rows, lens, H, cap=0.0, slopes=None, window=0, prefix=None):
    """(values, tolerance) of every row"""
    out, tol, at, D = [], [], 0, c.D
    many = max(rows) * (H // c.Hkv) > 64
    for i, (r, n) in enumerate(zip(rows, lens)):
        if r == 0:
            continue
        x = q[at:at + r].reshape(r, H, D)
        k, v = c.k[i].values()[:n], c.v[i].values()[:n]
        n = len(k)
        pre = min(max(prefix[i], 0), n) if prefix is not None else 0
        if r > n:       # rows before the first position see the prefix alone
            y = np.zeros((r, H, D))
            y[r - n:] = O.attention(x[r - n:], k, v, cap, slopes, window, pre)
            for j in range(r - n if pre else 0):
                bias = None if slopes is None else slopes
                y[j] = early_row(x[j], k, v, n - r + j, cap, bias, pre)
        else:
            y = O.attention(x, k, v, cap, slopes, window, pre)
        big = np.abs(v).max() if n else 0.0
        step = 0.0
        if n:
            kk = np.repeat(np.abs(k), H // c.Hkv, axis=1)
            most = np.einsum("rhd,nhd->rhn", np.abs(x.astype(np.float64)), kk).max()
            bias = 0.0 if slopes is None else float(np.abs(slopes).max()) * n
            step = D * 2.0 ** -24 * most + 2.0 ** -21 * cap + 2.0 ** -22 * (min(most, cap or most) + bias)
        out.append(y.reshape(r, -1))
        tol.append(HALF * np.abs(y.reshape(r, -1)) + (2 * step + (HALF if many else 2.0 ** -20)) * big +
                   2.0 ** -25)
        at += r
    return np.concatenate(out), np.concatenate(tol)


def early_row(x, k, v, pos, cap, slopes, pre):
    out = np.zeros(x.shape)
    for h in range(len(x)):
        s = k[:pre, h // (len(x) // k.shape[1])] @ x[h].astype(np.float64)
        s = cap * np.tanh(s / cap) if cap else s
        s = s if slopes is None else s - float(slopes[h]) * np.abs(pos - np.arange(pre))
        p = np.exp(s - s.max())
        out[h] = p @ v[:pre, h // (len(x) // k.shape[1])] / p.sum()
    return out


def check(got, want, tol, what):
    bad = ~(np.abs(got.astype(np.float64) - want) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])


def check_error(got, want, many, what=""):
    """all in all: the output's rounding (rms 2^-11 / root 3), and one of the weights"""
    if want.size > 500 and want.any():   # (zeros, of rows that see nothing, are equal)
        err = np.linalg.norm(got.astype(np.float64) - want) / np.linalg.norm(want)
        assert err <= np.sqrt((2 if many else 1) / 3) * HALF * 1.1, (what, err)


def draw_q(rng, M, H, D, std=1.5):
    return (rng.standard_normal((M, H * D)) * std * D ** -0.5).astype(np.float16)


# ---------------------------------------------------------------------------
@BOTH
@pytest.mark.parametrize("lens,Hkv,D,ps,shift,pad", [
    ([1], 1, 64, 16, 0, 0), ([5, 0, 17], 3, 128, 16, 0, 8), ([33, 64, 1, 100], 8, 128, 64, 0, 0),
    ([40, 3], 2, 64, 32, 1, 3), ([300], 5, 128, 256, 0, 0), ([129, 128, 127], 1, 128, 128, 5, 0),
    ([250, 31, 7], 13, 64, 64, 0, 0)])
def test_append_and_read(lens, Hkv, D, ps, shift, pad, fmt):
    """Whole prompts, in one call, of rows whose sizes differ; nothing else is written."""
    print(f"append lens={lens} Hkv={Hkv} D={D} ps={ps} shift={shift} pad={pad} {fmt}", flush=True)
    rng = np.random.default_rng(sum(lens) + ps)
    c = Cache(lens, Hkv, D, ps, fmt, rng, layers=2, fill=0xA5)
    k, v = ([(rng.standard_normal((n, Hkv * D)) * np.exp(2 * rng.standard_normal((n, 1)))).astype(
        np.float16) for n in lens] for _ in "kv")
    k[0][0, :5] = np.inf, -np.inf, np.nan, 65504, -57344
    v[0][0] = 0
    v[-1][-1] = rng.integers(-40, 40, Hkv * D) * 2.0 ** -24        # the least halves there are
    c.append(k, v, layer=1, shift=shift, pad=pad)
    c.check_all(layer=1, shift=shift, pad=pad)
    b = c.bytes()
    assert (b[0] == 0xA5).all()
    used = {int(p) for row, n in zip(c.table, lens) for p in row[:-(-n // ps)]}
    assert all((b[1, p] == 0xA5).all() for p in range(c.n_pages) if p not in used)
    tiles = sum(-(-n // 16) for n in lens) * Hkv
    assert (b[1] != 0xA5).sum() <= sum(lens) * Hkv * 2 * D + 8 * tiles


@BOTH
@pytest.mark.parametrize("D,ps", [(64, 16), (128, 32)])
def test_append_by_pieces(D, ps, fmt):
    """Rows that get larger and smaller as they come: scales of blocks grow under the codes
    that are there, by one power of two or by many, at every place in a block."""
    print(f"append by pieces D={D} ps={ps} {fmt}", flush=True)
    rng = np.random.default_rng(D)
    n, Hkv = 5, 3
    c = Cache([150] * n, Hkv, D, ps, fmt, rng, fill=0xA5)
    at = [0] * n
    while max(at) < 110:
        rows = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 3, 17], n)]
        k, v = ([(rng.standard_normal((r, Hkv * D)) * 2.0 ** rng.integers(-12, 9, (r, 1))).astype(
            np.float16) for r in rows] for _ in "kv")
        c.append(k, v)
        at = [len(b.units) for b in c.k]
    c.check_all()
    # some positions go again, and others come in their place: blocks keep their scales
    cut = [max(x - 5, 0) for x in at]
    k, v = ([(rng.standard_normal((3, Hkv * D)) * 0.01).astype(np.float16) for _ in at] for _ in "kv")
    c.append(k, v, lens=[x + 3 for x in cut])
    c.check_all()


@BOTH
def test_append_of_infinities_anywhere(fmt):
    """One element out of range or not a number, at every place of a row and a block."""
    rng = np.random.default_rng(20)
    n, bad = 128, [np.inf, -np.inf, np.nan, 60000, -65504]
    c = Cache([n], 1, 128, 32, fmt, rng)
    k, v = (rng.standard_normal((n, 128)).astype(np.float16) for _ in "kv")
    for i in range(0, n, 8):       # some blocks have one, some more
        k[i + i // 8 % 8, (37 * i) % 128] = bad[i // 8 % 5]
        v[i // 2, (i + 53) % 128] = bad[(i // 8 + 1) % 5]
    c.append([k], [v])
    c.check_all()


@BOTH
def test_append_extremes(fmt):
    """The largest and least scales; a begun block whose scale is above what new rows need."""
    rng = np.random.default_rng(8)
    c = Cache([40, 40, 40], 1, 128, 16, fmt, rng)
    big, tiny = np.float16(60000), np.float16(2.0 ** -24)
    rows = lambda *xs: [np.full((1, 128), x, np.float16) for x in xs]  # noqa: E731
    c.append(rows(big, tiny, 0.0), rows(tiny, big, 0.0))
    c.append(rows(tiny, big, tiny), rows(big, tiny, 1.0))
    c.append(rows(1.0, 1.0, 1.0), rows(1.0, 1.0, big))
    c.check_all()


@BOTH
def test_append_skips_what_has_no_place(fmt):
    """Wrong tables, positions before the first, starts out of range: the others' rows
    are written and nothing else."""
    rng = np.random.default_rng(2)
    c = Cache([40, 20, 30, 16], 2, 128, 16, fmt, rng, fill=0xA5)
    t = np.full((4, 3), -1, np.int32)
    t[0] = c.table[0, 0], -1, c.n_pages
    t[1] = 1 << 30, c.table[1, 0], -(1 << 31)
    t[2] = c.table[2, :3] if c.width >= 3 else -1
    t[3, 0] = c.table[3, 0]
    c.set_table(t)
    x = rng.standard_normal((100, 256)).astype(np.float16)
    # sequence 0: 48 rows up to 48; 1: up to 100, past its row; 2: ten rows up to 4, six of
    # them before position 0; 3: none
    c.call(None, [48, 100, 4, 16], x, x, starts=[0, 48, 88, 98, 98])
    for i, (a, r) in enumerate(((0, 16), (76 - 60, 16))):
        b = O.Blocks(2, 128, fmt)
        if i == 0:
            b.append(x[:16].reshape(16, 2, 128), 16)
            pos = np.arange(16)
        else:       # position 60 + j is row 48 + j: none of them is at 16 .. 31
            continue
        got = c.read(np.zeros(16, int), pos)
        assert np.array_equal(got[0].astype(np.float64), b.values().reshape(16, -1))
        assert np.array_equal(got[1], got[0])
    b = O.Blocks(2, 128, fmt)
    b.append(x[94:98].reshape(4, 2, 128), 4)
    got = c.read(np.full(4, 2), np.arange(4))
    assert np.array_equal(got[0].astype(np.float64), b.values().reshape(4, -1))
    by = c.bytes()[0]
    ours = {int(t[0, 0]), int(t[2, 0])}
    assert all((by[p] == 0xA5).all() for p in range(c.n_pages) if p not in ours)
    # starts outside [0, M] count as the nearer end; lengths below 0 have no rows
    before = c.bytes()
    for starts, lens in (([-5, -1, 0, 0, 0], [16] * 4), ([200, 300, 400, 400, 1 << 30], [16] * 4),
                         ([0, 10, 20, 30, 40], [-3, 0, -(1 << 31), -1])):
        c.call(None, lens, x, x, starts=starts)
        assert np.array_equal(before, c.bytes())


@BOTH
def test_read_skips_rows_without_a_slot(fmt):
    rng = np.random.default_rng(3)
    c = Cache([40, 20], 2, 64, 16, fmt, rng)
    c.fill(rng)
    c.set_table(np.array([[c.table[0, 0], -1, c.n_pages], [c.table[1, 0], 1 << 30, -(1 << 31)]], np.int32))
    rows = [(-1, 0), (2, 0), (1 << 30, 3), (0, -1), (0, 16), (0, 47), (0, 48), (1, 1 << 30), (1, 17),
            (1, 33), (0, 2 ** 31 - 1), (-(2 ** 31), -(2 ** 31)), (0, 3)]
    k, v = c.read(*np.array(rows).T)
    assert (k[:-1] == 7).all() and (v[:-1] == 7).all()
    assert np.array_equal(k[-1].astype(np.float64), c.k[0].values()[3].reshape(-1))
    assert np.array_equal(v[-1].astype(np.float64), c.v[0].values()[3].reshape(-1))


@pytest.mark.parametrize("n", [63, 64, 65, 130, 4100])
def test_append_of_many_sequences(n):
    """Over the counts at which workgroups find their sequence in another way."""
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.choice([0, 1, 2, 16, 17, 33], n)]
    c = Cache(lens, 1, 64, 16, "e4m3", rng)
    c.fill(rng)
    c.check_all()


def test_copy_and_shared_pages():
    """A beam's last page copied in every layer, the pages before it shared."""
    rng = np.random.default_rng(4)
    c = Cache([40, 40], 2, 64, 16, "int8", rng, layers=2)
    for layer in range(2):
        c.k, c.v = ([O.Blocks(2, 64, "int8") for _ in range(2)] for _ in "kv")
        c.fill(rng, layer=layer)
    t = c.table.copy()
    t[1, :2] = t[0, :2]
    pairs, count = dev(np.array([[t[0, 2], t[1, 2]], [0, 1]]), np.int32), dev([1], np.int32)
    B.pipo_op_kv8_pages_copy(c.c(), pairs.ptr, count.ptr, 2)
    B.pipo_dev_synchronize()
    c.set_table(t)
    a, b = (c.read(np.full(40, i), np.arange(40), layer=1) for i in range(2))
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    by = c.bytes()
    assert np.array_equal(by[:, t[0, 2]], by[:, t[1, 2]])


# ---------------------------------------------------------------------------
SHAPES = [
    ([1], [1], 1, 1, 64, 16), ([1, 15, 16, 17], [1] * 4, 4, 4, 128, 16),
    ([31, 32, 33, 0, 100], [1] * 5, 8, 2, 128, 32), ([130, 7], [1, 1], 6, 2, 64, 64),
    ([257, 255, 256], [1] * 3, 10, 2, 128, 256), ([40, 90], [1, 1], 7, 1, 128, 128),
    ([65, 20], [1, 1], 32, 2, 64, 16), ([50, 300], [1, 1], 71, 1, 64, 64),
    ([20, 33, 64], [2, 0, 3], 8, 2, 128, 32), ([70, 16, 5], [5, 16, 5], 12, 4, 128, 16),
    ([200, 100], [17, 100], 4, 4, 64, 64), ([150, 330, 40], [130, 1, 40], 8, 2, 128, 64),
    ([700, 600], [300, 257], 4, 1, 128, 32), ([333], [333], 3, 3, 64, 16),
    ([530, 90, 260, 33], [1, 90, 129, 2], 10, 2, 128, 64)]


def run_attention(lens, rows, H, Hkv, D, ps, fmt, shift=0, pad=0, seed=0, cap=0.0, slopes=False,
                  window=0, prefix=0, split=True, std=1.5):
    rng = np.random.default_rng(sum(lens) + H + seed)
    c = Cache(lens, Hkv, D, ps, fmt, rng, layers=2)
    c.fill(rng, layer=1)
    q = draw_q(rng, sum(rows), H, D, std)
    f = dict(cap=cap, window=window, slopes=rng.uniform(0, 0.2, H).astype(np.float32) if slopes else None,
             prefix=[max(0, prefix - 3 * i) for i in range(len(lens))] if prefix else None)
    got = attend(c, q, rows, H, layer=1, shift=shift, pad=pad, split=split, **f)
    want, tol = want_attention(c, q, rows, lens, H, **f)
    check(got[:len(q)], want, tol, "attention")
    assert (got[len(q):] == 9).all()
    check_error(got[:len(q)], want, max(rows) * H // Hkv > 64)


@BOTH
@pytest.mark.parametrize("shift,pad", [(0, 0), (1, 3)])
@pytest.mark.parametrize("lens,rows,H,Hkv,D,ps", SHAPES)
def test_attention(lens, rows, H, Hkv, D, ps, shift, pad, fmt):
    print(f"attn lens={lens} rows={rows} H={H}/{Hkv} D={D} ps={ps} shift={shift} {fmt}", flush=True)
    run_attention(lens, rows, H, Hkv, D, ps, fmt, shift, pad)


@BOTH
@pytest.mark.parametrize("cap,slopes,window,prefix", [
    (5.0, False, 0, 0), (0.0, True, 0, 0), (30.0, True, 0, 0), (0.0, False, 1, 0), (0.0, False, 40, 0),
    (0.0, False, 0, 50), (2.0, True, 33, 20), (0.0, True, 5, 200)])
@pytest.mark.parametrize("lens,rows,H,Hkv,D,ps", SHAPES[2:])
def test_attention_scores(lens, rows, H, Hkv, D, ps, cap, slopes, window, prefix, fmt):
    print(f"attn lens={lens} rows={rows} H={H}/{Hkv} D={D} ps={ps} cap={cap} slopes={slopes} "
          f"window={window} prefix={prefix} {fmt}", flush=True)
    run_attention(lens, rows, H, Hkv, D, ps, fmt, cap=cap, slopes=slopes, window=window, prefix=prefix,
                  seed=1, std=4.0 if cap else 1.5)


@BOTH
@pytest.mark.parametrize("lens,rows,window,prefix", [
    ([5000], [1], 0, 0), ([3001, 2999], [1, 1], 0, 0), ([9000], [1], 2000, 100), ([4096, 1], [2, 1], 0, 33),
    ([2500, 900], [200, 1], 0, 0), ([3000], [150], 700, 64)])
def test_attention_in_parts(lens, rows, window, prefix, fmt):
    """Keys split over workgroups, and the same without a workspace."""
    print(f"attn parts lens={lens} rows={rows} window={window} prefix={prefix} {fmt}", flush=True)
    for split in (True, False):
        run_attention(lens, rows, 4, 2, 128, 64, fmt, window=window, prefix=prefix, split=split)


@pytest.mark.parametrize("n", [64, 65, 200])
def test_attention_of_many_sequences(n):
    """Prompts' pieces among single rows, over the counts at which workgroups find
    their sequence in another way; columns at 64, 65, 128 and 129."""
    print(f"attn sequences n={n}", flush=True)
    rng = np.random.default_rng(n)
    rows = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 32, 33, 64, 65, 90], n)]
    lens = [r + int(x) for r, x in zip(rows, rng.integers(0, 60, n))]
    run_attention(lens, rows, 4, 2, 64, 16, "e4m3", slopes=n == 65, window=40 if n == 200 else 0)


@BOTH
def test_rows_that_see_nothing(fmt):
    """More rows than keys, no keys, no pages; a prefix makes the early rows see."""
    rng = np.random.default_rng(6)
    for rows in ([9, 4, 3], [80, 70, 3]):
        lens, H = [5, 0, 20], 4
        c = Cache(lens, 2, 64, 16, fmt, rng)
        c.fill(rng)
        q = draw_q(rng, sum(rows), H, 64)
        got = attend(c, q, rows, H)
        want, tol = want_attention(c, q, rows, lens, H)
        check(got[:len(q)], want, tol, "early rows")
        assert (got[:rows[0] - 5] == 0).all() and (got[rows[0]:rows[0] + rows[1]] == 0).all()
        f = dict(slopes=np.array([0.1, 0.2, 0.0, -0.1], np.float32), window=2, prefix=[3, 3, 3], cap=4.0)
        got = attend(c, q, rows, H, **f)
        want, tol = want_attention(c, q, rows, lens, H, **f)
        check(got[:len(q)], want, tol, "early rows with a prefix")
        c.set_table(np.full_like(c.table, -1))
        got = attend(c, q, rows, H, **f)
        assert (got[:len(q)] == 0).all() and (got[len(q):] == 9).all()


@BOTH
@pytest.mark.parametrize("rows", [[1, 1], [40, 70]])
def test_wrong_entries_and_bounds(rows, fmt):
    """Keys on entries that are no pages are not seen; lengths past max_len, prefixes past
    max_prefix, rows past max_q and starts out of range count as the header says."""
    rng = np.random.default_rng(7)
    H, Hkv, D, ps, lens = 4, 2, 64, 16, [100, 90]
    c = Cache(lens, Hkv, D, ps, fmt, rng)
    c.fill(rng)
    q = draw_q(rng, sum(rows), H, D)
    whole, right = attend(c, q, rows, H), c.table.copy()
    want, tol = want_attention(c, q, rows, lens, H)
    check(whole[:len(q)], want, tol, "before")
    t = right.copy()
    t[0, 1], t[0, 3], t[1, 0] = -1, c.n_pages, -(1 << 31)
    c.set_table(t)
    got = attend(c, q, rows, H)
    at = 0
    for i, (r, n) in enumerate(zip(rows, lens)):
        gone = np.repeat((t[i, :-(-n // ps)] < 0) | (t[i, :-(-n // ps)] >= c.n_pages), ps)[:n]
        x, k, v = q[at:at + r].reshape(r, H, D), c.k[i].values(), c.v[i].values()
        seen = O.seen(r, n) & ~gone
        for h in range(H):
            s = np.where(seen, x[:, h].astype(np.float64) @ k[:, h // 2].T, -np.inf)
            p = np.exp(s - np.maximum(s.max(1, keepdims=True), -1e300))
            total = p.sum(1, keepdims=True)
            y = np.where(total > 0, p @ v[:, h // 2] / np.where(total > 0, total, 1), 0)
            check(got[at:at + r].reshape(r, H, D)[:, h], y, tol.reshape(-1, H, D)[at:at + r, h] + HALF * 4,
                  "holes")
        at += r
    c.set_table(right)
    # bounds: a length above max_len counts as max_len
    got = attend(c, q, rows, H, max_len=90, lens=[1 << 30, 90])
    c.k[0].append(np.zeros((0, Hkv, D)), 90)
    c.v[0].append(np.zeros((0, Hkv, D)), 90)
    want, tol = want_attention(c, q, rows, [90, 90], H)
    check(got[:len(q)], want, tol, "max_len")
    got = attend(c, q, rows, H, lens=[90, 90], prefix=[1 << 30, -5], max_prefix=7)
    want, tol = want_attention(c, q, rows, [90, 90], H, prefix=[7, 0])
    check(got[:len(q)], want, tol, "max_prefix")
    if max(rows) > 1:
        got = attend(c, q, rows, H, lens=[90, 90], max_q=50)
        want, tol = want_attention(c, q, rows, [90, 90], H)
        check(got[:90], want[:90], tol[:90], "max_q")
        assert (got[90:] == 9).all()
        got = attend(c, q, rows, H, lens=[90, 90], starts=[-7, 40, 1 << 30], max_q=200, behind=0)
        assert np.isfinite(got.astype(np.float64)).all()


@BOTH
@pytest.mark.parametrize("nq", [1, 100])
def test_infinite_queries(nq, fmt):
    """A row with infinities or NaN is NaN where its scores are; the others are not touched."""
    rng = np.random.default_rng(9)
    lens, rows, H = [130, 140], [nq, nq], 2
    c = Cache(lens, 1, 128, 32, fmt, rng)
    c.fill(rng)
    q = draw_q(rng, 2 * nq, H, 128)
    clean = attend(c, q, rows, H)
    q[nq, 5], q[nq, 128 + 7] = np.inf, np.nan
    got = attend(c, q, rows, H)
    assert np.isnan(got[nq].astype(np.float64)).all()
    keep = np.arange(len(clean)) != nq
    assert np.array_equal(got[keep], clean[keep])


@BOTH
def test_large_scores(fmt):
    """Scores far apart, and large ones that hardly differ: the weights' errors are those of
    the scores' sums."""
    rng = np.random.default_rng(10)
    for std, n in ((40.0, 300), (1000.0, 64)):
        c = Cache([n], 1, 128, 64, fmt, rng)
        k = rng.standard_normal((n, 128))
        k = (k * 0.002 + rng.standard_normal(128)).astype(np.float16) if std > 100 else k.astype(np.float16)
        c.append([k], [rng.standard_normal((n, 128)).astype(np.float16)])
        for rows in ([1], [64]):
            q = draw_q(rng, rows[0], 2, 128, std)
            got = attend(c, q, rows, 2)
            want, tol = want_attention(c, q, rows, [n], 2)
            check(got[:len(q)], want, tol, "large scores")


@BOTH
@pytest.mark.parametrize("nq", [1, 70])
def test_equal_weights_over_a_long_context(nq, fmt):
    """Sums over many keys lose nothing: nearly equal weights, values of both signs and
    values of one."""
    rng = np.random.default_rng(11)
    n = 20000
    c = Cache([n], 1, 64, 256, fmt, rng)
    k, v = rng.standard_normal((2, n, 64))
    v[:, 32:] = 1 + 0.1 * v[:, 32:]
    c.append([k.astype(np.float16)], [v.astype(np.float16)])
    q = draw_q(rng, nq, 1, 64, 0.05)
    for split in (True, False):
        got = attend(c, q, [nq], 1, split=split)[:nq].astype(np.float64)
        want, _ = want_attention(c, q, [nq], [n], 1)
        for part in (slice(0, 32), slice(32, 64)):
            err = np.linalg.norm(got[:, part] - want[:, part]) / np.linalg.norm(want[:, part])
            assert err <= np.sqrt(2 / 3) * HALF * 1.1, (part, err)


def test_values_of_very_different_sizes():
    """Blocks whose scales are far apart: small values beside large ones keep their size."""
    for fmt in ("e4m3", "int8"):
        rng = np.random.default_rng(12)
        n = 64
        c = Cache([n], 1, 64, 16, fmt, rng)
        size = np.repeat(2.0 ** np.array([-14, 0, 14, -6]), 16)[:, None]
        k = rng.standard_normal((n, 64)) * 0.3
        c.append([k.astype(np.float16)], [(rng.standard_normal((n, 64)) * size).astype(np.float16)])
        for nq in (1, 64, 80):
            rows = min(nq, n)
            q = draw_q(rng, rows, 2, 64)
            got = attend(c, q, [rows], 2)[:rows].astype(np.float64).reshape(rows, 2, 64)
            want, tol = want_attention(c, q, [rows], [n], 2)
            check(got.reshape(rows, -1), want, tol, fmt)
            if rows > 20:   # rows before the large block: an error relative to their own values
                first = want.reshape(rows, 2, 64)[:16 - (n - rows)] if rows == n else None
                if first is not None and len(first):
                    y = got[:len(first)]
                    assert np.abs(y - first).max() <= 4 * HALF * 2.0 ** -12


def test_a_stream_and_another_run():
    """On a stream of the caller's; the same bits as on the default one and on every run."""
    rng = np.random.default_rng(13)
    lens, rows, H = [900, 40, 333], [1, 3, 130], 4
    c = Cache(lens, 2, 128, 64, "e4m3", rng)
    c.fill(rng)
    q = draw_q(rng, sum(rows), H, 128)
    first = attend(c, q, rows, H, cap=20.0)
    stream = Hip().stream()
    for _ in range(3):
        assert np.array_equal(first, attend(c, q, rows, H, cap=20.0, stream=stream))


def test_far_offsets():
    """A pool whose pages lie past 2^32 bytes."""
    rng = np.random.default_rng(14)
    Hkv, D, ps = 16, 128, 256
    page = B.pipo_kv8_page_bytes(ps, Hkv, D)
    n_pages = (1 << 32) // page + 40
    c = Cache([300, 20], Hkv, D, ps, "int8", rng, fill=0, extra=0)
    c.n_pages = n_pages
    c.pool = DB(n_pages * page)
    t = c.table.copy()
    t[t >= 0] = n_pages - 1 - t[t >= 0]
    c.set_table(t)
    c.fill(rng)
    c.check_all()
    q = draw_q(rng, 2, Hkv, D)
    got = attend(c, q, [1, 1], Hkv)
    want, tol = want_attention(c, q, [1, 1], c.lens, Hkv)
    check(got[:2], want, tol, "far")


@BOTH
def test_steps_captured_and_replayed(fmt):
    """A decode loop in a graph: resize, append, attention and the draw of tokens, replayed
    with other data and eager work between, against the same calls made one by one."""
    hip = Hip()
    rng = np.random.default_rng(15)
    n, H, Hkv, D, ps, V = 5, 8, 2, 128, 16, 9000
    lens, w = [30, 16, 5, 900, 15], 2 * Hkv * D
    kv, q, o = DB(n * w * 2), DB(n * H * D * 2), DB(n * H * D * 2)
    logits, u, want = DB(n * V * 4), DB(n * 4), DB(n * 4)
    nxt, logp, start = DB(n * 4), DB(n * 4), dev(np.arange(n + 1), np.int32)
    T, topk = dev([1.0, 0.7, 0.0, 2.0, 1.0], np.float32), dev([0, 20, 0, 5, 0], np.int32)
    top_p, min_p = dev([1, 0.9, 1, 0.8, 0.5], np.float32), dev([0, 0.01, 0, 0, 0.1], np.float32)
    slopes = dev(rng.uniform(0, 0.1, H), np.float32)
    f = B.PipoAttnScores(30.0, 600, slopes.ptr, None, 0)

    class Loop:
        def __init__(self):
            r = np.random.default_rng(16)
            self.c = Cache(lens, Hkv, D, ps, fmt, r, extra=12, width=3)
            self.c.fill(r)
            self.len, self.missing = dev(lens, np.int32), dev([0], np.int32)
            self.max_len = self.c.width * ps
            self.ws_bytes = max(B.pipo_op_sample_workspace_bytes(n, V),
                                B.pipo_op_attn_kv8_pages_workspace_bytes(self.c.c(), f, H, n, 1,
                                                                         self.max_len))
            self.ws = DB(self.ws_bytes)

        def run(self, st):
            c, t = self.c, self.c.d_table.ptr
            B.pipo_op_kv_pages_resize(t, self.len.ptr, want.ptr, t, self.len.ptr, c.width, n, c.n_pages,
                                      ps, self.missing.ptr, st)
            B.pipo_op_kv8_pages_append(c.c(), 0, start.ptr, self.len.ptr, kv.ptr, w,
                                       kv.ptr + 2 * Hkv * D, w, n, st)
            B.pipo_op_attn_kv8_pages(c.c(), 0, f, q.ptr, H * D, start.ptr, self.len.ptr, o.ptr, H * D, H,
                                     n, 1, self.max_len, self.ws.ptr, self.ws_bytes, st)
            B.pipo_op_sample(logits.ptr, V, T.ptr, topk.ptr, top_p.ptr, min_p.ptr, u.ptr, nxt.ptr,
                             logp.ptr, n, V, self.ws.ptr, self.ws_bytes, st)

        def results(self):
            return [o.to_array(np.uint16, (n, H * D)), nxt.to_array(np.int32, (n,)),
                    logp.to_array(np.uint32, (n,)), self.len.to_array(np.int32, (n,)),
                    self.c.d_table.to_array(np.int32, self.c.table.shape), self.c.bytes()]

    def put(buf, a, dtype):
        a = np.ascontiguousarray(a, dtype)
        assert B.lib().pipo_copy_h2d(buf.ptr, a.ctypes.data, a.nbytes) == 0

    eager, captured, stream = Loop(), Loop(), hip.stream()
    put(want, [x + 1 for x in lens], np.int32)
    graph = hip.capture(stream, lambda: captured.run(stream))
    seen = set()
    for i in range(5):
        put(kv, rng.standard_normal((n, w)) * 2.0 ** i, np.float16)
        put(q, draw_q(rng, n, H, D), np.float16)
        put(logits, rng.standard_normal((n, V)) * 3, np.float32)
        put(u, rng.random(n), np.float32)
        put(want, [x + 1 + i for x in lens], np.int32)
        eager.run(stream)
        hip("hipStreamSynchronize", stream)
        one = eager.results()
        for buf in (o, nxt, logp):
            put(buf, np.zeros(buf.nbytes, np.uint8), np.uint8)
        hip("hipGraphLaunch", graph, stream)
        hip("hipStreamSynchronize", stream)
        for a, b in zip(one, captured.results()):
            assert np.array_equal(a, b)
        assert captured.missing.to_array(np.int32, (1,))[0] == 0
        seen.add(tuple(one[1]))
    assert len(seen) == 5


def test_a_batch_from_prompts_to_tokens():
    """Prompts in pieces beside single tokens, forks that share pages, a draw from what
    comes out: every step against the definitions."""
    rng = np.random.default_rng(17)
    H, Hkv, D, ps, n, V = 4, 2, 64, 16, 3, 400
    head = rng.standard_normal((V, H * D)).astype(np.float32)
    c = Cache([0] * n, Hkv, D, ps, "int8", rng, width=8)
    c.n_pages = 24
    c.pool = dev(np.full(c.n_pages * c.page, 255, np.uint8))
    c.set_table(np.full((n, 8), -1, np.int32))
    length, missing = dev([0] * n, np.int32), dev([0], np.int32)

    def grow(to):
        want = dev(to, np.int32)
        B.pipo_op_kv_pages_resize(c.d_table.ptr, length.ptr, want.ptr, c.d_table.ptr, length.ptr, c.width,
                                  n, c.n_pages, ps, missing.ptr)
        B.pipo_dev_synchronize()
        assert missing.to_array(np.int32, (1,))[0] == 0

    def step(rows):
        to = [len(b.units) + r for b, r in zip(c.k, rows)]
        grow(to)
        k, v = ([rng.standard_normal((r, Hkv * D)).astype(np.float16) for r in rows] for _ in "kv")
        c.append(k, v)
        q = draw_q(rng, sum(rows), H, D)
        got = attend(c, q, rows, H, lens=to, cap=10.0, window=20, prefix=[4] * n)[:len(q)]
        want, tol = want_attention(c, q, rows, to, H, cap=10.0, window=20, prefix=[4] * n)
        check(got, want, tol, rows)
        x = dev(got[np.cumsum(rows) - 1].astype(np.float32) @ head.T, np.float32)
        u, m = rng.random(n).astype(np.float32), dev([0.05] * n, np.float32)
        du, nxt = dev(u, np.float32), dev([0] * n, np.int32)
        B.pipo_op_sample(x.ptr, V, None, None, None, m.ptr, du.ptr, nxt.ptr, None, n, V)
        B.pipo_dev_synchronize()
        logits = x.to_array(np.float32, (n, V))
        assert nxt.to_array(np.int32, (n,)).tolist() == [
            sample(logits[i], float(u[i]), min_p=float(np.float32(0.05)))[0] for i in range(n)]

    step([20, 37, 5])
    step([1, 30, 1])
    step([1, 1, 1])
    # sequence 0 and 2 continue from 1: full pages shared, the last one copied
    parent, t2, l2 = dev([1, 1, 1], np.int32), DB(n * 8 * 4), DB(n * 4)
    pairs, counts = DB(n * 8), DB(8)
    B.pipo_op_kv_pages_fork(c.d_table.ptr, length.ptr, n, parent.ptr, t2.ptr, l2.ptr, n, c.width,
                            c.n_pages, ps, pairs.ptr, counts.ptr, counts.ptr + 4)
    B.pipo_op_kv8_pages_copy(c.c(), pairs.ptr, counts.ptr, n)
    B.pipo_dev_synchronize()
    c.set_table(t2.to_array(np.int32, (n, 8)))
    length = l2
    for blocks in (c.k, c.v):
        for i in (0, 2):
            blocks[i].units, blocks[i].exps = blocks[1].units.copy(), blocks[1].exps.copy()
    c.check_all()
    step([1, 2, 20])
    c.check_all()
