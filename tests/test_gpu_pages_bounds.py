"""The paged 4-bit cache where the bounds of test_gpu_pages.py have room: what
attention must not read and how far it may be off (there the error of a score is
that of codes held 256 above their value, and of the largest query and scale of a
batch), and counts of pages that go far past a table."""
import numpy as np
import pytest

from oracle import pages as O
from paper_2504_03664_amd import binding as B
from paper_2504_03664_amd.binding import DeviceBuffer as DB
from test_gpu_pages import HALF, Cache, attend, check, dev, draw_rows

pytestmark = pytest.mark.gpu


class CacheWithoutPage0(Cache):
    """No sequence holds page 0: whatever it contains is no key's or value's."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        spare = min(set(range(1, self.n_pages)) - set(self.table.reshape(-1).tolist()))
        t = self.table.copy()
        t[t == 0] = spare
        self.set_table(t)

    def set_page0(self, byte):
        x = np.full(self.page, byte, np.uint8)
        B._check(B.lib().pipo_copy_h2d(self.pool.ptr, x.ctypes.data, x.nbytes), "pipo_copy_h2d")


@pytest.mark.parametrize("lens,rows,H,Hkv,D", [
    ([1500], [1], 2, 1, 128), ([1500], [4], 2, 1, 64), ([300, 700], [1, 3], 40, 2, 64),
    ([1500], [60], 2, 1, 128), ([1500], [60], 2, 1, 64), ([1500], [300], 4, 2, 128),
    ([900, 40, 700, 300], [150, 1, 1, 30], 8, 2, 128),        # both kinds in one launch
    ([900, 40, 700, 300], [150, 1, 1, 30], 8, 2, 64),
    ([400] * 12, [130] * 12, 64, 8, 64)])                     # one team a workgroup
@pytest.mark.parametrize("split", [True, False])
def test_attention_reads_nothing_of_a_page_that_is_none(lens, rows, H, Hkv, D, split):
    """Entries that are no pages, beside a page 0 of no sequence whose bytes are
    NaNs (255), finite scales and mins of 61280 (0x7B) or zeros: the same bits each
    time, and those of the keys that there are."""
    print(f"attn page 0 lens={lens[:4]} rows={rows[:4]} D={D} split={split}", flush=True)
    rng = np.random.default_rng(sum(lens) + sum(rows) + D)
    ps = 16
    c = CacheWithoutPage0(lens, Hkv, D, ps, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((sum(rows), H * D)) * 0.1).astype(np.float16)
    t, bad, holes = c.table.copy(), [-1, c.n_pages, 1 << 30, -(1 << 31)], []
    for i, n in enumerate(lens):
        pages = -(-n // ps)
        at = np.nonzero(rng.random(pages) < 0.2)[0]
        if pages > 4:
            at = np.union1d(at, [0, pages // 2])
        t[i, at] = [bad[x % 4] for x in range(len(at))]
        holes.append(at)
    c.set_table(t)
    got = []
    for byte in (255, 0x7B, 0):
        c.set_page0(byte)
        got.append(attend(c, q, rows, H, split=split)[:len(q)])
    at = 0
    for i, (r, n) in enumerate(zip(rows, lens)):
        seen = np.arange(n)[None] <= (n - r + np.arange(r))[:, None]
        for j in holes[i]:
            seen[:, j * ps:(j + 1) * ps] = False
        x = q[at:at + r].reshape(r, H, D)
        o = O.page_attention(x, k[i], v[i], seen).reshape(r, -1)
        # the output's rounding and, of many columns, the weights' (2^-11 of values
        # of at most max|V|); the errors of scores are below 2^-13
        tol = HALF * np.abs(o) + 1.25 * HALF * np.abs(v[i]).max() + 2.0 ** -25
        for y in got:
            check(y[at:at + r], o, tol, (i, "page 0"))
        at += r
    assert np.array_equal(got[0], got[2]) and np.array_equal(got[1], got[2])


@pytest.mark.parametrize("lens,H,Hkv,D", [
    ([16384] + [1] * 1100, 2, 1, 64),      # two waves a workgroup, 64 keys at a time
    ([16384] + [1] * 1100, 16, 1, 64),     # 32 keys at a time
    ([16384] + [1] * 1100, 2, 1, 128),
    ([65536] + [1] * 300, 2, 1, 64),       # four waves
    ([65536] + [1] * 1100, 4, 1, 64),
    ([65536], 2, 1, 64), ([65536], 16, 1, 128), ([262144], 2, 1, 64)])
def test_attention_over_long_contexts_in_one_part(lens, H, Hkv, D):
    """Weights nearly alike over one part of many keys: the outputs are as small as
    one over the root of the keys, and sums of magnitudes are hundreds of times
    larger.  The output's own rounding has an rms of 2^-11 / root 3 of it at most.
    fp32 sums that stay of its size, of T / 32 terms at most, are off by root(T / 32)
    roundings of 2^-25, below 2^-18; sums of codes, 7.5 in the mean where a value's
    deviation is 4.6, over 32 blocks of 32 keys, by 7.5 / 4.6 * 2^-25 * root(1024) *
    root(32) together, below 2^-16: a tenth of the first, and 2^-13 for any element,
    leave room for both."""
    print(f"attn uniform lens={lens[:2]} H={H}/{Hkv} D={D}", flush=True)
    rng = np.random.default_rng(lens[0] + H + D)
    c = Cache(lens, Hkv, D, 64, rng)
    k, v = c.fill(draw_rows(lens, Hkv * D, rng), draw_rows(lens, Hkv * D, rng))
    q = (rng.standard_normal((len(lens), H * D)) * 0.02).astype(np.float16)
    got = attend(c, q, [1] * len(lens), H, split=False)[:1].astype(np.float64)
    o = O.page_attention(q[:1].reshape(1, H, D), k[0], v[0], np.ones((1, lens[0]), bool)).reshape(1, -1)
    rms = np.sqrt((o * o).mean())
    assert np.linalg.norm(got - o) <= 1.1 * HALF / np.sqrt(3) * np.linalg.norm(o)
    check(got, o, HALF * np.abs(o) + 2.0 ** -13 * rms + 2.0 ** -25, "uniform")


def alike_keys(n, Hkv, D, rng, size):
    """Keys of one value each but in sixteen dimensions of a group of 64, where they
    differ: the same scale and min in each, and 15 steps of it"""
    base = rng.uniform(-1, 1, (Hkv, D // 64, 64))
    base[..., 16], base[..., 17] = -1, 1
    k = np.broadcast_to(base, (n,) + base.shape).copy()
    k[..., :16] = rng.uniform(-1, 1, k[..., :16].shape)
    return (k * size).reshape(n, Hkv * D).astype(np.float16)


@pytest.mark.parametrize("rows,H,Hkv,D", [(1, 4, 2, 128), (1, 32, 1, 128), (3, 4, 2, 64), (70, 4, 2, 128),
                                          (70, 4, 2, 64)])
@pytest.mark.parametrize("size", [8.0, 75.0])
def test_attention_of_large_scores_that_hardly_differ(rows, H, Hkv, D, size):
    """Scores of up to thousands whose differences of about one decide.  A score is
    the sum over groups of s (q . c) + m sum(q) with codes c from 0 to 15: roundings
    in fp32 of sums up to 15 s sum|q| + |m sum(q)|, by half a step, 2^-24 of that, and
    2^-24 / root 3 in the rms.  There are four a group (two products of 32 terms, two
    multiply-adds); an error d of a score changes the output by p d (v - o)."""
    print(f"attn alike rows={rows} H={H}/{Hkv} D={D} size={size}", flush=True)
    rng = np.random.default_rng(8)
    T, G = 200, D // 64
    c = Cache([T], Hkv, D, 64, rng)
    k, v = c.fill([alike_keys(T, Hkv, D, rng, size)], draw_rows([T], Hkv * D, rng))
    q = rng.standard_normal((rows, H, G, 64)) * 4
    q[..., :16] *= 0.1 / size
    q = q.reshape(rows, H * D).astype(np.float16)
    got = attend(c, q, [rows], H)[:rows].astype(np.float64).reshape(rows, H, D)
    x, kk, vv = q.reshape(rows, H, D).astype(np.float64), *(np.repeat(y[0], H // Hkv, 1) for y in (k, v))
    s = np.einsum("nhd,thd->nht", x, kk)
    g, xg = kk.reshape(T, H, G, 64), x.reshape(rows, H, G, 64)
    mn, sc = g.min(-1), (g.max(-1) - g.min(-1)) / 15
    top = np.sqrt(np.einsum("nhg,thg->nht", np.abs(xg).sum(-1) ** 2, (15 * sc) ** 2) +
                  np.einsum("nhg,thg->nht", xg.sum(-1) ** 2, mn ** 2))
    err = np.sqrt(4 / 3) * 2.0 ** -24 * top
    p = np.where(np.arange(T)[None] <= (T - rows + np.arange(rows))[:, None], 1.0, 0.0)[:, None] * np.exp(
        s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o = np.einsum("nht,thd->nhd", p, vv)
    off = sum(((p[..., t] * err[..., t])[..., None] * (vv[t] - o)) ** 2 for t in range(T))
    many = rows * H // Hkv > 64                    # whose weights are rounded as well
    tol = 1.1 * np.sqrt(2 if many else 1) * HALF / np.sqrt(3) * np.sqrt((o * o).mean()) + np.sqrt(off.mean())
    assert np.sqrt(((got - o) ** 2).mean()) <= tol


@pytest.mark.parametrize("n,width,ps,n_pages", [(1, 1, 16, 1), (3, 4, 16, 9), (15, 7, 16, 100), (17, 3, 16, 50),
                                                (300, 5, 256, 1500), (1030, 3, 64, 5000),
                                                (2048, 3, 16, 5000)])
@pytest.mark.parametrize("inplace", [False, True])
def test_resize_counts_every_page_that_is_lacking(n, width, ps, n_pages, inplace):
    """Rows far too short, alone and beside others that grow: up to 2^38 pages."""
    print(f"resize lacking n={n} width={width} ps={ps}", flush=True)
    rng = np.random.default_rng(n)
    t = np.full((n, width), -1, np.int32)
    t[0, 0] = 0
    lens = np.zeros(n, np.int32)
    lens[0] = 5
    some = np.where(rng.random(n) < 0.5, rng.integers(0, width * ps + 1, n), -1)
    for want in (np.full(n, 2 ** 31 - 1), np.where(np.arange(n) == n - 1, 2 ** 31 - 1, some),
                 np.where(np.arange(n) % 7 == 0, width * ps + 1 + ps * 600000, some),
                 np.full(n, width * ps + 1)):
        want = want.astype(np.int32)
        a, b, lack = O.resize(t, lens.tolist(), want.tolist(), n_pages, ps)
        dt, dl, dw, dm = dev(t), dev(lens), dev(want), dev(np.full(1, 77, np.int32))
        ot, ol = (dt, dl) if inplace else (DB(t.nbytes), DB(lens.nbytes))
        B.pipo_op_kv_pages_resize(dt.ptr, dl.ptr, dw.ptr, ot.ptr, ol.ptr, width, n, n_pages, ps, dm.ptr)
        B.pipo_dev_synchronize()
        assert lack > 0 and dm.to_array(np.int32, (1,))[0] == min(lack, 2 ** 31 - 1)
        assert np.array_equal(ol.to_array(np.int32, (n,)), lens)
        assert np.array_equal(ot.to_array(np.int32, t.shape), t)
