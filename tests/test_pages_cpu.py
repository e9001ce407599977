"""Refusals of the calls on a paged 4-bit KV cache, without a GPU: nothing is
launched for arguments that a kernel could not take."""
import numpy as np
import pytest

from oracle import pages as O
from paper_2504_03664_amd import binding as B

P = 1 << 20     # an address that no refused call touches


def cache(**kw):
    base = dict(pool=P, layer_bytes=1 << 30, table=P, table_stride=8, n_layers=2, n_pages=100,
                page_size=64, n_kv_heads=8, head_dim=128, n_seq=4)
    base.update(kw)
    return B.PipoKvPages(**base)


def status(fn, *args):
    with pytest.raises(B.PipoError) as e:
        fn(*args)
    assert B.pipo_last_error() != ""
    return B.STATUS_NAMES[e.value.status]


def test_page_bytes():
    assert B.pipo_kv_page_bytes(64, 8, 128) == 64 * 8 * 144
    assert B.pipo_kv_page_bytes(16, 1, 64) == 16 * 72
    for ps, h, d in ((8, 8, 128), (48, 8, 128), (512, 8, 128), (64, 0, 128), (64, 8, 96), (-64, 1, 64),
                     (256, 1 << 17, 128)):
        assert B.pipo_kv_page_bytes(ps, h, d) == 0


BAD_CACHES = [
    (dict(pool=None), "PIPO_ERR_ARG"), (dict(table=None), "PIPO_ERR_ARG"),
    (dict(pool=P + 8), "PIPO_ERR_ARG"), (dict(n_pages=0), "PIPO_ERR_ARG"),
    (dict(n_seq=0), "PIPO_ERR_ARG"), (dict(table_stride=0), "PIPO_ERR_ARG"),
    (dict(layer_bytes=100 * 64 * 8 * 144 - 16), "PIPO_ERR_ARG"),
    (dict(layer_bytes=100 * 64 * 8 * 144 + 8), "PIPO_ERR_ARG"),
    (dict(n_layers=0), "PIPO_ERR_ARG"), (dict(page_size=24), "PIPO_ERR_UNSUPPORTED"),
    (dict(head_dim=96), "PIPO_ERR_UNSUPPORTED"), (dict(n_kv_heads=0), "PIPO_ERR_UNSUPPORTED"),
]


@pytest.mark.parametrize("kw,want", BAD_CACHES)
def test_bad_caches(kw, want):
    c = cache(**kw)
    assert status(B.pipo_op_kv_pages_append, c, 0, P, P, P, 1024, P, 1024, 1) == want
    assert status(B.pipo_op_kv_pages_read, c, 0, P, P, P, 1024, P, 1024, 1) == want
    assert status(B.pipo_op_attn_pages, c, 0, P, 4096, P, P, P, 4096, 32, 4, 1, 512) == want
    assert status(B.pipo_op_kv_pages_copy, c, P, P, 1) == want


@pytest.mark.parametrize("layer", [-1, 2])
def test_bad_layers(layer):
    assert status(B.pipo_op_kv_pages_append, cache(), layer, P, P, P, 1024, P, 1024, 1) == "PIPO_ERR_ARG"
    assert status(B.pipo_op_attn_pages, cache(), layer, P, 4096, P, P, P, 4096, 32, 4, 1,
                  512) == "PIPO_ERR_ARG"


@pytest.mark.parametrize("kw,want", [
    (dict(seq=None), "PIPO_ERR_ARG"), (dict(pos=None), "PIPO_ERR_ARG"), (dict(k=None), "PIPO_ERR_ARG"),
    (dict(v=None), "PIPO_ERR_ARG"), (dict(ldk=1023), "PIPO_ERR_ARG"), (dict(ldv=0), "PIPO_ERR_ARG"),
    (dict(M=-1), "PIPO_ERR_ARG"), (dict(M=1 << 31), "PIPO_ERR_UNSUPPORTED")])
def test_bad_rows(kw, want):
    a = dict(seq=P, pos=P, k=P, ldk=1024, v=P, ldv=1024, M=1)
    a.update(kw)
    assert status(B.pipo_op_kv_pages_append, cache(), 0, *a.values()) == want
    assert status(B.pipo_op_kv_pages_read, cache(), 0, *a.values()) == want


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), "PIPO_ERR_ARG"), (dict(q_start=None), "PIPO_ERR_ARG"),
    (dict(kv_len=None), "PIPO_ERR_ARG"), (dict(o=None), "PIPO_ERR_ARG"),
    (dict(ldq=4095), "PIPO_ERR_ARG"), (dict(ldo=4095), "PIPO_ERR_ARG"),
    (dict(n_heads=33), "PIPO_ERR_ARG"), (dict(n_heads=0), "PIPO_ERR_ARG"), (dict(M=-1), "PIPO_ERR_ARG"),
    (dict(max_q=-1), "PIPO_ERR_ARG"), (dict(max_len=513), "PIPO_ERR_ARG"),
    (dict(max_len=-1), "PIPO_ERR_ARG"), (dict(wsb=-1), "PIPO_ERR_ARG"),
    (dict(M=1 << 26), "PIPO_ERR_UNSUPPORTED"),
    (dict(M=1 << 25, max_q=1 << 25), "PIPO_ERR_UNSUPPORTED"),
    (dict(n_heads=65536, ldq=1 << 24, ldo=1 << 24), "PIPO_ERR_UNSUPPORTED")])
def test_bad_attention(kw, want):
    a = dict(q=P, ldq=4096, q_start=P, kv_len=P, o=P, ldo=4096, n_heads=32, M=4, max_q=1, max_len=512,
             ws=None, wsb=0)
    a.update(kw)
    assert status(B.pipo_op_attn_pages, cache(), 0, *a.values()) == want


def test_attention_workspace():
    c = cache(n_seq=1, table_stride=1024, pool=None, table=None)
    n = B.pipo_op_attn_pages_workspace_bytes(c, 32, 1, 1, 65536)
    assert n > 0 and n % (32 * 130 * 4) == 0
    assert B.pipo_op_attn_pages_workspace_bytes(c, 33, 1, 1, 65536) == 0
    assert B.pipo_op_attn_pages_workspace_bytes(c, 32, 0, 1, 65536) == 0
    assert B.pipo_op_attn_pages_workspace_bytes(c, 32, 1, 1, 100) == 0       # too short to split
    many = cache(n_seq=4096, table_stride=1024, pool=None, table=None)
    assert B.pipo_op_attn_pages_workspace_bytes(many, 32, 4096, 1, 4096) == 0  # enough workgroups


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), "PIPO_ERR_ARG"), (dict(k_out=None), "PIPO_ERR_ARG"), (dict(pos=None), "PIPO_ERR_ARG"),
    (dict(cs=None), "PIPO_ERR_ARG"), (dict(ldq=511), "PIPO_ERR_ARG"), (dict(ldk=255), "PIPO_ERR_ARG"),
    (dict(ldqo=0), "PIPO_ERR_ARG"), (dict(ldko=255), "PIPO_ERR_ARG"), (dict(M=-1), "PIPO_ERR_ARG"),
    (dict(H=0), "PIPO_ERR_ARG"), (dict(Hkv=0), "PIPO_ERR_ARG"), (dict(n_pos=0), "PIPO_ERR_ARG"),
    (dict(eps=-1.0), "PIPO_ERR_ARG"), (dict(eps=float("nan")), "PIPO_ERR_ARG"),
    (dict(D=96), "PIPO_ERR_UNSUPPORTED"), (dict(M=1 << 31), "PIPO_ERR_UNSUPPORTED")])
def test_bad_norm_rope(kw, want):
    a = dict(q=P, ldq=512, k=P, ldk=256, gq=P, gk=P, cs=P, n_pos=10, pos=P, q_out=P, ldqo=512, k_out=P,
             ldko=256, M=3, H=4, Hkv=2, D=128, eps=1e-5, scale=1.0)
    a.update(kw)
    assert status(B.pipo_op_qk_norm_rope, *a.values()) == want


TABLES = dict(table=P, len=2 * P, want=3 * P, out=4 * P, len_out=5 * P, stride=8, n=4, pages=100, ps=64)


@pytest.mark.parametrize("kw,want", [
    (dict(table=None), "PIPO_ERR_ARG"), (dict(len=None), "PIPO_ERR_ARG"), (dict(want=None), "PIPO_ERR_ARG"),
    (dict(out=None), "PIPO_ERR_ARG"), (dict(len_out=None), "PIPO_ERR_ARG"), (dict(stride=0), "PIPO_ERR_ARG"),
    (dict(n=0), "PIPO_ERR_ARG"), (dict(pages=0), "PIPO_ERR_ARG"), (dict(ps=15), "PIPO_ERR_ARG"),
    (dict(ps=0), "PIPO_ERR_ARG"), (dict(out=P + 4), "PIPO_ERR_ARG"),       # shifted by one entry
    (dict(len_out=2 * P + 4), "PIPO_ERR_ARG"), (dict(len_out=3 * P), "PIPO_ERR_ARG"),
    (dict(len_out=P + 8), "PIPO_ERR_ARG"), (dict(missing=P), "PIPO_ERR_ARG"),
    (dict(missing=None), "PIPO_ERR_ARG"), (dict(n=2049), "PIPO_ERR_UNSUPPORTED"),
    (dict(pages=(1 << 20) + 1), "PIPO_ERR_UNSUPPORTED"), (dict(stride=1 << 30), "PIPO_ERR_UNSUPPORTED")])
def test_bad_resize(kw, want):
    a = dict(TABLES, missing=6 * P)
    a.update(kw)
    assert status(B.pipo_op_kv_pages_resize, *a.values()) == want


@pytest.mark.parametrize("kw,want", [
    (dict(parent=None), "PIPO_ERR_ARG"), (dict(n_out=0), "PIPO_ERR_ARG"), (dict(out=P), "PIPO_ERR_ARG"),
    (dict(len_out=2 * P), "PIPO_ERR_ARG"), (dict(pairs=None), "PIPO_ERR_ARG"),
    (dict(n_pairs=7 * P), "PIPO_ERR_ARG"), (dict(missing=8 * P), "PIPO_ERR_ARG"),
    (dict(pairs=4 * P + 16), "PIPO_ERR_ARG"), (dict(ps=31), "PIPO_ERR_ARG"),
    (dict(n_out=2049), "PIPO_ERR_UNSUPPORTED"), (dict(n=2049), "PIPO_ERR_UNSUPPORTED"),
    (dict(pages=1 << 21), "PIPO_ERR_UNSUPPORTED")])
def test_bad_fork(kw, want):
    a = dict(table=P, len=2 * P, n=4, parent=3 * P, out=4 * P, len_out=5 * P, n_out=6, stride=8,
             pages=100, ps=64, pairs=7 * P, n_pairs=8 * P, missing=9 * P)
    a.update(kw)
    assert status(B.pipo_op_kv_pages_fork, *a.values()) == want


@pytest.mark.parametrize("kw,want", [
    (dict(table=None), "PIPO_ERR_ARG"), (dict(out=P + 4), "PIPO_ERR_ARG"), (dict(out=2 * P), "PIPO_ERR_ARG"),
    (dict(pairs=None), "PIPO_ERR_ARG"), (dict(n_pairs=7 * P + 4), "PIPO_ERR_ARG"),
    (dict(pairs=4 * P), "PIPO_ERR_ARG"), (dict(pages=(1 << 20) + 1), "PIPO_ERR_UNSUPPORTED")])
def test_bad_compact(kw, want):
    a = dict(table=P, len=2 * P, out=4 * P, stride=8, n=4, pages=100, ps=64, pairs=7 * P, n_pairs=8 * P)
    a.update(kw)
    assert status(B.pipo_op_kv_pages_compact, *a.values()) == want


@pytest.mark.parametrize("kw", [dict(pairs=None), dict(n_pairs=None), dict(n=-1)])
def test_bad_copy(kw):
    a = dict(pairs=P, n_pairs=P, n=1)
    a.update(kw)
    assert status(B.pipo_op_kv_pages_copy, cache(), *a.values()) == "PIPO_ERR_ARG"


def test_nothing_to_do_launches_nothing():
    """No rows and no pairs succeed without a device."""
    B.pipo_op_kv_pages_append(cache(), 0, P, P, P, 1024, P, 1024, 0)
    B.pipo_op_kv_pages_read(cache(), 1, P, P, P, 1024, P, 1024, 0)
    B.pipo_op_attn_pages(cache(), 0, P, 4096, P, P, P, 4096, 32, 0, 1, 512)
    B.pipo_op_attn_pages(cache(), 0, P, 4096, P, P, P, 4096, 32, 4, 0, 512)
    B.pipo_op_qk_norm_rope(P, 512, P, 256, P, P, P, 10, P, P, 512, P, 256, 0, 4, 2, 128, 1e-5, 1.0)
    B.pipo_op_kv_pages_copy(cache(), P, P, 0)


# --- the oracle's own definitions ---
def test_oracle_tables():
    table = np.array([[3, 5, -1], [7, -1, -1], [2, 6, 9]], np.int32)
    lens = [20, 16, 40]
    t, n, lack = O.resize(table, lens, [33, 0, -1], 10, 16)
    assert t.tolist() == [[3, 5, 0], [-1, -1, -1], [2, 6, 9]] and n.tolist() == [33, 0, 40] and lack == 0
    t, n, lack = O.resize(table, lens, [49, 17, 0], 4, 16)      # one entry past the row
    assert lack == 1 and n.tolist() == lens and t.tolist() == table.tolist()
    t, n, pairs, lack = O.fork(table, lens, [0, 0, 2, -1, 0, 1, 1], 12, 16)
    assert pairs == [(5, 0), (5, 1)] and lack == 0 and n.tolist() == [20, 20, 40, 0, 20, 16, 16]
    assert t.tolist() == [[3, 5, -1], [3, 0, -1], [2, 6, 9], [-1] * 3, [3, 1, -1], [7, -1, -1], [7, -1, -1]]
    t, pairs = O.compact(table, lens, 12, 16)
    assert pairs == [(6, 0), (7, 1), (9, 4)]
    assert t.tolist() == [[3, 5, -1], [1, -1, -1], [2, 0, 4]]


def test_oracle_attention_of_rows_that_see_nothing():
    q, k = np.ones((2, 2, 64)), np.ones((3, 1, 64))
    out = O.page_attention(q, k, 5 * k, np.array([[False] * 3, [True, False, False]]))
    assert (out[0] == 0).all() and (out[1] == 5).all()
