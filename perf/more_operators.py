"""The paged 8-bit cache's operators and the draw of the next tokens: what they
are measured on, their plain forms and their 64-bit values.

A batch of sequences of different lengths keeps keys and values in pages of
8-bit codes with a scale for every 16 positions of a head (pipo_kv8_pages in
include/pipo_ops.h); a step ends with a token drawn for each sequence.  The kinds of case:

  append   new rows' k and v into their pages, the scales of blocks that were
           begun before growing with them, and the newest positions read back
  attn     attention of each sequence's newest rows over its pages; the scores
           plain, capped, with a bias by distance, in a window, with a prefix
  sample   a token for each row of logits: temperature, top-k, min-p, top-p and
           a given random number

Sizes are those of the workloads this repository runs (OPT-125m / 13B / 30B and
LLaMA-3.1-8B heads and vocabularies, batch 1 to 128, prompts of 32 to 512
tokens) with contexts up to 65536 tokens; draw() spreads over the ranges between and
around them.
"""
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEV = "cuda"
CLAMP = 57344.0                 # of an element before it is quantized
TOP = {"e4m3": 448.0, "int8": 127.0}
LOW, HIGH = {"e4m3": -15, "int8": -24}, {"e4m3": 7, "int8": 9}   # exponents of a scale
TOP_WORK = 1.2e12               # flops of the largest attention case
TOP_CACHE = 4.5e8               # padded cache elements (sequences x longest x Hkv x D)
TOP_LOGITS = 128 * 128256


def _attn(name, n, H, Hkv, D, ps, lo, hi, nq=1, long=0, fmt="e4m3", cap=0.0, slopes=False, window=0,
          prefix=0):
    return dict(name=name, kind="attn", n=n, H=H, Hkv=Hkv, D=D, ps=ps, lo=lo, hi=hi, nq=nq, long=long,
                fmt=fmt, cap=cap, slopes=slopes, window=window, prefix=prefix)


# ---------------------------------------------------------------------------
def listed():
    return [
        # a decode step's new rows, in blocks that earlier tokens began
        dict(name="append_llama8b_b16", kind="append", n=16, nq=1, lo=100, hi=2100, Hkv=8, D=128,
             ps=64, fmt="e4m3"),
        # eight prompts of 512 tokens, every head its own keys
        dict(name="append_opt30b_prompts", kind="append", n=8, nq=512, lo=512, hi=600, Hkv=56,
             D=128, ps=64, fmt="int8"),
        # the smallest model just after short prompts: launch latency
        _attn("attn_opt125m_b4", 4, 12, 12, 64, 16, 33, 40),
        # 16 users at different lengths, grouped heads, capped scores
        _attn("attn_llama8b_b16_cap", 16, 32, 8, 128, 64, 100, 2100, fmt="int8", cap=30.0),
        # one key/value head per query head, a bias by distance
        _attn("attn_opt30b_b64_bias", 64, 56, 56, 128, 32, 513, 544, slopes=True),
        # one user with a long document: the cache split over the chip
        _attn("attn_llama8b_long", 1, 32, 8, 128, 128, 65000, 65000),
        # 32 long conversations that look 1024 tokens back, and at their first 16
        _attn("attn_llama8b_window", 32, 32, 8, 128, 64, 3001, 12007, fmt="int8", window=1024, prefix=16),
        # four long prompts in pieces of 509 tokens
        _attn("attn_llama8b_chunk", 4, 32, 8, 128, 64, 509, 4099, nq=509),
        # eight whole prompts whose first 100 tokens all see each other, scores capped and biased
        _attn("attn_llama8b_prefix", 8, 32, 8, 128, 64, 512, 512, nq=512, fmt="int8", cap=50.0,
              slopes=True, prefix=100),
        # one sequence's next token
        dict(name="sample_opt_b1", kind="sample", rows=1, V=50272, ld=50272, T=0.8, k=0, p=0.9, m=0.0,
             mixed=False, std=2.5),
        # 64 users, each with settings of their own, some greedy; a padded row
        dict(name="sample_llama8b_b64", kind="sample", rows=64, V=128256, ld=128384, T=0.7, k=50, p=0.9,
             m=0.02, mixed=True, std=2.5),
        # 128 users draw from everything
        dict(name="sample_llama8b_b128", kind="sample", rows=128, V=128256, ld=128256, T=1.0, k=0, p=1.0,
             m=0.0, mixed=False, std=2.0),
    ]


LONG = 509          # tokens of the prompts in a mixed batch


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "attn", "sample"])
    if kind == "sample":
        V = _log(rng, 500, 256000)
        rows = max(1, min(_log(rng, 1, 256), TOP_LOGITS // (V + 64)))
        return dict(kind=kind, rows=rows, V=V, ld=V + rng.choice([0, 0, 1, 64]),
                    T=round(rng.uniform(0.3, 1.5), 3), k=rng.choice([0, 1, 20, 50, _log(rng, 2, V)]),
                    p=rng.choice([1.0, 0.5, 0.9, 0.95, 0.99]), m=rng.choice([0.0, 0.0, 0.01, 0.1]),
                    mixed=rng.random() < 0.5, std=round(rng.uniform(0.5, 4.0), 2))
    D, fmt, ps = rng.choice([64, 128, 128]), rng.choice(["e4m3", "int8"]), rng.choice([16, 32, 64, 128, 256])
    if kind == "append":
        Hkv = rng.randint(1, 56)
        n, nq = _log(rng, 1, 128), _log(rng, 1, 1024) if rng.random() < 0.5 else 1
        nq = max(1, min(nq, 8 * 512 * 56 * 128 // (n * Hkv * D)))
        lo = nq + rng.randint(0, 500)
        return dict(kind=kind, n=n, nq=nq, lo=lo, hi=lo + rng.randint(0, 600), Hkv=Hkv, D=D, ps=ps,
                    fmt=fmt)
    G = rng.choice([1, 1, 2, 3, 4, 4, 5, 7, 8, 16])
    Hkv = rng.randint(1, 8) if G > 1 else rng.randint(1, 56)
    shape = rng.choice(["one", "one", "one", "few", "chunk", "mixed"])
    nq = {"one": 1, "few": rng.randint(2, 8), "chunk": _log(rng, 17, 1024), "mixed": 1}[shape]
    long = rng.randint(1, 3) if shape == "mixed" else 0
    n = _log(rng, 1, 8) if shape == "chunk" else _log(rng, 4, 32) if long else _log(rng, 1, 128)
    floor = LONG if long else nq
    hi = max(floor + 1, _log(rng, 33, 65536))
    hi = max(floor + 1, min(hi, int(TOP_CACHE / (n * Hkv * D))))
    hi = max(floor + 1, min(hi, int(TOP_WORK / (4 * n * floor * G * Hkv * D))))
    c = _attn("", n, G * Hkv, Hkv, D, ps, rng.randint(floor, hi), hi, nq, long, fmt,
              rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.3,
              rng.choice([0, 0, _log(rng, 16, 8192)]), rng.choice([0, 0, rng.randint(1, 200)]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# shapes of a case (not of its seed)
def _lens(c):
    n = c["n"]
    return [c["lo"] + (c["hi"] - c["lo"]) * (i * 37 % n) // max(n - 1, 1) for i in range(n)]


def _rows(c):
    """new rows of each sequence"""
    return [LONG if i < c.get("long", 0) else c["nq"] for i in range(c["n"])]


def _back(c):
    """positions of each sequence that are read back: the new ones, 16 at least"""
    return [min(n, max(r, 16)) for n, r in zip(_lens(c), _rows(c))]


def _code_bytes(c):
    return c["Hkv"] * c["ps"] * 2 * c["D"]


def _page_bytes(c):
    return _code_bytes(c) + -(-c["Hkv"] * c["ps"] // 16 * 8 // 128) * 128


def work(case):
    c = case
    if c["kind"] == "sample":
        return {"bytes": c["rows"] * (4 * c["V"] + 28), "flops": 0}
    D, Hkv = c["D"], c["Hkv"]
    if c["kind"] == "append":
        M, back = c["n"] * c["nq"], sum(_back(c))
        # halves in and codes out; codes in and halves out
        return {"bytes": (M + back) * 2 * Hkv * D * 3, "flops": 0}
    keys = pairs = 0
    for n, r in zip(_lens(c), _rows(c)):
        at = np.arange(n - r, n)
        first = np.maximum(at - (c["window"] or n) + 1, 0)
        pre = min(c["prefix"], n)
        # seen in the window, and of the prefix what is before it or ahead of the row
        seen = at + 1 - first + np.minimum(first, pre) + np.maximum(pre - at - 1, 0)
        pairs += int(seen.sum())
        keys += n - int(first[0]) + min(int(first[0]), pre)
    return {"bytes": keys * Hkv * D * 2 + sum(_rows(c)) * c["H"] * D * 4, "flops": 4 * D * c["H"] * pairs}


def _table(c, rng, extra):
    """Pages in random order: (table [n][width], pages in the pool)."""
    need = [-(-n // c["ps"]) for n in _lens(c)]
    n_pages = sum(need) + extra
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((c["n"], max(need) + 3), -1, np.int32)
    at = 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    return table, n_pages


# ---------------------------------------------------------------------------
# the pages' layout (pipo_kv8_pages in include/pipo_ops.h), written out in
# elementary operations: the tiles of 16 keys of each head, in them K codes and V codes,
# and behind all tiles of the page the scales (K, V) of each
def _round(x, fmt):
    """fp32 in units of the scale -> codes as bytes"""
    if fmt == "int8":
        return x.round().to(torch.int8).view(torch.uint8)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def _units(b, fmt):
    """codes as bytes -> fp32 in units of the scale"""
    return b.view(torch.int8).float() if fmt == "int8" else b.view(torch.float8_e4m3fn).float()


def _scale(amax, fmt):
    """the least power of two that holds the largest magnitude"""
    m, e = torch.frexp(amax)                                   # amax = m 2^e, 0.5 <= m < 1
    t, x = np.frexp(np.float32(TOP[fmt]))
    e = torch.where(m <= float(t), e - int(x), e - int(x) + 1)
    e = torch.where(amax > 0, e, LOW[fmt]).clamp(LOW[fmt], HIGH[fmt])
    return torch.ldexp(torch.ones_like(amax), e)


def _k_bytes(x):
    """[..., 16, D] -> [..., 16 D]: byte 1024 c + 16 (key + 16 g) + 8 j + b holds dimension
    64 c + 32 j + 8 g + b"""
    D, lead = x.shape[-1], x.shape[:-2]
    return x.reshape(-1, 16, D // 64, 2, 4, 8).permute(0, 2, 4, 1, 3, 5).reshape(*lead, 16 * D)


def _v_bytes(x):
    """[..., 16, D] -> [..., 16 D]: byte 1024 c + 16 (r + 16 g) + 4 m + b holds key 4 g + b,
    dimension 64 c + 16 m + r"""
    D, lead = x.shape[-1], x.shape[:-2]
    return x.reshape(-1, 4, 4, D // 64, 4, 16).permute(0, 3, 1, 5, 4, 2).reshape(*lead, 16 * D)


def _k_rows(b, D):
    x = b.reshape(-1, D // 64, 4, 16, 2, 8).permute(0, 3, 1, 4, 2, 5)
    return x.reshape(*b.shape[:-1], 16, D)


def _v_rows(b, D):
    x = b.reshape(-1, D // 64, 4, 16, 4, 4).permute(0, 2, 5, 1, 4, 3)
    return x.reshape(*b.shape[:-1], 16, D)


def _codes(s, pool=None):
    """view [page, head, tile, 32 D] of the pool's codes"""
    c, pool = s.c, s.pool if pool is None else pool
    return pool[:, :_code_bytes(c)].view(-1, c["Hkv"], c["ps"] // 16, 32 * c["D"])


def _scales(s, pool=None):
    """view [page, head, tile, 2] of the pool's scales"""
    c, pool = s.c, s.pool if pool is None else pool
    f, n = pool.view(torch.float32), c["Hkv"] * (c["ps"] // 16) * 2
    return f[:, _code_bytes(c) // 4:_code_bytes(c) // 4 + n].view(-1, c["Hkv"], c["ps"] // 16, 2)


# ---------------------------------------------------------------------------
# inputs
def _gen(seed, *salt):
    s = seed
    for v in salt:
        s = (s * 1000003 + v + 1) % (1 << 62)
    return torch.Generator(DEV).manual_seed(s)


def _normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std).half()


def _int(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


def _prepare_sample(s, seed):
    c, g = s.c, _gen(seed, 5)
    rows, V = c["rows"], c["V"]
    s.full = torch.randn(rows, c["ld"], generator=g, device=DEV) * c["std"]
    s.logits = s.full[:, :V]
    # some tokens are likely, some are not allowed
    at = torch.randint(0, V, (rows, max(1, V // 1000)), generator=g, device=DEV)
    s.logits.scatter_add_(1, at, torch.rand(at.shape, generator=g, device=DEV) * 3 * c["std"])
    at = torch.randint(1, V, (rows, V // 50), generator=g, device=DEV)
    s.logits.scatter_(1, at, -float("inf"))
    i = torch.arange(rows, device=DEV)
    s.T = torch.full((rows,), c["T"], device=DEV)
    s.k = torch.full((rows,), c["k"], dtype=torch.int32, device=DEV)
    s.p, s.m = torch.full((rows,), c["p"], device=DEV), torch.full((rows,), c["m"], device=DEV)
    if c["mixed"]:      # greedy ones, and ones without one of the limits
        s.T = torch.where(i % 8 == 7, torch.zeros_like(s.T), s.T * (1 + (i % 5) * 0.1))
        s.k = torch.where(i % 3 == 1, torch.zeros_like(s.k), s.k)
        s.p = torch.where(i % 4 == 2, torch.ones_like(s.p), s.p)
    s.u = torch.rand(rows, generator=g, device=DEV)
    s.next = torch.empty(rows, dtype=torch.int32, device=DEV)
    s.logprob = torch.empty(rows, device=DEV)
    s.ws = None
    return s


def prepare(case, seed):
    c, kind = case, case["kind"]
    s = SimpleNamespace(c=c, kind=kind)
    if kind == "sample":
        return _prepare_sample(s, seed)
    rng = np.random.default_rng(seed % (1 << 63))
    D, Hkv, ps, fmt = c["D"], c["Hkv"], c["ps"], c["fmt"]
    lens, rows = _lens(c), _rows(c)
    table, s.n_pages = _table(c, rng, 64)
    starts = np.concatenate([[0], np.cumsum(rows)])
    s.M, s.max_q, s.max_len = int(starts[-1]), max(rows), max(lens)
    s.table, s.q_start, s.len = _int(table), _int(starts), _int(lens)
    g = _gen(seed, 2)
    gain = torch.exp(0.5 * torch.randn(Hkv, 1, 1, D, generator=g, device=DEV)).half()
    s.pool = torch.zeros(s.n_pages, _page_bytes(c), dtype=torch.uint8, device=DEV)
    codes, scales = _codes(s), _scales(s)
    step = max(1, (1 << 27) // (Hkv * ps * D))
    for p in range(0, s.n_pages, step):
        for i in range(2):
            x = _normal(g, min(step, s.n_pages - p), Hkv, ps // 16, 16, D) * (1 if i else gain)
            x = x.float()
            sc = _scale(x.abs().amax((-1, -2)), fmt)
            b = _round(x / sc[..., None, None], fmt)
            codes[p:p + step, ..., 16 * D * i:16 * D * (i + 1)] = (_v_bytes if i else _k_bytes)(b)
            scales[p:p + step, ..., i] = sc
    if kind == "append":
        # (some rows larger than what their block holds)
        s.kv = _normal(g, s.M, 2 * Hkv * D) * torch.exp(
            0.5 * torch.randn(s.M, 1, generator=g, device=DEV)).half()
        s.k, s.v = s.kv[:, :Hkv * D], s.kv[:, Hkv * D:]
        back = _back(c)
        s.seq = _int(np.repeat(np.arange(c["n"]), back))
        s.pos = _int(np.concatenate([np.arange(n - r, n) for n, r in zip(lens, back)]))
        s.ko, s.vo = (torch.empty(sum(back), Hkv * D, dtype=torch.float16, device=DEV) for _ in "kv")
        return s
    s.q = _normal(g, s.M, c["H"] * D, std=(4.0 if c["cap"] else 1.2) * D ** -0.5)
    s.slopes = 2.0 ** (-8.0 * (torch.arange(c["H"], device=DEV).float() + 1) / c["H"]) if c["slopes"] else None
    # (not all of a batch's prefixes are as long)
    s.prefix = _int([max(0, c["prefix"] - i % 4) for i in range(c["n"])]) if c["prefix"] else None
    s.o = torch.empty_like(s.q)
    s.ws = None
    return s


# ---------------------------------------------------------------------------
# plain forms
def _places(s):
    """sequence and position of every new row"""
    m = torch.arange(s.M, device=DEV)
    seq = torch.searchsorted(s.q_start, m.int(), right=True) - 1
    return m, seq, s.len[seq].long() - s.q_start[seq + 1].long() + m


def _append(s):
    """The blocks that get rows (slots): their old codes, the new rows, a scale for
    both, codes of both; then the values that the newest positions stand for."""
    c, fmt = s.c, s.c["fmt"]
    Hkv, D, ps = c["Hkv"], c["D"], c["ps"]
    m, seq, pos = _places(s)
    first = (s.len.long() - s.q_start.diff().long()) // 16
    slot = s.q_start[seq].long() // 16 + 2 * seq + pos // 16 - first[seq]
    n = s.M // 16 + 2 * c["n"]
    page, tile = torch.zeros(2, n, dtype=torch.long, device=DEV)
    page[slot], tile[slot] = s.table[seq, pos // ps].long(), pos // 16 % (ps // 16)
    new = torch.zeros(n, 16, dtype=torch.bool, device=DEV)
    new[slot, pos % 16] = True
    key = torch.arange(16, device=DEV)
    old = key < torch.where(new, key, 16).amin(1, keepdim=True)
    used = new.any(1)
    begun = (old[:, :1] & used[:, None])[:, :, None, None]      # [slot, 1, 1, 1]
    codes, scales = _codes(s), _scales(s)
    was, sc = codes[page, :, tile], scales[page, :, tile]
    out, out_scale = [], []
    for i, x in enumerate((s.k, s.v)):
        x = x.float()
        x = torch.where(x != x, torch.zeros_like(x), x).clamp(-CLAMP, CLAMP)
        rows = torch.zeros(n, 16, Hkv, D, device=DEV)
        rows[slot, pos % 16] = x.view(s.M, Hkv, D)
        rows = rows.transpose(1, 2)
        before = sc[..., i, None, None]
        scale = _scale(rows.abs().amax((-1, -2), keepdim=True), fmt)
        scale = torch.where(begun, torch.maximum(scale, before), scale)
        b = (_v_rows if i else _k_rows)(was[..., 16 * D * i:16 * D * (i + 1)], D)
        kept = _round(_units(b.contiguous(), fmt) * (before / scale), fmt)
        mine = lambda mask: mask[:, None, :, None]  # noqa: E731
        b = torch.where(mine(new), _round(rows / scale, fmt), torch.where(mine(old), kept, b))
        out.append((_v_bytes if i else _k_bytes)(b))
        out_scale.append(scale[..., 0, 0])
    keep = lambda x: x[used]  # noqa: E731
    codes[keep(page), :, keep(tile)] = keep(torch.cat(out, -1))
    scales[keep(page), :, keep(tile)] = keep(torch.stack(out_scale, -1))
    p, seq = s.pos.long(), s.seq.long()
    page, tile = s.table[seq, p // ps].long(), p // 16 % (ps // 16)
    d = torch.arange(D, device=DEV)
    kat = 1024 * (d // 64) + 16 * ((p % 16)[:, None] + 16 * (d % 32 // 8)) + 8 * (d % 64 // 32) + d % 8
    vat = 16 * D + 1024 * (d // 64) + 16 * (d % 16 + 16 * (p % 16 // 4)[:, None]) + 4 * (
        d % 64 // 16) + (p % 4)[:, None]
    h = torch.arange(Hkv, device=DEV)[None, :, None]
    return [(_units(codes[page[:, None, None], h, tile[:, None, None], at[:, None]], fmt)
             * scales[page, :, tile, i][..., None]).half().view(-1, Hkv * D)
            for i, at in enumerate((kat, vat))]


def _attention(s):
    c = s.c
    n, H, Hkv, D, ps = c["n"], c["H"], c["Hkv"], c["D"], c["ps"]
    G, pages = H // Hkv, -(-s.max_len // ps)
    L = pages * ps
    t = s.table[:, :pages].clamp(min=0).long()
    codes, scales = _codes(s)[t].transpose(1, 2), _scales(s)[t].transpose(1, 2)   # n, Hkv, page, tile
    k = _units(_k_rows(codes[..., :16 * D], D), c["fmt"]) * scales[..., 0, None, None]
    v = _units(_v_rows(codes[..., 16 * D:], D), c["fmt"]) * scales[..., 1, None, None]
    k, v = k.reshape(n, Hkv, L, D), v.reshape(n, Hkv, L, D)
    m, seq, pos = _places(s)
    rows, j = s.q_start.diff().long(), torch.arange(s.max_q, device=DEV)
    row = (s.q_start[:-1, None] + j).clamp(max=s.M - 1).long()
    q = s.q[row].float().view(n, s.max_q, Hkv, G, D).transpose(1, 2).reshape(n, Hkv, s.max_q * G, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(n, Hkv, s.max_q, G, L)
    if c["cap"]:
        x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
    last, key = ((s.len.long() - rows)[:, None] + j)[..., None], torch.arange(L, device=DEV)
    if c["slopes"]:
        far = (last - key).abs().float()[:, None, :, None]
        x = x.sub_(far * s.slopes.view(1, Hkv, 1, G, 1))
    seen = key <= last
    if c["window"]:
        seen = seen & (last - key < c["window"])
    if c["prefix"]:
        seen = seen | (key < s.prefix[:, None, None])
    seen = seen & (key < s.len[:, None, None])
    x = x.masked_fill_(~seen[:, None, :, None], -float("inf"))
    x = x.sub_(x.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(n, Hkv, s.max_q * G, L), v).view(n, Hkv, s.max_q, G, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).transpose(1, 2)
    return o[seq, m - s.q_start[seq].long()].reshape(s.M, H * D).half()


def _sample(s):
    """In the order of falling logits (equal ones by index): the first k, of them those of
    at least m times the largest's weight, of these the shortest run with a share of p,
    and in it the token at which the running share passes u."""
    x = s.logits
    x = torch.where(x != x, -float("inf"), x)
    x, order = torch.sort(x, dim=-1, descending=True, stable=True)
    x, top = x.double(), x[:, :1].double()
    T = torch.where(s.T > 0, s.T, torch.ones_like(s.T)).double()[:, None]
    z = torch.where(x == top, 0.0, (x - top) / T)
    w = z.exp()
    rank = torch.arange(x.shape[1], device=DEV)
    k = torch.where((s.k > 0) & (s.k < x.shape[1]), s.k, x.shape[1])
    k = torch.where(s.T > 0, k, 1)[:, None]
    w = torch.where((rank < k) & (w >= s.m.double().clamp(max=1)[:, None]), w, 0.0)
    run = w.cumsum(-1)
    before = torch.cat([torch.zeros_like(run[:, :1]), run[:, :-1]], -1)
    keep = (w > 0) & ((before < s.p.double()[:, None] * run[:, -1:]) | (rank == 0))
    total = torch.where(keep, w, 0.0).sum(-1, keepdim=True)
    at = ((run <= s.u.double()[:, None] * total) & keep).sum(-1, keepdim=True)
    at = torch.minimum(at, keep.sum(-1, keepdim=True) - 1)
    return [order.gather(1, at)[:, 0].int(), (z.gather(1, at) - total.log())[:, 0].float()]


# ---------------------------------------------------------------------------
# the framework's calls
def _stream():
    return torch.cuda.current_stream().cuda_stream


def _cache(s):
    from paper_2504_03664_amd import binding as B
    c = s.c
    fmt = B.PIPO_KV8_INT8 if c["fmt"] == "int8" else B.PIPO_KV8_E4M3
    return B.PipoKv8Pages(s.pool.data_ptr(), _page_bytes(c) * s.n_pages, s.table.data_ptr(),
                          s.table.shape[1], 1, s.n_pages, c["ps"], c["Hkv"], c["D"], c["n"], fmt)


def _run_own(s):
    from paper_2504_03664_amd import binding as B
    c, st = s.c, _stream()
    if s.kind == "sample":
        if s.ws is None:
            n = B.pipo_op_sample_workspace_bytes(c["rows"], c["V"])
            s.ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
        B.pipo_op_sample(s.logits.data_ptr(), s.logits.stride(0), s.T.data_ptr(), s.k.data_ptr(),
                         s.p.data_ptr(), s.m.data_ptr(), s.u.data_ptr(), s.next.data_ptr(),
                         s.logprob.data_ptr(), c["rows"], c["V"], s.ws.data_ptr(), s.ws.numel(), st)
        return [s.next, s.logprob]
    if getattr(s, "cache", None) is None:
        s.cache = _cache(s)
    if s.kind == "append":
        B.pipo_op_kv8_pages_append(s.cache, 0, s.q_start.data_ptr(), s.len.data_ptr(), s.k.data_ptr(),
                                   s.k.stride(0), s.v.data_ptr(), s.v.stride(0), s.M, st)
        B.pipo_op_kv8_pages_read(s.cache, 0, s.seq.data_ptr(), s.pos.data_ptr(), s.ko.data_ptr(),
                                 s.ko.stride(0), s.vo.data_ptr(), s.vo.stride(0), s.ko.shape[0], st)
        return [s.ko, s.vo]
    if s.ws is None:
        s.scores = B.PipoAttnScores(c["cap"], c["window"], s.slopes.data_ptr() if c["slopes"] else None,
                                    s.prefix.data_ptr() if c["prefix"] else None, c["prefix"])
        n = B.pipo_op_attn_kv8_pages_workspace_bytes(s.cache, s.scores, c["H"], s.M, s.max_q, s.max_len)
        s.ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
    B.pipo_op_attn_kv8_pages(s.cache, 0, s.scores, s.q.data_ptr(), s.q.stride(0), s.q_start.data_ptr(),
                             s.len.data_ptr(), s.o.data_ptr(), s.o.stride(0), c["H"], s.M, s.max_q,
                             s.max_len, s.ws.data_ptr(), s.ws.numel(), st)
    return s.o


def run(state):
    if own:
        return _run_own(state)
    return {"append": _append, "attn": _attention, "sample": _sample}[state.kind](state)


# ---------------------------------------------------------------------------
# 64-bit values
def _number(code, fmt):
    """what a code stands for, from its bits"""
    code = code.to(torch.int64)
    if fmt == "int8":
        return (code - 256 * (code > 127)).double()
    e, m = code >> 3 & 15, (code & 7).double()
    x = torch.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7).double(), m * 2.0 ** -9)
    return torch.where(code > 127, -x, x)


def _element(s, page, tile, head, key, dim, value):
    """The number at (key, dim), by its address."""
    c, D = s.c, s.c["D"]
    at = (head * (c["ps"] // 16) + tile) * 32 * D
    if value:
        at = at + 16 * D + dim // 64 * 1024 + (dim % 16 + key // 4 * 16) * 16 + dim % 64 // 16 * 4 + key % 4
    else:
        at = at + dim // 64 * 1024 + (key + dim % 32 // 8 * 16) * 16 + dim % 64 // 32 * 8 + dim % 8
    sc = _code_bytes(c) // 4 + (head * (c["ps"] // 16) + tile) * 2 + int(value)
    return _number(s.pool[page, at], c["fmt"]) * s.pool.view(torch.float32)[page, sc].double()


def _sequence(s, i, n, head, value):
    """[n, D] of a sequence's head"""
    p, d = torch.arange(n, device=DEV)[:, None], torch.arange(s.c["D"], device=DEV)[None]
    page = s.table[i].long()[p // s.c["ps"]]
    return _element(s, page, p % s.c["ps"] // 16, head, p % 16, d, value)


def _exact_attention(s):
    c = s.c
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    G, at = H // Hkv, 0
    out = torch.zeros(s.M, H, D, dtype=torch.float64, device=DEV)
    for i, (n, r) in enumerate(zip(_lens(c), _rows(c))):
        pos, key = torch.arange(n - r, n, device=DEV)[:, None], torch.arange(n, device=DEV)[None]
        gone = key > pos
        if c["window"]:
            gone |= key <= pos - c["window"]
        if c["prefix"]:
            gone &= key >= int(s.prefix[i])
        for h in range(Hkv):
            k, v = (_sequence(s, i, n, h, value) for value in (False, True))
            for g in range(h * G, (h + 1) * G):
                x = s.q[at:at + r, g * D:(g + 1) * D].double() @ k.T
                if c["cap"]:
                    x = torch.tanh(x / c["cap"]) * c["cap"]
                if c["slopes"]:
                    x = x - s.slopes[g].double() * (pos - key).abs()
                x[gone] = -float("inf")
                out[at:at + r, g] = torch.softmax(x, -1) @ v
        at += r
    return out.view(s.M, H * D)


def _exact_append(s):
    """Block by block in numpy, the scales found by trying one after the other."""
    c, fmt, D, Hkv = s.c, s.c["fmt"], s.c["D"], s.c["Hkv"]

    def nearest(x):
        if fmt == "int8":
            return np.rint(x)
        step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -30))), -6) - 3)
        return np.rint(x / step) * step

    out = []
    for value, rows in ((False, s.k), (True, s.v)):
        rows = np.clip(np.nan_to_num(rows.cpu().numpy().astype(np.float64), nan=0.0), -CLAMP, CLAMP)
        rows, at, got = rows.reshape(-1, Hkv, D), 0, []
        for i, (n, r, back) in enumerate(zip(_lens(c), _rows(c), _back(c))):
            low = (n - max(r, back)) // 16 * 16
            p = torch.arange(low, n, device=DEV)[:, None, None]
            h, d = torch.arange(Hkv, device=DEV)[None, :, None], torch.arange(D, device=DEV)[None, None]
            page = s.table[i].long()[p // c["ps"]]
            x = _element(s, page, p % c["ps"] // 16, h, p % 16, d, value).cpu().numpy()
            sc = _scales(s)[page[:, 0, 0], :, p[:, 0, 0] % c["ps"] // 16, int(value)].cpu().numpy()
            x[n - r - low:] = rows[at:at + r]
            for b in range((n - r) // 16 * 16, n, 16):
                block = x[b - low:b - low + 16]
                fresh = block[max(n - r - b, 0):]
                scale = np.full(Hkv, 2.0 ** LOW[fmt])
                for e in range(LOW[fmt], HIGH[fmt]):
                    scale = np.where(np.abs(fresh).max((0, 2)) > TOP[fmt] * 2.0 ** e, 2.0 ** (e + 1), scale)
                if b < n - r:
                    scale = np.maximum(scale, sc[b - low].astype(np.float64))
                block[:] = nearest(block / scale[None, :, None]) * scale[None, :, None]
            got.append(x[n - back - low:].reshape(back, Hkv * D))
            at += r
        out.append(torch.from_numpy(np.concatenate(got)))
    return out


def _exact_sample(s):
    """One row after the other in numpy."""
    c, tokens, logs = s.c, [], []
    x = s.logits.cpu().numpy().astype(np.float64)
    T, k, p, m, u = (a.cpu().numpy().astype(np.float64) for a in (s.T, s.k, s.p, s.m, s.u))
    for i in range(c["rows"]):
        order = np.lexsort((np.arange(c["V"]), -x[i]))
        if T[i] <= 0:
            tokens.append(order[0])
            logs.append(0.0)
            continue
        if 0 < k[i] < c["V"]:
            order = order[:int(k[i])]
        z = (x[i][order] - x[i][order[0]]) / T[i]
        z = z[np.exp(z) >= m[i]]
        run = np.cumsum(np.exp(z))
        z = z[:np.searchsorted(run, p[i] * run[-1], side="left") + 1]
        total = run[min(len(z), len(run)) - 1]
        at = min(int(np.searchsorted(run[:len(z)], u[i] * total, side="right")), len(z) - 1)
        tokens.append(order[at])
        logs.append(z[at] - np.log(total))
    return [torch.tensor(np.array(tokens), dtype=torch.int32), torch.tensor(logs, dtype=torch.float64)]


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attention, "sample": _exact_sample}[s.kind](s)
