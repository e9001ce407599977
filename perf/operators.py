"""The paged 4-bit cache's operators: what they are measured on, their plain
forms and their 64-bit values.

A batch of sequences of different lengths keeps keys and values in pages of
4-bit codes (pipo_kv_pages in include/pipo_ops.h).  The kinds of case:

  norm_rope   per-head RMSNorm of q and k and their rotation, one position a row
  append      new rows' k and v quantized into their pages and read back
  attn        attention of each sequence's newest rows over its pages
  beam        a beam-search step: every beam grows by a token (resize), beams
              continue from their parents (fork), shared last pages are copied
  compact     sequences end (resize to 0), the pages in use move to the front

Sizes are those of the workloads this repository runs (OPT-125m / 13B / 30B and
LLaMA-3.1-8B heads, batch 1 to 128, prompts of 32 to 512 tokens) with contexts
up to 65536 tokens; draw() spreads over the ranges between and around them.
"""
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5
CLAMP = 57344.0                 # of an element before it is quantized
TOP_WORK = 1.2e12               # flops of the largest attention case
TOP_CACHE = 4.5e8               # padded cache elements (sequences x longest x Hkv x D)


# ---------------------------------------------------------------------------
def listed():
    return [
        # a decode step's q and k, 16 users: launch latency
        dict(name="norm_rope_llama8b_b16", kind="norm_rope", M=16, H=32, Hkv=8, D=128, first=0,
             top=2048),
        # 16 prompts of 512 tokens
        dict(name="norm_rope_llama8b_prompts", kind="norm_rope", M=8192, H=32, Hkv=8, D=128,
             first=0, top=4096),
        # a decode step's new rows
        dict(name="append_llama8b_b16", kind="append", n=16, nq=1, lo=100, hi=2100, Hkv=8, D=128,
             ps=64),
        # eight prompts of 512 tokens, every head its own keys
        dict(name="append_opt30b_prompts", kind="append", n=8, nq=512, lo=512, hi=512, Hkv=56,
             D=128, ps=64),
        # the smallest model just after short prompts: launch latency
        dict(name="attn_opt125m_b4", kind="attn", n=4, H=12, Hkv=12, D=64, ps=16, lo=33, hi=40,
             nq=1, long=0),
        # 16 users at different lengths, grouped heads
        dict(name="attn_llama8b_b16", kind="attn", n=16, H=32, Hkv=8, D=128, ps=64, lo=100,
             hi=2100, nq=1, long=0),
        # one key/value head per query head, prompts of 512 tokens and up to 32 generated
        dict(name="attn_opt30b_b64", kind="attn", n=64, H=56, Hkv=56, D=128, ps=32, lo=513, hi=544,
             nq=1, long=0),
        # one user with a long document: the cache split over the chip
        dict(name="attn_llama8b_long", kind="attn", n=1, H=32, Hkv=8, D=128, ps=128, lo=65000,
             hi=65000, nq=1, long=0),
        # four long prompts in pieces of 512 tokens
        dict(name="attn_llama8b_chunk", kind="attn", n=4, H=32, Hkv=8, D=128, ps=64, lo=509,
             hi=4099, nq=509, long=0),
        # 28 users decode while two prompts of 509 tokens come in
        dict(name="attn_llama8b_mixed", kind="attn", n=30, H=32, Hkv=8, D=128, ps=64, lo=520,
             hi=2100, nq=1, long=2),
        # 16 requests of four beams
        dict(name="beam_llama8b_b64", kind="beam", n=64, width=4, lo=520, hi=1300, Hkv=8, D=128,
             ps=64, layers=2),
        # half of 96 sequences end, small pages
        dict(name="compact_llama8b_b96", kind="compact", n=96, keep=2, lo=200, hi=1400, Hkv=8,
             D=128, ps=16, layers=2),
    ]


LONG = 509          # tokens of the prompts in a mixed batch


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["norm_rope", "append", "attn", "attn", "attn", "beam", "compact"])
    D = rng.choice([64, 128, 128])
    if kind == "norm_rope":
        G, Hkv = rng.choice([1, 2, 3, 4, 5, 8]), rng.randint(1, 16)
        top = _log(rng, 64, 65536)
        return dict(kind=kind, M=max(1, min(_log(rng, 1, 16384), 8192 * 40 * 128 // (Hkv * (G + 1) * D))),
                    H=G * Hkv, Hkv=Hkv, D=D, first=rng.randint(0, top // 2), top=top)
    ps = rng.choice([16, 32, 64, 128])
    if kind == "append":
        Hkv = rng.randint(1, 56)
        n, nq = _log(rng, 1, 128), _log(rng, 1, 1024) if rng.random() < 0.5 else 1
        nq = max(1, min(nq, 8 * 512 * 56 * 128 // (n * Hkv * D)))
        lo = nq + rng.randint(0, 500)
        return dict(kind=kind, n=n, nq=nq, lo=lo, hi=lo + rng.randint(0, 600), Hkv=Hkv, D=D, ps=ps)
    if kind == "attn":
        G = rng.choice([1, 1, 2, 3, 4, 4, 5, 7, 8, 16])
        Hkv = rng.randint(1, 8) if G > 1 else rng.randint(1, 56)
        shape = rng.choice(["one", "one", "one", "few", "chunk", "mixed"])
        nq = {"one": 1, "few": rng.randint(2, 8), "chunk": _log(rng, 17, 1024), "mixed": 1}[shape]
        long = rng.randint(1, 3) if shape == "mixed" else 0
        n = _log(rng, 1, 8) if shape == "chunk" else _log(rng, 4, 32) if long else _log(rng, 1, 128)
        floor = LONG if long else nq
        hi = max(floor + 1, _log(rng, 33, 65536))
        hi = max(floor + 1, min(hi, int(TOP_CACHE / (n * Hkv * D))))
        most = LONG if long else nq
        hi = max(floor + 1, min(hi, int(TOP_WORK / (4 * n * most * G * Hkv * D))))
        return dict(kind=kind, n=n, H=G * Hkv, Hkv=Hkv, D=D, ps=ps, lo=rng.randint(floor, hi), hi=hi,
                    nq=nq, long=long)
    Hkv = rng.randint(1, 12)
    n, hi = _log(rng, 4, 128), _log(rng, 40, 4000)
    page = Hkv * ps * 9 * D // 8
    hi = max(40, min(hi, int(1.5e8 / (n * page) * ps)))
    out = dict(kind=kind, n=n, lo=rng.randint(1, hi), hi=hi, Hkv=Hkv, D=D, ps=ps,
               layers=rng.randint(1, 2))
    out.update(dict(width=rng.choice([2, 4, 8])) if kind == "beam" else dict(keep=rng.choice([2, 3])))
    return out


# ---------------------------------------------------------------------------
# shapes of a case (not of its seed)
def _lens(c):
    n = c["n"]
    return [c["lo"] + (c["hi"] - c["lo"]) * (i * 37 % n) // max(n - 1, 1) for i in range(n)]


def _rows(c):
    """new rows of each sequence"""
    return [LONG if i < c.get("long", 0) else c["nq"] for i in range(c["n"])]


def _page_bytes(c):
    return c["Hkv"] * c["ps"] * (c["D"] + c["D"] // 8)


def work(case):
    c, kind = case, case["kind"]
    if kind == "norm_rope":
        row = (c["H"] + c["Hkv"]) * c["D"]
        return {"bytes": c["M"] * (4 * row + 4) + min(c["M"], c["top"] - c["first"]) * 4 * c["D"],
                "flops": 8 * c["M"] * row}
    if kind == "append":
        M, dkv = c["n"] * c["nq"], c["Hkv"] * c["D"]
        # fp16 in, codes written and read, fp16 out
        return {"bytes": M * 2 * dkv * (2 + 2 * 9 / 16 + 2), "flops": M * 2 * dkv * 8}
    if kind == "attn":
        lens, rows = _lens(c), _rows(c)
        cache = sum(lens) * c["Hkv"] * 2 * 9 * c["D"] // 16
        pairs = sum(r * (n - r) + r * (r + 1) // 2 for n, r in zip(lens, rows))
        return {"bytes": cache + sum(rows) * c["H"] * c["D"] * 4, "flops": 4 * c["D"] * c["H"] * pairs}
    # what moves and the tables; as many last pages as there are beams that share one
    t = sum(-(-n // c["ps"]) for n in _lens(c)) * 4
    if kind == "beam":
        return {"bytes": 2 * t + _beam_copies(c) * 2 * _page_bytes(c) * c["layers"], "flops": 0}
    return {"bytes": 2 * t + _compact_moves(c) * 2 * _page_bytes(c) * c["layers"], "flops": 0}


def _parents(c):
    """Beams continue from one of their group's; one group of eight ends."""
    rng, w, out = random.Random(c["n"] * 1000 + c["hi"]), c["width"], []
    for i in range(c["n"]):
        g = i // w * w
        out.append(-1 if i // w % 8 == 7 else min(g + rng.randrange(w), c["n"] - 1))
    return out


def _beam_copies(c):
    lens, parents = _lens(c), _parents(c)
    return sum(1 for i, p in enumerate(parents)
               if p >= 0 and (lens[p] + 1) % c["ps"] and p in parents[:i])


def _wants(c):
    """-1 keeps a sequence, 0 frees it"""
    return [-1 if i % c["keep"] == 0 else 0 for i in range(c["n"])]


def _table(c, rng, extra):
    """Pages in random order: (table [n][width], pages in the pool)."""
    lens = _lens(c)
    need = [-(-n // c["ps"]) for n in lens]
    n_pages = sum(need) + extra
    order = rng.permutation(n_pages).astype(np.int32)
    width = max(need) + 3
    table = np.full((c["n"], width), -1, np.int32)
    at = 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    return table, n_pages


def _compact_moves(c):
    """Expected number of pages that move (the table's order is random)."""
    lens = _lens(c)
    need = [-(-n // c["ps"]) for n in lens]
    used = sum(k for i, k in enumerate(need) if i % c["keep"] == 0)
    total = sum(need) + 64
    return used * (total - used) // total


# ---------------------------------------------------------------------------
# the pages' layout (pipo_kv_pages in include/pipo_ops.h), written out in
# elementary operations: tiles of 16 keys of a head, in them K codes, V codes,
# and the (min, scale) pairs of both
def _quantize(x):
    """[..., D] fp16 -> codes uint8 [..., D], (min, scale) fp16 [..., D/64, 2]"""
    v = x.float()
    v = torch.where(v != v, torch.zeros_like(v), v).clamp(-CLAMP, CLAMP)
    v = v.view(*x.shape[:-1], x.shape[-1] // 64, 64)
    lo, hi = v.amin(-1, keepdim=True), v.amax(-1, keepdim=True)
    s, m = ((hi - lo) / 15).half(), lo.half()
    q = torch.where(s != 0, (v - m.float()) / s.float(), torch.zeros_like(v))
    return q.round().clamp(0, 15).to(torch.uint8).view(x.shape), torch.cat([m, s], -1)


def _k_bytes(codes):
    """[..., 16, D] -> [..., 8 D]: byte (key + 16 g) D/8 + 4 kk + j of a tile holds the codes of
    dimensions 32 kk + 8 g + ..., those at 2 i + h in nibble 4 h + i of a word"""
    D, lead = codes.shape[-1], codes.shape[:-2]
    x = codes.reshape(-1, 16, D // 32, 4, 4, 2)            # key, kk, g, i, h
    x = x.permute(0, 3, 1, 2, 5, 4).reshape(-1, 4, 16, D // 32, 4, 2)   # g, key, kk, byte, nibble
    return (x[..., 0] | (x[..., 1] << 4)).reshape(*lead, 8 * D)


def _v_bytes(codes):
    """[..., 16, D] -> [..., 8 D]: byte (r + 16 g) D/8 + 4 w + i holds key 4 g + i, dimension
    32 w + r in the low nibble and 32 w + 16 + r in the high one"""
    D, lead = codes.shape[-1], codes.shape[:-2]
    x = codes.reshape(-1, 4, 4, D // 32, 2, 16).permute(0, 1, 5, 3, 2, 4)  # g, r, w, i, half
    return (x[..., 0] | (x[..., 1] << 4)).reshape(*lead, 8 * D)


def _k_codes(b, D):
    x = b.reshape(-1, 4, 16, D // 32, 4)
    x = torch.stack([x & 15, x >> 4], -1).view(-1, 4, 16, D // 32, 2, 4)    # g, key, kk, h, i
    return x.permute(0, 2, 3, 1, 5, 4).reshape(*b.shape[:-1], 16, D)


def _v_codes(b, D):
    x = b.reshape(-1, 4, 16, D // 32, 4)
    x = torch.stack([x & 15, x >> 4], -1)                                  # g, r, w, i, half
    return x.permute(0, 1, 4, 3, 5, 2).reshape(*b.shape[:-1], 16, D)


def _pack(k, v):
    """[..., 16, D] fp16 keys and values -> tiles [..., 18 D] uint8"""
    (kc, kp), (vc, vp) = _quantize(k), _quantize(v)
    pairs = [p.reshape(*k.shape[:-2], -1).view(torch.uint8) for p in (kp, vp)]
    return torch.cat([_k_bytes(kc), _v_bytes(vc), *pairs], -1)


def _values(codes, pairs, D):
    x = codes.view(*codes.shape[:-1], D // 64, 64).float()
    return (x * pairs[..., 1:].float() + pairs[..., :1].float()).view(codes.shape)


def _unpack(tiles, D):
    """tiles [..., 18 D] -> fp32 keys and values [..., 16, D]"""
    lead = tiles.shape[:-1]
    kp = tiles[..., 16 * D:17 * D].contiguous().view(torch.float16).view(*lead, 16, D // 64, 2)
    vp = tiles[..., 17 * D:].contiguous().view(torch.float16).view(*lead, 16, D // 64, 2)
    return (_values(_k_codes(tiles[..., :8 * D], D), kp, D),
            _values(_v_codes(tiles[..., 8 * D:16 * D], D), vp, D))


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


def prepare(case, seed):
    c, kind = case, case["kind"]
    s = SimpleNamespace(c=c, kind=kind)
    rng = np.random.default_rng(seed % (1 << 63))
    D = c["D"]
    if kind == "norm_rope":
        g = _gen(seed, 1)
        M, H, Hkv = c["M"], c["H"], c["Hkv"]
        # rows as the fused projection leaves them: q, k, v side by side
        s.qkv = _normal(g, M, (H + 2 * Hkv) * D, std=1.5)
        s.gq, s.gk = 1 + _normal(g, D, std=0.2), 1 + _normal(g, D, std=0.2)
        i = torch.arange(D // 2, dtype=torch.float64, device=DEV)
        a = torch.arange(c["top"], dtype=torch.float64, device=DEV)[:, None] * 500000.0 ** (-2 * i / D)
        s.cs = torch.stack([a.cos(), a.sin()], -1).float().contiguous()
        span = max(1, c["top"] - c["first"])
        s.pos = (torch.arange(M, device=DEV) % span + c["first"]).int()
        s.q, s.k = s.qkv[:, :H * D], s.qkv[:, H * D:(H + Hkv) * D]
        s.qo, s.ko = torch.empty(M, H * D, dtype=torch.float16, device=DEV), torch.empty(
            M, Hkv * D, dtype=torch.float16, device=DEV)
        return s
    lens, Hkv, ps = _lens(c), c["Hkv"], c["ps"]
    table, s.n_pages = _table(c, rng, 64 + (c["n"] * 2 if kind == "beam" else 0))
    s.layers = c.get("layers", 1)
    if kind in ("beam", "compact"):
        s.pool = torch.randint(0, 256, (s.layers, s.n_pages, _page_bytes(c)), generator=_gen(seed, 4),
                               device=DEV, dtype=torch.uint8)
        s.table, s.len = _int(table), _int(lens)
        s.want = _int([n + 1 for n in lens] if kind == "beam" else _wants(c))
        s.cap = c["n"] if kind == "beam" else s.n_pages // 2
        s.table1, s.table2 = torch.empty_like(s.table), torch.empty_like(s.table)
        s.len1, s.len2 = torch.empty_like(s.len), torch.empty_like(s.len)
        s.pairs = torch.zeros(max(s.cap, 1), 2, dtype=torch.int32, device=DEV)
        s.count = torch.zeros(3, dtype=torch.int32, device=DEV)
        if kind == "beam":
            s.parent = _int(_parents(c))
        return s
    rows = _rows(c)
    starts = np.concatenate([[0], np.cumsum(rows)])
    s.M, s.max_q, s.max_len = int(starts[-1]), max(rows), max(lens)
    s.table = _int(table)
    s.seq = _int(np.repeat(np.arange(c["n"]), rows))
    s.col = _int(np.concatenate([np.arange(r) for r in rows]))
    s.pos = _int(np.concatenate([np.arange(n - r, n) for n, r in zip(lens, rows)]))
    s.q_start, s.len, s.rows = _int(starts), _int(lens), _int(rows)
    g = _gen(seed, 2)
    gain = torch.exp(0.5 * torch.randn(Hkv, 1, 1, D, generator=g, device=DEV)).half()
    s.pool = torch.empty(s.n_pages, Hkv, ps // 16, 18 * D, dtype=torch.uint8, device=DEV)
    if kind == "append":
        s.pool.zero_()
        s.kv = _normal(g, s.M, 2 * Hkv * D)
        s.k, s.v = s.kv[:, :Hkv * D], s.kv[:, Hkv * D:]
        s.ko, s.vo = (torch.empty(s.M, Hkv * D, dtype=torch.float16, device=DEV) for _ in "kv")
        return s
    step = max(1, (1 << 27) // (Hkv * ps * D))
    for p in range(0, s.n_pages, step):
        m = min(step, s.n_pages - p)
        shape = (m, Hkv, ps // 16, 16, D)
        s.pool[p:p + m] = _pack(_normal(g, *shape) * gain, _normal(g, *shape))
    s.q = _normal(g, s.M, c["H"] * D, std=1.2 * D ** -0.5)
    s.o = torch.empty_like(s.q)
    s.ws = None
    return s


# ---------------------------------------------------------------------------
# plain forms
def _norm_rope(x, gamma, cs, pos, heads, D, scale):
    x = x.reshape(x.shape[0], heads, D).float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma.float()
    a, b = x[..., :D // 2], x[..., D // 2:]
    t = cs[pos.long()]
    cos, sin = t[:, None, :, 0], t[:, None, :, 1]
    y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1) * scale
    return y.view(x.shape[0], heads * D).half()


def _append(s):
    """Rows into their slots (a tile's bytes each), then the values they stand for."""
    c = s.c
    M, Hkv, D, ps = s.M, c["Hkv"], c["D"], c["ps"]
    pos, tiles = s.pos.long(), s.pool.view(-1, 18 * D)
    page = s.table[s.seq.long(), pos // ps].long()
    tile = (page[:, None] * Hkv + torch.arange(Hkv, device=DEV)) * (ps // 16) + (pos % ps // 16)[:, None]
    key = (pos % 16)[:, None, None]
    (kc, kp), (vc, vp) = _quantize(s.k.reshape(M, Hkv, D)), _quantize(s.v.reshape(M, Hkv, D))
    x = kc.view(M, Hkv, D // 32, 4, 4, 2).permute(0, 1, 3, 2, 5, 4).reshape(M, Hkv, 4, D // 32, 4, 2)
    kb = (x[..., 0] | (x[..., 1] << 4)).reshape(M, Hkv, D // 2)                    # g, kk, byte
    x = vc.view(M, Hkv, D // 32, 2, 16).permute(0, 1, 4, 2, 3)                      # r, w, half
    vb = (x[..., 0] | (x[..., 1] << 4)).reshape(M, Hkv, D // 2)
    i = torch.arange(D // 2, device=DEV)
    ka = (key + 16 * (i // (D // 8))) * (D // 8) + i % (D // 8)
    va = 8 * D + (i // (D // 32) + 16 * (key // 4)) * (D // 8) + 4 * (i % (D // 32)) + key % 4
    j = torch.arange(D // 16, device=DEV)
    at = torch.cat([ka, va, 16 * D + key * (D // 16) + j, 17 * D + key * (D // 16) + j], -1)
    data = torch.cat([kb, vb, kp.reshape(M, Hkv, -1).view(torch.uint8),
                      vp.reshape(M, Hkv, -1).view(torch.uint8)], -1)
    flat = tiles.view(-1)
    flat[tile[..., None] * (18 * D) + at] = data
    got = flat[tile[..., None] * (18 * D) + at]
    h = D // 2
    kb, vb = got[..., :h], got[..., h:2 * h]
    x = torch.stack([kb & 15, kb >> 4], -1).view(M, Hkv, 4, D // 32, 2, 4)
    kc = x.permute(0, 1, 3, 2, 5, 4).reshape(M, Hkv, D)
    x = torch.stack([vb & 15, vb >> 4], -1).view(M, Hkv, 16, D // 32, 2)
    vc = x.permute(0, 1, 3, 4, 2).reshape(M, Hkv, D)
    kp = got[..., 2 * h:2 * h + D // 16].contiguous().view(torch.float16).view(M, Hkv, D // 64, 2)
    vp = got[..., 2 * h + D // 16:].contiguous().view(torch.float16).view(M, Hkv, D // 64, 2)
    return [_values(kc, kp, D).half().view(M, Hkv * D), _values(vc, vp, D).half().view(M, Hkv * D)]


def _attention(s):
    c = s.c
    n, H, Hkv, D, ps = c["n"], c["H"], c["Hkv"], c["D"], c["ps"]
    G, pages = H // Hkv, -(-s.max_len // ps)
    L = pages * ps
    t = s.table[:, :pages].clamp(min=0).long()
    k, v = _unpack(s.pool[t].transpose(1, 2).contiguous(), D)         # n, Hkv, page, tile, 16, D
    k, v = k.view(n, Hkv, L, D), v.view(n, Hkv, L, D)
    j = torch.arange(s.max_q, device=DEV)
    row = (s.q_start[:-1, None] + j).clamp(max=s.M - 1).long()
    q = s.q[row].float().view(n, s.max_q, Hkv, G, D).transpose(1, 2).reshape(n, Hkv, s.max_q * G, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous())
    last = (s.len - s.rows)[:, None] + j                              # a row's position
    seen = torch.arange(L, device=DEV) <= last[..., None]             # n, q, key
    x = x.view(n, Hkv, s.max_q, G, L).masked_fill_(~seen[:, None, :, None], -float("inf"))
    x = x - x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = x.exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(n, Hkv, s.max_q * G, L), v).view(n, Hkv, s.max_q, G, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    o = o.transpose(1, 2)[s.seq.long(), s.col.long()]
    return o.reshape(s.M, H * D).half()


def _pages_of(n, ps):
    return (n + ps - 1) // ps


def _free_list(used):
    """pages not in use, in order (and how many)"""
    free = used == 0
    n = used.numel()
    i = torch.arange(n, device=DEV)
    order = torch.zeros(n + 1, dtype=torch.long, device=DEV)
    order.scatter_(0, torch.where(free, free.long().cumsum(0) - 1, n), i)
    return order, free.sum()


def _used(table, mask, n_pages):
    used = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV)
    used.scatter_(0, torch.where(mask, table.long(), n_pages).flatten(), 1)
    return used[:n_pages]


def _resize(s):
    ps, j = s.c["ps"], torch.arange(s.table.shape[1], device=DEV)
    held, need = _pages_of(s.len, ps)[:, None], _pages_of(s.want, ps)[:, None]
    need = torch.where(s.want[:, None] < 0, held, need)
    keep, grow = (j < held) & (j < need), (j >= held) & (j < need)
    order, _ = _free_list(_used(s.table, keep, s.n_pages))
    rank = (grow.flatten().long().cumsum(0) - 1).clamp(min=0).view(grow.shape)
    table = torch.where(keep, s.table, torch.where(grow, order[rank].int(), -1))
    return table, torch.where(s.want < 0, s.len, s.want)


def _fork(s, table, length):
    ps, n = s.c["ps"], s.c["n"]
    j, i = torch.arange(table.shape[1], device=DEV), torch.arange(n, device=DEV)
    p = s.parent.long()
    ok, p = p >= 0, p.clamp(min=0)
    new_len = torch.where(ok, length[p], 0)
    first = torch.full((n,), n, device=DEV).scatter_reduce_(0, torch.where(ok, p, 0),
                                                            torch.where(ok, i, n), "amin")
    held, partial = _pages_of(new_len, ps), new_len % ps != 0
    fresh = ok & partial & (first[p] != i)
    rows = torch.where(j < held[:, None], table[p], -1)
    is_new = fresh[:, None] & (j == held[:, None] - 1)
    order, _ = _free_list(_used(rows, (j < held[:, None]) & ~is_new, s.n_pages))
    rank = (fresh.long().cumsum(0) - 1).clamp(min=0)
    page = order[rank]
    at = (held.long() - 1).clamp(min=0)
    src = rows.long().gather(1, at[:, None])[:, 0]
    rows = torch.where(is_new, page[:, None].int(), rows)
    pairs = torch.zeros(n + 1, 2, dtype=torch.long, device=DEV)
    pairs.scatter_(0, torch.where(fresh, rank, n)[:, None].expand(-1, 2), torch.stack([src, page], -1))
    return rows, new_len, pairs[:n], fresh.sum()


def _compact(s, table, length):
    n_pages, j = s.n_pages, torch.arange(table.shape[1], device=DEV)
    mask = j < _pages_of(length, s.c["ps"])[:, None]
    used = _used(table, mask, n_pages)
    U, page = used.sum(), torch.arange(n_pages, device=DEV)
    high, hole = (used > 0) & (page >= U), (used == 0) & (page < U)
    hi_rank, hole_rank = high.long().cumsum(0) - 1, hole.long().cumsum(0) - 1
    pairs = torch.zeros(n_pages + 1, 2, dtype=torch.long, device=DEV)
    pairs[:, 0].scatter_(0, torch.where(high, hi_rank, n_pages), page)
    pairs[:, 1].scatter_(0, torch.where(hole, hole_rank, n_pages), page)
    to = torch.where(high, pairs[hi_rank.clamp(min=0), 1], page)
    rows = torch.where(mask, to[table.clamp(min=0).long()].int(), -1)
    return rows, length, pairs[:s.cap], high.sum()


def _copy(s, pairs, count):
    # (past the last pair, the first again; none: page 0 onto itself)
    i = torch.arange(pairs.shape[0], device=DEV)
    pairs = torch.where((i < count)[:, None], pairs, pairs[:1] * (count > 0))
    s.pool[:, pairs[:, 1]] = s.pool[:, pairs[:, 0]]
    return s.pool


# ---------------------------------------------------------------------------
# the framework's calls
def _stream():
    return torch.cuda.current_stream().cuda_stream


def _cache(s):
    from paper_2504_03664_amd import binding as B
    c = s.c
    return B.PipoKvPages(s.pool.data_ptr(), _page_bytes(c) * s.n_pages, s.table.data_ptr(),
                         s.table.shape[1], s.layers, s.n_pages, c["ps"], c["Hkv"], c["D"], c["n"])


def _run_own(s):
    from paper_2504_03664_amd import binding as B
    c, st = s.c, _stream()
    if s.kind == "norm_rope":
        B.pipo_op_qk_norm_rope(s.q.data_ptr(), s.q.stride(0), s.k.data_ptr(), s.k.stride(0),
                               s.gq.data_ptr(), s.gk.data_ptr(), s.cs.data_ptr(), c["top"],
                               s.pos.data_ptr(), s.qo.data_ptr(), s.qo.stride(0), s.ko.data_ptr(),
                               s.ko.stride(0), c["M"], c["H"], c["Hkv"], c["D"], EPS,
                               c["D"] ** -0.5, st)
        return [s.qo, s.ko]
    if s.kind in ("append", "attn") and getattr(s, "cache", None) is None:
        s.cache = _cache(s)
    if s.kind == "append":
        B.pipo_op_kv_pages_append(s.cache, 0, s.seq.data_ptr(), s.pos.data_ptr(), s.k.data_ptr(),
                                  s.k.stride(0), s.v.data_ptr(), s.v.stride(0), s.M, st)
        B.pipo_op_kv_pages_read(s.cache, 0, s.seq.data_ptr(), s.pos.data_ptr(), s.ko.data_ptr(),
                                s.ko.stride(0), s.vo.data_ptr(), s.vo.stride(0), s.M, st)
        return [s.ko, s.vo]
    if s.kind == "attn":
        if s.ws is None:
            n = B.pipo_op_attn_pages_workspace_bytes(s.cache, c["H"], s.M, s.max_q, s.max_len)
            s.ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
        B.pipo_op_attn_pages(s.cache, 0, s.q.data_ptr(), s.q.stride(0), s.q_start.data_ptr(),
                             s.len.data_ptr(), s.o.data_ptr(), s.o.stride(0), c["H"], s.M, s.max_q,
                             s.max_len, s.ws.data_ptr(), s.ws.numel(), st)
        return s.o
    cnt, width = s.count.data_ptr(), s.table.shape[1]
    B.pipo_op_kv_pages_resize(s.table.data_ptr(), s.len.data_ptr(), s.want.data_ptr(),
                              s.table1.data_ptr(), s.len1.data_ptr(), width, c["n"], s.n_pages,
                              c["ps"], cnt, st)
    if s.kind == "beam":
        B.pipo_op_kv_pages_fork(s.table1.data_ptr(), s.len1.data_ptr(), c["n"], s.parent.data_ptr(),
                                s.table2.data_ptr(), s.len2.data_ptr(), c["n"], width, s.n_pages,
                                c["ps"], s.pairs.data_ptr(), cnt + 4, cnt + 8, st)
        table, length = s.table2, s.len2
    else:
        B.pipo_op_kv_pages_compact(s.table1.data_ptr(), s.len1.data_ptr(), s.table2.data_ptr(), width,
                                   c["n"], s.n_pages, c["ps"], s.pairs.data_ptr(), cnt + 4, st)
        table, length = s.table2, s.len1
    B.pipo_op_kv_pages_copy(_cache(s), s.pairs.data_ptr(), cnt + 4, s.cap, st)
    return [table, length, s.pool]


def run(state):
    s = state
    if own:
        return _run_own(s)
    c = s.c
    if s.kind == "norm_rope":
        return [_norm_rope(s.q, s.gq, s.cs, s.pos, c["H"], c["D"], c["D"] ** -0.5),
                _norm_rope(s.k, s.gk, s.cs, s.pos, c["Hkv"], c["D"], 1.0)]
    if s.kind == "append":
        return _append(s)
    if s.kind == "attn":
        return _attention(s)
    table, length = _resize(s)
    table, length, pairs, count = (_fork if s.kind == "beam" else _compact)(s, table, length)
    return [table, length.int(), _copy(s, pairs, count)]


# ---------------------------------------------------------------------------
# 64-bit values
def _element(tile, D, key, dim, value):
    """The number at (key, dim) of tiles [..., 18 D], by its address."""
    if value:
        g, i, w, half, r = key // 4, key % 4, dim // 32, dim % 32 // 16, dim % 16
        byte, nib = 8 * D + (r + 16 * g) * (D // 8) + 4 * w + i, half
    else:
        kk, g, i, h = dim // 32, dim % 32 // 8, dim % 8 // 2, dim % 2
        n = 4 * h + i
        byte, nib = (key + 16 * g) * (D // 8) + 4 * kk + n // 2, n % 2
    code = (tile[..., byte].to(torch.int32) >> (4 * nib)) & 15
    at = (17 if value else 16) * D + key * (D // 16) + dim // 64 * 4
    half16 = lambda a: (tile[..., a].to(torch.int32) | tile[..., a + 1].to(torch.int32) << 8).to(  # noqa: E731
        torch.int16).view(torch.float16).double()
    return code.double() * half16(at + 2) + half16(at)


def _exact_attention(s):
    c = s.c
    H, Hkv, D, ps = c["H"], c["Hkv"], c["D"], c["ps"]
    out = torch.zeros(s.M, H, D, dtype=torch.float64, device=DEV)
    key = torch.arange(16, device=DEV)[:, None].expand(16, D)
    dim = torch.arange(D, device=DEV)[None].expand(16, D)
    at = 0
    for i, (n, r) in enumerate(zip(_lens(c), _rows(c))):
        tiles = s.pool[s.table[i, :-(-n // ps)].long()]                    # pages, Hkv, tiles, bytes
        for h in range(Hkv):
            one = tiles[:, h].reshape(-1, 18 * D)
            k = _element(one, D, key, dim, False).view(-1, D)[:n]
            v = _element(one, D, key, dim, True).view(-1, D)[:n]
            heads = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
            q = s.q[at:at + r].view(r, H, D)[:, heads].double()
            x = q.reshape(-1, D) @ k.T
            pos = torch.arange(n - r, n, device=DEV).repeat_interleave(H // Hkv)
            x[torch.arange(n, device=DEV)[None] > pos[:, None]] = -float("inf")
            out[at:at + r, heads] = (torch.softmax(x, -1) @ v).view(r, H // Hkv, D)
        at += r
    return out.view(s.M, H * D)


def _exact_rows(x, heads, D):
    """What a quantized row stands for, element by element in numpy."""
    x = np.clip(np.nan_to_num(x.astype(np.float64), nan=0.0), -CLAMP, CLAMP)
    x = x.reshape(-1, 64)
    lo, hi = x.min(1, keepdims=True), x.max(1, keepdims=True)
    scale = ((hi - lo).astype(np.float32) / np.float32(15)).astype(np.float16).astype(np.float64)
    low = lo.astype(np.float16).astype(np.float64)
    q = np.where(scale > 0, ((x - low).astype(np.float32) /
                             np.where(scale > 0, scale, 1).astype(np.float32)), 0)
    return (np.clip(np.rint(q), 0, 15) * scale + low).reshape(-1, heads * D)


def _exact_pages(s):
    """Tables and pool after the calls, one sequence and page after the other."""
    c, ps = s.c, s.c["ps"]
    table, lens, want = s.table.cpu().numpy(), s.len.cpu().tolist(), s.want.cpu().tolist()
    rows = [list(t[:-(-n // ps)]) for t, n in zip(table, lens)]
    rows = [r if w < 0 else r[:-(-w // ps)] for r, w in zip(rows, want)]
    lens = [n if w < 0 else w for n, w in zip(lens, want)]
    free = iter(sorted(set(range(s.n_pages)) - {p for r in rows for p in r}))
    for r, n in zip(rows, lens):
        while len(r) < -(-n // ps):
            r.append(next(free))
    moves = []
    if s.kind == "beam":
        old, taken, rows, fresh = rows, set(), [], []
        parents = s.parent.cpu().tolist()
        for i, p in enumerate(parents):
            rows.append(list(old[p]) if p >= 0 else [])
            if p >= 0 and lens[p] % ps:
                if p in taken:
                    fresh.append(i)
                taken.add(p)
        lens = [lens[p] if p >= 0 else 0 for p in parents]
        kept = {q for i, r in enumerate(rows) for q in (r[:-1] if i in fresh else r)}
        free = iter(sorted(set(range(s.n_pages)) - kept))
        for i in fresh:
            moves.append((rows[i][-1], next(free)))
            rows[i][-1] = moves[-1][1]
    else:
        used = sorted({p for r in rows for p in r})
        holes = sorted(set(range(len(used))) - set(used))
        to = dict(zip([p for p in used if p >= len(used)], holes))
        moves = list(to.items())
        rows = [[to.get(p, p) for p in r] for r in rows]
    out = np.full(table.shape, -1, np.int32)
    for i, r in enumerate(rows):
        out[i, :len(r)] = r
    pool = s.pool.clone()
    for a, b in moves:
        pool[:, b] = s.pool[:, a]
    return [torch.from_numpy(out), torch.tensor(lens, dtype=torch.int32), pool]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if s.kind == "norm_rope":
        D, out = c["D"], []
        for x, gamma, heads, scale in ((s.q, s.gq, c["H"], D ** -0.5), (s.k, s.gk, c["Hkv"], 1.0)):
            x = x.double().view(-1, heads, 2, D // 2)
            norm = (x.pow(2).sum((2, 3), keepdim=True) / D + EPS).sqrt()
            z = torch.view_as_complex((x / norm * gamma.double().view(2, D // 2)).transpose(2, 3).contiguous())
            z = z * torch.view_as_complex(s.cs.double())[s.pos.long()][:, None] * scale
            out.append(torch.view_as_real(z).transpose(2, 3).reshape(-1, heads * D))
        return out
    if s.kind == "append":
        return [torch.from_numpy(_exact_rows(x.cpu().numpy(), c["Hkv"], c["D"])) for x in (s.k, s.v)]
    if s.kind == "attn":
        return _exact_attention(s)
    return _exact_pages(s)
