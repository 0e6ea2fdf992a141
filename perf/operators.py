"""The 4-bit key / value cache: its operators as cases, in plain torch form and through the framework's calls.

Kinds of cases:
  append     k and v rows quantised into the paged cache; returns the values that the cache then holds for them
  attention  rows of queries over the paged cache (decode, verification, prompt rows), with or without each cached
             token's attention weight added up
  step       one decode forward's use of a layer's cache: append of the new rows, then attention with weights
  evict      each head keeps the tokens of the largest added-up weights, moved together into other pages; returns which,
             their weights and the values that the new pages hold

The cache (the format and its layout are those of include/kangaroo.h): per token, key / value head and group of 32
components 16 numbers of 4 bits with a scale and a least value in half precision.  A physical page of T tokens holds for
each head, with G = D / 32 groups,
  keys    T rows of D / 2 bytes: words [q of 4][g of G], word (q, g) = components 32 g + 8 q + 0..7, lowest nibble first
  values  [T / 4][r of 16][h of D / 64][token of 4] halfwords of 4 nibbles i: component 16 (4 h + i) + r
  key scales [T / 4][G][4], key minima [T][G], value scales [T / 4][G][4], value minima [T / 4][G][4], all float16
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    def attn(name, **kw):
        c = {"name": name, "kind": "attention", "dtype": "f32", "D": 128, "heads": 32, "kv_heads": 32, "page": 128,
             "lens": "4096", "rows": "1", "max_len": 0, "weights": False}
        c.update(kw)
        return c
    return [
        # the smallest call: one row of the small model, a few tokens in the cache; latency of the launches
        attn("attn_toy_17", D=64, heads=4, kv_heads=4, page=16, lens="17"),
        # a token of the 7B model at the benchmark's context, float32 rows as they stand between its kernels
        attn("attn_7b_decode_500", lens="500"),
        # seven verification rows at the long context, the weights kept for the eviction
        attn("attn_7b_verify_4103", lens="4103", rows="7", weights=True),
        # one token of the 7B width over a very long cache: what reading the cache costs
        attn("attn_7b_decode_131001", lens="131001"),
        # ragged requests of a model with shared heads: one row each, from one token to thousands
        attn("attn_gqa_batch", dtype="bf16", heads=32, kv_heads=8, page=64, lens="1,37,513,1999,4096,7000,333,9001", rows="1,1,1,1,1,1,1,1"),
        # a chunk of a long prompt behind what is cached already
        attn("attn_7b_chunk_2048", dtype="bf16", lens="6144", rows="2048"),
        # uneven prompts of the 13B width, two at once, half-precision rows, the weights kept
        attn("attn_13b_prompts", dtype="f16", heads=40, kv_heads=40, page=32, lens="777,131", rows="777,131", weights=True),
        # a token's keys and values
        {"name": "append_7b_1", "kind": "append", "dtype": "f32", "D": 128, "kv_heads": 32, "page": 128, "lens": "4097", "rows": "1"},
        # a prompt's
        {"name": "append_7b_4096", "kind": "append", "dtype": "bf16", "D": 128, "kv_heads": 32, "page": 128, "lens": "4096", "rows": "4096"},
        # a layer's share of a decode step at the 33B width, weights kept
        {"name": "step_33b_2500", "kind": "step", "dtype": "f32", "D": 128, "heads": 52, "kv_heads": 52, "page": 128, "lens": "2500",
         "rows": "2", "max_len": 0, "weights": True},
        # a cache that has grown to twice its budget goes back to it
        {"name": "evict_7b_4096", "kind": "evict", "D": 128, "kv_heads": 32, "page": 128, "lens": "4096", "keep": 2048, "first": 4, "recent": 256},
        # several long requests with shared heads
        {"name": "evict_gqa_batch", "kind": "evict", "D": 128, "kv_heads": 8, "page": 64, "lens": "32768,16001,8000,30011", "keep": 8000,
         "first": 4, "recent": 1000},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "attention", "step", "append", "evict"])
    c = {"kind": kind, "D": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 64, 128])}
    g = rng.choice([1, 1, 1, 2, 4, 8])
    kv = rng.randint(1, 40) if g == 1 else rng.choice([1, 2, 4, 8])
    c["kv_heads"] = kv
    n_seqs = rng.choice([1, 1, 1, 2, rng.randint(3, 16)])
    if kind == "evict":
        lens = [_log(rng, 1, 32768 // n_seqs + 64) for _ in range(n_seqs)]
        keep = _log(rng, 1, max(2, max(lens)))
        first = rng.randint(0, min(4, keep))
        recent = rng.randint(0, keep - first)
        c.update(lens=_text(lens), keep=keep, first=first, recent=recent)
        return c
    c["dtype"] = rng.choice(["f32", "f32", "bf16", "f16"])
    if kind == "append":
        rows = [_log(rng, 1, 4096 // n_seqs) for _ in range(n_seqs)]
        c.update(lens=_text([r + _log(rng, 1, 2000) - 1 for r in rows]), rows=_text(rows))
        return c
    c["heads"] = kv * g
    few = kind == "step" or rng.random() < 0.6
    if few:
        rows = [rng.randint(1, 8) if rng.random() < 0.5 else 1 for _ in range(n_seqs)]
        lens = [r + _log(rng, 1, 60000 // n_seqs) - 1 for r in rows]
    else:
        rows = [_log(rng, 9, min(1500, 48000 // c["heads"]) // n_seqs) for _ in range(n_seqs)]
        lens = [r + _log(rng, 1, 4000) - 1 for r in rows]
    c.update(lens=_text(lens), rows=_text(rows), max_len=0 if rng.random() < 0.7 else max(lens) + _log(rng, 1, 4000),
             weights=kind == "step" or rng.random() < 0.4)
    return c


def _text(v):
    return ",".join(str(x) for x in v)


def _ints(t):
    return [int(x) for x in t.split(",")]


# ---- the format ---------------------------------------------------------------------------------

def _quantise(x):
    """x [..., D] -> (n uint8 [..., D], s, m float16 [..., D / 32])."""
    g = x.float().unflatten(-1, (-1, 32))
    bad = ~torch.isfinite(g).all(-1)
    g = g.clamp(-65504.0, 65504.0)
    lo, hi = g.amin(-1), g.amax(-1)
    m = lo.half()
    s = ((hi - lo) / 15.0).half()
    d = (g.double() - m.double()[..., None]) / torch.where(s == 0, 1.0, s.double())[..., None]     # 64 bits: next to a border 32 round the wrong way
    n = torch.where((s == 0)[..., None], 0.0, d.round().clamp(0.0, 15.0))
    n = torch.where(bad[..., None], 0.0, n)
    return n.to(torch.uint8).flatten(-2), torch.where(bad, math.nan, s.float()).half(), torch.where(bad, 0.0, m.float()).half()


def _block_bytes(T, D):
    return T * D * 5 // 4


def _pack(nk, sk, mk, nv, sv, mv, T, D):
    """Tokens [N][H] of the two quantised tensors, N a multiple of T -> blocks uint8 [N / T][H][bytes]."""
    N, H = nk.shape[:2]
    P, G = N // T, D // 32

    def page(t):                                               # [N, H, ...] -> [P, H, T, ...]
        return t.unflatten(0, (P, T)).transpose(1, 2)
    k = page(nk).reshape(P, H, T, G, 4, 8).transpose(3, 4)     # [T][q][g][8]
    k = k[..., 0::2] | (k[..., 1::2] << 4)
    v = page(nv).reshape(P, H, T // 4, 4, D // 64, 4, 16)      # [T/4][tok][h][i][r]
    v = v.permute(0, 1, 2, 6, 4, 3, 5)                         # [T/4][r][h][tok][i]
    v = v[..., 0::2] | (v[..., 1::2] << 4)

    def quads(t):                                              # [T][G] -> [T/4][G][4]
        return page(t).reshape(P, H, T // 4, 4, G).transpose(3, 4)

    def raw(t):
        return t.contiguous().view(torch.uint8).reshape(P, H, -1)
    return torch.cat([raw(k), raw(v), raw(quads(sk)), raw(page(mk)), raw(quads(sv)), raw(quads(mv))], -1)


def _unpack(blocks, T, D):
    """blocks uint8 [P][H][bytes] -> keys, values float32 [P * T][H][D]."""
    P, H = blocks.shape[:2]
    G = D // 32
    o = [0, T * D // 2, T * D, T * D + 2 * T * G, T * D + 4 * T * G, T * D + 6 * T * G, T * D + 8 * T * G]
    part = [blocks[..., o[i]:o[i + 1]].contiguous() for i in range(6)]
    k = part[0].reshape(P, H, T, 4, G, 4, 1)
    k = torch.cat([k & 15, k >> 4], -1).reshape(P, H, T, 4, G, 8).transpose(3, 4).reshape(P, H, T, G, 32)
    v = part[1].reshape(P, H, T // 4, 16, D // 64, 4, 2, 1)
    v = torch.cat([v & 15, v >> 4], -1).reshape(P, H, T // 4, 16, D // 64, 4, 4)
    v = v.permute(0, 1, 2, 5, 4, 6, 3).reshape(P, H, T, G, 32)

    def quads(t):
        return t.view(torch.float16).float().reshape(P, H, T // 4, G, 4).transpose(3, 4).reshape(P, H, T, G, 1)
    km = part[3].view(torch.float16).float().reshape(P, H, T, G, 1)
    keys = k.float() * quads(part[2]) + km
    values = v.float() * quads(part[4]) + quads(part[5])
    return (t.reshape(P, H, T, D).transpose(1, 2).reshape(P * T, H, D) for t in (keys, values))


def _cached(st, s, n):
    """Keys and values of the first n tokens of sequence s."""
    T, D, H = st["page"], st["D"], st["kv_heads"]
    pages = st["table"][s, : (n + T - 1) // T].long()
    blocks = st["pool"].view(-1, H, _block_bytes(T, D))[pages]
    return (t[:n] for t in _unpack(blocks, T, D))


# ---- what a program has in hand -----------------------------------------------------------------

def _gen(seed, *key):
    h = seed & 0xFFFFFFFF
    for k in key:
        h = (h * 1000003 + int(k) + 17) & 0x7FFFFFFFFFFF
    return torch.Generator(device="cuda").manual_seed(h)


def _rows(seed, key, n, heads, D, scale, dt):
    return (torch.randn(n, heads, D, generator=_gen(seed, *key), device="cuda") * scale).to(dt)


def _kv_rows(seed, key, n, heads, D, dt=torch.float32):
    """Keys and values as a model has them: a few components of the keys far larger than the others."""
    loud = 1.0 + 6.0 * (torch.rand(heads, D, generator=_gen(seed, 77), device="cuda") < 0.03)
    k = _rows(seed, key + (1,), n, heads, D, 1.0, torch.float32) * loud
    v = _rows(seed, key + (2,), n, heads, D, 0.5, torch.float32)
    return k.to(dt), v.to(dt)


def _table(seed, lens, page, spare):
    """Pages of the sequences in random order: page table [n_seqs][most pages of one], number of pages."""
    need = [(n + spare + page - 1) // page for n in lens]
    total = sum(need) + 3
    order = torch.randperm(total, generator=_gen(seed, 5), device="cuda").to(torch.int32)
    table = torch.zeros(len(lens), max(need), dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, total


def _starts(rows):
    out = [0]
    for r in rows:
        out.append(out[-1] + r)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    D, T, H, lens = case["D"], case["page"], case["kv_heads"], _ints(case["lens"])
    kind = case["kind"]
    st = dict(case, lens=lens)
    st["table"], n_pages = _table(seed, lens, T, 0)
    st["pool"] = torch.zeros(n_pages * H * _block_bytes(T, D), dtype=torch.uint8, device="cuda")
    st["len_dev"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if kind != "append":
        blocks = st["pool"].view(n_pages, H, -1)
        per = max(T, 8192 // T * T)
        for s, n in enumerate(lens):
            for t0 in range(0, n, per):
                m = min(per, (n - t0 + T - 1) // T * T)
                k, v = _kv_rows(seed, (6, s, t0), m, H, D)
                blocks[st["table"][s, t0 // T:(t0 + m) // T].long()] = _pack(*_quantise(k), *_quantise(v), T, D)
    cap = st["table"].shape[1] * T
    if kind == "evict":
        # what tens of thousands of softmax rows leave: a few tokens with most of it; tokens never looked at share a zero
        w = torch.randn(len(lens), H, cap, generator=_gen(seed, 9), device="cuda").mul_(2.0).exp_()
        st["w_in"] = torch.where(w < 0.05, 0.0, w)
        keep = case["keep"]
        st["dst_table"], dst_pages = _table(seed + 1, [keep] * len(lens), T, 0)
        st["dst_pool"] = torch.zeros(dst_pages * H * _block_bytes(T, D), dtype=torch.uint8, device="cuda")
        st["dst_len"] = torch.tensor([min(n, keep) for n in lens], dtype=torch.int32, device="cuda")
        st["dst_rows"] = [min(n, keep) for n in lens]
        st["w_out"] = torch.zeros(len(lens), H, st["dst_table"].shape[1] * T, device="cuda")
        st["kept"] = torch.empty(len(lens), H, keep, dtype=torch.int32, device="cuda")
        st["row_start"] = _starts(st["dst_rows"])
        n = sum(st["dst_rows"])
        st["k_out"], st["v_out"] = (torch.empty(n, H, D, device="cuda") for _ in range(2))
    else:
        rows = _ints(case["rows"])
        dt = DT[case["dtype"]]
        st["rows"], st["row_start"] = rows, _starts(rows)
        n = sum(rows)
        if kind in ("append", "step"):
            k, v = _kv_rows(seed, (7,), n, H, D, dt)
            st["kv_rows"] = torch.stack([k, v], 1)             # rows of one fused projection: k and v are strided views
        if kind == "append":
            st["k_out"], st["v_out"] = (torch.empty(n, H, D, device="cuda") for _ in range(2))
        else:
            st["q"] = _rows(seed, (8,), n, case["heads"], D, 1.5, dt)
            st["out"] = torch.empty_like(st["q"])
            st["scale"] = 1.0 / math.sqrt(D)
            if case["max_len"] == 0:
                st["max_len"] = max(lens)
            if case["weights"]:
                st["w_in"] = torch.rand(len(lens), H, cap, generator=_gen(seed, 9), device="cuda")
                st["w_out"] = torch.zeros_like(st["w_in"])
    if own:
        from paper_2404_18911_amd import binding as B
        st["B"] = B
        st["cache"] = B.Kv4Cache(st["pool"], st["table"], st["len_dev"], H, D, T)
        if kind == "evict":
            st["dst"] = B.Kv4Cache(st["dst_pool"], st["dst_table"], st["dst_len"], H, D, T)
        elif kind != "append":
            n_work = B.op_kv4_work_bytes(st["cache"], st["q"].shape[0], case["heads"], st["max_len"])
            st["work"] = torch.empty(n_work, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    return st


# ---- one pass -----------------------------------------------------------------------------------

def run(st):
    kind = st["kind"]
    if kind == "append":
        k, v = st["kv_rows"][:, 0], st["kv_rows"][:, 1]
        if own:
            st["B"].op_kv4_append(st["cache"], k, v, st["row_start"])
            st["B"].op_kv4_read(st["cache"], st["row_start"], st["k_out"], st["v_out"])
            return st["k_out"], st["v_out"]
        _plain_append(st, k, v)
        return _plain_read(st, st["lens"], st["rows"])
    if kind == "evict":
        if own:
            st["B"].op_kv4_evict(st["cache"], st["dst"], st["keep"], st["first"], st["recent"], st["w_in"], st["w_out"], st["kept"])
            st["B"].op_kv4_read(st["dst"], st["row_start"], st["k_out"], st["v_out"])
            return st["kept"], st["w_out"], st["k_out"], st["v_out"]
        return _plain_evict(st)
    if kind == "step":
        k, v = st["kv_rows"][:, 0], st["kv_rows"][:, 1]
        if own:
            st["B"].op_kv4_append(st["cache"], k, v, st["row_start"])
        else:
            _plain_append(st, k, v)
    if own:
        st["B"].op_kv4_attention(st["cache"], st["q"], st["row_start"], st["out"], st["max_len"], st["work"], st["scale"],
                                 st.get("w_in"), st.get("w_out"))
        return (st["out"], st["w_out"]) if st["weights"] else st["out"]
    return _plain_attention(st)


def _plain_append(st, k, v):
    """The rows' bytes put in their places, by pages: the pages that the rows fall into are taken apart, filled and stored."""
    T, D, H = st["page"], st["D"], st["kv_heads"]
    blocks = st["pool"].view(-1, H, _block_bytes(T, D))
    G, at = D // 32, 0
    qk, qv = _quantise(k), _quantise(v)
    for s, (n, r) in enumerate(zip(st["lens"], st["rows"])):
        t = torch.arange(n - r, n, device="cuda")
        page = st["table"][s, t // T].long()[:, None]
        tok, head = (t % T)[:, None], torch.arange(H, device="cuda")[None]
        quad, sub = tok // 4, tok % 4
        rows = slice(at, at + r)
        at += r
        o = [0, T * D // 2, T * D, T * D + 2 * T * G, T * D + 4 * T * G, T * D + 6 * T * G, T * D + 8 * T * G]

        def part(i, dt, *shape):
            return blocks[..., o[i]:o[i + 1]].view(dt).unflatten(-1, shape)
        kw = qk[0][rows].reshape(r, H, G, 4, 8).transpose(2, 3)
        kw = (kw[..., 0::2] | (kw[..., 1::2] << 4)).reshape(r, H, -1)
        part(0, torch.uint8, T, D // 2)[page, head, tok] = kw
        vw = qv[0][rows].reshape(r, H, D // 64, 4, 16).permute(0, 1, 4, 2, 3)          # [r][h][i]
        vw = (vw[..., 0::2] | (vw[..., 1::2] << 4))
        part(1, torch.uint8, T // 4, 16, D // 64, 4, 2)[page, head, quad, :, :, sub] = vw
        part(2, torch.float16, T // 4, G, 4)[page, head, quad, :, sub] = qk[1][rows]
        part(3, torch.float16, T, G)[page, head, tok] = qk[2][rows]
        part(4, torch.float16, T // 4, G, 4)[page, head, quad, :, sub] = qv[1][rows]
        part(5, torch.float16, T // 4, G, 4)[page, head, quad, :, sub] = qv[2][rows]


def _plain_read(st, lens, rows):
    ks, vs = [], []
    for s, (n, r) in enumerate(zip(lens, rows)):
        k, v = _cached(st, s, n)
        ks.append(k[n - r:])
        vs.append(v[n - r:])
    return torch.cat(ks), torch.cat(vs)


def _plain_attention(st):
    H, g, D = st["kv_heads"], st["heads"] // st["kv_heads"], st["D"]
    out, at = [], 0
    w_out = st["w_in"] * (torch.arange(st["w_in"].shape[2], device="cuda") < st["len_dev"][:, None])[:, None] if st["weights"] else None
    for s, (n, r) in enumerate(zip(st["lens"], st["rows"])):
        k, v = (t.transpose(0, 1) for t in _cached(st, s, n))                          # [H][n][D]
        q = st["q"][at:at + r].float().reshape(r, H, g, D).permute(1, 0, 2, 3).reshape(H, r * g, D)
        at += r
        z = (q * st["scale"]) @ k.transpose(1, 2).contiguous()
        if r > 1:
            pos = torch.arange(n - r, n, device="cuda").repeat_interleave(g)
            z.masked_fill_(torch.arange(n, device="cuda")[None] > pos[:, None], -math.inf)
        z = (z - z.amax(-1, keepdim=True)).exp_()
        z = z / z.sum(-1, keepdim=True)
        out.append((z @ v.contiguous()).reshape(H, r, g, D).permute(1, 0, 2, 3).reshape(r, H * g, D))
        if w_out is not None:
            w_out[s, :, :n] += z.sum(1)
    out = torch.cat(out).to(st["q"].dtype)
    return (out, w_out) if st["weights"] else out


def _plain_evict(st):
    T, D, H, keep = st["page"], st["D"], st["kv_heads"], st["keep"]
    kept = torch.full((len(st["lens"]), H, keep), -1, dtype=torch.int32, device="cuda")
    w_out = torch.zeros_like(st["w_out"])
    ks, vs = [], []
    G = D // 32
    dst = st["dst_pool"].view(-1, H, _block_bytes(T, D))
    for s, n in enumerate(st["lens"]):
        m = min(n, keep)
        w = st["w_in"][s, :, :n].clone()
        if n > keep:
            w[:, : st["first"]] = math.inf
            w[:, n - st["recent"]:] = math.inf
            order = torch.sort(w, dim=-1, descending=True, stable=True).indices[:, :keep]
            idx = order.sort(-1).values
        else:
            idx = torch.arange(n, device="cuda").expand(H, n)
        kept[s, :, :m] = idx.to(torch.int32)
        w_out[s, :, :m] = st["w_in"][s].gather(1, idx)
        # every token's bytes, in the order of the tokens
        src = st["pool"].view(-1, H, _block_bytes(T, D))[st["table"][s, : (n + T - 1) // T].long()]
        P, Q = src.shape[0], (m + T - 1) // T
        o = [0, T * D // 2, T * D, T * D + 2 * T * G, T * D + 4 * T * G, T * D + 6 * T * G, T * D + 8 * T * G]
        page = st["dst_table"][s, :Q].long()
        new = torch.zeros(Q, H, _block_bytes(T, D), dtype=torch.uint8, device="cuda")
        for i in range(6):
            b = src[..., o[i]:o[i + 1]]
            if i in (0, 3):                                    # [T][bytes]
                b = b.reshape(P, H, T, -1)
            else:                                              # [T / 4][pieces][4 tokens][2 bytes]
                b = b.reshape(P, H, T // 4, -1, 4, 2).transpose(3, 4).reshape(P, H, T, -1)
            b = b.transpose(0, 1).reshape(H, P * T, -1).gather(1, idx[..., None].expand(-1, -1, b.shape[-1]))
            f = torch.zeros(H, Q * T, b.shape[-1], dtype=torch.uint8, device="cuda")
            f[:, :m] = b
            f = f.reshape(H, Q, T, -1).transpose(0, 1)
            if i not in (0, 3):
                f = f.reshape(Q, H, T // 4, 4, -1, 2).transpose(3, 4)
            new[..., o[i]:o[i + 1]] = f.reshape(Q, H, -1)
        dst[page] = new
        k, v = _unpack(new, T, D)
        ks.append(k[:m])
        vs.append(v[:m])
    return kept, w_out, torch.cat(ks), torch.cat(vs)


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    D, H, lens = case["D"], case["kv_heads"], _ints(case["lens"])
    token = H * D * 5 // 4                                     # a cached token's bytes
    if case["kind"] == "evict":
        kept = sum(min(n, case["keep"]) for n in lens)
        # weights and kept tokens read; kept tokens, their weights and indices written; the new pages read and widened
        return {"bytes": 4 * H * sum(lens) + 2 * token * kept + 8 * H * kept + token * kept + 8 * H * D * kept, "flops": 4 * H * D * kept}
    rows = _ints(case["rows"])
    n, e = sum(rows), 4 if case["dtype"] == "f32" else 2
    append = n * (2 * H * D * e + token)
    if case["kind"] == "append":
        return {"bytes": append + n * (token + 8 * H * D), "flops": n * 12 * H * D}
    seen = sum(r * m - r * (r - 1) // 2 for r, m in zip(rows, lens))
    out = {"bytes": sum(lens) * token + 2 * n * case["heads"] * D * e, "flops": 4 * case["heads"] * D * seen}
    if case["weights"]:
        out["bytes"] += 8 * H * sum(lens)
    if case["kind"] == "step":
        out["bytes"] += append
        out["flops"] += n * 12 * H * D
    return out


# ---- the same in 64 bits ------------------------------------------------------------------------

def _exact_values(x):
    """What the cache holds of x [n][H][D], by the format's definition."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for c in range(0, x.shape[2], 32):
        g = x[:, :, c:c + 32].double().clamp(-65504.0, 65504.0)
        lo, hi = g.min(2, keepdim=True)[0], g.max(2, keepdim=True)[0]
        m = lo.to(torch.float32).to(torch.float16).double()
        span = (hi - lo).to(torch.float32)
        s = (span / 15).to(torch.float16).double()
        step = torch.round((g - m) / torch.where(s > 0, s, torch.ones_like(s)))
        step = torch.where(s > 0, step, torch.zeros_like(step)).clamp(0, 15)
        out[:, :, c:c + 32] = m + s * step
    return out


def _exact_token(st, pool, table, s, head, n):
    """Keys and values [n][D] of one head, looked up component by component."""
    T, D = st["page"], st["D"]
    G = D // 32
    dev = pool.device
    base = (table[s].long()[torch.arange(n, device=dev) // T] * st["kv_heads"] + head) * _block_bytes(T, D)
    t = (torch.arange(n, device=dev) % T)[:, None]
    d = torch.arange(D, device=dev)[None]
    g, base = d // 32, base[:, None]
    half = pool.view(torch.float16)
    kb = pool[base + t * (D // 2) + ((d % 32 // 8) * G + g) * 4 + d % 8 // 2]
    k = torch.where(d % 2 == 1, kb >> 4, kb & 15).double()
    j, r = d // 16, d % 16
    vb = pool[base + T * D // 2 + ((t // 4 * 16 + r) * (D // 64) + j // 4) * 8 + t % 4 * 2 + j % 4 // 2]
    v = torch.where(j % 2 == 1, vb >> 4, vb & 15).double()
    o = (base + T * D) // 2
    quad = (t // 4 * G + g) * 4 + t % 4
    k = k * half[o + quad].double() + half[o + T * G + t * G + g].double()
    v = v * half[o + 2 * T * G + quad].double() + half[o + 3 * T * G + quad].double()
    return k, v


def exact(case, seed):
    st = prepare(case, seed)
    kind, H = case["kind"], case["kv_heads"]
    if kind == "append":
        return tuple(_exact_values(st["kv_rows"][:, i]) for i in range(2))
    if kind == "evict":
        keep = case["keep"]
        w_out = torch.zeros(st["w_out"].shape, dtype=torch.float64, device="cuda")
        ks, vs = [], []
        for s, n in enumerate(st["lens"]):
            m = min(n, keep)
            k = torch.empty(m, H, case["D"], dtype=torch.float64, device="cuda")
            v = torch.empty_like(k)
            for h in range(H):
                w = st["w_in"][s, h, :n].double()
                ids = torch.arange(n, device="cuda")
                if n > keep:
                    free = (ids >= case["first"]) & (ids < n - case["recent"])
                    cand = ids[free]
                    # largest weight first, lowest index among equals
                    best = cand[torch.argsort(-w[cand], stable=True)][: keep - case["first"] - case["recent"]]
                    ids = torch.sort(torch.cat([ids[~free], best]))[0]
                w_out[s, h, :m] = w[ids]
                kh, vh = _exact_token(st, st["pool"], st["table"], s, h, n)
                k[:, h], v[:, h] = kh[ids], vh[ids]
            ks.append(k)
            vs.append(v)
        return None, w_out, torch.cat(ks), torch.cat(vs)
    D, g = case["D"], case["heads"] // H
    if H * sum(st["lens"]) * D > 6e8:
        return None
    new = [_exact_values(st["kv_rows"][:, i]) for i in range(2)] if kind == "step" else None
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    w = None
    if case["weights"]:
        w = torch.zeros(st["w_in"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for s, (n, r) in enumerate(zip(st["lens"], st["rows"])):
        pos = torch.arange(n - r, n, device="cuda")[:, None]
        hidden = torch.arange(n, device="cuda")[None] > pos
        for h in range(H):
            k, v = _exact_token(st, st["pool"], st["table"], s, h, n)
            if new is not None:
                k[n - r:], v[n - r:] = new[0][at:at + r, h], new[1][at:at + r, h]
            if w is not None:
                w[s, h, :n] = st["w_in"][s, h, :n].double()
            for j in range(h * g, h * g + g):
                z = st["q"][at:at + r, j].double() @ k.T * st["scale"]
                p = torch.softmax(z.masked_fill(hidden, -math.inf), -1)
                out[at:at + r, j] = p @ v
                if w is not None:
                    w[s, h, :n] += p.sum(0)
        at += r
    return (out, w) if case["weights"] else out
