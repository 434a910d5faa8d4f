"""Performance cases of the attention half of a hybrid model: the norm and
rotation of query and key heads, the append of keys and values to a paged cache
held in E4M3 with one scale for each page and head, and the attention that reads
that cache, from one decode token to a whole prompt.

With ``own`` false, ``run`` computes each operator from elementary torch
operations; with ``own`` true it calls ``paper_2609_04098_amd.attention``.

Cache layout (bytes of one page and head, ``page`` tokens of ``d`` elements, in
groups of 16 tokens):
  keys    [page / 16][d / 16][16 tokens][16 elements]
  values  [page / 16][d / 64][4: t / 4][16: e % 16][4: e / 16 % 4][4: t % 4]
for token t of the group and element e of the head.
"""

import math

import torch

own = False

EPS = 1e-6
THETA = 1e6
SCALE_FLOOR = 2.0 ** -100      # the scale of a page that holds only zeros


def listed():
    return [
        # One token of a single user: the heads of one layer, latency only.
        dict(name="norm_rope_1", op="norm_rope", seqs=1, new=1, ctx=1000, ragged=False, hq=40, hkv=8, d=128, rot=128,
             interleaved=False, page=32),
        # A prompt of several users, wide heads, a quarter of each rotated.
        dict(name="norm_rope_prompts", op="norm_rope", seqs=6, new=2500, ctx=2500, ragged=True, hq=24, hkv=4, d=256,
             rot=64, interleaved=False, page=32),
        # One decode step of many users, each somewhere inside a page.
        dict(name="append_decode_96", op="append", seqs=96, new=1, ctx=700, ragged=True, hq=40, hkv=8, d=128,
             rot=128, interleaved=False, page=64),
        # A long prompt goes into fresh pages behind a shared first part.
        dict(name="append_prompt", op="append", seqs=1, new=16000, ctx=16391, ragged=False, hq=32, hkv=8, d=128,
             rot=128, interleaved=True, page=32),
        # One token of a single user in a short chat: latency.
        dict(name="attn_1_short", op="attention", seqs=1, new=1, ctx=500, ragged=False, hq=40, hkv=8, d=128, page=16,
             causal=True, window=0, lse=False),
        # One token of a single user behind a very long document: little to run side by side but the keys.
        dict(name="attn_1_long", op="attention", seqs=1, new=1, ctx=131072, ragged=False, hq=64, hkv=8, d=128,
             page=64, causal=True, window=0, lse=False),
        # A decode batch of chats of all lengths.
        dict(name="attn_decode_128", op="attention", seqs=128, new=1, ctx=8000, ragged=True, hq=40, hkv=8, d=128,
             page=16, causal=True, window=0, lse=True),
        # A decode batch of long documents, wide heads.
        dict(name="attn_decode_wide", op="attention", seqs=16, new=1, ctx=32768, ragged=True, hq=24, hkv=4, d=256,
             page=32, causal=True, window=0, lse=False),
        # Drafted tokens being verified by a model whose layers see a window.
        dict(name="attn_verify_window", op="attention", seqs=24, new=6, ctx=9000, ragged=True, hq=16, hkv=4, d=64,
             page=32, causal=True, window=4096, lse=False),
        # A whole prompt.
        dict(name="attn_prompt", op="attention", seqs=1, new=8192, ctx=8192, ragged=False, hq=40, hkv=8, d=128,
             page=64, causal=True, window=0, lse=False),
        # Prompts served in pieces: a piece of each behind what the cache already holds, wide heads.
        dict(name="attn_pieces_wide", op="attention", seqs=5, new=1024, ctx=7001, ragged=True, hq=16, hkv=2, d=256,
             page=64, causal=True, window=0, lse=True),
        # One decode step of one layer: norm and rotation, append, attention.
        dict(name="layer_decode_32", op="layer", seqs=32, new=1, ctx=3000, ragged=True, hq=32, hkv=8, d=128, rot=128,
             interleaved=False, page=32, causal=True, window=0, lse=False),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rope", "append", "attention", "attention", "attention", "layer"])
    d = rng.choice([64, 128, 128, 256])
    hkv = rng.choice([1, 2, 3, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 5, 6, 7, 8, 16])
    page = rng.choice([16, 32, 64, 128] if d < 256 else [16, 32, 64])
    c = dict(op=op, hq=hq, hkv=hkv, d=d, page=page, ragged=rng.random() < 0.7)
    if op != "attention":
        c.update(rot=rng.choice([0, 16 * rng.randint(1, d // 16), d]), interleaved=rng.random() < 0.4)
    if op in ("norm_rope", "append"):
        rows = max(1, _spread(rng, 1, 90e6 / ((hq + hkv) * d)))
        seqs = min(rows, _spread(rng, 1, 128))
        new = max(1, rows // seqs)
        c.update(seqs=seqs, new=new, ctx=new + _spread(rng, 1, 2000))
        return c
    prompt = op == "attention" and rng.random() < 0.4
    if prompt:
        ctx = _spread(rng, 1, 8192)
        new = max(1, int(ctx * rng.choice([1.0, rng.random()])))
        pairs = 8192 * 8192 * 40 * 128 // 2
        seqs = max(1, min(6, pairs // (ctx * new * hq * d)))
    else:
        new = rng.choice([1, 1, 1, rng.randint(2, 9)])
        ctx = new + _spread(rng, 1, 60000)
        seqs = max(1, min(_spread(rng, 1, 160), 260_000_000 // (ctx * hkv * d)))
    c.update(seqs=seqs, new=new, ctx=ctx, causal=op == "layer" or rng.random() < 0.85,
             window=rng.choice([0, 0, 0, rng.randint(1, ctx)]), lse=rng.random() < 0.5)
    return c


def _lengths(case):
    """Per sequence: (new rows, cached tokens with the new ones).  Ragged
    lengths go down to nothing from the stated largest ones."""
    got = []
    for b in range(case["seqs"]):
        if not case["ragged"] or b == 0:
            got.append((case["new"], max(case["ctx"], case["new"])))
            continue
        f = (b * 0.6180339887) % 1.0
        new = case["new"] if case["new"] == 1 and f > 0.03 else int(case["new"] * f)
        got.append((new, max(new, int(case["ctx"] * ((b * 0.7548776662) % 1.0)))))
    return got


def _pow2(e):
    """2^e in 64 bits, from its bits (powers computed on the GPU are not exact)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _pow2_scale(amax):
    """The smallest power of two s with amax <= 448 s, at least SCALE_FLOOR."""
    m, e = torch.frexp(amax.double() / 448.0)
    s = _pow2(torch.where(m == 0.5, e - 1, e)).clamp(min=SCALE_FLOOR)
    return torch.where(amax > 0, s, torch.full_like(s, SCALE_FLOOR)).to(amax.dtype)


def _k_pages(nat):
    """Keys [n, heads, page, d] in the cache's order."""
    n, h, p, d = nat.shape
    return nat.view(n, h, p // 16, 16, d // 16, 16).permute(0, 1, 2, 4, 3, 5).reshape(n, h, p * d)


def _k_tokens(k, p):
    n, h, b = k.shape
    d = b // p
    return k.view(n, h, p // 16, d // 16, 16, 16).permute(0, 1, 2, 4, 3, 5).reshape(n, h, p, d)


def _v_pages(nat):
    n, h, p, d = nat.shape
    return nat.view(n, h, p // 16, 4, 4, d // 64, 4, 16).permute(0, 1, 2, 5, 3, 7, 6, 4).reshape(n, h, p * d)


def _v_tokens(v, p):
    n, h, b = v.shape
    d = b // p
    return v.view(n, h, p // 16, d // 64, 4, 16, 4, 4).permute(0, 1, 2, 4, 7, 3, 6, 5).reshape(n, h, p, d)


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    lens = _lengths(case)
    p, d, hq, hkv = case["page"], case["d"], case["hq"], case["hkv"]
    rows = sum(n for n, _ in lens)
    cu = [0]
    for n, _ in lens:
        cu.append(cu[-1] + n)
    st = {"case": case, "rows": rows, "max_new": max(n for n, _ in lens), "max_len": max(c for _, c in lens)}
    i32 = dict(dtype=torch.int32, device=dev)
    st["cu"] = torch.tensor(cu, **i32)
    st["len"] = torch.tensor([c for _, c in lens], **i32)
    # Each row's sequence, its place among the sequence's new rows and its place in the cache.
    seq = [b for b, (n, _) in enumerate(lens) for _ in range(n)]
    off = [i for n, _ in lens for i in range(n)]
    st["row_seq"] = torch.tensor(seq, dtype=torch.int64, device=dev)
    st["row_off"] = torch.tensor(off, dtype=torch.int64, device=dev)
    slot = [lens[b][1] - lens[b][0] + i for b, i in zip(seq, off)]
    st["positions"] = torch.tensor(slot, **i32)
    # The projections of the new rows, as one fused GEMM leaves them.
    qkv = torch.randn(rows, (hq + 2 * hkv) * d, generator=gen, device=dev)
    qkv[:, (hq + hkv) * d:] *= torch.rand(hkv * d, generator=gen, device=dev) * 2
    qkv = qkv.to(torch.bfloat16)
    st["q"], st["k"], st["v"] = (qkv[:, a * d:b * d].view(rows, b - a, d) for a, b in
                                 ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    if "rot" in case:
        gamma = torch.rand(2, d, generator=gen, device=dev) + 0.5
        st["q_gamma"], st["k_gamma"] = gamma.to(torch.bfloat16)
        st["inv_freq"] = (THETA ** (-torch.arange(0, case["rot"], 2, device=dev).double() / max(1, case["rot"]))).float()
    if case["op"] == "norm_rope":
        return st
    if case["op"] == "attention":
        st["q"].mul_(2.0)
    # Pages in any order over the cache; a page and head has values of its own size.
    pages = [-(-c // p) for _, c in lens]
    width = max(1, max(pages))
    order = torch.randperm(sum(pages) + 3, generator=gen, device=dev).to(torch.int32)
    table, at = torch.zeros(len(lens), width, dtype=torch.int64), 0
    for b, n in enumerate(pages):
        table[b, :n] = torch.arange(at, at + n)
        at += n
    st["table"] = order[table.to(dev)]
    n_pages = order.numel()
    for name, pack in (("k", _k_pages), ("v", _v_pages)):
        nat = torch.randn(n_pages, hkv, p, d, generator=gen, device=dev)
        nat *= torch.rand(n_pages, hkv, 1, 1, generator=gen, device=dev) + 0.5
        s = _pow2_scale(nat.abs().amax(dim=(2, 3)))
        nat /= s[:, :, None, None]
        st[name + "_cache"] = pack(nat.to(torch.float8_e4m3fn).view(torch.uint8))
        st[name + "_scale"] = s
        del nat
    if case["op"] != "attention":
        page_of = st["table"].long()[st["row_seq"], st["positions"].long() // p]
        st["row_page"], st["row_slot"] = page_of, st["positions"].long() % p
        st["touched"] = torch.unique(page_of)          # the pages that this step writes to
    return st


def run(st):
    c = st["case"]
    if own:
        return _run_own(st, c)
    if c["op"] == "norm_rope":
        return {"q": _norm_rope(st["q"], st["q_gamma"], st["positions"], st["inv_freq"], c).to(torch.bfloat16),
                "k": _norm_rope(st["k"], st["k_gamma"], st["positions"], st["inv_freq"], c).to(torch.bfloat16)}
    if c["op"] == "append":
        return _append(st, c)
    if c["op"] == "attention":
        return _attention(st["q"], st, c)
    q = _norm_rope(st["q"], st["q_gamma"], st["positions"], st["inv_freq"], c).to(torch.bfloat16)
    got = _append(st, c)
    got.update(_attention(q, st, c))
    return got


def _run_own(st, c):
    from paper_2609_04098_amd import attention as A
    if "handles" not in st:     # what a serving loop holds: the rotation, the step's batch, the cache
        st["rope"] = A.Rope(st["inv_freq"], c["interleaved"]) if "rot" in c else None
        if "table" in st:
            st["batch"] = A.Batch(st["table"], st["len"], st["cu"], rows=st["rows"], max_len=st["max_len"])
            st["cache"] = A.KVCache(st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], c["page"])
        st["handles"] = True
    got = {}
    if c["op"] == "norm_rope":
        got["q"], got["k"] = A.qk_norm_rope(st["q"], st["k"], st["positions"], st["rope"], st["q_gamma"],
                                            st["k_gamma"], EPS)
        return got
    q = st["q"]
    if c["op"] == "layer":
        q, _ = A.qk_norm_rope(q, None, st["positions"], st["rope"], st["q_gamma"], None, EPS)
    if c["op"] != "attention":
        A.kv_append(st["cache"], st["batch"], st["k"], st["v"], st["k_gamma"], EPS, st["rope"])
        got = _cache_values(st)
    if c["op"] != "append":
        y = A.attention(q, st["cache"], st["batch"], causal=c["causal"], window=c["window"], return_lse=c["lse"])
        got["y"], got["lse"] = y if c["lse"] else (y, None)
    return got


def _cache_values(st):
    return {"k": st["k_cache"].view(torch.float8_e4m3fn), "v": st["v_cache"].view(torch.float8_e4m3fn),
            "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _norm_rope(x, gamma, positions, inv_freq, c, wide=torch.float32):
    """Norm of each head, then the rotation of its first elements; angles in 64 bits."""
    x = x.to(wide)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma.to(wide)
    rot = c["rot"]
    if rot == 0:
        return y
    angle = positions.double()[:, None] * inv_freq.double()[None, :]
    cos, sin = angle.cos().to(wide)[:, None, :], angle.sin().to(wide)[:, None, :]
    head, rest = y[..., :rot], y[..., rot:]
    if c["interleaved"]:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((turned, rest), dim=-1)


def _append(st, c):
    """New rows into their pages.  A page's scale is a power of two that only
    grows while the page fills (a page written from its first slot starts
    anew); tokens that it holds are brought to the grown scale."""
    p, hkv = c["page"], c["hkv"]
    # In 64 bits: the 8-bit rounding decides between neighbours 6 to 12 % apart.
    new = {"k": _norm_rope(st["k"], st["k_gamma"], st["positions"], st["inv_freq"], c, torch.float64),
           "v": st["v"].double()}
    page, slot, n_pages = st["row_page"], st["row_slot"], st["k_cache"].shape[0]
    first = torch.full((n_pages,), p, dtype=torch.int64, device=page.device).scatter_reduce(0, page, slot, "amin")
    for name, pack, unpack in (("k", _k_pages, _k_tokens), ("v", _v_pages, _v_tokens)):
        cache, scale = st[name + "_cache"], st[name + "_scale"]
        amax = torch.zeros(n_pages, hkv, dtype=torch.float64, device=page.device)
        amax.scatter_reduce_(0, page[:, None].expand(-1, hkv), new[name].abs().amax(-1), "amax")
        held = torch.where(first[:, None] > 0, scale.double(), torch.zeros_like(amax))
        grown = torch.maximum(held, _pow2_scale(amax))
        t = st["touched"]
        codes = unpack(cache[t], p).view(torch.float8_e4m3fn).float()
        behind = torch.arange(p, device=page.device)[None, :] >= first[t][:, None]      # left as they are
        codes *= torch.where(behind[:, None, :], 1.0, (held / grown)[t].float()[:, :, None])[..., None]
        values = (new[name] / grown[page][:, :, None]).float()
        codes = codes.to(torch.float8_e4m3fn).view(torch.uint8)
        where = torch.searchsorted(t, page)
        codes[where, :, slot] = values.to(torch.float8_e4m3fn).view(torch.uint8)
        cache[t] = pack(codes)
        scale[t] = grown[t].float()
    return _cache_values(st)


def _attention(q, st, c):
    """softmax(q k' / sqrt(d)) v over the cached tokens that each row sees."""
    p, d, hq, hkv = c["page"], c["d"], c["hq"], c["hkv"]
    group, seqs, n = hq // hkv, c["seqs"], st["max_new"]
    table = st["table"].long()
    length = table.shape[1] * p

    def gathered(cache, scale, unpack):
        x = unpack(cache[table.flatten()], p).view(torch.float8_e4m3fn).float()
        x *= scale[table.flatten()][:, :, None, None]
        return x.view(seqs, -1, hkv, p, d).transpose(1, 2).reshape(seqs, hkv, length, d)

    place = torch.arange(length, device=table.device)
    held = place[None, :] < st["len"][:, None]
    k = gathered(st["k_cache"], st["k_scale"], _k_tokens)
    row = (st["cu"][:-1, None].long() + torch.arange(n, device=table.device)).clamp(max=max(0, st["rows"] - 1))
    x = q.float()[row].view(seqs, n, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, group * n, d)
    s = torch.matmul(x, k.transpose(2, 3)).view(seqs, hkv, group, n, length) * (1 / math.sqrt(d))
    del k
    new = (st["cu"][1:] - st["cu"][:-1])
    at = (st["len"] - new)[:, None] + torch.arange(n, device=table.device)
    seen = held[:, None, :].expand(seqs, n, length)
    if c["causal"]:
        seen = seen & (place[None, None, :] <= at[:, :, None])
    if c["window"] > 0:
        seen = seen & (place[None, None, :] > at[:, :, None] - c["window"])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s -= torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    s.exp_()
    total = s.sum(-1, keepdim=True)
    v = gathered(st["v_cache"], st["v_scale"], _v_tokens).masked_fill_(~held[:, None, :, None], 0.0)
    y = torch.matmul(s.view(seqs, hkv, group * n, length), v).view(seqs, hkv, group, n, d)
    y = torch.where(total > 0, y / total, torch.zeros_like(y))
    b, i = st["row_seq"], st["row_off"]
    out = {"y": y.permute(0, 3, 1, 2, 4)[b, i].reshape(-1, hq, d).to(torch.bfloat16), "lse": None}
    if c["lse"]:
        out["lse"] = (top + total.log())[..., 0].permute(0, 3, 1, 2)[b, i].reshape(-1, hq)
    return out


def _seen(case):
    """Pairs of a query row and a token that it sees, and tokens that some row sees."""
    pairs = tokens = 0
    for n, length in _lengths(case):
        start, w = length - n, case["window"]
        lo = start
        for i in range(n):
            end = min(length, start + i + 1) if case["causal"] else length
            begin = max(0, start + i - w + 1) if w > 0 else 0
            pairs += max(0, end - begin)
            lo = begin if i == 0 else lo
        if n:
            tokens += length - lo
    return pairs, tokens


def work(case):
    lens = _lengths(case)
    rows, d, hq, hkv = sum(n for n, _ in lens), case["d"], case["hq"], case["hkv"]
    nbytes = flops = 0
    if case["op"] in ("norm_rope", "layer"):
        heads = hq + (hkv if case["op"] == "norm_rope" else 0)
        nbytes += 4 * rows * heads * d + 4 * rows + 4 * d
        flops += 7 * rows * heads * d
    if case["op"] in ("append", "layer"):
        pages = sum(-(-c // case["page"]) - (c - n) // case["page"] for n, c in lens if n)
        nbytes += rows * hkv * d * 2 * 3 + 16 * pages * hkv + 4 * pages + 8 * case["seqs"]
        flops += 10 * rows * hkv * d
    if case["op"] in ("attention", "layer"):
        pairs, tokens = _seen(case)
        # (a layer's queries, and the tokens that it appends, are produced by the same pass)
        nbytes += rows * hq * d * (4 if case["op"] == "attention" else 2) + (4 * rows * hq if case["lse"] else 0)
        nbytes += (tokens - (rows if case["op"] == "layer" else 0)) * hkv * 2 * d
        nbytes += -(-tokens // case["page"]) * (8 * hkv + 4)
        flops += 4 * pairs * hq * d
    return {"bytes": max(1, nbytes), "flops": flops}


# The definitions in 64 bits, by index arithmetic on the cache's bytes.


def _e4m3(code):
    """Values of E4M3 bytes, from their bits."""
    e, m = (code >> 3) & 15, (code & 7).double()
    v = torch.where(e > 0, (1 + m / 8) * _pow2(e - 7), m / 8 * 2.0 ** -6)
    v = torch.where((code & 127) == 127, torch.full_like(v, math.nan), v)
    return torch.where(code >= 128, -v, v)


def _to_e4m3(x):
    """The nearest E4M3 value of |x| <= 448, ties to the even one."""
    _, e = torch.frexp(x)
    step = _pow2((e - 1).clamp(min=-6) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _byte_of(p, d, values, device):
    """Place in a page's bytes of token t's element e, [p, d]."""
    t, e = torch.arange(p, device=device)[:, None], torch.arange(d, device=device)[None, :]
    g, u = t // 16, t % 16
    if values:
        return g * 16 * d + (e // 64) * 1024 + ((u // 4) * 16 + e % 16) * 16 + (e // 16 % 4) * 4 + u % 4
    return g * 16 * d + (e // 16) * 256 + u * 16 + e % 16


def _exact_rows(x, gamma, st, c):
    x = x.double()
    y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["d"] + EPS) * gamma.double()
    half = c["rot"] // 2
    if half:
        i = torch.arange(half, device=x.device)
        lo, hi = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device),
                           torch.outer(st["positions"].double(), st["inv_freq"].double()))[:, None, :]
        z = torch.complex(y[..., lo], y[..., hi]) * turn
        y[..., lo], y[..., hi] = z.real, z.imag
    return y


def _exact_append(st, c):
    p, d, dev = c["page"], c["d"], st["k"].device
    table, out = st["table"].cpu(), {}
    for name, values, rows in (("k", False, _exact_rows(st["k"], st["k_gamma"], st, c)), ("v", True, st["v"].double())):
        val = _e4m3(st[name + "_cache"].int())
        scale = st[name + "_scale"].double()
        place, r = _byte_of(p, d, values, dev), 0
        for b, (n, length) in enumerate(_lengths(c)):
            at = length - n
            while at < length:
                page, first = int(table[b, at // p]), at % p
                count = min(p - first, length - at)
                x = rows[r:r + count]                                  # [count, heads, d]
                big = x.abs().amax(dim=(0, 2)) / 448
                s = _pow2(torch.ceil(torch.log2(big.clamp(min=SCALE_FLOOR))))
                s = torch.where(s / 2 >= big, s / 2, s).clamp(min=SCALE_FLOOR)      # (log2 rounds)
                s = torch.where(s < big, s * 2, s)
                if first:
                    s = torch.maximum(s, scale[page])
                    old = place[:first].flatten()
                    val[page][:, old] = _to_e4m3(val[page][:, old] * (scale[page] / s)[:, None])
                val[page][:, place[first:first + count].flatten()] = \
                    _to_e4m3(x / s[None, :, None]).transpose(0, 1).reshape(c["hkv"], -1)
                scale[page] = s
                at, r = at + count, r + count
        out[name], out[name + "_scale"] = val, scale
    return out


def _exact_attention(q, kv, st, c):
    p, d, hkv, dev = c["page"], c["d"], c["hkv"], q.device
    group = c["hq"] // hkv
    y = torch.zeros(st["rows"], c["hq"], d, dtype=torch.float64, device=dev)
    lse = torch.full((st["rows"], c["hq"]), -math.inf, dtype=torch.float64, device=dev)
    kb, vb = _byte_of(p, d, False, dev).flatten(), _byte_of(p, d, True, dev).flatten()
    r = 0
    for b, (n, length) in enumerate(_lengths(c)):
        pages = st["table"][b, :-(-length // p)].long()
        for h in range(hkv if n and length else 0):
            k = (kv["k"][pages, h][:, kb] * kv["k_scale"][pages, h][:, None]).view(-1, d)[:length]
            v = (kv["v"][pages, h][:, vb] * kv["v_scale"][pages, h][:, None]).view(-1, d)[:length]
            for i in range(0, n, 2048):
                m = min(2048, n - i)
                x = q[r + i:r + i + m, h * group:(h + 1) * group].double().transpose(0, 1).reshape(-1, d)
                at = length - n + i + torch.arange(m, device=dev)[:, None]
                j = torch.arange(length, device=dev)[None, :]
                hide = (j > at) if c["causal"] else torch.zeros(m, length, dtype=torch.bool, device=dev)
                if c["window"] > 0:
                    hide = hide | (j <= at - c["window"])
                s = (x @ k.T / math.sqrt(d)).view(group, m, length).masked_fill(hide[None], -math.inf)
                total = torch.logsumexp(s, -1)
                w = torch.exp(s - torch.where(total.isinf(), torch.zeros_like(total), total)[..., None])
                y[r + i:r + i + m, h * group:(h + 1) * group] = (w.view(-1, length) @ v).view(group, m, d).transpose(0, 1)
                lse[r + i:r + i + m, h * group:(h + 1) * group] = total.T
        r += n
    return {"y": y, "lse": lse if c["lse"] else None}


def exact(case, seed):
    st = prepare(case, seed)
    c = case
    if c["op"] == "norm_rope":
        return {"q": _exact_rows(st["q"], st["q_gamma"], st, c), "k": _exact_rows(st["k"], st["k_gamma"], st, c)}
    q = st["q"]
    out = {}
    if c["op"] == "attention":
        kv = {n + "_scale": st[n + "_scale"].double() for n in "kv"}
        kv.update({n: _Codes(st[n + "_cache"]) for n in "kv"})
    else:
        kv = out = _exact_append(st, c)
    if c["op"] == "layer":
        q = _exact_rows(q, st["q_gamma"], st, c).to(torch.bfloat16)      # the queries are handed on in 16 bits
    if c["op"] != "append":
        out = {**out, **_exact_attention(q, kv, st, c)}
    return out


class _Codes:
    """Cache bytes that are decoded where they are read."""

    def __init__(self, codes):
        self.codes = codes

    def __getitem__(self, at):
        return _e4m3(self.codes[at].int())
