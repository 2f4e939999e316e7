"""The rotated append and the cache held in 4 bits, as measured cases.

A layer behind the boundary computes queries, keys and values, turns queries and keys by
their positions and puts keys and values into the paged cache; a cache whose pages hold 4
bits a value keeps 3.6 times as many tokens, and a decoded token reads as much less.  Four
operators of the package:

  rope     queries turned by their positions into a tensor of their own, keys turned and
           written to the cache's pages with their values (``gmc.cache_append_rope``); of a
           4-bit cache the new rows are read back as the values they stand for
           (``gmc.cache_read``)
  decode   one new token a sequence, its row already in the cache: its attention over a
           4-bit cache, and the weight that every key received added to the key's running
           score (``gmc.decode``)
  attend   the new tokens' causal attention over a 4-bit cache (``gmc.attend``)
  evict    every head's best-scored rows of a 4-bit cache moved to fresh pages
           (``gmc.evict``), and read back

What 4 bits hold: blocks of 16 channels of a bf16 row.  The scale s of a block is its
largest magnitude over 6, rounded to 3 bits behind the point of a half-precision number
(at least 2^-17, at most 8192), and a value is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4 and 6
times s, ties to the even one of these.  A head's part of a page holds the codes of its
slots, d / 2 bytes each with the even channel in the low half, and then their scales,
d / 16 bytes each: the upper bits of a positive half without its last seven.

Fields of a case (all plain values):
  op        rope | decode | attend | evict
  cache     "fp4", "bf16" or "f32": what the pages hold (rows are bf16, of "f32" fp32)
  B         sequences; ragged: their lengths differ, the first one has the largest
  H, Hkv, d query heads, key heads, head size
  L         tokens a sequence holds, the new ones included (the largest)
  T         new tokens a sequence (the largest of a ragged call)
  page      slots of a page
  window, sinks   keys that a query sees: itself and the window - 1 before it, and the
            first `sinks` of the sequence (window 0: every key up to itself)
  scores    decode: whether the running scores are kept
  keep, recent    evict: rows kept a head, and the last rows and the first `sinks` always are
  rot       rope: channels that turn, from the first on
  near      rope: a channel's partner is its neighbour, not the one half of `rot` further
  mrope     rope: (t, h, w) positions, each of which turns a section of the pairs
  packed    rope: queries, keys and values lie in rows of one projection's output
"""

import math

import torch

own = False

QWEN = dict(H=28, Hkv=4, d=128)
LLAVA = dict(H=32, Hkv=32, d=128)
GROUPED = dict(H=4, Hkv=2, d=64)
GRID = 36  # patches along a side of a prompt's image


def _case(name, op, cache, L, model, **more):
    c = dict(op=op, cache=cache, B=1, L=L, T=1, page=64, ragged=False, window=0, sinks=0,
             scores=False, keep=0, recent=0, rot=0, near=False, mrope=False, packed=False, **model)
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's next token: 28 query heads and 4 key heads turned, nothing but latency
        _case("rope qwen step", "rope", "bf16", 322, QWEN, page=16, rot=128, mrope=True,
              packed=True),
        # 32 questions of 16 to 256 tokens behind compressed prompts
        _case("rope serving questions", "rope", "bf16", 513, QWEN, B=32, T=256, ragged=True,
              rot=128, mrope=True, packed=True),
        # a LLaVA-1.5 prompt (576 visual and 32 text tokens) through a layer in fp32
        _case("rope llava prompt f32", "rope", "f32", 608, LLAVA, T=608, page=32, rot=128),
        # eight document prompts go into a cache of 4 bits
        _case("rope documents fp4", "rope", "fp4", 16004, QWEN, B=8, T=16004, page=128, rot=128,
              mrope=True, packed=True),
        # one user's next token after a compressed prompt
        _case("decode fp4 qwen", "decode", "fp4", 322, QWEN, page=16, scores=True),
        # the next token of 32 users at different points of their answers
        _case("decode fp4 serving", "decode", "fp4", 2085, QWEN, B=32, ragged=True, scores=True),
        # eight users' next token about uncompressed documents
        _case("decode fp4 documents", "decode", "fp4", 16005, QWEN, B=8, page=128),
        # 32 compressed prompts, 257 carriers each, whose questions of 16 to 256 tokens go
        # through the layers after the boundary
        _case("attend fp4 serving questions", "attend", "fp4", 513, QWEN, B=32, T=256, ragged=True),
        # a question of 128 tokens about an uncompressed document: few rows, many keys
        _case("attend fp4 document question", "attend", "fp4", 16004, QWEN, T=128),
        # the last piece of a document prompt that is prefilled 2,048 tokens at a time
        _case("attend fp4 document piece", "attend", "fp4", 16004, QWEN, T=2048, page=128),
        # a document's cache cut to a quarter, the question and the first tokens kept
        _case("evict fp4 document", "evict", "fp4", 16004, QWEN, keep=4096, recent=128, sinks=4),
        # 32 users' caches cut back to the size that they had after the compression
        _case("evict fp4 serving", "evict", "fp4", 1027, QWEN, B=32, ragged=True, keep=385,
              recent=64, sinks=4, page=16),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    model = rng.choice([QWEN, QWEN, QWEN, LLAVA, GROUPED, dict(H=8, Hkv=1, d=128),
                        dict(H=12, Hkv=2, d=64), dict(H=16, Hkv=1, d=64), dict(H=8, Hkv=2, d=256)])
    op = rng.choice(["rope"] * 4 + ["decode"] * 4 + ["attend"] * 3 + ["evict"] * 2)
    page = rng.choice([16, 16, 32, 48, 64, 64, 128, 256])
    H, Hkv, d = model["H"], model["Hkv"], model["d"]
    window = sinks = 0
    if rng.random() < 0.4:
        window, sinks = _log(rng, 16, 4096), rng.choice([0, 1, 4, 16, 64])
    L = _log(rng, 1, 16004)
    if op == "rope":
        cache = rng.choice(["fp4", "fp4", "bf16", "bf16", "f32"])
        if cache != "fp4" and rng.random() < 0.25:  # a head size of its own
            model = dict(H=H, Hkv=Hkv, d=rng.choice([80, 96]))
            d = model["d"]
        T = L if rng.random() < 0.5 else _log(rng, 1, L)
        # elements in and out, at most those of the eight documents
        row = (2 * H + (6 if cache == "fp4" else 4) * Hkv) * d * (2 if cache == "f32" else 1)
        B = _log(rng, 1, max(1, min(64, int(8 * 16004 * 72 * 128 / (row * T)), 8 * 16004 // L)))
        return _case(None, op, cache, L, model, B=B, T=T, page=page,
                     ragged=B > 1 and rng.random() < 0.6, rot=d if rng.random() < 0.6 else 32,
                     near=rng.random() < 0.3, mrope=rng.random() < 0.5, packed=rng.random() < 0.5)
    if op == "attend":
        T = L if rng.random() < 0.4 else _log(rng, 1, L)
        most = 16004 * 2048 * 28 * 128 / 2  # half of the listed document piece's products
        if d > 128:  # on the CUDA cores
            most /= 8
        while T > 1 and T * L * H * d > most:
            T = max(1, T // 2)
            L = max(T, L * 3 // 4)
        B = _log(rng, 1, max(1, min(32, int(most / (T * L * H * d)), 60000 // L)))
        return _case(None, op, "fp4", L, model, B=B, T=T, page=page,
                     ragged=B > 1 and rng.random() < 0.7, window=window, sinks=sinks)
    B = _log(rng, 1, max(1, min(64, 8 * 16004 * 512 // (Hkv * d * L))))
    while B == 1 and Hkv * d * L > 8 * 16004 * 512:
        L //= 2
    ragged = B > 1 and rng.random() < 0.7
    if op == "decode":
        return _case(None, op, "fp4", L, model, B=B, page=page, ragged=ragged, window=window,
                     sinks=sinks, scores=rng.random() < 0.6)
    B = min(B, max(1, 64020 // L))  # no more places than four documents' are sorted
    keep = max(1, int(L * rng.uniform(0.1, 0.9)))
    sinks = min(rng.choice([0, 1, 4]), keep)
    recent = rng.randint(0, (keep - sinks) // 2)
    return _case(None, op, "fp4", L, model, B=B, page=page, ragged=ragged and B > 1, keep=keep,
                 recent=recent, sinks=sinks)


def _lengths(c):
    """Tokens and new tokens of every sequence, the first with the largest: (lens, news)."""
    if not c["ragged"]:
        return [c["L"]] * c["B"], [c["T"]] * c["B"]
    import random
    rng = random.Random("lengths %d %d %d" % (c["B"], c["L"], c["T"]))
    lens, news = [c["L"]], [c["T"]]
    for _ in range(c["B"] - 1):
        if c["op"] in ("attend", "rope"):
            t = rng.randint(max(1, c["T"] // 16), c["T"])
            # what was there before the new tokens stays: the prompt's carriers
            lens.append(c["L"] - c["T"] + t)
            news.append(t)
        else:
            lens.append(rng.randint(max(1, c["L"] // 8), c["L"]))
            news.append(1)
    return lens, news


def _sections(c):
    """Pairs that turn by t, h and w: a quarter, three eighths and three eighths of them."""
    n = c["rot"] // 2
    return (n // 4, n // 4 + n // 8, n // 4 + n // 8) if c["mrope"] else (0, 0, 0)


def _ints(v, dev="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _sums(v):
    at = [0]
    for t in v:
        at.append(at[-1] + t)
    return at


# ---- 4 bits ------------------------------------------------------------------------------
def _levels():
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")


def _encode(x):
    """Codes [..., d / 2] and scales [..., d / 16], bytes, of rows [..., d] (bf16 values)."""
    x = x.float().unflatten(-1, (-1, 16))
    top = x.abs().amax(-1, keepdim=True)
    top = top / torch.full_like(top, 6.0)  # divided: a product with 1/6 misses ties
    # three bits behind the point: multiples of 2^-3 of the power of two below
    _, e = torch.frexp(top)
    unit = ((e - 4).clamp(min=-17) + 127 << 23).view(torch.float32)  # its bits: exact
    s = torch.round(top / unit) * unit
    s = torch.where(top > 0, s.clamp(2.0 ** -17, 8192.0), torch.zeros_like(s))
    y = x.abs() / torch.where(s > 0, s, torch.ones_like(s))
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5)
            + (y >= 3.5) + (y > 5.0))
    code = (code + 8 * (x < 0)).flatten(-2).to(torch.uint8)
    half = s.squeeze(-1).half().view(torch.int16).to(torch.int32) >> 7
    return code[..., 0::2] | (code[..., 1::2] << 4), half.to(torch.uint8)


def _decode_bytes(codes, scales):
    """The values of codes [..., d / 2] and scales [..., d / 16], fp32 [..., d]."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    v = _levels()[code & 7]
    v = torch.where(code >= 8, -v, v).unflatten(-1, (-1, 16))
    s = (scales.to(torch.int16) << 7).view(torch.half).float()
    return (v * s[..., None]).flatten(-2)


def _halves(c, pool):
    """Views of a pool's codes [pages, Hkv, page, d / 2] and scales [pages, Hkv, page, d / 16]."""
    n = c["page"] * c["d"] // 2
    return (pool[..., :n].unflatten(-1, (c["page"], c["d"] // 2)),
            pool[..., n:n + n // 8].unflatten(-1, (c["page"], c["d"] // 16)))


def _values(c, pool):
    """A pool's values, [pages, Hkv, page, d]."""
    return _decode_bytes(*_halves(c, pool)) if c["cache"] == "fp4" else pool


# ---- the inputs --------------------------------------------------------------------------
def _pages(c, rows, gen):
    """A pool of pages in no order, some of them another's: (k, v, page table)."""
    per = -(-rows // c["page"])
    n = c["B"] * per + 3
    shape = (n, c["Hkv"], c["page"], c["d"])

    def pool():
        x = torch.randn(shape, generator=gen, device="cuda").to(
            torch.float32 if c["cache"] == "f32" else torch.bfloat16)
        if c["cache"] != "fp4":
            return x
        codes, scales = _encode(x)
        # a head's part of a page in whole pieces of 16 bytes
        size = -(-c["page"] * c["d"] * 9 // 16 // 16) * 16
        p = torch.zeros(n, c["Hkv"], size, dtype=torch.uint8, device="cuda")
        a, b = _halves(c, p)
        a.copy_(codes)
        b.copy_(scales)
        return p

    table = torch.randperm(n, generator=gen, device="cuda")[:c["B"] * per]
    return pool(), pool(), table.to(torch.int32).reshape(c["B"], per).contiguous()


def _positions(c, lens, news):
    """Position ids of the new rows: one row of all (1-D), or three rows a sequence, one
    sequence after another.  An image of `side` x `side` patches lies at the start."""
    side = 126 if c["L"] >= 15876 else GRID
    got = []
    for n, t in zip(lens, news):
        j = torch.arange(n - t, n)
        if not c["mrope"]:
            got.append(j)
            continue
        seen = j < side * side
        text = j - side * side + side
        row = torch.div(j, side, rounding_mode="floor")
        got += [torch.where(seen, torch.zeros_like(j), text), torch.where(seen, row, text),
                torch.where(seen, j % side, text)]
    return torch.cat(got).to(torch.int32).cuda()


def _table(c, rows):
    """cos and sin of position p in row p: rot / 2 of each, from angles in 64 bits."""
    n = c["rot"] // 2
    rate = 1e6 ** (-torch.arange(n, dtype=torch.float64) / n)
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * rate
    return torch.cat([angle.cos(), angle.sin()], 1).float().cuda()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(6131 * int(seed) + 29)
    B, H, Hkv, d, L = c["B"], c["H"], c["Hkv"], c["d"], c["L"]
    dtype = torch.float32 if c["cache"] == "f32" else torch.bfloat16
    lens, news = _lengths(c)
    total = sum(news)
    s = {"case": c, "lens": _ints(lens), "ragged": c["ragged"]}
    s["k"], s["v"], s["table"] = _pages(c, L, gen)

    def rows(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    if c["op"] in ("attend", "rope"):
        at = _sums(news)
        s["at"] = torch.tensor(at, device="cuda")
        if c["ragged"]:
            s["offsets"] = _ints(at)
    if c["op"] == "rope":
        if c["packed"]:
            x = rows(total, H + 2 * Hkv, d).to(dtype)
            s["q"], s["k_new"], s["v_new"] = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
        else:
            s["q"], s["k_new"], s["v_new"] = (rows(total, n, d).to(dtype) for n in (H, Hkv, Hkv))
        s["positions"] = _positions(c, lens, news)
        s["cos_sin"] = _table(c, L + 1)
        s["out"] = torch.empty(total, H, d, device="cuda", dtype=dtype)
        if c["cache"] == "fp4":
            s["k_read"], s["v_read"] = (torch.empty(total, Hkv, d, device="cuda", dtype=dtype)
                                        for _ in range(2))
    if c["op"] in ("attend", "decode"):
        # every head's queries share a direction that the first keys of a sequence answer to
        u = rows(Hkv, d)
        n = min(4, c["page"])
        first = s["table"][:, 0].long()
        codes, scales = _encode((1.5 * u[None, :, None] + 0.3 * rows(B, Hkv, n, d)).to(dtype))
        a, b = _halves(c, s["k"])
        a[first, :, :n], b[first, :, :n] = codes, scales
        q = 2.0 * rows(total, Hkv, H // Hkv, d) + 0.5 * u[None, :, None]
        s["q"] = q.reshape(total, H, d).to(dtype)
        s["out"] = torch.empty(total, H, d, device="cuda", dtype=dtype)
        s["lse"] = torch.empty(total, H, device="cuda", dtype=torch.float32)
    if c["op"] == "evict" or c["scores"]:
        # what a key gathered so far: a few large sums, many small ones, some nothing
        x = torch.rand(B, Hkv, L, generator=gen, device="cuda")
        s["scores"] = torch.where(x < 0.05, torch.zeros_like(x), (rows(B, Hkv, L) * 1.5 - 3).exp())
        if c["op"] == "decode":
            s["new_scores"] = torch.zeros_like(s["scores"])
    if c["op"] == "evict":
        keep = c["keep"]
        kept = [min(keep, n) for n in lens]
        s["to_k"], s["to_v"], s["to_table"] = _pages(c, keep, gen)
        s["to_lens"] = _ints([0] * B)
        s["idx"] = torch.empty(B, Hkv, keep, dtype=torch.int32, device="cuda")
        s["kept"] = torch.empty(B, Hkv, keep, dtype=torch.float32, device="cuda")
        s["to_offsets"] = _ints(_sums(kept))
        s["k_read"], s["v_read"] = (torch.empty(sum(kept), Hkv, d, device="cuda", dtype=dtype)
                                    for _ in range(2))
    if own:  # the handles of the caches and the workspace of the calls, which a program keeps
        from paper_2608_02134_gb300 import gmc

        def cache(k, v, table, lens, most):
            if c["cache"] == "fp4":
                return gmc.KVCache4(k, v, table, lens, page_size=c["page"], d=d, max_len=most)
            return gmc.KVCache(k, v, table, lens, max_len=most)

        s["cache"] = cache(s["k"], s["v"], s["table"], s["lens"], L)
        if c["op"] == "rope":
            s["rope"] = gmc.Rope(s["cos_sin"], interleaved=c["near"],
                                 sections=_sections(c) if c["mrope"] else None)
        elif c["op"] == "attend":
            s["workspace"] = gmc.alloc_workspace(gmc.attend_workspace_size(s["cache"], H, c["T"]))
        elif c["op"] == "decode":
            s["workspace"] = gmc.alloc_workspace(gmc.decode_workspace_size(s["cache"], H))
        else:
            s["to"] = cache(s["to_k"], s["to_v"], s["to_table"], s["to_lens"], c["keep"])
            s["workspace"] = gmc.alloc_workspace(gmc.evict_workspace_size(s["cache"], c["keep"]))
    return s


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2608_02134_gb300 import gmc
        if c["op"] == "rope":
            gmc.cache_append_rope(s["cache"], s["rope"], s["k_new"], s["v_new"], c["T"],
                                  positions=s["positions"], q=s["q"], out=s["out"],
                                  offsets=s.get("offsets"))
            if c["cache"] != "fp4":
                return s["out"], s["k"], s["v"]
            gmc.cache_read(s["cache"], s["k_read"], s["v_read"], c["T"], offsets=s.get("offsets"))
            return s["out"], s["k_read"], s["v_read"]
        if c["op"] == "attend":
            gmc.attend(s["cache"], s["q"], s["out"], c["T"], q_offsets=s.get("offsets"),
                       window=c["window"], sinks=c["sinks"], lse=s["lse"],
                       workspace=s["workspace"])
            return s["out"], s["lse"]
        if c["op"] == "decode":
            gmc.decode(s["cache"], s["q"], s["out"], window=c["window"], sinks=c["sinks"],
                       lse=s["lse"], scores=s.get("scores"), out_scores=s.get("new_scores"),
                       workspace=s["workspace"])
            return s["out"], s["lse"], s.get("new_scores")
        gmc.evict(s["cache"], s["to"], s["scores"], c["keep"], s["idx"], s["kept"],
                  sinks=c["sinks"], recent=c["recent"], workspace=s["workspace"])
        gmc.cache_read(s["to"], s["k_read"], s["v_read"], c["keep"], offsets=s["to_offsets"])
        return s["idx"], s["kept"], s["to_lens"], s["k_read"], s["v_read"]
    return {"rope": _rope, "decode": _decode, "attend": _attend, "evict": _evict}[c["op"]](s)


# ---- the plain forms -------------------------------------------------------------------
def _owner(s):
    """Sequence, place among its new tokens and number of its new tokens, of every new row."""
    at = s["at"]
    row = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(at[1:], row, right=True)
    return b, row - at[b], (at[1:] - at[:-1])[b]


def _angles(s, wide):
    """cos and sin of every new row's pairs, [rows, 1, rot / 2]."""
    c, n = s["case"], s["case"]["rot"] // 2
    pos = s["positions"].long()
    if c["mrope"]:
        b, t, count = _owner(s)
        sect = torch.repeat_interleave(torch.arange(3, device="cuda"),
                                       torch.tensor(_sections(c), device="cuda"), output_size=n)
        where = (3 * s["at"][b] + t)[:, None] + sect * count[:, None]
        pos = pos[where]
    else:
        pos = pos[:, None].expand(-1, n)
    j = torch.arange(n, device="cuda")
    table = s["cos_sin"].to(wide)
    return table[pos, j][:, None], table[pos, j + n][:, None]


def _turn(c, x, cos, sin):
    """Rows [rows, heads, d] with their pairs turned."""
    n = c["rot"] // 2
    y = x.clone()
    i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if c["near"] else (slice(0, n), slice(n, 2 * n))
    a, b = x[..., i], x[..., j]
    y[..., i] = a * cos - b * sin
    y[..., j] = b * cos + a * sin
    return y


def _rope(s):
    c = s["case"]
    b, t, n = _owner(s)
    slot = s["lens"].long()[b] - n + t
    page = s["table"].long()[b, slot // c["page"]]
    slot = slot % c["page"]
    cos, sin = _angles(s, torch.float32)
    out = _turn(c, s["q"].float(), cos, sin).to(s["q"].dtype)
    if c["cache"] != "fp4":
        s["k"][page, :, slot] = _turn(c, s["k_new"].float(), cos, sin).to(s["k"].dtype)
        s["v"][page, :, slot] = s["v_new"]
        return out, s["k"], s["v"]
    cos, sin = _angles(s, torch.float64)  # a code goes by which side of a border a value lies on
    k = _turn(c, s["k_new"].double(), cos, sin).float().bfloat16()
    got = []
    for x, pool in ((k, s["k"]), (s["v_new"], s["v"])):
        a, z = _halves(c, pool)
        a[page, :, slot], z[page, :, slot] = _encode(x)
        got.append(_decode_bytes(a[page, :, slot], z[page, :, slot]).to(x.dtype))
    return out, got[0], got[1]


def _gather(s, pool, rows):
    """The first rows of every sequence, [B, Hkv, rows, d]."""
    B, Hkv, d = s["case"]["B"], s["case"]["Hkv"], s["case"]["d"]
    x = _values(s["case"], pool[s["table"].long()])
    return x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)[:, :, :rows]


def _softmax(logits, seen):
    """exp(x - max) over the seen keys, its sum and its logarithm; nothing seen gives zeros."""
    logits.masked_fill_(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return p, total, (top + total.log()).squeeze(-1)


def _attend(s):
    c = s["case"]
    B, H, Hkv, d, L, T = c["B"], c["H"], c["Hkv"], c["d"], c["L"], c["T"]
    b, t, _ = _owner(s)
    lens = s["lens"].long()
    news = s["at"][1:] - s["at"][:-1]
    place = torch.arange(T, device="cuda")
    where = (s["at"][:-1, None] + place).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][where].float().reshape(B, T, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4)
    j = torch.arange(L, device="cuda")
    held = j < lens[:, None]
    k = _gather(s, s["k"], L)
    v = _gather(s, s["v"], L).masked_fill(~held[:, None, :, None], 0.0)
    i = (lens - news)[:, None] + place
    seen = (j <= i[..., None]) & held[:, None]
    if c["window"]:
        seen = seen & ((j < c["sinks"]) | (i[..., None] - j < c["window"]))
    logits = (q.reshape(B, Hkv, -1, d) * (1.0 / math.sqrt(d))) @ k.transpose(2, 3)
    logits = logits.reshape(B, Hkv, H // Hkv, T, L)
    p, total, lse = _softmax(logits, seen[:, None, None])
    out = (p.reshape(B, Hkv, -1, L) @ v).reshape(B, Hkv, H // Hkv, T, d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    out = out.permute(0, 3, 1, 2, 4).reshape(B, T, H, d)[b, t]
    return out.to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B, T, H)[b, t]


def _decode(s):
    c = s["case"]
    B, H, Hkv, d, L = c["B"], c["H"], c["Hkv"], c["d"], c["L"]
    last = s["lens"].long() - 1
    j = torch.arange(L, device="cuda")
    seen = j <= last[:, None]
    k = _gather(s, s["k"], L)
    v = _gather(s, s["v"], L).masked_fill(~seen[:, None, :, None], 0.0)
    held = seen
    if c["window"]:
        seen = seen & ((j < c["sinks"]) | (last[:, None] - j < c["window"]))
    q = s["q"].float().reshape(B, Hkv, H // Hkv, d) * (1.0 / math.sqrt(d))
    p, total, lse = _softmax(q @ k.transpose(2, 3), seen[:, None, None])
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    out = (p @ v).reshape(B, H, d).to(s["q"].dtype)
    if c["scores"]:
        s["new_scores"] = torch.where(held[:, None], s["scores"] + p.sum(2), s["new_scores"])
    return out, lse.reshape(B, H), s.get("new_scores")


def _evict(s):
    c = s["case"]
    B, Hkv, L, keep, page = c["B"], c["Hkv"], c["L"], c["keep"], c["page"]
    lens = s["lens"].long()
    j = torch.arange(L, device="cuda")
    x = torch.where(torch.isnan(s["scores"]), -math.inf, s["scores"])
    always = (j < c["sinks"]) | (j >= lens[:, None] - c["recent"])
    x = torch.where(always[:, None], math.inf, x)
    x = torch.where((j < lens[:, None])[:, None], x, -math.inf)
    order = x.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    n = lens.clamp(max=keep)
    r = torch.arange(keep, device="cuda")
    there = (r < n[:, None])[:, None].expand(B, Hkv, keep)
    idx = torch.where(there, order, L).sort(-1).values
    safe = idx.clamp(max=L - 1)
    s["idx"] = torch.where(there, idx, -1).to(torch.int32)
    s["kept"] = torch.where(there, s["scores"].gather(2, safe), torch.zeros_like(s["kept"]))
    s["to_lens"] = n.to(torch.int32)
    head = torch.arange(Hkv, device="cuda")[None, :, None].expand(B, Hkv, keep)
    seq = torch.arange(B, device="cuda")[:, None, None]
    at = s["table"].long()[seq, safe // page]
    to = s["to_table"].long()[:, r // page][:, None].expand(B, Hkv, keep)
    slot = (r % page)[None, None].expand(B, Hkv, keep)
    got = []
    for pool, dest in ((s["k"], s["to_k"]), (s["v"], s["to_v"])):
        moved = []
        for a, z in zip(_halves(c, pool), _halves(c, dest)):
            rows = a[at, head, safe % page]
            z[to, head, slot] = torch.where(there[..., None], rows, z[to, head, slot])
            moved.append(z[to, head, slot].transpose(1, 2)[there.transpose(1, 2)[..., 0]])
        got.append(_decode_bytes(*moved).to(torch.bfloat16))
    return s["idx"], s["kept"], s["to_lens"], got[0], got[1]


# ---- what a pass cannot do without -------------------------------------------------------
def _pairs(c, n, t):
    """Query-key pairs that t new tokens of a sequence of n see, and the keys seen by any."""
    w, sk = c["window"], c["sinks"]
    if not w:
        return t * (n - t) + t * (t + 1) // 2, n
    i = torch.arange(n - t, n)
    lo = (i - w + 1).clamp(min=0)
    total = int((i - lo + 1 + lo.clamp(max=sk)).sum())
    lo = max(0, n - t - w + 1)
    return total, n - lo + min(sk, lo)


def work(case):
    c = case
    size = 4 if c["cache"] == "f32" else 2
    lens, news = _lengths(c)
    row = c["Hkv"] * c["d"] * size                                  # new or read back
    held = c["Hkv"] * c["d"] * 9 // 16 if c["cache"] == "fp4" else row  # in the cache
    if c["op"] == "rope":
        n = sum(news)
        pos = _positions_seen(c, lens, news)
        moved = n * (2 * c["H"] * c["d"] * size + 2 * row + 2 * held + (12 if c["mrope"] else 4))
        if c["cache"] == "fp4":
            moved += 2 * n * row  # read back
        return {"bytes": moved + 4 * c["rot"] * pos,
                "flops": 3 * c["rot"] * n * (c["H"] + c["Hkv"])}
    if c["op"] == "evict":
        kept = sum(min(c["keep"], n) for n in lens)
        return {"bytes": c["Hkv"] * (4 * sum(lens) + 8 * kept) + (4 * held + 2 * row) * kept,
                "flops": 0}
    pairs = keys = 0
    for n, t in zip(lens, news):
        p, u = _pairs(c, n, t)
        pairs, keys = pairs + p, keys + u
    moved = 2 * held * keys + (2 * c["d"] * size + 4) * c["H"] * sum(news)
    if c["scores"]:
        moved += 8 * c["Hkv"] * sum(lens)
    return {"bytes": moved, "flops": 4 * c["d"] * c["H"] * pairs}


def _positions_seen(c, lens, news):
    """Rows of the table that the new tokens' positions name."""
    if not c["mrope"]:
        return max(lens) - min(n - t for n, t in zip(lens, news))
    side = 126 if c["L"] >= 15876 else GRID
    last = max(lens) - 1
    return min(side, last + 1) + max(0, last - side * side + 1)


# ---- the definitions in 64 bits ------------------------------------------------------------
def _power(e):
    """2^e in 64 bits, exactly."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _nearest(x):
    """bf16 rows [..., d] as the values that 4 bits keep of them, in 64 bits."""
    x = x.double().unflatten(-1, (-1, 16))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=1e-30) / 6)).clamp(min=-14.0)
    e = torch.where(top >= 6 * _power(e + 1), e + 1, e)  # whatever the logarithm's last bit said
    e = torch.where(top < 6 * _power(e), e - 1, e).clamp(min=-14.0)
    unit = _power(e - 3)
    s = (torch.round(top / (6 * unit)) * unit).clamp(2.0 ** -17, 8192.0)
    s = torch.where(top > 0, s, torch.zeros_like(s))
    y = x.abs() / torch.where(s > 0, s, torch.ones_like(s))
    # spacing 0.5 below 2, 1 below 4, 2 below 6 and above; half of it goes to the even one
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    got = (torch.round(y / step) * step).clamp(max=6.0)
    return (torch.sign(x) * got * s).flatten(-2)


def _one(c, pool, table, b, n):
    """Rows 0 .. n-1 of sequence b, [n, Hkv, d] in 64 bits."""
    j = torch.arange(n, device="cuda")
    page = table[b].long()[torch.div(j, c["page"], rounding_mode="floor")]
    if c["cache"] != "fp4":
        return pool[page, :, j % c["page"]].double()
    x = pool[page]  # the row's bytes out of its page's
    half, sixteenth = c["d"] // 2, c["d"] // 16
    slot = (j % c["page"])[:, None, None]
    code = x.gather(2, (slot * half + torch.arange(half, device="cuda")).expand(n, x.shape[1], half))
    scale = x.gather(2, (c["page"] * half + slot * sixteenth + torch.arange(
        sixteenth, device="cuda")).expand(n, x.shape[1], sixteenth)).long()
    e, m = scale >> 3, (scale & 7).double()
    s = torch.where(e > 0, (1 + m / 8) * _power(e - 15), m * 2.0 ** -17)
    q = torch.stack([code & 15, code >> 4], -1).flatten(-2).long()
    e, m = (q >> 1) & 3, (q & 1).double()
    v = torch.where(e > 0, (1 + m / 2) * _power(e - 1), m / 2)
    v = torch.where(q > 7, -v, v)
    return v * s.repeat_interleave(16, -1)


def exact(case, seed):
    c = case
    if work(c)["flops"] > 2e12:
        return None
    s = prepare(c, seed)
    lens, news = _lengths(c)
    H, Hkv, d, L = c["H"], c["Hkv"], c["d"], c["L"]
    G = H // Hkv
    if c["op"] == "rope":
        n, at = c["rot"] // 2, 0
        which = [sum(([x] * m for x, m in enumerate(_sections(c))), [])] if c["mrope"] else [[0] * n]
        which = torch.tensor(which[0], device="cuda")
        out, kk, vv = [], [], []
        k_all, v_all = s["k"].double() if c["cache"] != "fp4" else None, None
        if k_all is not None:
            v_all = s["v"].double()
        pair = torch.arange(n, device="cuda")
        for b, (m, t) in enumerate(zip(lens, news)):
            pos = s["positions"][3 * at:3 * (at + t)].reshape(3, t) if c["mrope"] \
                else s["positions"][at:at + t].reshape(1, t)
            p = pos.long()[which].T
            w = torch.complex(s["cos_sin"][p, pair].double(), s["cos_sin"][p, pair + n].double())

            def turned(x):
                x = x.double()
                if c["near"]:
                    z = torch.view_as_complex(x[..., :2 * n].unflatten(-1, (n, 2)).contiguous())
                    y = torch.view_as_real(z * w[:, None]).flatten(-2)
                else:
                    z = torch.complex(x[..., :n].contiguous(), x[..., n:2 * n].contiguous())
                    z = z * w[:, None]
                    y = torch.cat([z.real, z.imag], -1)
                return torch.cat([y, x[..., 2 * n:]], -1)

            k, v = turned(s["k_new"][at:at + t]), s["v_new"][at:at + t].double()
            out.append(turned(s["q"][at:at + t]))
            if c["cache"] == "fp4":
                kk.append(_nearest(k.float().bfloat16()))
                vv.append(_nearest(v))
            else:
                j = torch.arange(m - t, m, device="cuda")
                page = s["table"][b].long()[torch.div(j, c["page"], rounding_mode="floor")]
                k_all[page, :, j % c["page"]] = k
                v_all[page, :, j % c["page"]] = v
            at += t
        if c["cache"] == "fp4":
            return torch.cat(out), torch.cat(kk), torch.cat(vv)
        return torch.cat(out), k_all, v_all
    if c["op"] == "evict":
        idx = torch.full((c["B"], Hkv, c["keep"]), -1, dtype=torch.int32)
        kept = torch.zeros(c["B"], Hkv, c["keep"], dtype=torch.float64)
        scores = s["scores"].double().cpu().numpy()
        k, v = [], []
        for b, n in enumerate(lens):
            m = min(c["keep"], n)
            K, V = _one(c, s["k"], s["table"], b, n), _one(c, s["v"], s["table"], b, n)
            rows = torch.empty(2, m, Hkv, d, dtype=torch.float64, device="cuda")
            for h in range(Hkv):
                rank = sorted(range(n), key=lambda j: (
                    not (j < c["sinks"] or j >= n - c["recent"]), -scores[b, h, j], j))
                got = sorted(rank[:m])
                idx[b, h, :m] = torch.tensor(got, dtype=torch.int32)
                kept[b, h, :m] = torch.from_numpy(scores[b, h, got])
                at = torch.tensor(got, device="cuda")
                rows[0, :, h], rows[1, :, h] = K[at, h], V[at, h]
            k.append(rows[0])
            v.append(rows[1])
        return idx, kept, _ints([min(c["keep"], n) for n in lens]), torch.cat(k), torch.cat(v)
    out = torch.zeros(sum(news), H, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(sum(news), H, dtype=torch.float64, device="cuda")
    sums = torch.zeros(c["B"], Hkv, L, dtype=torch.float64, device="cuda") if c["scores"] else None
    at = 0
    for b, (n, t) in enumerate(zip(lens, news)):
        K, V = _one(c, s["k"], s["table"], b, n), _one(c, s["v"], s["table"], b, n)
        i = torch.arange(n - t, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None]
        ok = j <= i
        if c["window"]:
            ok &= (j > i - c["window"]) | (j < c["sinks"])
        for h in range(H):
            w = s["q"][at:at + t, h].double() @ K[:, h // G].T / math.sqrt(d)
            w = w.masked_fill(~ok, -math.inf)
            z = torch.logsumexp(w, 1)
            w = (w - z[:, None]).exp()
            out[at:at + t, h], lse[at:at + t, h] = w @ V[:, h // G], z
            if sums is not None:
                sums[b, h // G, :n] += w[0]
        if sums is not None:
            sums[b, :, :n] += s["scores"][b, :, :n].double()
        at += t
    return (out, lse) if c["op"] == "attend" else (out, lse, sums)
