"""What a program does with the key-value cache after the boundary compression, as measured cases.

A compressed prompt goes on in a paged cache: its kept rows are appended to the
cache's pages, the next tokens attend over them, single tokens are decoded one
after another, and a cache that has grown too long is cut back to the rows that
gathered the most attention.  Four operators of the package:

  append   rows of several sequences written to their pages (``gmc.cache_append``)
  attend   the new tokens' causal attention over the pages, whole or over a window and a
           few first tokens that stay visible (``gmc.attend``)
  decode   one new token a sequence: its key and value appended, its attention over the
           pages, and the weight that every key received added to the key's running score
           (``gmc.decode``)
  evict    every head's best-scored rows of a sequence moved to fresh pages
           (``gmc.evict``)

Fields of a case (all plain values):
  op        append | attend | decode | evict
  B         sequences; ragged: their lengths differ, the first one has the largest
  H, Hkv, d, dtype   query heads, key heads, head size, "bf16" or "f32"
  L         tokens a sequence holds, the new ones included (the largest)
  T         new tokens a sequence (append, attend; the largest of a ragged call)
  page      slots of a page
  window, sinks   keys that a query sees: itself and the window - 1 before it, and the
            first `sinks` of the sequence (window 0: every key up to itself)
  scores    decode: whether the running scores are kept
  keep, recent    evict: rows kept a head, and the last rows and the first `sinks` always are
  packed    append: the rows lie as the compression's output does, a sequence's keys and
            then its values
"""

import math

import torch

own = False

QWEN = dict(H=28, Hkv=4, d=128, dtype="bf16")
LLAVA = dict(H=32, Hkv=32, d=128, dtype="bf16")
LLAVA32 = dict(H=32, Hkv=32, d=128, dtype="f32")
SMALL32 = dict(H=4, Hkv=4, d=64, dtype="f32")
GROUPED = dict(H=4, Hkv=2, d=64, dtype="bf16")
GROUPED32 = dict(H=4, Hkv=2, d=64, dtype="f32")


def _case(name, op, L, model, **more):
    c = dict(op=op, B=1, L=L, T=1, page=64, ragged=False, window=0, sinks=0, scores=False, keep=0,
             recent=0, packed=False, **model)
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a LLaVA-1.5 prompt (576 visual and 32 text tokens) through a layer in fp32
        _case("attend llava prompt f32", "attend", 608, LLAVA32, T=608, page=32),
        # 32 compressed prompts, 257 carriers each, whose questions of 16 to 256 tokens
        # go through the layers after the boundary
        _case("attend serving questions", "attend", 513, QWEN, B=32, T=256, ragged=True),
        # a question of 128 tokens about an uncompressed document page: few rows, many keys
        _case("attend document question", "attend", 16004, QWEN, T=128, page=64),
        # the document prompt through a layer before the boundary
        _case("attend document prompt", "attend", 16004, QWEN, T=16004, page=128),
        # the same prompt where layers see a window of 4,096 and 16 first tokens
        _case("attend document window", "attend", 16004, QWEN, T=16004, page=64, window=4096,
              sinks=16),
        # one user's next token after a compressed prompt: nothing but latency
        _case("decode qwen", "decode", 322, QWEN, page=16, scores=True),
        # the next token of 32 users at different points of their answers
        _case("decode serving", "decode", 2085, QWEN, B=32, ragged=True, scores=True),
        # eight users' next token about uncompressed documents
        _case("decode documents", "decode", 16005, QWEN, B=8, page=128),
        # a document's cache cut to a quarter, the question and the first tokens kept
        _case("evict document", "evict", 16004, QWEN, keep=4096, recent=128, sinks=4),
        # 32 users' caches cut back to the size that they had after the compression
        _case("evict serving", "evict", 1027, QWEN, B=32, ragged=True, keep=385, recent=64,
              sinks=4, page=16),
        # 32 compressed prompts go into the cache: 257 carriers and 16 to 256 text tokens
        _case("append serving prompts", "append", 513, QWEN, B=32, T=513, ragged=True, packed=True),
        # eight document prompts go into the cache
        _case("append documents", "append", 16004, QWEN, B=8, T=16004, page=128),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    model = rng.choice([QWEN, QWEN, QWEN, LLAVA, GROUPED, dict(H=8, Hkv=1, d=128, dtype="bf16"),
                        dict(H=12, Hkv=2, d=64, dtype="bf16"), LLAVA32, SMALL32, GROUPED32,
                        dict(H=28, Hkv=4, d=128, dtype="f32")])
    op = rng.choice(["attend"] * 4 + ["decode"] * 4 + ["evict"] * 2 + ["append"] * 2)
    page = rng.choice([16, 16, 32, 48, 64, 64, 128, 256])
    size = 2 if model["dtype"] == "bf16" else 4
    window = sinks = 0
    if rng.random() < 0.4:
        window, sinks = _log(rng, 16, 4096), rng.choice([0, 1, 4, 16, 64])
    L = _log(rng, 1, 16004)
    if op == "attend":
        T = L if rng.random() < 0.4 else _log(rng, 1, L)
        # at most a tenth of the document prompt's products (fp32: a hundredth)
        most = (7e9 if size == 2 else 7e8) / 28
        while T > 1 and T * L * model["H"] * model["d"] > most * 28 * 128:
            T = max(1, T // 2)
            L = max(T, L * 3 // 4)
        B = _log(rng, 1, max(1, min(32, int(most * 28 * 128 / (T * L * model["H"] * model["d"])),
                                    200000 // L)))
        return _case(None, op, L, model, B=B, T=T, page=page, ragged=B > 1 and rng.random() < 0.7,
                     window=window, sinks=sinks)
    # bytes of the rows: at most those of the eight documents
    row = 2 * model["Hkv"] * model["d"] * size
    B = _log(rng, 1, max(1, min(64, int(8 * 16004 * 2048 / (row * L)))))
    ragged = B > 1 and rng.random() < 0.7
    while B == 1 and row * L > 8 * 16004 * 2048:
        L = L // 2
    if op == "decode":
        return _case(None, op, L, model, B=B, page=page, ragged=ragged, window=window, sinks=sinks,
                     scores=rng.random() < 0.6)
    if op == "evict":
        keep = max(1, int(L * rng.uniform(0.1, 0.9)))
        sinks = min(rng.choice([0, 1, 4]), keep)
        recent = rng.randint(0, (keep - sinks) // 2)
        return _case(None, op, L, model, B=B, page=page, ragged=ragged, keep=keep, recent=recent,
                     sinks=sinks)
    T = L if rng.random() < 0.6 else _log(rng, 1, L)
    return _case(None, op, L, model, B=B, T=T, page=page, ragged=ragged,
                 packed=rng.random() < 0.5)


def _lengths(c):
    """Tokens and new tokens of every sequence, the first with the largest: (lens, news)."""
    if not c["ragged"]:
        return [c["L"]] * c["B"], [c["T"]] * c["B"]
    import random
    rng = random.Random("lengths %d %d %d" % (c["B"], c["L"], c["T"]))
    lens, news = [c["L"]], [c["T"]]
    for _ in range(c["B"] - 1):
        if c["op"] in ("attend", "append"):
            t = rng.randint(max(1, c["T"] // 16), c["T"])
            # what was there before the new tokens stays: the prompt's carriers
            lens.append(c["L"] - c["T"] + t)
            news.append(t)
        else:
            lens.append(rng.randint(max(1, c["L"] // 8), c["L"]))
            news.append(1)
    return lens, news


def _ints(v, dev="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _pages(c, rows, gen, dtype):
    """A pool of pages in no order, some of them another's: (k, v, page table)."""
    per = -(-rows // c["page"])
    n = c["B"] * per + 3
    shape = (n, c["Hkv"], c["page"], c["d"])
    k = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)
    v = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)
    table = torch.randperm(n, generator=gen, device="cuda")[:c["B"] * per]
    return k, v, table.to(torch.int32).reshape(c["B"], per).contiguous()


def prepare(case, seed):
    c = case
    dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(7919 * int(seed) + 17)
    B, H, Hkv, d, L = c["B"], c["H"], c["Hkv"], c["d"], c["L"]
    lens, news = _lengths(c)
    s = {"case": c, "lens": _ints(lens), "ragged": c["ragged"]}
    s["k"], s["v"], s["table"] = _pages(c, L, gen, dtype)

    def rows(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    if c["op"] in ("attend", "decode"):
        total = sum(news)
        # every head's queries share a direction that the first keys of a sequence answer to
        u = rows(Hkv, d)
        first = s["table"][:, 0].long()
        n = min(4, c["page"])
        s["k"][first, :, :n] = (1.5 * u[None, :, None] + 0.3 * rows(B, Hkv, n, d)).to(dtype)
        q = 2.0 * rows(total, Hkv, H // Hkv, d) + 0.5 * u[None, :, None]
        s["q"] = q.reshape(total, H, d).to(dtype)
        s["out"] = torch.empty(total, H, d, device="cuda", dtype=dtype)
        s["lse"] = torch.empty(total, H, device="cuda", dtype=torch.float32)
    if c["op"] in ("attend", "append") and c["ragged"]:
        at = [0]
        for t in news:
            at.append(at[-1] + t)
        s["offsets"] = _ints(at)
    if c["op"] == "append":
        total = sum(news)
        if c["packed"]:
            s["kv"] = rows(2 * total, Hkv, d).to(dtype)
        else:
            s["k_new"], s["v_new"] = rows(total, Hkv, d).to(dtype), rows(total, Hkv, d).to(dtype)
    if c["op"] == "decode":
        s["k_new"], s["v_new"] = rows(B, Hkv, d).to(dtype), rows(B, Hkv, d).to(dtype)
    if c["op"] == "evict" or c["scores"]:
        # what a key gathered so far: a few large sums, many small ones, some nothing
        x = torch.rand(B, Hkv, L, generator=gen, device="cuda")
        s["scores"] = torch.where(x < 0.05, torch.zeros_like(x), (rows(B, Hkv, L) * 1.5 - 3).exp())
        if c["op"] == "decode":
            s["new_scores"] = torch.zeros_like(s["scores"])
    if c["op"] == "evict":
        keep = c["keep"]
        s["to_k"], s["to_v"], s["to_table"] = _pages(c, keep, gen, dtype)
        s["to_lens"] = _ints([0] * B)
        s["idx"] = torch.empty(B, Hkv, keep, dtype=torch.int32, device="cuda")
        s["kept"] = torch.empty(B, Hkv, keep, dtype=torch.float32, device="cuda")
    if own:  # the handles of the caches and the workspace of the calls, which a program keeps
        from paper_2608_02134_gb300 import gmc
        s["cache"] = gmc.KVCache(s["k"], s["v"], s["table"], s["lens"], max_len=L)
        if c["op"] == "attend":
            n = gmc.attend_workspace_size(s["cache"], H, c["T"])
        elif c["op"] == "decode":
            n = gmc.decode_workspace_size(s["cache"], H)
        elif c["op"] == "evict":
            s["to"] = gmc.KVCache(s["to_k"], s["to_v"], s["to_table"], s["to_lens"],
                                  max_len=c["keep"])
            n = gmc.evict_workspace_size(s["cache"], c["keep"])
        else:
            n = 0
        s["workspace"] = gmc.alloc_workspace(n)
    return s


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2608_02134_gb300 import gmc
        if c["op"] == "attend":
            gmc.attend(s["cache"], s["q"], s["out"], c["T"], q_offsets=s.get("offsets"),
                       window=c["window"], sinks=c["sinks"], lse=s["lse"],
                       workspace=s["workspace"])
            return s["out"], s["lse"]
        if c["op"] == "decode":
            gmc.decode(s["cache"], s["q"], s["out"], k_new=s["k_new"], v_new=s["v_new"],
                       window=c["window"], sinks=c["sinks"], lse=s["lse"],
                       scores=s.get("scores"), out_scores=s.get("new_scores"),
                       workspace=s["workspace"])
            return s["out"], s["lse"], s["k"], s["v"], s.get("new_scores")
        if c["op"] == "evict":
            gmc.evict(s["cache"], s["to"], s["scores"], c["keep"], s["idx"], s["kept"],
                      sinks=c["sinks"], recent=c["recent"], workspace=s["workspace"])
            return s["idx"], s["kept"], s["to_lens"], s["to_k"], s["to_v"]
        if c["packed"]:
            gmc.cache_append(s["cache"], s["kv"], None, c["T"], offsets=s.get("offsets"))
        else:
            gmc.cache_append(s["cache"], s["k_new"], s["v_new"], c["T"], offsets=s.get("offsets"))
        return s["k"], s["v"]
    return {"attend": _attend, "decode": _decode, "evict": _evict, "append": _append}[c["op"]](s)


# ---- the plain forms -------------------------------------------------------------------
def _gather(s, pool, rows):
    """The first rows of every sequence, [B, Hkv, rows, d]."""
    B, Hkv, d = s["case"]["B"], s["case"]["Hkv"], s["case"]["d"]
    x = pool[s["table"].long()]
    return x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)[:, :, :rows]


def _owner(s):
    """Sequence, place among its new tokens and number of its new tokens, of every new row."""
    c = s["case"]
    if s["ragged"]:
        at = s["offsets"].long()
    else:
        at = torch.arange(c["B"] + 1, device="cuda") * c["T"]
    total = s["k_new"].shape[0] if "k_new" in s else s["kv"].shape[0] // 2 if "kv" in s \
        else s["q"].shape[0]
    row = torch.arange(total, device="cuda")
    b = torch.searchsorted(at[1:], row, right=True)
    return b, row - at[b], (at[1:] - at[:-1])[b], at


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
    b, t, n, at = _owner(s)
    lens = s["lens"].long()
    news = at[1:] - at[:-1]
    place = torch.arange(T, device="cuda")
    where = (at[:-1, None] + place).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][where].float().reshape(B, T, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4)
    j = torch.arange(L, device="cuda")
    held = j < lens[:, None]
    k = _gather(s, s["k"], L).float()
    v = _gather(s, s["v"], L).float().masked_fill(~held[:, None, :, None], 0.0)
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
    lens = s["lens"].long()
    last = lens - 1
    page = s["table"].long().gather(1, (last // c["page"])[:, None])[:, 0]
    s["k"][page, :, last % c["page"]] = s["k_new"]
    s["v"][page, :, last % c["page"]] = s["v_new"]
    j = torch.arange(L, device="cuda")
    seen = j < lens[:, None]
    k = _gather(s, s["k"], L).float()
    v = _gather(s, s["v"], L).float().masked_fill(~seen[:, None, :, None], 0.0)
    held = seen
    if c["window"]:
        seen = seen & ((j < c["sinks"]) | (last[:, None] - j < c["window"]))
    q = s["q"].float().reshape(B, Hkv, H // Hkv, d) * (1.0 / math.sqrt(d))
    p, total, lse = _softmax(q @ k.transpose(2, 3), seen[:, None, None])
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    out = (p @ v).reshape(B, H, d).to(s["q"].dtype)
    if c["scores"]:
        before = torch.where(j == last[:, None], 0.0, 1.0)[:, None] * s["scores"]
        s["new_scores"] = torch.where(held[:, None], before + p.sum(2), s["new_scores"])
    return out, lse.reshape(B, H), s["k"], s["v"], s.get("new_scores")


def _evict(s):
    c = s["case"]
    B, Hkv, d, L, keep = c["B"], c["Hkv"], c["d"], c["L"], c["keep"]
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
    page = s["to_table"].long()[:, r // c["page"]][:, None].expand(B, Hkv, keep)
    head = torch.arange(Hkv, device="cuda")[None, :, None].expand(B, Hkv, keep)
    slot = (r % c["page"])[None, None].expand(B, Hkv, keep)
    where = safe[..., None].expand(B, Hkv, keep, d)
    s["to_k"][page, head, slot] = torch.where(there[..., None], _gather(s, s["k"], L).gather(2, where),
                                              s["to_k"][page, head, slot])
    s["to_v"][page, head, slot] = torch.where(there[..., None], _gather(s, s["v"], L).gather(2, where),
                                              s["to_v"][page, head, slot])
    s["to_lens"] = n.to(torch.int32)
    return s["idx"], s["kept"], s["to_lens"], s["to_k"], s["to_v"]


def _append(s):
    c = s["case"]
    b, t, n, at = _owner(s)
    slot = s["lens"].long()[b] - n + t
    page = s["table"].long()[b, slot // c["page"]]
    if c["packed"]:
        k, v = s["kv"][2 * at[b] + t], s["kv"][2 * at[b] + n + t]
    else:
        k, v = s["k_new"], s["v_new"]
    s["k"][page, :, slot % c["page"]] = k
    s["v"][page, :, slot % c["page"]] = v
    return s["k"], s["v"]


# ---- what a pass cannot do without -------------------------------------------------------
def _pairs(c, n, t):
    """Query-key pairs that t new tokens of a sequence of n see, and the keys seen by any."""
    w, sk = c["window"], c["sinks"]
    if not w:
        return t * (n - t) + t * (t + 1) // 2, n
    total = 0
    for i in (range(n - t, n) if t <= 4096 else ()):
        lo = max(0, i - w + 1)
        total += i - lo + 1 + min(sk, lo)
    if t > 4096:
        i = torch.arange(n - t, n)
        lo = (i - w + 1).clamp(min=0)
        total = int((i - lo + 1 + lo.clamp(max=sk)).sum())
    lo = max(0, n - t - w + 1)
    return total, n - lo + min(sk, lo)


def work(case):
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    lens, news = _lengths(c)
    row = c["Hkv"] * c["d"] * size
    if c["op"] == "append":
        return {"bytes": 4 * row * sum(news), "flops": 0}
    if c["op"] == "evict":
        kept = sum(min(c["keep"], n) for n in lens)
        return {"bytes": c["Hkv"] * (4 * sum(lens) + 8 * kept) + 4 * row * kept, "flops": 0}
    pairs = keys = 0
    for n, t in zip(lens, news):
        p, u = _pairs(c, n, t)
        pairs, keys = pairs + p, keys + u
    moved = 2 * row * keys + 2 * c["H"] * c["d"] * size * sum(news) + 4 * c["H"] * sum(news)
    if c["op"] == "decode":
        moved += 2 * row * c["B"] + (8 * c["Hkv"] * sum(lens) if c["scores"] else 0)
    return {"bytes": moved, "flops": 4 * c["d"] * c["H"] * pairs}


# ---- the definitions in 64 bits ------------------------------------------------------------
def _one(s, pool, b, h, n):
    """Rows 0 .. n-1 of one sequence and head in 64 bits."""
    ps = s["case"]["page"]
    j = torch.arange(n, device="cuda")
    return pool[s["table"][b].long()[torch.div(j, ps, rounding_mode="floor")], h, j % ps].double()


def _seen(c, i, n):
    """[queries, n] truth values: key j of n is visible to the query at place i."""
    j = torch.arange(n, device="cuda")[None]
    ok = j <= i[:, None]
    if c["window"]:
        ok &= (j > i[:, None] - c["window"]) | (j < c["sinks"])
    return ok


def exact(case, seed):
    c = case
    if work(c)["flops"] > 4e12:
        return None
    s = prepare(c, seed)
    lens, news = _lengths(c)
    G, d = c["H"] // c["Hkv"], c["d"]
    if c["op"] == "append":
        k, v, at = s["k"].double(), s["v"].double(), 0
        for b, (n, t) in enumerate(zip(lens, news)):
            for x in range(0, t, c["page"]):  # from one page's border to the next
                pos = torch.arange(n - t + x, min(n - t + x + c["page"], n), device="cuda")
                page = s["table"][b].long()[torch.div(pos, c["page"], rounding_mode="floor")]
                m = pos.numel()
                if c["packed"]:
                    kn, vn = s["kv"][2 * at + x:][:m], s["kv"][2 * at + t + x:][:m]
                else:
                    kn, vn = s["k_new"][at + x:][:m], s["v_new"][at + x:][:m]
                k[page, :, pos % c["page"]] = kn.double()
                v[page, :, pos % c["page"]] = vn.double()
            at += t
        return k, v
    if c["op"] == "evict":
        k, v = s["to_k"].double(), s["to_v"].double()
        idx = torch.full((c["B"], c["Hkv"], c["keep"]), -1, dtype=torch.int32)
        kept = torch.zeros(c["B"], c["Hkv"], c["keep"], dtype=torch.float64)
        scores = s["scores"].double().cpu().numpy()
        for b, n in enumerate(lens):
            m = min(c["keep"], n)
            for h in range(c["Hkv"]):
                rank = sorted(range(n), key=lambda j: (
                    not (j < c["sinks"] or j >= n - c["recent"]), -scores[b, h, j], j))
                got = sorted(rank[:m])
                idx[b, h, :m] = torch.tensor(got, dtype=torch.int32)
                kept[b, h, :m] = torch.from_numpy(scores[b, h, got])
                r = torch.arange(m, device="cuda")
                page = s["to_table"][b].long()[torch.div(r, c["page"], rounding_mode="floor")]
                at = torch.tensor(got, device="cuda")
                k[page, h, r % c["page"]] = _one(s, s["k"], b, h, n)[at]
                v[page, h, r % c["page"]] = _one(s, s["v"], b, h, n)[at]
        return idx, kept, _ints([min(c["keep"], n) for n in lens]), k, v
    total = sum(news)
    out = torch.zeros(total, c["H"], d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(total, c["H"], dtype=torch.float64, device="cuda")
    k_all, v_all, sums = s["k"], s["v"], None
    if c["op"] == "decode":
        k_all, v_all = k_all.clone(), v_all.clone()
        for b, n in enumerate(lens):
            page = int(s["table"][b, (n - 1) // c["page"]])
            k_all[page, :, (n - 1) % c["page"]] = s["k_new"][b]
            v_all[page, :, (n - 1) % c["page"]] = s["v_new"][b]
        if c["scores"]:
            sums = torch.zeros_like(s["scores"], dtype=torch.float64)
    at = 0
    for b, (n, t) in enumerate(zip(lens, news)):
        for h in range(c["Hkv"]):
            k, v = _one(s, k_all, b, h, n), _one(s, v_all, b, h, n)
            if sums is not None:
                sums[b, h, :n - 1] = s["scores"][b, h, :n - 1].double()
            for x in range(0, t, 4096):
                m = min(4096, t - x)
                i = torch.arange(n - t + x, n - t + x + m, device="cuda")
                ok = _seen(c, i, n)
                for g in range(h * G, (h + 1) * G):
                    w = s["q"][at + x:at + x + m, g].double() @ k.T / math.sqrt(d)
                    w = w.masked_fill(~ok, -math.inf)
                    z = torch.logsumexp(w, 1)
                    w = (w - z[:, None]).exp()
                    out[at + x:at + x + m, g] = w @ v
                    lse[at + x:at + x + m, g] = z
                    if sums is not None:
                        sums[b, h, :n] += w[0]
        at += t
    if c["op"] == "attend":
        return out, lse
    return out, lse, k_all.double(), v_all.double(), sums
