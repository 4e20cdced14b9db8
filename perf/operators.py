"""Cases of the paged cache's operators: appending rows, attention of one new token, both in one launch, and
eviction by accumulated attention weight.

With ``own`` false ``run`` computes an operator from elementary torch operations in 32 bits; with ``own`` true it
makes the calls that a user of ``paper_2510_18716_b200.binding.PagedKV`` makes.  A cache is a pool of pages
[n_pages, n_kv_heads, page_size, head_dim] (the tensor may be a view of another order in memory), a table of page
numbers per sequence (or per sequence and head), and the number of tokens held per sequence (or per sequence and
head).  The scores are the attention weights that each cached token has had so far, summed over the steps and over
the query heads that share its key head.
"""
import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------ the cases
def _case(name, op, **kw):
    c = dict(name=name, op=op, dtype="bf16", q_dtype="bf16", n_seqs=1, kv_heads=8, group=1, head_dim=128, page=16, min_len=1, max_len=640,
             ragged=1, order="head", per_head=False, weights=False, tokens=0, prefix=0, budget=0, recent=0, window=0, sink_heads=0)
    c.update(kw)
    return c


def listed():
    return [
        # one chat-sized sequence decoding alone: nothing but latency
        _case("decode_one_sequence", "decode", kv_heads=8, group=4, min_len=613, max_len=613),
        # the decode step of the janus7b batch over an uncompressed paged cache, sequences at different image steps
        _case("decode_batch_mha", "decode", n_seqs=64, kv_heads=32, min_len=65, max_len=640),
        # long contexts of very different lengths, shared heads, and the weights accumulated for a later eviction
        _case("decode_long_weights", "decode", n_seqs=16, kv_heads=8, group=8, page=64, min_len=1000, max_len=32768, order="token", weights=True),
        # a padded batch (sequences of no and of one token), an odd group, pages that do not divide a tile
        _case("decode_odd_weights_fp16", "decode", dtype="fp16", q_dtype="fp16", n_seqs=47, kv_heads=4, group=7, head_dim=64, page=24,
              min_len=0, max_len=5003, weights=True),
        # one very long document in 8 bits: the work of few heads has to be split over the whole GPU
        _case("decode_one_long_e4m3", "decode", dtype="e4m3", kv_heads=4, group=16, page=32, min_len=200001, max_len=200001),
        # the decode step after an eviction: every head has a table and a length of its own
        _case("append_decode_small", "append_decode", n_seqs=8, kv_heads=16, min_len=152, max_len=153, per_head=True, weights=True),
        # the hires7b step, rows in 8 bits, quantised on the way in
        _case("append_decode_hires_e4m3", "append_decode", dtype="e4m3", n_seqs=16, kv_heads=32, min_len=2500, max_len=4224),
        # the rows of one decode step of the janus7b batch
        _case("append_step", "append", n_seqs=64, kv_heads=32, tokens=1, min_len=65, max_len=640),
        # a chunk of prompts of ragged lengths, quantised on the way in
        _case("append_prompts_e4m3", "append", dtype="e4m3", n_seqs=23, kv_heads=8, page=32, tokens=700, min_len=701, max_len=4100, order="token"),
        # one janus1b sequence refreshed: latency
        _case("evict_one_sequence", "evict", kv_heads=16, min_len=305, max_len=305, prefix=64, budget=64, recent=24, window=64, sink_heads=8),
        # the refresh of the janus7b batch with its head split
        _case("evict_batch", "evict", n_seqs=64, kv_heads=32, min_len=185, max_len=640, prefix=64, budget=96, recent=24, window=64, sink_heads=13),
        # long contexts cut down to a fixed budget
        _case("evict_long", "evict", dtype="e4m3", n_seqs=16, kv_heads=8, page=64, min_len=5000, max_len=32768, order="token", prefix=128, budget=4096,
              recent=256, sink_heads=8),
    ]


def _between(rng, lo, hi):
    """Spread over the logarithm of the range."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["decode", "decode", "append_decode", "append", "evict"])
    dtype = rng.choice(["bf16", "fp16", "e4m3"])
    c = _case("", op, dtype=dtype, q_dtype=dtype if dtype != "e4m3" else rng.choice(["bf16", "fp16"]),
              n_seqs=_between(rng, 1, 96), kv_heads=rng.choice([1, 2, 4, 5, 8, 16, 32]), group=rng.choice([1, 1, 2, 3, 4, 6, 8, 16]),
              head_dim=rng.choice([64, 128, 128]), page=rng.choice([8, 16, 16, 20, 32, 64, 128]), order=rng.choice(["head", "token"]),
              per_head=rng.random() < 0.3, ragged=rng.randrange(1 << 30))
    del c["name"]
    budget = 1_200_000   # slots of all heads: below the largest listed case
    top = max(2, min(131072, budget // (c["n_seqs"] * c["kv_heads"])))
    c["max_len"] = _between(rng, 2, top)
    c["min_len"] = rng.choice([0, 1, c["max_len"] // 2, c["max_len"]])
    if op in ("decode", "append_decode"):
        c["weights"] = rng.random() < 0.4
    if op == "append":
        c["tokens"] = rng.choice([1, _between(rng, 1, c["max_len"])])
        c["min_len"] = max(c["min_len"], c["tokens"])
    if op == "evict":
        c["prefix"] = rng.choice([0, 1, 32, 64])
        c["recent"] = rng.choice([1, 8, 24, 64])
        c["budget"] = _between(rng, 1, max(2, c["max_len"]))
        c["window"] = rng.choice([1, 16, 64])
        c["sink_heads"] = rng.randint(0, c["kv_heads"])
        c["group"] = 1
    return c


# ------------------------------------------------------------------------------------------------ sizes
def _lengths(c):
    """Tokens held, [n_seqs, kv_heads], the appended ones included."""
    r = np.random.RandomState(c["ragged"] & 0x7fffffff)
    shape = (c["n_seqs"], c["kv_heads"]) if c["per_head"] else (c["n_seqs"], 1)
    n = r.randint(c["min_len"], c["max_len"] + 1, size=shape)
    n.flat[0] = c["max_len"]
    if n.shape[0] > 2 and c["min_len"] <= 1:
        n[1, :] = c["min_len"]
        n[2, :] = 1
    return np.ascontiguousarray(np.broadcast_to(n, (c["n_seqs"], c["kv_heads"])))


def _tokens(c):
    """Tokens appended per sequence."""
    if c["tokens"] <= 1:
        return np.full(c["n_seqs"], c["tokens"], np.int64)
    r = np.random.RandomState((c["ragged"] + 1) & 0x7fffffff)
    n = r.randint(1, c["tokens"] + 1, size=c["n_seqs"])
    n[0] = c["tokens"]
    return n


def _policy(c):
    """(budget, recent) of every head: sink heads keep the best tokens and a short window, the others a window."""
    sink = np.arange(c["kv_heads"]) * 7 % c["kv_heads"] < c["sink_heads"] if c["kv_heads"] % 7 else np.arange(c["kv_heads"]) < c["sink_heads"]
    return np.where(sink, c["budget"], 0).tolist(), np.where(sink, c["recent"], max(1, c["window"])).tolist()


def _keep(c):
    b, r = _policy(c)
    return c["prefix"] + np.asarray(b) + np.asarray(r)


def work(case):
    c = case
    n, d = _lengths(c), c["head_dim"]
    row = 2 * (d * 2 if c["dtype"] != "e4m3" else d + 4)      # K and V row of one token of one head
    fresh = 2 * d * 2                                         # the same as it arrives
    slots = int(n.sum())
    if c["op"] in ("decode", "append_decode"):
        heads = c["n_seqs"] * c["kv_heads"] * c["group"]
        b = slots * row + heads * (d * 4 + 4) + (8 * slots if c["weights"] else 0)
        if c["op"] == "append_decode":
            b += int((n > 0).sum()) * fresh                   # the new rows are read as they arrive, and written once
        return {"bytes": b, "flops": 4 * d * slots * c["group"]}
    if c["op"] == "append":
        t = int(_tokens(c).sum()) * c["kv_heads"]
        return {"bytes": t * (row + fresh), "flops": 0}
    kept = int(np.minimum(n, _keep(c)[None, :]).sum())
    return {"bytes": 4 * slots + kept * (2 * row + 8), "flops": 0}


# ------------------------------------------------------------------------------------------------ inputs
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


def _pages(c, n_pages, g):
    """A pool of pages in the case's order of memory, and its row scales (8 bits only)."""
    h, p, d = 1 if c["per_head"] else c["kv_heads"], c["page"], c["head_dim"]
    shape = (n_pages, h, p, d) if c["order"] == "head" else (n_pages, p, h, d)
    x = torch.randn(shape, generator=g, device="cuda")
    s = None
    if c["dtype"] == "e4m3":
        s = torch.rand(shape[:3], generator=g, device="cuda") * 0.01 + 0.005
        x = (x * 110.0).clamp(-E4M3_MAX, E4M3_MAX)
    x = x.to(_TYPES[c["dtype"]])
    if c["order"] == "token":
        x = x.transpose(1, 2)
        s = None if s is None else s.transpose(1, 2)
    return x, s


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    h, d, group, page, n_seqs = c["kv_heads"], c["head_dim"], c["group"], c["page"], c["n_seqs"]
    n = _lengths(c)
    rows = h if c["per_head"] else 1
    need = -(-n[:, :rows] // page)                            # pages of each table row
    wide = max(1, int(need.max()))
    total = int(need.sum())
    kept_pages = 0
    if c["op"] == "evict":                                    # the kept tokens go into fresh pages of the same pool
        kept = np.minimum(n, _keep(c)[None, :])
        kept = kept if c["per_head"] else kept.max(axis=1, keepdims=True)
        kept_need = -(-kept // page)
        kept_pages = int(kept_need.sum())
    n_pages = total + kept_pages + 2
    s = {"case": c}
    # a page holds the rows of every head; with a table of its own per head, those of one head
    s["k"], s["ks"] = _pages(c, n_pages, g)
    s["v"], s["vs"] = _pages(c, n_pages, g)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)

    def table(need, first, width):
        at = np.full((need.shape[0] * need.shape[1], width), -1, np.int64)
        k = first
        for i, m in enumerate(need.reshape(-1)):
            at[i, :m] = np.arange(k, k + m)
            k += m
        at = torch.from_numpy(at).cuda()
        t = torch.where(at >= 0, order[at.clamp(min=0)], torch.full_like(order[:1], -1))
        return t.view(need.shape[0], need.shape[1], width) if c["per_head"] else t

    s["table"] = table(need, 0, wide)
    lens = torch.from_numpy(n.astype(np.int32)).cuda()
    evict = c["op"] == "evict"
    s["lengths"] = lens if c["per_head"] or evict else lens[:, 0].contiguous()
    qt = _TYPES[c["q_dtype"]]
    if c["op"] in ("decode", "append_decode"):
        s["q"] = (1.5 * torch.randn((n_seqs, h * group, d), generator=g, device="cuda")).to(qt)
    if c["op"] in ("append", "append_decode"):
        t = _tokens(c) if c["op"] == "append" else np.ones(n_seqs, np.int64)
        s["k_new"] = torch.randn((int(t.sum()), h, d), generator=g, device="cuda").to(qt)
        s["v_new"] = torch.randn((int(t.sum()), h, d), generator=g, device="cuda").to(qt)
        s["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(t)]).astype(np.int32)).cuda() if c["tokens"] > 1 else None
    s["scores"] = None
    if c["weights"] or evict:
        # weights so far: a few tokens have most of them, the newest have none yet
        x = torch.exp(2.0 * torch.randn((n_seqs, h, max(1, c["max_len"])), generator=g, device="cuda"))
        s["scores"] = torch.where(torch.rand(x.shape, generator=g, device="cuda") < 0.02, torch.zeros_like(x), x)
    if evict:
        most = min(int(_keep(c).max()), wide * page)          # columns that any of the heads may need
        s["dst_table"] = table(kept_need, total, -(-most // page))
        s["dst_lengths"] = torch.zeros_like(lens)
        s["dst_scores"] = torch.zeros((n_seqs, h, most), device="cuda")
    if own:
        from paper_2510_18716_b200 import binding
        s["cache"] = binding.PagedKV(s["k"], s["v"], s["table"], s["lengths"], k_scales=s["ks"], v_scales=s["vs"], scores=s["scores"])
        if evict:
            s["dst"] = binding.PagedKV(s["k"], s["v"], s["dst_table"], s["dst_lengths"], k_scales=s["ks"], v_scales=s["vs"],
                                       scores=s["dst_scores"])
            s["policy"] = _policy(c)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _table3(s, name="table"):
    t, h = s[name], s["case"]["kv_heads"]
    return t if t.dim() == 3 else t[:, None, :].expand(-1, h, -1)


def _lens2(s):
    n, h = s["lengths"], s["case"]["kv_heads"]
    return (n if n.dim() == 2 else n[:, None].expand(-1, h)).long()


def _where(s, slot, name="table"):
    """Page and row in it of slots [n_seqs, kv_heads, n]."""
    page = s["case"]["page"]
    t = _table3(s, name).long()
    return torch.gather(t, 2, (slot // page).clamp(0, t.shape[2] - 1)).clamp(min=0), slot % page


def _head(s, like):
    """Which head of its page each of the slots `like` [n, kv_heads, ..] is in."""
    h = torch.arange(s["k"].shape[1], device="cuda")
    return h.view(1, -1, *[1] * (like.dim() - 2)).expand_as(like)


def _values(pages, scales, at):
    x = pages.view(torch.uint8)[at].view(pages.dtype).float() if pages.dtype == torch.float8_e4m3fn else pages[at].float()
    return x if scales is None else x * scales[at][..., None]


def _plain_attend(s):
    c = s["case"]
    q = s["q"].float().view(c["n_seqs"], c["kv_heads"], c["group"], c["head_dim"])
    n = _lens2(s)
    slot = torch.arange(max(1, c["max_len"]), device="cuda").expand(c["n_seqs"], c["kv_heads"], -1)
    page, row = _where(s, slot)
    head = _head(s, slot)
    held = slot < n[:, :, None]
    k = _values(s["k"], s["ks"], (page, head, row))
    x = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(c["head_dim"]))
    del k
    x = torch.where(held[:, :, None, :], x, torch.full_like(x[:1, :1, :1, :1], -math.inf))
    m = x.amax(dim=3, keepdim=True)
    p = torch.exp(x - torch.where(torch.isfinite(m), m, torch.zeros_like(m)))
    total = p.sum(dim=3, keepdim=True)
    w = p / torch.where(total > 0, total, torch.ones_like(total))
    v = _values(s["v"], s["vs"], (page, head, row))
    v = torch.where(held[..., None], v, torch.zeros_like(v[:1, :1, :1, :1]))
    out = torch.matmul(w, v).view(c["n_seqs"], c["kv_heads"] * c["group"], c["head_dim"]).to(s["q"].dtype)
    lse = (m + torch.log(total)).view(c["n_seqs"], -1)
    got = {"out": out, "lse": lse}
    if c["weights"]:
        s["scores"] += w.sum(dim=2)
        got["scores"] = s["scores"]
    return got


def _quantize(x):
    top = x.abs().amax(dim=-1)
    scale = top / torch.full_like(top, E4M3_MAX)              # a true division: by a plain number, torch multiplies by its inverse
    by = torch.where(scale > 0, scale, torch.ones_like(scale))
    return (x / by[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale


def _store(pages, scales, at, x):
    if scales is not None:
        x, s = _quantize(x.float())
        scales[at] = s
        pages.view(torch.uint8)[at] = x.view(torch.uint8)
    else:
        pages[at] = x.to(pages.dtype)


def _plain_append(s):
    c = s["case"]
    n = _lens2(s)
    t = s["k_new"].shape[0]
    if s["cu"] is None:
        seq, ago = torch.arange(t, device="cuda"), torch.ones(t, dtype=torch.long, device="cuda")
    else:
        i = torch.arange(t, device="cuda")
        seq = torch.searchsorted(s["cu"].long(), i, right=True) - 1
        ago = s["cu"].long()[seq + 1] - i                     # 1 for a sequence's newest token
    slot = n[seq] - ago[:, None]                              # [tokens, kv_heads]
    page = torch.gather(_table3(s).long()[seq], 2, (slot.clamp(min=0) // c["page"])[..., None])[..., 0]
    head = _head(s, slot)
    ok = slot >= 0
    at = (page[ok], head[ok], (slot % c["page"])[ok])
    _store(s["k"], s["ks"], at, s["k_new"][ok])
    _store(s["v"], s["vs"], at, s["v_new"][ok])
    if s["scores"] is not None:                               # a new token has had no weight yet
        s["scores"][seq[:, None].expand_as(slot)[ok], torch.arange(c["kv_heads"], device="cuda").expand_as(slot)[ok], slot[ok]] = 0.0
    return _cache(s)


def _cache(s):
    return {x: s[x] for x in ("k", "v", "ks", "vs") if s[x] is not None}


def _plain_evict(s):
    c = s["case"]
    n = _lens2(s)[..., None]
    budget, recent = (torch.tensor(x, device="cuda")[None, :, None] for x in _policy(c))
    x = s["scores"]
    slot = torch.arange(x.shape[2], device="cuda").expand_as(x)
    candidate = (slot >= c["prefix"]) & (slot < n - recent)
    order = torch.sort(torch.where(candidate, x, torch.full_like(x, -math.inf)), dim=2, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(2, order, slot.contiguous())
    keep = c["prefix"] + budget + recent
    kept = (slot < n) & ((n <= keep) | ~candidate | (rank < budget))
    new = kept.sum(dim=2)
    to = torch.arange(s["dst_scores"].shape[2], device="cuda").expand(c["n_seqs"], c["kv_heads"], -1)
    live = to < new[..., None]
    first = torch.sort((~kept).to(torch.uint8), dim=2, stable=True).indices
    src = torch.gather(first, 2, to.clamp(max=first.shape[2] - 1))
    head = _head(s, to)
    a, b = _where(s, src), _where(s, to, "dst_table")
    at, put = (a[0][live], head[live], a[1][live]), (b[0][live], head[live], b[1][live])
    for name in ("k", "v", "ks", "vs"):
        if s[name] is not None:
            raw = s[name].view(torch.uint8) if s[name].dtype == torch.float8_e4m3fn else s[name]
            raw[put] = raw[at]
    s["dst_lengths"].copy_(new)
    s["dst_scores"][live] = torch.gather(x, 2, src)[live]
    return {"kept": torch.where(live, src, torch.full_like(src, -1)).to(torch.int32), "lengths": s["dst_lengths"], "scores": s["dst_scores"], **_cache(s)}


# ------------------------------------------------------------------------------------------------ one pass
def _own(s):
    c, cache = s["case"], s["cache"]
    if c["op"] == "decode":
        out, lse = cache.decode_attn(s["q"], return_lse=True, accumulate=c["weights"])
        return {"out": out, "lse": lse, **({"scores": s["scores"]} if c["weights"] else {})}
    if c["op"] == "append_decode":
        out, lse = cache.append_decode(s["k_new"], s["v_new"], s["q"], return_lse=True, accumulate=c["weights"])
        return {"out": out, "lse": lse, **({"scores": s["scores"]} if c["weights"] else {}), **_cache(s)}
    if c["op"] == "append":
        cache.append(s["k_new"], s["v_new"], s["cu"])
        return _cache(s)
    kept = cache.evict(c["prefix"], s["policy"][0], s["policy"][1], into=s["dst"])
    return {"kept": kept, "lengths": s["dst_lengths"], "scores": s["dst_scores"], **_cache(s)}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "decode":
        return _plain_attend(state)
    if op == "append_decode":
        _plain_append(state)
        return {**_plain_attend(state), **_cache(state)}
    if op == "append":
        return _plain_append(state)
    return _plain_evict(state)


# ------------------------------------------------------------------------------------------------ 64 bits
def _row64(pages, scales, table, head, page, n):
    """The first n rows of one head of one sequence, in 64 bits."""
    head %= pages.shape[1]
    x = pages[table[: -(-n // page)].long(), head].double()
    if scales is not None:
        x = x * scales[table[: -(-n // page)].long(), head].double()[..., None]
    return x.reshape(-1, pages.shape[3])[:n]


def exact(case, seed):
    c = case
    if c["op"] == "evict" or (c["op"] == "append" and c["dtype"] != "e4m3"):
        return None                                           # rows are moved: nothing is computed
    s = prepare(case, seed)
    none = {x: None for x in _cache(s)}
    n, page = _lengths(c), c["page"]
    if c["op"] == "append":
        t = _tokens(c)
        first = np.concatenate([[0], np.cumsum(t)])
        ks, vs = s["ks"].double(), s["vs"].double()
        for i in range(c["n_seqs"]):
            for h in range(c["kv_heads"]):
                slot = torch.arange(int(n[i, h] - t[i]), int(n[i, h]), device="cuda")
                pages = (s["table"][i, h] if c["per_head"] else s["table"][i])[slot // page].long()
                for new, to in ((s["k_new"], ks), (s["v_new"], vs)):
                    to[pages, h % to.shape[1], slot % page] = new[first[i]:first[i + 1], h].double().abs().amax(dim=1) / E4M3_MAX
        return {**none, "ks": ks, "vs": vs}
    group, d = c["group"], c["head_dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    scores = s["scores"].double() if c["weights"] else None
    for i in range(c["n_seqs"]):
        for h in range(c["kv_heads"]):
            m = int(n[i, h])
            if m == 0:
                continue
            table = s["table"][i, h] if c["per_head"] else s["table"][i]
            k, v = (_row64(s[x], s[x + "s"], table, h, page, m) for x in ("k", "v"))
            if c["op"] == "append_decode":
                for new, to in ((s["k_new"], k), (s["v_new"], v)):
                    x = new[i, h]
                    if c["dtype"] == "e4m3":                  # the codes are decided in 32 bits
                        code, by = _quantize(x.float())
                        to[m - 1] = code.double() * by.double()
                    else:
                        to[m - 1] = x.double()
            q = s["q"][i, h * group:(h + 1) * group].double()
            x = q @ k.T / math.sqrt(d)
            top = x.amax(dim=1, keepdim=True)
            e = (x - top).exp()
            z = e.sum(dim=1, keepdim=True)
            out[i, h * group:(h + 1) * group] = (e / z) @ v
            lse[i, h * group:(h + 1) * group] = (top + z.log())[:, 0]
            if scores is not None:
                if c["op"] == "append_decode":
                    scores[i, h, m - 1] = 0.0                 # the new token's
                scores[i, h, :m] += (e / z).sum(dim=0)
    got = {"out": out, "lse": lse, **({"scores": scores} if c["weights"] else {})}
    if c["op"] == "append_decode":
        got.update(none)
        if c["dtype"] == "e4m3":
            for x, new in (("ks", s["k_new"]), ("vs", s["v_new"])):
                to = s[x].double()
                for i in range(c["n_seqs"]):
                    for h in range(c["kv_heads"]):
                        if n[i, h]:
                            table = s["table"][i, h] if c["per_head"] else s["table"][i]
                            to[int(table[(n[i, h] - 1) // page]), h % to.shape[1], int((n[i, h] - 1) % page)] = new[i, h].double().abs().amax() / E4M3_MAX
                got[x] = to
    return got
