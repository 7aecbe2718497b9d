"""What a serving loop over the paged key/value cache does beside attention, as measurable cases: the next token of every row from its
logits, and the bound on what a sequence keeps in the cache.

`kind` names the entry point:
  sample  sample: one token a row from logits by temperature, top-k, top-p and min-p, each row with its own, from given uniform numbers
  weigh   paged_weigh: how much attention a chunk's rows give to each cached token, summed over rows and a kv head's queries
  evict   paged_evict: of a sequence's tokens the first, the last and those of most weight move to the front of its pages, in every
          layer and kv head by its own weights

Sampling, exactly: the tokens of a row in order of their logits (equal ones by id) with weights w = exp((logit - largest) / temperature).  Kept are
the first top_k of them; of those, with W their weights' sum, each one before which less than top_p W lies; of those, what weighs
min_p of the first at least; the first always.  The token is the lowest id at which the kept weights' sum over ids up to it is above u times the
sum of all kept.  Temperature 0: the first of the order.

A page holds planes [kv head][page_size * head_dim] in blocks of 32 slots, in the order of esp_kv: K [head_dim/16][2][32 slots][8], V
[head_dim/32][2][2][32 features][2][4].
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases -----------------------------------------------------------------------------------------

def _sample(name, rows, vocab, settings, dtype="f32", banned=0.0):
    """settings: which of the limits the rows have; "mixed": some rows each.  banned: share of tokens that a grammar forbids (logit -inf)."""
    c = dict(kind="sample", rows=rows, vocab=vocab, settings=settings, dtype=dtype, banned=banned)
    return dict(c, name=name) if name else c


def _weigh(name, hq, hkv, hd, page, batch, len_lo, len_hi, rows_lo, rows_hi, last, dtype="bf16", mix=0):
    """len, rows: committed tokens and new rows of a sequence, from lo to hi over the batch; last: so many of the rows count (0: all)."""
    c = dict(kind="weigh", dtype=dtype, hq=hq, hkv=hkv, hd=hd, page=page, batch=batch, len_lo=len_lo, len_hi=len_hi, rows_lo=rows_lo,
             rows_hi=rows_hi, last=last, mix=mix)
    return dict(c, name=name) if name else c


def _evict(name, hkv, hd, page, layers, batch, len_lo, len_hi, keep, first, recent, dtype="bf16", mix=0):
    c = dict(kind="evict", dtype=dtype, hkv=hkv, hd=hd, page=page, layers=layers, batch=batch, len_lo=len_lo, len_hi=len_hi, keep=keep, first=first,
             recent=recent, mix=mix)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the small fp32 model, one user: latency
        _sample("sample_row1_vocab4096", 1, 4096, "top_k"),
        # one user of a large vocabulary, the usual top-p
        _sample("sample_row1_vocab128256", 1, 128256, "top_p"),
        # a serving batch, every request with limits of its own
        _sample("sample_rows64_vocab128256", 64, 128256, "mixed"),
        # all rows of a tree of 320, drawn without limits, logits in bf16
        _sample("sample_rows320_vocab151936_bf16", 320, 151936, "none", "bf16"),
        # many requests under a grammar that forbids most tokens
        _sample("sample_rows256_vocab128256_banned", 256, 128256, "mixed", "f32", 0.6),
        # the small fp32 model's block of 60 rows
        _weigh("weigh_f32_rows60_kv128", 4, 4, 64, 32, 1, 128, 128, 60, 60, 0, "f32"),
        # one user, ordinary decoding
        _weigh("weigh_decode_kv2048", 32, 8, 128, 64, 1, 2047, 2047, 1, 1, 0),
        # serving: one row of each of 32 sequences whose lengths differ
        _weigh("weigh_decode_b32_ragged", 32, 8, 128, 64, 32, 1000, 16384, 1, 1, 0, mix=1),
        # the last 64 rows of each prompt say what of it will matter
        _weigh("weigh_last64_b4", 32, 8, 128, 64, 4, 0, 512, 2000, 8192, 64, mix=2),
        # every row of a prompt
        _weigh("weigh_prompt_4096", 32, 8, 128, 128, 1, 0, 0, 4096, 4096, 0),
        # one user's prompt cut to half, 32 layers
        _evict("evict_b1_kv4096", 8, 128, 64, 32, 1, 4096, 4096, 2048, 4, 256),
        # a batch in which some are over their bound and some are not, 8 layers
        _evict("evict_b16_ragged", 8, 128, 64, 8, 16, 200, 3000, 1024, 4, 128, mix=3),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = [(32, 8), (32, 8), (32, 32), (28, 4), (16, 2), (8, 1), (6, 2), (40, 8), (12, 12)]


def _draw(rng):
    kind = rng.choice(["sample"] * 4 + ["weigh"] * 5 + ["evict"] * 3)
    if kind == "sample":
        vocab = rng.choice([4096, 128256, 151936, _log_int(rng, 1000, 200000), _log_int(rng, 1000, 200000)])
        return _sample(None, _log_int(rng, 1, 400), vocab, rng.choice(["none", "greedy", "top_k", "top_p", "min_p", "mixed", "mixed"]),
                       rng.choice(["f32", "f32", "bf16"]), rng.choice([0.0, 0.0, 0.0, 0.5, 0.9]))
    hq, hkv = rng.choice(_HEADS)
    hd = rng.choice([128, 128, 64])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([32, 64, 64, 96, 128, 256])
    batch = rng.choice([1, 1, 2, 3, 7, 16, 33, 64])
    mix = rng.randint(10, 10 ** 6)
    if kind == "evict":
        len_hi = _log_int(rng, 64, 12000)
        keep = _log_int(rng, 16, max(16, len_hi - 1))
        first = rng.choice([0, 1, 4, min(16, keep)])
        recent = rng.randint(0, keep - first)
        return _evict(None, hkv, hd, page, rng.randint(1, 36), batch, rng.choice([1, len_hi // 2, len_hi]), len_hi, keep, first, recent, dtype, mix)
    len_hi = _log_int(rng, 1, 32768 if batch <= 7 else 8192)
    len_lo = rng.choice([0, len_hi // 8, len_hi])
    rows = 1 if rng.random() < 0.4 else _log_int(rng, 2, 4096)
    last = rng.choice([0, 0, 16, 64, _log_int(rng, 1, 300)])
    return _weigh(None, hq, hkv, hd, page, batch, len_lo, len_hi, rng.choice([1, rows]), rows, last, dtype, mix)


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        if c["kind"] == "sample":
            fits = c["rows"] * c["vocab"] <= 320 * 151936
        elif c["kind"] == "weigh":         # what the plain form pads to
            fits = w["flops"] <= (7e10 if c["dtype"] == "bf16" else 2e10) and c["batch"] * c["hq"] * _counted(c, c["rows_hi"]) * (
                c["len_hi"] + c["rows_hi"]) <= 1.2e9 and w["bytes"] <= 1.2e9
        else:
            fits = c["layers"] * c["hkv"] * c["hd"] * (2 if c["dtype"] == "bf16" else 4) * 2 * sum(_lens(c)) <= 1.0e9
        if fits:
            return c


def _spread(lo, hi, n, mix, stream):
    """n whole numbers from lo to hi that depend on nothing but these; one of them is hi."""
    r = random.Random(1000003 * mix + stream)
    v = [r.randint(lo, hi) for _ in range(n)]
    v[r.randrange(n)] = hi
    return v


def _lens(c):
    return _spread(c["len_lo"], c["len_hi"], c["batch"], c["mix"], 1)


def _rows(c):
    return _spread(c["rows_lo"], c["rows_hi"], c["batch"], c["mix"], 2)


def _counted(c, rows):
    return min(rows, c["last"]) if c["last"] else rows


# ---- inputs ----------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 7 + 3)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _limits(c, g):
    """temperature, top_k, top_p, min_p of every row, or None where no row has it."""
    n, s = c["rows"], c["settings"]
    t = 0.5 + torch.rand(n, generator=g, device="cuda")
    k = torch.randint(1, 100, (n,), generator=g, device="cuda", dtype=torch.int32)
    p = 0.5 + 0.499 * torch.rand(n, generator=g, device="cuda")
    m = 0.3 * torch.rand(n, generator=g, device="cuda") ** 2
    if s == "mixed":
        has = torch.arange(n, device="cuda") % 8               # a greedy row, rows with every combination of limits, one with none
        t = torch.where(has == 0, 0.0, t)
        k = torch.where((has & 1) == 1, k, 0).to(torch.int32)
        p = torch.where((has & 2) == 2, p, 1.0)
        m = torch.where((has & 4) == 4, m, 0.0)
        return t, k, p, m
    if s == "greedy":
        t = torch.zeros_like(t)
    return t, k if s == "top_k" else None, p if s == "top_p" else None, m if s == "min_p" else None


def _pages(c, need, spare, g):
    """(pages in the pool, one page table for each list of needs): pages in random order, some more than are needed."""
    n = sum(sum(k) for k in need) + spare
    order = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    tables, at = [], 0
    for pages in need:
        table = torch.zeros((len(pages), max(max(pages), 1)), dtype=torch.int32, device="cuda")
        for b, k in enumerate(pages):
            table[b, :k] = order[at:at + k]
            at += k
        tables.append(table)
    return n, tables


def _pool(c, layers, pages, g):
    """K of some channels larger than of others, as models have it; V of size one."""
    hd, dt = c["hd"], DTYPES[c["dtype"]]
    k = torch.randn((layers, pages, c["hkv"], c["page"] // 32, hd // 16, 2, 32, 8), generator=g, device="cuda", dtype=dt)
    k *= torch.exp(0.4 * torch.randn((c["hkv"], 1, hd // 16, 2, 1, 8), generator=g, device="cuda")).to(dt)
    v = torch.randn((layers, pages, c["hkv"], c["page"] * hd), generator=g, device="cuda", dtype=dt)
    shape = (layers, pages, c["hkv"], c["page"], hd)
    return k.reshape(shape), v.reshape(shape)


def prepare(case, seed):
    c, g = case, _gen(seed)
    if c["kind"] == "sample":
        n, vocab = c["rows"], c["vocab"]
        x = 2.2 * torch.randn((n, vocab), generator=g, device="cuda")
        # some tokens of each row are likely ones, in sure rows by more than in others
        at = (torch.randint(0, vocab, (n, 1), generator=g, device="cuda") + torch.arange(40, device="cuda") * (vocab // 41)) % vocab
        sure = 14 * torch.rand((n, 1), generator=g, device="cuda")
        x.scatter_(1, at, x.gather(1, at) + sure * torch.rand((n, 40), generator=g, device="cuda"))
        if c["banned"]:
            x.masked_fill_(torch.rand((n, vocab), generator=g, device="cuda") < c["banned"], -math.inf)
        t, k, p, m = _limits(c, g)
        return dict(case=c, logits=x.to(DTYPES[c["dtype"]]), temperature=t, top_k=k, top_p=p, min_p=m, u=torch.rand(n, generator=g, device="cuda"),
                    ids=torch.empty(n, dtype=torch.int32, device="cuda"), probs=torch.empty(n, device="cuda"))
    lens, page = _lens(c), c["page"]
    if c["kind"] == "evict":
        pages, tables = _pages(c, [[(l + page - 1) // page for l in lens], [(min(l, c["keep"]) + page - 1) // page for l in lens]], 2, g)
        kp, vp = _pool(c, c["layers"], pages, g)
        room = tables[0].shape[1] * page
        # attention goes to few tokens; many have got none of it
        mass = torch.randn((c["layers"], c["batch"], c["hkv"], room), generator=g, device="cuda").clamp_min(0).pow(3)
        shape = (c["layers"], c["batch"], c["hkv"], c["keep"])
        # a table's entries past a sequence's pages are not used, and the new table has room for all that is kept
        wide = torch.zeros((c["batch"], (c["keep"] + page - 1) // page), dtype=torch.int32, device="cuda")
        wide[:, :tables[1].shape[1]] = tables[1]
        return dict(case=c, k_pool=kp, v_pool=vp, table=tables[0], table_out=wide, lens=_i32(lens), mass=mass,
                    mass_out=torch.zeros_like(mass), len_out=_i32([0] * c["batch"]), kept=torch.zeros(shape, dtype=torch.int32, device="cuda"))
    rows = _rows(c)
    pages, tables = _pages(c, [[(l + r + page - 1) // page for l, r in zip(lens, rows)]], 2, g)
    kp, vp = _pool(c, 1, pages, g)
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    q = (1.5 * torch.randn((starts[-1], c["hq"], c["hd"]), generator=g, device="cuda")).to(DTYPES[c["dtype"]])
    before = torch.randn((1, c["batch"], c["hkv"], tables[0].shape[1] * page), generator=g, device="cuda").pow(2)
    return dict(case=c, k_pool=kp, v_pool=vp, table=tables[0], lens=_i32(lens), row0=_i32(starts), total=starts[-1], q=q, before=before,
                mass=torch.zeros_like(before))


# ---- the framework's entry points --------------------------------------------------------------------------

def _run_own(s):
    from paper_2603_17942_amd import binding as B
    c = s["case"]
    if c["kind"] == "sample":
        return B.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], ids=s["ids"],
                        probs=s["probs"])
    if "handles" not in s:       # what a program keeps around its own tensors from step to step
        h = dict(kv=B.PagedKv(s["k_pool"], s["v_pool"], s["table"], s["lens"], len_bound=c["len_hi"]))
        if c["kind"] == "weigh":
            h["rows"] = B.ChunkRows(s["row0"], s["total"], c["rows_hi"])
            h["scratch"] = torch.empty(B.paged_weigh_scratch_bytes(h["kv"], h["rows"], c["hq"], last_rows=c["last"]), dtype=torch.uint8, device="cuda")
        s["handles"] = h
    h = s["handles"]
    if c["kind"] == "weigh":
        return B.paged_weigh(h["kv"], 0, h["rows"], s["q"], s["mass"], before=s["before"], last_rows=c["last"], scratch=h["scratch"])
    B.paged_evict(h["kv"], s["mass"], c["keep"], first=c["first"], recent=c["recent"], table_out=s["table_out"], mass_out=s["mass_out"],
                  len_out=s["len_out"], kept=s["kept"])
    return s["kept"], s["k_pool"], s["v_pool"], s["mass_out"], s["len_out"]


# ---- the plain forms -----------------------------------------------------------------------------------------

def _plain_sample(s):
    x = s["logits"].double()
    n, vocab = x.shape
    t = s["temperature"].double()[:, None]
    top = x.amax(1, keepdim=True)
    w = torch.where(t > 0, ((x - top) / t.clamp_min(1e-300)).exp(), (x == top).double())
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    sorted_w = w.gather(1, order)
    place = torch.arange(vocab, device=x.device)
    keep = torch.ones_like(x, dtype=torch.bool)
    if s["top_k"] is not None:
        keep &= (place < s["top_k"][:, None]) | (s["top_k"][:, None] <= 0)
    if s["top_p"] is not None:
        total = torch.where(keep, sorted_w, 0.0).cumsum(1)
        p = s["top_p"].double()[:, None]
        keep &= (total - sorted_w < p * total[:, -1:]) | (p >= 1)
    if s["min_p"] is not None:
        keep &= sorted_w >= s["min_p"].double()[:, None]
    keep &= (t > 0) | (place == 0)
    keep[:, 0] = True
    kept_w = torch.zeros_like(x).scatter_(1, order, torch.where(keep, sorted_w, 0.0))
    total = kept_w.cumsum(1)
    pick = torch.searchsorted(total, s["u"].double()[:, None] * total[:, -1:], right=True)
    s["ids"].copy_(pick[:, 0])
    s["probs"].copy_((kept_w.gather(1, pick) / total[:, -1:])[:, 0])
    return s["ids"], s["probs"]


def _plain_weigh(s):
    c = s["case"]
    B, hq, hkv, hd, page = c["batch"], c["hq"], c["hkv"], c["hd"], c["page"]
    G, n = hq // hkv, s["table"].shape[1]
    T, R = n * page, _counted(c, c["rows_hi"])
    k = s["k_pool"][0][s["table"].long()].view(B, n, hkv, page // 32, hd // 16, 2, 32, 8).permute(0, 2, 4, 5, 7, 1, 3, 6).reshape(B, hkv, hd, T).float()
    row0, lens = s["row0"].long(), s["lens"].long()
    rows = row0[1:] - row0[:-1]
    r = rows[:, None] - R + torch.arange(R, device="cuda")                          # the last R rows of each
    live = r >= 0
    at = torch.where(live, row0[:-1, None] + r, 0)
    slot = torch.arange(T, device="cuda")
    seen = (slot <= (lens[:, None] + r)[:, :, None]) & live[:, :, None]
    q = s["q"][at].float().view(B, R, hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(B, hkv, R * G, hd)
    x = torch.matmul(q, k).mul_(1 / math.sqrt(hd)).view(B, hkv, R, G, T)
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    x /= x.sum(-1, keepdim=True).clamp_min(1e-30)
    given = x.sum((2, 3))                                                           # [B, hkv, T]
    old = torch.where(slot < lens[:, None, None], s["before"][0], 0.0)
    there = (slot < (lens + rows)[:, None, None]).expand_as(given)
    s["mass"][0] = torch.where(there, old + given, s["mass"][0])
    return s["mass"]


def _k_places(slot, hd):
    """Where the elements of slots lie in a plane of a page, K."""
    d = torch.arange(hd, device=slot.device)
    return (slot // 32 * hd * 32 + slot % 32 * 8)[..., None] + (d // 16 * 64 + d // 8 % 2 * 32) * 8 + d % 8


def _v_places(slot, hd):
    key, d = slot % 32, torch.arange(hd, device=slot.device)
    at = slot // 32 * hd * 32 + (key // 16 * 64 + key // 4 % 2 * 32) * 8 + key // 8 % 2 * 4 + key % 4
    return at[..., None] + d // 32 * 1024 + d % 32 * 8


def _plain_evict(s):
    c = s["case"]
    lens, keep, hkv, hd, page = s["lens"].long(), c["keep"], c["hkv"], c["hd"], c["page"]
    slot = torch.arange(s["mass"].shape[3], device="cuda")
    L = lens[:, None, None]
    rank = torch.where((slot < c["first"]) | (slot >= L - c["recent"]), math.inf, s["mass"])
    rank = torch.where(slot < L, rank, -math.inf)
    order = torch.sort(rank, dim=3, descending=True, stable=True).indices[..., :keep]
    if order.shape[3] < keep:
        order = torch.cat([order, order.new_zeros(order.shape[:3] + (keep - order.shape[3],))], 3)
    order = order.sort(3).values
    place = torch.arange(keep, device="cuda")
    order = torch.where(L <= keep, torch.where(place < L, place, -1), order)
    s["kept"].copy_(order)
    n = torch.minimum(lens, torch.tensor(keep, device="cuda"))
    seq, new = (place < n[:, None]).nonzero(as_tuple=True)                          # all kept tokens: whose and to which slot
    shape, head = s["k_pool"].shape, torch.arange(hkv, device="cuda")
    to_page = s["table_out"].long()[seq, new // page]
    to = (to_page[:, None] * hkv + head)[..., None] * (page * hd)
    for layer in range(c["layers"]):
        old = order[layer][seq, :, new]                                             # [tokens, hkv]
        frm = (s["table"].long()[seq[:, None], old // page] * hkv + head)[..., None] * (page * hd)
        for pool, of in ((s["k_pool"], _k_places), (s["v_pool"], _v_places)):
            flat = pool[layer].view(-1)
            flat[to + of(new % page, hd)[:, None]] = flat[frm + of(old % page, hd)]
        s["mass_out"][layer][seq, :, new] = s["mass"][layer][seq[:, None], head, old]
    s["len_out"].copy_(n)
    return s["kept"], s["k_pool"], s["v_pool"], s["mass_out"], s["len_out"]


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    return _plain_sample(state) if kind == "sample" else _plain_weigh(state) if kind == "weigh" else _plain_evict(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    if c["kind"] == "sample":
        return {"bytes": c["rows"] * (c["vocab"] * e + 28), "flops": 3 * c["rows"] * c["vocab"]}
    lens = _lens(c)
    if c["kind"] == "evict":       # every weight once, what is kept once from its old place and once to its new one
        n = sum(min(l, c["keep"]) for l in lens)
        return {"bytes": c["layers"] * c["hkv"] * (4 * sum(lens) + n * (4 * c["hd"] * e + 8)), "flops": 0}
    rows = _rows(c)
    seen = nq = 0
    for r, l in zip(rows, lens):
        w = _counted(c, r)
        seen += w * (l + r) - w * (w - 1) // 2
        nq += w
    t = sum(r + l for r, l in zip(rows, lens))
    return {"bytes": nq * c["hq"] * c["hd"] * e + c["hkv"] * (t * (c["hd"] * e + 4) + 4 * sum(lens)), "flops": 2 * c["hd"] * c["hq"] * seen}


# ---- from the definition, in 64 bits -----------------------------------------------------------------------------

def _exact_sample(c, s):
    x = s["logits"].double().cpu().numpy()
    lim = {k: None if s[k] is None else s[k].double().cpu().numpy() for k in ("temperature", "top_k", "top_p", "min_p", "u")}
    ids, probs = [], []
    for i in range(c["rows"]):
        row, T = x[i], lim["temperature"][i]
        if T == 0:
            ids.append(int(np.flatnonzero(row == row.max())[0]))
            probs.append(1.0)
            continue
        alive = np.flatnonzero(row > -np.inf)
        order = alive[np.lexsort((alive, -row[alive]))]
        w = np.exp((row[order] - row[order[0]]) / T)
        if lim["top_k"] is not None and lim["top_k"][i] > 0:
            w = w[:int(lim["top_k"][i])]
        if lim["top_p"] is not None and lim["top_p"][i] < 1:
            before = np.concatenate([[0.0], np.cumsum(w)])
            w = w[:max(1, int(np.count_nonzero(before[:-1] < lim["top_p"][i] * before[-1])))]
        if lim["min_p"] is not None:
            w = w[:max(1, int(np.count_nonzero(w >= lim["min_p"][i])))]
        by_id = np.argsort(order[:len(w)])
        run_, goal = np.cumsum(w[by_id]), lim["u"][i] * math.fsum(w)
        at = by_id[min(int(np.count_nonzero(run_ <= goal)), len(w) - 1)]
        ids.append(int(order[at]))
        probs.append(w[at] / math.fsum(w))
    return _i32(ids), torch.tensor(probs, dtype=torch.float64, device="cuda")


def _exact_planes(c, page, slots, h, of_v):
    """For slots of pages: the elements' places in the flat pool of a layer, [slots, hd], of kv head h."""
    hd = c["hd"]
    d = torch.arange(hd, device="cuda")
    inside = slots % c["page"]
    block, key = torch.div(inside, 32, rounding_mode="floor"), inside % 32
    if of_v:
        piece = ((d >> 5) * 2 + (key >> 4)[:, None]) * 64 + ((key >> 2) & 1)[:, None] * 32 + (d & 31)
        place = piece * 8 + (4 * ((key >> 3) & 1) + (key & 3))[:, None]
    else:
        place = ((d >> 4) * 64 + ((d >> 3) & 1) * 32 + key[:, None]) * 8 + (d & 7)
    return place + (block * (32 * hd) + (page * c["hkv"] + h) * (c["page"] * hd))[:, None]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "sample":
        return _exact_sample(c, s)
    lens, page = _lens(c), c["page"]
    if c["kind"] == "evict":
        mass, kept = s["mass"].cpu().numpy(), np.full(tuple(s["kept"].shape), -1, dtype=np.int64)
        pools = [s["k_pool"].double(), s["v_pool"].double()]
        mass_out = s["mass_out"].double()
        for b, n in enumerate(lens):
            m = min(n, c["keep"])
            new = torch.arange(m, device="cuda")
            to_page = s["table_out"][b].long()[torch.div(new, page, rounding_mode="floor")]
            for layer in range(c["layers"]):
                for h in range(c["hkv"]):
                    old = np.arange(m)
                    if n > m:
                        mid = np.arange(c["first"], n - c["recent"])
                        chosen = mid[np.lexsort((mid, -mass[layer, b, h, mid]))][:m - c["first"] - c["recent"]]
                        old = np.sort(np.concatenate([np.arange(c["first"]), chosen, np.arange(n - c["recent"], n)]))
                    kept[layer, b, h, :m] = old
                    frm = torch.from_numpy(old).cuda()
                    from_page = s["table"][b].long()[torch.div(frm, page, rounding_mode="floor")]
                    for out, pool, of_v in ((pools[0], s["k_pool"], False), (pools[1], s["v_pool"], True)):
                        out[layer].view(-1)[_exact_planes(c, to_page, new, h, of_v)] = pool[layer].view(-1)[
                            _exact_planes(c, from_page, frm, h, of_v)].double()
                    mass_out[layer, b, h, :m] = s["mass"][layer, b, h, frm].double()
        return torch.from_numpy(kept).cuda().to(torch.int32), pools[0], pools[1], mass_out, _i32([min(n, c["keep"]) for n in lens])
    G, at, mass = c["hq"] // c["hkv"], 0, s["mass"].double()
    for b, (l, r) in enumerate(zip(lens, _rows(c))):
        slots, w = torch.arange(l + r, device="cuda"), _counted(c, r)
        pages = s["table"][b].long()[torch.div(slots, page, rounding_mode="floor")]
        hidden = torch.ones((w, l + r), dtype=torch.bool, device="cuda").triu(l + r - w + 1)
        for h in range(c["hkv"]):
            k = s["k_pool"].reshape(-1)[_exact_planes(c, pages, slots, h, False)].double()
            m = torch.zeros(l + r, dtype=torch.float64, device="cuda")
            m[:l] = s["before"][0, b, h, :l].double()
            for g in range(G):
                x = s["q"][at + r - w:at + r, h * G + g].double() @ k.t().contiguous() / math.sqrt(c["hd"])
                e = (x - x.masked_fill(hidden, -math.inf).max(-1, keepdim=True).values).exp().masked_fill(hidden, 0.0)
                m += (e / e.sum(-1, keepdim=True)).sum(0)
            mass[0, b, h, :l + r] = m
        at += r
    return mass
