"""The paged key/value cache as measurable cases: what rotates queries and keys, what appends to the pages, what attends to
them and what moves the accepted rows of a verified tree.

`kind` names the entry point:
  rope    rope_qk: rotary positions on query and key rows, with the norm of every head where the model has one
  append  paged_append: the same on the way into the pages of one layer, queries to a buffer of their own
  attn    paged_attn: a chunk of new rows of every sequence over its pages, causal or under a tree's ancestor bitsets
  commit  paged_commit: the rows of the accepted paths move behind the committed tokens, in all layers

Rows of q, k and v are the three parts of one projection's output, as a model hands them over, so their stride is longer than
they are.  Pages of a sequence lie anywhere in the pool.  A page holds planes [kv head][page_size * head_dim] in blocks of 32
slots, in the order of esp_kv: K [head_dim/16][2][32 slots][8], V [head_dim/32][2][2][32 features][2][4].
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases -----------------------------------------------------------------------------------------

def _attn(name, hq, hkv, hd, page, batch, len_lo, len_hi, rows_lo, rows_hi, mask="causal", dtype="bf16", mix=0):
    """len, rows: committed tokens and new rows of a sequence, from lo to hi over the batch."""
    c = dict(kind="attn", dtype=dtype, hq=hq, hkv=hkv, hd=hd, page=page, batch=batch, len_lo=len_lo, len_hi=len_hi, rows_lo=rows_lo,
             rows_hi=rows_hi, mask=mask, mix=mix)
    return dict(c, name=name) if name else c


def _append(name, hq, hkv, hd, page, batch, len_lo, len_hi, rows_lo, rows_hi, norm, rot, interleaved, factor, given, dtype="bf16", mix=0):
    """given: positions are an input (a tree's, by depth); otherwise a row's position is its place in the sequence."""
    c = dict(kind="append", dtype=dtype, hq=hq, hkv=hkv, hd=hd, page=page, batch=batch, len_lo=len_lo, len_hi=len_hi, rows_lo=rows_lo,
             rows_hi=rows_hi, norm=norm, rot=rot, interleaved=interleaved, factor=factor, given=given, mix=mix)
    return dict(c, name=name) if name else c


def _rope(name, hq, hkv, hd, rows, norm, rot, interleaved, factor, far, dtype="bf16"):
    """far: positions are below it."""
    c = dict(kind="rope", dtype=dtype, hq=hq, hkv=hkv, hd=hd, rows=rows, norm=norm, rot=rot, interleaved=interleaved, factor=factor, far=far)
    return dict(c, name=name) if name else c


def _commit(name, hkv, hd, page, layers, batch, len_lo, len_hi, path, dtype="bf16", mix=0):
    """path: tokens emitted by a sequence, 1 to path over the batch."""
    c = dict(kind="commit", dtype=dtype, hkv=hkv, hd=hd, page=page, layers=layers, batch=batch, len_lo=len_lo, len_hi=len_hi, path=path, mix=mix)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the small fp32 model's block of 60 rows: launches and latency
        _attn("attn_f32_rows60_kv128", 4, 4, 64, 32, 1, 128, 128, 60, 60, "tree", "f32"),
        # one user, ordinary decoding: one row over a short cache
        _attn("attn_decode_kv2048", 32, 8, 128, 64, 1, 2047, 2047, 1, 1),
        # serving: one row of each of 32 sequences whose lengths differ
        _attn("attn_decode_b32_ragged", 32, 8, 128, 64, 32, 1000, 16384, 1, 1, mix=1),
        # a tree of 64 nodes with four mask rows each, verified over a cache of 2048 tokens
        _attn("attn_tree_rows320_kv2048", 32, 8, 128, 64, 1, 2048, 2048, 320, 320, "tree"),
        # prompts that come in by chunks beside sequences that decode: chunks of 1 to 512 rows
        _attn("attn_chunk_b8_ragged", 32, 8, 128, 64, 8, 0, 8192, 1, 512, mix=2),
        # a long prompt at once
        _attn("attn_prefill_8192", 32, 8, 128, 128, 1, 0, 0, 8192, 8192),
        # a decode step's rows of 64 sequences, model with norms on q and k
        _append("append_decode_b64", 32, 8, 128, 64, 64, 100, 4000, 1, 1, True, 128, False, 1.0, False),
        # chunks of four prompts, frequencies scaled for a long context
        _append("append_chunk_b4", 32, 8, 128, 64, 4, 0, 1500, 700, 2048, False, 128, False, 8.0, False, mix=3),
        # one row at a far position, interleaved pairs on half of the head
        _rope("rope_row1_interleaved", 32, 8, 128, 1, False, 64, True, 1.0, 131072),
        # a long prompt's rows, norms and scaled frequencies
        _rope("rope_rows8192_norm", 32, 8, 128, 8192, True, 128, False, 4.0, 131072),
        # one user's accepted path after a step, 32 layers
        _commit("commit_b1", 8, 128, 64, 32, 1, 2000, 2000, 3),
        # a batch's paths
        _commit("commit_b16", 8, 128, 64, 32, 16, 1, 250, 5, mix=4),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = [(32, 8), (32, 8), (32, 32), (28, 4), (16, 2), (8, 1), (6, 2), (40, 8), (12, 12)]


def _draw(rng):
    kind = rng.choice(["attn"] * 6 + ["append"] * 2 + ["rope", "commit"])
    hq, hkv = rng.choice(_HEADS)
    hd = rng.choice([128, 128, 64])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([32, 64, 64, 96, 128, 256])
    batch = rng.choice([1, 1, 2, 3, 7, 16, 33, 64])
    mix = rng.randint(10, 10 ** 6)
    norm, interleaved, factor = rng.random() < 0.4, rng.random() < 0.4, rng.choice([1.0, 1.0, 2.0, 8.0, 32.0])
    rot = rng.choice([hd, hd, hd // 2, 32, 16])
    if kind == "rope":
        return _rope(None, hq, hkv, hd, _log_int(rng, 1, 8192), norm, rot, interleaved, factor, _log_int(rng, 64, 1 << 20), dtype)
    if kind == "commit":
        return _commit(None, hkv, hd, page, rng.randint(1, 36), min(batch, 16), rng.randint(0, 20), _log_int(rng, 21, 300), rng.randint(1, 9), dtype, mix)
    len_hi = _log_int(rng, 1, 32768 if batch <= 7 else 8192)
    len_lo = rng.choice([0, len_hi // 8, len_hi])
    if kind == "append":
        rows = rng.choice([1, 1, _log_int(rng, 2, 300), _log_int(rng, 16, 2048)])
        return _append(None, hq, hkv, hd, page, batch, min(len_lo, 4000), min(len_hi, 4000), rng.choice([1, rows]), rows, norm, rot, interleaved,
                       factor, rng.random() < 0.4, dtype, mix)
    mask = rng.choice(["causal", "causal", "tree"])
    rows = 1 if rng.random() < 0.35 else _log_int(rng, 2, 700 if mask == "tree" else 4096)
    return _attn(None, hq, hkv, hd, page, batch, len_lo, len_hi, rng.choice([1, rows]), rows, mask, dtype, mix)


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        scores = 0
        if c["kind"] == "attn":        # what the plain form pads to
            scores = c["batch"] * c["hq"] * c["rows_hi"] * (c["len_hi"] + c["rows_hi"])
        if w["bytes"] <= 1.2e9 and w["flops"] <= (6e11 if c["dtype"] == "bf16" else 6e10) and scores <= 2.2e9:
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


def _parents(n, mix, b):
    """A tree of n rows, parents before children, about log2 n deep."""
    r = random.Random(7919 * mix + 31 * b + n)
    return [-1] + [r.randrange(max(0, i // 4 - 3), i // 2 + 1) if i > 1 else 0 for i in range(1, n)]


def _depths(parents):
    d = [0] * len(parents)
    for i, p in enumerate(parents[1:], 1):
        d[i] = d[p] + 1
    return d


def _ancestors(parents):
    """Rows that each row sees: itself and what is above it, as bits."""
    a = [1] * len(parents)
    for i, p in enumerate(parents[1:], 1):
        a[i] = a[p] | (1 << i)
    return a


def _path(c, b):
    """A sequence's accepted rows: the root and one row of each further level, level i + 1 beginning behind the path's last place."""
    n = _spread(1, c["path"], c["batch"], c["mix"], 3)[b]
    r = random.Random(104729 * c["mix"] + b)
    rows, at = [0], 8
    for _ in range(1, n):
        at += r.randint(1, 4)
        rows.append(at)
    return rows


_TREE_ROWS = 48                 # rows of a tree block that commit's paths lie in


# ---- inputs ----------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 7 + 3)


def _pages(c, lens, rows, g):
    """(pages in the pool, page table): pages in random order, two more than are needed."""
    need = [(l + r + c["page"] - 1) // c["page"] for l, r in zip(lens, rows)]
    n, most = sum(need) + 2, max(max(need), 1)
    order = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((len(lens), most), dtype=torch.int32, device="cuda")
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    return n, table


def _pool(c, layers, pages, g):
    """K of some channels larger than of others, as models have it; V of size one."""
    hd = c["hd"]
    dt = DTYPES[c["dtype"]]
    k = torch.randn((layers, pages, c["hkv"], c["page"] // 32, hd // 16, 2, 32, 8), generator=g, device="cuda", dtype=dt)
    k *= torch.exp(0.4 * torch.randn((c["hkv"], 1, hd // 16, 2, 1, 8), generator=g, device="cuda")).to(dt)
    v = torch.randn((layers, pages, c["hkv"], c["page"] * hd), generator=g, device="cuda", dtype=dt)
    shape = (layers, pages, c["hkv"], c["page"], hd)
    return k.reshape(shape), v.reshape(shape)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _projection(c, rows, g):
    """q, k, v: parts of the rows that one projection leaves."""
    hq, hkv, hd = c["hq"], c["hkv"], c["hd"]
    x = (1.5 * torch.randn((rows, hq + 2 * hkv, hd), generator=g, device="cuda")).to(DTYPES[c["dtype"]])
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _gains(c, g):
    if not c["norm"]:
        return None, None
    return tuple((1 + 0.1 * torch.randn(c["hd"], generator=g, device="cuda")).to(DTYPES[c["dtype"]]) for _ in range(2))


def _rotation(c):
    """theta 5e5; scaled frequencies keep what turns 4 times or more within 8192 positions."""
    scaled = c["factor"] != 1.0
    return dict(rot_dim=c["rot"], theta=5e5, interleaved=c["interleaved"], factor=c["factor"], orig_len=8192 if scaled else 0, low_turns=1.0,
                high_turns=4.0, amplitude=1.0 + 0.1 * math.log(c["factor"]))


def prepare(case, seed):
    c, g = case, _gen(seed)
    if c["kind"] == "rope":
        q, k, _ = _projection(c, c["rows"], g)
        qg, kg = _gains(c, g)
        pos = torch.randint(0, c["far"], (c["rows"],), generator=g, device="cuda", dtype=torch.int32)
        return dict(case=c, q=q, k=k, q_gain=qg, k_gain=kg, pos=pos, rotation=_rotation(c), q_out=torch.empty_like(q).contiguous(),
                    k_out=torch.empty_like(k).contiguous())
    lens = _lens(c)
    rows = [_TREE_ROWS] * c["batch"] if c["kind"] == "commit" else _rows(c)
    pages, table = _pages(c, lens, rows, g)
    kp, vp = _pool(c, c["layers"] if c["kind"] == "commit" else 1, pages, g)
    s = dict(case=c, k_pool=kp, v_pool=vp, table=table, lens=_i32(lens))
    if c["kind"] == "commit":
        paths = [_path(c, b) for b in range(c["batch"])]
        s.update(n_emit=_i32([len(p) for p in paths]), accepted=_i32([p + [0] * (9 - len(p)) for p in paths]), len_out=torch.zeros_like(s["lens"]))
        return s
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    s.update(row0=_i32(starts), total=starts[-1])
    if c["kind"] == "append":
        q, k, v = _projection(c, starts[-1], g)
        qg, kg = _gains(c, g)
        pos = None
        if c["given"]:
            pos = _i32([l + d for b, (l, r) in enumerate(zip(lens, rows)) for d in _depths(_parents(r, c["mix"], b))])
        s.update(q=q, k=k, v=v, q_gain=qg, k_gain=kg, pos=pos, rotation=_rotation(c), q_out=torch.empty_like(q).contiguous())
        return s
    q = (1.5 * torch.randn((starts[-1], c["hq"], c["hd"]), generator=g, device="cuda")).to(DTYPES[c["dtype"]])
    s.update(q=q, out=torch.empty_like(q), anc=None)
    if c["mask"] == "tree":
        words = (c["rows_hi"] + 63) // 64
        bits = [a for b, r in enumerate(rows) for a in _ancestors(_parents(r, c["mix"], b))]
        signed = [[(w ^ (1 << 63)) - (1 << 63) for w in ((a >> (64 * i)) & ((1 << 64) - 1) for i in range(words))] for a in bits]
        s["anc"] = torch.tensor(signed, dtype=torch.int64, device="cuda")
    return s


# ---- the framework's entry points --------------------------------------------------------------------------

def _run_own(s):
    from paper_2603_17942_amd import binding as B
    c = s["case"]
    if "handles" not in s:       # what a program keeps around its own tensors from step to step
        h = {}
        if "rotation" in s:
            h["rope"] = B.rope_spec(c["hd"], **s["rotation"])
        if "table" in s:
            h["kv"] = B.PagedKv(s["k_pool"], s["v_pool"], s["table"], s["lens"], len_bound=c["len_hi"])
        if "row0" in s:
            h["rows"] = B.ChunkRows(s["row0"], s["total"], c["rows_hi"])
        if c["kind"] == "attn":
            h["scratch"] = torch.empty(B.paged_attn_scratch_bytes(h["kv"], h["rows"], c["hq"]), dtype=torch.uint8, device="cuda")
        s["handles"] = h
    h = s["handles"]
    if c["kind"] == "rope":
        return B.rope_qk(s["q"], s["k"], s["pos"], h["rope"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=1e-6, q_out=s["q_out"], k_out=s["k_out"])
    if c["kind"] == "append":
        q = B.paged_append(h["kv"], 0, h["rows"], s["q"], s["k"], s["v"], rope=h["rope"], positions=s["pos"], q_gain=s["q_gain"],
                           k_gain=s["k_gain"], eps=1e-6, q_out=s["q_out"])
        return q, s["k_pool"], s["v_pool"]
    if c["kind"] == "commit":
        B.paged_commit(h["kv"], s["n_emit"], s["accepted"], s["len_out"])
        return s["k_pool"], s["v_pool"], s["len_out"]
    return B.paged_attn(h["kv"], 0, h["rows"], s["q"], anc=s["anc"], out=s["out"], scratch=h["scratch"])


# ---- the plain forms -----------------------------------------------------------------------------------------

def _plain_rotated(x, gain, pos, rot):
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gain.float()
    r = rot["rot_dim"]
    f = rot["theta"] ** (-torch.arange(0, r, 2, dtype=torch.float64, device=x.device) / r)
    turns = rot["orig_len"] * f / (2 * math.pi)
    keep = ((turns - rot["low_turns"]) / (rot["high_turns"] - rot["low_turns"])).clamp(0, 1)
    a = pos.double()[:, None] * (f * (keep + (1 - keep) / rot["factor"]))
    cos, sin = ((rot["amplitude"] * t).float()[:, None] for t in (a.cos(), a.sin()))
    if rot["interleaved"]:
        u, w = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2)
    else:
        u, w = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([u * cos - w * sin, w * cos + u * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _k_places(slot, hd):
    """Where the elements of slots lie in a plane of a page, K."""
    d = torch.arange(hd, device=slot.device)
    return (slot // 32 * hd * 32 + slot % 32 * 8)[..., None] + (d // 16 * 64 + d // 8 % 2 * 32) * 8 + d % 8


def _v_places(slot, hd):
    key, d = slot % 32, torch.arange(hd, device=slot.device)
    at = slot // 32 * hd * 32 + (key // 16 * 64 + key // 4 % 2 * 32) * 8 + key // 8 % 2 * 4 + key % 4
    return at[..., None] + d // 32 * 1024 + d % 32 * 8


def _sequence_and_slot(s):
    """For every row its sequence, and its place there."""
    row = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(s["row0"][1:].long(), row, right=True)
    return seq, s["lens"].long()[seq] + row - s["row0"].long()[seq]


def _plain_append(s):
    c = s["case"]
    seq, slot = _sequence_and_slot(s)
    pos = slot if s["pos"] is None else s["pos"]
    page = s["table"][seq, slot // c["page"]].long()
    q = _plain_rotated(s["q"], s["q_gain"], pos, s["rotation"]).to(s["q"].dtype)
    k = _plain_rotated(s["k"], s["k_gain"], pos, s["rotation"]).to(s["k"].dtype)
    planes = (page[:, None] * c["hkv"] + torch.arange(c["hkv"], device="cuda"))[..., None] * (c["page"] * c["hd"])
    inside = slot % c["page"]
    s["k_pool"].view(-1)[planes + _k_places(inside, c["hd"])[:, None]] = k
    s["v_pool"].view(-1)[planes + _v_places(inside, c["hd"])[:, None]] = s["v"]
    return q, s["k_pool"], s["v_pool"]


def _plain_commit(s):
    c = s["case"]
    i = torch.arange(1, s["accepted"].shape[1], device="cuda")
    lens = s["lens"].long()[:, None]
    wanted = i < s["n_emit"][:, None]
    # a place that is not wanted moves onto itself: the root's own
    src, dst = (torch.where(wanted, lens + t, lens) for t in (s["accepted"][:, 1:].long(), i))
    shape = s["k_pool"].shape

    def places(slot, of):
        page = torch.gather(s["table"].long(), 1, slot // c["page"])
        planes = (page[..., None] * c["hkv"] + torch.arange(c["hkv"], device="cuda"))[..., None] * (c["page"] * c["hd"])
        return planes + of(slot % c["page"], c["hd"])[:, :, None]
    for pool, of in ((s["k_pool"], _k_places), (s["v_pool"], _v_places)):
        flat = pool.view(shape[0], -1)
        flat[:, places(dst, of)] = flat[:, places(src, of)]
    torch.add(s["lens"], s["n_emit"], out=s["len_out"])
    return s["k_pool"], s["v_pool"], s["len_out"]


def _plain_attn(s):
    c = s["case"]
    B, R, hq, hkv, hd, page = c["batch"], c["rows_hi"], c["hq"], c["hkv"], c["hd"], c["page"]
    G, T = hq // hkv, s["table"].shape[1] * c["page"]
    kp, vp = (p[0][s["table"].long()] for p in (s["k_pool"], s["v_pool"]))         # [B, pages, hkv, page, hd]
    n, blocks = s["table"].shape[1], page // 32
    k = kp.view(B, n, hkv, blocks, hd // 16, 2, 32, 8).permute(0, 2, 4, 5, 7, 1, 3, 6).reshape(B, hkv, hd, T).float()
    v = vp.view(B, n, hkv, blocks, hd // 32, 2, 2, 32, 2, 4).permute(0, 2, 1, 3, 5, 8, 6, 9, 4, 7).reshape(B, hkv, T, hd).float()
    row0, lens = s["row0"].long(), s["lens"].long()
    r = torch.arange(R, device="cuda")
    live = r < (row0[1:] - row0[:-1])[:, None]
    at = torch.where(live, row0[:-1, None] + r, 0)                                   # [B, R]
    slot = torch.arange(T, device="cuda")
    behind = slot - lens[:, None]                                                    # slots of the new rows count from 0
    if c["mask"] == "causal":
        seen = behind[:, None] <= r[:, None]
    else:
        words = s["anc"][at]                                                         # [B, R, words]
        place = behind.clamp(0, words.shape[2] * 64 - 1)[:, None].expand(B, R, T)
        seen = (torch.gather(words, 2, place // 64) >> (place % 64)) & 1 == 1
        seen = seen & (behind[:, None] < words.shape[2] * 64) | (behind[:, None] < 0)
    seen = seen & live[:, :, None] & (slot < (lens + row0[1:] - row0[:-1])[:, None])[:, None]
    q = s["q"][at].float().view(B, R, hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(B, hkv, R * G, hd)
    x = torch.matmul(q, k).mul_(1 / math.sqrt(hd)).view(B, hkv, R, G, T)
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, hkv, R * G, T), v).view(B, hkv, R, G, hd) / total.clamp_min(1e-30)
    s["out"].copy_(o.permute(0, 2, 1, 3, 4).reshape(B, R, hq, hd)[live])
    return s["out"]


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "append":
        return _plain_append(state)
    if kind == "commit":
        return _plain_commit(state)
    if kind == "attn":
        return _plain_attn(state)
    for x, gain, out in (("q", "q_gain", "q_out"), ("k", "k_gain", "k_out")):
        state[out].copy_(_plain_rotated(state[x], state[gain], state["pos"], state["rotation"]))
    return state["q_out"], state["k_out"]


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    if c["kind"] == "rope":
        heads = c["hq"] + c["hkv"]
        return {"bytes": 2 * c["rows"] * heads * c["hd"] * e + 4 * c["rows"], "flops": c["rows"] * heads * (3 * c["rot"] + 3 * c["hd"] * c["norm"])}
    if c["kind"] == "commit":
        moved = sum(len(_path(c, b)) - 1 for b in range(c["batch"]))
        return {"bytes": 4 * c["layers"] * c["hkv"] * c["hd"] * e * moved + 48 * c["batch"], "flops": 0}
    rows, lens = _rows(c), _lens(c)
    if c["kind"] == "append":
        n, heads = sum(rows), c["hq"] + c["hkv"]
        return {"bytes": 2 * n * (heads + c["hkv"]) * c["hd"] * e, "flops": n * heads * (3 * c["rot"] + 3 * c["hd"] * c["norm"])}
    if c["mask"] == "causal":
        seen = sum(r * l + r * (r + 1) // 2 for r, l in zip(rows, lens))
    else:
        seen = sum(r * l + sum(_depths(_parents(r, c["mix"], b))) + r for b, (r, l) in enumerate(zip(rows, lens)))
    return {"bytes": 2 * sum(rows) * c["hq"] * c["hd"] * e + 2 * sum(r + l for r, l in zip(rows, lens)) * c["hkv"] * c["hd"] * e,
            "flops": 4 * c["hd"] * c["hq"] * seen}


# ---- from the definition, in 64 bits -----------------------------------------------------------------------------

def _exact_rotated(c, x, gain, pos):
    """Pairs as complex numbers that turn."""
    x = x.double().clone()
    if gain is not None:
        x *= gain.double() / (x.pow(2).sum(-1, keepdim=True) / c["hd"] + 1e-6).sqrt()
    R = c["rot"]
    first = [2 * i if c["interleaved"] else i for i in range(R // 2)]
    second = [2 * i + 1 if c["interleaved"] else i + R // 2 for i in range(R // 2)]
    speed = []
    for i in range(R // 2):
        w = 5e5 ** (-2.0 * i / R)
        part = 1.0
        if c["factor"] != 1.0:
            part = min(1.0, max(0.0, (8192 * w / (2 * math.pi) - 1.0) / 3.0))
        speed.append(part * w + (1 - part) * w / c["factor"])
    angle = pos.double()[:, None, None] * torch.tensor(speed, dtype=torch.float64, device=x.device)
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.full_like(angle, 1.0 + 0.1 * math.log(c["factor"])), angle)
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_planes(c, s, b, slots, of_v):
    """For slots of sequence b: the elements' places in the flat pool of a layer, [slots, hkv, hd]."""
    hd, out = c["hd"], []
    d = torch.arange(hd, device="cuda")
    inside = slots % c["page"]
    block, key = torch.div(inside, 32, rounding_mode="floor"), inside % 32
    if of_v:
        lane = ((key >> 2) & 1)[:, None] * 32 + (d & 31)
        piece = ((d >> 5) * 2 + (key >> 4)[:, None]) * 64 + lane
        place = piece * 8 + (4 * ((key >> 3) & 1) + (key & 3))[:, None]
    else:
        place = ((d >> 4) * 64 + ((d >> 3) & 1) * 32 + key[:, None]) * 8 + (d & 7)
    place = place + (block * (32 * hd))[:, None]
    page = s["table"][b].long()[torch.div(slots, c["page"], rounding_mode="floor")]
    for h in range(c["hkv"]):
        out.append(place + ((page * c["hkv"] + h) * (c["page"] * hd))[:, None])
    return torch.stack(out, 1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "rope":
        return _exact_rotated(c, s["q"], s["q_gain"], s["pos"]), _exact_rotated(c, s["k"], s["k_gain"], s["pos"])
    lens, rows = _lens(c), None
    if c["kind"] == "commit":
        pools = []
        for pool, of_v in ((s["k_pool"], False), (s["v_pool"], True)):
            flat, out = pool.reshape(c["layers"], -1), pool.double().reshape(c["layers"], -1)
            for b in range(c["batch"]):
                for i, r in enumerate(_path(c, b)):
                    to, frm = (_exact_planes(c, s, b, torch.tensor([lens[b] + t], device="cuda"), of_v).reshape(-1) for t in (i, r))
                    out[:, to] = flat[:, frm].double()
            pools.append(out.reshape(pool.shape))
        return pools[0], pools[1], _i32([lens[b] + len(_path(c, b)) for b in range(c["batch"])])
    rows = _rows(c)
    if c["kind"] == "append":
        at, qs, pools = 0, [], [s["k_pool"].double().reshape(-1), s["v_pool"].double().reshape(-1)]
        for b, (l, r) in enumerate(zip(lens, rows)):
            slots = l + torch.arange(r, device="cuda")
            pos = slots if s["pos"] is None else s["pos"][at:at + r]
            qs.append(_exact_rotated(c, s["q"][at:at + r], s["q_gain"], pos))
            pools[0][_exact_planes(c, s, b, slots, False)] = _exact_rotated(c, s["k"][at:at + r], s["k_gain"], pos)
            pools[1][_exact_planes(c, s, b, slots, True)] = s["v"][at:at + r].double()
            at += r
        return torch.cat(qs), pools[0].reshape(s["k_pool"].shape), pools[1].reshape(s["v_pool"].shape)
    G, at, outs = c["hq"] // c["hkv"], 0, []
    for b, (l, r) in enumerate(zip(lens, rows)):
        slots = torch.arange(l + r, device="cuda")
        k = s["k_pool"].reshape(-1)[_exact_planes(c, s, b, slots, False)].double()
        v = s["v_pool"].reshape(-1)[_exact_planes(c, s, b, slots, True)].double()
        hidden = torch.zeros((r, l + r), dtype=torch.bool, device="cuda")
        if c["mask"] == "causal":
            hidden[:, l:] = torch.ones((r, r), dtype=torch.bool, device="cuda").triu(1)
        else:
            sees = _ancestors(_parents(r, c["mix"], b))
            hidden[:, l:] = torch.tensor([[not (a >> j) & 1 for j in range(r)] for a in sees], device="cuda")
        o = torch.empty((r, c["hq"], c["hd"]), dtype=torch.float64, device="cuda")
        for h in range(c["hq"]):
            x = s["q"][at:at + r, h].double() @ k[:, h // G].t().contiguous() / math.sqrt(c["hd"])
            x = x.masked_fill(hidden, -math.inf)
            w = (x - x.max(-1, keepdim=True).values).exp()
            o[:, h] = w @ v[:, h // G] / w.sum(-1, keepdim=True)
        outs.append(o)
        at += r
    return torch.cat(outs)
