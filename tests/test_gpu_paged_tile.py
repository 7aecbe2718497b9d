"""Attention over pages where the tile kernel has the work: whole items and shares, one sequence and many, what nobody sees holding no numbers.

References and tolerances are those of test_gpu_paged.py; of long chunks some rows are compared.  Every case says what it is planned as, so that a
rule that moves it to another kernel fails here."""
import copy
import ctypes as C
import functools
import math

import numpy as np
import pytest
import torch

from test_gpu_paged import DT, Cache, attention, k_place, pack_anc, queries, random_tree, v_place, visible
from util import internal

from paper_2603_17942_amd import binding as B

pytestmark = pytest.mark.gpu


class Plan(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("cap", "q_tiles", "shares", "least")]


@functools.lru_cache(None)
def plans():
    return internal("paged_attn_plan", *[C.c_int] * 8, restype=Plan)


MANY = [(37 * i) % 1001 for i in range(64)], [(i * 5) % 17 for i in range(64)]                       # 0 to 1000 keys, 0 to 16 rows
PAIRS = [(613 * i) % 3001 for i in range(20)], [1 + (i * 5) % 16 for i in range(20)]                 # two column tiles a sequence and kv head
BATCH = [(311 * i) % 2001 for i in range(40)], [1 + (i * 7) % 16 for i in range(40)]

# dtype, hd, hq, hkv, page, lens, rows, column tiles of an item at most, in shares
TILE = {
    "prompt_bf16_128": ("bf16", 128, 32, 8, 64, [0], [2304], 8, False),
    "prompt_bf16_64": ("bf16", 64, 64, 16, 32, [0], [2311], 8, False),
    "prompt_f32_128": ("f32", 128, 32, 8, 64, [0], [2100], 4, False),
    "prompt_f32_64": ("f32", 64, 32, 16, 96, [100], [2100], 4, False),
    "many_bf16_128": ("bf16", 128, 32, 8, 32, *MANY, 8, False),
    "many_bf16_64": ("bf16", 64, 32, 8, 64, *MANY, 8, False),
    "many_f32_128": ("f32", 128, 32, 8, 32, *MANY, 4, False),
    "chunk_bf16_128": ("bf16", 128, 32, 8, 64, [9000], [300], 8, True),
    "chunk_bf16_64": ("bf16", 64, 32, 8, 128, [21001], [333], 8, True),
    "chunk_f32_128": ("f32", 128, 4, 1, 32, [6000], [200], 4, True),
    "batch_bf16_128": ("bf16", 128, 32, 8, 64, *BATCH, 8, True),
    "batch_f32_64": ("f32", 64, 32, 8, 32, *BATCH, 4, True),
    "pairs_bf16_128": ("bf16", 128, 32, 8, 64, *PAIRS, 2, True),
    "pairs_bf16_64": ("bf16", 64, 32, 8, 96, *PAIRS, 2, True),
    "pairs_f32_128": ("f32", 128, 32, 8, 32, *PAIRS, 2, True),
}


ALL = dict(TILE, **{      # and of the stream kernel, whole and in shares
    "stream_bf16_128": ("bf16", 128, 8, 2, 32, [50, 7], [40, 9], 1, False),
    "stream_bf16_64": ("bf16", 64, 8, 2, 32, [4000, 7], [1, 9], 1, True),
    "stream_f32_128": ("f32", 128, 8, 2, 64, [40, 90], [33, 5], 1, False),
    "stream_f32_64": ("f32", 64, 8, 2, 32, [2500, 1], [12, 3], 1, True),
})


@functools.lru_cache(None)
def built(name, single_rows=False):
    dtype, hd, hq, hkv, page, lens, rows, cap, shares = ALL[name]
    if single_rows:
        lens, rows = list(lens), [1 if b % 2 == 0 else r for b, r in enumerate(rows)]
        lens[2] = lens[6] = 0
    c = Cache(DT[dtype], hkv, hd, page, lens, rows, 501)
    p = plans()(c.kv.struct.dtype, hd, len(lens), hq, hkv, c.chunk.total_rows, c.chunk.max_rows, c.kv.len_bound)
    assert (p.cap, p.shares > 0) == (cap, shares), (p.cap, p.shares)
    return c, queries(c.starts[-1], hq, hd, DT[dtype], 502)


def make(name, single_rows=False):
    """A cache of the case and its queries, the test's own to spoil."""
    first, q = built(name, single_rows)
    c = copy.copy(first)
    c.table, c.v, kv = first.table.clone(), [v.clone() for v in first.v], first.kv
    c.kv = B.PagedKv(kv.k.clone(), kv.v.clone(), kv.page_table.clone(), kv.lens.clone(), kv.len_bound)
    return c, q


def some_rows(r, b):
    """Of many rows 16 at most, the ends among them."""
    return list(range(r)) if r <= 40 else sorted({0, 1, 31, 32, 33, r - 2, r - 1} | set(np.random.default_rng(b).integers(0, r, 9).tolist()))


def some_sequences(c):
    """Of many with rows, the first eight and every second."""
    return [b for b, r in enumerate(c.rows) if r and (b < 8 or b % 2)]


def check(c, q, out, seen_of):
    """seen_of(b): [rows, keys] of sequence b, what its rows see."""
    out = out.cpu().double()
    for b in some_sequences(c):
        r = c.rows[b]
        pick = torch.tensor(some_rows(r, b))
        at = c.starts[b] + pick
        want, tol = attention(q.cpu()[at], c.k[b], c.v[b], seen_of(b)[pick], c.hd ** -0.5)
        assert torch.isfinite(out[at]).all(), b
        worst = ((out[at] - want).abs() - tol).max()
        assert worst <= 0, (b, float(worst))
    assert torch.isfinite(out).all()


def clear_page_0(c):
    """What is in page 0 moves to a page that is free, and page 0, nobody's then, holds no numbers."""
    free = next(p for p in range(c.kv.k.shape[1] - 1, 0, -1) if not (c.table == p).any())
    for pool in (c.kv.k, c.kv.v):
        pool[:, free] = pool[:, 0]
        pool[:, 0] = math.nan
    c.table[c.table == 0] = free
    c.kv.page_table.copy_(c.table)


@pytest.mark.parametrize("name", TILE)
@pytest.mark.parametrize("tree", [False, True])
def test_whole_items_and_shares(name, tree):
    c, q = make(name)
    ancs = [random_tree(r, 570 + b) for b, r in enumerate(c.rows)] if tree else None
    anc = pack_anc(ancs, c.rows, (max(c.rows) + 63) // 64 + 1) if tree else None
    out = torch.full_like(q, 7.0)
    B.paged_attn(c.kv, 0, c.chunk, q, anc=anc, out=out)
    check(c, q, out, lambda b: visible(c.lens[b], c.rows[b], ancs[b] if tree else None))
    assert torch.equal(out, B.paged_attn(c.kv, 0, c.chunk, q, anc=anc)) and c.kv.device_status() == 0


@pytest.mark.parametrize("name", [n for n in TILE if not n.startswith("prompt")])
@pytest.mark.parametrize("tree", [False, True])
def test_rows_that_are_not_finite_and_missing_pages(name, tree):
    """Of ragged sequences: who sees a row whose K and V are no numbers is not finite, everybody else is right."""
    c, q = make(name)
    hkv, d = c.kv.n_kv_heads, np.arange(c.hd)
    clear_page_0(c)
    bad = {b: sorted({l + r - 1, l + r // 2}) for b, (l, r) in enumerate(zip(c.lens, c.rows)) if r > 2 and b % 4 != 1}
    for b, slots in bad.items():
        for i, s in enumerate(slots):
            for pool, place in ((c.kv.k, k_place), (c.kv.v, v_place)):
                pool[0, int(c.table[b, s // c.page])].view(hkv, -1)[:, torch.from_numpy(place(s % c.page, d, c.hd)).cuda()] = (math.nan, math.inf)[(b + i) % 2]
    gone = [b for b, l in enumerate(c.lens) if l >= 2 * c.page and b % 3 == 0]
    for b in gone:
        c.kv.page_table[b, 1] = -1 - b
    ancs = [random_tree(r, 590 + b) for b, r in enumerate(c.rows)] if tree else None
    out = B.paged_attn(c.kv, 0, c.chunk, q, anc=pack_anc(ancs, c.rows, (max(c.rows) + 63) // 64) if tree else None).cpu().double()
    assert c.kv.device_status() == 16 and gone
    clean = 0
    for b in some_sequences(c):
        l, r = c.lens[b], c.rows[b]
        seen = visible(l, r, ancs[b] if tree else None)
        if b in gone:
            seen[:, c.page:2 * c.page] = False
        hit = seen[:, bad[b]].any(1) if b in bad else torch.zeros(r, dtype=torch.bool)
        got = out[c.starts[b]:c.starts[b] + r]
        assert not torch.isfinite(got[hit]).any(), b
        pick = torch.tensor([i for i in some_rows(r, b) if not hit[i]], dtype=torch.long)
        want, tol = attention(q.cpu()[c.starts[b] + pick], c.k[b], c.v[b], seen[pick], c.hd ** -0.5)
        assert torch.isfinite(got[~hit]).all() and ((got[pick] - want).abs() <= tol).all(), b
        clean += len(pick)
    assert clean > 10


@pytest.mark.parametrize("name", TILE)
@pytest.mark.parametrize("tree", [False, True])
def test_missing_pages_beside_a_page_that_is_not_finite(name, tree):
    """The slots of pages outside the pool are not seen, whatever the pool's own pages hold."""
    c, q = make(name)
    clear_page_0(c)
    missing = {b: [p for p in (0, 2, (l - 1) // c.page - 1) if 0 <= p < l // c.page] for b, l in enumerate(c.lens) if b % 3 == 0}
    if len(c.lens) == 1 and c.lens[0] == 0:
        missing = {0: [0, 2]}
    for b, pages in missing.items():
        for i, p in enumerate(pages):
            c.kv.page_table[b, p] = (-1, 10 ** 6)[i % 2]
    ancs = [random_tree(r, 510 + b) for b, r in enumerate(c.rows)] if tree else None
    out = B.paged_attn(c.kv, 0, c.chunk, q, anc=pack_anc(ancs, c.rows, (max(c.rows) + 63) // 64) if tree else None)

    def seen(b):
        m = visible(c.lens[b], c.rows[b], ancs[b] if tree else None)
        for p in missing.get(b, []):
            m[:, p * c.page:(p + 1) * c.page] = False
        return m
    check(c, q, out, seen)
    assert c.kv.device_status() == 16


@pytest.mark.parametrize("name", ["many_bf16_128", "many_bf16_64", "many_f32_128", "batch_bf16_128", "batch_f32_64", "pairs_bf16_64"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_one_row_that_does_not_see_itself(name, what):
    """A sequence's only row, hidden from itself, whose K and V are no numbers: zeros where there is nothing before it, else attention to that."""
    c, q = make(name, True)
    lens, rows, hd, hkv, page = c.lens, c.rows, c.hd, c.kv.n_kv_heads, c.page
    d = np.arange(hd)
    ancs = [random_tree(r, 530 + b) for b, r in enumerate(rows)]
    for b, r in enumerate(rows):
        if r != 1:
            continue
        ancs[b][0, 0] = False
        pg, inside = int(c.table[b, lens[b] // page]), lens[b] % page
        for pool, place in ((c.kv.k, k_place), (c.kv.v, v_place)):
            pool[0, pg].view(hkv, -1)[:, torch.from_numpy(place(inside, d, hd)).cuda()] = what
    out = B.paged_attn(c.kv, 0, c.chunk, q, anc=pack_anc(ancs, rows, 1))
    check(c, q, out, lambda b: visible(lens[b], rows[b], ancs[b]))
    for b in (2, 6):
        assert (out[c.starts[b]] == 0).all()
    assert c.kv.device_status() == 0


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("tree", [False, True])
def test_infinities_keep_their_sign(name, tree):
    """Infinities among the values a row sees make its output that infinity, NaN and infinities of both signs make it NaN, in committed slots and in
    the chunk's own; who does not see them has its own output.  (The scores are of size 1.5, so no probability comes to nothing.)"""
    c, q = make(name)
    lens, rows, hd, hkv, hq, page = c.lens, c.rows, c.hd, c.kv.n_kv_heads, q.shape[1], c.page
    kvh, inf, nan = hkv - 1, math.inf, math.nan
    for b, (l, r) in enumerate(zip(lens, rows)):
        slots = [s for s, there in ((l // 2, l > 0), (l + r // 3, r > 0), (l + r // 2, r > 3), (l + r - 1, r > 5)) if there]
        for i, s in enumerate(slots):
            for d, what in ((1, -inf), (2, inf), (3 if i % 2 else hd - 1, -inf), (4, inf if i else -inf), (5, -inf if i else inf), (6, nan if i == 1 else -inf),
                            (40, -inf if i == 2 else 0.5), (41, inf if i == 2 else -0.5)):
                c.v[b][s, kvh, d] = what
                pg, inside = int(c.table[b, s // page]), s % page
                c.kv.v[0, pg].view(hkv, -1)[kvh, v_place(inside, d, hd)] = what
    ancs = [random_tree(r, 550 + b) for b, r in enumerate(rows)] if tree else None
    out = B.paged_attn(c.kv, 0, c.chunk, q, anc=pack_anc(ancs, rows, (max(rows) + 63) // 64) if tree else None).cpu().double()
    hit = 0
    for b in some_sequences(c):
        l, r = lens[b], rows[b]
        pick = torch.tensor(some_rows(r, b))
        at, seen = c.starts[b] + pick, visible(l, r, ancs[b] if tree else None)[pick]
        v = c.v[b].double()
        want, tol = attention(q.cpu()[at], c.k[b], torch.where(torch.isfinite(v), v, 0.0).to(c.dt), seen, hd ** -0.5)
        s = seen.double()
        up, down, none = (torch.einsum("rt,thd->rhd", s, m.double()) > 0 for m in (v == inf, v == -inf, v.isnan()))
        odd = torch.where(none | (up & down), nan, torch.where(up, inf, torch.where(down, -inf, 0.0))).repeat_interleave(hq // hkv, 1)
        got = out[at]
        same = (got == odd) | (got.isnan() & odd.isnan())
        fine = (got - want).abs() <= tol
        assert torch.where(odd == 0, fine, same).all(), b
        hit += int((odd != 0).sum())
    assert hit > 0
