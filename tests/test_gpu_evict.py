"""Attention weights of cached tokens (paged_weigh) and the bound on what a sequence keeps (paged_evict) against plain forms in 64 bits, and a serving loop
over the cache that samples, weighs and evicts.

Tolerance of a token's mass, sum of p over n columns (row, query head).  A score is a sum of hd products, off by hd 2^-24 sum |q k| at most; scale and
reference add 4 roundings of the largest score, twice (the reference is off too, but it is the same number everywhere and cancels); the exponent
instruction is off by 2^-22; a row's sum of t exponentials by (t / 32 + 64) 2^-24, which over the units that a lane adds up is what a run of additions
can do, its reciprocal by 2^-23; adding up n columns and `before` by (n + 8) 2^-24 of the mass, the number stored by 2^-24 of itself.
Eviction moves numbers as they are: lists, pages and masses have to be equal."""
import math

import numpy as np
import pytest
import torch

from util import ROOT  # noqa: F401

from paper_2603_17942_amd import binding as B
from test_gpu_paged import DT, U, gen, i32, k_place, queries, v_place

pytestmark = pytest.mark.gpu


class Plain:
    """A paged cache whose contents the test knows in every layer: K and V of sequence b as rows [layers, tokens, kv heads, hd]; everything else NaN.
    table_out: pages of `keep` tokens for each, behind the others."""

    def __init__(self, dt, layers, hkv, hd, page, lens, rows, seed, room=None, keep=0, std=1.0):
        g = gen(seed)
        self.dt, self.layers, self.hkv, self.hd, self.page, self.lens, self.rows = dt, layers, hkv, hd, page, lens, rows
        need = [(l + r + page - 1) // page for l, r in zip(lens, rows)]
        also = (keep + page - 1) // page
        n = sum(need) + also * len(lens) + 3
        order = torch.randperm(n, generator=g).to(torch.int32)
        stride = max(max(need), 1, room or 0)
        table = torch.full((len(lens), stride), 2 ** 31 - 1, dtype=torch.int32)
        self.pages = n
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = order[at:at + k]
            at += k
        self.fresh = order[at:at + also * len(lens)].reshape(len(lens), also).clone() if also else None
        self.table = table
        self.kn = torch.full((layers, n, hkv, page * hd), math.nan)
        self.vn = self.kn.clone()
        self.k = [(torch.randn((layers, l + r, hkv, hd), generator=g) * std).to(dt) for l, r in zip(lens, rows)]
        self.v = [torch.randn((layers, l + r, hkv, hd), generator=g).to(dt) for l, r in zip(lens, rows)]
        for b, (l, r) in enumerate(zip(lens, rows)):
            self.put(self.kn, self.vn, table[b], self.k[b], self.v[b], l + r)
        shape = (layers, n, hkv, page, hd)
        self.kv = B.PagedKv(self.kn.to(dt).reshape(shape).cuda(), self.vn.to(dt).reshape(shape).cuda(), table.cuda(), i32(lens), max(lens))
        self.starts = np.concatenate([[0], np.cumsum(rows)]).tolist()
        self.chunk = B.ChunkRows(i32(self.starts), self.starts[-1], max(max(rows), 1))

    def put(self, kn, vn, table, k, v, n, only=None):
        """rows [layers, n, hkv, hd] into slots 0.. of a sequence's pages (only: of these heads' tokens per layer)."""
        d = np.arange(self.hd)
        for s in range(n):
            pg, inside = int(table[s // self.page]), s % self.page
            kn[:, pg][:, :, k_place(inside, d, self.hd)] = k[:, s].float()
            vn[:, pg][:, :, v_place(inside, d, self.hd)] = v[:, s].float()

    def pools(self):
        return tuple(t.cpu().float().reshape(self.kn.shape) for t in (self.kv.k, self.kv.v))


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0))


# ---- weights ---------------------------------------------------------------------------------------------------

def weights(c, layer, b, q, last, scale):
    """(mass, tolerance) [hkv, tokens] of a sequence, without `before`."""
    l, r = c.lens[b], c.rows[b]
    n = min(r, last) if last else r
    G = q.shape[1] // c.hkv
    seen = torch.arange(l + r) <= (l + torch.arange(r - n, r))[:, None]
    mass, tol = torch.zeros((c.hkv, l + r), dtype=torch.float64), torch.zeros((c.hkv, l + r), dtype=torch.float64)
    rows = q[c.starts[b + 1] - n:c.starts[b + 1]].cpu().double()
    for h in range(c.hkv):
        k = c.k[b][layer, :, h].double()
        for g in range(G):
            x = rows[:, h * G + g] @ k.T * scale
            size = (rows[:, h * G + g].abs() @ k.abs().T * scale).masked_fill(~seen, 0.0).amax(1, keepdim=True)
            p = torch.softmax(x.masked_fill(~seen, -math.inf), 1)
            off = 2 * U * (c.hd * size + 8 * torch.where(seen, x.abs(), 0.0).amax(1, keepdim=True)) + 2.0 ** -21 + ((l + r) / 32 + 68) * U
            mass[h] += p.sum(0)
            tol[h] += (p * off).sum(0)
        tol[h] += (n * G + 8) * U * mass[h] + 1e-30
    return mass, tol


def check_mass(c, layer, q, got, before, last=0, scale=None):
    """got, before [layers, batch, hkv, slots] on the CPU; slots that nobody writes are as `before`'s own."""
    scale = c.hd ** -0.5 if scale is None else scale
    for b, (l, r) in enumerate(zip(c.lens, c.rows)):
        if r == 0:
            continue
        want, tol = weights(c, layer, b, q, last, scale)
        old = before[layer, b].double()
        want[:, :l] += old[:, :l]
        tol[:, :l] += 9 * U * old[:, :l]
        mine = got[layer, b, :, :l + r].double()
        assert torch.isfinite(mine).all(), b
        worst = ((mine - want).abs() - tol - U * want).max()
        assert worst <= 0, (b, float(worst), float((mine - want).abs().max()))


WEIGH = [  # dtype, hd, hq, hkv, page, lens, rows, last
    ("bf16", 128, 32, 8, 64, [0], [1], 0),
    ("bf16", 128, 32, 8, 64, [2047], [1], 0),
    ("bf16", 128, 8, 2, 32, [31, 32, 33, 0, 127, 128, 129], [1] * 7, 0),
    ("bf16", 128, 32, 8, 64, [0, 1, 63, 64, 500], [1, 7, 8, 9, 0], 0),
    ("bf16", 128, 32, 8, 64, [0, 1, 63, 64, 500], [1, 7, 8, 9, 0], 3),
    ("bf16", 128, 4, 4, 96, [95, 96, 97, 191, 300], [33, 1, 2, 65, 31], 0),
    ("bf16", 128, 4, 4, 96, [95, 96, 97, 191, 300], [33, 1, 2, 65, 31], 32),
    ("bf16", 128, 28, 4, 128, [130, 700], [5, 40], 0),
    ("bf16", 128, 8, 1, 32, [64, 5], [3, 300], 16),
    ("bf16", 128, 16, 2, 64, [0, 1000], [257, 129], 0),
    ("bf16", 128, 6, 2, 64, [4000, 3], [1, 1], 0),
    ("bf16", 128, 5, 5, 32, [0, 0, 0], [1, 2, 3], 0),
    ("bf16", 64, 8, 2, 64, [0, 33, 1000], [1, 31, 100], 0),
    ("bf16", 64, 3, 1, 32, [77, 640], [1, 1], 0),
    ("bf16", 64, 12, 12, 256, [300], [70], 64),
    ("bf16", 128, 64, 1, 64, [200, 70], [1, 6], 0),
    ("bf16", 128, 64, 2, 64, [200, 7000], [1, 1], 0),
    ("f32", 64, 4, 4, 32, [128], [60], 0),
    ("f32", 64, 8, 2, 64, [0, 1, 31, 500], [1, 1, 1, 1], 0),
    ("f32", 128, 8, 2, 64, [0, 65, 700], [40, 3, 130], 0),
    ("f32", 128, 8, 2, 64, [0, 65, 700], [40, 3, 130], 4),
    ("f32", 128, 4, 1, 32, [1500], [1], 0),
    ("f32", 128, 7, 7, 96, [95, 10], [33, 9], 0),
    ("bf16", 128, 8, 1, 32, [(37 * i) % 90 for i in range(70)], [(5 * i) % 21 for i in range(70)], 0),
    ("f32", 64, 4, 1, 32, [(29 * i) % 70 for i in range(130)], [1 + i % 2 for i in range(130)], 0),
    ("bf16", 64, 2, 1, 32, [10, 0], [1500, 700], 0),
]


@pytest.mark.parametrize("dtype,hd,hq,hkv,page,lens,rows,last", WEIGH)
def test_weights(dtype, hd, hq, hkv, page, lens, rows, last):
    dt = DT[dtype]
    c = Plain(dt, 2, hkv, hd, page, lens, rows, 11)
    q = queries(c.starts[-1], hq, hd, dt, 12)
    slots = max(l + r for l, r in zip(lens, rows)) + 5
    before = 3 * torch.rand((2, len(lens), hkv, slots), generator=gen(13))
    mass = before.cuda()
    assert B.paged_weigh(c.kv, 1, c.chunk, q, mass, last_rows=last) is mass
    got = mass.cpu()
    check_mass(c, 1, q, got, before, last)
    assert c.kv.device_status() == 0
    assert torch.equal(got[0], before[0])              # the other layer, and what lies behind the rows
    for b, (l, r) in enumerate(zip(lens, rows)):
        assert torch.equal(got[1, b, :, l + r if r else 0:], before[1, b, :, l + r if r else 0:])
    # planned for longer ones, out of place, the same bits
    c.kv.len_bound = 40000
    other = torch.full_like(mass, -5.0)
    B.paged_weigh(c.kv, 1, c.chunk, q, other, before=before.cuda(), last_rows=last)
    check_mass(c, 1, q, other.cpu(), before, last)
    again = torch.full_like(mass, -5.0)
    B.paged_weigh(c.kv, 1, c.chunk, q, again, before=before.cuda(), last_rows=last)
    assert torch.equal(other, again)


def test_weights_of_nothing_before():
    c = Plain(torch.bfloat16, 1, 2, 64, 32, [40], [1], 5)
    q = queries(1, 4, 64, torch.bfloat16, 6)
    mass = torch.full((1, 1, 2, 64), math.nan).cuda()
    scratch = torch.full((B.paged_weigh_scratch_bytes(c.kv, c.chunk, 4),), 255, dtype=torch.uint8, device="cuda")
    lib = B.load_library()
    assert lib.esp_paged_weigh(B._stream_ptr(), c.kv._ref, 0, c.chunk._ref, 4, q.data_ptr(), 256, 0.125, 0, None, mass.data_ptr(), 64, scratch.data_ptr(),
                               scratch.numel()) == 0
    check_mass(c, 0, q, mass.cpu(), torch.zeros(1, 1, 2, 64))
    assert torch.isnan(mass[..., 41:]).all()
    assert abs(float(mass[..., :41].sum()) - 4) < 1e-5


@pytest.mark.parametrize("n", [1, 30])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_tokens_that_are_not_finite(dtype, n, what):
    """K of the chunk's last row is no number: that row's scores make NaN of all that it sees, or give that token nothing; the other sequence is as it was."""
    dt = DT[dtype]
    c = Plain(dt, 1, 2, 64, 32, [70, 10], [n, n], 21)
    d = np.arange(64)
    s = 70 + n - 1
    at = torch.from_numpy(k_place(s % 32, d, 64)).cuda()
    c.kv.k[0, int(c.table[0, s // 32])].view(2, -1)[:, at] = what
    q = queries(2 * n, 8, 64, dt, 22).abs()            # (a score of one sign)
    before = torch.rand((1, 2, 2, 128), generator=gen(23))
    mass = before.cuda()
    B.paged_weigh(c.kv, 0, c.chunk, q, mass)
    got = mass.cpu()
    rest = Plain(dt, 1, 2, 64, 32, [70, 10], [n, n], 21)
    other = before.cuda()
    B.paged_weigh(rest.kv, 0, rest.chunk, q, other)
    assert torch.equal(got[0, 1], other.cpu()[0, 1])   # the other sequence
    if what == -math.inf:                              # (its features all count alike: a score of minus infinity or, mixed with zeros, NaN)
        assert torch.isfinite(got[0, 0, :, :s]).all() and (got[0, 0, :, s] == 0).all()
    else:
        assert torch.isnan(got[0, 0, :, :s + 1]).all()
    assert torch.equal(got[0, 0, :, s + 1:], before[0, 0, :, s + 1:])


@pytest.mark.parametrize("n", [1, 30])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_minus_infinity_among_scores_that_are_not_finite(dtype, n):
    """A row with a score of plus infinity makes NaN of all that it sees, tokens with a score of minus infinity among them; a row whose scores are all minus
    infinity gives nothing."""
    c = Plain(DT[dtype], 1, 2, 64, 32, [70, 40], [n, n], 25)
    d = np.arange(64)
    for s, what in ((5, math.inf), (9, -math.inf)):
        c.kv.k[0, int(c.table[0, 0])].view(2, -1)[:, torch.from_numpy(k_place(s, d, 64)).cuda()] = what
    for page in c.table[1, :(40 + n + 31) // 32].tolist():
        c.kv.k[0, page] = -math.inf
    q = queries(2 * n, 8, 64, DT[dtype], 26).abs()     # (a score of one sign)
    assert (q > 0).all()
    before = torch.rand((1, 2, 2, 128), generator=gen(27))
    mass = before.cuda()
    B.paged_weigh(c.kv, 0, c.chunk, q, mass)
    got = mass.cpu()
    assert torch.isnan(got[0, 0, :, :70 + n]).all() and torch.equal(got[0, 0, :, 70 + n:], before[0, 0, :, 70 + n:])
    assert torch.equal(got[0, 1, :, :40], before[0, 1, :, :40]) and (got[0, 1, :, 40:40 + n] == 0).all()
    assert torch.equal(got[0, 1, :, 40 + n:], before[0, 1, :, 40 + n:])


@pytest.mark.parametrize("hq", [4, 64])
def test_rows_that_do_not_see_a_bad_token_are_not_touched_by_it(hq):
    """A row whose scores are NaN makes NaN of what it sees, not of tokens behind it."""
    n = 40
    c = Plain(torch.bfloat16, 1, 2, 64, 32, [33], [n], 31)
    q = queries(n, hq, 64, torch.bfloat16, 32)
    q[7] = math.nan
    mass = torch.zeros((1, 1, 2, 96)).cuda()
    B.paged_weigh(c.kv, 0, c.chunk, q, mass)
    got = mass.cpu()[0, 0]
    assert torch.isnan(got[:, :33 + 8]).all() and torch.isfinite(got[:, 33 + 8:33 + n]).all() and (got[:, 33 + n:] == 0).all()
    assert (got[:, 33 + n - 1] > 0).all()


@pytest.mark.parametrize("rows", [1, 50])
def test_pages_outside_the_pool_are_not_seen(rows):
    c = Plain(torch.bfloat16, 1, 2, 128, 32, [200, 100], [rows, rows], 41)
    table = c.table.clone()
    table[0, 2], table[0, 4] = -1, c.pages
    c.kv.page_table.copy_(table)
    q = queries(2 * rows, 8, 128, torch.bfloat16, 42)
    before = torch.rand((1, 2, 2, 256), generator=gen(43))
    mass = before.cuda()
    B.paged_weigh(c.kv, 0, c.chunk, q, mass)
    got = mass.cpu()
    assert c.kv.device_status() == B.DEV_BAD_PAGE
    gone = torch.zeros(200 + rows, dtype=torch.bool)
    gone[64:96] = gone[128:160] = True
    assert torch.equal(got[0, 0, :, :200][:, gone[:200]], before[0, 0, :, :200][:, gone[:200]])
    # what is left: as if these tokens were not there
    G = 4
    seen = (torch.arange(200 + rows) <= (200 + torch.arange(rows))[:, None]) & ~gone
    for h in range(2):
        x = torch.einsum("rgd,td->rgt", q[:rows].cpu().double()[:, h * G:h * G + G], c.k[0][0, :, h].double()) * 128 ** -0.5
        p = torch.softmax(x.masked_fill(~seen[:, None], -math.inf), -1).sum((0, 1))
        p[:200] += before[0, 0, h, :200].double()
        assert ((got[0, 0, h, :200 + rows].double() - p).abs() <= 2e-5 * (1 + p))[~gone].all()


@pytest.mark.parametrize("rows", [1, 50])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sequences_that_share_pages(dtype, rows):
    """Three sequences begin with the same 64 tokens, on the same pages: weighed, then evicted to pages of their own; the shared ones stay as they are."""
    c = Plain(DT[dtype], 2, 2, 64, 32, [100, 90, 64], [rows] * 3, 45, keep=48)
    for b in (1, 2):
        c.table[b, :2] = c.table[0, :2]
        c.k[b][:, :64], c.v[b][:, :64] = c.k[0][:, :64], c.v[0][:, :64]
    c.kv.page_table.copy_(c.table)
    q = queries(3 * rows, 8, 64, DT[dtype], 46)
    before = torch.rand((2, 3, 2, 200), generator=gen(47))
    mass = before.cuda()
    for layer in range(2):
        B.paged_weigh(c.kv, layer, c.chunk, q, mass)
        check_mass(c, layer, q, mass.cpu(), before)
    c.lens = [n + rows for n in c.lens]
    c.kv.lens.copy_(i32(c.lens))
    c.kv.len_bound = max(c.lens)
    check_evict(c, mass.cpu(), 48, 4, 8, in_place=False)        # (all of the pools against what they were, but the new pages)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 7, 50])
def test_rows_that_see_nothing(dtype, rows):
    """Pages outside the pool: all of one sequence's, the first two of another's, whose first rows see nothing and whose later ones see what is behind, and none of a
    third's."""
    dt = DT[dtype]
    c = Plain(dt, 1, 2, 64, 32, [70, 20, 40], [rows] * 3, 48)
    table = c.table.clone()
    table[0], table[1, :2] = -1, c.pages
    c.kv.page_table.copy_(table)
    q = queries(3 * rows, 8, 64, dt, 49)
    before = torch.rand((1, 3, 2, 130), generator=gen(50))
    for bound in (70, 40000):                          # (as planned for their lengths and for long ones)
        c.kv.len_bound = bound
        mass = before.cuda()
        B.paged_weigh(c.kv, 0, c.chunk, q, mass)
        got = mass.cpu()
        assert c.kv.device_status() == B.DEV_BAD_PAGE
        assert torch.equal(got[0, 0, :, :70], before[0, 0, :, :70]) and (got[0, 0, :, 70:70 + rows] == 0).all()
        assert torch.equal(got[0, 1, :, :20], before[0, 1, :, :20]) and (got[0, 1, :, 20:min(64, 20 + rows)] == 0).all()
        for b, (l, gone) in enumerate(((70, 70 + rows), (20, 64), (40, 0))):
            assert torch.equal(got[0, b, :, l + rows:], before[0, b, :, l + rows:])
            if l + rows <= gone:
                continue
            # rows that see something, over what there is
            seen = (torch.arange(gone, l + rows) <= (l + torch.arange(rows))[:, None])
            some = seen.any(1)
            for h in range(2):
                rq = q[b * rows:(b + 1) * rows].cpu().double()[some, 4 * h:4 * h + 4]
                x = torch.einsum("rgd,td->rgt", rq, c.k[b][0, gone:, h].double()) * 0.125
                p = torch.softmax(x.masked_fill(~seen[some][:, None], -math.inf), -1).sum((0, 1))
                old = before[0, b, h, gone:l + rows].double()
                old[max(l - gone, 0):] = 0
                # a score: 64 products, below 64 2^-24 64; twice, and 8 roundings of it; the rest of it as above
                size = (rq.abs() @ c.k[b][0, gone:, h].double().abs().T * 0.125).amax()
                tol = 2 * U * 72 * float(size) + 2.0 ** -21 + ((l + rows) / 32 + 68) * U + (4 * rows + 8) * U
                assert ((got[0, b, h, gone:l + rows].double() - p - old).abs() <= tol * p + 10 * U * old + 1e-30).all(), (b, h)


def test_malformed_sequences_are_left_out():
    c = Plain(torch.bfloat16, 1, 2, 64, 32, [40, 50, 60, 70], [1, 1, 1, 1], 51)
    c.kv.lens.copy_(i32([-1, 50, 71, 70]))             # the bound is 70
    q = queries(4, 4, 64, torch.bfloat16, 52)
    before = torch.rand((1, 4, 2, 80), generator=gen(53))
    mass = before.cuda()
    B.paged_weigh(c.kv, 0, c.chunk, q, mass)
    assert c.kv.device_status() == B.DEV_LEN_OVER_BOUND
    got = mass.cpu()
    assert torch.equal(got[0, [0, 2]], before[0, [0, 2]])
    c.lens = [0, 50, 0, 70]
    c.rows = [0, 1, 0, 1]
    c.starts = [0, 1, 2, 3, 4]
    for b in (1, 3):
        want, tol = weights(c, 0, b, q, 0, 0.125)
        want[:, :c.lens[b]] += before[0, b, :, :c.lens[b]].double()
        assert ((got[0, b, :, :c.lens[b] + 1].double() - want).abs() <= tol + 9 * U * want.abs()).all()
    # masses too short for a sequence
    c = Plain(torch.bfloat16, 1, 2, 64, 32, [40, 50], [30, 30], 51)
    mass = torch.zeros((1, 2, 2, 75)).cuda()
    B.paged_weigh(c.kv, 0, c.chunk, queries(60, 4, 64, torch.bfloat16, 52), mass)
    assert c.kv.device_status() == B.DEV_LEN_OVER_BOUND and (mass[0, 1] == 0).all() and (mass[0, 0, :, :70] > 0).all()


@pytest.mark.parametrize("rows", [1, 20])
def test_captured_weights_follow_the_lengths(rows):
    c = Plain(torch.bfloat16, 1, 2, 128, 64, [500, 300], [rows, rows], 61)
    c.kv.len_bound = 500
    q = queries(2 * rows, 8, 128, torch.bfloat16, 62)
    mass = torch.zeros((1, 2, 2, 600)).cuda()
    scratch = torch.zeros(B.paged_weigh_scratch_bytes(c.kv, c.chunk, 8), dtype=torch.uint8, device="cuda")
    B.paged_weigh(c.kv, 0, c.chunk, q, mass, scratch=scratch)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.paged_weigh(c.kv, 0, c.chunk, q, mass, scratch=scratch)
    for lens in ([500, 300], [0, 299], [63, 64], [480, 1]):
        c.kv.lens.copy_(i32(lens))
        mass.fill_(0.25)
        scratch.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.full_like(mass, 0.25)
        B.paged_weigh(c.kv, 0, c.chunk, q, eager)
        assert torch.equal(mass, eager)
        assert abs(float(mass[0, 0, :, :lens[0] + rows].double().sum()) - 0.25 * 2 * lens[0] - 8 * rows) < 1e-3


# ---- eviction --------------------------------------------------------------------------------------------------

def chosen(mass, n, keep, first, recent):
    """Old slots of what stays of n tokens with these masses (numpy fp32), ascending."""
    if n <= keep:
        return np.arange(n)
    mid = np.arange(first, n - recent)
    x = np.where(np.isnan(mass[mid]), -np.inf, mass[mid].astype(np.float64))
    least = np.isnan(mass[mid])
    order = mid[np.lexsort((mid, least, -x))][:keep - first - recent]
    return np.sort(np.concatenate([np.arange(first), order, np.arange(n - recent, n)]))


def check_evict(c, mass, keep, first, recent, in_place, slots_out=None):
    """mass [layers, batch, hkv, slots] CPU."""
    k0, v0 = c.pools()
    m = mass.cuda()
    table = c.table.clone() if in_place else c.fresh
    kw = {}
    if not in_place:
        kw = dict(table_out=c.fresh.cuda(), mass_out=torch.full((*mass.shape[:3], slots_out or keep), -3.0).cuda(), len_out=i32([-4] * len(c.lens)))
    kept = B.paged_evict(c.kv, m, keep, first, recent, **kw)
    assert c.kv.device_status() == 0
    mass_out = (m if in_place else kw["mass_out"]).cpu()
    want_mass = mass.clone() if in_place else torch.full_like(mass_out, -3.0)
    lens = [min(n, keep) for n in c.lens]
    assert (c.kv.lens if in_place else kw["len_out"]).tolist() == lens
    if not in_place:
        assert c.kv.lens.tolist() == c.lens
    got = kept.cpu().numpy()
    for b, n in enumerate(c.lens):
        k, v = torch.empty((c.layers, lens[b], c.hkv, c.hd), dtype=c.dt), torch.empty((c.layers, lens[b], c.hkv, c.hd), dtype=c.dt)
        for layer in range(c.layers):
            for h in range(c.hkv):
                old = chosen(mass[layer, b, h].numpy(), n, keep, first, recent)
                assert got[layer, b, h].tolist() == old.tolist() + [-1] * (keep - len(old)), (layer, b, h)
                k[layer, :, h], v[layer, :, h] = c.k[b][layer, old, h], c.v[b][layer, old, h]
                want_mass[layer, b, h, :len(old)] = mass[layer, b, h, old]
        c.put(k0, v0, table[b], k, v, lens[b])
    k1, v1 = c.pools()
    assert same(k0, k1) and same(v0, v1)
    assert same(want_mass, mass_out)
    return kept


EVICT = [  # dtype, hd, hkv, page, layers, lens, keep, first, recent
    ("bf16", 128, 2, 32, 2, [100, 64, 65, 0, 1, 63], 64, 4, 8),
    ("bf16", 128, 8, 64, 3, [300, 10, 129], 128, 0, 0),
    ("bf16", 64, 1, 96, 2, [500, 96, 97, 95], 95, 1, 94),
    ("bf16", 64, 3, 32, 1, [40, 33], 1, 0, 0),
    ("bf16", 128, 1, 32, 1, [40, 33, 1], 1, 1, 0),
    ("bf16", 128, 1, 64, 2, [1500], 1499, 0, 3),
    ("bf16", 64, 2, 32, 1, [2500, 1025, 1024], 1024, 16, 100),
    ("f32", 64, 2, 64, 2, [200, 31, 77], 33, 2, 5),
    ("f32", 128, 4, 32, 1, [321, 65], 64, 0, 64),
    ("f32", 128, 1, 128, 3, [130, 500], 129, 128, 1),
    ("bf16", 128, 2, 32, 1, [(53 * i) % 200 for i in range(40)], 70, 3, 10),
    ("bf16", 64, 1, 128, 1, [20001, 7000], 6999, 5, 700),
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("dtype,hd,hkv,page,layers,lens,keep,first,recent", EVICT)
def test_evict(dtype, hd, hkv, page, layers, lens, keep, first, recent, in_place):
    c = Plain(DT[dtype], layers, hkv, hd, page, lens, [0] * len(lens), 71, room=(keep + page - 1) // page, keep=keep)
    mass = torch.randn((layers, len(lens), hkv, max(lens) + 3), generator=gen(72))
    if not in_place:
        mass = mass.clamp_min(0)                       # half of them equal
    check_evict(c, mass, keep, first, recent, in_place)


@pytest.mark.parametrize("what", ["equal", "two", "special", "steps"])
def test_masses_that_are_equal_or_not_finite(what):
    c = Plain(torch.bfloat16, 2, 2, 64, 32, [1200, 90], [0, 0], 81, keep=60)
    shape = (2, 2, 2, 1200)
    mass = {"equal": torch.full(shape, 0.5), "two": torch.randint(0, 2, shape, generator=gen(82)).float(),
            "special": torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1e-45, 3e38, -3e38])[torch.randint(0, 9, shape, generator=gen(83))],
            "steps": torch.randint(0, 40, shape, generator=gen(84)).float() * 1e-3 + 7}[what]
    if what == "special":
        mass[0, 0, 0] = math.nan
    check_evict(c, mass, 60, 4, 10, True)


def test_evict_keeps_whole_pages_where_they_are():
    """Blocks of which nothing goes are not moved, and a table may take some of its pages from the old one."""
    c = Plain(torch.bfloat16, 1, 2, 128, 32, [300], [0], 91, keep=128)
    mass = torch.arange(300, 0, -1).float().expand(1, 1, 2, 300).contiguous()        # the earliest stay
    table = torch.cat([c.table[:, :2], c.fresh[:, 2:]], 1)
    k0, v0 = c.pools()
    kept = B.paged_evict(c.kv, mass.cuda(), 128, table_out=table.cuda(), mass_out=torch.zeros((1, 1, 2, 128)).cuda())
    assert kept.cpu().tolist() == [[[list(range(128))] * 2]]
    c.put(k0, v0, table[0], c.k[0][:, :128], c.v[0][:, :128], 128)
    k1, v1 = c.pools()
    assert same(k0, k1) and same(v0, v1)


def test_evict_malformed_sequences_and_pages():
    c = Plain(torch.bfloat16, 1, 1, 64, 32, [100, 100, 100, 100, 100], [0] * 5, 95, keep=40)
    c.kv.lens.copy_(i32([-3, 101, 100, 100, 100]))
    table, fresh = c.table.clone(), c.fresh.clone()
    table[2, 1] = c.pages                              # old page of slots 32 .. 63 of sequence 2
    fresh[3, 1] = -1                                   # new page of slots 32 .. 39 of sequence 3
    c.kv.page_table.copy_(table)
    mass = torch.rand((1, 5, 1, 100), generator=gen(96))
    k0, v0 = c.pools()
    out, len_out = torch.zeros((1, 5, 1, 40)).cuda(), i32([7] * 5)
    kept = B.paged_evict(c.kv, mass.cuda(), 40, 0, 0, table_out=fresh.cuda(), mass_out=out, len_out=len_out).cpu()
    assert c.kv.device_status() == B.DEV_LEN_OVER_BOUND | B.DEV_BAD_PAGE
    assert len_out.tolist() == [-3, 101, 40, 40, 40]
    assert (kept[0, :2] == -1).all() and (out[0, :2] == 0).all()
    for b in (2, 3, 4):
        old = chosen(mass[0, b, 0].numpy(), 100, 40, 0, 0)
        assert kept[0, b, 0].tolist() == old.tolist()
        k, v = c.k[b][:, old].clone(), c.v[b][:, old].clone()
        if b == 2:
            k[:, (old >= 32) & (old < 64)] = 0
            v[:, (old >= 32) & (old < 64)] = 0
        c.put(k0, v0, fresh[b].clamp_min(0), k, v, 32 if b == 3 else 40)
    k1, v1 = c.pools()
    assert same(k0, k1) and same(v0, v1)


def test_captured_eviction_follows_the_lengths():
    keep, lens = 96, [200, 300]
    mass0 = torch.rand((2, 2, 2, 320), generator=gen(98))
    runs = []
    for captured in (False, True):
        c = Plain(torch.bfloat16, 2, 2, 128, 32, lens, [0, 0], 97)
        mass = mass0.cuda()
        pools = c.kv.k.clone(), c.kv.v.clone()
        kept = torch.zeros((2, 2, 2, keep), dtype=torch.int32, device="cuda")
        graph = torch.cuda.CUDAGraph()
        if captured:
            B.paged_evict(c.kv, mass, keep, 4, 16, kept=kept)
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                B.paged_evict(c.kv, mass, keep, 4, 16, kept=kept)
        for now in ([200, 300], [96, 97], [0, 299], [150, 95]):
            c.kv.k.copy_(pools[0])
            c.kv.v.copy_(pools[1])
            mass.copy_(mass0)
            c.kv.lens.copy_(i32(now))
            kept.fill_(5)
            graph.replay() if captured else B.paged_evict(c.kv, mass, keep, 4, 16, kept=kept)
            torch.cuda.synchronize()
            assert c.kv.lens.tolist() == [min(keep, n) for n in now]
            runs.append([t.clone() for t in (c.kv.k, c.kv.v, mass, kept)])
    for a, b in zip(runs[:4], runs[4:]):
        for x, y in zip(a, b):
            assert same(x.float(), y.float())


@pytest.mark.parametrize("rows", [1, 40])
def test_pools_behind_31_and_32_bits(rows):
    """A sequence whose pages and layer lie behind 2^31 and 2^32 elements of a pool does what the same does in a small one."""
    small = Plain(torch.bfloat16, 1, 8, 128, 64, [400, 90], [rows, rows], 111, keep=128)
    pages, layers = 50000, 2                           # 3.3e9 elements a layer
    shape = (layers, pages, 8, 64, 128)
    kv = B.PagedKv(torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(shape, dtype=torch.bfloat16, device="cuda"),
                   torch.zeros_like(small.kv.page_table), i32([400, 90]), 400)
    n = small.pages
    base = pages - n - 3
    kv.k[1, base:base + n] = small.kv.k[0]
    kv.v[1, base:base + n] = small.kv.v[0]
    kv.page_table.copy_(torch.where(small.table < n, small.table + base, small.table))
    q = queries(2 * rows, 32, 128, torch.bfloat16, 112)
    mass, far = torch.zeros((1, 2, 8, 500), device="cuda"), torch.zeros((2, 2, 8, 500), device="cuda")
    B.paged_weigh(small.kv, 0, small.chunk, q, mass)
    B.paged_weigh(kv, 1, small.chunk, q, far)
    assert torch.equal(mass[0], far[1]) and (far[0] == 0).all() and float(mass[0, 0, :, 400].min()) > 0
    far[0] = far[1]
    fresh = small.fresh.cuda()
    a = B.paged_evict(small.kv, mass, 128, 4, 16, table_out=fresh)
    b = B.paged_evict(kv, far, 128, 4, 16, table_out=(fresh + base).to(torch.int32))
    assert torch.equal(a[0], b[1]) and torch.equal(mass[0], far[1]) and kv.lens.tolist() == [128, 90]
    assert same(kv.k[1, base:base + n].float(), small.kv.k[0].float()) and same(kv.v[1, base:base + n].float(), small.kv.v[0].float())
    assert (kv.k[0, base:base + n] == 0).all() and (kv.k[1, :base] == 0).all() and (kv.v[1, base + n:] == 0).all()
    assert kv.device_status() == 0 and small.kv.device_status() == 0


def test_queries_that_lie_apart_and_at_any_place():
    """Rows of a projection, and rows whose addresses 16-byte loads cannot take."""
    for rows in (1, 40):
        c = Plain(torch.bfloat16, 1, 2, 128, 32, [70, 9], [rows, rows], 121)
        q = queries(2 * rows, 8, 128, torch.bfloat16, 122)
        want = torch.zeros((1, 2, 2, 128), device="cuda")
        B.paged_weigh(c.kv, 0, c.chunk, q, want)
        for off, pad in ((0, 256), (8, 8), (1, 0), (3, 5)):
            big = torch.full((2 * rows, off + 1024 + pad), math.nan, dtype=torch.bfloat16, device="cuda")
            big[:, off:off + 1024] = q.reshape(2 * rows, 1024)
            got = torch.zeros_like(want)
            B.paged_weigh(c.kv, 0, c.chunk, big[:, off:off + 1024].unflatten(1, (8, 128)), got)
            assert torch.equal(got, want)


def test_two_streams_with_a_workspace_each():
    c = Plain(torch.bfloat16, 1, 4, 128, 32, [900, 400, 30], [20, 20, 20], 131)
    q = queries(60, 16, 128, torch.bfloat16, 132)
    want = torch.zeros((1, 3, 4, 1000), device="cuda")
    B.paged_weigh(c.kv, 0, c.chunk, q, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(want) for _ in range(6)]
    scratch = [torch.empty(B.paged_weigh_scratch_bytes(c.kv, c.chunk, 16), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        with torch.cuda.stream(streams[i % 2]):
            B.paged_weigh(c.kv, 0, c.chunk, q, o, scratch=scratch[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


# ---- a run of them together ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_bounded_serving_loop(dtype):
    """Two sequences decode over a cache that holds 64 tokens of each: append, attention, weights, the next token, eviction.  The same loop on plain rows
    in 64 bits, with the GPU's own lists (checked against the GPU's own masses) says what attention, masses and tokens have to be."""
    dt, hkv, hq, hd, page, vocab, keep, first, recent = DT[dtype], 2, 8, 64, 32, 500, 64, 2, 16
    g = gen(101)
    emb = torch.randn((vocab, hq + 2 * hkv, hd), generator=g)                       # a token's q, k, v
    head = torch.randn((hq * hd, vocab), generator=g) * 0.1
    kv = B.PagedKv.zeros(1, 10, hkv, page, hd, 2, 5, dtype=dt)
    kv.page_table.copy_(torch.randperm(10, generator=g).reshape(2, 5).to(torch.int32))
    mass = torch.zeros((1, 2, hkv, 160), device="cuda")
    rope = B.rope_spec(hd)
    prompts = [torch.randint(0, vocab, (n,), generator=g) for n in (90, 20)]
    seen = [0, 0]                                       # tokens so far: positions
    rows_k = [torch.zeros((0, hkv, hd)), torch.zeros((0, hkv, hd))]                  # what the cache holds, per kv head
    rows_v = [torch.zeros((0, hkv, hd)), torch.zeros((0, hkv, hd))]
    tokens, lens, evictions = prompts, [0, 0], 0
    lim = [torch.tensor(x).cuda() for x in ([0.9, 0.0], [0.95, 1.0])]
    for step in range(40):
        rows = [len(t) for t in tokens]
        x = emb[torch.cat(tokens)].to(dt).cuda()
        starts = [0, rows[0], rows[0] + rows[1]]
        ch = B.ChunkRows(i32(starts), starts[-1], max(rows))
        pos = torch.cat([s + torch.arange(r) for s, r in zip(seen, rows)]).to(torch.int32).cuda()
        kv.len_bound = max(lens)
        q = B.paged_append(kv, 0, ch, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], rope=rope, positions=pos)
        _, k_rot = B.rope_qk(None, x[:, hq:hq + hkv].contiguous(), pos, rope)
        out = B.paged_attn(kv, 0, ch, q)
        old = mass.clone()
        B.paged_weigh(kv, 0, ch, q, mass)
        logits = torch.stack([out[starts[b + 1] - 1].float().reshape(-1) @ head.cuda() for b in range(2)])
        u = torch.rand(2, generator=g).cuda()
        ids, _ = B.sample(logits, u, temperature=lim[0], top_p=lim[1])
        for b in range(2):
            a, e, l, r = starts[b], starts[b + 1], lens[b], rows[b]
            rows_k[b] = torch.cat([rows_k[b], k_rot[a:e].cpu().float()])
            rows_v[b] = torch.cat([rows_v[b], x[a:e, hq + hkv:].cpu().float()])
            hidden = torch.arange(l + r) > (l + torch.arange(r))[:, None]
            s = torch.einsum("rhgd,thd->hgrt", q[a:e].cpu().double().view(r, hkv, hq // hkv, hd), rows_k[b].double()) * hd ** -0.5
            p = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
            o = torch.einsum("hgrt,thd->rhgd", p, rows_v[b].double()).reshape(r, hq, hd)
            tol = 2.0 ** -7 if dt == torch.bfloat16 else 1e-5       # p and the output rounded, and the size of V (up to 4) in sums of p = 1
            assert (out[a:e].cpu().double() - o).abs().max() <= 4 * tol
            want = p.sum((1, 2))
            want[:, :l] += old[0, b, :, :l].cpu().double()
            assert ((mass[0, b, :, :l + r].cpu().double() - want).abs() <= 2e-5 * (1 + want)).all()
            lens[b], seen[b] = l + r, seen[b] + r
        kv.lens.copy_(i32(lens))
        kv.len_bound = max(lens)
        m0 = mass.cpu()
        kept = B.paged_evict(kv, mass, keep, first, recent).cpu()
        assert kv.device_status() == 0
        for b in range(2):
            evictions += lens[b] > keep
            n = min(lens[b], keep)
            for h in range(hkv):
                old_slots = chosen(m0[0, b, h].numpy(), lens[b], keep, first, recent)
                assert kept[0, b, h, :n].tolist() == old_slots.tolist()
            rows_k[b] = torch.stack([rows_k[b][kept[0, b, h, :n].long(), h] for h in range(hkv)], 1)
            rows_v[b] = torch.stack([rows_v[b][kept[0, b, h, :n].long(), h] for h in range(hkv)], 1)
            lens[b] = n
            k, v = B.paged_load(kv, 0, b, 0, n)
            assert torch.equal(k.cpu().float(), rows_k[b]) and torch.equal(v.cpu().float(), rows_v[b])
        assert kv.lens.tolist() == lens
        assert int(ids[1]) == int(logits[1].argmax()) and 0 <= int(ids[0]) < vocab
        tokens = [ids[b:b + 1].cpu().long() for b in range(2)]
    assert evictions > 35


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_verified_tree_is_weighed(dtype):
    """Two sequences verify a tree each step: its rows appended, attention by ancestors, the accepted rows moved (new lengths to a tensor of their own), and these alone
    weighed, with the lengths of before; then eviction.  Masses against the accepted rows' softmax in 64 bits over what the cache holds."""
    dt, hkv, hq, hd, page, keep, first, recent = DT[dtype], 2, 8, 64, 32, 80, 2, 20
    g = gen(151)
    kv = B.PagedKv.zeros(1, 12, hkv, page, hd, 2, 6, dtype=dt)
    kv.page_table.copy_(torch.randperm(12, generator=g).reshape(2, 6).to(torch.int32))
    rope, lens, seen = B.rope_spec(hd), [0, 0], [0, 0]
    mass, after = torch.zeros((1, 2, hkv, 192), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    rows_k = [torch.zeros((0, hkv, hd)), torch.zeros((0, hkv, hd))]
    # parents of a tree's rows (-1: the root, row 0), and the paths that are accepted, by steps
    trees = [[-1, 0, 0, 1, 1, 2, 3, 5, 5, 6], [-1, 0, 1, 0, 3, 3, 2, 2, 4, 4, 8, 8, 10]]
    paths = [([0, 1, 3, 6, 9], [0, 3, 4, 8, 10, 12]), ([0], [0, 3, 5]), ([0, 2, 5, 8], [0]), ([0, 1, 4], [0, 1, 2, 7])]
    evictions = 0
    for step in range(9):
        rows = [60, 75] if step == 0 else [len(t) for t in trees]
        starts = [0, rows[0], sum(rows)]
        x = torch.randn((sum(rows), hq + 2 * hkv, hd), generator=g).to(dt).cuda()
        ch = B.ChunkRows(i32(starts), starts[-1], max(rows))
        kv.len_bound = max(lens)
        if step == 0:                                  # prompts
            depth, accepted, anc = [list(range(r)) for r in rows], [list(range(r)) for r in rows], None
        else:
            depth, accepted = [], list(paths[step % 4])
            anc = torch.zeros((sum(rows), 1), dtype=torch.int64)
            for b, t in enumerate(trees):
                depth.append([])
                for i, parent in enumerate(t):
                    depth[b].append(0 if parent < 0 else depth[b][parent] + 1)
                    anc[starts[b] + i, 0] = (0 if parent < 0 else int(anc[starts[b] + parent, 0])) | 1 << i
            anc = anc.cuda()
        pos = torch.cat([s + torch.tensor(d) for s, d in zip(seen, depth)]).to(torch.int32).cuda()
        q = B.paged_append(kv, 0, ch, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], rope=rope, positions=pos)
        _, k_rot = B.rope_qk(None, x[:, hq:hq + hkv].contiguous(), pos, rope)
        B.paged_attn(kv, 0, ch, q, anc=anc)
        if anc is None:
            after.copy_(kv.lens + i32(rows))
        else:
            B.paged_commit(kv, i32([len(p) for p in accepted]), i32([p + [0] * (B.MAX_MASKS + 1 - len(p)) for p in accepted]), after)
        assert after.tolist() == [n + len(p) for n, p in zip(lens, accepted)] and kv.lens.tolist() == lens
        took = [starts[b] + i for b in range(2) for i in accepted[b]]
        n = [len(p) for p in accepted]
        old = mass.cpu()
        B.paged_weigh(kv, 0, B.ChunkRows(i32([0, n[0], sum(n)]), sum(n), max(n)), q[took].contiguous(), mass)
        got = mass.cpu()
        for b in range(2):
            mine = [starts[b] + i for i in accepted[b]]
            rows_k[b] = torch.cat([rows_k[b], k_rot[mine].cpu().float()])
            l, r = lens[b], n[b]
            hidden = torch.arange(l + r) > (l + torch.arange(r))[:, None]
            rq = q[mine].cpu().double().view(r, hkv, hq // hkv, hd)
            s = torch.einsum("rhgd,thd->hgrt", rq, rows_k[b].double()) * hd ** -0.5
            want = torch.softmax(s.masked_fill(hidden, -math.inf), -1).sum((1, 2))
            was = old[0, b, :, :l + r].double()
            was[:, l:] = 0
            size = torch.einsum("rhgd,thd->hgrt", rq.abs(), rows_k[b].double().abs()).amax() * hd ** -0.5
            tol = 2 * U * (hd + 8) * float(size) + 2.0 ** -21 + ((l + r) / 32 + 68) * U + (4 * r + 8) * U
            assert ((got[0, b, :, :l + r].double() - want - was).abs() <= tol * want + 10 * U * was + 1e-30).all(), (step, b)
            assert torch.equal(got[0, b, :, l + r:], old[0, b, :, l + r:])
            lens[b], seen[b] = l + r, seen[b] + r
        kv.lens.copy_(after)
        kv.len_bound = max(lens)
        kept = B.paged_evict(kv, mass, keep, first, recent).cpu()
        assert kv.device_status() == 0
        for b in range(2):
            evictions += lens[b] > keep
            m = min(lens[b], keep)
            for h in range(hkv):
                assert kept[0, b, h, :m].tolist() == chosen(got[0, b, h].numpy(), lens[b], keep, first, recent).tolist()
            rows_k[b] = torch.stack([rows_k[b][kept[0, b, h, :m].long(), h] for h in range(hkv)], 1)
            lens[b] = m
            assert torch.equal(B.paged_load(kv, 0, b, 0, m)[0].cpu().float(), rows_k[b])
        assert kv.lens.tolist() == lens
    assert evictions == 2 + 6                          # lengths 60, 61, 65, 68, 73, 74, 78, 81, 80 + 5 and 75, 78, 79, 83, 80 + 6, + 3, + 1, + 4, + 6
