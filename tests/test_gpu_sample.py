"""The choice of tokens from logits (sample) against its definition in 64 bits.

Whole numbers have to be equal.  The kernel's weights are off by 1.1e-12 of themselves (its polynomial; 3e-12 with the roundings) and by half of 2^-S, S = min(45, 62 - ceil
log2 vocab), where the largest weighs 1.  A sum of n of them is off by n times that at most, a border's place among all, W, by twice (3e-12 + n 2^-S-1 / W);
beside it 1e-13 for the reference's own sums.  Where the number u, or a limit, is nearer to a border than that, both sides of it are right and the row
says nothing; a test says how many such rows it may have.  probs: the quotient rounded to fp32, and those errors."""
import math

import numpy as np
import pytest
import torch

from util import ROOT  # noqa: F401

from paper_2603_17942_amd import binding as B

pytestmark = pytest.mark.gpu

def gen(seed):
    return torch.Generator().manual_seed(seed)


def choose(x, T, k, p, m, u):
    """(id, share, nearest border) of one row x (float64 numpy) by the definition."""
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, float(np.finfo(np.float32).max)))
    alive = np.flatnonzero(x > -np.inf)
    if len(alive) == 0 or not (0 <= T < math.inf) or math.isnan(p) or math.isnan(m):
        return -1, 0.0, math.inf
    order = alive[np.lexsort((alive, -x[alive]))]
    if T == 0:
        return int(order[0]), 1.0, math.inf
    w = np.exp((x[order] - x[order[0]]) / T)
    near = math.inf                                    # nearest border, in units of what it may be off by
    half_step = 2.0 ** -(min(45, 62 - math.ceil(math.log2(len(x)))) + 1)
    allowed = lambda n, total: 2 * (3e-12 + n * half_step / total) + 1e-13          # noqa: E731
    if k > 0:
        w = w[:k]
    if p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)])
        goal = max(p, 0.0) * before[-1]
        if goal > 0:
            near = min(near, np.abs(before[1:-1] - goal).min(initial=math.inf) / before[-1] / allowed(len(w), before[-1]))
        w = w[:max(1, int(np.count_nonzero(before[:-1] < goal)))]
    if m > 0:
        # (what weighs less than 1e-9 makes no difference that the other errors do not make)
        near = min(near, (np.abs(w - min(m, 1.0)) / (3e-12 * w + 2 * half_step))[(w < 1) & (w > 1e-9)].min(initial=math.inf))
        w = w[:max(1, int(np.count_nonzero(w >= min(m, 1.0))))]
    by_id = np.argsort(order[:len(w)])
    run, total = np.cumsum(w[by_id]), math.fsum(w)
    goal = min(max(u, 0.0), 1 - 2.0 ** -24) * total if u == u else 0.0
    at = min(int(np.count_nonzero(run <= goal)), len(w) - 1)
    if goal > 0:
        near = min(near, np.abs(run - goal).min() / total / allowed(len(w), total))
    return int(order[by_id[at]]), float(w[by_id[at]] / total), near


def dev(t):
    return None if t is None else t.cuda()


def check(x, u, T=None, k=None, p=None, m=None, silent=0):
    """x: CPU logits; returns ids.  silent: rows that may be too near a border."""
    ids, probs = B.sample(x.cuda(), u.cuda(), dev(T), dev(k), dev(p), dev(m))
    n, quiet = x.shape[0], 0
    for r in range(n):
        want, share, near = choose(x[r].double().numpy(), 1.0 if T is None else float(T[r]), 0 if k is None else int(k[r]), 1.0 if p is None else float(p[r]),
                                   0.0 if m is None else float(m[r]), float(u[r]))
        if near < 1:
            quiet += 1
            continue
        assert int(ids[r]) == want, (r, int(ids[r]), want, share)
        assert abs(float(probs[r]) - share) <= 2.0 ** -23 * share + 1e-9, (r, float(probs[r]), share)
    assert quiet <= silent
    again, _ = B.sample(x.cuda(), u.cuda(), dev(T), dev(k), dev(p), dev(m))
    assert torch.equal(ids, again)
    return ids


def limits(n, seed):
    """Every combination of limits, a greedy row in eight."""
    g = gen(seed)
    has = torch.arange(n) % 8
    T = torch.where(has == 0, 0.0, 0.3 + 1.2 * torch.rand(n, generator=g))
    k = torch.where((has & 1) == 1, torch.randint(1, 200, (n,), generator=g), 0).to(torch.int32)
    p = torch.where((has & 2) == 2, torch.rand(n, generator=g), 1.0)
    m = torch.where((has & 4) == 4, torch.rand(n, generator=g) ** 3, 0.0)
    return T, k, p, m


def logits(n, vocab, seed, spread=2.0, dtype=torch.float32):
    g = gen(seed)
    x = spread * torch.randn((n, vocab), generator=g)
    # some rows are sure of a few tokens
    for r in range(0, n, 2):
        at = torch.randint(0, vocab, (min(20, vocab),), generator=g)
        x[r, at] += 12 * torch.rand(len(at), generator=g)
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 3, 63, 64, 255, 257, 1000, 4096, 4097, 8197, 50001, 128256])
def test_every_combination_of_limits(vocab, dtype):
    n = 48 if vocab < 10000 else 24
    check(logits(n, vocab, vocab, dtype=dtype), torch.rand(n, generator=gen(vocab + 1)), *limits(n, vocab + 2))


@pytest.mark.parametrize("vocab", [151936, 200003])
def test_large_vocabularies_without_limits(vocab):
    check(logits(12, vocab, 5), torch.rand(12, generator=gen(6)))
    check(logits(12, vocab, 7, dtype=torch.bfloat16), torch.rand(12, generator=gen(8)), T=torch.full((12,), 0.7))


@pytest.mark.parametrize("spread", [1e-4, 1e-2, 0.3, 8.0, 60.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_flat_and_steep_rows(spread, dtype):
    """1e-4 and 1e-2: far more tokens in one step of the first division than LDS holds."""
    n, vocab = 16, 40000
    x = (spread * torch.randn((n, vocab), generator=gen(1))).to(dtype)
    T, k, p, m = limits(n, 2)
    k = torch.where(torch.arange(n) % 3 == 0, k * 150, k).to(torch.int32)
    check(x, torch.rand(n, generator=gen(3)), T, k, p, m, silent=1)
    check(x + 50.0, torch.rand(n, generator=gen(4)), T, k, p, m, silent=1)


@pytest.mark.parametrize("vocab", [7, 5000, 60000])
@pytest.mark.parametrize("values", [1, 2, 5, 70])
def test_equal_logits_go_by_id(vocab, values):
    n = 24
    g = gen(values)
    table = torch.randn(values, generator=g)
    x = table[torch.randint(0, values, (n, vocab), generator=g)]
    T, k, p, m = limits(n, 4)
    k[1], k[3] = 1, vocab // 2 + 1
    check(x, torch.rand(n, generator=g), T, k, p, m, silent=1)
    if values == 1:                                    # one value: the lowest ids, evenly
        k = torch.full((n,), min(vocab, 5), dtype=torch.int32)
        ids = check(x, (torch.arange(n) % 5 + 0.5) / 5, k=k)
        if vocab >= 5:
            assert ids.tolist() == [i % 5 for i in range(n)]
        p = torch.full((n,), 0.5)
        ids = check(torch.zeros((n, 64)), torch.full((n,), 0.99999), p=p, silent=n)
        assert ids.tolist() == [31] * n                # before the 33rd lies half of all, not less


def test_zeros_of_both_signs_are_equal():
    x = torch.full((2, 300), -0.0)
    x[0, 5], x[1, 200] = 0.0, 0.0
    assert B.sample(x.cuda(), torch.zeros(2).cuda(), temperature=torch.zeros(2).cuda())[0].tolist() == [0, 0]
    assert check(x, torch.full((2,), 0.99), k=torch.tensor([3, 3], dtype=torch.int32)).tolist() == [2, 2]


def test_masks_infinities_and_nan():
    vocab, low = 9000, float(torch.finfo(torch.float32).min)
    x = logits(12, vocab, 9)
    mask = torch.rand((12, vocab), generator=gen(10)) < 0.7
    x[0:3] = x[0:3].masked_fill(mask[0:3], -math.inf)
    x[3:5] = x[3:5].masked_fill(mask[3:5], low)
    x[5:7] = x[5:7].masked_fill(mask[5:7], math.nan)
    x[7] = -math.inf                                   # nothing left
    x[8] = math.nan
    x[9] = low                                         # all masked alike: all alike
    x[10, [17, 4000, 8999]] = math.inf
    x[11] = -math.inf
    x[11, 8998] = -3.0
    for T, k, p, m in ((None,) * 4, limits(12, 11), (torch.zeros(12), None, None, None), (None, torch.full((12,), 2, dtype=torch.int32), torch.full((12,), 0.9), None)):
        ids = check(x, torch.rand(12, generator=gen(12)), T, k, p, m)
        assert ids[7] == -1 and ids[8] == -1 and ids[11] == 8998 and int(ids[10]) in (17, 4000, 8999)
        assert all(not bool(mask[r, int(ids[r])]) for r in range(7))


def test_limits_at_their_ends():
    x = logits(8, 3000, 20)
    u = torch.rand(8, generator=gen(21))
    ones = torch.ones(8)
    for T in (1e-30, 1e-45, 1e-3, 100.0, 3e38):
        check(x, u, T=T * ones, silent=1)
    for k in (-5, 0, 1, 2999, 3000, 3001, 2 ** 31 - 1):
        check(x, u, k=torch.full((8,), k, dtype=torch.int32))
    for p in (-1.0, 0.0, 1e-30, 0.999999, 1.0, 7.0):
        check(x, u, p=p * ones, silent=1)
    for m in (-1.0, 0.0, 1e-30, 1e-12, 1.0, 7.0):
        check(x, u, m=m * ones)
    for v in (0.0, -1.0, 1.0, 2.0, math.nan, 1 - 2.0 ** -24, 1e-38):
        check(x, torch.full((8,), v))
        check(x, torch.full((8,), v), k=torch.full((8,), 40, dtype=torch.int32))
    for bad in (dict(T=-ones), dict(T=math.inf * ones), dict(T=math.nan * ones), dict(p=math.nan * ones), dict(m=math.nan * ones)):
        assert check(x, u, **bad).tolist() == [-1] * 8


def test_even_numbers_give_every_token_its_share():
    """u on a grid of n: the inverse of a distribution function, so a token of share s is chosen n s times, one more or less."""
    vocab, n = 37, 20000
    x = 1.5 * torch.randn((1, vocab), generator=gen(30))
    u = ((torch.arange(n) + 0.5) / n)
    ids, _ = B.sample(x.cuda().expand(n, vocab).contiguous(), u.cuda(), temperature=torch.full((n,), 0.8).cuda())
    share = torch.softmax(x[0].double() / 0.8, 0)
    got = torch.bincount(ids.cpu().long(), minlength=vocab).double()
    assert (got - n * share).abs().max() <= 1.0 + 1e-3


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off,pad", [(0, 0), (1, 3), (8, 8), (3, 5)])
def test_rows_that_lie_apart(off, pad, dtype):
    n, vocab = 9, 5003
    big = torch.full((n, off + vocab + pad), math.inf, dtype=dtype)          # what is around would be chosen
    big[:, off:off + vocab] = logits(n, vocab, 40, dtype=dtype)
    u, lim = torch.rand(n, generator=gen(41)), limits(n, 42)
    want = check(big[:, off:off + vocab].contiguous(), u, *lim)
    got, _ = B.sample(big.cuda()[:, off:off + vocab], u.cuda(), *(t.cuda() for t in lim))
    assert torch.equal(got, want)


def test_outputs_without_probs_and_no_rows():
    x, u = logits(5, 700, 50).cuda(), torch.rand(5, generator=gen(51)).cuda()
    ids, probs = torch.full((5,), -7, dtype=torch.int32).cuda(), torch.full((5,), -7.0).cuda()
    a, b = B.sample(x, u, ids=ids, probs=probs)
    assert a is ids and b is probs and (ids >= 0).all() and (probs > 0).all()
    scratch = torch.full((B.sample_scratch_bytes(5, 700),), 255, dtype=torch.uint8).cuda()
    lib, only = B.load_library(), torch.full((6,), -7, dtype=torch.int32).cuda()
    assert lib.esp_sample(B._stream_ptr(), B.ESP_F32, x.data_ptr(), 700, 5, 700, None, None, None, None, u.data_ptr(), only.data_ptr(), None, scratch.data_ptr(),
                          scratch.numel()) == 0
    assert torch.equal(only[:5], ids) and int(only[5]) == -7
    assert B.sample(x[:0], u[:0])[0].numel() == 0


def test_a_captured_call_follows_its_inputs():
    n, vocab = 6, 20000
    x, u = torch.empty((n, vocab)).cuda(), torch.empty(n).cuda()
    T, k, p, m = (torch.empty_like(t).cuda() for t in limits(n, 1))
    ids, probs = torch.empty(n, dtype=torch.int32).cuda(), torch.empty(n).cuda()
    B.sample(x.zero_(), u.zero_(), T.fill_(1), k.zero_(), p.fill_(1), m.zero_(), ids=ids, probs=probs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sample(x, u, T, k, p, m, ids=ids, probs=probs)
    for i in range(4):
        new = [logits(n, vocab, 60 + i), torch.rand(n, generator=gen(70 + i)), *limits(n, 80 + i)]
        for t, v in zip((x, u, T, k, p, m), new):
            t.copy_(v)
        ids.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        want = check(*new)
        assert torch.equal(ids, want)


def test_two_streams_at_once():
    n, vocab = 40, 60000
    x, u, lim = logits(n, vocab, 90).cuda(), torch.rand(n, generator=gen(91)).cuda(), [t.cuda() for t in limits(n, 92)]
    want = B.sample(x, u, *lim)[0]
    torch.cuda.synchronize()
    streams, out = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            out.append(B.sample(x, u, *lim)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in out)


def test_rows_behind_31_bits_of_elements():
    vocab, n = 131072, 16390                           # the last rows' first elements lie behind 2^31
    x = torch.zeros((n, vocab), dtype=torch.bfloat16, device="cuda")
    at = (torch.arange(n, device="cuda") * 7919) % vocab
    x[torch.arange(n, device="cuda"), at] = 30.0       # weight of all others: 1.2e-8
    ids, _ = B.sample(x, torch.full((n,), 0.5, device="cuda"))
    assert torch.equal(ids, at.int())


def test_more_rows_than_are_done_at_once_and_a_workspace_of_anything():
    n, vocab = 2100, 5003                              # three lots
    x, u, lim = logits(n, vocab, 110), torch.rand(n, generator=gen(111)), limits(n, 112)
    rows = torch.tensor([0, 1, 2, 3, 1022, 1023, 1024, 1025, 2047, 2048, 2049, 2097, 2098, 2099])
    want = check(x[rows], u[rows], *(t[rows] for t in lim))
    args = [x.cuda(), u.cuda(), *(t.cuda() for t in lim)]
    ids = B.sample(*args)[0]
    assert torch.equal(ids[rows.cuda()], want)
    scratch = torch.empty(B.sample_scratch_bytes(n, vocab), dtype=torch.uint8, device="cuda")
    for fill in (0, 255, 127):
        scratch.fill_(fill)
        assert torch.equal(B.sample(*args, scratch=scratch)[0], ids)


@pytest.mark.parametrize("vocab,k", [(30000, 5000), (30000, 29999), (140000, 20000), (140000, 3)])
def test_more_tokens_left_than_are_listed(vocab, k):
    n = 8
    x = logits(n, vocab, 120)
    u = torch.rand(n, generator=gen(121))
    ks = torch.full((n,), k, dtype=torch.int32)
    check(x, u, k=ks)
    check(x, u, k=ks, p=torch.full((n,), 0.97), T=torch.full((n,), 1.3))
    # (the rows that are sure of a few: at 0.9999 the sum's border lies among tokens that weigh some 1e-8 of W each, and it may be off
    # by 2 (3e-12 + 140000 2^-45 / W) = 8e-9 at W = 1: whatever the kernel does, up to these four say nothing)
    check(x, u, p=torch.full((n,), 0.9999), m=torch.full((n,), 1e-4), silent=4 if vocab == 140000 else 0)
    check(x.bfloat16(), u, k=ks, m=torch.full((n,), 1e-3))


def test_logits_far_from_zero():
    """Steps of log w are counted from zero: far from it logits are divided another way."""
    n, vocab = 6, 20000
    x = logits(n, vocab, 130)
    u, lim = torch.rand(n, generator=gen(131)), limits(n, 132)
    lim[0][0] = 0.9
    for shift in (300.0, -300.0, 4.0e4, -4.0e4, 1.0e6):         # (1e6: a sixteenth apart at least)
        check(x + shift, u, *lim)
    check(x * 1e6, u, lim[0] * 1e6, *lim[1:])
    check(x * 1e-30, u, lim[0] * 1e-10, *lim[1:])


def test_outputs_and_inputs_of_others_are_left_alone():
    n, vocab = 5, 6000
    x, u, lim = logits(n, vocab, 140).cuda(), torch.rand(n, generator=gen(141)).cuda(), [t.cuda() for t in limits(n, 142)]
    before = [t.clone() for t in (x, u, *lim)]
    ids, probs = torch.full((n + 2,), -7, dtype=torch.int32).cuda(), torch.full((n + 2,), -7.0).cuda()
    B.sample(x, u, *lim, ids=ids[1:-1], probs=probs[1:-1])
    assert ids[0] == -7 and ids[-1] == -7 and probs[0] == -7 and probs[-1] == -7 and (ids[1:-1] >= 0).all()
    assert all(torch.equal(a, b) for a, b in zip(before, (x, u, *lim)))


@pytest.mark.parametrize("value", [-1e-10, -1e-30, -2.0 ** -149, 0.0])
def test_a_part_of_equal_logits_a_little_below_zero(value):
    """8192 of them lie at the very end of their step."""
    n, vocab = 64, 140000
    x = torch.full((n, vocab), -math.inf)
    x[:, 8192:16384] = value
    x[:, 20000:23000] = -0.04 - 0.3 * torch.rand((n, 3000), generator=gen(150))
    x[:, 139999] = 0.0
    check(x, torch.rand(n, generator=gen(151)), p=torch.linspace(0.70, 0.99, n))
    check(x, torch.rand(n, generator=gen(152)), k=torch.linspace(8180, 8210, n).to(torch.int32))


@pytest.mark.parametrize("vocab", [5000, 2 ** 22])
def test_the_largest_top_p_below_one(vocab):
    """Weights that are none in integers and much more than 1 - top_p of all together are tokens that are not chosen."""
    for octaves in (42.5, 41.2, 47.0, 60.0):
        x = torch.full((2, vocab), -octaves * math.log(2))
        x[:, 1234] = 0.0
        x[:, 4321] = -1.0
        p, u = torch.full((2,), 1 - 2.0 ** -24), torch.tensor([0.5, 0.9])
        ids, probs = B.sample(x.cuda(), u.cuda(), top_p=p.cuda())
        share = 1 / (1 + math.exp(-1))
        assert ids.tolist() == [1234, 4321], octaves
        # 2^22 tokens of 2^-41.2 at most weigh 1.7e-6; fp32
        assert torch.allclose(probs.cpu(), torch.tensor([share, 1 - share]), rtol=0, atol=2e-6 + 2.0 ** -24)
        ids, _ = B.sample(x.cuda(), u.cuda(), top_p=p.cuda(), top_k=torch.full((2,), 4000, dtype=torch.int32).cuda(), min_p=torch.full((2,), 1e-12).cuda())
        assert ids.tolist() == [1234, 4321], octaves


@pytest.mark.parametrize("vocab", [262145, 300001, 1000003])
def test_more_parts_than_a_wave_has_lanes(vocab):
    x, u = logits(16, vocab, 160), torch.rand(16, generator=gen(161))
    # (a border may be off by 2 (3e-12 + 1000003 2^-43 / W), 2.3e-7 of a row whose W is 1: one of these rows has its top-p's border that near)
    check(x, u, *limits(16, 162), silent=int(vocab == 1000003))
    check(x[:4], u[:4])
    flat = logits(4, vocab, 163, spread=1e-3)[1::2]    # (all parts alike, and a row that cannot be narrowed down)
    for share in (0.0, 0.3, 0.7, 0.999):
        check(flat, torch.full((2,), share))
        check(flat, torch.full((2,), share), k=torch.tensor([vocab // 3, 7], dtype=torch.int32))


@pytest.mark.parametrize("rows", [1, 600])
@pytest.mark.parametrize("vocab,also", [(8192, None), (12288, 100)])
def test_tokens_of_less_than_half_a_unit_are_not_chosen(vocab, also, rows):
    """4096 tokens of 2^-50 of the largest, in a part without it (one row) and in a part with it (600 rows of 8192); `also`: among them one that counts.
    Their sum is 128 units, and none of them may be chosen, whatever the parts are."""
    x = torch.full((rows, vocab), -math.inf)
    x[:, :4096] = -50 * math.log(2)
    x[:, 5000] = 0.0
    if also is not None:
        x[:, also] = -20 * math.log(2)
    x = x.cuda()
    ones, zeros = torch.ones(rows).cuda(), torch.zeros(rows).cuda()
    want, share = (5000, 1 / (1 + 2.0 ** -20)) if also is None else (also, 2.0 ** -20)
    if also is None:
        share = 1.0
    for lim in ({}, dict(temperature=ones), dict(top_p=ones), dict(top_k=zeros.int()), dict(min_p=zeros), dict(min_p=1e-30 * ones)):
        ids, probs = B.sample(x, zeros, **lim)
        assert (ids == want).all(), (lim, ids[:4])
        # one rounding of the quotient; 128 units of 2^-45 that the part's sum has more of; the logit's rounding, 2^-24 of 13.9
        assert ((probs.double().cpu() - share).abs() <= share * (2.0 ** -23 + 14 * 2.0 ** -24) + 128 * 2.0 ** -45).all(), lim
        ids, _ = B.sample(x, torch.full((rows,), 0.5).cuda(), **lim)
        assert (ids == 5000).all(), lim


@pytest.mark.parametrize("rows", [1, 400])
def test_limits_do_not_leave_tokens_of_less_than_half_a_unit(rows):
    """6000 of 2^-46.6 and 2^-46.3 of the largest, where the steps of log w still reach: a min-p below them, a top-k among them."""
    vocab = 20000
    x = torch.full((rows, vocab), -math.inf)
    x[:, :3000] = -46.3 * math.log(2)
    x[:, 3000:4000] = -46.6 * math.log(2)
    x[:, 4096:6096] = -46.6 * math.log(2)
    x[:, 7000] = -20 * math.log(2)
    x[:, 19000] = 0.0
    x = x.cuda()
    for lim in (dict(min_p=torch.full((rows,), 1e-30)), dict(top_k=torch.full((rows,), 5500, dtype=torch.int32)),
                dict(top_k=torch.full((rows,), 5500, dtype=torch.int32), min_p=torch.full((rows,), 1e-20)), dict(top_p=torch.full((rows,), 1 - 2.0 ** -24))):      # (2^-24 of all is less than 2^-20)
        lim = {name: t.cuda() for name, t in lim.items()}
        ids, _ = B.sample(x, torch.zeros(rows).cuda(), **lim)
        assert (ids == 7000).all(), (lim, ids[:4])


def test_top_p_is_of_all_weights_however_the_cut_is_found():
    """The first token, the second one of e^-6.5 and 4 million of 0.9 half units, 1.7e-6 together: top_p lies between what the first one is of all and of the two
    alone, so the second one is in.  At 40000 the same logits, to the bit, are divided by going over the row."""
    vocab, faint = 2 ** 22, -7302 / 256
    second, rest = math.exp(-6.5), (vocab - 2) * math.exp(faint)
    assert math.exp(faint) < 2.0 ** -41 and 1.6e-6 < rest < 1.8e-6
    p = torch.full((1,), 0.5 / (1 + second) + 0.5 / (1 + second + rest), dtype=torch.float64).float()
    assert 1 / (1 + second + rest) + 5e-7 < float(p) < 1 / (1 + second) - 5e-7
    u = torch.full((1,), 0.9995)
    for shift in (0.0, 40000.0):
        x = torch.full((1, vocab), faint + shift)
        x[0, 100], x[0, 4000000] = shift, shift - 6.5
        assert float(x[0, 0]) == faint + shift
        ids, _ = B.sample(x.cuda(), u.cuda(), top_p=p.cuda())
        assert ids.tolist() == [4000000], shift


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [4095, 4097, 50257, 151643])
def test_one_row_of_an_odd_size_is_as_among_others(vocab, dtype):
    """By itself and at an aligned address it is read 16 bytes at a time, whatever its stride: what lies behind it would be chosen."""
    n = 8
    x, u, lim = logits(n, vocab, 170, dtype=dtype), torch.rand(n, generator=gen(171)), limits(n, 172)
    want = check(x, u, *lim)
    probs = B.sample(x.cuda(), u.cuda(), *(t.cuda() for t in lim))[1]
    for off in (0, 1):
        big = torch.full((vocab + off + 8,), math.inf, dtype=dtype, device="cuda")
        for r in range(n):
            big[off:off + vocab] = x[r].cuda()
            one = [t[r:r + 1].cuda() for t in (u, *lim)]
            got = B.sample(big[off:off + vocab].unsqueeze(0), one[0], *one[1:])
            assert int(got[0]) == int(want[r]) and float(got[1]) == float(probs[r]), (r, off)
