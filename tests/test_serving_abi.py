"""Host side of sampling, attention weights and eviction: what the entry points refuse before any GPU work, scratch sizes, and the checks of the
Python functions.  No call here needs a GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_2603_17942_amd import binding as B
from test_paged_abi import BAD_CACHE, ECAPACITY, EDTYPE, EINVAL, ESHAPE, P, chunk, paged
from util import internal


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def test_sample_refusals(lib):
    def call(dtype=B.ESP_F32, logits=P, stride=100, rows=3, vocab=100, u=P, ids=P, scratch=P, n=1 << 30):
        return lib.esp_sample(None, dtype, logits, stride, rows, vocab, None, None, None, None, u, ids, None, scratch, n)
    assert call(logits=None) == EINVAL and call(u=None) == EINVAL and call(ids=None) == EINVAL
    assert call(rows=-1) == EINVAL and call(vocab=0) == EINVAL and call(vocab=-5) == EINVAL
    assert call(dtype=2) == EDTYPE and call(dtype=-1) == EDTYPE
    assert call(stride=99) == ESHAPE and call(stride=0) == ESHAPE
    assert call(vocab=2 ** 22 + 1, stride=2 ** 25) == ECAPACITY
    assert call(rows=0) == 0
    for rows, vocab in ((1, 1), (3, 4097), (64, 128256), (320, 151936), (2 ** 31 - 1, 2 ** 22)):
        need, lot = lib.esp_sample_scratch_bytes(rows, vocab), min(rows, 1024)
        parts = [lot * ((vocab + n - 1) // n) for n in (8192, 4096)]
        if vocab <= 4096:
            assert need == 16 * lot
        else:
            assert parts[0] * 9248 <= need - lot * (4096 * 8 + 28) <= parts[1] * 9248 + 16
        assert call(rows=rows, vocab=vocab, stride=vocab, n=need - 1) == ECAPACITY and call(rows=rows, vocab=vocab, stride=vocab, scratch=None) == ECAPACITY
        assert call(rows=rows, vocab=vocab, stride=vocab, scratch=P + 8, n=need) == EINVAL
    assert lib.esp_sample_scratch_bytes(0, 10) == 0 and lib.esp_sample_scratch_bytes(10, 0) == 0 and lib.esp_sample_scratch_bytes(1, 2 ** 22 + 1) == 0


@pytest.mark.parametrize("change,code", BAD_CACHE)
def test_malformed_caches_are_refused(lib, change, code):
    kv, ch = C.byref(paged(**change)), C.byref(chunk())
    assert lib.esp_paged_weigh(None, kv, 0, ch, 32, P, 4096, 0.1, 0, P, P, 4096, P, 1 << 40) == code
    assert lib.esp_paged_weigh_scratch_bytes(kv, ch, 32, 0) == 0
    assert lib.esp_paged_evict(None, kv, P, 4096, 100, 4, 8, P, 50, P, 4096, P, P) == code


def test_weigh_refusals(lib):
    def call(kv=paged(), layer=0, ch=chunk(), nq=32, q=P, stride=4096, scale=0.1, last=0, before=None, mass=P, slots=4096, scratch=P, n=1 << 40):
        return lib.esp_paged_weigh(None, C.byref(kv), layer, None if ch is None else C.byref(ch), nq, q, stride, scale, last, before, mass, slots, scratch, n)
    assert call(layer=2) == EINVAL and call(layer=-1) == EINVAL
    assert call(ch=None) == EINVAL and call(ch=chunk(row0=None)) == EINVAL
    assert call(ch=chunk(total_rows=-1)) == EINVAL and call(ch=chunk(max_rows=-1)) == EINVAL
    assert call(q=None) == EINVAL and call(mass=None) == EINVAL and call(slots=0) == EINVAL and call(last=-1) == EINVAL
    assert call(nq=12) == ESHAPE and call(nq=0) == EINVAL and call(stride=4095) == ESHAPE
    for bad in (0.0, -1.0, math.inf, math.nan, 1e-30):
        assert call(scale=bad) == EINVAL
    assert call(kv=paged(len_bound=2 ** 31 - 10)) == ECAPACITY
    assert call(ch=chunk(total_rows=0)) == 0 and call(ch=chunk(max_rows=0)) == 0
    for last in (0, 1):
        need = lib.esp_paged_weigh_scratch_bytes(C.byref(paged()), C.byref(chunk()), 32, last)
        assert need > 0
        assert call(last=last, scratch=None) == ECAPACITY and call(last=last, n=need - 1) == ECAPACITY and call(last=last, scratch=P + 8, n=need) == EINVAL
    assert call(kv=paged(n_kv_heads=70000, n_pages=10), nq=70000, stride=70000 * 128) == ECAPACITY
    assert call(ch=chunk(max_rows=2 ** 30 // 4 + 1, total_rows=2 ** 30)) == ECAPACITY
    assert call(kv=paged(batch=65535, n_kv_heads=512, n_layers=1, n_pages=10), nq=512, stride=512 * 128) == ECAPACITY


def test_weigh_scratch_is_what_its_arrays_take(lib):
    def need(batch, rows, max_rows, bound, last, nq=32, nkv=8, hd=128, dtype=B.ESP_BF16):
        kv, ch = paged(batch=batch, table_stride=30000, len_bound=bound, n_kv_heads=nkv, head_dim=hd, dtype=dtype), chunk(total_rows=rows, max_rows=max_rows)
        return lib.esp_paged_weigh_scratch_bytes(C.byref(kv), C.byref(ch), nq, last)
    # a decode step: a score of four queries a token, and little beside
    assert 32 * 8 * 16384 * 16 <= need(32, 32, 1, 16384, 0) <= 1.05 * 32 * 8 * 16416 * 16
    assert need(4, 8000, 4000, 100, 1) == need(4, 4, 1, 3999 + 100, 0)      # one counted row each, as many tokens
    assert need(1, 4096, 4096, 0, 64) < need(1, 4096, 4096, 0, 0)
    assert need(1, 10, 10, 100, 0) > 0 and need(1, 10, 10, 100, 0, nq=8, hd=64, dtype=B.ESP_F32) > 0
    assert need(1, 10, 10, 100, -1) == 0 and need(1, 10, 10, 100, 0, nq=12) == 0 and need(1, 0, 10, 100, 0) == 0


def test_evict_refusals(lib):
    def call(kv=paged(), mass=P, slots=4096, keep=100, first=4, recent=8, table=P + 64, stride=50, mass_out=P + 64, out_slots=4096, len_out=P, kept=P):
        return lib.esp_paged_evict(None, C.byref(kv), mass, slots, keep, first, recent, table, stride, mass_out, out_slots, len_out, kept)
    for name in ("mass", "table", "mass_out", "len_out", "kept"):
        assert call(**{name: None}) == EINVAL, name
    assert call(slots=0) == EINVAL and call(out_slots=0) == EINVAL and call(stride=0) == EINVAL
    assert call(keep=0) == EINVAL and call(keep=-1) == EINVAL and call(first=-1) == EINVAL and call(recent=-1) == EINVAL
    assert call(first=60, recent=41) == EINVAL and call(keep=2 ** 31 - 1, first=2 ** 31 - 1, recent=2 ** 31 - 1) == EINVAL
    assert call(mass_out=P, out_slots=4000) == EINVAL and call(table=P, stride=49) == EINVAL
    assert call(out_slots=99) == ECAPACITY and call(stride=1) == ECAPACITY and call(kv=paged(len_bound=2 ** 31 - 1)) == ECAPACITY
    assert call(kv=paged(batch=60000, n_layers=100)) == ECAPACITY


def test_python_checks_of_tensors():
    x, u = torch.zeros((3, 50)), torch.zeros(3)
    for bad in (x.half(), x[0], x.t()):
        with pytest.raises(ValueError):
            B.sample(bad, u)
    for kw in (dict(temperature=torch.zeros(2)), dict(temperature=u.double()), dict(top_k=u), dict(top_k=torch.zeros(3, dtype=torch.int64)), dict(top_p=u.half()),
               dict(min_p=torch.zeros((3, 1))), dict(scratch=torch.zeros(1000)), dict(ids=torch.zeros(3)), dict(probs=torch.zeros(3, dtype=torch.float64)), dict(temperature=torch.zeros(6)[::2])):
        with pytest.raises(ValueError):
            B.sample(x, u, **kw)
    with pytest.raises(ValueError):
        B.sample(x, torch.zeros(4))
    with pytest.raises(ValueError, match="no CPU fallback"):
        B.sample(x, u)
    k = torch.zeros((1, 4, 2, 32, 64))
    kv = B.PagedKv(k, k.clone(), torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 0)
    rows, q, mass = B.ChunkRows(torch.tensor([0, 2], dtype=torch.int32), 2, 2), torch.zeros((2, 2, 64)), torch.zeros((1, 1, 2, 64))
    for bad in (mass[0], mass.double(), torch.zeros((1, 1, 64, 2)).transpose(2, 3), torch.zeros((2, 1, 2, 64))):
        with pytest.raises(ValueError):
            B.paged_weigh(kv, 0, rows, q, bad)
        with pytest.raises(ValueError):
            B.paged_weigh(kv, 0, rows, q, mass, before=bad)
        with pytest.raises(ValueError):
            B.paged_evict(kv, bad, 8)
    with pytest.raises(ValueError):
        B.paged_weigh(kv, 0, rows, q, mass, before=torch.zeros((1, 1, 2, 32)))
    with pytest.raises(ValueError):
        B.paged_weigh(kv, 0, rows, q[:1], mass)
    with pytest.raises(ValueError):
        B.paged_weigh(kv, 0, rows, q, mass, scratch=torch.zeros(10))
    for kw in (dict(keep=0), dict(keep=8, table_out=torch.zeros(2, dtype=torch.int32)), dict(keep=8, table_out=torch.zeros((2, 2), dtype=torch.int32)),
               dict(keep=8, len_out=torch.zeros(2, dtype=torch.int32)), dict(keep=8, kept=torch.zeros((1, 1, 2, 9), dtype=torch.int32)),
               dict(keep=8, mass_out=mass.half())):
        with pytest.raises(ValueError):
            B.paged_evict(kv, mass, **kw)
    with pytest.raises(ValueError, match="no CPU fallback"):
        B.paged_evict(kv, mass, 8)


@pytest.mark.parametrize("vocab", [1, 4096, 4097, 32000, 128256, 2 ** 22])
def test_a_workspace_for_more_rows_is_enough_for_fewer(vocab):
    lib = B.load_library()
    need = [lib.esp_sample_scratch_bytes(n, vocab) for n in range(1, 2100)]
    assert all(a <= b for a, b in zip(need, need[1:]))
    assert need[-1] == need[1023]


def test_python_numbers_beyond_32_bits():
    k = torch.zeros((1, 4, 2, 32, 64))
    kv = B.PagedKv(k, k.clone(), torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 0)
    mass = torch.zeros((1, 1, 2, 64))
    for kw in (dict(keep=2 ** 32 + 8), dict(keep=8, first=2 ** 32), dict(keep=8, recent=2 ** 32 + 1), dict(keep=8, first=-2 ** 32), dict(keep=8, first=5, recent=4)):
        with pytest.raises(ValueError, match="keep: 1 or more wanted"):
            B.paged_evict(kv, mass, **kw)


class SampleLot(C.Structure):
    _fields_ = [("first", C.c_int64), ("rows", C.c_int)]


@pytest.mark.parametrize("rows", [0, 1, 1023, 1024, 1025, 2048, 2 ** 31 - 1025, 2 ** 31 - 1024, 2 ** 31 - 1023, 2 ** 31 - 2, 2 ** 31 - 1])
def test_lots_of_rows_end_where_the_rows_do(rows):
    """Also where the number behind the last lot is none of 32 bits."""
    lot = internal("sample_lot", C.c_int, C.c_int, restype=SampleLot)
    lots = (rows + 1023) // 1024
    for i in {0, 1, lots - 2, lots - 1, lots, lots + 1}:
        if i >= 0:
            got = lot(rows, i)
            assert got.rows == max(0, min(1024, rows - 1024 * i))
            assert got.first == min(1024 * i, rows)


@pytest.mark.parametrize("keep", [65, 2 ** 31 - 1])
def test_keeping_more_than_there_is_room_for_is_refused_before_anything_is_allocated(keep, monkeypatch):
    k = torch.zeros((1, 4, 2, 32, 64))
    kv = B.PagedKv(k, k.clone(), torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 0)
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: pytest.fail("allocated"))
    for slots, pages in ((64, 100), (200, 2)):
        with pytest.raises(B.EspError, match="ESP_ECAPACITY"):
            B.paged_evict(kv, torch.zeros((1, 1, 2, slots)), keep, table_out=torch.zeros((1, pages), dtype=torch.int32))
