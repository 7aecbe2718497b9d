"""Host side of the paged KV cache's entry points: what they refuse before any GPU work, the frequencies of esp_rope_make, and
what the plans ask for as scratch.  No call here needs a GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_2603_17942_amd import binding as B

EINVAL, ESHAPE, ECAPACITY, EDTYPE = 1, 2, 3, 4
P = 4096          # an address that no call of this file reaches


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def paged(**kw):
    f = dict(k=P, v=P, page_table=P, len=P, status=None, dtype=B.ESP_BF16, n_layers=2, n_kv_heads=8, head_dim=128, page_size=64, n_pages=100,
             batch=2, table_stride=50, len_bound=1000)
    f.update(kw)
    return B.PagedKvStruct(*(f[n] for n, _ in B.PagedKvStruct._fields_))


def chunk(row0=P, total_rows=8, max_rows=8):
    return B.ChunkStruct(row0, total_rows, max_rows)


def rope(**kw):
    f = dict(head_dim=128, rot_dim=128, interleaved=0, theta=1e4, factor=1.0, orig_len=0, low=1.0, high=32.0, amplitude=1.0)
    f.update(kw)
    r = B.Rope()
    code = B.load_library().esp_rope_make(*(f[n] for n in ("head_dim", "rot_dim", "interleaved", "theta", "factor", "orig_len", "low", "high", "amplitude")),
                                          C.byref(r))
    return code, r


BAD_CACHE = [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(page_table=None), EINVAL), (dict(len=None), EINVAL), (dict(dtype=7), EDTYPE),
             (dict(n_layers=0), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(n_pages=0), EINVAL), (dict(batch=0), EINVAL), (dict(table_stride=0), EINVAL),
             (dict(len_bound=-1), EINVAL), (dict(head_dim=96), ESHAPE), (dict(page_size=16), ESHAPE), (dict(page_size=48), ESHAPE), (dict(page_size=0), EINVAL),
             (dict(k=P + 8), EINVAL), (dict(n_pages=2 ** 30), ECAPACITY), (dict(table_stride=2 ** 26), ECAPACITY)]


@pytest.mark.parametrize("change,code", BAD_CACHE)
def test_malformed_caches_are_refused_by_every_call(lib, change, code):
    kv, ch, (ok, r) = paged(**change), chunk(), rope()
    assert ok == 0
    kv, ch = C.byref(kv), C.byref(ch)
    assert lib.esp_paged_append(None, kv, 0, ch, C.byref(r), None, 32, P, 4096, P, 1024, P, 1024, None, None, 1e-6, P, 4096) == code
    assert lib.esp_paged_attn(None, kv, 0, ch, 32, P, 4096, 0.1, None, 0, P, P, 1 << 30) == code
    assert lib.esp_paged_attn_scratch_bytes(kv, ch, 32) == 0
    assert lib.esp_paged_commit(None, kv, P, P, P) == code
    assert lib.esp_paged_load(None, kv, 0, 0, 0, 1, P, P) == code


def test_attention_refusals(lib):
    kv = paged()

    def call(kv=kv, layer=0, ch=chunk(), nq=32, q=P, stride=4096, scale=0.1, anc=None, words=0, out=P, scratch=P, n=1 << 30):
        return lib.esp_paged_attn(None, C.byref(kv), layer, None if ch is None else C.byref(ch), nq, q, stride, scale, anc, words, out, scratch, n)
    assert call(layer=2) == EINVAL and call(layer=-1) == EINVAL
    assert call(ch=None) == EINVAL and call(ch=chunk(row0=None)) == EINVAL
    assert call(ch=chunk(total_rows=-1)) == EINVAL and call(ch=chunk(max_rows=-1)) == EINVAL
    assert call(q=None) == EINVAL and call(out=None) == EINVAL
    assert call(nq=12) == ESHAPE and call(nq=0) == EINVAL
    assert call(stride=4095) == ESHAPE
    for bad in (0.0, -1.0, math.inf, math.nan, 1e-30):
        assert call(scale=bad) == EINVAL
    assert call(anc=P, words=0) == ESHAPE and call(ch=chunk(max_rows=65), anc=P, words=1) == ESHAPE
    assert call(kv=paged(len_bound=2 ** 31 - 10)) == ECAPACITY
    assert call(ch=chunk(total_rows=0)) == 0 and call(ch=chunk(max_rows=0)) == 0     # nothing to do
    kv = paged(len_bound=3000)
    need = lib.esp_paged_attn_scratch_bytes(C.byref(kv), C.byref(chunk()), 32)
    assert need > 0                                                                     # 8 rows on 3000 keys: shares
    assert call(kv, scratch=None) == ECAPACITY and call(kv, n=need - 1) == ECAPACITY and call(kv, scratch=P + 4) == EINVAL


def test_append_and_rope_refusals(lib):
    kv, (_, r) = paged(), rope()

    def append(kv=kv, layer=0, ch=chunk(), rope=r, nq=32, q=P, qs=4096, k=P, ks=1024, v=P, vs=1024, eps=1e-6, qo=P, qos=4096):
        return lib.esp_paged_append(None, C.byref(kv), layer, C.byref(ch), None if rope is None else C.byref(rope), None, nq, q, qs, k, ks, v, vs, None,
                                    None, eps, qo, qos)
    assert append(layer=2) == EINVAL and append(k=None) == EINVAL and append(v=None) == EINVAL
    assert append(q=None) == EINVAL and append(qo=None) == EINVAL and append(nq=0) == EINVAL
    assert append(eps=-1.0) == EINVAL and append(eps=math.nan) == EINVAL
    assert append(qs=4095) == ESHAPE and append(ks=1023) == ESHAPE and append(vs=1023) == ESHAPE and append(qos=4095) == ESHAPE
    assert append(qs=8192) == EINVAL                                                    # in place with another stride
    assert append(kv=paged(head_dim=64)) == ESHAPE                                      # the rope's is 128
    bad = B.Rope(128, 24, 0, 1.0)
    assert append(rope=bad) == ESHAPE
    bad = B.Rope(128, 32, 0, math.nan)
    assert append(rope=bad) == EINVAL
    assert append(ch=chunk(total_rows=2 ** 30, max_rows=8)) == ECAPACITY
    assert append(ch=chunk(total_rows=0)) == 0

    def qk(dtype=B.ESP_BF16, rope=r, rows=4, nq=32, nk=8, q=P, qs=4096, k=P, ks=1024, pos=P, eps=0.0, qo=P, qos=4096, ko=P, kos=1024):
        return lib.esp_rope_qk(None, dtype, None if rope is None else C.byref(rope), rows, nq, nk, q, qs, k, ks, pos, None, None, eps, qo, qos, ko, kos)
    assert qk(dtype=3) == EDTYPE and qk(rope=None) == EINVAL and qk(rows=-1) == EINVAL and qk(pos=None) == EINVAL
    assert qk(q=None, k=None, qo=None, ko=None) == EINVAL and qk(q=None) == EINVAL and qk(ko=None) == EINVAL
    assert qk(nq=0) == EINVAL and qk(nk=0) == EINVAL and qk(eps=math.inf) == EINVAL
    assert qk(qs=4095) == ESHAPE and qk(kos=1023) == ESHAPE and qk(ks=2048) == EINVAL
    assert qk(rows=2 ** 27) == ECAPACITY
    assert qk(rows=0) == 0


def test_commit_and_load_refusals(lib):
    kv = C.byref(paged())
    assert lib.esp_paged_commit(None, kv, None, P, P) == EINVAL
    assert lib.esp_paged_commit(None, kv, P, None, P) == EINVAL
    assert lib.esp_paged_commit(None, kv, P, P, None) == EINVAL
    for layer, seq, slot, n, kp in ((2, 0, 0, 1, P), (0, 2, 0, 1, P), (0, -1, 0, 1, P), (0, 0, -1, 1, P), (0, 0, 0, -1, P), (0, 0, 0, 1, None)):
        assert lib.esp_paged_load(None, kv, layer, seq, slot, n, kp, P) == EINVAL
    assert lib.esp_paged_load(None, kv, 0, 0, 50 * 64 - 1, 2, P, P) == ECAPACITY
    assert lib.esp_paged_load(None, kv, 0, 0, 50 * 64, 0, P, P) == 0


def test_more_than_a_launch_can_have_is_refused(lib):
    """A launch counts threads in 32 bits: 2^24 - 1 workgroups of 256."""
    (_, r), many = rope(), 2 ** 26 - 3                                              # four rows a workgroup

    def qk(rows, nq=1):
        return lib.esp_rope_qk(None, B.ESP_BF16, C.byref(r), rows, nq, 0, P, nq * 128, None, 0, P, None, None, 1e-6, P, nq * 128, None, 0)
    assert qk(many) == ECAPACITY and qk(2 ** 24, 128) == ECAPACITY and qk(1, 2 ** 22) == ECAPACITY
    kv = paged(n_kv_heads=1)
    assert lib.esp_paged_append(None, C.byref(kv), 0, C.byref(chunk(total_rows=many)), None, None, 0, None, 0, P, 128, P, 128, None, None, 1e-6, None,
                                0) == ECAPACITY
    kv = paged(batch=65535, len_bound=0)                                             # 65535 x 8 items of a sequence and kv head, 64 each
    ch = chunk(total_rows=2 ** 28, max_rows=4096)
    assert lib.esp_paged_attn_scratch_bytes(C.byref(kv), C.byref(ch), 32) == 0
    assert lib.esp_paged_attn(None, C.byref(kv), 0, C.byref(ch), 32, P, 4096, 0.1, None, 0, P, P, 1 << 30) == ECAPACITY
    assert lib.esp_paged_commit(None, C.byref(paged(n_layers=40000, n_kv_heads=512)), P, P, P) == ECAPACITY


def test_rope_make_refusals():
    for kw, code in ((dict(head_dim=80), ESHAPE), (dict(rot_dim=8), ESHAPE), (dict(rot_dim=130), ESHAPE), (dict(rot_dim=144), ESHAPE), (dict(theta=0.0), EINVAL),
                     (dict(theta=math.inf), EINVAL), (dict(factor=0.0), EINVAL), (dict(factor=math.nan), EINVAL), (dict(orig_len=-1), EINVAL),
                     (dict(orig_len=10, low=2.0, high=2.0), EINVAL), (dict(amplitude=math.nan), EINVAL), (dict(amplitude=1e39), EINVAL)):
        assert rope(**kw)[0] == code, kw
    assert B.load_library().esp_rope_make(128, 128, 0, 1e4, 1.0, 0, 1.0, 32.0, 1.0, None) == EINVAL


def test_rope_make_refuses_what_gives_no_speeds():
    """theta and factor finite, but not the speeds that they make; nothing is written then."""
    for kw in (dict(theta=5e-324), dict(theta=1e-300, factor=1e-20), dict(factor=1e-320), dict(factor=1e-310, orig_len=4096, low=1.0, high=4.0),
               dict(orig_len=4096, low=-1e308, high=1e308), dict(theta=5e-324, orig_len=4096)):
        code, r = rope(**kw)
        assert code == EINVAL and r.head_dim == 0 and not any(r.turns), kw
    assert rope(theta=1e-300)[0] == 0 and rope(factor=1e-300)[0] == 0 and rope(theta=1e300)[0] == 0


@pytest.mark.parametrize("rot", [16, 64, 96, 128])
@pytest.mark.parametrize("factor,orig", [(1.0, 0), (4.0, 0), (8.0, 8192), (0.5, 4096)])
def test_rope_make_frequencies(rot, factor, orig):
    """Against the formula term by term; pow and four roundings of double: 1e-14."""
    code, r = rope(rot_dim=rot, theta=5e5, factor=factor, orig_len=orig, low=1.0, high=4.0, amplitude=1.25)
    assert code == 0 and (r.head_dim, r.rot_dim, r.interleaved, r.amplitude) == (128, rot, 0, 1.25)
    for i in range(rot // 2):
        f = 1.0 / (5e5 ** (2 * i / rot))
        keep = 0.0
        if orig:
            keep = (orig * f / (2 * math.pi) - 1.0) / 3.0
            keep = 0.0 if keep < 0 else 1.0 if keep > 1 else keep
        want = (keep * f + (1 - keep) * f / factor) / (2 * math.pi)
        assert abs(r.turns[i] - want) <= 1e-14 * want
    if factor == 1.0:                   # one turn of the first pair in 2 pi positions, whatever the scaling's other numbers
        assert abs(r.turns[0] * 2 * math.pi - 1) < 1e-15


def test_scratch_is_for_work_that_is_cut(lib):
    """Where every workgroup has whole items nothing is wanted; where work is cut, what it wants does not grow with the batch's rows
    beyond what all workgroups' pieces take, and a refused call wants nothing."""
    def need(batch, rows, max_rows, bound, nq=32, nkv=8, hd=128, dtype=B.ESP_BF16):
        kv, ch = paged(batch=batch, table_stride=30000, len_bound=bound, n_kv_heads=nkv, head_dim=hd, dtype=dtype), chunk(total_rows=rows, max_rows=max_rows)
        return lib.esp_paged_attn_scratch_bytes(C.byref(kv), C.byref(ch), nq)
    assert need(1, 1, 1, 40) == 0 and need(3, 9, 3, 0) == 0                   # a few keys
    assert need(1, 8192, 8192, 0) == 0                                          # enough items
    assert need(1, 1, 1, 2000) > 0 and need(1, 1, 1, 10 ** 6, 8, 1, 64) > 0
    assert need(1, 300, 300, 20000) > 0 and need(1, 300, 300, 20000, dtype=B.ESP_F32) > 0
    for hd in (64, 128):
        for rows in (1, 8, 33, 500):
            for bound in (0, 100, 5000, 10 ** 6):
                assert need(4, 4 * rows, rows, bound, hd=hd) <= 2 * 512 * (32 * (hd + 2) * 4 + 16) * (1 if rows <= 8 else 4) + 4096
    assert lib.esp_paged_attn_scratch_bytes(C.byref(paged()), C.byref(chunk()), 12) == 0


def test_python_checks_of_tensors():
    k = torch.zeros((1, 4, 2, 32, 64))
    table, lens = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    kv = B.PagedKv(k, k.clone(), table, lens, 0)
    rows = B.ChunkRows(torch.tensor([0, 2], dtype=torch.int32), 2, 2)
    x = torch.zeros((2, 2, 64))
    with pytest.raises(ValueError):
        B.PagedKv(k, k[:, :3], table, lens, 0)
    with pytest.raises(ValueError):
        B.PagedKv(k.half(), k.half(), table, lens, 0)
    with pytest.raises(ValueError):
        B.PagedKv(k, k.clone(), table.long(), lens, 0)
    with pytest.raises(ValueError):
        B.ChunkRows(torch.tensor([0, 2]), 2, 2)
    for bad in (x.bfloat16(), x[:, :1], x[:1], torch.zeros((2, 64, 2)).transpose(1, 2)):
        with pytest.raises(ValueError):
            B.paged_append(kv, 0, rows, None, bad, x)
        with pytest.raises(ValueError):
            B.paged_append(kv, 0, rows, None, x, bad)
    with pytest.raises(ValueError):
        B.paged_attn(kv, 0, B.ChunkRows(torch.tensor([0, 1, 2], dtype=torch.int32), 2, 2), x)
    with pytest.raises(ValueError):
        B.paged_attn(kv, 0, rows, x, out=torch.zeros((2, 4, 64)))
    with pytest.raises(ValueError):
        B.paged_attn(kv, 0, rows, x, anc=torch.zeros((2, 1), dtype=torch.int32))
    with pytest.raises(ValueError):
        B.rope_qk(None, None, lens, B.rope_spec(64))
    with pytest.raises(ValueError):
        B.rope_qk(x, x, torch.zeros(3, dtype=torch.int32), B.rope_spec(64))
    with pytest.raises(ValueError):
        B.rope_qk(x, None, torch.zeros(2, dtype=torch.int32), B.rope_spec(64), q_gain=torch.ones(32))
    with pytest.raises(ValueError):                # no CPU path
        B.rope_qk(x, None, torch.zeros(2, dtype=torch.int32), B.rope_spec(64))
    with pytest.raises(B.EspError):
        B.rope_spec(64, rot_dim=20)


def test_tensors_whose_addresses_are_held_cannot_be_replaced():
    k = torch.zeros((1, 4, 2, 32, 64))
    table, lens = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    kv, rows = B.PagedKv(k, k.clone(), table, lens, 0), B.ChunkRows(torch.tensor([0, 2], dtype=torch.int32), 2, 2)
    for name in ("k", "v", "page_table", "lens", "status", "dtype", "struct"):
        with pytest.raises(AttributeError):
            setattr(kv, name, getattr(kv, name).clone() if torch.is_tensor(getattr(kv, name)) else None)
    for name, value in (("row0", rows.row0.clone()), ("total_rows", 3), ("max_rows", 1)):
        with pytest.raises(AttributeError):
            setattr(rows, name, value)
    kv.len_bound = 40                     # the one that may be set, and what is changed in place is seen
    kv.lens[0] = 33
    assert kv.struct.len_bound == 40 and C.cast(kv.struct.len, C.POINTER(C.c_int32))[0] == 33
    assert kv.struct.len == lens.data_ptr() and rows.struct.row0 == rows.row0.data_ptr()


def test_bitsets_of_no_words_are_not_causal_attention():
    k = torch.zeros((1, 4, 2, 32, 64))
    kv = B.PagedKv(k, k.clone(), torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 0)
    rows, x = B.ChunkRows(torch.tensor([0, 2], dtype=torch.int32), 2, 2), torch.zeros((2, 2, 64))
    with pytest.raises(ValueError, match="anc"):
        B.paged_attn(kv, 0, rows, x, anc=torch.zeros((2, 0), dtype=torch.int64))
