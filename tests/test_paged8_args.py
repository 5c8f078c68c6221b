"""Refusals of the page plan, the norm and rotation, and the 8-bit cache, through the C ABI: decided on the host before any CUDA call, so
they need no GPU."""
import ctypes as C

import pytest

NULL, SHAPE, DTYPE, ALIGN = 1, 2, 3, 4
P = 0x10000                                    # stands for a device pointer; nothing is launched


def _moa():
    from paper_2410_03804_b200 import moa
    return moa


def _struct(cls, base, kw):
    f = dict(base)
    f.update(kw)
    return cls(*(f[n] for n, _ in cls._fields_))


POOL = dict(page_table=P, held=P, free_pages=P, free_count=P, batch=2, max_pages=4, n_pages=9, page_size=16)


def _pool(**kw):
    return _struct(_moa().MoaPagePool, POOL, kw)


PLAN = dict(len=P, n_new=P, seen=P, rows=P, row_start=P, row_seq=P, row_pos=P, slot=P, max_rows=10)


def _plan(pool, out=None, **kw):
    a = dict(PLAN)
    a.update(kw)
    return _moa().load_library().moa_page_plan(pool and C.byref(pool), out and C.byref(out), *a.values(), None)


@pytest.mark.parametrize("change,status", [
    (dict(page_table=None), NULL), (dict(held=None), NULL), (dict(free_pages=None), NULL), (dict(free_count=None), NULL), (dict(batch=0), SHAPE),
    (dict(batch=65), SHAPE), (dict(max_pages=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(page_size=0), SHAPE), (dict(page_size=24), SHAPE),
    (dict(page_size=2048), SHAPE), (dict(max_pages=1 << 27), SHAPE), (dict(n_pages=(1 << 28) + 1), SHAPE)])
def test_plan_refuses_a_bad_pool(change, status):
    assert _plan(_pool(**change)) == status


def test_plan_refuses_bad_arguments():
    assert _plan(None) == NULL
    for k in ("len", "rows", "row_start", "row_seq", "row_pos", "slot"):
        assert _plan(_pool(), **{k: None}) == NULL, k
    assert _plan(_pool(), max_rows=0) == SHAPE and _plan(_pool(), max_rows=-1) == SHAPE and _plan(_pool(), max_rows=(1 << 30) + 1) == SHAPE
    assert _plan(_pool(), slot=P + 4) == ALIGN
    assert _plan(_pool(), _pool(page_table=None)) == NULL
    assert _plan(_pool(), _pool(batch=3)) == SHAPE and _plan(_pool(), _pool(page_size=32)) == SHAPE
    assert _plan(_pool(), _pool(held=2 * P)) == SHAPE                  # some arrays of its own, some not


ARGS = dict(q=P, k=P, v=None, q_stride=4096, kv_stride=1024, q_gain=P, k_gain=P, pos=P, freq=P, q_out=P, q_out_stride=4096, k_out=P, k_out_stride=1024,
            cache=None, slot=None, rows=3, hq=32, hkv=8, head_dim=128, rot_dim=128, interleaved=0, dtype=1, eps=1e-5)
PAGED = dict(k=P, v=P, page_stride=16 * 8 * 128, page_table=P, len=P, weight=None, pos=None, seen=None, batch=2, max_pages=4, n_pages=9, page_size=16,
             hkv=8, head_dim=128, dtype=1)


def _norm(cache=None, **kw):
    moa = _moa()
    held = None
    if cache is not None:
        held = _struct(moa.MoaPagedCache, PAGED, cache)
        kw = dict(dict(k_out=None, v=P, slot=P), **kw, cache=C.addressof(held))
    a = _struct(moa.MoaQkNormRopeArgs, ARGS, kw)
    return moa.load_library().moa_qk_norm_rope(C.byref(a), None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(pos=None), NULL), (dict(q_out=None), NULL), (dict(k_out=None), NULL), (dict(q_gain=None), NULL),
    (dict(k_gain=None), NULL), (dict(freq=None), NULL), (dict(v=P), NULL), (dict(slot=P), NULL), (dict(dtype=2), DTYPE), (dict(rows=0), SHAPE),
    (dict(rows=(1 << 24) + 1), SHAPE), (dict(hq=0), SHAPE), (dict(hkv=0), SHAPE), (dict(hq=1025, q_stride=1 << 20, q_out_stride=1 << 20), SHAPE),
    (dict(head_dim=96), SHAPE), (dict(rot_dim=-16), SHAPE), (dict(rot_dim=144), SHAPE), (dict(rot_dim=24), SHAPE), (dict(eps=-1.0), SHAPE),
    (dict(eps=float("nan")), SHAPE), (dict(q_stride=4088), SHAPE), (dict(kv_stride=1016), SHAPE), (dict(q_out_stride=4088), SHAPE),
    (dict(k_out_stride=1016), SHAPE), (dict(q_stride=4100), ALIGN), (dict(kv_stride=1028), ALIGN), (dict(q_out_stride=4100), ALIGN),
    (dict(k_out_stride=1028), ALIGN), (dict(q=P + 8), ALIGN), (dict(k=P + 8), ALIGN), (dict(q_out=P + 2), ALIGN), (dict(k_out=P + 2), ALIGN),
    (dict(q_gain=P + 2), ALIGN), (dict(k_gain=P + 2), ALIGN)])
def test_norm_refuses(change, status):
    assert _norm(**change) == status


@pytest.mark.parametrize("cache,change,status", [
    (dict(k=None), {}, NULL), (dict(dtype=0, page_stride=16 * 8 * 128), {}, DTYPE), (dict(hkv=4), {}, SHAPE), (dict(head_dim=64), {}, SHAPE), ({}, dict(v=None), NULL),
    ({}, dict(slot=None), NULL), ({}, dict(k_out=P), NULL), ({}, dict(v=P + 4), ALIGN), ({}, dict(slot=P + 4), ALIGN)])
def test_norm_to_pages_refuses(cache, change, status):
    assert _norm(cache=cache, **change) == status


CACHE8 = dict(pages=P, page_stride=8 * 4112, k_ring=P, v_ring=P, page_table=P, len=P, seen=None, batch=2, max_pages=4, n_pages=9, page_size=16, hkv=8, head_dim=128)


def _cache8(**kw):
    return _struct(_moa().MoaPagedCache8, CACHE8, kw)


@pytest.mark.parametrize("change,status", [
    (dict(pages=None), NULL), (dict(k_ring=None), NULL), (dict(v_ring=None), NULL), (dict(page_table=None), NULL), (dict(len=None), NULL), (dict(batch=0), SHAPE),
    (dict(batch=65), SHAPE), (dict(max_pages=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(hkv=0), SHAPE), (dict(hkv=1025), SHAPE), (dict(head_dim=96), SHAPE),
    (dict(page_size=8), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=2048, page_stride=1 << 30), SHAPE), (dict(max_pages=1 << 27), SHAPE),
    (dict(page_stride=8 * 4112 - 16), SHAPE), (dict(page_stride=8 * 4112 + 8), ALIGN), (dict(pages=P + 8), ALIGN), (dict(k_ring=P + 8), ALIGN),
    (dict(v_ring=P + 2), ALIGN)])
def test_every_call_refuses_a_bad_cache8(change, status):
    lib, c, n = _moa().load_library(), _cache8(**change), C.c_size_t()
    assert lib.moa_paged8_workspace_bytes(C.byref(c), 1, 8, C.byref(n)) == status
    assert lib.moa_paged8_append(C.byref(c), P, P, 1024, 1, None, 1, None) == status
    assert lib.moa_paged8_attention(C.byref(c), P, 4096, P, P, 1024, 1, 1, 32, None, 0.0, P, P, 1 << 40, None) == status
    assert lib.moa_paged8_commit(C.byref(c), 1, None, None, 0, 1, None) == status
    assert lib.moa_paged8_read(C.byref(c), 1, None, None, P, P, 1, None) == status


ATT = dict(q=P, q_stride=4096, k_new=P, v_new=P, new_stride=1024, n=1, n_new=1, hq=32, mask=None, scale=0.0, out=P, ws=P, ws_bytes=1 << 40)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(ws=None), NULL), (dict(k_new=None), NULL), (dict(v_new=None), NULL), (dict(n=0, n_new=0), SHAPE),
    (dict(n=65, n_new=65), SHAPE), (dict(n=2, n_new=1), SHAPE), (dict(n_new=0), SHAPE), (dict(hq=12), SHAPE), (dict(hq=0), SHAPE),
    (dict(hq=8 * 129, q_stride=1 << 20), SHAPE), (dict(q_stride=4088), SHAPE), (dict(new_stride=1016), SHAPE), (dict(scale=-1.0), SHAPE),
    (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(scale=2.5e38), SHAPE), (dict(q=P + 8), ALIGN), (dict(out=P + 8), ALIGN),
    (dict(ws=P + 8), ALIGN), (dict(k_new=P + 8), ALIGN), (dict(v_new=P + 8), ALIGN), (dict(q_stride=4100), ALIGN), (dict(new_stride=1028), ALIGN)])
def test_attention8_refuses(change, status):
    a = dict(ATT)
    a.update(change)
    assert _moa().load_library().moa_paged8_attention(C.byref(_cache8()), *a.values(), None) == status


def test_the_other_calls_refuse():
    lib, c, n = _moa().load_library(), _cache8(), C.c_size_t()
    r = C.byref(c)
    assert lib.moa_paged8_workspace_bytes(r, 1, 8, None) == NULL
    assert [lib.moa_paged8_workspace_bytes(r, *a, C.byref(n)) for a in ((0, 8), (65, 8), (1, 12), (1, 8 * 129))] == [SHAPE] * 4
    assert lib.moa_paged8_append(r, None, P, 1024, 1, None, 1, None) == NULL and lib.moa_paged8_append(r, P, None, 1024, 1, None, 1, None) == NULL
    assert lib.moa_paged8_append(r, P, P, 1016, 1, None, 1, None) == SHAPE and lib.moa_paged8_append(r, P, P, 1024, 0, None, 1, None) == SHAPE
    assert lib.moa_paged8_append(r, P + 8, P, 1024, 1, None, 1, None) == ALIGN and lib.moa_paged8_append(r, P, P, 1028, 1, None, 1, None) == ALIGN
    assert lib.moa_paged8_commit(r, 1, P, None, 4, 1, None) == NULL and lib.moa_paged8_commit(r, 1, P, P, 0, 1, None) == SHAPE
    assert lib.moa_paged8_commit(r, 0, None, None, 0, 1, None) == SHAPE and lib.moa_paged8_commit(r, 65, None, None, 0, 1, None) == SHAPE
    assert lib.moa_paged8_read(r, 1, None, None, None, P, 1, None) == NULL and lib.moa_paged8_read(r, 1, None, None, P, None, 1, None) == NULL
    assert lib.moa_paged8_read(r, 0, None, None, P, P, 1, None) == SHAPE and lib.moa_paged8_read(r, 1, None, None, P, P, 2, None) == DTYPE
    assert lib.moa_paged8_read(r, 1, None, None, P + 8, P, 1, None) == ALIGN


def test_plan_refuses_outputs_over_inputs():
    """Decided by address: every array of the call a page of 64 KB apart, then one output moved into another array."""
    at = {n: P * (2 + i) for i, n in enumerate(("page_table", "held", "free_pages", "free_count", "len", "n_new", "seen", "rows", "row_start", "row_seq",
                                                "row_pos", "slot"))}
    pool = {n: at[n] for n in ("page_table", "held", "free_pages", "free_count")}
    other = {n: 32 * P + at[n] for n in pool}
    args = {n: at[n] for n in PLAN if n in at}
    outs = ("rows", "row_start", "row_seq", "row_pos", "slot")
    for second in (None, other):
        call = lambda p=pool, s=second, **kw: _plan(_pool(**p), s and _pool(**s), **dict(args, **kw))  # noqa: E731
        for o in outs:
            for name, there in {**args, **pool, **(second or {})}.items():
                if name != o and (o, name) != ("rows", "n_new"):
                    assert call(**{o: there}) == SHAPE, (o, name)
        # the end of one inside of the other: 2 sequences, 10 rows, 4 pages each
        assert call(rows=at["len"] + 4 - 8 + 4) == SHAPE and call(row_start=at["n_new"] + 4) == SHAPE and call(rows=at["n_new"] + 4) == SHAPE
        assert call(slot=at["row_pos"] + 32) == SHAPE and call(row_pos=at["slot"] + 76) == SHAPE and call(rows=at["page_table"] + 28) == SHAPE
        assert call(row_start=at["free_pages"] + 32) == SHAPE
    for n in pool:                                                   # a second pool that lies in the first one, or in an input
        assert _plan(_pool(**pool), _pool(**dict(other, **{n: pool["page_table"] + 16})), **args) == SHAPE
        assert _plan(_pool(**pool), _pool(**dict(other, **{n: at["seen"]})), **args) == SHAPE


def test_norm_refuses_outputs_over_other_rows():
    """bf16, 3 rows: q 32 heads and k 8 heads of 128. In place means the same rows; the parts of one projection may lie between each other."""
    q, k, qo, ko, row = P, 2 * P, 3 * P, 4 * P, 1024                  # bytes between k's rows: 2048
    base = dict(q=q, k=k, q_out=qo, k_out=ko)
    for change in (
            dict(q_out=q, q_out_stride=8192), dict(q_out=q, q_stride=8192),      # the same start, other rows behind it
            dict(k_out=k, k_out_stride=2 * row), dict(q_out=q + 16), dict(k_out=k + 2048), dict(k_out=k - 16), dict(q_out=q + 8192),
            dict(q_out=k), dict(k_out=q), dict(k_out=q + 3 * 8192 - 16), dict(q_out=ko), dict(k_out=qo), dict(rows=1, q_out=q + 16), dict(rows=1, k_out=qo + 64),
            # one projection of 48 heads per row (12288 bytes): results that reach into the next part, or into the next row's
            dict(k=q + 8192, q_stride=6144, kv_stride=6144, q_out=q + 4096, q_out_stride=6144),
            dict(k=q + 8192, q_stride=6144, kv_stride=6144, k_out=q + 8192 + 1024, k_out_stride=6144),
            dict(k=q + 8192, q_stride=6144, kv_stride=6144, k_out=q + 12288 - 16, k_out_stride=6144)):
        assert _norm(**dict(base, **change)) == SHAPE, change
    for change in (dict(q_out=k), dict(q_out=5 * P), dict(q_out=5 * P + 1024, q_out_stride=4096)):
        assert _norm(cache={}, q=q, k=k, v=5 * P, slot=6 * P, **change) == SHAPE, change
