"""Refusals of the serving operators, through the C ABI: all are decided on the host before any CUDA call, so they need no GPU."""
import ctypes as C

import pytest

NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
P = 0x10000                                    # stands for a device pointer; nothing is launched


def _lib():
    from paper_2410_03804_b200 import moa
    return moa.load_library()


def _cache(**kw):
    from paper_2410_03804_b200 import moa
    f = dict(k=P, v=P, page_stride=16 * 8 * 128, page_table=P, len=P, weight=None, pos=None, seen=None, batch=2, max_pages=4, n_pages=9,
             page_size=16, hkv=8, head_dim=128, dtype=1)
    f.update(kw)
    return moa.MoaPagedCache(*(f[n] for n, _ in moa.MoaPagedCache._fields_))


BAD_CACHES = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(page_table=None), NULL), (dict(len=None), NULL), (dict(dtype=2), DTYPE),
              (dict(batch=0), SHAPE), (dict(batch=65), SHAPE), (dict(max_pages=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(hkv=0), SHAPE),
              (dict(head_dim=96), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=0), SHAPE), (dict(page_size=2048, page_stride=1 << 30), SHAPE),
              (dict(max_pages=1 << 28), SHAPE), (dict(page_stride=16 * 8 * 128 - 8), SHAPE), (dict(page_stride=16 * 8 * 128 + 4), ALIGN),
              (dict(k=P + 8), ALIGN), (dict(v=P + 2), ALIGN), (dict(pos=P), NULL), (dict(pos=P, weight=P), NULL), (dict(pos=P, seen=P), NULL)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(change, status):
    lib, c, n = _lib(), _cache(**change), C.c_size_t()
    assert lib.moa_paged_workspace_bytes(C.byref(c), 1, 8, 0, C.byref(n)) == status
    assert lib.moa_paged_append(C.byref(c), P, P, 1024, 1, None, None) == status
    assert lib.moa_paged_attention(C.byref(c), P, 4096, P, P, 1024, 1, 1, 32, None, 0.0, P, None, P, 1 << 40, None) == status
    assert lib.moa_paged_commit(C.byref(c), 1, None, None, 0, 1, None) == status
    assert lib.moa_paged_evict_workspace_bytes(C.byref(c), 8, C.byref(n)) == status
    assert lib.moa_paged_evict(C.byref(c), 8, 0, 0, P, P, None, P, 1 << 40, None) == status


def test_null_cache_and_sizes():
    lib, n = _lib(), C.c_size_t()
    assert lib.moa_paged_append(None, P, P, 1024, 1, None, None) == NULL
    assert lib.moa_paged_workspace_bytes(C.byref(_cache()), 1, 8, 0, None) == NULL
    assert lib.moa_paged_workspace_bytes(C.byref(_cache()), 0, 8, 0, C.byref(n)) == SHAPE
    assert lib.moa_paged_workspace_bytes(C.byref(_cache()), 65, 8, 0, C.byref(n)) == SHAPE
    assert lib.moa_paged_workspace_bytes(C.byref(_cache()), 1, 12, 0, C.byref(n)) == SHAPE
    assert lib.moa_paged_evict_workspace_bytes(C.byref(_cache()), 0, C.byref(n)) == SHAPE
    assert lib.moa_paged_evict_workspace_bytes(C.byref(_cache()), 20, C.byref(n)) == 0 and n.value >= 2 * 2 * 8 * 20 * 4


ATT = dict(q=P, q_stride=4096, k_new=P, v_new=P, new_stride=1024, n=1, n_new=1, hq=32, mask=None, scale=0.0, out=P, weight_out=None, ws=P,
           ws_bytes=1 << 40)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(ws=None), NULL), (dict(k_new=None), NULL), (dict(v_new=None), NULL),
    (dict(n=0, n_new=0), SHAPE), (dict(n=65, n_new=65), SHAPE), (dict(n=2, n_new=1), SHAPE), (dict(n_new=0), SHAPE), (dict(hq=12), SHAPE),
    (dict(hq=0), SHAPE), (dict(hq=8 * 129, q_stride=1 << 20), SHAPE), (dict(q_stride=4088), SHAPE), (dict(new_stride=1016), SHAPE),
    (dict(n=2, n_new=2, weight_out=P), SHAPE), (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(scale=2.5e38), SHAPE),
    (dict(q_stride=4100), ALIGN), (dict(new_stride=1028), ALIGN), (dict(q=P + 8), ALIGN), (dict(out=P + 8), ALIGN), (dict(ws=P + 4), ALIGN),
    (dict(k_new=P + 2), ALIGN)])
def test_attention_refuses(change, status):
    a = dict(ATT, **change)
    c = _cache()
    assert _lib().moa_paged_attention(C.byref(c), a["q"], a["q_stride"], a["k_new"], a["v_new"], a["new_stride"], a["n"], a["n_new"], a["hq"],
                                      a["mask"], a["scale"], a["out"], a["weight_out"], a["ws"], a["ws_bytes"], None) == status


def test_append_commit_and_evict_refuse():
    lib, c, t = _lib(), _cache(), _cache(weight=P, pos=P, seen=P)
    r = C.byref
    assert lib.moa_paged_append(r(c), None, P, 1024, 1, None, None) == NULL
    assert lib.moa_paged_append(r(c), P, P, 1024, 0, None, None) == SHAPE
    assert lib.moa_paged_append(r(c), P, P, 512, 1, None, None) == SHAPE
    assert lib.moa_paged_append(r(c), P + 8, P, 1024, 1, None, None) == ALIGN
    assert lib.moa_paged_append(r(c), P, P, 1028, 1, None, None) == ALIGN
    assert lib.moa_paged_commit(r(c), 0, None, None, 0, 1, None) == SHAPE
    assert lib.moa_paged_commit(r(c), 5, P, None, 7, 1, None) == NULL
    assert lib.moa_paged_commit(r(c), 65, P, P, 7, 1, None) == SHAPE
    assert lib.moa_paged_commit(r(c), 5, P, P, 0, 1, None) == SHAPE
    assert lib.moa_paged_evict(r(c), 8, 0, 0, P, P, None, P, 1 << 30, None) == NULL
    assert lib.moa_paged_evict(r(t), 0, 0, 0, P, P, None, P, 1 << 30, None) == SHAPE
    assert lib.moa_paged_evict(r(t), 8, -1, 0, P, P, None, P, 1 << 30, None) == SHAPE
    assert lib.moa_paged_evict(r(t), 8, 4, 5, P, P, None, P, 1 << 30, None) == SHAPE
    assert lib.moa_paged_evict(r(t), 8, 2, 2, None, P, None, P, 1 << 30, None) == NULL
    assert lib.moa_paged_evict(r(t), 8, 2, 2, P, P, None, None, 1 << 30, None) == NULL
    assert lib.moa_paged_evict(r(t), 8, 2, 2, P, P, None, P + 4, 1 << 30, None) == ALIGN


def test_rules_refuse():
    from paper_2410_03804_b200 import moa
    lib, r = _lib(), C.byref
    none = moa.MoaLogitRuleSet(*([None] * 8), 0)
    bias = moa.MoaLogitRuleSet(*([None] * 8), 3)
    many = moa.MoaLogitRuleSet(*([None] * 5), P, P, None, 1025)
    call = lambda s=none, tok=P, parent=P, b=1, n=4, x=P, dt=0, v=64, out=P, ch=P: lib.moa_logit_rules(  # noqa: E731
        r(s), tok, parent, b, n, x, dt, v, out, ch, None)
    assert lib.moa_logit_rules(None, P, P, 1, 4, P, 0, 64, P, P, None) == NULL
    assert call(x=None) == NULL and call(tok=None) == NULL and call(out=None, ch=None) == NULL and call(s=bias) == NULL
    assert call(b=0) == SHAPE and call(b=65) == SHAPE and call(n=0) == SHAPE and call(n=257) == SHAPE and call(v=0) == SHAPE
    assert call(v=(1 << 20) + 1) == SHAPE and call(s=many) == SHAPE and call(b=64, n=1025, tok=None, parent=None) == SHAPE
    assert call(dt=2) == DTYPE and call(x=P + 2) == ALIGN and call(dt=1, out=P + 1) == ALIGN
    full = lambda **k: lib.moa_verify_greedy_rules(r(none), k.get("tok", P), P, 1, 4, k.get("x", P), 1, 64, k.get("cap", 3), k.get("ch", P), P, P, P,  # noqa: E731
                                                   P, None)
    assert full(tok=None) == NULL and full(ch=None) == NULL and full(x=None) == NULL and full(cap=0) == SHAPE
    assert lib.moa_token_record(None, None, 1, 8, P, None, 4, None) == NULL
    assert lib.moa_token_record(P, P, 1, 8, None, None, 4, None) == NULL
    assert lib.moa_token_record(P, P, 65, 8, P, None, 4, None) == SHAPE
    assert lib.moa_token_record(P, P, 1, 0, P, None, 4, None) == SHAPE
    assert lib.moa_token_record(P, P, 1, 8, P, None, 0, None) == SHAPE
