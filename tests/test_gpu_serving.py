"""The serving operators on the GPU against plain definitions in 64 bits: paged attention with its append, commit and
accumulated weights, eviction, logit rules, and one cycle of all of them."""
import numpy as np
import pytest
import torch

from oracle import moa_oracle as O

pytestmark = pytest.mark.gpu

NAN = float("nan")
T = {"bf16": torch.bfloat16, "f32": torch.float32}


def _moa():
    from paper_2410_03804_b200 import moa
    return moa


def _cache(rng, dtype, lens, hkv, dh, page, extra, gap=False, track=False, spare=2):
    """A PagedCache whose committed slots hold random rows and whose every other byte is NaN. extra: slots behind len."""
    batch = len(lens)
    per = max(1, -(-(max(max(lens), 0) + extra) // page))
    total = batch * per + spare
    table = torch.from_numpy(rng.permutation(total)[:batch * per].astype(np.int32).reshape(batch, per)).cuda()
    shape = (total, page, hkv, dh)
    if gap:
        both = torch.full((total, 2) + shape[1:], NAN, dtype=T[dtype], device="cuda")
        k, v = both[:, 0], both[:, 1]
    else:
        k, v = (torch.full(shape, NAN, dtype=T[dtype], device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(int(rng.integers(1 << 30)))
    for b, L in enumerate(lens):
        for j0 in range(0, max(L, 0), page):
            m = min(page, L - j0)
            p = int(table[b, j0 // page])
            k[p, :m] = torch.randn((m, hkv, dh), generator=g).to(T[dtype]).cuda()
            v[p, :m] = torch.randn((m, hkv, dh), generator=g).to(T[dtype]).cuda()
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    w = p = seen = None
    if track:
        w = torch.rand((batch, hkv, per * page), generator=g).cuda() * 3
        p = torch.arange(per * page, dtype=torch.int32).expand(batch, hkv, per * page).contiguous().cuda()
        seen = torch.tensor([max(L, 0) + 5 for L in lens], dtype=torch.int32, device="cuda")
    return _moa().PagedCache(k, v, table, ln, w, p, seen)


def _slots(c, b, n):
    """Rows of slots 0 .. n-1 of sequence b in float64: (k, v) [n, hkv, dh]."""
    ps = c.k.shape[1]
    idx = torch.arange(n, device="cuda")
    page = c.page_table[b].long()[idx // ps]
    return c.k[page, idx % ps].double().cpu().numpy(), c.v[page, idx % ps].double().cpu().numpy()


def _attend(q, K, V, see, scale):
    """One head: q [dh], K, V [m, dh], see [m] -> (out, weights, sum of p |v|, largest sum of |q k|)."""
    idx = np.nonzero(see)[0]
    w = np.zeros(len(K))
    if len(idx) == 0:
        return np.zeros(K.shape[1]), w, np.zeros(K.shape[1]), 0.0
    z = K[idx] @ q * scale
    p = np.exp(z - z.max())
    p /= p.sum()
    w[idx] = p
    return p @ V[idx], w, p @ np.abs(V[idx]), float((np.abs(K[idx]) @ np.abs(q)).max() * scale)


def _bound(dtype, dh, keys, spread, mass, ref, once=False):
    """How far an output may be off: its own rounding (half a step), and relative to sum p |v|:
      scores    dh products summed in fp32, each sum off by at most 2^-23 of the running sum (the tensor cores may cut where
                an addition rounds): |error| <= dh * 2^-23 * sum |q k|, and 2^-23 of the scaled score; a score's error is a
                relative error of its p, once above and once below the fraction's line;
      exp       2^-21 per p, above and below;
      p         as two bf16 terms: 2^-16 (bf16 path; none in fp32). Several rows per sequence (`once`) may take the kernel that
                rounds each p once to bf16 for the product with v, its sum being taken before: each p is off by at most half
                a step, 2^-8 of itself, and so the output by at most 2^-8 * sum p |v|;
      sums      at most `keys` additions in fp32, above and below: 2 * keys * 2^-24 (products: 2^-23 each)."""
    score = (dh + 1) * 2.0**-23 * spread
    rel = 2 * score + 2 * 2.0**-21 + ((2.0**-8 if once else 2.0**-16) if dtype == "bf16" else 0.0) + 3 * keys * 2.0**-24
    half = 2.0**-8 if dtype == "bf16" else 2.0**-23
    return half * np.abs(ref) * (1 + rel) + rel * mass


def _check_attention(c, dtype, q, k_new, v_new, mask, out, lens, n_new, scale=None, weight_out=None, weight_in=None, before=None):
    """out [batch, n, hq, dh] (and weight_out) against the definition."""
    batch, n, hq, dh = q.shape
    hkv, cap = c.hkv, c.slots
    G = hq // hkv
    scale = dh ** -0.5 if scale is None else scale
    o, qd = out.double().cpu().numpy(), q.double().cpu().numpy()
    wo = None if weight_out is None else weight_out.double().cpu().numpy()
    for b, L in enumerate(lens):
        if L < 0:
            if before is not None:
                assert torch.equal(out[b], before[b])
            continue
        K, V = _slots(c, b, L)
        if n_new:
            K = np.concatenate([K, k_new[b].double().cpu().numpy()])
            V = np.concatenate([V, v_new[b].double().cpu().numpy()])
        for i in range(n):
            see = np.ones(len(K), bool)
            word = (2 << i) - 1 if mask is None else int(mask[b, i]) & (2**64 - 1)
            if n_new:
                see[L:] = [(word >> j) & 1 for j in range(n_new)]
            if word == 0:
                see[:] = False
            see &= np.arange(len(K)) < cap
            acc = np.zeros((hkv, len(K)))
            for h in range(hq):
                ref, w, mass, spread = _attend(qd[b, i, h], K[:, h // G], V[:, h // G], see, scale)
                tol = _bound(dtype, dh, len(K), spread, mass, ref, once=n > 1)
                assert np.all(np.abs(o[b, i, h] - ref) <= tol), (b, i, h, np.max(np.abs(o[b, i, h] - ref) - tol), np.abs(ref).max())
                acc[h // G] += w
            if wo is not None:
                m = min(len(K), cap)
                old = weight_in[b].double().cpu().numpy().copy()
                old[:, L:] = 0
                want = old[:, :m] + acc[:, :m]
                # each weight: the errors of p above; the sum over the group and the addition round in fp32
                rel = 2 * (dh + 1) * 2.0**-23 * 60 + 2.0**-20 + 3 * m * 2.0**-24 + (G + 1) * 2.0**-24
                assert np.all(np.abs(wo[b, :, :m] - want) <= rel * acc[:, :m] + 2.0**-23 * want + 1e-37)
                behind = weight_in[b, :, m:].cpu().numpy() if weight_out is c.weight else -7.0          # as they were
                assert np.all(wo[b, :, m:] == behind)


def _rows_of(rng, dtype, batch, n, hq, hkv, dh):
    g = torch.Generator().manual_seed(int(rng.integers(1 << 30)))
    qkv = torch.randn((batch, n, (hq + 2 * hkv) * dh), generator=g).to(T[dtype]).cuda()
    return (qkv[..., :hq * dh].unflatten(-1, (hq, dh)), qkv[..., hq * dh:(hq + hkv) * dh].unflatten(-1, (hkv, dh)),
            qkv[..., (hq + hkv) * dh:].unflatten(-1, (hkv, dh)))


TOKEN_CASES = [
    # dtype, dh, hq, hkv, page, gap, lens
    ("bf16", 128, 4, 1, 16, False, [0]),
    ("bf16", 128, 4, 2, 16, False, [1]),
    ("bf16", 128, 32, 8, 16, False, [0, 1, 15, 16, 17, 63, 64, 65, -1, 300]),
    ("bf16", 64, 8, 8, 8, True, [5, 1000, 0, 31, 32, 33]),
    ("bf16", 128, 16, 1, 1, False, [77, 3]),
    ("bf16", 64, 48, 2, 128, False, [700, 127, 128, 129]),
    ("bf16", 128, 8, 1, 64, True, [5003]),
    ("f32", 64, 4, 4, 16, False, [64, 0, 7, 8, 9]),
    ("f32", 128, 16, 2, 32, True, [513, -1, 31, 32, 33]),
    ("f32", 64, 20, 1, 4, False, [2500, 1]),
]


@pytest.mark.parametrize("dtype,dh,hq,hkv,page,gap,lens", TOKEN_CASES)
@pytest.mark.parametrize("weights", [False, True])
def test_token_attention(dtype, dh, hq, hkv, page, gap, lens, weights):
    """One row per sequence, appended by the call: uneven lengths, sequences without a slot or not in use, NaN in every slot
    that nobody may read, pages that end inside a tile."""
    moa, rng = _moa(), np.random.default_rng(len(lens) * 1000 + dh + hq)
    c = _cache(rng, dtype, lens, hkv, dh, page, 1, gap, track=weights)
    q, kn, vn = _rows_of(rng, dtype, len(lens), 1, hq, hkv, dh)
    k0, v0 = c.k.clone(), c.v.clone()
    out = torch.full((len(lens), 1, hq, dh), 5.0, dtype=T[dtype], device="cuda")
    before = out.clone()
    wo = torch.full_like(c.weight, -7.0) if weights else None
    pos0 = c.pos.clone() if weights else None
    w_in = c.weight.clone() if weights else None
    moa.moa_paged_attention(c, q, kn, vn, out=out, weight_out=wo)
    torch.cuda.synchronize()
    _check_attention(c, dtype, q, kn, vn, None, out, lens, 1, weight_out=wo, weight_in=w_in, before=before)
    for b, L in enumerate(lens):                # the new rows are in the pages, nothing else changed
        if L >= 0:
            p, r = int(c.page_table[b, L // page]), L % page
            assert torch.equal(c.k[p, r], kn[b, 0]) and torch.equal(c.v[p, r], vn[b, 0])
            k0[p, r], v0[p, r] = kn[b, 0], vn[b, 0]
            if weights:
                assert torch.all(c.pos[b, :, L] == L + 5) and torch.all(c.weight[b, :, L] == 0)
                pos0[b, :, L] = L + 5
    assert torch.equal(c.k.view(torch.uint8), k0.view(torch.uint8)) and torch.equal(c.v.view(torch.uint8), v0.view(torch.uint8))
    assert c.len.tolist() == lens and (not weights or torch.equal(c.pos, pos0))
    again = moa.moa_paged_attention(c, q, kn, vn, out=out.clone())
    assert torch.equal(again.view(torch.uint8), out.view(torch.uint8))          # the same bits again, with or without weights
    rows_there = moa.moa_paged_attention(c, q, out=before.clone())           # the rows are in the pages now
    assert torch.equal(rows_there.view(torch.uint8), out.view(torch.uint8))


def _word(bits):
    w = sum(1 << j for j, x in enumerate(bits) if x)
    return w - 2**64 if w >= 2**63 else w


def _trees(rng, batch, n, unused):
    """Random trees; the last `unused` slots of each are not in use. Returns parent [batch, n] and the packed words."""
    parent = np.full((batch, n), -1, np.int32)
    anc = np.zeros((batch, n, n), bool)
    for b in range(batch):
        for i in range(n - unused):
            if i:
                parent[b, i] = rng.integers(0, i)
                anc[b, i] = anc[b, parent[b, i]]
            anc[b, i, i] = True
    return parent, anc, torch.tensor([[_word(anc[b, i]) for i in range(n)] for b in range(batch)], dtype=torch.int64).cuda()


TREE_CASES = [
    # dtype, dh, hq, hkv, n, unused, page, lens
    ("bf16", 128, 8, 2, 61, 3, 16, [300, 0, 61, -1]),
    ("bf16", 128, 8, 1, 64, 0, 64, [129, 1]),
    ("bf16", 64, 4, 4, 7, 2, 8, [40, 64, 57]),
    ("bf16", 128, 16, 2, 17, 0, 32, [2500]),
    ("bf16", 128, 3, 1, 2, 1, 16, [15, 14]),
    ("bf16", 64, 16, 2, 63, 5, 16, [700, 130]),
    ("f32", 64, 4, 2, 13, 1, 16, [100, 0]),
    ("f32", 128, 4, 1, 33, 4, 16, [77]),
]


@pytest.mark.parametrize("dtype,dh,hq,hkv,n,unused,page,lens", TREE_CASES)
def test_tree_attention(dtype, dh, hq, hkv, n, unused, page, lens):
    """Rows of a kept tree under its packed mask: rows of unused slots see nothing and give zeros, whatever those slots hold."""
    moa, rng = _moa(), np.random.default_rng(n * 77 + dh)
    batch = len(lens)
    c = _cache(rng, dtype, lens, hkv, dh, page, n, track=False)
    q, kn, vn = _rows_of(rng, dtype, batch, n, hq, hkv, dh)
    if unused:
        kn[:, n - unused:], vn[:, n - unused:] = NAN, float("inf")
    parent, anc, mask = _trees(rng, batch, n, unused)
    words = moa.moa_tree_attn_mask(torch.from_numpy(parent).cuda(), packed=True)
    assert torch.equal(words.reshape(batch, n), mask)
    out = torch.full((batch, n, hq, dh), 5.0, dtype=T[dtype], device="cuda")
    before = out.clone()
    moa.moa_paged_attention(c, q, kn, vn, mask=words, out=out)
    torch.cuda.synchronize()
    _check_attention(c, dtype, q, kn, vn, mask.cpu().numpy(), out, lens, n, before=before)
    for b, L in enumerate(lens):
        for i in range(n - unused if L >= 0 else 0):
            p, r = int(c.page_table[b, (L + i) // page]), (L + i) % page
            assert torch.equal(c.k[p, r], kn[b, i]) and torch.equal(c.v[p, r], vn[b, i])


@pytest.mark.parametrize("dtype,dh,hq,hkv,n,unused,page,lens", [c for c in TREE_CASES if c[0] == "bf16"])
def test_tree_attention_in_a_large_cache(dtype, dh, hq, hkv, n, unused, page, lens):
    """The same rows in caches with room for many more positions, which take another kernel from 17 rows on."""
    moa, rng = _moa(), np.random.default_rng(n * 77 + dh + 1)
    batch = len(lens)
    tiles = -(-n * hq // hkv // 8)
    c = _cache(rng, dtype, lens, hkv, dh, page, n + 2**17 // (batch * hkv * tiles) + page)
    q, kn, vn = _rows_of(rng, dtype, batch, n, hq, hkv, dh)
    if unused:
        kn[:, n - unused:], vn[:, n - unused:] = NAN, float("inf")
    _, _, mask = _trees(rng, batch, n, unused)
    out = torch.full((batch, n, hq, dh), 5.0, dtype=T[dtype], device="cuda")
    before = out.clone()
    moa.moa_paged_attention(c, q, kn, vn, mask=mask, out=out)
    torch.cuda.synchronize()
    _check_attention(c, dtype, q, kn, vn, mask.cpu().numpy(), out, lens, n, before=before)
    for b, L in enumerate(lens):
        for i in range(n - unused if L >= 0 else 0):
            p, r = int(c.page_table[b, (L + i) // page]), (L + i) % page
            assert torch.equal(c.k[p, r], kn[b, i]) and torch.equal(c.v[p, r], vn[b, i])


def test_causal_rows_and_committed_only():
    """Without a mask the rows are causal; new_rows=False leaves the committed slots, and a sequence without any gives zeros."""
    moa, rng = _moa(), np.random.default_rng(3)
    for dtype in ("bf16", "f32"):
        lens, n, hq, hkv, dh = [70, 0, 33], 9, 6, 2, 64
        c = _cache(rng, dtype, lens, hkv, dh, 16, n)
        q, kn, vn = _rows_of(rng, dtype, 3, n, hq, hkv, dh)
        out = moa.moa_paged_attention(c, q, kn, vn, scale=0.3)
        _check_attention(c, dtype, q, kn, vn, None, out, lens, n, scale=float(np.float32(0.3)))
        out = moa.moa_paged_attention(c, q, new_rows=False)
        _check_attention(c, dtype, q, None, None, None, out, lens, 0)
        assert torch.all(out[1] == 0)


def test_append_in_place_weights_and_advance():
    """A prompt appended in ragged pieces, then ten tokens one by one with weights kept in the cache's own buffer: the same
    as attending over what was appended."""
    moa, rng = _moa(), np.random.default_rng(8)
    lens, hkv, hq, dh, page = [0, 0, -1, 0], 2, 8, 128, 16
    c = _cache(rng, "bf16", lens, hkv, dh, page, 200, track=True)
    c.seen.zero_()
    c.weight.fill_(9.0)
    q, kn, vn = _rows_of(rng, "bf16", 4, 90, hq, hkv, dh)
    n_new = torch.tensor([90, 17, 50, 0], dtype=torch.int32, device="cuda")
    moa.moa_paged_append(c, kn, vn, n_new)
    moa.moa_paged_commit(c, 90, acc_len=n_new)
    assert c.len.tolist() == [90, 17, -1, 0] and c.seen.tolist() == [90, 17, 0, 0]
    for b, m in ((0, 90), (1, 17)):
        K, V = _slots(c, b, m)
        assert np.array_equal(K, kn[b, :m].double().cpu().numpy()) and np.array_equal(V, vn[b, :m].double().cpu().numpy())
        assert c.pos[b, :, :m].tolist() == [list(range(m))] * hkv and torch.all(c.weight[b, :, :m] == 0)
        assert torch.all(c.weight[b, :, m:] == 9.0)
    total = [c.weight.clone().double().cpu().numpy() for _ in range(1)][0]
    for step in range(10):
        q, kn, vn = _rows_of(rng, "bf16", 4, 1, hq, hkv, dh)
        at = [90 + step, 17 + step, -1, step]
        w_in = c.weight.clone()
        out = moa.moa_paged_attention(c, q, kn, vn, weight_out=c.weight)
        torch.cuda.synchronize()
        _check_attention(c, "bf16", q, kn, vn, None, out, at, 1, weight_out=c.weight, weight_in=w_in)
        moa.moa_paged_commit(c, 1)
    assert c.len.tolist() == [100, 27, -1, 10] and c.seen.tolist() == [100, 27, 0, 10]
    # every token gave each key / value head the group's weight in all: 4 heads
    got = c.weight.double().cpu().numpy()
    for b, m in ((0, 100), (1, 27), (3, 10)):
        assert np.allclose(got[b, :, :m].sum(-1), 10 * (hq // hkv), rtol=1e-4)
    assert np.all(got[2] == total[2])


def test_commit_keeps_the_accepted_path():
    moa, rng = _moa(), np.random.default_rng(4)
    for dtype, dh in (("bf16", 128), ("f32", 128), ("f32", 64)):
        lens, n, hkv, page = [30, 0, 7, -1], 61, 3, 16
        c = _cache(rng, dtype, lens, hkv, dh, page, n, track=True)
        seen0 = c.seen.clone()
        _, kn, vn = _rows_of(rng, dtype, 4, n, hkv, hkv, dh)
        moa.moa_paged_append(c, kn, vn)
        path = torch.tensor([[0, 1, 5, 9, 60, -1, -1], [0, 1, 2, 3, 4, 5, 6], [0, -1, -1, -1, -1, -1, -1], [0, 7, 9, -1, -1, -1, -1]],
                            dtype=torch.int32, device="cuda")
        m = torch.tensor([5, 7, 1, 3], dtype=torch.int32, device="cuda")
        heads = [_slots(c, b, max(L, 0)) for b, L in enumerate(lens)]
        moa.moa_paged_commit(c, n, path, m, advance=False)
        assert c.len.tolist() == lens
        moa.moa_paged_commit(c, n, acc_len=m)
        assert c.len.tolist() == [35, 7, 8, -1] and c.seen.tolist() == [int(seen0[0]) + 5, int(seen0[1]) + 7, int(seen0[2]) + 1, int(seen0[3])]
        for b, L in enumerate(lens[:3]):
            K, V = _slots(c, b, L + int(m[b]))
            assert np.array_equal(K[:L], heads[b][0]) and np.array_equal(V[:L], heads[b][1])
            keep = path[b, :int(m[b])].long()
            assert np.array_equal(K[L:], kn[b, keep].double().cpu().numpy()) and np.array_equal(V[L:], vn[b, keep].double().cpu().numpy())


def test_pages_that_do_not_exist_and_a_full_cache():
    """Positions on a page outside the pool are left out; new rows behind the last slot are neither stored nor seen."""
    moa, rng = _moa(), np.random.default_rng(6)
    for dtype in ("bf16", "f32"):
        lens, hq, hkv, dh, page = [90, 64], 4, 2, 64, 16
        c = _cache(rng, dtype, lens, hkv, dh, page, 1, track=True)
        per = c.page_table.shape[1]
        table = c.page_table.clone()
        table[0, 1], table[0, 3] = -1, c.k.shape[0]
        c2 = moa.PagedCache(c.k, c.v, table, c.len)
        q, _, _ = _rows_of(rng, dtype, 2, 1, hq, hkv, dh)
        out = moa.moa_paged_attention(c2, q, new_rows=False)
        K, V = _slots(c, 0, 90)
        see = np.ones(90, bool)
        see[16:32] = see[48:64] = False
        for h in range(hq):
            ref, _, mass, spread = _attend(q[0, 0, h].double().cpu().numpy(), K[:, h // 2], V[:, h // 2], see, dh ** -0.5)
            assert np.all(np.abs(out[0, 0, h].double().cpu().numpy() - ref) <= _bound(dtype, dh, 90, spread, mass, ref))
        full = torch.tensor([per * page, per * page - 2], dtype=torch.int32, device="cuda")
        c.k[torch.isnan(c.k)] = 0.25
        c.v[torch.isnan(c.v)] = 0.5
        c3 = moa.PagedCache(c.k, c.v, c.page_table, full)
        q, kn, vn = _rows_of(rng, dtype, 2, 5, hq, hkv, dh)
        k0 = c.k.clone()
        out = moa.moa_paged_attention(c3, q, kn, vn)
        torch.cuda.synchronize()
        _check_attention(c3, dtype, q, kn, vn, None, out, full.tolist(), 5)
        last = int(c.page_table[1, per - 1])
        k0[last, page - 2:] = kn[1, :2]
        assert torch.equal(c.k, k0)
        moa.moa_paged_append(c3, kn, vn)
        assert torch.equal(c.k, k0)


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes and 2^31 elements per tensor: pages at its end are read and written there."""
    moa = _moa()
    hkv, dh, page = 8, 128, 1024
    n_pages = (2**31) // (page * hkv * dh) + 3
    k = torch.empty((n_pages, page, hkv, dh), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    table = torch.tensor([[n_pages - 1, 0], [n_pages - 2, 1]], dtype=torch.int32, device="cuda")
    for p in (0, 1, n_pages - 2, n_pages - 1):
        k[p].normal_()
        v[p].normal_()
    length = torch.tensor([1000, 1030], dtype=torch.int32, device="cuda")
    c = moa.PagedCache(k, v, table, length)
    rng = np.random.default_rng(2)
    q, kn, vn = _rows_of(rng, "bf16", 2, 1, 16, hkv, dh)
    out = moa.moa_paged_attention(c, q, kn, vn)
    torch.cuda.synchronize()
    _check_attention(c, "bf16", q, kn, vn, None, out, [1000, 1030], 1)
    assert torch.equal(k[n_pages - 1, 1000], kn[0, 0]) and torch.equal(k[1, 6], kn[1, 0])


def test_attention_on_another_stream_and_replayed():
    """A captured call follows the lengths and rows of each replay; a second graph has a workspace of its own."""
    moa, rng = _moa(), np.random.default_rng(12)
    lens, hq, hkv, dh = [40, 200], 16, 4, 128
    c = _cache(rng, "bf16", lens, hkv, dh, 16, 400, track=True)
    c.k[torch.isnan(c.k)] = 0.25
    c.v[torch.isnan(c.v)] = 0.5
    q, kn, vn = _rows_of(rng, "bf16", 2, 1, hq, hkv, dh)
    side = torch.cuda.Stream()
    out = torch.zeros((2, 1, hq, dh), dtype=torch.bfloat16, device="cuda")
    wo = torch.zeros_like(c.weight)
    ws = c.workspace(1, hq, True)
    torch.cuda.synchronize()
    moa.moa_paged_attention(c, q, kn, vn, out=out, weight_out=wo, ws=ws, stream=side)
    side.synchronize()
    first = out.clone()
    _check_attention(c, "bf16", q, kn, vn, None, out, lens, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moa.moa_paged_attention(c, q, kn, vn, out=out, weight_out=wo, ws=ws)
        moa.moa_paged_commit(c, 1)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first) and c.len.tolist() == [41, 201]
    for step in range(2):
        q2, kn2, vn2 = _rows_of(rng, "bf16", 2, 1, hq, hkv, dh)
        q.copy_(q2); kn.copy_(kn2); vn.copy_(vn2)
        at = c.len.tolist()
        graph.replay()
        torch.cuda.synchronize()
        _check_attention(c, "bf16", q, kn, vn, None, out, at, 1)
    c.len.copy_(torch.tensor([-1, 350], dtype=torch.int32))
    out.fill_(3.0)
    before = out.clone()
    graph.replay()
    torch.cuda.synchronize()
    _check_attention(c, "bf16", q, kn, vn, None, out, [-1, 350], 1, before=before)
    assert c.len.tolist() == [-1, 351]


STEEP_CASES = [
    # dtype, dh, hq, hkv, n, page, len
    ("bf16", 128, 16, 2, 1, 16, 1500),
    ("f32", 64, 4, 2, 1, 8, 700),
    ("bf16", 128, 16, 2, 40, 16, 1700),
    ("bf16", 64, 32, 1, 52, 128, 1001),
]


@pytest.mark.parametrize("dtype,dh,hq,hkv,n,page,L", STEEP_CASES)
@pytest.mark.parametrize("shape", ["rising", "falling", "peaks"])
def test_scores_far_apart(dtype, dh, hq, hkv, n, page, L, shape):
    """Scores that climb by hundreds over the positions, fall, or stand out at single ones: the running maximum moves often,
    by more than one factor of 2^8 at a time, or never again."""
    moa, rng = _moa(), np.random.default_rng(L + n)
    c = _cache(rng, dtype, [L], hkv, dh, page, n)
    u = torch.from_numpy(rng.choice([-1.0, 1.0], dh)).to(T[dtype]).cuda()              # the direction that queries share
    j = torch.arange(L, dtype=torch.float64)
    a = {"rising": 30 * j / L, "falling": 30 - 30 * j / L, "peaks": torch.where(j % 131 == 77, 25.0 + j / L, 0.0)}[shape]
    for x in range(0, L, page):
        p, m = int(c.page_table[0, x // page]), min(page, L - x)
        c.k[p, :m] += (a[x:x + m, None, None].cuda() * u.double()).to(T[dtype])
    q, kn, vn = _rows_of(rng, dtype, 1, n, hq, hkv, dh)
    q += u
    _, anc, mask = _trees(rng, 1, n, 0)
    out = moa.moa_paged_attention(c, q, kn, vn, mask=mask)
    torch.cuda.synchronize()
    _check_attention(c, dtype, q, kn, vn, mask.cpu().numpy(), out, [L], n)


@pytest.mark.parametrize("page,hq,n", [(8, 128, 64), (128, 64, 21), (256, 32, 21), (1024, 16, 21)])
def test_tree_rows_on_missing_pages_and_at_the_end_of_the_cache(page, hq, n):
    """Rows of several tokens: pages that the table does not have are left out, new rows behind the last slot are neither
    stored nor seen, unused slots in a causal batch of uneven lengths."""
    moa, rng = _moa(), np.random.default_rng(page)
    hkv, dh = 2, 128
    lens = [3 * page + 5, 2 * page, 0]
    c = _cache(rng, "bf16", lens, hkv, dh, page, n)
    per = c.page_table.shape[1]
    table = c.page_table.clone()
    table[0, 1], table[1, 0] = -1, c.k.shape[0]
    q, _, _ = _rows_of(rng, "bf16", 3, n, hq, hkv, dh)
    out = moa.moa_paged_attention(moa.PagedCache(c.k, c.v, table, c.len), q, new_rows=False).double().cpu().numpy()
    for b, gone in ((0, 1), (1, 0)):
        K, V = _slots(c, b, lens[b])
        see = np.arange(lens[b]) // page != gone
        for i in range(0, n, 5):
            for h in range(hq):
                ref, _, mass, spread = _attend(q[b, i, h].double().cpu().numpy(), K[:, h // (hq // 2)], V[:, h // (hq // 2)], see, dh ** -0.5)
                assert np.all(np.abs(out[b, i, h] - ref) <= _bound("bf16", dh, lens[b], spread, mass, ref, once=True))
    assert np.all(out[2] == 0)
    c.k[torch.isnan(c.k)] = 0.25
    c.v[torch.isnan(c.v)] = 0.5
    full = torch.tensor([per * page, per * page - 2, per * page - n], dtype=torch.int32, device="cuda")
    c3 = moa.PagedCache(c.k, c.v, c.page_table, full)
    q, kn, vn = _rows_of(rng, "bf16", 3, n, hq, hkv, dh)
    k0 = c.k.clone()
    out = moa.moa_paged_attention(c3, q, kn, vn)
    torch.cuda.synchronize()
    _check_attention(c3, "bf16", q, kn, vn, None, out, full.tolist(), n)
    for b, m in ((1, 2), (2, n)):
        for i in range(m):
            s = int(full[b]) + i
            k0[int(c.page_table[b, s // page]), s % page] = kn[b, i]
    assert torch.equal(c.k, k0)


def test_one_workspace_for_calls_of_every_kind():
    """One workspace, zeroed once, serves tokens, trees and weights in turn, on one stream, and each call answers as with a
    workspace of its own."""
    moa, rng = _moa(), np.random.default_rng(21)
    lens, hq, hkv, dh = [900, 3, 2100, -1], 32, 4, 128
    c = _cache(rng, "bf16", lens, hkv, dh, 16, 64, track=True)
    kinds = [(1, True), (61, False), (1, False), (2, False), (64, False), (1, True)]
    ws = max((c.workspace(n, hq, w) for n, w in kinds), key=lambda t: t.numel())
    got, want = [], []
    for n, w in kinds * 2:
        q, kn, vn = _rows_of(rng, "bf16", 4, n, hq, hkv, dh)
        outs = []
        for space in (ws, c.workspace(n, hq, w)):
            wo = torch.full_like(c.weight, -7.0) if w else None
            out = torch.full((4, n, hq, dh), 5.0, dtype=torch.bfloat16, device="cuda")
            moa.moa_paged_attention(c, q, kn, vn, out=out, weight_out=wo, ws=space)
            outs.append((out, wo))
        got.append(outs[0])
        want.append(outs[1])
    torch.cuda.synchronize()
    for (a, wa), (b, wb) in zip(got, want):
        assert torch.equal(a, b) and (wa is None or torch.equal(wa, wb))


def test_two_streams_at_once():
    """Calls of two streams, each with its own workspace and output, over one cache whose rows are in the pages."""
    moa, rng = _moa(), np.random.default_rng(31)
    lens, hq, hkv, dh = [3000, 1, 777], 32, 8, 128
    c = _cache(rng, "bf16", lens, hkv, dh, 16, 1)
    q1, _, _ = _rows_of(rng, "bf16", 3, 1, hq, hkv, dh)
    q2, _, _ = _rows_of(rng, "bf16", 3, 30, hq, hkv, dh)
    want = [moa.moa_paged_attention(c, q, new_rows=False) for q in (q1, q2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[torch.empty_like(w) for _ in range(20)] for w in want]
    spaces = [c.workspace(1, hq), c.workspace(30, hq)]
    torch.cuda.synchronize()
    for i in range(20):
        for s, q, o, ws in zip(streams, (q1, q2), outs, spaces):
            moa.moa_paged_attention(c, q, new_rows=False, out=o[i], ws=ws, stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w, x) for x in o)


def test_scratch_of_a_call_on_another_stream():
    """Scratch and results that a call on a given stream makes for itself do not wait for, or overtake, the current stream."""
    moa, rng = _moa(), np.random.default_rng(51)
    c = _cache(rng, "bf16", [3000, 500], 4, 128, 16, 1)
    q, _, _ = _rows_of(rng, "bf16", 2, 1, 16, 4, 128)
    want = moa.moa_paged_attention(c, q, new_rows=False)
    size = c.workspace(1, 16).numel()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        dirt = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for _ in range(3)]
        del dirt
    dirt = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    del dirt
    torch.cuda._sleep(50_000_000)                # the current stream is busy for some 25 ms
    got = [moa.moa_paged_attention(c, q, new_rows=False, stream=side) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(g, want) for g in got)
    torch.cuda.synchronize()


def test_evict_replayed():
    """A captured eviction in place follows the length of each replay."""
    moa, rng = _moa(), np.random.default_rng(41)
    c = _cache(rng, "bf16", [70, 40], 2, 64, 16, 2, track=True)
    ws = c.evict_workspace(64)
    start = [t.clone() for t in (c.k, c.v, c.weight, c.pos)]
    moa.moa_paged_evict(c, 64, 4, 8, ws=ws)
    torch.cuda.synchronize()
    want = [t.clone() for t in (c.k, c.v, c.weight, c.pos)]
    assert c.len.tolist() == [64, 40]
    def back():
        for t, s in zip((c.k, c.v, c.weight, c.pos), start):
            t.copy_(s)
        c.len.copy_(torch.tensor([70, 40], dtype=torch.int32))
    back()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moa.moa_paged_evict(c, 64, 4, 8, ws=ws)
    for _ in range(2):
        back()
        graph.replay()
        torch.cuda.synchronize()
        assert c.len.tolist() == [64, 40]
        assert all(torch.equal(t.view(torch.uint8), w.view(torch.uint8)) for t, w in zip((c.k, c.v, c.weight, c.pos), want))
        graph.replay()                           # nothing is left to evict
        torch.cuda.synchronize()
        assert all(torch.equal(t.view(torch.uint8), w.view(torch.uint8)) for t, w in zip((c.k, c.v, c.weight, c.pos), want))


# ------------------------------------------------------------------------------------------------------------ eviction
def _evict_reference(w, pos, L, seen, budget, sink, recent):
    """(kept slots, [(source, destination)]) of one head."""
    if L <= budget:
        return list(range(max(L, 0))), []
    def key(j):
        must = pos[j] < sink or pos[j] >= seen - recent
        return (0 if must else 1 if not np.isnan(w[j]) else 2, 0.0 if must or np.isnan(w[j]) else -float(w[j]), j)
    kept = set(sorted(range(L), key=key)[:budget])
    src, dst = [j for j in range(budget, L) if j in kept], [j for j in range(budget) if j not in kept]
    assert len(src) == len(dst)
    return sorted(kept), list(zip(src, dst))


EVICT_CASES = [
    # dtype, dh, hkv, page, lens, budget, sink, recent, weights
    ("bf16", 128, 8, 16, [2049], 2048, 4, 64, "random"),
    ("bf16", 128, 2, 16, [100, 64, 63, 0, -1, 65, 1000], 64, 4, 20, "random"),
    ("f32", 64, 3, 8, [50, 51], 10, 0, 0, "ties"),
    ("bf16", 64, 1, 64, [20000, 13000], 300, 4, 100, "ties"),
    ("f32", 128, 2, 32, [700, 400], 399, 10, 389, "odd"),
    ("bf16", 128, 1, 16, [5], 1, 0, 0, "odd"),
    ("bf16", 64, 2, 16, [600, 599], 598, 0, 3, "odd"),
    ("f32", 64, 1, 1024, [12289, 12288], 6000, 4, 0, "random"),
    ("bf16", 64, 8, 16, [1500, 1301, 1300, 1299, 0, -1, 3000, 1302, 2600, 1900], 1300, 4, 64, "random"),      # many heads
    ("f32", 64, 40, 8, [300, 40, 129], 40, 2, 5, "odd"),
    ("bf16", 128, 38, 32, [5000], 4999, 0, 0, "ties"),
]


@pytest.mark.parametrize("dtype,dh,hkv,page,lens,budget,sink,recent,kind", EVICT_CASES)
@pytest.mark.parametrize("apart", [False, True])
def test_evict(dtype, dh, hkv, page, lens, budget, sink, recent, kind, apart):
    moa, rng = _moa(), np.random.default_rng(budget)
    c = _cache(rng, dtype, lens, hkv, dh, page, 2, track=True)
    w = c.weight.cpu().numpy()
    if kind == "ties":
        w = np.floor(w * 2).astype(np.float32) / 2
    if kind == "odd":                            # values at which an order of bits and one of numbers part
        pick = rng.choice([0.0, -0.0, NAN, np.inf, -np.inf, 1e-45, -1.0, 2.5], size=w.shape)
        w = np.where(rng.random(w.shape) < 0.7, pick, w).astype(np.float32)
    pos = np.stack([np.stack([rng.permutation(w.shape[2]) for _ in range(hkv)]) for _ in lens]).astype(np.int32)
    c.weight.copy_(torch.from_numpy(w))
    c.pos.copy_(torch.from_numpy(pos))
    seen = c.seen.cpu().numpy()
    k0, v0 = c.k.clone(), c.v.clone()
    wo, po = (torch.full_like(c.weight, -7.0), torch.full_like(c.pos, -7)) if apart else (c.weight, c.pos)
    lo = torch.full_like(c.len, -9) if apart else c.len
    moa.moa_paged_evict(c, budget, sink, recent, weight_out=wo, pos_out=po, len_out=lo)
    torch.cuda.synchronize()
    assert lo.tolist() == [min(L, budget) for L in lens]
    want_w, want_p = (np.full_like(w, -7.0), np.full_like(pos, -7)) if apart else (w.copy(), pos.copy())
    for b, L in enumerate(lens):
        for h in range(hkv):
            kept, moves = _evict_reference(w[b, h], pos[b, h], L, int(seen[b]), budget, sink, recent)
            n = min(max(L, 0), budget)
            stay = [j for j in kept if j < n]
            want_w[b, h, stay], want_p[b, h, stay] = w[b, h, stay], pos[b, h, stay]
            for s, d in moves:
                want_w[b, h, d], want_p[b, h, d] = w[b, h, s], pos[b, h, s]
            if moves:
                s, d = (torch.tensor(x, device="cuda") for x in zip(*moves))
                page_of = c.page_table[b].long()
                ks, vs = c.k[page_of[s // page], s % page, h], c.v[page_of[s // page], s % page, h]
                k0[page_of[d // page], d % page, h], v0[page_of[d // page], d % page, h] = ks, vs
    assert torch.equal(c.k.view(torch.uint8), k0.view(torch.uint8)) and torch.equal(c.v.view(torch.uint8), v0.view(torch.uint8))
    assert np.array_equal(po.cpu().numpy(), want_p)
    assert np.array_equal(wo.cpu().numpy().view(np.int32), want_w.view(np.int32))


# --------------------------------------------------------------------------------------------------------- logit rules
def _bits(x):
    x = np.concatenate([x, np.zeros(x.shape[:-1] + (-x.shape[-1] % 32,), bool)], -1)
    return np.packbits(x, axis=-1, bitorder="little").view(np.uint32).view(np.int32)


def _rules_reference(x, counts, seen, rep, freq, pres, bias_id, bias_val, allow, path):
    """One row in fp32, step by step as the header says; x float32 [V]."""
    V = len(x)
    f = np.float32
    c = np.zeros(V, np.int64) if counts is None else counts.astype(np.int64).copy()
    known = (c > 0) if seen is None else seen.copy()
    if seen is not None:
        c = np.where(seen, c, 0)
    for t in path:
        if 0 <= t < V:
            c[t] += 1
            known[t] = True
    x = x.copy()
    with np.errstate(all="ignore"):
        if rep is not None:
            x = np.where(known, np.where(x > 0, x / f(rep), x * f(rep)), x).astype(f)
        x = np.where(c > 0, x - f(freq or 0) * c.astype(f), x).astype(f)
        x = np.where(c > 0, x - f(pres or 0), x).astype(f)
        if bias_id is not None:
            add = {}
            for t, v in zip(bias_id, bias_val):
                if 0 <= t < V:
                    add[t] = f(add[t] + f(v)) if t in add else f(v)
            for t, v in add.items():
                x[t] = f(x[t] + v)
    if allow is not None:
        x = np.where(allow, x, f(-np.inf)).astype(f)
    best = np.where(np.isnan(x), -np.inf, x)
    choice = int(np.argmax(best)) if best.max() > -np.inf else 0
    return x, choice


def _path(parent, i):
    if i and parent[i] < 0:
        return []
    got = [i]
    while got[-1] > 0 and 0 <= parent[got[-1]] < got[-1]:
        got.append(int(parent[got[-1]]))
    return got


RULE_CASES = [
    # dtype, batch, n, vocab, tree, bias, allow, record
    ("f32", 1, 1, 7, False, 0, False, "both"),
    ("bf16", 3, 1, 1024, False, 5, True, "both"),
    ("f32", 2, 17, 5003, True, 300, True, "both"),
    ("bf16", 2, 61, 5003, True, 8, False, "counts"),
    ("bf16", 4, 5, 32001, True, 0, True, "seen"),
    ("f32", 1, 2, 128256, True, 1024, False, "none"),
    ("bf16", 16, 40, 999, True, 40, True, "both"),
    ("f32", 2, 300, 640, False, 3, True, "both"),
    ("f32", 64, 61, 32, True, 4, True, "both"),
    ("bf16", 1, 1, 300001, False, 7, True, "both"),
    ("bf16", 1, 1, 518400, False, 1024, False, "both"),
]


@pytest.mark.parametrize("dtype,batch,n,vocab,tree,n_bias,allow,record", RULE_CASES)
def test_logit_rules(dtype, batch, n, vocab, tree, n_bias, allow, record):
    """Bit for bit the steps of the definition in fp32: odd vocabularies, rows off a 16-byte boundary, an id twice in the bias
    list, ids out of range, rows with nothing allowed, NaN and infinities among the logits, unused slots."""
    moa, rng = _moa(), np.random.default_rng(vocab + n)
    x = (rng.standard_normal((batch, n, vocab)) * 3).astype(np.float32)
    odd = rng.random(x.shape) < 0.02
    x[odd] = rng.choice([NAN, np.inf, -np.inf, 0.0, -0.0, 3.0], size=int(odd.sum()))
    x[0, 0] = NAN
    xt = torch.from_numpy(x).to(T[dtype]).cuda()
    x = xt.float().cpu().numpy()
    made = rng.integers(0, vocab, (batch, 60))
    counts = np.zeros((batch, vocab), np.int32)
    for b in range(batch):
        np.add.at(counts[b], made[b], 1)
    seen = counts > 0
    for b in range(batch):
        seen[b, rng.integers(0, vocab, 90)] = True
    counts = counts if record in ("both", "counts") else None
    seen = seen if record in ("both", "seen") else None
    rep, freq, pres = (rng.random(batch).astype(np.float32) + s for s in (0.8, 0.1, -0.3))
    bias_id = bias_val = None
    if n_bias:
        bias_id = rng.integers(-1, vocab + 2, (batch, n_bias)).astype(np.int32)
        bias_id[:, -1] = bias_id[:, 0]
        bias_val = (rng.standard_normal((batch, n_bias)) * 5).astype(np.float32)
    may = None
    if allow:
        may = rng.random((batch, n, vocab)) < 0.4
        may[-1, -1] = False
    tok = parent = None
    if tree:
        parent, _, _ = _trees(rng, batch, n, 1 if n > 2 else 0)
        tok = rng.integers(0, vocab, (batch, n)).astype(np.int32)
        tok[0, 0] = vocab + 3                    # a token that does not exist is on no path
        if n > 4:
            tok[:, 3] = tok[:, 1]
    dev = lambda a, dt=None: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    rules = moa.LogitRules(vocab, dev(counts), dev(_bits(seen)) if seen is not None else None, dev(rep), dev(freq), dev(pres), dev(bias_id),
                           dev(bias_val), dev(_bits(may)) if may is not None else None)
    got, choice = moa.moa_logit_rules(rules, xt, dev(tok), dev(parent))
    want, want_c = np.empty_like(x), np.empty((batch, n), np.int32)
    for b in range(batch):
        for i in range(n):
            path = [int(tok[b, j]) for j in _path(parent[b], i)] if tree else []
            want[b, i], want_c[b, i] = _rules_reference(x[b, i], None if counts is None else counts[b], None if seen is None else seen[b],
                                                       rep[b], freq[b], pres[b], None if bias_id is None else bias_id[b],
                                                       None if bias_val is None else bias_val[b], None if may is None else may[b, i], path)
    wt = torch.from_numpy(want).to(T[dtype]).float().numpy()
    assert np.array_equal(got.float().cpu().numpy(), wt, equal_nan=True)
    assert np.array_equal(choice.cpu().numpy(), want_c)
    again = xt.clone()
    moa.moa_logit_rules(rules, again, dev(tok), dev(parent), out=again)
    assert np.array_equal(again.float().cpu().numpy(), wt, equal_nan=True)
    if tree:
        ok = parent.copy()
        tok[0, 0] = 0
        t_dev, p_dev = dev(tok), dev(ok)
        _, c2 = moa.moa_logit_rules(rules, xt, t_dev, p_dev)
        five = moa.moa_verify_greedy_rules(rules, t_dev, p_dev, xt, 7)
        assert torch.equal(five[0], c2)
        one_hot = torch.zeros((batch, n, vocab)).scatter_(2, c2.long().cpu()[..., None], 1.0)
        plain = moa.moa_verify_greedy(t_dev, p_dev, one_hot.cuda(), 7)
        for a, b in zip(five, plain):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,n,vocab", [(1, 3, 20011), (10, 61, 2003)])
def test_rules_when_everything_was_said(dtype, batch, n, vocab):
    """A record that holds every token, more than a CTA lists, with the output off the logits' 16-byte boundaries or alike."""
    moa, rng = _moa(), np.random.default_rng(vocab)
    xt = torch.from_numpy((rng.standard_normal((batch, n, vocab)) * 3).astype(np.float32)).to(T[dtype]).cuda()
    counts = rng.integers(0, 4, (batch, vocab)).astype(np.int32)
    seen = np.ones((batch, vocab), bool)
    rep, freq, pres = (rng.random(batch).astype(np.float32) + s for s in (0.8, 0.1, -0.3))
    may = rng.random((batch, n, vocab)) < 0.7
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    rules = moa.LogitRules(vocab, dev(counts), dev(_bits(seen)), dev(rep), dev(freq), dev(pres), None, None, dev(_bits(may)))
    x = xt.float().cpu().numpy()
    want, want_c = np.empty_like(x), np.empty((batch, n), np.int32)
    for b in range(batch):
        for i in range(n):
            want[b, i], want_c[b, i] = _rules_reference(x[b, i], counts[b], seen[b], rep[b], freq[b], pres[b], None, None, may[b, i], [])
    wt = torch.from_numpy(want).to(T[dtype]).float().numpy()
    for shift in (0, 1, 4):
        flat = torch.full((x.size + 8,), 9.0, dtype=T[dtype], device="cuda")
        out = flat[shift:shift + x.size].view(batch, n, vocab)
        got, choice = moa.moa_logit_rules(rules, xt, out=out)
        assert np.array_equal(got.float().cpu().numpy(), wt)
        assert np.array_equal(choice.cpu().numpy(), want_c)
        assert torch.all(flat[:shift] == 9.0) and torch.all(flat[shift + x.size:] == 9.0)


def test_no_rules_is_the_plain_arg_max():
    moa, rng = _moa(), np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((2, 3, 4097)).astype(np.float32)).cuda()
    out, choice = moa.moa_logit_rules(moa.LogitRules(4097), x)
    assert torch.equal(out, x) and torch.equal(choice.long(), x.argmax(-1))


def test_token_record():
    moa, rng = _moa(), np.random.default_rng(5)
    V, b, cap = 777, 3, 3000
    counts, seen = torch.zeros((b, V), dtype=torch.int32, device="cuda"), torch.zeros((b, 25), dtype=torch.int32, device="cuda")
    tok = rng.integers(-2, V + 2, (b, cap)).astype(np.int32)
    n = np.array([3000, 0, 41], np.int32)
    t = torch.from_numpy(tok).cuda()
    moa.moa_token_record(t, V, counts, seen, torch.from_numpy(n).cuda())
    prompt = rng.integers(0, V, (b, 10)).astype(np.int32)
    moa.moa_token_record(torch.from_numpy(prompt).cuda(), V, None, seen)
    want, bits = np.zeros((b, V), np.int32), np.zeros((b, V), bool)
    for i in range(b):
        for x in tok[i, :n[i]]:
            if 0 <= x < V:
                want[i, x] += 1
                bits[i, x] = True
        bits[i, prompt[i]] = True
    assert np.array_equal(counts.cpu().numpy(), want) and np.array_equal(seen.cpu().numpy(), _bits(bits))


# --------------------------------------------------------------------------------------------------------------- cycle
def test_cycle_of_all_operators():
    """Prompt, then cycles of a kept tree: attend with the tree's rows, logits of a fixed projection, rules, verification,
    record, commit; tokens without a tree with weights; eviction. The caches, lengths, records and outputs follow a plain
    model of all of it."""
    moa, rng = _moa(), np.random.default_rng(21)
    batch, hq, hkv, dh, V, n, page = 2, 4, 2, 64, 997, 13, 16
    g = torch.Generator().manual_seed(7)
    head = torch.randn((V, hq * dh), generator=g).cuda()
    c = _cache(rng, "bf16", [0, 0], hkv, dh, page, 300, track=True)
    c.k.zero_(); c.v.zero_(); c.seen.zero_(); c.weight.zero_()
    counts, seen = torch.zeros((batch, V), dtype=torch.int32, device="cuda"), torch.zeros((batch, 32), dtype=torch.int32, device="cuda")
    rules = moa.LogitRules(V, counts, seen, *(torch.tensor(x, device="cuda") for x in ([1.3, 1.1], [0.4, 0.2], [0.3, 0.1])))
    prompt = torch.from_numpy(rng.integers(0, V, (batch, 40)).astype(np.int32)).cuda()
    _, kp, vp = _rows_of(rng, "bf16", batch, 40, hq, hkv, dh)
    m = torch.tensor([40, 23], dtype=torch.int32, device="cuda")
    moa.moa_paged_append(c, kp, vp, m)
    moa.moa_paged_commit(c, 40, acc_len=m)
    moa.moa_token_record(prompt, V, None, seen, m)
    held = [(kp[b, :int(m[b])], vp[b, :int(m[b])]) for b in range(batch)]
    want_counts = np.zeros((batch, V), np.int32)
    want_seen = np.zeros((batch, V), bool)
    for b in range(batch):
        want_seen[b, prompt[b, :int(m[b])].cpu().numpy()] = True
    root = torch.tensor([3, 5], dtype=torch.int32, device="cuda")
    for cycle in range(3):
        parent, anc, words = _trees(rng, batch, n, 1)
        tok = torch.from_numpy(np.stack([rng.permutation(V)[:n] for _ in range(batch)]).astype(np.int32)).cuda()
        tok[:, 0] = root
        par = torch.from_numpy(parent).cuda()
        q, kn, vn = _rows_of(rng, "bf16", batch, n, hq, hkv, dh)
        at = c.len.tolist()
        out = moa.moa_paged_attention(c, q, kn, vn, mask=moa.moa_tree_attn_mask(par, packed=True))
        _check_attention(c, "bf16", q, kn, vn, words.cpu().numpy(), out, at, n)
        logits = out.float().reshape(batch, n, -1) @ head.T
        for b in range(batch):                   # the LLM likes one child of most slots
            for i in range(1, n - 1):
                if rng.random() < 0.7:
                    logits[b, parent[b, i], tok[b, i].long()] = 60.0 + float(i)
        choice, slot, acc, k, nxt = moa.moa_verify_greedy_rules(rules, tok, par, logits, 7)
        moa.moa_token_record(acc, V, counts, seen, k)
        moa.moa_paged_commit(c, n, slot, k)
        torch.cuda.synchronize()
        for b in range(batch):
            t, z = tok[b].cpu().numpy(), logits[b].cpu().numpy()
            adj = np.stack([_rules_reference(z[i], want_counts[b], want_seen[b], *(float(getattr(rules.held[j][b], "item")()) for j in (2, 3, 4)),
                                             None, None, None, [int(t[j]) for j in _path(parent[b], i)])[0] for i in range(n)])
            slots, follow, _ = O.verify_greedy(t, parent[b], adj)
            slots = slots[:7]
            assert int(k[b]) == len(slots) and slot[b, :len(slots)].tolist() == list(slots)
            assert len(slots) == 7 or int(nxt[b]) == follow
            held[b] = tuple(torch.cat([x, y[b, torch.tensor(list(slots), device="cuda")]]) for x, y in zip(held[b], (kn, vn)))
            np.add.at(want_counts[b], t[slots], 1)
            want_seen[b, t[slots]] = True
            K, V_ = _slots(c, b, int(c.len[b]))
            assert np.array_equal(K, held[b][0].double().cpu().numpy()) and np.array_equal(V_, held[b][1].double().cpu().numpy())
        assert np.array_equal(counts.cpu().numpy(), want_counts) and np.array_equal(seen.cpu().numpy(), _bits(want_seen))
        root = nxt
    c.weight.zero_()
    for step in range(3):
        q, kn, vn = _rows_of(rng, "bf16", batch, 1, hq, hkv, dh)
        at, w_in = c.len.tolist(), c.weight.clone()
        out = moa.moa_paged_attention(c, q, kn, vn, weight_out=c.weight)
        _check_attention(c, "bf16", q, kn, vn, None, out, at, 1, weight_out=c.weight, weight_in=w_in)
        moa.moa_paged_commit(c, 1)
    w, pos, lens = c.weight.cpu().numpy(), c.pos.cpu().numpy(), c.len.tolist()
    rows = [_slots(c, b, lens[b]) for b in range(batch)]
    moa.moa_paged_evict(c, 30, sink=4, recent=8)
    assert c.len.tolist() == [min(30, L) for L in lens]
    for b in range(batch):
        K, V_ = _slots(c, b, int(c.len[b]))
        for h in range(hkv):
            kept, moves = _evict_reference(w[b, h], pos[b, h], lens[b], int(c.seen[b]), 30, 4, 8)
            order = list(range(len(K)))
            for s, d in moves:
                order[d] = s
            assert sorted(order) == kept
            assert np.array_equal(K[:, h], rows[b][0][order, h]) and np.array_equal(V_[:, h], rows[b][1][order, h])
            assert c.pos[b, h, :len(K)].tolist() == pos[b, h, order].tolist()
    q, kn, vn = _rows_of(rng, "bf16", batch, 1, hq, hkv, dh)
    out = moa.moa_paged_attention(c, q, kn, vn)
    _check_attention(c, "bf16", q, kn, vn, None, out, c.len.tolist(), 1)
