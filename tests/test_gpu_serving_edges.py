"""The serving operators on the GPU where their parts meet: items of one block, pages that are missing, entries that nobody
sees, values that are not finite, scores far from zero. Definitions and tolerances are those of the operators' other tests."""
import numpy as np
import pytest
import torch

from tests.test_gpu_serving import NAN, T, _attend, _bound, _cache, _check_attention, _evict_reference, _moa, _rows_of, _slots, _trees, _word  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh,hkv,hq,n", [(128, 2, 4, 20), (64, 3, 48, 17)])
def test_tree_items_of_one_block(dh, hkv, hq, n):
    """Stretches of several short items, the first of one block of positions: the queries of the second item may be there
    before its keys are asked for."""
    moa, rng = _moa(), np.random.default_rng(dh)
    lens = [int(x) for x in rng.integers(1, 128 - n, 40)]
    c = _cache(rng, "bf16", lens, hkv, dh, 16, 600)
    q, kn, vn = _rows_of(rng, "bf16", 40, n, hq, hkv, dh)
    _, _, mask = _trees(rng, 40, n, 0)
    out = moa.moa_paged_attention(c, q, kn, vn, mask=mask)
    torch.cuda.synchronize()
    _check_attention(c, "bf16", q, kn, vn, mask.cpu().numpy(), out, lens, n)
    for _ in range(50):
        assert torch.equal(moa.moa_paged_attention(c, q, mask=mask), out)


@pytest.mark.parametrize("dtype,hq,n,extra", [("bf16", 8, 1, 0), ("f32", 4, 1, 0), ("bf16", 2, 5, 0), ("f32", 8, 19, 0),
                                              ("bf16", 16, 19, 0), ("bf16", 16, 19, 5000)])
def test_new_rows_on_missing_pages(dtype, hq, n, extra):
    """New rows whose page the table does not have are left out, whichever kernel a cache's size leads to, and whether the
    call appends them or they were appended before; their slots get no weight."""
    moa, rng = _moa(), np.random.default_rng(n + extra + hq)
    hkv, dh, page = 2, 64, 8
    lens = [40, 37, 64, 16]                      # the rows begin with a page, inside one, ...
    c = _cache(rng, dtype, lens, hkv, dh, page, n + extra, track=True)
    table = c.page_table.clone()
    gone = [(0, 5), (1, 4), (2, 9 if n > 8 else 8), (3, 2)]
    for b, p in gone:
        table[b, p] = -1 if b % 2 else c.k.shape[0] + b
    c2 = moa.PagedCache(c.k, c.v, table, c.len, c.weight, c.pos, c.seen)
    q, kn, vn = _rows_of(rng, dtype, 4, n, hq, hkv, dh)
    _, _, mask = _trees(rng, 4, n, 0)
    w_in = c.weight.clone()
    wo = torch.full_like(c.weight, -7.0) if n == 1 else None
    k0 = c.k.clone()
    out = moa.moa_paged_attention(c2, q, kn, vn, mask=mask, weight_out=wo)
    torch.cuda.synchronize()
    words = mask.cpu().numpy()
    for b, L in enumerate(lens):
        K, V = _slots(c, b, L)
        K, V = np.concatenate([K, kn[b].double().cpu().numpy()]), np.concatenate([V, vn[b].double().cpu().numpy()])
        there = np.arange(L + n) // page != gone[b][1]
        for i in range(n):
            see = there.copy()
            see[L:] &= [bool((int(words[b, i]) >> j) & 1) for j in range(n)]
            for h in range(hq):
                g = h // (hq // hkv)
                ref, w, mass, spread = _attend(q[b, i, h].double().cpu().numpy(), K[:, g], V[:, g], see, dh ** -0.5)
                assert np.all(np.abs(out[b, i, h].double().cpu().numpy() - ref) <= _bound(dtype, dh, L + n, spread, mass, ref, once=n > 1)), (b, i, h)
        for i in range(n):
            if there[L + i]:
                k0[int(table[b, (L + i) // page]), (L + i) % page] = kn[b, i]
        if wo is not None:                       # the group's weights are shared out among the slots that are there
            got = (wo[b, :, :L].double() - w_in[b, :, :L].double()).cpu().numpy()[:, there[:L]].sum(-1)
            got = got + (wo[b, :, L].double().cpu().numpy() if there[L] else 0.0)
            assert np.allclose(got, hq // hkv, rtol=1e-4)
    assert torch.equal(c.k.view(torch.uint8), k0.view(torch.uint8))
    assert torch.equal(moa.moa_paged_attention(c2, q, mask=mask), out)


@pytest.mark.parametrize("dtype,n,extra", [("bf16", 1, 0), ("f32", 1, 0), ("bf16", 3, 0), ("f32", 9, 0), ("bf16", 40, 5000)])
@pytest.mark.parametrize("scale", [3e5, 1e8, 7e11, 1e30, 1e36, 2e38])
@pytest.mark.parametrize("below", [False, True])
def test_scores_far_from_zero(dtype, n, extra, scale, below):
    """Scores are whole numbers, exact in fp32, and the scale sets them so far apart that a row's largest share the weight
    evenly: out = the mean of their values. Off by: p = 1 and their count are exact; the sum of m products and the division
    round in fp32 (m + 1 times 2^-23 of the mean of |v| with room for the order), the result once to its type."""
    moa, rng = _moa(), np.random.default_rng(n)
    L, hq, hkv, dh = 333, 16, 2, 128
    c = _cache(rng, dtype, [L], hkv, dh, 16, n + extra, track=n == 1)
    q, kn, vn = _rows_of(rng, dtype, 1, n, hq, hkv, dh)
    g = torch.Generator().manual_seed(n)
    whole = lambda shape: torch.randint(-2, 0 if below else 3, shape, generator=g).to(T[dtype]).cuda()  # noqa: E731
    q.copy_(whole(q.shape).abs() if below else whole(q.shape))
    kn.copy_(whole(kn.shape))
    c.k.copy_(whole(c.k.shape))
    _, anc, mask = _trees(rng, 1, n, 0)
    wo = torch.zeros_like(c.weight) if n == 1 else None
    if n == 1:
        c.weight.zero_()
    out = moa.moa_paged_attention(c, q, kn, vn, mask=mask, scale=scale, weight_out=wo)
    K, V = _slots(c, 0, L + n)
    acc = np.zeros((hkv, L + n))
    for i in range(n):
        see = np.concatenate([np.ones(L, bool), anc[0, i]])
        for h in range(hq):
            s = np.where(see, K[:, h // 8] @ q[0, i, h].double().cpu().numpy(), -np.inf)
            top = s == s.max()
            acc[h // 8] += top / top.sum()
            v, m = V[top, h // 8], top.sum()
            ref, mass = v.mean(0), np.abs(v).mean(0)
            tol = (2.0**-8 if dtype == "bf16" else 2.0**-24) * np.abs(ref) + (m + 1) * 2.0**-23 * mass
            assert np.all(np.abs(out[0, i, h].double().cpu().numpy() - ref) <= tol), (i, h)
    if n == 1:
        assert np.all(np.abs(wo[0, :, :L + 1].double().cpu().numpy() - acc) <= 9 * 2.0**-23 * acc)


@pytest.mark.parametrize("dtype,dh,hq,hkv,n,extra,lens", [("bf16", 128, 2, 2, 5, 0, [30, 0]), ("bf16", 64, 6, 2, 16, 0, [121]), ("f32", 128, 8, 2, 9, 0, [70]),
                                                          ("f32", 64, 3, 3, 33, 0, [15, 250]), ("bf16", 128, 64, 8, 61, 600, [100, 0, 700]),
                                                          ("bf16", 64, 8, 2, 40, 5000, [333, 1])])
@pytest.mark.parametrize("there", [False, True])
def test_values_that_are_not_finite(dtype, dh, hq, hkv, n, extra, lens, there):
    """Infinities and NaN among the keys and values of a tree's slots reach the rows that see those slots, in the columns they
    stand in, and no other row."""
    moa, rng = _moa(), np.random.default_rng(n + dh)
    B = len(lens)
    c = _cache(rng, dtype, lens, hkv, dh, 16, n + extra)
    q, kn, vn = _rows_of(rng, dtype, B, n, hq, hkv, dh)
    parent, anc, mask = _trees(rng, B, n, 0)
    for b in range(B):                           # leaves and inner slots, but not the root
        i, j, k, m = rng.permutation(np.arange(1, n))[:4]
        vn[b, i, :, 3] = float("inf")
        vn[b, j, 0] = -float("inf")
        vn[b, k, :, dh - 9:] = NAN
        kn[b, m, hkv - 1, 5] = NAN
    if there:
        moa.moa_paged_append(c, kn, vn)
    out = moa.moa_paged_attention(c, q, *(() if there else (kn, vn)), mask=mask).double().cpu().numpy()
    for b, L in enumerate(lens):
        K, V = _slots(c, b, L + n)
        assert np.array_equal(V[L:], vn[b].double().cpu().numpy(), equal_nan=True) and np.array_equal(K[L:], kn[b].double().cpu().numpy(), equal_nan=True)
        for i in range(n):
            see = np.concatenate([np.ones(L, bool), anc[b, i]])
            for h in range(hq):
                g = h // (hq // hkv)
                seen = np.where(see[:, None], V[:, g], 0.0)
                qi = q[b, i, h].double().cpu().numpy()
                ref, _, _, _ = _attend(qi, K[:, g], seen, see, dh ** -0.5)
                sure = np.isfinite(ref)
                if sure.any():
                    fin, _, mass, spread = _attend(qi, K[:, g], np.where(np.isfinite(seen), seen, 0.0), see, dh ** -0.5)
                    tol = _bound(dtype, dh, L + n, spread, mass, fin, once=True)
                    assert np.all(np.abs(out[b, i, h] - fin)[sure] <= tol[sure]), (b, i, h)
                assert np.array_equal(out[b, i, h][~sure], ref[~sure], equal_nan=True), (b, i, h, out[b, i, h][~sure], ref[~sure])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("track", [False, True])
def test_weights_of_slots_that_the_row_does_not_see(dtype, own, track):
    """weight_out has entries for the slots that the row sees: not for pages that the table does not have, a row whose mask
    word is 0, or a row that does not see its own slot."""
    moa, rng = _moa(), np.random.default_rng(17)
    hq, hkv, dh, page = 6, 2, 64, 16
    lens, words = [90, 300, 40, 32, 33, -1, 0, 0], [1, 1, 0, 2, 1, 1, 2, 0]
    c = _cache(rng, dtype, lens, hkv, dh, page, 1, track=True)
    table = c.page_table.clone()
    gone = {0: 1, 1: 18, 4: 2}                   # inside, the new slot's and the last cached ones', the new slot's page
    for b, p in gone.items():
        table[b, p] = -5 if b else c.k.shape[0]
    w_in = c.weight.clone()
    c2 = moa.PagedCache(c.k, c.v, table, c.len, c.weight, *((c.pos, c.seen) if track else ()))
    q, kn, vn = _rows_of(rng, dtype, len(lens), 1, hq, hkv, dh)
    wo = c.weight if own else torch.full_like(c.weight, -7.0)
    mask = torch.tensor(words, dtype=torch.int64).reshape(-1, 1).cuda()
    moa.moa_paged_attention(c2, q, kn, vn, mask=mask, weight_out=wo)
    got = wo.double().cpu().numpy()
    for b, L in enumerate(lens):
        want = (w_in if own else torch.full_like(wo, -7.0))[b].double().cpu().numpy()
        rel = np.zeros_like(want)
        if L >= 0:
            if own and track:
                want[:, L] = 0.0                 # the new slot's weight, as moa_paged_append sets it
            K, V = _slots(c, b, L)
            K, V = np.concatenate([K, kn[b].double().cpu().numpy()]), np.concatenate([V, vn[b].double().cpu().numpy()])
            see = np.arange(L + 1) // page != gone.get(b, -1)
            see[:L] &= words[b] != 0
            see[L] &= words[b] & 1 != 0
            old = w_in[b].double().cpu().numpy()[:, :L + 1].copy()
            old[:, L] = 0.0
            acc = np.zeros_like(old)
            for h in range(hq):
                acc[h // 3] += _attend(q[b, 0, h].double().cpu().numpy(), K[:, h // 3], V[:, h // 3], see, dh ** -0.5)[1]
            want[:, :L + 1][:, see] = (old + acc)[:, see]
            # as in the weights' other tests: the errors of p, then the group's sum and the addition in fp32
            rel[:, :L + 1][:, see] = ((2 * (dh + 1) * 2.0**-23 * 60 + 2.0**-20 + 3 * (L + 1) * 2.0**-24 + 4 * 2.0**-24) * acc + 2.0**-23 * (old + acc))[:, see]
        assert np.all(np.abs(got[b] - want) <= rel), (b, np.argwhere(np.abs(got[b] - want) > rel)[:4])


@pytest.mark.parametrize("dtype,dh,hkv,page,lens,budget,sink,recent", [
    ("bf16", 64, 2, 16, [300, 100, 65, 640], 64, 4, 20),
    ("f32", 128, 20, 8, [300, 99, 41, 640], 40, 2, 5),                    # many heads
    ("bf16", 64, 1, 32, [13000, 20000, 12288, 700], 6400, 4, 100),        # more slots than keys in shared memory
])
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("gone", ["low", "high", "both", "most"])
def test_evict_with_missing_pages(dtype, dh, hkv, page, lens, budget, sink, recent, apart, gone):
    """Slots on pages that the table does not have: before the budget they stay and count, behind it they go first. Every row
    that moves takes its weight and position along, and none moves from or to such a page."""
    moa, rng = _moa(), np.random.default_rng(budget + len(gone))
    c = _cache(rng, dtype, lens, hkv, dh, page, 2, track=True)
    c.weight.copy_(torch.from_numpy(np.floor(rng.random(tuple(c.weight.shape)) * 40).astype(np.float32) / 8))
    c.weight[:, :, 1::7] = NAN
    c.pos.copy_(torch.from_numpy(np.stack([np.stack([rng.permutation(c.slots) for _ in range(hkv)]) for _ in lens]).astype(np.int32)))
    table, edge = c.page_table.clone(), -(-budget // page)
    for b, L in enumerate(lens):
        last = (L - 1) // page
        low, high = rng.permutation(edge)[:max(1, edge // 3)], edge + rng.permutation(max(0, last + 1 - edge))[:max(1, (last - edge) // 3)]
        if gone == "most":
            low, high = rng.permutation(edge)[:edge // 2], np.arange(edge, last + 1)[1:]
        for p in ([] if gone == "high" else low.tolist()) + ([] if gone == "low" else high.tolist()):
            table[b, p] = -1 if p % 2 else c.k.shape[0] + p
    c2 = moa.PagedCache(c.k, c.v, table, c.len, c.weight, c.pos, c.seen)
    w, pos, seen = c.weight.cpu().numpy(), c.pos.cpu().numpy(), c.seen.cpu().numpy()
    k0, v0 = c.k.clone(), c.v.clone()
    wo, po = (torch.full_like(c.weight, -7.0), torch.full_like(c.pos, -7)) if apart else (c.weight, c.pos)
    moa.moa_paged_evict(c2, budget, sink, recent, weight_out=wo, pos_out=po)
    torch.cuda.synchronize()
    assert c.len.tolist() == [min(L, budget) for L in lens]
    want_w, want_p = (np.full_like(w, -7.0), np.full_like(pos, -7)) if apart else (w.copy(), pos.copy())
    there = ((table >= 0) & (table < c.k.shape[0])).cpu().numpy()
    for b, L in enumerate(lens):
        for h in range(hkv):
            def key(j):
                if not there[b, j // page]:
                    return (0 if j < budget else 3, 0.0, j)
                if pos[b, h, j] < sink or pos[b, h, j] >= seen[b] - recent:
                    return (0, 0.0, j)
                return (2, 0.0, j) if np.isnan(w[b, h, j]) else (1, -float(w[b, h, j]), j)
            kept = set(sorted(range(L), key=key)[:budget])
            src, dst = [j for j in range(budget, L) if j in kept], [j for j in range(min(L, budget)) if j not in kept]
            assert len(src) == len(dst) and all(there[b, j // page] for j in src + dst)
            stay = [j for j in kept if j < budget]
            want_w[b, h, stay], want_p[b, h, stay] = w[b, h, stay], pos[b, h, stay]
            want_w[b, h, dst], want_p[b, h, dst] = w[b, h, src], pos[b, h, src]
            if src:
                s, d = torch.tensor(src, device="cuda"), torch.tensor(dst, device="cuda")
                at = table[b].long()
                ks, vs = c.k[at[s // page], s % page, h].clone(), c.v[at[s // page], s % page, h].clone()
                k0[at[d // page], d % page, h], v0[at[d // page], d % page, h] = ks, vs
    assert torch.equal(c.k.view(torch.uint8), k0.view(torch.uint8)) and torch.equal(c.v.view(torch.uint8), v0.view(torch.uint8))
    assert np.array_equal(po.cpu().numpy(), want_p)
    assert np.array_equal(wo.cpu().numpy().view(np.int32), want_w.view(np.int32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_commit_with_missing_pages(dtype):
    """A listed row that comes from a missing page leaves its new slot as it was, one that goes to such a page is lost; the
    others are kept, and nothing else is written."""
    moa, rng = _moa(), np.random.default_rng(5)
    lens, n, hkv, dh, page = [30, 13, 24], 40, 2, 64, 8
    c = _cache(rng, dtype, lens, hkv, dh, page, n)
    _, kn, vn = _rows_of(rng, dtype, 3, n, hkv, hkv, dh)
    moa.moa_paged_append(c, kn, vn)
    table = c.page_table.clone()
    table[0, 6], table[1, 2], table[2, 3] = -1, c.k.shape[0], -9
    path = torch.tensor([[0, 1, 5, 18, 19, 33, 39], [0, 3, 4, 10, 12, 30, -1], [0, 2, 30, 31, -1, -1, -1]], dtype=torch.int32, device="cuda")
    m = torch.tensor([7, 6, 4], dtype=torch.int32, device="cuda")
    k0, v0 = c.k.clone(), c.v.clone()
    k1, v1, at, there = c.k.clone(), c.v.clone(), table.tolist(), lambda p: 0 <= p < c.k.shape[0]
    for b, L in enumerate(lens):
        for j in range(int(m[b])):
            s, d = L + int(path[b, j]), L + j
            ps, pd = at[b][s // page], at[b][d // page]
            if there(ps) and there(pd):
                k1[pd, d % page], v1[pd, d % page] = k0[ps, s % page], v0[ps, s % page]
    moa.moa_paged_commit(moa.PagedCache(c.k, c.v, table, c.len), n, path, m)
    assert c.len.tolist() == [37, 19, 28]
    assert torch.equal(c.k.view(torch.uint8), k1.view(torch.uint8)) and torch.equal(c.v.view(torch.uint8), v1.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [2003, 32001])
def test_rules_in_small_and_large_calls(dtype, vocab):
    """The rows of a large call, which take a CTA each, and the same rows in small ones, which take a cluster each: the same bits."""
    moa, rng = _moa(), np.random.default_rng(vocab)
    batch, n = 12, 9
    g = torch.Generator().manual_seed(vocab)
    x = (torch.randn((batch, n, vocab), generator=g) * 3).to(T[dtype]).cuda()
    x[:, 3, ::7] = NAN
    x[:, 5] = x[:, 5].round()
    counts = (torch.rand((batch, vocab), generator=g) < 0.1).int().cuda() * 2
    word = lambda may: (torch.nn.functional.pad(may, (0, -vocab % 32)).unflatten(-1, (-1, 32)).long() << torch.arange(32)).sum(-1)  # noqa: E731
    bits = lambda may: torch.where((w := word(may)) >= 2**31, w - 2**32, w).int().cuda()  # noqa: E731
    seen = bits((counts.cpu() > 0) | (torch.rand((batch, vocab), generator=g) < 0.05))
    allow = bits(torch.rand((batch, n, vocab), generator=g) < 0.5)
    rep, freq, pres = (torch.rand(batch, generator=g).cuda() + 0.5 for _ in range(3))
    bias_id = torch.randint(-1, vocab + 1, (batch, 70), generator=g).int().cuda()
    bias_val = torch.randn((batch, 70), generator=g).cuda()
    parent, _, _ = _trees(rng, batch, n, 2)
    tok, par = torch.randint(0, vocab, (batch, n), generator=g).int().cuda(), torch.from_numpy(parent).cuda()
    out, choice = moa.moa_logit_rules(moa.LogitRules(vocab, counts, seen, rep, freq, pres, bias_id, bias_val, allow), x, tok, par)
    for b in range(batch):
        one = slice(b, b + 1)
        rules = moa.LogitRules(vocab, *(t[one].contiguous() for t in (counts, seen, rep, freq, pres, bias_id, bias_val, allow)))
        o, c = moa.moa_logit_rules(rules, x[one].contiguous(), tok[one].contiguous(), par[one].contiguous())
        assert torch.equal(o.view(torch.uint8), out[one].view(torch.uint8)) and torch.equal(c, choice[one])


@pytest.mark.parametrize("dh,hq,hkv,n,lens", [(128, 4, 2, 2, [700, 33]), (64, 8, 8, 16, [300]), (128, 16, 2, 2, [5000, 1]), (64, 6, 2, 5, [64, 0, 999])])
def test_rows_of_small_calls_keep_probabilities_in_two_terms(dh, hq, hkv, n, lens):
    """Up to 16 query rows per key / value head a bf16 call keeps its probabilities in two bf16 terms, like a token's: the
    tolerance is that of one row."""
    moa, rng = _moa(), np.random.default_rng(n * hq)
    c = _cache(rng, "bf16", lens, hkv, dh, 16, n)
    q, kn, vn = _rows_of(rng, "bf16", len(lens), n, hq, hkv, dh)
    _, anc, mask = _trees(rng, len(lens), n, 0)
    out = moa.moa_paged_attention(c, q, kn, vn, mask=mask)
    for b, L in enumerate(lens):
        K, V = _slots(c, b, L)
        K, V = np.concatenate([K, kn[b].double().cpu().numpy()]), np.concatenate([V, vn[b].double().cpu().numpy()])
        for i in range(n):
            see = np.concatenate([np.ones(L, bool), anc[b, i]])
            for h in range(hq):
                ref, _, mass, spread = _attend(q[b, i, h].double().cpu().numpy(), K[:, h * hkv // hq], V[:, h * hkv // hq], see, dh ** -0.5)
                assert np.all(np.abs(out[b, i, h].double().cpu().numpy() - ref) <= _bound("bf16", dh, L + n, spread, mass, ref)), (b, i, h)


def test_line_of_work_beyond_its_limit_is_refused():
    """The documented bound on sequences x heads x query tiles x positions: refused on the host, before anything is launched."""
    import ctypes as C
    moa = _moa()
    fake, lib = 0x10000, moa.load_library()
    cache = moa.MoaPagedCache(fake, fake, 1024 * 8 * 64, fake, fake, None, None, None, 64, 1024, 9, 1024, 8, 64, 0)
    call = lambda hq: lib.moa_paged_attention(C.byref(cache), fake, hq * 64, None, None, 0, 64, 64, hq, None, 0.0, fake, None, fake, 0, None)  # noqa: E731
    assert call(8 * 128) == 2                    # 64 * 8 * (64 * 128 / 8) * (1024 * 1024 / 64) = 2^33: a shape
    assert call(8 * 16) == 5                     # 2^30: accepted, and refused for its workspace of no bytes
