"""The 8-bit paged cache on the GPU against plain definitions in 64 bits: append, read, attention, commit, and cycles of them."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

NAN = float("nan")
BF = torch.bfloat16


def _moa():
    from paper_2410_03804_b200 import moa
    return moa


def _codes(x):
    """One block [16, hkv, dh] of bf16 rows: (codes float64, scales float32 [hkv]) by the documented fp32 steps."""
    x = x.float().numpy()
    top = np.abs(x).max((0, 2))
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        none = top < 2.0**-100
        scale = np.where(none, np.float32(0), top / np.float32(127)).astype(np.float32)
        r = np.where(none, np.float32(0), np.float32(127) / top).astype(np.float32)
        code = np.rint((x * r[None, :, None]).astype(np.float32))
    bad = ~np.isfinite(x).all((0, 2))
    return np.where(bad[None, :, None], 0.0, code).astype(np.float64), np.where(bad, np.float32(NAN), scale)


def _held(rows):
    """Committed rows [m, hkv, dh] bf16 as the cache holds them: float32 values of closed blocks, the rest as they are."""
    out = rows.float().numpy().copy()
    for j in range(0, len(rows) // 16 * 16, 16):
        code, scale = _codes(rows[j:j + 16])
        out[j:j + 16] = code.astype(np.float32) * scale[None, :, None]
    return out


class Model:
    """A cache and, on the host, the rows that were committed to it."""

    def __init__(self, rng, lens, hkv, dh, page, extra=64, gap=0, spare=2, chunks=1):
        self.rng, self.hkv, self.dh, self.page, self.batch = rng, hkv, dh, page, len(lens)
        per = max(1, -(-(max(max(lens), 0) + extra) // page))
        total = self.batch * per + spare
        self.g = torch.Generator().manual_seed(int(rng.integers(1 << 30)))
        table = torch.from_numpy(rng.permutation(total)[:self.batch * per].astype(np.int32).reshape(self.batch, per)).cuda()
        rec = hkv * (page // 16) * (32 * dh + 16)
        flat = torch.full((total, rec + gap), 255, dtype=torch.uint8, device="cuda")          # scales of unwritten records are NaN
        pages = flat[:, :rec].unflatten(1, (hkv, page // 16, 32 * dh + 16))
        kr, vr = (torch.full((self.batch, 80, hkv, dh), NAN, dtype=BF, device="cuda") for _ in range(2))
        self.len = torch.tensor([min(L, 0) for L in lens], dtype=torch.int32, device="cuda")
        self.seen = torch.arange(self.batch, dtype=torch.int32, device="cuda") * 10
        self.c = _moa().PagedCache8(pages, kr, vr, table, self.len, page, self.seen)
        self.rows = [(torch.zeros((0, hkv, dh), dtype=BF),) * 2 for _ in lens]
        if max(lens) > 0:
            k, v = self.fresh(max(lens)), self.fresh(max(lens))
            self.append(k, v, lens)

    def fresh(self, n, scale=1.0):
        return (torch.randn((self.batch, n, self.hkv, self.dh), generator=self.g) * scale).to(BF)

    def append(self, k, v, n_new, advance=True, stride=0):
        n = torch.tensor(n_new, dtype=torch.int32, device="cuda")
        kv = torch.full((self.batch, k.shape[1], 2 + (stride > 0), self.hkv, self.dh), NAN, dtype=BF)          # side by side, as a projection leaves them
        kv[:, :, 0], kv[:, :, 1] = k, v
        kv = kv.cuda()
        _moa().moa_paged8_append(self.c, kv[:, :, 0], kv[:, :, 1], n, advance=advance)
        for b, m in enumerate(n_new):
            if int(self.len[b]) >= 0:
                m = max(0, min(m, k.shape[1]))
                self.keep(b, k[b, :m], v[b, :m])

    def keep(self, b, k, v):
        self.rows[b] = tuple(torch.cat([a, x]) for a, x in zip(self.rows[b], (k, v)))

    def held(self, b):
        return tuple(_held(x) for x in self.rows[b])

    def check_rows(self, first=None, n=None):
        """The whole cache, read back in both types, bit for bit."""
        most = max(len(r[0]) for r in self.rows)
        n = n or most + 20
        f = torch.zeros(self.batch, dtype=torch.int32) if first is None else torch.tensor(first, dtype=torch.int32)
        for dt in (torch.float32, BF):
            got = _moa().moa_paged8_read(self.c, n, first=None if first is None else f.cuda(), dtype=dt)
            for b in range(self.batch):
                live = int(self.len[b]) >= 0
                for x, y in zip(got, self.held(b)):
                    want = torch.zeros((n, self.hkv, self.dh), dtype=dt)
                    at = torch.arange(n) + int(f[b])
                    ok = (at >= 0) & (at < len(y)) & live
                    want[ok] = torch.from_numpy(y)[at[ok]].to(dt)
                    same = (x[b].cpu() == want) | (torch.isnan(x[b].cpu()) & torch.isnan(want))
                    assert bool(same.all()), (dt, b, (~same).nonzero()[:4].tolist())


def _attend(q, K, V, see, scale):
    idx = np.nonzero(see)[0]
    if len(idx) == 0:
        return np.zeros(K.shape[1]), np.zeros(K.shape[1]), 0.0
    z = K[idx] @ q * scale
    p = np.exp(z - z.max())
    p /= p.sum()
    return p @ V[idx], p @ np.abs(V[idx]), float((np.abs(K[idx]) @ np.abs(q)).max() * scale)


def _bound(dh, keys, spread, mass, ref, most):
    """How far an output may be off: its own rounding to bf16 (half a step), and
      scores  dh exact products summed in fp32 (at most 2^-23 of the running sum each, as the tensor cores may cut), two products
              with scales (2^-24 each) and 2^-23 of the scaled score: (dh + 3) * 2^-23 * sum |q k|, above and below the fraction's line
      exp     2^-21 per p, above and below
      p       times the values' scale, rounded once to fp16: 2^-11 of itself, or 2^-29 of the largest p times the largest scale,
              and so 2^-29 of the largest value (a code is at most 127 scales) for each position
      sums    at most `keys` additions in fp32: 3 * keys * 2^-24"""
    score = (dh + 3) * 2.0**-23 * spread
    rel = 2 * score + 2 * 2.0**-21 + 2.0**-11 + 3 * keys * 2.0**-24
    return 2.0**-8 * np.abs(ref) * (1 + rel) + rel * mass + keys * 2.0**-29 * most


def _word(mask, b, i):
    return (2 << i) - 1 if mask is None else int(mask[b, i]) & (2**64 - 1)


def _check_attention(m, q, k_new, v_new, mask, out, n_new, scale=None, before=None, missing=()):
    """out [batch, n, hq, dh] against the definition over what the cache holds. missing: (sequence, block) that are not there."""
    batch, n, hq, dh = q.shape
    G = hq // m.hkv
    scale = dh**-0.5 if scale is None else scale
    o, qd = out.double().cpu().numpy(), q.double().cpu().numpy()
    for b in range(batch):
        if int(m.len[b]) < 0:
            if before is not None:
                assert torch.equal(out[b], before[b])
            continue
        K, V = (x.astype(np.float64) for x in m.held(b))
        L = len(K)
        there = np.ones(L, bool)
        for bb, blk in missing:
            if bb == b:
                there[blk * 16:blk * 16 + 16] = False
        K[~there], V[~there] = 0, 0
        if n_new:
            K = np.concatenate([K, k_new[b].double().cpu().numpy()])
            V = np.concatenate([V, v_new[b].double().cpu().numpy()])
        most = np.abs(np.where(np.isfinite(V), V, 0)).max() if len(V) else 0.0
        for i in range(n):
            see = np.concatenate([there, np.ones(len(K) - L, bool)])
            word = _word(mask, b, i)
            if n_new:
                see[L:] = [(word >> j) & 1 for j in range(n_new)]
            if word == 0:
                see[:] = False
            see &= np.arange(len(K)) < m.c.slots
            for h in range(hq):
                ref, mass, spread = _attend(qd[b, i, h], K[:, h // G], V[:, h // G], see, scale)
                tol = _bound(dh, len(K), spread, mass, ref, most)
                assert np.all(np.abs(o[b, i, h] - ref) <= tol), (b, i, h, np.max(np.abs(o[b, i, h] - ref) - tol), np.abs(ref).max())


def _new_rows(m, n, hq, scale=1.0):
    """q, k, v of n new rows side by side, on the GPU."""
    x = torch.cat([torch.randn((m.batch, n, hq, m.dh), generator=m.g) * scale, torch.randn((m.batch, n, 2 * m.hkv, m.dh), generator=m.g)], 2).to(BF).cuda()
    return x[:, :, :hq], x[:, :, hq:hq + m.hkv], x[:, :, hq + m.hkv:]


def _tree(rng, batch, n, empty=0):
    """Masks of random trees, int64 [batch, n]; some rows unused."""
    mask = np.zeros((batch, n), np.uint64)
    for b in range(batch):
        for i in range(n):
            up = int(mask[b, int(rng.integers(0, i))]) if i else 0
            mask[b, i] = up | (1 << i)
        for i in rng.permutation(n)[:empty]:
            mask[b, i] = 0
    return torch.from_numpy(mask.view(np.int64)).cuda()


# ------------------------------------------------------------------------------------------------------- append and read
@pytest.mark.parametrize("dh,hkv,page,lens", [
    (64, 1, 16, [0, 1, 15, 16]), (128, 2, 16, [17, 31, 32, 33]), (128, 8, 64, [100, 0, 63, 257]), (64, 3, 128, [5, -1, 130, 300]),
    (128, 1, 1024, [1500])])
def test_append_and_read(dh, hkv, page, lens):
    rng = np.random.default_rng(dh + hkv + page)
    m = Model(rng, lens, hkv, dh, page, extra=220, gap=48)
    m.check_rows()
    at = [max(L, 0) for L in lens]
    for step in ([1] * len(lens), [int(x) for x in rng.integers(0, 40, len(lens))], [100 + 16 * i for i in range(len(lens))]):
        n = max(step)
        m.append(m.fresh(n), m.fresh(n), step, stride=1)
        at = [a + s if L >= 0 else a for a, s, L in zip(at, step, lens)]
        assert m.len.tolist() == [a if L >= 0 else L for a, L in zip(at, lens)]
        m.check_rows()
    m.check_rows(first=[int(x) for x in rng.integers(-20, 60, len(lens))], n=37)
    assert m.seen.tolist() == [10 * i + (len(m.rows[i][0]) if L >= 0 else 0) for i, L in enumerate(lens)]


def test_append_n_new_out_of_range_and_no_rows():
    m = Model(np.random.default_rng(2), [20, 3, 0], 2, 64, 16, extra=64)
    m.append(m.fresh(7), m.fresh(7), [-4, 0, 9])
    assert m.len.tolist() == [20, 3, 7]
    m.check_rows()


def test_record_layout():
    m = Model(np.random.default_rng(3), [48], 2, 128, 32)
    rec = m.c.pages[m.c.page_table[0, 1].item(), 1, 0].cpu()                 # block 2, head 1
    for kv in (0, 1):
        code, scale = _codes(m.rows[0][kv][32:48])
        t, d = np.meshgrid(np.arange(16), np.arange(128), indexing="ij")
        at = (t % 2 * 2 + d // 64) * 512 + t // 2 * 64 + d % 64 if kv == 0 else 2048 + d // 32 * 512 + d % 8 * 64 + t // 4 * 16 + d // 8 % 4 * 4 + t % 4
        assert np.array_equal(rec.numpy()[at].astype(np.float64) - 128, code[:, 1])
        assert rec[4096 + 4 * kv:4100 + 4 * kv].view(torch.float32).item() == scale[1]


def test_blocks_of_zeros_tiny_and_unfinite_values():
    m = Model(np.random.default_rng(4), [0], 3, 64, 16)
    k, v = m.fresh(64), m.fresh(64)
    k[0, 0:16, 0] = 0
    k[0, 0:16, 1] *= 2.0**-110
    k[0, 16:32, 2] *= 2.0**-97
    v[0, 33, 0, 5], v[0, 40, 1, 9] = float("inf"), NAN
    k[0, 50, 2, 0] = 3e38
    m.append(k, v, [64])
    m.check_rows()


def test_pages_beyond_four_gigabytes():
    hkv, dh, page = 1, 64, 16
    rec = 32 * dh + 16
    stride = 2_500_000_000 // 16 * 16
    if torch.cuda.mem_get_info()[0] < 3 * stride:
        pytest.skip("not enough memory")
    m = Model(np.random.default_rng(5), [0], hkv, dh, page, extra=48, spare=0)
    flat = torch.empty(2 * stride + rec, dtype=torch.uint8, device="cuda")
    pages = torch.as_strided(flat, (3, hkv, 1, rec), (stride, rec, rec, 1))
    m.c = _moa().PagedCache8(pages, m.c.k_ring, m.c.v_ring, torch.tensor([[2, 1, 0]], dtype=torch.int32, device="cuda"), m.len, page, m.seen)
    m.append(m.fresh(40), m.fresh(40), [40])
    m.check_rows()
    q, k, v = _new_rows(m, 1, 2)
    out = _moa().moa_paged8_attention(m.c, q, k, v)
    _check_attention(m, q, k, v, None, out, 1)


# ------------------------------------------------------------------------------------------------------- attention
@pytest.mark.parametrize("dh,hq,hkv,page,lens", [
    (64, 4, 4, 16, [0]), (64, 4, 2, 16, [1, 15, 16, 17]), (128, 8, 1, 32, [31, -1, 0, 33]), (128, 32, 8, 16, [2048]), (128, 7, 7, 64, [500, 3]),
    (128, 40, 4, 16, [129, 700]), (64, 128, 1, 128, [300]), (128, 16, 2, 1024, [4000, 1, 127, 128]), (64, 5, 1, 16, [25000, 1300])])
def test_one_token(dh, hq, hkv, page, lens):
    m = Model(np.random.default_rng(dh + hq + page), lens, hkv, dh, page)
    ws = m.c.workspace(1, hq)
    for _ in range(3):                                                       # the workspace is left as it was found
        q, k, v = _new_rows(m, 1, hq)
        out = torch.full((m.batch, 1, hq, dh), 7.0, dtype=BF, device="cuda")
        before = out.clone()
        _moa().moa_paged8_attention(m.c, q, k, v, out=out, ws=ws)
        _check_attention(m, q, k, v, None, out, 1, before=before)
        again = _moa().moa_paged8_attention(m.c, q, out=before.clone(), ws=ws)       # the rows are in the ring now
        assert torch.equal(again, out)
        _moa().moa_paged8_commit(m.c, 1)
        for b in range(m.batch):
            if int(m.len[b]) >= 0:
                m.keep(b, k[b].cpu(), v[b].cpu())
        m.check_rows()
    assert not bool(ws.view(torch.int32)[:ws.numel() // 4].ne(0)[:64].any())


@pytest.mark.parametrize("dh,hq,hkv,page,lens,n", [
    (64, 4, 4, 16, [5], 2), (128, 8, 2, 16, [100, 15], 3), (128, 8, 4, 32, [16, -1, 47, 0], 17), (128, 16, 4, 16, [333, 40], 61),
    (64, 8, 1, 64, [1000], 64), (128, 8, 1, 128, [1, 255, 511], 64), (128, 64, 8, 64, [600], 61), (64, 6, 2, 16, [79, 80, 81], 33)])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("room", [64, 20000])
def test_rows_of_trees(dh, hq, hkv, page, lens, n, masked, room):
    """room: slots behind the longest sequence. The kernel is chosen by the size of the cache, so both are met at all lengths."""
    rng = np.random.default_rng(n + dh + hq)
    m = Model(rng, lens, hkv, dh, page, extra=room)
    mask = _tree(rng, m.batch, n, empty=n // 5) if masked else None
    q, k, v = _new_rows(m, n, hq)
    if masked:                                                               # rows that nobody sees may hold anything
        for b in range(m.batch):
            any_word = 0
            for i in range(n):
                any_word |= _word(mask, b, i)
            for j in range(n):
                if not (any_word >> j) & 1:
                    k[b, j], v[b, j] = NAN, NAN
    out = torch.full((m.batch, n, hq, dh), 7.0, dtype=BF, device="cuda")
    before = out.clone()
    ws = m.c.workspace(n, hq)
    kk, vv = k.clone(), v.clone()
    kk[torch.isnan(kk)], vv[torch.isnan(vv)] = 0, 0
    _moa().moa_paged8_attention(m.c, q, k, v, mask=mask, out=out, ws=ws)
    _check_attention(m, q, kk, vv, mask, out, n, before=before)
    again = _moa().moa_paged8_attention(m.c, q, mask=mask, out=before.clone(), ws=ws)
    assert torch.equal(again, out)


def test_committed_slots_only():
    m = Model(np.random.default_rng(8), [0, 40, 300], 2, 128, 32, extra=10000)
    for n in (1, 5, 61):
        q = _new_rows(m, n, 8)[0]
        out = _moa().moa_paged8_attention(m.c, q, new_rows=False)
        _check_attention(m, q, None, None, None, out, 0)


@pytest.mark.parametrize("n", [1, 40])
def test_missing_pages_are_left_out(n):
    m = Model(np.random.default_rng(9), [400, 250], 2, 128, 32, extra=10000)
    m.c.page_table[0, 3], m.c.page_table[0, 0], m.c.page_table[1, 1] = -1, m.c.pages.shape[0], 1 << 30
    missing = [(0, 6), (0, 7), (0, 0), (0, 1), (1, 2), (1, 3)]
    q, k, v = _new_rows(m, n, 16)
    out = _moa().moa_paged8_attention(m.c, q, k, v)
    _check_attention(m, q, k, v, None, out, n, missing=missing)
    k2, _ = _moa().moa_paged8_read(m.c, 400, dtype=torch.float32)
    for b, blk in missing:
        assert not bool(k2[b, blk * 16:blk * 16 + 16].any())


@pytest.mark.parametrize("n", [1, 61])
def test_slots_end_with_the_table(n):
    """New rows behind the last slot are neither kept nor seen."""
    hkv = 2 if n == 1 else 8
    m = Model(np.random.default_rng(10), [94, 96], hkv, 64, 32, extra=0)
    assert m.c.slots == 96
    q, k, v = _new_rows(m, n, 16 * hkv)
    out = _moa().moa_paged8_attention(m.c, q, k, v)
    _check_attention(m, q, k, v, None, out, n)
    _moa().moa_paged8_commit(m.c, n)
    assert m.len.tolist() == [min(94 + n, 96), 96]
    m.keep(0, k[0, :2][:n].cpu(), v[0, :2][:n].cpu())
    m.check_rows()


@pytest.mark.parametrize("n", [1, 61])
@pytest.mark.parametrize("size,scale", [(60.0, None), (1e-3, 4.0), (1.0, 1e-6), (3e4, 1e-3), (1e30, 1e-30), (1e-30, 1e30)])
def test_steep_flat_large_and_small_scores(n, size, scale):
    m = Model(np.random.default_rng(11), [700, 33], 2, 128, 16, extra=64 if n == 1 else 9000)
    q, k, v = _new_rows(m, n, 16, scale=size)
    out = _moa().moa_paged8_attention(m.c, q, k, v, scale=scale or 0.0)
    _check_attention(m, q, k, v, None, out, n, scale=scale)


@pytest.mark.parametrize("n", [1, 61])
def test_blocks_of_very_different_scales(n):
    m = Model(np.random.default_rng(12), [0], 2, 128, 16, extra=600 if n == 1 else 9000)
    k, v = m.fresh(400), m.fresh(400)
    for j in range(0, 400, 16):
        v[0, j:j + 16] *= 2.0 ** float(m.rng.integers(-30, 30))
        k[0, j:j + 16] *= 2.0 ** float(m.rng.integers(-12, 2))
    v[0, 64:80] = 0
    k[0, 80:96] = 0
    m.append(k, v, [400])
    m.check_rows()
    q, kn, vn = _new_rows(m, n, 16)
    vn *= 1000
    out = _moa().moa_paged8_attention(m.c, q, kn, vn)
    _check_attention(m, q, kn, vn, None, out, n)


@pytest.mark.parametrize("size", [2.0**-60, 2.0**60])
@pytest.mark.parametrize("n", [1, 61])
def test_values_far_from_one(n, size):
    m = Model(np.random.default_rng(13), [0, 0], 1, 64, 16, extra=600 if n == 1 else 9000)
    m.append(m.fresh(300), m.fresh(300, size), [300, 170])
    q, kn, vn = _new_rows(m, n, 8)
    vn *= size
    out = _moa().moa_paged8_attention(m.c, q, kn, vn)
    _check_attention(m, q, kn, vn, None, out, n)


@pytest.mark.parametrize("hq,room", [(2, 64), (16, 64), (16, 9000)])
def test_unfinite_new_values_reach_only_the_rows_that_see_them(hq, room):
    rng = np.random.default_rng(14)
    n = 40
    m = Model(rng, [200, 31], 2, 128, 16, extra=room)
    mask = _tree(rng, 2, n)
    q, k, v = _new_rows(m, n, hq)
    v[0, 20, 1, 3], v[1, 7, 0, 100], k[1, 11, 1, 0] = float("inf"), NAN, NAN
    out = _moa().moa_paged8_attention(m.c, q, k, v, mask=mask)
    clean_k, clean_v = torch.nan_to_num(k, 0.0, 0.0, 0.0), torch.nan_to_num(v, 0.0, 0.0, 0.0)
    G = hq // 2
    for b in range(2):
        for i in range(n):
            w = _word(mask, b, i)
            for h in range(hq):
                o = out[b, i, h].float().cpu()
                bad = torch.zeros(128, dtype=torch.bool)
                if b == 0 and h // G == 1 and (w >> 20) & 1:
                    assert o[3] == float("inf")
                    bad[3] = True
                if b == 1 and h // G == 0 and (w >> 7) & 1:
                    assert torch.isnan(o[100])
                    bad[100] = True
                if b == 1 and h // G == 1 and (w >> 11) & 1:
                    assert torch.isnan(o).all()
                    bad[:] = True
                assert torch.isfinite(o[~bad]).all(), (b, i, h)
                out[b, i, h, bad.cuda()] = NAN
    seen = out.clone()
    fresh = _moa().moa_paged8_attention(m.c, q, clean_k, clean_v, mask=mask)
    same = torch.isnan(seen)
    # the scores of rows that do not see the NaN key are those of the clean call
    assert torch.equal(torch.where(same, fresh, seen), fresh)


@pytest.mark.parametrize("room", [128, 40000])
def test_a_closed_block_with_a_nan_is_nan_for_its_head_only(room):
    m = Model(np.random.default_rng(15), [0], 2, 64, 16, extra=room)
    k, v = m.fresh(64), m.fresh(64)
    v[0, 20, 1, 0] = NAN
    m.append(k, v, [64])
    for n in (1, 40):
        mask = _tree(m.rng, 1, n)
        mask[0, n - 1] = 0 if n > 1 else mask[0, n - 1]
        q, kn, vn = _new_rows(m, n, 4)
        out = _moa().moa_paged8_attention(m.c, q, kn, vn, mask=mask).float().cpu()
        assert torch.isfinite(out[:, :, :2]).all()
        rows = slice(0, n - 1) if n > 1 else slice(0, 1)
        assert torch.isnan(out[:, rows, 2:]).all()
        if n > 1:
            assert not out[:, n - 1].any()                                   # sees nothing


@pytest.mark.parametrize("room", [128, 40000])
def test_a_query_that_is_not_finite_spoils_its_own_row_only(room):
    m = Model(np.random.default_rng(16), [200], 2, 128, 16, extra=room)
    for n in (1, 61):
        q, k, v = _new_rows(m, n, 8)
        q[0, 0, 1, 5] = float("inf")
        out = _moa().moa_paged8_attention(m.c, q, k, v).float().cpu()
        assert torch.isnan(out[0, 0, 1]).all()
        out[0, 0, 1] = 0
        assert torch.isfinite(out).all()


# ------------------------------------------------------------------------------------------------------- cycles
@pytest.mark.parametrize("dh,hq,hkv,page,lens,n", [(128, 8, 2, 16, [10, 77, -1, 0], 13), (64, 16, 2, 32, [64, 15], 61), (128, 32, 8, 64, [200, 201], 64)])
def test_draft_verify_commit_cycles(dh, hq, hkv, page, lens, n):
    rng = np.random.default_rng(n)
    m = Model(rng, lens, hkv, dh, page, extra=400 if n < 60 else 6000)
    ws = m.c.workspace(n, hq)
    for cycle in range(5):
        mask = _tree(rng, m.batch, n)
        q, k, v = _new_rows(m, n, hq)
        out = _moa().moa_paged8_attention(m.c, q, k, v, mask=mask, ws=ws)
        _check_attention(m, q, k, v, mask, out, n)
        cap = n
        slot, length = torch.full((m.batch, cap), -1, dtype=torch.int32), torch.zeros(m.batch, dtype=torch.int32)
        for b in range(m.batch):
            leaf = int(rng.integers(0, n)) if cycle < 4 else n - 1
            path = [j for j in range(n) if (_word(mask, b, leaf) >> j) & 1] if cycle != 2 else list(range(n))       # all rows once
            slot[b, :len(path)] = torch.tensor(path, dtype=torch.int32)
            length[b] = len(path)
            if lens[b] >= 0:
                m.keep(b, k[b, path].cpu(), v[b, path].cpu())
        _moa().moa_paged8_commit(m.c, n, slot.cuda(), length.cuda())
        assert m.len.tolist() == [len(r[0]) if L >= 0 else L for r, L in zip(m.rows, lens)]
        m.check_rows()


def test_commit_of_leading_rows_and_without_advance():
    m = Model(np.random.default_rng(17), [30, 14], 2, 64, 16)
    q, k, v = _new_rows(m, 20, 4)
    _moa().moa_paged8_attention(m.c, q, k, v)
    kept = torch.tensor([3, 20], dtype=torch.int32, device="cuda")
    _moa().moa_paged8_commit(m.c, 20, acc_len=kept, advance=False)
    assert m.len.tolist() == [30, 14]
    end = m.len + kept
    m.keep(0, k[0, :3].cpu(), v[0, :3].cpu())
    m.keep(1, k[1].cpu(), v[1].cpu())
    got = _moa().moa_paged8_read(m.c, 40, length=end, dtype=torch.float32)
    for b in range(2):
        for x, y in zip(got, m.held(b)):
            assert torch.equal(x[b, :len(y)].cpu(), torch.from_numpy(y)) and not bool(x[b, len(y):].any())


def test_captured_decode_follows_the_lengths():
    m = Model(np.random.default_rng(18), [13, 500], 2, 128, 32, extra=100)
    ws = m.c.workspace(1, 8)
    q, k, v = _new_rows(m, 1, 8)
    out = torch.zeros((2, 1, 8, 128), dtype=BF, device="cuda")
    step = lambda: (_moa().moa_paged8_attention(m.c, q, k, v, out=out, ws=ws), _moa().moa_paged8_commit(m.c, 1))  # noqa: E731
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
    for _ in range(36):
        for dst, src in zip((q, k, v), _new_rows(m, 1, 8)):
            dst.copy_(src)
        g.replay()
        _check_attention(m, q, k, v, None, out, 1)
        for b in range(2):
            m.keep(b, k[b].cpu(), v[b].cpu())
    m.check_rows()


def test_calls_on_a_stream_of_their_own():
    m = Model(np.random.default_rng(19), [300], 2, 128, 16, extra=9000)
    n = 40
    q, k, v = _new_rows(m, n, 16)
    want = _moa().moa_paged8_attention(m.c, q, k, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda._sleep(20_000_000)                                            # a busy current stream must not matter
    got = _moa().moa_paged8_attention(m.c, q, k, v, stream=side)
    rows = _moa().moa_paged8_read(m.c, 300, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(rows[0], _moa().moa_paged8_read(m.c, 300)[0])


def test_two_caches_of_one_table_on_two_streams():
    m = Model(np.random.default_rng(20), [700, 90], 4, 64, 16)
    q, k, v = _new_rows(m, 1, 16)
    want = _moa().moa_paged8_attention(m.c, q, k, v)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [m.c.workspace(1, 16) for _ in streams]
    outs = [torch.zeros_like(want) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, w, o in zip(streams, ws, outs):
            _moa().moa_paged8_attention(m.c, q, out=o, ws=w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("hq,hkv,lens", [(16, 2, [3000, 90, 1500]), (64, 32, [2500])])
def test_a_workspace_serves_fewer_rows_and_both_kernels_in_turn(hq, hkv, lens):
    m = Model(np.random.default_rng(21), lens, hkv, 128, 64, extra=9000)
    ws = m.c.workspace(61, hq)
    for n in (61, 1, 5, 40, 61, 1, 2):
        assert m.c.workspace(n, hq).numel() <= ws.numel()
        q, k, v = _new_rows(m, n, hq)
        want = _moa().moa_paged8_attention(m.c, q, k, v)
        out = torch.full_like(want, NAN)
        assert torch.equal(_moa().moa_paged8_attention(m.c, q, k, v, out=out, ws=ws), want), n
