"""Page plans and the norm and rotation of queries and keys on the GPU against plain definitions, and a serving loop of all of them."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

T = {"bf16": torch.bfloat16, "f32": torch.float32}


def _moa():
    from paper_2410_03804_b200 import moa
    return moa


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------------- page plans
class Pool:
    """The definition, one sequence after another."""

    def __init__(self, batch, per, n_pages, page):
        self.per, self.page, self.n = per, page, n_pages
        self.table, self.free = [[] for _ in range(batch)], list(range(n_pages - 1, -1, -1))

    def plan(self, lens, new, max_rows=None, seen=None):
        new = [max(0, x) for x in new]
        want = [0 if L < 0 else -(-(L + n) // self.page) for L, n in zip(lens, new)]
        for b, w in enumerate(want):
            self.free += self.table[b][w:]
            del self.table[b][w:]
        have, asked, used = len(self.free), 0, 0
        rows, start = [], []
        for b, w in enumerate(want):
            need = max(0, w - len(self.table[b])) if lens[b] >= 0 and w <= self.per else 0
            asked += need
            ok = lens[b] >= 0 and w <= self.per and (need == 0 or asked <= have)
            if ok:
                used += new[b]
                ok = max_rows is None or used <= max_rows
            start.append(sum(rows))
            rows.append(new[b] if ok else 0)
            if ok:
                self.table[b] += [self.free.pop() for _ in range(need)]
        start.append(sum(rows))
        maps = [[], [], []]
        if max_rows is not None:
            for b, n in enumerate(rows):
                for i in range(n):
                    s = lens[b] + i
                    maps[0].append(b)
                    maps[1].append((lens if seen is None else seen)[b] + i)
                    maps[2].append(self.table[b][s // self.page] * self.page + s % self.page)
            for x in maps:
                x += [-1] * (max_rows - len(x))
        return rows, start, maps


def _check_pool(p, ref):
    per = p.page_table.shape[1]
    assert p.held.tolist() == [len(t) for t in ref.table]
    assert p.page_table.tolist() == [t + [-1] * (per - len(t)) for t in ref.table]
    n = int(p.free_count)
    assert n == len(ref.free) and p.free_pages[:n].tolist() == ref.free


def _check_maps(maps, want):
    rows, start, m = want
    assert maps[0].tolist() == rows and maps[1].tolist() == start
    for got, x in zip(maps[2:], m):
        assert (got is None and not x) or got.tolist() == x


@pytest.mark.parametrize("batch,per,n_pages,page,max_rows,seed", [
    (1, 1, 1, 16, 1, 0), (3, 4, 7, 1, 9, 1), (64, 40, 900, 16, 300, 2), (17, 100, 1000, 32, 20000, 3), (64, 700, 30000, 16, 9000, 4), (5, 9, 20, 1024, None, 5),
    (64, 300, 17000, 8, None, 6), (64, 100, 3000, 16, 2500, 7), (2, 9, 9, 4, 60, 8)])
def test_plans_of_a_changing_batch(batch, per, n_pages, page, max_rows, seed):
    """Requests come, grow, shrink and end; some do not fit. In place, and to a second pool, alternately."""
    rng = np.random.default_rng(seed)
    ref = Pool(batch, per, n_pages, page)
    p = _moa().PagePool.make(batch, per, n_pages, page)
    other = _moa().PagePool(*(torch.full_like(t, 99) for t in (p.page_table, p.held, p.free_pages, p.free_count)), page)
    lens = [-1] * batch
    for step in range(12):
        for b in range(batch):
            x = rng.random()
            if lens[b] < 0 and x < 0.6:
                lens[b] = 0
            elif lens[b] >= 0 and x < 0.15:
                lens[b] = -1
            elif lens[b] > 0 and x < 0.3:
                lens[b] = int(rng.integers(0, lens[b] + 1))          # an eviction
        new = [int(x) for x in rng.choice([-1, 0, 1, 1, 1, 13, 61, per * page // 2 + 1, per * page + 1], batch)]
        seen = [max(L, 0) + 3 * b for b, L in enumerate(lens)] if step % 2 else None
        want = ref.plan(lens, new, max_rows, seen)
        kw = dict(max_rows=max_rows or 0, seen=None if seen is None else _i32(seen))
        if step % 3 == 2:
            before = [t.clone() for t in (p.page_table, p.held, p.free_count)]
            maps = _moa().moa_page_plan(p, _i32(lens), _i32(new), pool_out=other, **kw)
            assert all(torch.equal(a, t) for a, t in zip(before, (p.page_table, p.held, p.free_count)))
            p, other = other, p
        else:
            maps = _moa().moa_page_plan(p, _i32(lens), _i32(new), **kw)
        _check_pool(p, ref)
        _check_maps(maps, want)
        lens = [L + n if L >= 0 else L for L, n in zip(lens, want[0])]


@pytest.mark.parametrize("per", [100, 1000])
@pytest.mark.parametrize("second", [False, True])
def test_pages_that_come_back_are_taken_in_the_same_call(per, second):
    """Half of the batch gives all of its pages to the other half, over and over: every page is read, put back and taken at once."""
    batch, page = 64, 8
    ref, p, other = Pool(batch, per, batch // 2 * per, page), *(_moa().PagePool.make(batch, per, batch // 2 * per, page) for _ in range(2))
    for step in range(20):
        lens = [-1 if (b + step) % 2 else 0 for b in range(batch)]
        new = [per * page] * batch
        want = ref.plan(lens, new)
        _moa().moa_page_plan(p, _i32(lens), _i32(new), pool_out=other if second else None)
        if second:
            p, other = other, p
        _check_pool(p, ref)
        assert want[0] == [0 if L < 0 else per * page for L in lens]
        assert sorted(p.free_pages.tolist()) == list(range(batch // 2 * per))       # what was taken is still there, behind the count


def test_plan_without_counts_gives_a_row_each():
    p = _moa().PagePool.make(3, 4, 12, 16)
    ref = Pool(3, 4, 12, 16)
    maps = _moa().moa_page_plan(p, _i32([15, -1, 16]), max_rows=4)
    _check_maps(maps, ref.plan([15, -1, 16], [1, 1, 1], 4))
    _check_pool(p, ref)


def test_plan_nobody_overtakes_who_waits_and_others_go_on():
    p, ref = _moa().PagePool.make(4, 8, 10, 16), Pool(4, 8, 10, 16)
    for lens, new in (([0, 0, 0, 0], [16, 32, 16, 48]), ([16, 32, 16, 48], [1, 80, 17, 0]), ([17, 32, 16, 48], [1, 1, 17, 0]), ([17, 32, -1, 48], [1, 200, 1, 1])):
        _check_maps(_moa().moa_page_plan(p, _i32(lens), _i32(new), max_rows=200), ref.plan(lens, new, 200))
        _check_pool(p, ref)


def test_plan_of_the_largest_batch_and_sizes_that_pass_32_bits():
    """64 prompts whose needs together pass 32 bits wait; maps of many rows take the second kernel."""
    page, per = 1, 1 << 26
    p = _moa().PagePool(torch.full((2, per), -1, dtype=torch.int32, device="cuda"), _i32([0, 0]), torch.arange(50000, dtype=torch.int32, device="cuda"), _i32([50000]), page)
    big = (1 << 31) - 1
    maps = _moa().moa_page_plan(p, _i32([big - 1, 0]), _i32([big, 40000]), max_rows=60000)
    assert maps[0].tolist() == [0, 40000] and p.held.tolist() == [0, 40000] and int(p.free_count) == 10000
    assert torch.equal(maps[4][:40000], torch.arange(49999, 9999, -1, device="cuda")) and bool((maps[4][40000:] == -1).all())
    assert torch.equal(p.page_table[1, :40000].long(), maps[4][:40000])


def test_plan_captured_and_replayed():
    p, ref = _moa().PagePool.make(4, 20, 60, 16), Pool(4, 20, 60, 16)
    lens = _i32([0, 5, -1, 40])
    new = _i32([1, 1, 1, 1])
    maps = _moa().moa_page_plan(_moa().PagePool.make(4, 20, 60, 16), lens, new, max_rows=70)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            _moa().moa_page_plan(p, lens, new, maps=maps)
    for L, n in (([0, 5, -1, 40], [3, 61, 9, 1]), ([3, 66, 0, -1], [1, 1, 30, 1]), ([4, -1, 30, -1], [1, 1, 1, 1])):
        lens.copy_(_i32(L))
        new.copy_(_i32(n))
        g.replay()
        _check_maps(maps, ref.plan(L, n, 70))
        _check_pool(p, ref)


# ------------------------------------------------------------------------------------------------------- norm and rotation
def _turned(x, gain, pos, freq, inter, eps):
    """[rows, heads, dh] in float64."""
    x = x.double().cpu()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double().cpu()
    if freq is None:
        return x
    rot = 2 * len(freq)
    a = pos.double().cpu()[:, None] * freq.cpu()
    turn = torch.polar(torch.ones_like(a), a)[:, None]
    y = x.clone()
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(x[..., i].contiguous(), x[..., j].contiguous()) * turn
    y[..., i], y[..., j] = z.real, z.imag
    return y


def _near(got, want, x, gain, eps, dtype):
    """Half a step of the output's type, and 40 steps of fp32 (2^-24 each) of the largest element that took part: the sum of squares has
    head_dim additions whose errors are halved by the root (64 at most for 128, and far less since its terms are positive and
    summed in a tree: 3 + 4 levels), the root 2 ulp, gain, cosine and sine 1 to 2 ulp each, the angle 2^-24 of a turn / 2 pi."""
    size = want.abs().amax(-1, keepdim=True)
    tol = (2.0**-8 if dtype == "bf16" else 2.0**-24) * want.abs() + 40 * 2.0**-24 * size
    d = (got.double().cpu() - want).abs()
    assert bool((d <= tol).all()), float((d - tol).max())


def _rows(rng, rows, hq, hkv, dh, dtype):
    g = torch.Generator().manual_seed(int(rng.integers(1 << 30)))
    x = torch.randn((rows, hq + 2 * hkv, dh), generator=g)
    x[..., ::9] *= 20
    x = x.to(T[dtype]).cuda()
    gains = [(1 + 0.2 * torch.randn(dh, generator=g)).to(T[dtype]).cuda() for _ in range(2)]
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], gains


def _freq(rot, theta=500000.0):
    return theta ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot) if rot else None


@pytest.mark.parametrize("rows,hq,hkv,dh", [(1, 1, 1, 64), (1, 32, 8, 128), (7, 5, 3, 64), (61, 64, 8, 128), (300, 4, 4, 64), (5000, 9, 1, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot,inter,norm", [(1.0, False, True), (0.5, False, True), (1.0, True, True), (0.25, True, False), (0.0, False, True), (1.0, False, False)])
def test_norm_and_rotation(rows, hq, hkv, dh, dtype, rot, inter, norm):
    rng = np.random.default_rng(rows + dh)
    q, k, _, gains = _rows(rng, rows, hq, hkv, dh, dtype)
    rot = int(rot * dh)
    pos, freq = _i32(rng.integers(0, 1 << 20, rows).tolist()), _freq(rot)
    gains = gains if norm else (None, None)
    qo, ko = _moa().moa_qk_norm_rope(q, k, pos, freq, *gains, eps=1e-5, interleaved=inter)
    for got, x, g in ((qo, q, gains[0]), (ko, k, gains[1])):
        _near(got, _turned(x, g, pos, freq, inter, 1e-5), x, g, 1e-5, dtype)
    if rot < dh and not norm:
        assert torch.equal(qo[..., rot:], q[..., rot:])              # what neither turns nor is normalised passes bit for bit
    # in place
    q2, k2 = q.clone(), k.clone()
    big = torch.cat([q2, k2], 1)
    qi, ki = big[:, :hq], big[:, hq:]
    _moa().moa_qk_norm_rope(qi, ki, pos, freq, *gains, eps=1e-5, interleaved=inter, q_out=qi, k_out=ki)
    assert torch.equal(qi, qo) and torch.equal(ki, ko)


def test_positions_at_the_end_of_int32():
    rng = np.random.default_rng(1)
    q, k, _, gains = _rows(rng, 4, 2, 2, 128, "f32")
    pos, freq = _i32([0, 1, 2**31 - 1, 2**30 + 7]), _freq(128, 10000.0)
    qo, _ = _moa().moa_qk_norm_rope(q, k, pos, freq, *gains)
    # the angle's 64-bit product is off by 2^-53 of 2^31 radians, twice: 2^-21, far below the 40 steps only for small positions
    want = _turned(q, gains[0], pos, freq, False, 1e-5)
    size = want.abs().amax(-1, keepdim=True)
    assert bool(((qo.double().cpu() - want).abs() <= (40 * 2.0**-24 + 2.0**-20) * size).all())


def test_padding_and_zero_and_unfinite_rows():
    rng = np.random.default_rng(2)
    q, k, _, gains = _rows(rng, 9, 6, 2, 64, "bf16")
    q[4], q[5, 2, 7], k[6, 0, 0] = 0, float("nan"), float("inf")
    pos = _i32([3, -1, 5, -7, 8, 9, 10, 11, -1])
    qo, ko = torch.full_like(q, 5.0), torch.full_like(k, 5.0)
    _moa().moa_qk_norm_rope(q, k, pos, _freq(64), *gains, q_out=qo, k_out=ko)
    for r in (1, 3, 8):
        assert bool((qo[r] == 5).all()) and bool((ko[r] == 5).all())
    assert not bool(qo[4].any())
    assert bool(torch.isnan(qo[5, 2]).all()) and bool(torch.isfinite(qo[5, [0, 1, 3, 4, 5]]).all())
    assert bool(torch.isfinite(ko[6, 1]).all()) and not bool(torch.isfinite(ko[6, 0]).all())
    assert bool(torch.isfinite(qo[6]).all())
    # without norm a value that does not turn keeps what is not finite to itself
    q[5, 2, 40] = float("nan")
    qo, _ = _moa().moa_qk_norm_rope(q, k, pos, _freq(32))
    assert torch.isnan(qo[5, 2]).nonzero().flatten().tolist() == [7, 23, 40]


@pytest.mark.parametrize("dtype,dh,hkv,page,gap", [("bf16", 128, 8, 16, False), ("f32", 64, 3, 64, True), ("bf16", 64, 1, 1, False)])
def test_keys_and_values_to_their_pages(dtype, dh, hkv, page, gap):
    rng = np.random.default_rng(page)
    rows, n_pages, hq = 50, 70, 2 * hkv
    q, k, v, gains = _rows(rng, rows, hq, hkv, dh, dtype)
    shape = (n_pages, 2, page, hkv, dh) if gap else (2, n_pages, page, hkv, dh)
    both = torch.full(shape, 3.0, dtype=T[dtype], device="cuda")
    pk, pv = (both[:, 0], both[:, 1]) if gap else (both[0], both[1])
    cache = _moa().PagedCache(pk, pv, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), _i32([0]))
    slot = torch.from_numpy(rng.permutation(n_pages * page)[:rows].astype(np.int64)).cuda()
    pos = _i32(rng.integers(0, 5000, rows).tolist())
    slot[7], slot[9], slot[11], pos[13] = -1, n_pages * page, 1 << 40, -1
    want_k, want_v = pk.clone(), pv.clone()
    qo, none = _moa().moa_qk_norm_rope(q, k, pos, _freq(dh), *gains, cache=cache, slot=slot, v=v)
    assert none is None
    qr, kr = _moa().moa_qk_norm_rope(q, k, pos, _freq(dh), *gains)
    keep = [r for r in range(rows) if r not in (7, 9, 11, 13)]
    s = slot[keep]
    want_k[s // page, s % page], want_v[s // page, s % page] = kr[keep], v[keep]
    assert torch.equal(pk, want_k) and torch.equal(pv, want_v) and torch.equal(qo, qr)


# ------------------------------------------------------------------------------------------------------- all of them together
@pytest.mark.parametrize("eight", [False, True])
def test_a_serving_loop(eight):
    """Requests of uneven prompts come, are decoded and end: pages planned, rows normalised, rotated and appended, attended, committed. Checked
    against attention in 64 bits over every row that a request ever had (8-bit rows as the cache holds them)."""
    moa = _moa()
    rng = np.random.default_rng(30)
    batch, per, page, hq, hkv, dh = 4, 8, 16, 8, 2, 64
    pool = moa.PagePool.make(batch, per, 22, page)
    length, seen = _i32([-1] * batch), _i32([0] * batch)
    freq = _freq(dh)
    gains = [(1 + 0.2 * torch.randn(dh, generator=torch.Generator().manual_seed(i))).bfloat16().cuda() for i in range(2)]
    if eight:
        cache = moa.PagedCache8.make(pool.page_table, length, 22, page, hkv, dh, seen=seen)
    else:
        k, v = (torch.zeros((22, page, hkv, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        cache = moa.PagedCache(k, v, pool.page_table, length)
    ws = cache.workspace(1, hq)
    rows = [[] for _ in range(batch)]                                # (key as it is held, value) in float64

    def project(n):
        x = torch.randn((n, hq + 2 * hkv, dh), generator=torch.Generator().manual_seed(int(rng.integers(1 << 30)))).bfloat16().cuda()
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]

    plan = {0: [(0, 20), (1, 33)], 3: [(2, 1)], 5: [(3, 40)], 9: [(0, 50)]}
    ends = {7: [0], 12: [1]}
    for step in range(15):
        for b in ends.get(step, ()):
            length[b] = -1
            rows[b] = []
        fresh = dict(plan.get(step, ()))
        for b in fresh:
            length[b], seen[b] = 0, 0
        # prompts: all their rows in one packed batch; their attention among themselves is not this test's
        if fresh:
            new = [fresh.get(b, 0) for b in range(batch)]
            maps = moa.moa_page_plan(pool, length, _i32(new), max_rows=sum(new) + 5, seen=seen)
            assert maps[0].tolist() == new
            q, k, v = project(sum(new) + 5)
            if eight:
                _, ko = moa.moa_qk_norm_rope(q, k, maps[3], freq, *gains)
                kn, vn = (torch.zeros((batch, max(new), hkv, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
                for b, n in enumerate(new):
                    kn[b, :n], vn[b, :n] = ko[maps[1][b]:maps[1][b] + n], v[maps[1][b]:maps[1][b] + n]
                moa.moa_paged8_append(cache, kn, vn, _i32(new))
            else:
                moa.moa_qk_norm_rope(q, k, maps[3], freq, *gains, cache=cache, slot=maps[4], v=v)
                length += torch.where(length >= 0, maps[0], 0)
                seen += maps[0]
                _, ko = moa.moa_qk_norm_rope(q, k, maps[3], freq, *gains)
            for b, n in enumerate(new):
                at = int(maps[1][b])
                rows[b] += [(ko[at + i].double().cpu(), v[at + i].double().cpu()) for i in range(n)]
        # one token each
        maps = moa.moa_page_plan(pool, length, max_rows=batch, seen=seen)
        live = [b for b in range(batch) if int(length[b]) >= 0]
        assert maps[0].tolist() == [1 if b in live else 0 for b in range(batch)]
        x = project(batch)
        q, k = moa.moa_qk_norm_rope(x[0], x[1], seen, freq, *gains)
        call = moa.moa_paged8_attention if eight else moa.moa_paged_attention
        out = call(cache, q[:, None], k[:, None], x[2][:, None].contiguous(), ws=ws)
        for b in live:
            rows[b].append((k[b].double().cpu(), x[2][b].double().cpu()))
            K, V = (torch.stack([r[i] for r in rows[b]]) for i in (0, 1))
            if eight:                                                # blocks that were closed before this token, by the documented fp32 steps
                for j in range(0, (len(K) - 1) // 16 * 16, 16):
                    for t in (K, V):
                        x32 = t[j:j + 16].float()
                        top = x32.abs().amax((0, 2), keepdim=True)
                        most = torch.full_like(top, 127.0)           # (tensor by tensor: rounded once)
                        t[j:j + 16] = torch.round(x32 * (most / top)).double() * (top / most).double()
            z = torch.einsum("hgd,shd->hgs", q[b].double().cpu().reshape(hkv, hq // hkv, dh), K) * dh**-0.5
            p = torch.softmax(z, -1)
            want = torch.einsum("hgs,shd->hgd", p, V).reshape(hq, dh)
            mass = torch.einsum("hgs,shd->hgd", p, V.abs()).reshape(hq, dh)
            # half a step of bf16; probabilities to 2^-11 of themselves, and as much for scores summed in fp32 (64 products of at most some tens)
            over = float(((out[b, 0].double().cpu() - want).abs() - 2.0**-8 * want.abs() - 2.0**-10 * mass).max())
            assert over <= 0, (step, b, len(K), over)
        if eight:
            moa.moa_paged8_commit(cache, 1)
        else:
            moa.moa_paged_commit(cache, 1)
            seen += (length >= 0).int()
        assert length.tolist() == [len(rows[b]) if b in live else -1 for b in range(batch)]


@pytest.mark.parametrize("second", [False, True])
@pytest.mark.parametrize("batch,per,n_pages,page,max_rows", [(64, 700, 30000, 16, 9000), (64, 3000, 100000, 16, 40000), (3, 4, 7, 1, 9)])
def test_granted_rows_over_the_numbers_asked_for(batch, per, n_pages, page, max_rows, second):
    """rows may be n_new: every sum is made of what was asked for, whichever CTA writes first."""
    rng = np.random.default_rng(batch + per)
    ref, p, other = Pool(batch, per, n_pages, page), *(_moa().PagePool.make(batch, per, n_pages, page) for _ in range(2))
    lens, new = [0] * batch, torch.zeros(batch, dtype=torch.int32, device="cuda")
    maps = (new,) + _moa().moa_page_plan(_moa().PagePool.make(batch, per, n_pages, page), _i32(lens), _i32([0] * batch), max_rows=max_rows)[1:]
    for step in range(20):
        lens = [0 if L > per * page // 2 else L for L in lens]
        ask = [int(x) for x in rng.choice([0, 1, 61, 500, per * page // 3], batch)]
        want = ref.plan(lens, ask, max_rows)
        new.copy_(_i32(ask))
        _moa().moa_page_plan(p, _i32(lens), new, pool_out=other if second else None, maps=maps)
        if second:
            p, other = other, p
        _check_pool(p, ref)
        _check_maps(maps, want)
        lens = [L + n for L, n in zip(lens, want[0])]


def test_results_between_the_rows_that_are_read():
    """Results in columns of their own of the buffer that holds the projection, and in place."""
    rng = np.random.default_rng(40)
    for rows in (1, 90):
        q, k, _, gains = _rows(rng, rows, 6, 2, 64, "bf16")
        pos = _i32(rng.integers(0, 5000, rows).tolist())
        want = _moa().moa_qk_norm_rope(q, k, pos, _freq(64), *gains)
        x = torch.zeros((rows, 16, 64), dtype=torch.bfloat16, device="cuda")
        x[:, 2:8], x[:, 12:14] = q, k
        got = _moa().moa_qk_norm_rope(x[:, 2:8], x[:, 12:14], pos, _freq(64), *gains, k_out=x[:, 14:16])
        assert torch.equal(got[0], want[0]) and torch.equal(x[:, 14:16], want[1]) and torch.equal(x[:, 2:8], q) and torch.equal(x[:, 12:14], k)
        _moa().moa_qk_norm_rope(x[:, 2:8], x[:, 12:14], pos, _freq(64), *gains, q_out=x[:, 2:8], k_out=x[:, :2])
        assert torch.equal(x[:, 2:8], want[0]) and torch.equal(x[:, :2], want[1])


@pytest.mark.parametrize("second", [False, True])
def test_needs_that_together_pass_32_bits(second):
    """64 sequences of which each would fit, 2^26 pages each: the sums pass 2^31 at the 33rd and come to 2^32 - 2^26 + 5 at the last.
    There are pages for the first one's five rows only."""
    batch, page, per, free = 64, 1, 1 << 26, 50000
    if torch.cuda.mem_get_info()[0] < (2 if second else 1) * batch * per * 4 + (4 << 30):
        pytest.skip("not enough memory")
    new = lambda: _moa().PagePool(torch.full((batch, per), -1, dtype=torch.int32, device="cuda"), _i32([0] * batch),  # noqa: E731
                                  torch.arange(free, dtype=torch.int32, device="cuda"), _i32([free]), page)
    p, other = new(), new() if second else None
    ask = [5] + [per] * 63
    maps = _moa().moa_page_plan(p, _i32([0] * batch), _i32(ask), max_rows=1000, pool_out=other)
    p = other or p
    assert maps[0].tolist() == [5] + [0] * 63 and maps[1].tolist() == [0] + [5] * 64
    assert p.held.tolist() == [5] + [0] * 63 and int(p.free_count) == free - 5
    assert p.page_table[0, :6].tolist() == [free - 1 - i for i in range(5)] + [-1] and bool((p.page_table[1:, 0] == -1).all())


@pytest.mark.parametrize("second", [False, True])
def test_rows_that_together_pass_31_bits(second):
    """Sequences that hold all of their pages already: without maps the rows are bounded by what row_start can hold, 2^31 - 1."""
    batch, page, per = 6, 1024, 1 << 20
    new = lambda: _moa().PagePool(torch.arange(batch * per, dtype=torch.int32, device="cuda").reshape(batch, per), _i32([per] * batch),  # noqa: E731
                                  torch.arange(batch * per, dtype=torch.int32, device="cuda"), _i32([0]), page)
    p, other = new(), new() if second else None
    many = (1 << 30) - 1
    maps = _moa().moa_page_plan(p, _i32([1, 0, 5, 1, 0, -1]), _i32([many, many, 1, many, many, 7]), pool_out=other)
    # 2^31 - 2 rows, one more, and no room for any behind it; the last one is not in use and gives its pages back
    assert maps[0].tolist() == [many, many, 1, 0, 0, 0] and maps[1].tolist() == [0, many, 2 * many] + [2 * many + 1] * 4
    p = other or p
    assert p.held.tolist() == [per, per, 1, per, per, 0] and int(p.free_count) == 2 * per - 1
    assert torch.equal(p.free_pages[:2 * per - 1].long(), torch.cat([torch.arange(2 * per + 1, 3 * per), torch.arange(5 * per, 6 * per)]).cuda())
