"""Edges of the 8-bit paged cache on the GPU: values far apart, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests.test_gpu_paged8 import Model, _attend, _bound, _moa, _new_rows, _tree, _word

pytestmark = pytest.mark.gpu


def _check_rows(m, q, k_new, v_new, mask, out, per_row=False):
    """out [batch, n, hq, dh] against the definition. per_row: "the largest scale" of the bound is that of the slots that the row sees."""
    batch, n, hq, dh = q.shape
    G = hq // m.hkv
    o, qd = out.double().cpu().numpy(), q.double().cpu().numpy()
    assert np.isfinite(o).all()
    for b in range(batch):
        K, V = (np.concatenate([x.astype(np.float64), y[b].double().cpu().numpy()]) for x, y in zip(m.held(b), (k_new, v_new)))
        L = len(K) - n
        for i in range(n):
            see = np.ones(len(K), bool)
            see[L:] = [(_word(mask, b, i) >> j) & 1 for j in range(n)]
            most = np.abs(V[see] if per_row else V).max()
            for h in range(hq):
                ref, mass, spread = _attend(qd[b, i, h], K[:, h // G], V[:, h // G], see, dh**-0.5)
                tol = _bound(dh, len(K), spread, mass, ref, most)
                assert np.all(np.abs(o[b, i, h] - ref) <= tol), (b, i, h, np.max(np.abs(o[b, i, h] - ref) - tol), np.abs(ref).max())


# ------------------------------------------------------------------------------------------------------- values far apart
# A long sequence is cut into pieces of two tiles of 128 positions: the open block's warp has a closed block in hand, too. (n, hq): few rows
# and rows of trees, by the room's size.
@pytest.mark.parametrize("n,hq", [(1, 8), (40, 4), (61, 8)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("large,small", [(2.0**19, 2.0**-99), (1e20, 1e-16), (2.0**110, 2.0**-90), (1.0, 2.0**-98), (2.0**-60, 2.0**-99), (1e-16, 1e20)])
def test_open_values_far_from_the_closed_ones(n, hq, dh, large, small):
    """New rows' values, and those of two committed rows of the open block, of one size behind closed blocks of another."""
    _far_apart(n, hq, dh, large, small)


@pytest.mark.parametrize("n,hq", [(1, 8), (40, 4), (61, 8)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("large,small", [(2.0**122, 1.0), (2.0**122, 2.0**122), (1.0, 2.0**122)])
def test_values_near_the_largest(n, hq, dh, large, small):
    """Sums of probabilities times values are divided at the end; values of up to 2^125 still do not leave fp32 on the way."""
    _far_apart(n, hq, dh, large, small)


def _far_apart(n, hq, dh, large, small):
    m = Model(np.random.default_rng(n + dh), [0, 0], 2, dh, 16, extra=5392)
    k, v = m.fresh(5314), m.fresh(5314, small)
    v[:, 5312:] = m.fresh(2, large)
    m.append(k, v, [5314, 194])
    q, kn, vn = _new_rows(m, n, hq)
    vn *= large
    mask = _tree(m.rng, 2, n)
    out = _moa().moa_paged8_attention(m.c, q, kn, vn, mask=mask)
    _check_rows(m, q, kn, vn, mask, out)


@pytest.mark.parametrize("dh", [64, 128])
def test_few_rows_keep_their_bits_beside_large_open_values(dh):
    """A tree slot with values 2^60 times the others' takes nothing off the rows that do not see it, where few rows are attended."""
    m = Model(np.random.default_rng(dh), [5309], 2, dh, 16, extra=70)
    n, large = 3, 2.0**60
    q, kn, vn = _new_rows(m, n, 8)
    vn[0, 1] *= large
    mask = torch.tensor([[0b001, 0b011, 0b101]], dtype=torch.int64, device="cuda")
    out = _moa().moa_paged8_attention(m.c, q, kn, vn, mask=mask)
    _check_rows(m, q, kn, vn, mask, out, per_row=True)


def test_infinity_among_small_open_values_before_large_closed_ones():
    """The outputs' unit passes from the open values' to the closed blocks', a factor that is zero in fp32: infinity stays what it is."""
    m = Model(np.random.default_rng(3), [0], 2, 64, 16, extra=5392)
    m.append(m.fresh(5314), m.fresh(5314, 2.0**122), [5314])
    q, kn, vn = _new_rows(m, 1, 8)
    vn *= 2.0**-60
    vn[0, 0, 1, 7] = float("inf")
    out = _moa().moa_paged8_attention(m.c, q, kn, vn).float().cpu()[0, 0]
    assert bool((out[4:, 7] == float("inf")).all())
    out[4:, 7] = 0
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dh,lens,n", [(64, [5, 0], 1), (128, [5309, 13], 1), (64, [30, 2000], 3)])
def test_tiny_open_values_keep_their_bits_where_few_rows_are_attended(dh, lens, n):
    """Values of 2^-108 behind closed blocks that are held as zeros."""
    m = Model(np.random.default_rng(dh + n), [0] * len(lens), 2, dh, 16, extra=max(lens) + 70)
    if max(lens):
        m.append(m.fresh(max(lens)), m.fresh(max(lens), 2.0**-108), lens)
    q, kn, vn = _new_rows(m, n, 8)
    vn *= 2.0**-108
    out = _moa().moa_paged8_attention(m.c, q, kn, vn)
    _check_rows(m, q, kn, vn, None, out)


# ------------------------------------------------------------------------------------------------------- rows read back
@pytest.mark.parametrize("dh,hkv,lens,cut", [(64, 2, [40, 7, 160], [33, 3, 90]), (128, 3, [95, -1, 300], [16, 5, 17]), (128, 1, [64, 81, 200], [0, 80, 199])])
def test_fewer_rows_than_are_committed(dh, hkv, lens, cut):
    """The rows of a prefix that ends inside a closed block, as they stand for; a block with NaN behind the prefix's end leaves zeros there."""
    m = Model(np.random.default_rng(dh + hkv), [min(L, 0) for L in lens], hkv, dh, 16, extra=320)
    k, v = m.fresh(max(lens)), m.fresh(max(lens))
    m.append(k, v, lens)
    n = max(lens) + 5
    for first in (None, [11, -3, 2]):
        f = [0, 0, 0] if first is None else first
        for dt in (torch.float32, torch.bfloat16):
            got = _moa().moa_paged8_read(m.c, n, first=None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda"),
                                         length=torch.tensor(cut, dtype=torch.int32, device="cuda"), dtype=dt)
            for b, L in enumerate(lens):
                for x, y in zip(got, m.held(b)):
                    want, at = torch.zeros((n, hkv, dh), dtype=dt), torch.arange(n) + f[b]
                    ok = (at >= 0) & (at < cut[b]) & (L >= 0)
                    want[ok] = torch.from_numpy(y)[at[ok]].to(dt)
                    assert torch.equal(x[b].cpu(), want), (b, f[b], dt)


def test_a_prefix_of_a_block_that_holds_a_nan():
    m = Model(np.random.default_rng(5), [0], 2, 64, 16)
    k, v = m.fresh(32), m.fresh(32)
    v[0, 20, 1, 3] = float("nan")
    m.append(k, v, [32])
    _, got = _moa().moa_paged8_read(m.c, 32, length=torch.tensor([18], dtype=torch.int32, device="cuda"))
    assert bool(torch.isnan(got[0, 16:18, 1]).all()) and not bool(got[0, 18:].any()) and bool(torch.isfinite(got[0, :, 0]).all())


# ------------------------------------------------------------------------------------------------------- lengths
@pytest.mark.parametrize("back", [0, 16, 48, 96])
def test_a_length_lowered_to_a_multiple_of_16(back):
    m = Model(np.random.default_rng(back), [0, 0], 2, 64, 16, extra=400)
    m.append(m.fresh(107), m.fresh(107), [107, 99])
    m.len.fill_(back)
    m.rows = [tuple(x[:back] for x in r) for r in m.rows]
    m.check_rows()
    for n in (1, 30):
        q, k, v = _new_rows(m, n, 8)
        mask = _tree(m.rng, 2, n)
        out = _moa().moa_paged8_attention(m.c, q, k, v, mask=mask)
        _check_rows(m, q, k, v, mask, out)
        _moa().moa_paged8_commit(m.c, n)
        for b in range(2):
            m.keep(b, k[b].cpu(), v[b].cpu())
        m.check_rows()


@pytest.mark.parametrize("dh,hkv", [(64, 3), (128, 8)])
@pytest.mark.parametrize("lens,rows", [([5, 5, 5], [75, 78, 82]), ([15, 15, 15], [65, 79, 80]), ([1, 20, 33], [95, 60 + 16, 79]), ([79, 80, 81], [1 + 15, 80, 79])])
def test_appended_rows_that_stay_open_where_the_open_block_lay(lens, rows, dh, hkv):
    """The ring has 80 rows: a prompt's last rows take the places of those that the same call closes a block with."""
    m = Model(np.random.default_rng(dh + sum(rows)), lens, hkv, dh, 16, extra=300)
    for _ in range(2):
        m.append(m.fresh(max(rows)), m.fresh(max(rows)), rows)
        m.check_rows()
        q, k, v = _new_rows(m, 1, 2 * hkv)
        out = _moa().moa_paged8_attention(m.c, q, k, v)
        _check_rows(m, q, k, v, None, out)


# ------------------------------------------------------------------------------------------------------- workspaces and streams
def _counters(ws):
    return ws.view(torch.int32)[:2 * torch.cuda.get_device_properties(0).multi_processor_count]


@pytest.mark.parametrize("dh,hq,hkv,lens,n", [
    (128, 8, 8, [30000], 1), (64, 4, 1, [60000], 1), (64, 128, 1, [20000, 300], 1), (128, 16, 2, [9000, 1, 777], 1), (64, 8, 2, [3000] * 40, 1),
    (128, 16, 4, [5000, 300], 3), (128, 16, 4, [5000, 300], 61), (64, 64, 32, [2500], 40)])
def test_every_join_counter_is_zero_between_calls(dh, hq, hkv, lens, n):
    m = Model(np.random.default_rng(n + hq), lens, hkv, dh, 64)
    ws = m.c.workspace(n, hq)
    q, k, v = _new_rows(m, n, hq)
    want = None
    for _ in range(3):
        out = _moa().moa_paged8_attention(m.c, q, k, v, ws=ws)
        assert not bool(_counters(ws).any())
        assert want is None or torch.equal(out, want)                # the order in which pieces come in changes nothing
        want = out


@pytest.mark.parametrize("n", [1, 40])
def test_two_layers_of_one_table_on_two_streams(n):
    """Two caches of the same table and lengths, each with pages and rings of its own, appended to, attended and committed at the same time."""
    moa, lens, hkv, dh, page, hq = _moa(), [700, 90], 4, 64, 16, 16
    a = Model(np.random.default_rng(20), [0, 0], hkv, dh, page, extra=9000)
    layers = [a.c] + [moa.PagedCache8(torch.zeros_like(a.c.pages), torch.zeros_like(a.c.k_ring), torch.zeros_like(a.c.v_ring), a.c.page_table, a.len, page)]
    prompt = [tuple(x.cuda() for x in (a.fresh(700), a.fresh(700))) for _ in layers]
    count, grown = torch.tensor(lens, dtype=torch.int32, device="cuda"), a.len.clone()
    rows, mask = [_new_rows(a, n, hq) for _ in layers], _tree(a.rng, 2, n)
    ws = [c.workspace(n, hq) for c in layers]
    streams = [torch.cuda.Stream() for _ in layers]

    def run(side):
        for c in layers:
            for t in (c.pages, c.k_ring, c.v_ring):
                t.zero_()
        a.len.copy_(grown)
        torch.cuda.synchronize()
        st = streams if side else [None, None]
        for c, (k, v), s in zip(layers, prompt, st):
            moa.moa_paged8_append(c, k, v, count, advance=False, stream=s)
        torch.cuda.synchronize()
        a.len.copy_(count)
        torch.cuda.synchronize()
        outs = []
        for _ in range(5):
            for c, (q, k, v), w, s in zip(layers, rows, ws, st):
                outs.append(moa.moa_paged8_attention(c, q, k, v, mask=mask, ws=w, stream=s))
        for c, s in zip(layers, st):
            moa.moa_paged8_commit(c, n, advance=False, stream=s)
        torch.cuda.synchronize()
        a.len.add_(n)
        return outs + [x for c in layers for x in moa.moa_paged8_read(c, 800)]

    want, got = run(False), run(True)
    for x, y in zip(want, got):
        assert torch.equal(x, y)
    assert not torch.equal(want[0], want[1])
