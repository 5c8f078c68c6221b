"""A captured step of a drafting loop over the 8-bit cache, replayed while requests come, grow, wait for pages and end."""
import numpy as np
import pytest
import torch

from tests.test_gpu_paged8 import _bound, _held, _moa
from tests.test_gpu_plan_norm import Pool, _check_pool, _freq, _i32, _near, _turned

pytestmark = pytest.mark.gpu

BATCH, PAGE, HQ, HKV, DH, N, VOCAB, CAP = 3, 16, 16, 2, 64, 13, 97, 8


def _tree(rng):
    """tok, parent, depth [N] of a random tree; the last slots may be unused."""
    used = int(rng.integers(1, N + 1))
    parent, depth = [-1] * N, [0] * N
    for i in range(1, used):
        parent[i] = int(rng.integers(0, i))
        depth[i] = depth[parent[i]] + 1
    return [int(x) for x in rng.integers(0, VOCAB, N)], parent, depth, used


def _accepted(tok, parent, used, score):
    """The path from the root along the arg-max children, CAP slots at most."""
    path = [0]
    while len(path) < CAP:
        best = int(np.argmax(score[path[-1]]))
        child = [c for c in range(1, used) if parent[c] == path[-1] and tok[c] == best]
        if not child:
            break
        path.append(child[0])
    return path


def _check_rows(o, q, K, V, see):
    """o, q [N, HQ, DH]; K, V [keys, HKV, DH]; see [N, keys]: softmax attention in 64 bits, zeros for a row that sees nothing."""
    K, V = (np.repeat(t, HQ // HKV, 1) for t in (K, V))
    z = np.where(see[:, None], np.einsum("nhd,khd->nhk", q, K) * DH**-0.5, -np.inf)
    blind = ~see.any(1)
    p = np.exp(z - np.where(blind[:, None, None], 0, z.max(-1, keepdims=True)))
    p /= np.where(blind[:, None, None], 1, p.sum(-1, keepdims=True))
    want, mass = (np.einsum("nhk,khd->nhd", p, t) for t in (V, np.abs(V)))
    spread = np.where(see[:, None], np.einsum("nhd,khd->nhk", np.abs(q), np.abs(K)), 0).max(-1)[..., None] * DH**-0.5
    assert not o[blind].any()
    assert np.all(np.abs(o - want) <= _bound(DH, len(K), spread, mass, want, np.abs(V).max()))


@pytest.mark.parametrize("per", [24, 600])                           # few rows' kernel, tensor memory: chosen by the table's size
def test_a_captured_drafting_step(per):
    moa, rng = _moa(), np.random.default_rng(per)
    n_pages = 14                                                     # too few from time to time
    pool, ref = moa.PagePool.make(BATCH, per, n_pages, PAGE), Pool(BATCH, per, n_pages, PAGE)
    length, seen = _i32([-1] * BATCH), _i32([0] * BATCH)
    layers = [moa.PagedCache8.make(pool.page_table, length, n_pages, PAGE, HKV, DH, seen=seen) for _ in range(2)]
    ws, freq = layers[0].workspace(N, HQ), _freq(DH)
    gains = [(1 + 0.2 * torch.randn(DH, generator=torch.Generator().manual_seed(i))).bfloat16().cuda() for i in range(2)]
    ids = torch.arange(4, dtype=torch.int32).repeat(BATCH, 1).cuda()
    bias = torch.full((BATCH, 4), 1.5, device="cuda")
    rules = moa.LogitRules(VOCAB, bias_id=ids, bias_value=bias)
    # what a step is given
    x = [torch.zeros((BATCH * N, HQ + 2 * HKV, DH), dtype=torch.bfloat16, device="cuda") for _ in layers]
    tok, parent, depth = (torch.zeros((BATCH, N), dtype=torch.int32, device="cuda") for _ in range(3))
    logits = torch.zeros((BATCH, N, VOCAB), device="cuda")
    ask = _i32([N] * BATCH)
    counts = (torch.zeros(BATCH, dtype=torch.int32, device="cuda"), torch.zeros(BATCH + 1, dtype=torch.int32, device="cuda"), None, None, None)

    def step():
        moa.moa_page_plan(pool, length, ask, maps=counts)
        pos = torch.where(length[:, None] >= 0, seen[:, None] + depth, -1).flatten().contiguous()
        mask = moa.moa_tree_attn_mask(parent, packed=True).view(BATCH, N)
        outs = []
        for c, y in zip(layers, x):
            q, k, v = y[:, :HQ], y[:, HQ:HQ + HKV], y[:, HQ + HKV:]
            moa.moa_qk_norm_rope(q, k, pos, freq, *gains, q_out=q, k_out=k)
            q, k, v = (t.unflatten(0, (BATCH, N)) for t in (q, k, v))
            outs.append(moa.moa_paged8_attention(c, q, k, v, mask=mask, ws=ws))
        _, slot, _, acc, _ = moa.moa_verify_greedy_rules(rules, tok, parent, logits, CAP)
        kept = torch.where(counts[0] > 0, acc, 0)                    # who waits for pages keeps nothing
        moa.moa_paged8_commit(layers[0], N, slot, kept, advance=False)
        moa.moa_paged8_commit(layers[1], N, slot, kept)
        return outs, slot, acc

    step()                                                           # nobody is in use: nothing happens
    assert length.tolist() == [-1] * BATCH and seen.tolist() == [0] * BATCH
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs, slot, acc = step()
    torch.cuda.synchronize()

    gen = torch.Generator().manual_seed(per)
    rows = [[[torch.zeros((0, HKV, DH), dtype=torch.bfloat16)] * 2 for _ in layers] for _ in range(BATCH)]       # per sequence and layer: keys, values
    lens, comes, ends = [-1] * BATCH, {0: (0, 37), 2: (1, 100), 5: (2, 1), 13: (0, 64), 17: (1, 16)}, {12: 0, 15: 1}
    waited = grew = 0
    for t in range(22):
        if t in ends:
            lens[ends[t]] = -1
        if t in comes:                                               # a prompt: planned, and appended to both layers
            b, n = comes[t]
            lens[b] = 0
            length.copy_(_i32(lens))
            seen[b] = 0
            new = [n if i == b else 0 for i in range(BATCH)]
            got = moa.moa_page_plan(pool, length, _i32(new))
            assert got[0].tolist() == new == ref.plan(lens, new)[0]
            for i, c in enumerate(layers):
                k, v = (torch.randn((BATCH, n, HKV, DH), generator=gen).bfloat16() for _ in range(2))
                moa.moa_paged8_append(c, k.cuda(), v.cuda(), _i32(new), advance=i == 1)
                rows[b][i] = [k[b], v[b]]
            lens[b] = n
        length.copy_(_i32(lens))
        given = [torch.randn(y.shape, generator=gen).bfloat16() for y in x]
        trees = [_tree(rng) for _ in range(BATCH)]
        z = torch.randn((BATCH, N, VOCAB), generator=gen)
        for b, (tk, pa, _, used) in enumerate(trees):
            for i in range(used):
                child = [c for c in range(1, used) if pa[c] == i]
                if child and rng.random() < 0.8:
                    z[b, i, tk[child[int(rng.integers(0, len(child)))]]] += 9
        for dst, src in zip(x + [logits], given + [z]):
            dst.copy_(src)
        for i, dst in enumerate((tok, parent, depth)):
            dst.copy_(_i32([tr[i] for tr in trees]))
        g.replay()
        torch.cuda.synchronize()
        want_rows, want_start, _ = ref.plan(lens, [N] * BATCH)
        _check_pool(pool, ref)
        assert counts[0].tolist() == want_rows and counts[1].tolist() == want_start
        score = z.clone()
        score[..., :4] += 1.5
        for b in range(BATCH):
            if lens[b] < 0:
                continue
            tk, pa, de, used = trees[b]
            path = _accepted(tk, pa, used, score[b].numpy())
            assert int(acc[b]) == len(path) and slot[b, :len(path)].tolist() == path
            at = _i32([lens[b] + d for d in de])
            for i, y in enumerate(x):
                mine, had = y[b * N:(b + 1) * N].cpu(), given[i][b * N:(b + 1) * N]
                _near(mine[:, :HQ], _turned(had[:, :HQ], gains[0], at, freq, False, 1e-5), had, gains[0], 1e-5, "bf16")
                _near(mine[:, HQ:HQ + HKV], _turned(had[:, HQ:HQ + HKV], gains[1], at, freq, False, 1e-5), had, gains[1], 1e-5, "bf16")
                new = [mine[:, HQ:HQ + HKV], had[:, HQ + HKV:]]
                K, V = (np.concatenate([_held(old).astype(np.float64), now.double().numpy()]) for old, now in zip(rows[b][i], new))
                see = np.ones((N, len(K)), bool)                     # a row: the committed ones, itself and its ancestors
                for r in range(N):
                    see[r, lens[b]:] = False
                    j = r if r < used else -1
                    while j >= 0:
                        see[r, lens[b] + j] = True
                        j = pa[j]
                see[used:] = False
                _check_rows(outs[i][b].double().cpu().numpy(), mine[:, :HQ].double().numpy(), K, V, see)
                if want_rows[b]:
                    rows[b][i] = [torch.cat([old, now[path]]) for old, now in zip(rows[b][i], new)]
            waited += want_rows[b] == 0
            grew += len(path) - 1 if want_rows[b] else 0
            lens[b] += len(path) if want_rows[b] else 0
        assert length.tolist() == lens
        assert [s for s, L in zip(seen.tolist(), lens) if L >= 0] == [L for L in lens if L >= 0]
    assert waited > 0 and grew > 10                                  # both were met
    for i, c in enumerate(layers):
        got = moa.moa_paged8_read(c, max(lens), dtype=torch.float32)
        for b in range(BATCH):
            for y, old in zip(got, rows[b][i]):
                assert lens[b] < 0 or torch.equal(y[b, :lens[b]].cpu(), torch.from_numpy(_held(old)))
