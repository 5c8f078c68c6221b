"""Operators of a paged serving loop, as cases to be measured.

Three families, in the order of one step of a batch: the page tables and slot maps of the batch's rows, from the requests'
lengths; norm and rotation of their queries and keys, with the append to a paged cache; and a paged cache that holds its rows
in 8 bits, a scale for each block of 16 positions and head, with the attention over it. Sizes are those of the framework's
configurations: c1 (float32, head size 64, 4 heads), c2 / c4 (32 query and 8 key / value heads of 128, contexts of 2048 and
32768), c5 (64 / 8 heads, 16 sequences of 4096), trees of 61 kept slots, 64 sequences at most.
"""
import math

import torch

own = False

NEG = float("-inf")
KEPT, DEPTH = 61, 6          # slots of a kept tree, its drafted levels
BLOCK, RING = 16, 80         # positions that share a scale; rows of the 16-bit ring behind the closed blocks


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    pl = dict(op="plan", ended=0, short=False)
    no = dict(op="norm", inter=False, gain=True, pad=0)
    c8 = dict(op="cache8", tree=False, ragged=False)
    ap = dict(op="append", ragged=False)
    return [
        # a decode step of a full batch: a row each, now and then a new page
        dict(pl, name="plan-64-tokens", batch=64, ctx=2048, rows=1, page=16),
        # prompts of a full batch, two of them behind requests that ended, and too few pages for the last ones
        dict(pl, name="plan-64-prompts", batch=64, ctx=64, rows=32768, page=16, ended=9, short=True),
        # c1's drafter geometry, one short prompt: what a call costs at least
        dict(no, name="norm-f32-33", rows=33, hq=4, hkv=4, dh=64, rot=64, dtype="f32", paged=False),
        # the rows of c5's 16 kept trees, padded to a captured size, keys and values to their pages
        dict(no, name="norm-16x61", rows=1024, hq=64, hkv=8, dh=128, rot=128, dtype="bf16", paged=True, pad=48),
        # c4's prompt: 32768 rows to their pages
        dict(no, name="norm-32768", rows=32768, hq=32, hkv=8, dh=128, rot=128, dtype="bf16", paged=True),
        # one user's prompt at c2's context enters the cache, and is read back
        dict(ap, name="append-1x2048", batch=1, hkv=8, dh=128, ctx=5, rows=2043, page=16),
        # c5's prompts
        dict(ap, name="append-16x4096", batch=16, hkv=8, dh=128, ctx=0, rows=4096, page=64, ragged=True),
        # one user at c2's context, one token
        dict(c8, name="token-1x2048", batch=1, hq=32, hkv=8, dh=128, ctx=2048, page=16),
        # one user at c4's long context
        dict(c8, name="token-1x32768", batch=1, hq=32, hkv=8, dh=128, ctx=32768, page=64),
        # c5's batch and heads, uneven lengths up to twice its context
        dict(c8, name="token-16x8192", batch=16, hq=64, hkv=8, dh=128, ctx=8192, page=32, ragged=True),
        # the LLM's verification of c2's kept tree, and the commit of the accepted path
        dict(c8, name="tree-1x2048", batch=1, hq=32, hkv=8, dh=128, ctx=2045, page=16, tree=True),
        # the same for c5's batch: 488 query rows per key / value head and sequence
        dict(c8, name="tree-16x4096", batch=16, hq=64, hkv=8, dh=128, ctx=4090, page=64, tree=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "norm", "norm", "append", "cache8", "cache8", "cache8"])
    if op == "plan":
        batch = rng.randint(1, 64)
        return dict(op="plan", batch=batch, ctx=_log_int(rng, 1, 32768), rows=rng.choice([1, KEPT, _log_int(rng, 2, 32768)]),
                    page=rng.choice([16, 32, 64, 128]), ended=rng.randint(0, batch // 4), short=rng.random() < 0.3)
    if op == "norm":
        hkv, group, dh = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        top = 32768 * 48 * 128 // ((hkv * group + 2 * hkv) * dh * (1 if dtype == "bf16" else 2))
        rows = _log_int(rng, 1, min(32768, top))
        return dict(op="norm", rows=rows, hq=hkv * group, hkv=hkv, dh=dh, rot=rng.choice([dh, dh, dh // 2]), inter=rng.random() < 0.3,
                    gain=rng.random() < 0.8, dtype=dtype, paged=rng.random() < 0.6, pad=rng.randint(0, rows // 8))
    hkv, dh = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128])
    if op == "append":
        batch = _log_int(rng, 1, 64)
        return dict(op="append", batch=batch, hkv=hkv, dh=dh, ctx=_log_int(rng, 1, 300) - 1,
                    rows=_log_int(rng, 1, max(2, min(16384, 16 * 8 * 4096 // (batch * hkv)))), page=rng.choice([16, 32, 64, 128]),
                    ragged=rng.random() < 0.6)
    tree, group = rng.random() < 0.4, rng.choice([1, 2, 4, 8])
    batch = _log_int(rng, 1, 16 if tree else 64)
    room = 16 * 8 * 8 * 4096 if tree else 16 * 8 * 8192
    top = max(2, min(32768, room // (batch * hkv * (group if tree else 1))))
    return dict(op="cache8", batch=batch, hq=hkv * group, hkv=hkv, dh=dh, ctx=_log_int(rng, 1, top), page=rng.choice([16, 32, 64, 128]),
                tree=tree, ragged=rng.random() < 0.6)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _uneven(case, most, salt=0):
    """A number for each sequence: `most`, or uneven parts of it."""
    if not case.get("ragged", True):
        return [most] * case["batch"]
    return [max(min(1, most), most - ((b + salt) * 2654435761 % 4294967296) * most // 5368709120) for b in range(case["batch"])]


# ---------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(1_000_003 * (seed + 1))
    return {"plan": _prepare_plan, "norm": _prepare_norm, "append": _prepare_cache8, "cache8": _prepare_cache8}[case["op"]](case, g, dev)


def _ints(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def _plan_sizes(case):
    """Committed positions, new rows and pages held of each sequence, and the most pages that one may have."""
    lens, new, ps = _uneven(case, case["ctx"]), _uneven(case, case["rows"], 7), case["page"]
    if case["rows"] <= KEPT:
        new = [case["rows"]] * case["batch"]
    held = [-(-n // ps) for n in lens]
    for i in range(case["ended"]):          # these ended, and still hold their pages
        lens[i * 7 % case["batch"]] = -1
    per = max(-(-(max(n, 0) + m) // ps) for n, m in zip(lens, new))
    return lens, new, held, max(per, max(held))


def _prepare_plan(case, g, dev):
    lens, new, held, per = _plan_sizes(case)
    B, ps, used = case["batch"], case["page"], sum(held)
    need = sum(max(0, -(-(n + m) // ps) - h) for n, m, h in zip(lens, new, held) if n >= 0)
    back = sum(h for n, h in zip(lens, held) if n < 0)
    spare = max(1, int(need * 0.8) - back) if case["short"] else need + 5
    total = used + spare
    order = torch.randperm(total, generator=g, device=dev).to(torch.int32)
    table = torch.full((B, per), -1, dtype=torch.int32, device=dev)
    at = torch.arange(per, device=dev)
    table[at < _ints(held, dev)[:, None]] = order[:used]
    free = torch.zeros(total, dtype=torch.int32, device=dev)
    free[:spare] = order[used:]
    s = {"case": case, "table": table, "held": _ints(held, dev), "free": free, "count": _ints([spare], dev)}
    s["len"] = _ints(lens, dev)
    jump = torch.randint(0, 40, (B,), generator=g, device=dev).to(torch.int32)          # positions that an eviction dropped
    s["seen"] = torch.where(s["len"] < 0, 0, s["len"] + jump)
    s["n_new"] = _ints(new, dev)
    rows = sum(m for n, m in zip(lens, new) if n >= 0) + 3
    new32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=dev)  # noqa: E731
    s["out"] = (torch.zeros_like(table), new32(B), torch.zeros_like(free), new32(1))
    s["maps"] = (new32(B), new32(B + 1), new32(rows), new32(rows), torch.zeros(rows, dtype=torch.int64, device=dev))
    if own:
        from paper_2410_03804_b200 import moa
        s["pool"] = moa.PagePool(s["table"], s["held"], s["free"], s["count"], ps)
        s["pool_out"] = moa.PagePool(*s["out"], ps)
    return s


def _prepare_norm(case, g, dev):
    R, hq, hkv, dh, T = case["rows"], case["hq"], case["hkv"], case["dh"], _type(case)
    real = R - case["pad"]
    # q, k, v of a row lie side by side, as one projection leaves them; some channels are larger than the others
    qkv = torch.randn((R, hq + 2 * hkv, dh), generator=g, device=dev)
    qkv[..., :: dh // 4] *= 6
    qkv = qkv.to(T)
    s = {"case": case, "q": qkv[:, :hq], "k": qkv[:, hq : hq + hkv], "v": qkv[:, hq + hkv :]}
    # positions of a few requests one after another; rows behind the last one are padding
    span = max(1, real // 3)
    first = torch.randint(0, 100_000, (R // span + 1,), generator=g, device=dev)
    at = torch.arange(R, device=dev)
    s["pos"] = torch.where(at < real, first[at // span] + at % span, -1).to(torch.int32)
    s["freq"] = 500000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=dev) / case["rot"])
    if case["gain"]:
        s["q_gain"], s["k_gain"] = ((1 + 0.1 * torch.randn(dh, generator=g, device=dev)).to(T) for _ in range(2))
    s["q_out"] = torch.zeros((R, hq, dh), dtype=T, device=dev)
    if case["paged"]:
        ps, pages = 16, -(-R // 16) + 5
        s["pk"], s["pv"] = (torch.zeros((pages, ps, hkv, dh), dtype=T, device=dev) for _ in range(2))
        order = torch.randperm(pages, generator=g, device=dev)
        s["slot"] = torch.where(at < real, order[at // ps] * ps + at % ps, -1)
    else:
        s["k_out"] = torch.zeros((R, hkv, dh), dtype=T, device=dev)
    if own and case["paged"]:
        from paper_2410_03804_b200 import moa
        s["cache"] = moa.PagedCache(s["pk"], s["pv"], order[None].to(torch.int32).contiguous(), _ints([0], dev))
    return s


def _codes(x):
    """Blocks [..., 16, dh] in 8 bits: codes -127 .. 127 and a scale [...] for each."""
    x = x.float()
    top = x.abs().amax((-1, -2))
    none, most = top < 2.0**-100, torch.full_like(top, 127.0)          # (divisions of tensors by tensors are rounded once, by numbers not)
    scale = torch.where(none, 0.0, top / most)
    r = torch.where(none, 0.0, most / top)
    return (x * r[..., None, None]).round().clamp(-127, 127), scale


def _records(k, v):
    """Blocks of keys and values [..., 16, dh] as the cache holds them, uint8 [..., 32 * dh + 16]: the keys' codes plus 128 in the
    order (token's parity, dim / 64, token / 2, dim % 64), the values' in the order (dim / 32, dim % 8, token / 4, (dim / 8) % 4,
    token % 4), both scales in fp32, 8 bytes unused."""
    lead, dh = k.shape[:-2], k.shape[-1]
    n = len(lead)
    (kc, ks), (vc, vs) = _codes(k), _codes(v)
    kc = (kc + 128).to(torch.uint8).reshape(*lead, 8, 2, dh // 64, 64).permute(*range(n), n + 1, n + 2, n, n + 3)
    vc = (vc + 128).to(torch.uint8).reshape(*lead, 4, 4, dh // 32, 4, 8).permute(*range(n), n + 2, n + 4, n, n + 3, n + 1)
    scales = torch.stack([ks, vs, torch.zeros_like(ks), torch.zeros_like(ks)], -1).view(torch.uint8)
    return torch.cat([kc.reshape(*lead, -1), vc.reshape(*lead, -1), scales], -1)


def _values(rec, dh):
    """The inverse: fp32 keys and values [..., 16, dh] of records."""
    lead = rec.shape[:-1]
    n, m = len(lead), 16 * dh
    scales = rec[..., 2 * m :].contiguous().view(torch.float32)
    k = rec[..., :m].reshape(*lead, 2, dh // 64, 8, 64).permute(*range(n), n + 2, n, n + 1, n + 3).reshape(*lead, 16, dh)
    v = rec[..., m : 2 * m].reshape(*lead, dh // 32, 8, 4, 4, 4).permute(*range(n), n + 2, n + 4, n, n + 3, n + 1).reshape(*lead, 16, dh)
    return (k.float() - 128) * scales[..., 0, None, None], (v.float() - 128) * scales[..., 1, None, None]


def _rows_in(case):
    """New rows of each sequence of an append. The row count avoids the lengths at which a prompt's last rows meet the first
    ones in the ring, so that a pass can be made again on what it left."""
    base = case["ctx"] // BLOCK
    out = []
    for m in _uneven(case, case["rows"], 3):
        end = (case["ctx"] + m) // BLOCK
        out.append(m - 16 if end > base and (end - base) % 5 == 0 and m > 16 else m)
    return out


def _prepare_cache8(case, g, dev):
    B, hkv, dh, ps = case["batch"], case["hkv"], case["dh"], case["page"]
    append = case["op"] == "append"
    n = max(_rows_in(case)) if append else KEPT if case["tree"] else 1
    lens = [case["ctx"]] * B if append else _uneven(case, case["ctx"])
    per = -(-(max(lens) + n) // ps)
    total, nb = B * per + 3, ps // BLOCK
    loud = torch.ones(dh, device=dev)
    loud[:: dh // 4] = 8                    # channels of the keys that are larger than the others
    rows = lambda *shape: torch.randn(shape + (dh,), generator=g, device=dev)  # noqa: E731
    s = {"case": case, "len": _ints(lens, dev)}
    if append:
        s["pages"] = torch.zeros((total, hkv, nb, 32 * dh + 16), dtype=torch.uint8, device=dev)
    else:
        s["pages"] = torch.cat([_records(rows(c, hkv, nb, BLOCK) * loud, rows(c, hkv, nb, BLOCK)) for c in _chunks(total, 2**27 // (hkv * ps * dh))])
    s["table"] = torch.randperm(total, generator=g, device=dev)[: B * per].to(torch.int32).reshape(B, per)
    s["k_ring"], s["v_ring"] = ((rows(B, RING, hkv) * f).to(torch.bfloat16) for f in (loud, 1.0))
    if append:
        kv = (torch.stack([rows(B, n, hkv) * loud, rows(B, n, hkv)], 2)).to(torch.bfloat16)          # keys and values of a row side by side
        s["k_new"], s["v_new"] = kv[:, :, 0], kv[:, :, 1]
        s["n_new"] = _ints(_rows_in(case), dev)
        s["first"] = s["len"] // BLOCK * BLOCK
        s["end"] = s["len"] + s["n_new"]
        span = n + BLOCK - 1
    else:
        hq = case["hq"]
        qkv = rows(B, n, hq + 2 * hkv)
        qkv[:, :, hq : hq + hkv] *= loud
        qkv = qkv.to(torch.bfloat16)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :, :hq], qkv[:, :, hq : hq + hkv], qkv[:, :, hq + hkv :]
        s["out"] = torch.zeros((B, n, hq, dh), dtype=torch.bfloat16, device=dev)
        span = BLOCK + DEPTH
        if case["tree"]:
            s["anc"] = _tree(g, B, n, dev)
            bit = torch.ones((), dtype=torch.int64, device=dev) << torch.arange(n, device=dev)
            s["mask"] = (s["anc"] * bit).sum(-1)          # one 64-bit word per row, as moa_tree_attn_mask packs it
            leaf = torch.randint(0, n, (B,), generator=g, device=dev)
            path = s["anc"][torch.arange(B, device=dev), leaf]          # the accepted path: the ancestors of some slot
            s["acc_len"] = path.sum(-1).to(torch.int32)
            order = torch.where(path, torch.arange(n, device=dev), n).sort(-1).values[:, : DEPTH + 1]
            s["acc_slot"] = torch.where(order < n, order, -1).to(torch.int32).contiguous()
            s["first"] = s["len"] // BLOCK * BLOCK
            s["end"] = s["len"] + s["acc_len"]
    if append or case["tree"]:
        s["k_read"], s["v_read"] = (torch.zeros((B, span, hkv, dh), dtype=torch.bfloat16, device=dev) for _ in range(2))
    if own:
        from paper_2410_03804_b200 import moa
        s["cache"] = moa.PagedCache8(s["pages"], s["k_ring"], s["v_ring"], s["table"], s["len"], ps)
        if not append:
            s["ws"] = s["cache"].workspace(n, case["hq"])
    return s


def _chunks(total, most):
    most = max(1, most)
    return [min(most, total - i) for i in range(0, total, most)]


def _tree(g, batch, n, dev):
    """Random trees in slot order, parents first, at most DEPTH deep: [batch, n, n], whether a slot sees another."""
    r = torch.Generator().manual_seed(int(torch.randint(0, 2**31 - 1, (1,), generator=g, device=dev)))
    anc = torch.zeros((batch, n, n), dtype=torch.bool)
    for b in range(batch):
        parent, depth, u = [0] * n, [0] * n, torch.rand(n, generator=r).tolist()
        anc[b, 0, 0] = True
        for i in range(1, n):
            q = int(u[i] * i)
            while depth[q] >= DEPTH:
                q = parent[q]
            parent[i], depth[i] = q, depth[q] + 1
            anc[b, i] = anc[b, q]
            anc[b, i, i] = True
    return anc.to(dev)


# ---------------------------------------------------------------------------------------------------------- passes
def run(s):
    op = s["case"]["op"]
    if own:
        return {"plan": _own_plan, "norm": _own_norm, "append": _own_append, "cache8": _own_cache8}[op](s)
    return {"plan": _plan, "norm": _norm, "append": _append, "cache8": _cache8}[op](s)


def _own_plan(s):
    from paper_2410_03804_b200 import moa
    moa.moa_page_plan(s["pool"], s["len"], s["n_new"], seen=s["seen"], pool_out=s["pool_out"], maps=s["maps"])
    return list(s["out"] + s["maps"])


def _own_norm(s):
    from paper_2410_03804_b200 import moa
    kw = dict(cache=s["cache"], slot=s["slot"], v=s["v"]) if s["case"]["paged"] else dict(k_out=s["k_out"])
    moa.moa_qk_norm_rope(s["q"], s["k"], s["pos"], s["freq"], q_gain=s.get("q_gain"), k_gain=s.get("k_gain"), eps=1e-5,
                         interleaved=s["case"]["inter"], q_out=s["q_out"], **kw)
    return [s["q_out"]] + ([s["pk"], s["pv"]] if s["case"]["paged"] else [s["k_out"]])


def _own_append(s):
    from paper_2410_03804_b200 import moa
    moa.moa_paged8_append(s["cache"], s["k_new"], s["v_new"], n_new=s["n_new"], advance=False)
    moa.moa_paged8_read(s["cache"], s["k_read"].shape[1], first=s["first"], length=s["end"], out=(s["k_read"], s["v_read"]))
    return [s["k_read"], s["v_read"], s["k_ring"], s["v_ring"]]


def _own_cache8(s):
    from paper_2410_03804_b200 import moa
    moa.moa_paged8_attention(s["cache"], s["q"], s["k_new"], s["v_new"], mask=s.get("mask"), out=s["out"], ws=s["ws"])
    outs = [s["out"], s["k_ring"], s["v_ring"]]
    if s["case"]["tree"]:
        moa.moa_paged8_commit(s["cache"], KEPT, s["acc_slot"], s["acc_len"], advance=False)
        moa.moa_paged8_read(s["cache"], s["k_read"].shape[1], first=s["first"], length=s["end"], out=(s["k_read"], s["v_read"]))
        outs += [s["k_read"], s["v_read"]]
    return outs


def _plan(s):
    case, ps = s["case"], s["case"]["page"]
    table, held, dev = s["table"], s["held"].long(), s["table"].device
    B, per = table.shape
    T, rows = s["free"].numel(), s["maps"][2].numel()
    n = s["n_new"].long().clamp(min=0)
    live = s["len"] >= 0
    want = torch.where(live, (s["len"].long() + n + ps - 1) // ps, 0)
    fits = live & (want <= per)
    # pages that are given back, on top of the free ones, in the order of sequences and pages
    keep = torch.where(live, torch.minimum(want, held), 0)
    at = torch.arange(per, device=dev)
    back = (at >= keep[:, None]) & (at < held[:, None])
    place = s["count"].long() + (back.flatten().cumsum(0) - 1).reshape(B, per)
    spot = torch.where(back, place, T)
    free = torch.nn.functional.pad(s["free"], (0, 1)).scatter(0, spot.flatten(), table.flatten())[:T]
    have = s["count"].long() + back.sum()
    # whose pages and rows fit, none overtaking one that waits
    need = torch.where(fits, (want - held).clamp(min=0), 0)
    ok = fits & ((need == 0) | (need.cumsum(0) <= have))
    ok = ok & (torch.where(ok, n, 0).cumsum(0) <= rows)
    take = torch.where(ok, need, 0)
    n = torch.where(ok, n, 0)
    # their pages, from the top
    fresh = (at >= held[:, None]) & (at < (held + take)[:, None])
    from_top = (take.cumsum(0) - take)[:, None] + at - held[:, None]
    source = torch.where(fresh, have - 1 - from_top, 0)
    new = torch.where(fresh, free[source], torch.where(at < keep[:, None], table, -1))
    now = torch.where(ok, keep + take, keep)
    used = torch.arange(T, device=dev) < have
    for out, x in zip(s["out"], (new, now, torch.where(used, free, s["out"][2]), have - take.sum())):
        out.copy_(x)
    # the rows, one request's after another's
    start = torch.nn.functional.pad(n.cumsum(0), (1, 0))
    r = torch.arange(rows, device=dev)
    b = (r[:, None] >= start[None, 1:]).sum(1)
    there = b < B
    b = b.clamp(max=B - 1)
    i = r - start[b]
    slot = s["len"].long()[b] + i
    page = new[b, (slot // ps).clamp(0, per - 1)].long()
    maps = (n, start, torch.where(there, b, -1), torch.where(there, s["seen"][b] + i, -1), torch.where(there & (page >= 0), page * ps + slot % ps, -1))
    for out, x in zip(s["maps"], maps):
        out.copy_(x)
    return list(s["out"] + s["maps"])


def _turned(x, gain, s):
    """Norm and rotation of heads [rows, heads, dh]."""
    case, rot = s["case"], s["case"]["rot"]
    x = x.float()
    if gain is not None:
        x = x * (x.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * gain.float()
    angle = s["pos"].double()[:, None] * s["freq"]
    c, d = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case["inter"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * d, b * c + a * d], -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2 : rot]
        y = torch.cat([a * c - b * d, b * c + a * d], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _norm(s):
    case = s["case"]
    real = case["rows"] - case["pad"]
    q, k = _turned(s["q"], s.get("q_gain"), s), _turned(s["k"], s.get("k_gain"), s)
    s["q_out"][:real] = q[:real].to(s["q_out"].dtype)
    if not case["paged"]:
        s["k_out"][:real] = k[:real].to(s["k_out"].dtype)
        return [s["q_out"], s["k_out"]]
    at = s["slot"][:real]
    s["pk"].flatten(0, 1)[at] = k[:real].to(s["pk"].dtype)
    s["pv"].flatten(0, 1)[at] = s["v"][:real]
    return [s["q_out"], s["pk"], s["pv"]]


def _put_blocks(s, first, k, v, there):
    """Closes blocks first + j (k, v [B, m, 16, hkv, dh]) where there [B, m]."""
    nb = s["case"]["page"] // BLOCK
    m = k.shape[1]
    g = first[:, None] + torch.arange(m, device=k.device)
    page = s["table"].gather(1, (g // nb).clamp(max=s["table"].shape[1] - 1)).long()
    rec = _records(k.transpose(2, 3), v.transpose(2, 3))
    s["pages"][page[there], :, (g % nb)[there]] = rec[there]


def _read(s):
    """Slots first .. first + span - 1 below end, in bf16, zeros behind them."""
    case, (B, span, hkv, dh) = s["case"], s["k_read"].shape
    nb, cap = case["page"] // BLOCK, s["table"].shape[1] * case["page"]
    slot = s["first"].long()[:, None] + torch.arange(span, device=s["len"].device)
    g = (slot // BLOCK).clamp(max=cap // BLOCK - 1)
    m = span // BLOCK + 2
    blocks = (s["first"].long()[:, None] // BLOCK + torch.arange(m, device=slot.device)).clamp(max=cap // BLOCK - 1)
    page = s["table"].gather(1, blocks // nb).long()
    inside = (g - s["first"].long()[:, None] // BLOCK) * BLOCK + slot % BLOCK
    b = torch.arange(B, device=slot.device)[:, None]
    closed = (slot < (s["end"].long() // BLOCK * BLOCK)[:, None])[..., None, None]
    there = (slot < s["end"][:, None])[..., None, None]
    for out, x, ring in zip((s["k_read"], s["v_read"]), _values(s["pages"][page, :, blocks % nb], dh), (s["k_ring"], s["v_ring"])):
        x = x.transpose(2, 3).reshape(B, m * BLOCK, hkv, dh)[b, inside].to(torch.bfloat16)
        out.copy_(torch.where(there, torch.where(closed, x, ring[b, slot % RING]), 0))


def _append(s):
    B, n = s["k_new"].shape[:2]
    dev = s["len"].device
    first, end = s["first"].long(), s["end"].long()
    m = (n + BLOCK - 1) // BLOCK + 1
    # positions from the open block on: its rows in the ring, then the new ones
    slot = first[:, None] + torch.arange(m * BLOCK, device=dev)
    old = (slot < s["len"][:, None])[..., None, None]
    i = (slot - s["len"][:, None]).clamp(0, n - 1)
    b = torch.arange(B, device=dev)[:, None]
    k, v = (torch.where(old, ring[b, slot % RING], new[b, i]) for ring, new in ((s["k_ring"], s["k_new"]), (s["v_ring"], s["v_new"])))
    closed = (slot[:, ::BLOCK] + BLOCK) <= end[:, None]
    _put_blocks(s, first // BLOCK, k.unflatten(1, (m, BLOCK)), v.unflatten(1, (m, BLOCK)), closed)
    # what stays open
    last = (end // BLOCK * BLOCK)[:, None] + torch.arange(BLOCK, device=dev)
    fresh = ((last < end[:, None]) & (last >= s["len"][:, None]))[..., None, None]
    at = (last - s["len"][:, None]).clamp(0, n - 1)
    for ring, new in ((s["k_ring"], s["k_new"]), (s["v_ring"], s["v_new"])):
        ring[b, last % RING] = torch.where(fresh, new[b, at], ring[b, last % RING])
    _read(s)
    return [s["k_read"], s["v_read"], s["k_ring"], s["v_ring"]]


def _cache8(s):
    case = s["case"]
    B, n, hq, dh = s["q"].shape
    hkv, ps, dev = case["hkv"], case["page"], s["q"].device
    nb, cap = ps // BLOCK, s["table"].shape[1] * ps
    length = s["len"].long()
    b = torch.arange(B, device=dev)[:, None]
    new = length[:, None] + torch.arange(n, device=dev)
    s["k_ring"][b, new % RING], s["v_ring"][b, new % RING] = s["k_new"], s["v_new"]
    slot = torch.arange(cap, device=dev)
    closed = (slot < (length // BLOCK * BLOCK)[:, None])[..., None, None]
    kv = []
    for x, ring in zip(_values(s["pages"][s["table"].long()], dh), (s["k_ring"], s["v_ring"])):
        x = x.permute(0, 1, 3, 4, 2, 5).reshape(B, cap, hkv, dh)
        kv.append(torch.where(closed, x, ring[b, (slot % RING)[None]].float()))
    sees = (slot < length[:, None])[:, None, :].expand(B, n, cap)
    if case["tree"]:
        sees = sees.scatter(2, new[:, None, :].expand(B, n, n), s["anc"])
    else:
        sees = sees | (slot == length[:, None])[:, None, :]
    q = s["q"].float().unflatten(2, (hkv, hq // hkv))
    score = torch.einsum("bnhgd,bshd->bhgns", q, kv[0]) / math.sqrt(dh)
    score = score.masked_fill(~sees[:, None, None], NEG)
    p = (score - score.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    s["out"].copy_(torch.einsum("bhgns,bshd->bnhgd", p, kv[1]).reshape(B, n, hq, dh))
    outs = [s["out"], s["k_ring"], s["v_ring"]]
    if case["tree"]:
        m = s["acc_slot"].shape[1]
        j = torch.arange(m, device=dev)
        src = torch.where(j < s["acc_len"][:, None], s["acc_slot"].long(), j)          # behind the path: a row onto itself
        frm, to = (length[:, None] + src) % RING, (length[:, None] + j) % RING
        s["k_ring"][b, to], s["v_ring"][b, to] = s["k_ring"][b, frm], s["v_ring"][b, frm]
        rows = (s["first"].long()[:, None] + torch.arange(2 * BLOCK, device=dev)) % RING
        done = (s["first"].long()[:, None] + torch.tensor([BLOCK, 2 * BLOCK], device=dev)) <= s["end"][:, None]
        _put_blocks(s, s["first"].long() // BLOCK, s["k_ring"][b, rows].unflatten(1, (2, BLOCK)), s["v_ring"][b, rows].unflatten(1, (2, BLOCK)), done)
        _read(s)
        outs += [s["k_read"], s["v_read"]]
    return outs


# ---------------------------------------------------------------------------------------------------------- floors
def work(case):
    if case["op"] == "plan":
        lens, new, held, per = _plan_sizes(case)
        rows = sum(m for n, m in zip(lens, new) if n >= 0)
        moved = sum(-(-(n + m) // case["page"]) for n, m in zip(lens, new) if n >= 0)
        return {"bytes": rows * 16 + moved * 8 + case["batch"] * 32, "flops": 0}
    e = 2 if case.get("dtype", "bf16") == "bf16" else 4
    hkv, dh = case["hkv"], case["dh"]
    if case["op"] == "norm":
        rows, heads = case["rows"] - case["pad"], case["hq"] + hkv
        per = heads + (hkv if case["paged"] else 0)
        return {"bytes": rows * (2 * per * dh * e + 4 + (8 if case["paged"] else 0)), "flops": rows * heads * dh * 8}
    if case["op"] == "append":
        # rows in as 16 bits, out as codes; read back as codes, out as 16 bits
        return {"bytes": sum(_rows_in(case)) * hkv * dh * 2 * (2 + 1 + 1 + 2), "flops": sum(_rows_in(case)) * hkv * dh * 6}
    n, lens = KEPT if case["tree"] else 1, _uneven(case, case["ctx"])
    shut = [L // BLOCK * BLOCK for L in lens]
    rows = sum(shut) * hkv * 2 * dh + sum(shut) // BLOCK * hkv * 8 + sum(L - c for L, c in zip(lens, shut)) * hkv * 4 * dh
    new = case["batch"] * n * (2 * case["hq"] + 4 * hkv) * dh * 2
    return {"bytes": rows + new, "flops": sum(4 * n * case["hq"] * dh * (L + n) for L in lens)}


# ---------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)
    return {"norm": _exact_norm, "append": _exact_append, "cache8": _exact_cache8}[case["op"]](case, s)


def _exact_norm(case, s):
    """The rotation as a product of complex numbers."""
    rot, real = case["rot"], case["rows"] - case["pad"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=s["q"].device), s["pos"][:real].double()[:, None] * s["freq"])[:, None]

    def heads(x, gain):
        x = x[:real].double()
        if gain is not None:
            x = x / torch.sqrt(torch.mean(x**2, -1, keepdim=True) + 1e-5) * gain.double()
        y = x.clone()
        if case["inter"]:
            z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * turn
            y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
        else:
            z = torch.complex(x[..., : rot // 2], x[..., rot // 2 : rot]) * turn
            y[..., : rot // 2], y[..., rot // 2 : rot] = z.real, z.imag
        return y

    q, k = s["q_out"].double(), heads(s["k"], s.get("k_gain"))
    q[:real] = heads(s["q"], s.get("q_gain"))
    if not case["paged"]:
        out = s["k_out"].double()
        out[:real] = k
        return [q, out]
    pk, pv = s["pk"].double(), s["pv"].double()
    page, row = s["slot"][:real] // 16, s["slot"][:real] % 16
    pk[page, row], pv[page, row] = k, s["v"][:real].double()
    return [q, pk, pv]


def _block64(x):
    """A block [16, ...] of rows of one sequence as it is held: the nearest multiples of its heads' largest value / 127."""
    x = x.double()
    top = x.abs().amax((0, 2), keepdim=True)
    unit = torch.where(top > 0, top / 127, 1.0)
    return torch.round(x / unit) * unit


def _exact_append(case, s):
    outs = [x.double().clone() for x in (s["k_read"], s["v_read"], s["k_ring"], s["v_ring"])]
    base, ctx = case["ctx"] // BLOCK * BLOCK, case["ctx"]
    for b, m in enumerate(_rows_in(case)):
        for w, (ring, new) in enumerate(((s["k_ring"], s["k_new"]), (s["v_ring"], s["v_new"]))):
            old = [ring[b, j % RING] for j in range(base, ctx)]
            rows = torch.cat([torch.stack(old), new[b, :m]] if old else [new[b, :m]])
            shut = len(rows) // BLOCK * BLOCK
            for j in range(0, shut, BLOCK):
                outs[w][b, j : j + BLOCK] = _block64(rows[j : j + BLOCK])
            outs[w][b, shut : len(rows)] = rows[shut:].double()
            for j in range(max(shut, ctx - base), len(rows)):
                outs[2 + w][b, (base + j) % RING] = rows[j].double()
    return outs


def _exact_cache8(case, s):
    """Sequence by sequence and key / value head by head: softmax(q k^T / sqrt(d)) v in 64 bits, the codes taken from their places one by one."""
    dev, ps, dh, n = s["q"].device, case["page"], case["dh"], s["q"].shape[1]
    G, t, d = case["hq"] // case["hkv"], torch.arange(BLOCK, device=dev)[:, None], torch.arange(dh, device=dev)
    at_k = ((t % 2) * (dh // 64) + d // 64) * 512 + t // 2 * 64 + d % 64
    at_v = 16 * dh + d // 32 * 512 + d % 8 * 64 + t // 4 * 16 + d // 8 % 4 * 4 + t % 4
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    kr, vr = s["k_ring"].double(), s["v_ring"].double()
    for b, L in enumerate(_uneven(case, case["ctx"])):
        shut = L // BLOCK
        g = torch.arange(shut, device=dev)
        rec = s["pages"][s["table"][b].long()[g * BLOCK // ps], :, g % (ps // BLOCK)]
        scale = rec[..., 32 * dh :].contiguous().view(torch.float32).double()
        kr[b, torch.arange(L, L + n, device=dev) % RING], vr[b, torch.arange(L, L + n, device=dev) % RING] = s["k_new"][b].double(), s["v_new"][b].double()
        tail = torch.arange(shut * BLOCK, L + n, device=dev) % RING
        new = s["anc"][b] if case["tree"] else torch.ones((1, 1), dtype=torch.bool, device=dev)
        hidden = torch.cat([torch.zeros((n, L), dtype=torch.bool, device=dev), ~new], 1)
        for h in range(case["hkv"]):
            K = ((rec[:, h][:, at_k].double() - 128) * scale[:, h, 0, None, None]).reshape(-1, dh)
            W = ((rec[:, h][:, at_v].double() - 128) * scale[:, h, 1, None, None]).reshape(-1, dh)
            K, W = torch.cat([K, kr[b, tail, h]]), torch.cat([W, vr[b, tail, h]])
            z = torch.matmul(s["q"][b, :, h * G : (h + 1) * G].double().transpose(0, 1), K.T) * dh**-0.5
            z = torch.softmax(z.masked_fill(hidden, NEG), -1)
            out[b, :, h * G : (h + 1) * G] = torch.matmul(z, W).transpose(0, 1)
    outs = [out, kr, vr]
    if case["tree"]:
        kd, vd = s["k_read"].double(), s["v_read"].double()
        for b, L in enumerate(_uneven(case, case["ctx"])):
            m, base = int(s["acc_len"][b]), L // BLOCK * BLOCK
            path = s["acc_slot"][b, :m].tolist()
            for ring, read in ((kr, kd), (vr, vd)):
                kept = [ring[b, (L + j) % RING].clone() for j in path]
                for j, x in enumerate(kept):
                    ring[b, (L + j) % RING] = x
                rows = torch.stack([ring[b, j % RING] for j in range(base, L + m)])
                for j in range(0, len(rows) // BLOCK * BLOCK, BLOCK):
                    rows[j : j + BLOCK] = _block64(rows[j : j + BLOCK])
                read[b, : len(rows)] = rows
        outs += [kd, vd]
    return outs
