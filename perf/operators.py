"""The serving operators beside the drafter, as cases to be measured.

Three families, in the order of one generation cycle: attention of new rows over a paged key / value cache (with the
append of their keys and values, and for a tree the commit of its accepted path), the rules that logits pass before
verification, and the eviction that bounds the cache. Sizes are those of the framework's configurations: c1 (float32,
head size 64, 4 heads), c2 / c4 (32 query and 8 key / value heads of 128, contexts of 2048 and 32768), c5 (64 / 8 heads,
16 sequences of 4096), trees of 61 kept slots, vocabularies of 1024 and 128256.
"""
import math

import torch

own = False

NEG = float("-inf")


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    att = dict(op="attention", tree=False, weights=False, ragged=False, gap=0)
    ev = dict(op="evict", hkv=8, dh=128, dtype="bf16", page=16, sink=4)
    ru = dict(op="rules", vocab=128256, tree=False, bias=0, allow=False, verify=False)
    return [
        # c1's drafter geometry, one short conversation: what a call costs at least
        dict(att, name="token-f32-64", batch=1, hq=4, hkv=4, dh=64, ctx=64, dtype="f32", page=16),
        # one user at c2's context; the weights feed the eviction
        dict(att, name="token-1x2048", batch=1, hq=32, hkv=8, dh=128, ctx=2048, dtype="bf16", page=16, weights=True),
        # one user at c4's long context
        dict(att, name="token-1x32768", batch=1, hq=32, hkv=8, dh=128, ctx=32768, dtype="bf16", page=64),
        # a full batch of short and uneven conversations, keys and values of a page in one block
        dict(att, name="token-64x1500", batch=64, hq=32, hkv=4, dh=128, ctx=1500, dtype="bf16", page=16, ragged=True, gap=1),
        # c5's batch and heads, uneven lengths up to its context, with weights
        dict(att, name="token-16x4096", batch=16, hq=64, hkv=8, dh=128, ctx=4096, dtype="bf16", page=32, ragged=True, weights=True),
        # the LLM's verification of c2's kept tree, and the commit of the accepted path
        dict(att, name="tree-1x2048", batch=1, hq=32, hkv=8, dh=128, ctx=2048, dtype="bf16", page=16, tree=True),
        # the same for c5's batch: 488 query rows per key / value head and sequence
        dict(att, name="tree-16x4096", batch=16, hq=64, hkv=8, dh=128, ctx=4096, dtype="bf16", page=64, tree=True),
        # steady state of a bounded cache: one slot over the budget
        dict(ev, name="evict-1x2049-one", batch=1, ctx=2049, budget=2048, recent=64, ragged=False),
        # c5's batch cut to half its context at once
        dict(ev, name="evict-16x4096-half", batch=16, ctx=4096, budget=2048, recent=256, ragged=True),
        # plain sampling of 16 users: penalties and a few biases, adjusted logits out
        dict(ru, name="rules-16-tokens", batch=16, n=1, dtype="f32", bias=32),
        # a constrained answer, verified over c2's kept tree: adjusted logits out
        dict(ru, name="rules-tree-61", batch=1, n=61, dtype="bf16", tree=True, bias=8, allow=True),
        # c5's verification with every rule on; only choices and the accepted path come out
        dict(ru, name="verify-16x61", batch=16, n=61, dtype="bf16", tree=True, bias=300, allow=True, verify=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "evict", "rules"])
    if op == "attention":
        tree = rng.random() < 0.35
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
        batch = _log_int(rng, 1, 16 if tree else 64)
        room = 16 * 8 * 8 * 4096 if tree else 64 * 4 * 1500 if dtype == "bf16" else 64 * 4 * 700
        top = max(2, min(32768, room // (batch * hkv * (group if tree else 1))))
        if tree and dtype == "f32":
            top = min(top, 2048)
        return dict(op="attention", batch=batch, hq=hkv * group, hkv=hkv, dh=rng.choice([64, 128, 128]),
                    ctx=_log_int(rng, 1, top), dtype=dtype, page=rng.choice([8, 16, 32, 64, 128]), tree=tree,
                    weights=not tree and rng.random() < 0.4, ragged=rng.random() < 0.6, gap=rng.choice([0, 0, 1]))
    if op == "evict":
        batch = _log_int(rng, 1, 32)
        hkv = rng.choice([1, 2, 4, 8])
        ctx = _log_int(rng, 40, max(41, min(32768, 16 * 8 * 4096 // (batch * hkv))))
        budget = max(24, int(ctx * rng.uniform(0.3, 1.0)))
        return dict(op="evict", batch=batch, hkv=hkv, dh=rng.choice([64, 128]), ctx=ctx, budget=budget,
                    sink=rng.choice([0, 4]), recent=rng.randint(0, budget // 4), dtype=rng.choice(["bf16", "f32"]),
                    page=rng.choice([8, 16, 32, 64]), ragged=rng.random() < 0.5)
    tree = rng.random() < 0.6
    batch, vocab = _log_int(rng, 1, 16 if tree else 64), _log_int(rng, 1000, 128256)
    return dict(op="rules", batch=batch, n=rng.randint(2, 61) if tree else 1, vocab=vocab, dtype=rng.choice(["f32", "bf16"]),
                tree=tree, bias=rng.choice([0, 0, 5, 64, 300]), allow=rng.random() < 0.5, verify=tree and rng.random() < 0.5)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lens(case):
    """Cached positions of each sequence: the context, or uneven parts of it."""
    c = case["ctx"]
    if not case["ragged"]:
        return [c] * case["batch"]
    return [max(1, c - (b * 2654435761 % 4294967296) * c // 5368709120) for b in range(case["batch"])]


KEPT = 61          # slots of a kept tree, the root among them
DEPTH = 6          # its drafted levels


# ---------------------------------------------------------------------------------------------------------- inputs
def _tree(g, batch, n, vocab, dev):
    """Random trees in slot order, parents first, at most DEPTH deep, siblings with different tokens."""
    r = torch.Generator().manual_seed(int(torch.randint(0, 2**31 - 1, (1,), generator=g, device=dev)))
    parent, tok = torch.full((batch, n), -1, dtype=torch.int32), torch.empty((batch, n), dtype=torch.int32)
    anc = torch.zeros((batch, n, n), dtype=torch.bool)
    for b in range(batch):
        tok[b] = torch.randperm(vocab, generator=r)[:n].to(torch.int32)
        depth, u = [0] * n, torch.rand(n, generator=r).tolist()
        anc[b, 0, 0] = True
        for i in range(1, n):
            q = int(u[i] * i)
            while depth[q] >= DEPTH:
                q = int(parent[b, q])
            parent[b, i], depth[i] = q, depth[q] + 1
            anc[b, i] = anc[b, q]
            anc[b, i, i] = True
    return tok.to(dev), parent.to(dev), anc.to(dev)


def _pages(g, case, cap_slots, dev):
    """A pool of pages in random order, some of them nobody's, and the table of each sequence's pages."""
    ps, B = case["page"], case["batch"]
    per = -(-cap_slots // ps)
    total = B * per + 3
    table = torch.randperm(total, generator=g, device=dev)[: B * per].to(torch.int32).reshape(B, per)
    shape = (total, ps, case["hkv"], case["dh"])
    if case.get("gap"):          # keys and values of a page side by side: a page stride of twice a page's values
        both = torch.randn((total, 2) + shape[1:], generator=g, device=dev).to(_type(case))
        k, v = both[:, 0], both[:, 1]
    else:
        k, v = (torch.randn(shape, generator=g, device=dev).to(_type(case)) for _ in range(2))
    return k, v, table, per * ps


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(1_000_003 * (seed + 1))
    B, T = case["batch"], _type(case)
    if case["op"] == "rules":
        return _prepare_rules(case, g, dev)
    lens = _lens(case)
    s = {"case": case, "len": torch.tensor(lens, dtype=torch.int32, device=dev)}
    n = (KEPT if case["tree"] else 1) if case["op"] == "attention" else 1
    s["k"], s["v"], s["table"], cap = _pages(g, case, max(lens) + n, dev)
    s["cap"] = cap
    hkv, dh = case["hkv"], case["dh"]
    s["seen"] = s["len"] + torch.randint(0, 50, (B,), generator=g, device=dev).to(torch.int32)
    if case["op"] == "evict" or case["weights"]:
        # accumulated weights: most positions got little, a few a lot
        s["weight"] = torch.rand((B, hkv, cap), generator=g, device=dev).pow(8) * 40
        gap = (s["seen"] - s["len"]).to(torch.int32)          # positions that earlier evictions dropped, behind the first four
        at = torch.arange(cap, device=dev, dtype=torch.int32)
        s["pos"] = (at + torch.where(at >= 4, gap[:, None], 0)).to(torch.int32)[:, None].expand(B, hkv, cap).contiguous()
        s["weight_out"], s["pos_out"] = torch.zeros_like(s["weight"]), torch.zeros_like(s["pos"])
    if case["op"] == "attention":
        hq = case["hq"]
        # q, k, v of the new rows lie side by side, as one projection leaves them
        qkv = torch.randn((B, n, (hq + 2 * hkv) * dh), generator=g, device=dev).to(T)
        s["q"] = qkv[..., : hq * dh].unflatten(-1, (hq, dh))
        s["k_new"] = qkv[..., hq * dh : (hq + hkv) * dh].unflatten(-1, (hkv, dh))
        s["v_new"] = qkv[..., (hq + hkv) * dh :].unflatten(-1, (hkv, dh))
        s["out"] = torch.empty((B, n, hq, dh), dtype=T, device=dev)
        if case["tree"]:
            _, parent, anc = _tree(g, B, n, 4096, dev)
            s["anc"] = anc
            bit = torch.ones((), dtype=torch.int64, device=dev) << torch.arange(n, device=dev)
            s["mask"] = (anc * bit).sum(-1)          # one 64-bit word per row, as moa_tree_attn_mask packs it
            # the accepted path: the ancestors of some slot
            leaf = torch.randint(0, n, (B,), generator=g, device=dev)
            path = anc[torch.arange(B, device=dev), leaf]
            s["acc_len"] = path.sum(-1).to(torch.int32)
            order = torch.where(path, torch.arange(n, device=dev), n).sort(-1).values[:, : DEPTH + 1]
            s["acc_slot"] = torch.where(order < n, order, -1).to(torch.int32).contiguous()
    else:
        s["len_out"] = torch.zeros_like(s["len"])
    if own:
        from paper_2410_03804_b200 import moa
        s["cache"] = moa.PagedCache(s["k"], s["v"], s["table"], s["len"], s.get("weight"), s.get("pos"), s["seen"])
        s["ws"] = s["cache"].workspace(n, case["hq"], case["weights"]) if case["op"] == "attention" else s["cache"].evict_workspace(case["budget"])
    return s


def _prepare_rules(case, g, dev):
    B, n, V = case["batch"], case["n"], case["vocab"]
    s = {"case": case}
    s["logits"] = (torch.randn((B, n, V), generator=g, device=dev) * 2.5).to(_type(case))
    s["out"] = torch.empty_like(s["logits"])
    s["choice"] = torch.empty((B, n), dtype=torch.int32, device=dev)
    # the record of a conversation: a prompt of a few hundred different tokens, a few dozen generated ones
    prompt = torch.randint(0, V, (B, 700), generator=g, device=dev)
    made = torch.randint(0, max(1, V // 20), (B, 180), generator=g, device=dev)
    s["counts"] = torch.zeros((B, V), dtype=torch.int32, device=dev).scatter_add_(1, made, torch.ones_like(made, dtype=torch.int32))
    known = (s["counts"] > 0).scatter_(1, prompt, True)
    s["known"] = known
    s["seen"] = _bits(known)
    s["repetition"] = 1 + torch.rand((B,), generator=g, device=dev) * 0.4
    s["frequency"] = torch.rand((B,), generator=g, device=dev) * 0.8
    s["presence"] = torch.rand((B,), generator=g, device=dev) * 0.6
    if case["bias"]:
        s["bias_id"] = torch.stack([torch.randperm(V, generator=g, device=dev)[: case["bias"]] for _ in range(B)]).to(torch.int32)
        s["bias_value"] = torch.randn((B, case["bias"]), generator=g, device=dev) * 4
    if case["allow"]:
        may = torch.rand((B, n, V), generator=g, device=dev) < 0.3
        s["may"], s["allow"] = may, _bits(may)
    if case["tree"]:
        s["tok"], s["parent"], s["anc"] = _tree(g, B, n, V, dev)
        # the LLM agrees with one child of most slots, so that paths get accepted
        at = torch.rand((B, n), generator=g, device=dev) < 0.8
        p = s["parent"].clamp(min=0).long()
        sel = (at & (s["parent"] >= 0)).nonzero(as_tuple=True)
        s["logits"][sel[0], p[sel], s["tok"][sel].long()] = 24.0
        if case["allow"]:
            s["may"][sel[0], p[sel], s["tok"][sel].long()] = True
            s["allow"] = _bits(s["may"])
        new = lambda *shape: torch.empty(shape, dtype=torch.int32, device=dev)  # noqa: E731
        s["walk"] = (s["choice"], new(B, DEPTH + 1), new(B, DEPTH + 1), new(B), new(B))
    if own:
        from paper_2410_03804_b200 import moa
        s["rules"] = moa.LogitRules(V, counts=s["counts"], seen=s["seen"], repetition=s["repetition"], frequency=s["frequency"],
                                    presence=s["presence"], bias_id=s.get("bias_id"), bias_value=s.get("bias_value"),
                                    allow=s.get("allow"))
    return s


def _bits(x):
    """Truth values [..., V] as little-endian words int32 [..., ceil(V / 32)]."""
    x = torch.nn.functional.pad(x, (0, -x.shape[-1] % 32)).unflatten(-1, (-1, 32))
    word = (x.to(torch.int64) << torch.arange(32, device=x.device)).sum(-1)
    return torch.where(word >= 2**31, word - 2**32, word).to(torch.int32)


# ---------------------------------------------------------------------------------------------------------- passes
def run(s):
    op = s["case"]["op"]
    if own:
        return {"attention": _own_attention, "evict": _own_evict, "rules": _own_rules}[op](s)
    return {"attention": _attention, "evict": _evict, "rules": _rules}[op](s)


def _own_attention(s):
    from paper_2410_03804_b200 import moa
    case, weights = s["case"], s["case"]["weights"]
    moa.moa_paged_attention(s["cache"], s["q"], s["k_new"], s["v_new"], mask=s.get("mask"), out=s["out"],
                            weight_out=s["weight_out"] if weights else None, ws=s["ws"])
    if case["tree"]:
        moa.moa_paged_commit(s["cache"], KEPT, s["acc_slot"], s["acc_len"], advance=False)
    return [s["out"], s["k"], s["v"]] + ([s["weight_out"]] if weights else [])


def _own_evict(s):
    from paper_2410_03804_b200 import moa
    case = s["case"]
    moa.moa_paged_evict(s["cache"], case["budget"], case["sink"], case["recent"], weight_out=s["weight_out"], pos_out=s["pos_out"],
                        len_out=s["len_out"], ws=s["ws"])
    return [s["k"], s["v"], s["weight_out"], s["pos_out"], s["len_out"]]


def _own_rules(s):
    from paper_2410_03804_b200 import moa
    case = s["case"]
    if case["verify"]:
        return list(moa.moa_verify_greedy_rules(s["rules"], s["tok"], s["parent"], s["logits"], DEPTH + 1, out=s["walk"]))
    moa.moa_logit_rules(s["rules"], s["logits"], s.get("tok"), s.get("parent"), out=s["out"], choice=s["choice"])
    return [s["out"], s["choice"]]


def _places(s, slot):
    """(page, row in the page) of slots [B, m] of the sequences."""
    ps = s["case"]["page"]
    return s["table"].gather(1, slot // ps).long(), slot % ps


def _attention(s):
    case = s["case"]
    B, n, hq, dh = s["q"].shape
    hkv, cap, dev = case["hkv"], s["cap"], s["q"].device
    new = s["len"].long()[:, None] + torch.arange(n, device=dev)
    at = _places(s, new)
    s["k"][at], s["v"][at] = s["k_new"], s["v_new"]
    k = s["k"][s["table"].long()].reshape(B, cap, hkv, dh).float()
    v = s["v"][s["table"].long()].reshape(B, cap, hkv, dh).float()
    slot = torch.arange(cap, device=dev)
    sees = (slot < s["len"][:, None])[:, None, :].expand(B, n, cap)
    if case["tree"]:
        sees = sees.scatter(2, new[:, None, :].expand(B, n, n), s["anc"])
    else:
        sees = sees | (slot == s["len"][:, None])[:, None, :]
    q = s["q"].float().unflatten(2, (hkv, hq // hkv))
    score = torch.einsum("bnhgd,bshd->bhgns", q, k) / math.sqrt(dh)
    score = score.masked_fill(~sees[:, None, None], NEG)
    p = (score - score.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    s["out"].copy_(torch.einsum("bhgns,bshd->bnhgd", p, v).reshape(B, n, hq, dh))
    outs = [s["out"], s["k"], s["v"]]
    if case["weights"]:
        old = torch.where(slot < s["len"][:, None, None], s["weight"], 0.0)
        got = old + p.sum((2, 3))
        s["weight_out"].copy_(torch.where(slot <= s["len"][:, None, None], got, s["weight_out"]))
        outs.append(s["weight_out"])
    if case["tree"]:
        m = s["acc_slot"].shape[1]
        j = torch.arange(m, device=dev)
        src = torch.where(j < s["acc_len"][:, None], s["acc_slot"].long(), j)          # behind the path: a row onto itself
        a, b = _places(s, s["len"].long()[:, None] + src), _places(s, s["len"].long()[:, None] + j)
        s["k"][b], s["v"][b] = s["k"][a], s["v"][a]
    return outs


def _evict(s):
    case = s["case"]
    B, hkv, cap = s["weight"].shape
    budget, dev = case["budget"], s["weight"].device
    slot = torch.arange(cap, device=dev)
    used = slot < s["len"][:, None, None]
    must = (s["pos"] < case["sink"]) | (s["pos"] >= s["seen"][:, None, None] - case["recent"])
    rank = torch.where(must, math.inf, s["weight"]).masked_fill(~used, -1.0)          # weights are sums of probabilities: >= 0
    order = rank.sort(dim=-1, descending=True, stable=True).indices
    keep = torch.zeros_like(used.expand(B, hkv, cap)).scatter(2, order[..., :budget], True) & used
    mover, hole = keep & (slot >= budget), ~keep & (slot < budget) & (s["len"][:, None, None] > budget)
    b, h, src = mover.nonzero(as_tuple=True)
    dst = hole.nonzero(as_tuple=True)[2]                  # both lists in the order of sequence, head, slot
    page = s["table"].long()
    to, frm = (page[b, dst // case["page"]], dst % case["page"], h), (page[b, src // case["page"]], src % case["page"], h)
    s["k"][to], s["v"][to] = s["k"][frm], s["v"][frm]
    w, p = s["weight"].clone(), s["pos"].clone()
    w[b, h, dst], p[b, h, dst] = s["weight"][b, h, src], s["pos"][b, h, src]
    s["len_out"].copy_(s["len"].clamp(max=budget))
    left = slot < s["len_out"][:, None, None]
    s["weight_out"].copy_(torch.where(left, w, s["weight_out"]))
    s["pos_out"].copy_(torch.where(left, p, s["pos_out"]))
    return [s["k"], s["v"], s["weight_out"], s["pos_out"], s["len_out"]]


def _rules(s):
    case = s["case"]
    B, n, V = s["logits"].shape
    x = s["logits"].float()
    count, known = s["counts"][:, None].expand(B, n, V), s["known"][:, None].expand(B, n, V)
    if case["tree"]:
        on = torch.zeros((B, n, V), dtype=torch.int32, device=x.device)
        on.scatter_add_(2, s["tok"].long()[:, None].expand(B, n, n), s["anc"].to(torch.int32))
        count, known = count + on, known | (on > 0)
    rep, freq, pres = (s[k][:, None, None] for k in ("repetition", "frequency", "presence"))
    x = torch.where(known, torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * count.float()
    x = torch.where(count > 0, x - pres, x)
    if case["bias"]:
        add = torch.zeros((B, V), device=x.device).scatter_add_(1, s["bias_id"].long(), s["bias_value"])
        x = x + add[:, None]
    if case["allow"]:
        x = x.masked_fill(~s["may"], NEG)
    best = x.amax(-1, keepdim=True)
    choice = torch.where(x == best, torch.arange(V, device=x.device), V).amin(-1)
    choice = torch.where(best[..., 0] > NEG, choice, 0).to(torch.int32)
    if not case["verify"]:
        return [s["out"].copy_(x), s["choice"].copy_(choice)]
    p = s["parent"].clamp(min=0).long()
    agreed = (s["tok"] == choice.gather(1, p)) | (s["parent"] < 0)
    taken = (agreed[:, None] | ~s["anc"]).all(-1)          # every slot of the path agreed: those slots form the path
    order = torch.where(taken, torch.arange(n, device=x.device), n)
    order = torch.nn.functional.pad(order, (0, max(0, DEPTH + 1 - n)), value=n).sort(-1).values[:, : DEPTH + 1]
    there = order < n
    acc_slot = torch.where(there, order, -1).to(torch.int32)
    acc_tok = torch.where(there, s["tok"].gather(1, order.clamp(max=n - 1)), -1).to(torch.int32)
    acc_len = there.sum(-1).to(torch.int32)
    last = order.gather(1, (acc_len - 1)[:, None].long())
    return [choice, acc_slot, acc_tok, acc_len, choice.gather(1, last)[:, 0]]


# ---------------------------------------------------------------------------------------------------------- floors
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rules":
        rows, V = case["batch"] * case["n"], case["vocab"]
        bits = V // 8 * (case["batch"] + (rows if case["allow"] else 0))
        return {"bytes": rows * V * e * (1 if case["verify"] else 2) + bits + case["batch"] * 180 * 4, "flops": rows * V * 2}
    hkv, dh, lens = case["hkv"], case["dh"], _lens(case)
    if case["op"] == "evict":
        total = 0
        for L in lens:
            # weights and positions once in, the kept ones out; rows move as often as kept slots lie behind the budget,
            # which for weights in no order is the share of the slots behind it
            total += hkv * 8 * (L + min(L, case["budget"]))
            if L > case["budget"]:
                total += hkv * 4 * dh * e * case["budget"] * (L - case["budget"]) // L
        return {"bytes": total, "flops": 0}
    n = KEPT if case["tree"] else 1
    rows = sum(lens) * hkv * dh * 2 * e
    new = case["batch"] * n * (2 * case["hq"] + 4 * hkv) * dh * e
    more = sum(lens) * hkv * 8 if case["weights"] else 0
    return {"bytes": rows + new + more, "flops": sum(4 * n * case["hq"] * dh * (L + n) for L in lens)}


# ---------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "evict": _exact_evict, "rules": _exact_rules}[case["op"]](case, s)


def _exact_attention(case, s):
    """Sequence by sequence and key / value head by head: softmax(q k^T / sqrt(d)) v in 64 bits."""
    ps, n, G = case["page"], s["q"].shape[1], case["hq"] // case["hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    got = s["weight_out"].double().clone() if case["weights"] else None
    for b, L in enumerate(_lens(case)):
        where = torch.arange(L, device=out.device)
        page = s["table"][b].long()[where // ps]
        K = torch.cat([s["k"][page, where % ps].double(), s["k_new"][b].double()])
        W = torch.cat([s["v"][page, where % ps].double(), s["v_new"][b].double()])
        new = s["anc"][b] if case["tree"] else torch.ones((1, 1), dtype=torch.bool, device=out.device)
        hidden = torch.cat([torch.zeros((n, L), dtype=torch.bool, device=out.device), ~new], 1)
        for h in range(case["hkv"]):
            q = s["q"][b, :, h * G : (h + 1) * G].double()
            z = torch.matmul(q.transpose(0, 1), K[:, h].T) * case["dh"] ** -0.5
            z = torch.softmax(z.masked_fill(hidden, NEG), -1)
            out[b, :, h * G : (h + 1) * G] = torch.matmul(z, W[:, h]).transpose(0, 1)
            if got is not None:
                got[b, h, :L] = s["weight"][b, h, :L].double() + z[:, 0, :L].sum(0)
                got[b, h, L] = z[:, 0, L].sum()
    return [out, None, None] + ([got] if got is not None else [])


def _exact_evict(case, s):
    """By sorting each head's slots on the host; what moves is copied, so the values have no rounding."""
    K, W, w, p = s["k"].double().cpu(), s["v"].double().cpu(), s["weight_out"].double().cpu(), s["pos_out"].cpu()
    weight, pos, table, m = s["weight"].double().cpu(), s["pos"].cpu(), s["table"].cpu().tolist(), case["budget"]
    ps = case["page"]
    for b, L in enumerate(_lens(case)):
        edge = int(s["seen"][b]) - case["recent"]
        for h in range(case["hkv"]):
            ww, pp = weight[b, h, :L].tolist(), pos[b, h, :L].tolist()
            w[b, h, : min(L, m)], p[b, h, : min(L, m)] = weight[b, h, : min(L, m)], pos[b, h, : min(L, m)]
            if L <= m:
                continue
            best = sorted(range(L), key=lambda j: (not (pp[j] < case["sink"] or pp[j] >= edge), -ww[j], j))
            kept = set(best[:m])
            frm, to = [j for j in range(m, L) if j in kept], [j for j in range(m) if j not in kept]
            for a, z in zip(frm, to):
                w[b, h, z], p[b, h, z] = ww[a], pp[a]
            a, z = torch.tensor(frm, dtype=torch.long), torch.tensor(to, dtype=torch.long)
            row = torch.tensor(table[b])
            for t in (K, W):
                t[row[z // ps], z % ps, h] = t[row[a // ps], a % ps, h]
    return [K, W, w, None, None]


def _exact_rules(case, s):
    y = s["logits"].double()
    B, n, V = y.shape
    for b in range(B):
        rep, freq, pres = (float(s[k][b].double()) for k in ("repetition", "frequency", "presence"))
        bias = torch.zeros(V, dtype=torch.float64, device=y.device)
        if case["bias"]:
            bias[s["bias_id"][b].long()] = s["bias_value"][b].double()
        for i in range(n):
            c = s["counts"][b].double()
            k = s["known"][b].clone()
            j = i if case["tree"] else -1
            while j >= 0:
                t = int(s["tok"][b, j])
                c[t] += 1
                k[t] = True
                j = int(s["parent"][b, j])
            row = y[b, i]
            row = torch.where(k & (row > 0), row / rep, torch.where(k, row * rep, row))
            row = row - freq * c - pres * (c > 0) + bias
            if case["allow"]:
                row = torch.where(s["may"][b, i], row, torch.full_like(row, NEG))
            y[b, i] = row
    return [y.argmax(-1).to(torch.int32), None, None, None, None] if case["verify"] else [y, None]
