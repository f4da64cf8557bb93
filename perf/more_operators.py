"""Operators of tree verification as cases that can be timed and checked, beside their plain forms.

A round may bring a tree of drafts instead of a chain: several continuations of the committed text that share their
beginnings.  A pass then has a row for the pending token and one for every draft; a row's parent is the row whose token comes
before its own, and a row sees the cached text, its ancestors and itself.  The operators work on a paged cache in the model's own
type, whose clients may share blocks:

  attend  the rows of a pass over their clients' caches, a tree or a chain each;
  pass    a whole pass: room for the rows, then keys and values in and attention, layer by layer;
  accept  the decision on a tree: which drafts stand, and the token that follows them;
  fork    clients that begin as another client's text, without its blocks being copied, and go on by themselves;
  keep    what lies behind a position is reduced to some of its tokens (a tree to its accepted path), in place;
  copy    a client's text into blocks of another's own.

The decision.  Row r has target distribution p_r and, behind it, the drafts of its children were drawn from q_r, one after the
other (with `distinct`: without putting back).  Children are tried in order.  With a = 0, b = 1, S = 1 before the first, child c
with token x is taken if u_c < min(1, w / (b q(x))), w = max(0, p(x) - a q(x)); 0 / 0 is not.  If it is not, a grows by b, S (if
`distinct`) falls by q(x), to no less than 2^-24, and b becomes T / S, T the sum over the vocabulary of max(0, p - a q).  What is
left when no child is taken is max(0, p - a q), of a row without children p, and the next token is drawn from it with u_0.  p, q, u
and a, b, w are 32-bit numbers; w is p - a q rounded once, b q is rounded before the division, S and T / S are formed in 64 bits.
T and the draw are sums of whole numbers floor(2^40 w): the token is the first whose running sum exceeds floor(2^24 u_0) W / 2^24,
W the sum over all; if W is 0 it is the lowest one of largest p.  Without q a child is taken if its token is that of the row's largest
p (the lowest index of several), which is also the next token.

Model shapes are the library's own workloads, and head layouts of its tests.
"""
import math
import random

import torch

own = False

_DEVICE = "cuda"
_BLOCK = 16  # tokens per cache block

# query heads, heads of the cache, head dim
_HEADS = {
    "tiny": (4, 4, 64),      # the small fp32 model
    "1b": (32, 8, 64),
    "8b": (32, 8, 128),      # the headline workload
    "13b": (40, 40, 128),    # every query head has its own keys
    "g3": (24, 8, 128),      # three query heads share one
    "g8": (128, 16, 64),     # eight do
}


def listed():
    return [
        # the small fp32 model: the pending token and four drafts in two branches, latency
        {"name": "attend_tiny_5", "do": "attend", "heads": "tiny", "dtype": "f32", "clients": 1, "context": 128, "rows": 5, "tree": True},
        # one token at a time behind a short context, head dim 64
        {"name": "attend_1b_decode", "do": "attend", "heads": "1b", "dtype": "bf16", "clients": 1, "context": 1023, "rows": 1, "tree": False},
        # the headline context with a full tree of drafts
        {"name": "attend_8b_tree64", "do": "attend", "heads": "8b", "dtype": "bf16", "clients": 1, "context": 2048, "rows": 64, "tree": True},
        # sixteen clients of all lengths with trees of all sizes
        {"name": "attend_8b_batch16", "do": "attend", "heads": "8b", "dtype": "bf16", "clients": 16, "context": 4096, "rows": 33, "tree": True},
        # a small tree at the far end of a long context
        {"name": "attend_8b_long", "do": "attend", "heads": "8b", "dtype": "bf16", "clients": 1, "context": 131071, "rows": 9, "tree": True},
        # an fp32 model, three query heads to a head of the cache, odd context
        {"name": "attend_g3_f32", "do": "attend", "heads": "g3", "dtype": "f32", "clients": 2, "context": 6001, "rows": 27, "tree": True},
        # a whole pass of eight clients through the layers of a model
        {"name": "pass_1b_8", "do": "pass", "heads": "1b", "dtype": "bf16", "layers": 16, "clients": 8, "context": 1531, "rows": 25},
        # a small tree over a small vocabulary: latency
        {"name": "accept_tiny", "do": "accept", "vocab": 4096, "clients": 1, "rows": 6, "children": 2, "distinct": False, "sample": True},
        # a full tree over the largest vocabulary
        {"name": "accept_8b_64", "do": "accept", "vocab": 128256, "clients": 1, "rows": 64, "children": 4, "distinct": True, "sample": True},
        # sixteen clients of ragged trees
        {"name": "accept_1b_batch16", "do": "accept", "vocab": 32000, "clients": 16, "rows": 25, "children": 3, "distinct": True, "sample": True},
        # sixteen clients that begin with the same text and go on by themselves, read back
        {"name": "fork_1b_16", "do": "fork", "heads": "1b", "dtype": "bf16", "layers": 2, "clients": 16, "context": 777, "rows": 9},
        # trees of drafts reduced to their accepted paths behind a text that others share, read back
        {"name": "keep_8b_4", "do": "keep", "heads": "8b", "dtype": "bf16", "layers": 4, "clients": 4, "context": 1531, "rows": 64, "kept": 6},
    ]


def draw(rng):
    def spread(low, high):
        return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))

    most = [work(c) for c in listed()]
    most_bytes, most_flops = (max(w[k] for w in most) for k in ("bytes", "flops"))
    while True:
        do = rng.choice(["attend", "attend", "attend", "pass", "accept", "accept", "fork", "keep", "copy"])
        heads, dtype = rng.choice(sorted(_HEADS)), rng.choice(["bf16", "bf16", "f32"])
        clients = spread(1, 16) if rng.random() < 0.6 else 1
        case = {"do": do, "heads": heads, "dtype": dtype, "clients": clients}
        if do == "attend":
            case.update(context=spread(1, 131072 // clients + 1) - 1, rows=spread(1, 64), tree=rng.random() < 0.7)
        elif do == "pass":
            case.update(layers=rng.randint(1, 16), context=spread(1, 8192 // clients + 1) - 1, rows=spread(1, 64))
        elif do == "accept":
            case = {"do": do, "vocab": spread(100, 128256), "clients": clients, "rows": spread(1, 64), "children": rng.randint(1, 5),
                    "distinct": rng.random() < 0.5, "sample": rng.random() < 0.8}
        else:
            case.update(layers=rng.randint(1, 8), context=spread(1, 4096))
            if do == "fork":
                case.update(rows=spread(1, 64))
            if do == "keep":
                case.update(rows=spread(1, 2048))
                case.update(kept=rng.randint(0, case["rows"]))
        w = work(case)
        if w["bytes"] <= most_bytes and w["flops"] <= most_flops and case.get("rows", 1) * clients * case.get("vocab", 1) <= 1 << 24:
            return case


# ---- sizes --------------------------------------------------------------------------------------


def _lengths(case):
    """(tokens that a client has cached before the pass, its new rows), per client; the first has the most of both."""
    r = random.Random(case["clients"] * 1000003 + case.get("context", 0) * 101 + case["rows"])
    before, rows = [case.get("context", 0)], [case["rows"]]
    for _ in range(case["clients"] - 1):
        before.append(r.randint(0, before[0]))
        rows.append(r.randint(1, rows[0]))
    return before, rows


def _parents(rows, children=4):
    """A tree's rows: the parent of each, -1 for the first (the pending token); no row has more than `children`."""
    r = random.Random(rows * 31 + children)
    parents, have = [-1], [0]
    for i in range(1, rows):
        may = [j for j in range(max(0, i - 2 * children - 2), i) if have[j] < children]
        j = r.choice(may)
        parents.append(j)
        have[j] += 1
        have.append(0)
    return parents


def _kept(case, client):
    """Which of a client's rows stay, rising."""
    r = random.Random(case["rows"] * 7919 + case["kept"] * 31 + client)
    return sorted(r.sample(range(case["rows"]), case["kept"]))


def work(case):
    if case["do"] == "accept":
        # the distributions that the draw is made from (rows that a client's walk does not come by need not be read)
        v, n = case["vocab"], case["clients"]
        return {"bytes": n * v * 4 * (2 if case["sample"] and case["rows"] > 1 else 1), "flops": 0}
    nq, nkv, dim = _HEADS[case["heads"]]
    size = 4 if case["dtype"] == "f32" else 2
    token = nkv * 2 * dim * size  # bytes of a token in the cache of a layer
    if case["do"] in ("attend", "pass"):
        before, rows = _lengths(case)
        layers = case.get("layers", 1)
        new = sum(rows) * token * 2 if case["do"] == "pass" else 0  # keys and values of the rows into the cache
        # (of the rows' own tokens a chain's row sees half, a tree's its ancestors: some few)
        own = sum(r * (r + 1) // 2 for r in rows) if not case.get("tree", True) else sum(r * min(r, 6) for r in rows)
        seen = sum(r * b for b, r in zip(before, rows)) + own
        return {"bytes": layers * (sum(b + r for b, r in zip(before, rows)) * token + sum(rows) * nq * dim * 2 * size + new),
                "flops": layers * 4 * dim * nq * seen}
    layers, clients, context = case["layers"], case["clients"], case["context"]
    if case["do"] == "fork":
        # the new rows in and into the cache; the read back: in (the text once) and out
        return {"bytes": layers * token * (clients * case["rows"] * 2 + context + clients * case["rows"] + clients * (context + case["rows"])), "flops": 0}
    if case["do"] == "keep":
        return {"bytes": layers * token * (clients * case["kept"] * 2 + context + clients * case["kept"] + clients * (context + case["kept"])), "flops": 0}
    return {"bytes": layers * token * clients * context * 4, "flops": 0}  # copied, and read back


# ---- inputs -------------------------------------------------------------------------------------


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _generator(seed, part):
    g = torch.Generator(device=_DEVICE)
    g.manual_seed(seed * 1009 + part)
    return g


def _keys_values(case, seed, part, tokens):
    """Keys and values [tokens][heads][dim].  A few channels of the keys are several times larger than the others, as in
    trained models."""
    _, nkv, dim = _HEADS[case["heads"]]
    g = _generator(seed, 2 + part)
    large = 1 + 3 * (torch.rand(nkv, dim, generator=g, device=_DEVICE) < 0.05)
    k = torch.randn((tokens, nkv, dim), generator=g, device=_DEVICE) * large
    v = torch.randn((tokens, nkv, dim), generator=g, device=_DEVICE)
    return k.to(_type(case)), v.to(_type(case))


def _queries(case, seed, layer, rows):
    nq, _, dim = _HEADS[case["heads"]]
    return (1.5 * torch.randn((rows, nq, dim), generator=_generator(seed, 100000 + layer), device=_DEVICE)).to(_type(case))


def _text(case, seed, layer, client, tokens):
    return _keys_values(case, seed, layer * 64 + client, tokens)


def _trees(case):
    """Per client, the parents of its rows."""
    _, rows = _lengths(case)
    if case["do"] == "attend" and not case["tree"]:
        return [list(range(-1, n - 1)) for n in rows]
    return [_parents(n, case.get("children", 4)) for n in rows]


def _distributions(case, seed):
    """Target and draft distributions [rows][vocab] of all clients' rows.  Draft models are near the target, and both are peaked."""
    _, rows = _lengths(case)
    g = _generator(seed, 0)
    z = 3.0 * torch.randn((sum(rows), case["vocab"]), generator=g, device=_DEVICE)
    p = torch.softmax(z, -1)
    return p, torch.softmax(z + 0.7 * torch.randn(z.shape, generator=g, device=_DEVICE), -1) if case["sample"] else None


def _drafts(case, seed, p, q):
    """A token for every row (the first of a client: any), drawn from the parent's draft distribution, and uniforms."""
    g = _generator(seed, 1)
    _, rows = _lengths(case)
    tokens, r0 = [], 0
    many = min(case["children"], case["vocab"])
    pool = torch.multinomial(p if q is None else q, many, replacement=not case["distinct"], generator=g).tolist()
    for n, parents in zip(rows, _trees(case)):
        given = [0] * n
        tokens.append(0)
        for j in parents[1:]:
            tokens.append(pool[r0 + j][given[j]])
            given[j] += 1
        r0 += n
    u = torch.randint(0, 1 << 24, (sum(rows),), generator=g, device=_DEVICE).float() * 2.0 ** -24
    return tokens, u.tolist()


def _ints(v):
    return torch.tensor(v, dtype=torch.int64, device=_DEVICE)


# ---- plain forms --------------------------------------------------------------------------------


def _plain_pages(case, layers, blocks):
    _, nkv, dim = _HEADS[case["heads"]]
    return [torch.zeros((layers, blocks, _BLOCK, nkv, dim), dtype=_type(case), device=_DEVICE) for _ in range(2)]


def _plain_attend(s, layer):
    """Attention of a pass's rows; queries in their own places [client][most rows] of a padded batch."""
    clients, most, nq, nkv, dim = s["sizes"]
    group = nq // nkv
    k, v = (page[layer][s["table"]].flatten(1, 2).permute(0, 2, 1, 3).float() for page in s["pages"])  # [client][head][token][dim]
    q = s["q"][layer].float()[s["row_at"]]                           # [client][most rows][query head][dim]
    q = q.view(clients, most, nkv, group, dim).permute(0, 2, 1, 3, 4).reshape(clients, nkv, most * group, dim)
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(dim)
    sees = s["sees"].unsqueeze(1).unsqueeze(3).expand(-1, nkv, -1, group, -1).reshape(score.shape)
    score = score.masked_fill(~sees, -torch.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -torch.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = torch.matmul(p, v.contiguous()).view(clients, nkv, most, group, dim).permute(0, 2, 1, 3, 4).reshape(clients * most, nq, dim)
    return o[s["row_of"]].to(s["type"])


def _run_pass(s):
    out = []
    for layer in range(len(s["k"])):
        for page, new in zip(s["pages"], (s["k"][layer], s["v"][layer])):
            page[layer][s["block"], s["token"]] = new
        out.append(_plain_attend(s, layer))
    return out


def _fixed(w):
    """floor(2^40 w) of 32-bit numbers."""
    return (w.double() * 2.0 ** 40).long()


def _left(p, q, a):
    """max(0, p - a q), rounded once (the product of two 32-bit numbers is exact in 64)."""
    return (p.double() - a.double() * q.double()).float().clamp(min=0)


def _run_accept(s):
    """All clients side by side, from row to row and from child to child."""
    p, q, kids, tokens, u, first = s["p"], s["q"], s["kids"], s["tokens"], s["u"], s["first"]
    clients, n = len(first), p.shape[1]
    result = torch.full((clients, s["width"]), -1, dtype=torch.int32, device=_DEVICE)
    row, length, walking = first.clone(), torch.zeros_like(first), torch.ones_like(first, dtype=torch.bool)
    every = torch.arange(clients, device=_DEVICE)
    a = torch.zeros(clients, device=_DEVICE)
    for _ in range(s["depth"]):
        a = torch.where(walking, 0.0, a)
        b, left = torch.ones_like(a), torch.ones(clients, dtype=torch.float64, device=_DEVICE)
        open_, taken = walking.clone(), torch.zeros_like(walking)
        best = p[row].argmax(-1) if q is None else None
        to = row
        for i in range(kids.shape[1]):
            child = kids[row, i]
            here = open_ & (child >= 0)
            c = child.clamp(min=0)
            if q is None:
                good = here & (tokens[c] == best)
            else:
                if i > 0:
                    total = _fixed(_left(p[row], q[row], a[:, None])).sum(-1)
                    b = torch.where(here, (total.double() * 2.0 ** -40 / left).float(), b)
                px, qx = p[row, tokens[c]], q[row, tokens[c]]
                good = here & (u[c] < (_left(px, qx, a) / (b * qx)).clamp(max=1))
                bad = here & ~good
                a = torch.where(bad, a + b, a)
                if s["distinct"]:
                    left = torch.where(bad, (left - qx.double()).clamp(min=2.0 ** -24), left)
            to, taken, open_ = torch.where(good, c, to), taken | good, open_ & ~good
        result[every, 2 + length] = torch.where(taken, (to - first).int(), result[every, 2 + length])
        length, row, walking = length + taken.long(), to, walking & taken
    if q is None:
        result[:, 1] = p[row].argmax(-1).int()
    else:
        w = _fixed(_left(p[row], q[row], a[:, None]))
        upto = w.cumsum(-1)
        whole = upto[:, -1]
        parts = (u[first] * 2.0 ** 24).long()
        # W of 41 bits, 24 bits of u: the product by halves of W
        at = ((whole >> 20) * parts + (((whole & 0xfffff) * parts) >> 20)) >> 4
        token = (upto <= at[:, None]).sum(-1).clamp(max=n - 1)
        result[:, 1] = torch.where(whole == 0, p[row].argmax(-1), token).int()
    result[:, 0] = length.int()
    return {"result": result}


def _plain_read(s, table, length):
    at = torch.arange(length, device=_DEVICE)
    return [page[:, table[:, at // _BLOCK], at % _BLOCK] for page in s["pages"]]  # [layer][client][token][head][dim]


def _run_fork(s):
    clients, context, rows = s["sizes"]
    table = s["table"]
    table[:, :s["shared"]] = s["text"][:s["shared"]]
    if context % _BLOCK:
        for page in s["pages"]:  # the block that the text ends in becomes a client's own
            page[:, table[:, s["shared"]]] = page[:, s["text"][s["shared"]]].unsqueeze(1)
    at = context + torch.arange(rows, device=_DEVICE)
    for page, new in zip(s["pages"], (s["k"], s["v"])):
        page[:, table[:, at // _BLOCK], at % _BLOCK] = new.unflatten(1, (clients, rows))
    k, v = _plain_read(s, table, context + rows)
    return {"k": k.flatten(1, 2), "v": v.flatten(1, 2)}


def _run_keep(s):
    clients, context, rows, kept = s["sizes"]
    table = s["table"]
    table[:, :s["shared"]] = s["text"][:s["shared"]]
    old = context + s["kept"]  # [client][kept]
    at = context + torch.arange(kept, device=_DEVICE)
    for page in s["pages"]:
        moved = page[:, s["text"][old // _BLOCK], old % _BLOCK]
        if context % _BLOCK:
            page[:, table[:, s["shared"]]] = page[:, s["text"][s["shared"]]].unsqueeze(1)
        page[:, table[:, at // _BLOCK], at % _BLOCK] = moved
    k, v = _plain_read(s, table, context + kept)
    return {"k": k.flatten(1, 2), "v": v.flatten(1, 2)}


def _run_copy(s):
    clients, context = s["sizes"]
    for page in s["pages"]:
        page[:, s["table"]] = page[:, s["text"]].unsqueeze(1)
    k, v = _plain_read(s, s["table"], context)
    return {"k": k.flatten(1, 2), "v": v.flatten(1, 2)}


# ---- what a program has in hand -----------------------------------------------------------------


def _cache(case, layers, clients, blocks):
    """The library's paged cache in the model's own type."""
    from paper_2605_13319_amd import inputs as I
    from paper_2605_13319_amd import nav

    nq, nkv, dim = _HEADS[case["heads"]]
    shape = I.ModelShape(case["heads"], layers, 512, nq, nkv, dim, 512, 512, dtype=I.DTYPE_F32 if case["dtype"] == "f32" else I.DTYPE_BF16)
    return nav.PageCache(shape, max_seqs=clients, n_blocks=blocks)


def _prepare_accept(case, seed):
    _, rows = _lengths(case)
    trees = _trees(case)
    p, q = _distributions(case, seed)
    tokens, u = _drafts(case, seed, p, q)
    s = {"do": "accept", "p": p, "q": q, "distinct": case["distinct"]}
    if own:
        from paper_2605_13319_amd import nav

        s.update(rows=rows, tokens=tokens, parents=[j for t in trees for j in t], u=u)
        s["result"] = torch.empty((len(rows), max(rows) + 1), dtype=torch.int32, device=_DEVICE)
        s["workspace"] = nav.tree_workspace(len(rows), sum(rows))
        return s
    kids, r0, depth = [], 0, 0
    for t in trees:
        mine, level = [[] for _ in t], [0] * len(t)
        for i, j in enumerate(t):
            if j >= 0:
                mine[j].append(r0 + i)
                level[i] = level[j] + 1
        kids += mine
        depth = max(depth, max(level))
        r0 += len(t)
    most = max([1] + [len(k) for k in kids])
    s.update(kids=_ints([k + [-1] * (most - len(k)) for k in kids]), tokens=_ints(tokens), u=torch.tensor(u, device=_DEVICE),
             first=_ints([sum(rows[:i]) for i in range(len(rows))]), width=max(rows) + 1, depth=max(1, depth))
    return s


def _prepare_shared(case, seed):
    """A text in client 0's blocks, and what becomes of it in others."""
    do, layers, clients, context = case["do"], case["layers"], case["clients"], case["context"]
    rows = case.get("rows", 0)
    length = context + (rows if do == "keep" else 0)            # of the text
    after = context + {"fork": rows, "keep": case.get("kept", 0), "copy": 0}[do]
    s = {"do": do, "type": _type(case), "after": after}
    text = [_text(case, seed, layer, 0, length) for layer in range(layers)]
    if do == "fork":
        new = [_text(case, seed, layer, 1, clients * rows) for layer in range(layers)]
        s["k"], s["v"] = torch.stack([k for k, _ in new]), torch.stack([v for _, v in new])
    old_blocks, new_blocks = -(-length // _BLOCK), -(-after // _BLOCK)
    if own:
        s["cache"] = cache = _cache(case, layers, clients + 1, old_blocks + clients * new_blocks)
        cache.extend([0], [length])
        for layer, (k, v) in enumerate(text):
            cache.append(layer, k, v)
        s.update(layers=layers, seqs=list(range(1, clients + 1)), zero=[0] * clients, context=[context] * clients, rows=[rows] * clients,
                 length=[length] * clients, count=[after] * clients)
        if do == "keep":
            s["kept"] = [_kept(case, c) for c in range(clients)]
        return s
    s["pages"] = _plain_pages(case, layers, old_blocks + clients * new_blocks)
    order = torch.randperm(old_blocks + clients * new_blocks, generator=_generator(seed, 99), device=_DEVICE)
    s["text"], s["table"] = order[:old_blocks], order[old_blocks:].view(clients, new_blocks)
    at = torch.arange(length, device=_DEVICE)
    for layer, kv in enumerate(text):
        for page, x in zip(s["pages"], kv):
            page[layer][s["text"][at // _BLOCK], at % _BLOCK] = x
    s["shared"] = context // _BLOCK
    s["sizes"] = {"fork": (clients, context, rows), "keep": (clients, context, rows, case.get("kept", 0)), "copy": (clients, context)}[do]
    if do == "keep":
        s["kept"] = _ints([_kept(case, c) for c in range(clients)]).view(clients, case["kept"])
    return s


def prepare(case, seed):
    if case["do"] == "accept":
        return _prepare_accept(case, seed)
    if case["do"] in ("fork", "keep", "copy"):
        return _prepare_shared(case, seed)
    nq, nkv, dim = _HEADS[case["heads"]]
    before, rows = _lengths(case)
    clients, layers, trees = case["clients"], case.get("layers", 1), _trees(case)
    total = [b + n for b, n in zip(before, rows)]
    s = {"do": case["do"], "type": _type(case)}
    text = [[_text(case, seed, layer, c, total[c]) for c in range(clients)] for layer in range(layers)]
    s["q"] = [_queries(case, seed, layer, sum(rows)) for layer in range(layers)]
    s["k"], s["v"] = ([torch.cat([kv[j][b:] for kv, b in zip(text[layer], before)]) for layer in range(layers)] for j in (0, 1))
    if own:
        s["cache"] = cache = _cache(case, layers, clients, sum(-(-n // _BLOCK) for n in total))
        for c in range(clients):
            if before[c]:
                cache.extend([c], [before[c]])
                for layer in range(layers):
                    cache.append(layer, *(x[:before[c]] for x in text[layer][c]))
        s.update(seqs=list(range(clients)), before=before, rows=rows, out=[torch.empty_like(q) for q in s["q"]])
        s["parents"] = [j for t in trees for j in t] if case.get("tree", True) else None
        if case["do"] == "attend":
            cache.extend(s["seqs"], rows, s["parents"])
            cache.append(0, s["k"][0], s["v"][0])
        return s
    blocks = [-(-n // _BLOCK) for n in total]
    s["pages"] = _plain_pages(case, layers, sum(blocks))
    order = torch.randperm(sum(blocks), generator=_generator(seed, 99), device=_DEVICE)
    table = torch.zeros((clients, max(blocks)), dtype=torch.int64, device=_DEVICE)
    most = max(rows)
    sees = torch.zeros((clients, most, max(blocks) * _BLOCK), dtype=torch.bool, device=_DEVICE)
    for c in range(clients):
        table[c, :blocks[c]] = order[sum(blocks[:c]):sum(blocks[:c + 1])]
        at = torch.arange(total[c], device=_DEVICE)
        for layer in range(layers):
            for page, x in zip(s["pages"], text[layer][c]):
                page[layer][table[c][at // _BLOCK], at % _BLOCK] = x
        sees[c, :rows[c], :before[c]] = True
        line = []  # a row's ancestors and itself
        for i, j in enumerate(trees[c]):
            line.append((line[j] if j >= 0 else []) + [i])
        pairs = _ints([[i, j] for i, l in enumerate(line) for j in l])
        sees[c, pairs[:, 0], before[c] + pairs[:, 1]] = True
    client = torch.repeat_interleave(torch.arange(clients, device=_DEVICE), _ints(rows))
    row = torch.cat([torch.arange(n, device=_DEVICE) for n in rows])
    pos = _ints(before)[client] + row
    row_at = torch.zeros((clients, most), dtype=torch.int64, device=_DEVICE)
    row_at[client, row] = torch.arange(len(client), device=_DEVICE)
    s.update(sizes=(clients, most, nq, nkv, dim), table=table, sees=sees, row_at=row_at, row_of=client * most + row,
             block=table[client, pos // _BLOCK], token=pos % _BLOCK)
    return s


def run(s):
    do = s["do"]
    if not own:
        if do == "attend":
            return {"out": _plain_attend(s, 0)}
        return {"pass": _run_pass, "accept": _run_accept, "fork": _run_fork, "keep": _run_keep, "copy": _run_copy}[do](s)
    if do == "accept":
        from paper_2605_13319_amd import nav

        return {"result": nav.tree_accept(s["p"], s["q"], s["tokens"], s["parents"], s["u"], rows=s["rows"], distinct=s["distinct"],
                                          result=s["result"], workspace=s["workspace"])}
    cache = s["cache"]
    if do == "attend":
        return {"out": cache.attend(0, s["q"][0], out=s["out"][0])}
    if do == "pass":
        cache.truncate(s["seqs"], s["before"])
        cache.extend(s["seqs"], s["rows"], s["parents"])
        for layer in range(len(s["k"])):
            cache.append(layer, s["k"][layer], s["v"][layer])
            cache.attend(layer, s["q"][layer], out=s["out"][layer])
        return s["out"]
    if do == "fork":
        cache.fork(s["zero"], s["seqs"], s["context"])
        cache.extend(s["seqs"], s["rows"])
        for layer in range(s["layers"]):
            cache.append(layer, s["k"][layer], s["v"][layer])
    elif do == "keep":
        cache.fork(s["zero"], s["seqs"], s["length"])
        cache.compact(s["seqs"], s["context"], s["kept"])
    else:
        cache.copy(s["zero"], s["seqs"], s["context"])
    k, v = cache.read(s["seqs"], [0] * len(s["seqs"]), s["count"])
    return {"k": k, "v": v}


# ---- the definition in 64 bits ------------------------------------------------------------------


def _exact_attend(case, seed, layer):
    nq, nkv, dim = _HEADS[case["heads"]]
    group = nq // nkv
    before, rows = _lengths(case)
    q, r0, out = _queries(case, seed, layer, sum(rows)).double(), 0, []
    for c, (b, n, parents) in enumerate(zip(before, rows, _trees(case))):
        k, v = _text(case, seed, layer, c, b + n)
        hidden = torch.ones((n, b + n), dtype=torch.bool)
        hidden[:, :b] = False
        for i in range(n):
            j = i
            while j >= 0:
                hidden[i, b + j] = False
                j = parents[j]
        hidden = hidden.to(_DEVICE)[None]
        o = torch.empty((n, nq, dim), dtype=torch.float64, device=_DEVICE)
        for h in range(nkv):
            z = (q[r0:r0 + n, h * group:(h + 1) * group].transpose(0, 1).reshape(group * n, dim) @ k[:, h].double().T.contiguous()).view(group, n, -1)
            w = torch.softmax((z / math.sqrt(dim)).masked_fill(hidden, -torch.inf), -1)
            o[:, h * group:(h + 1) * group] = (w.view(group * n, -1) @ v[:, h].double()).view(group, n, dim).transpose(0, 1)
        out.append(o)
        r0 += n
    return torch.cat(out)


def _exact_accept(case, seed):
    """A client at a time, on the host, in whole numbers where the definition has them."""
    import numpy as np

    _, rows = _lengths(case)
    p, q = _distributions(case, seed)
    tokens, u = _drafts(case, seed, p, q)
    result, r0 = np.full((len(rows), max(rows) + 1), -1, dtype=np.int32), 0

    def rest(r, a):
        return np.maximum(np.float32(0), (pr[r].astype(np.float64) - np.float64(a) * qr[r].astype(np.float64)).astype(np.float32))

    def whole(w):
        return np.floor(w.astype(np.float64) * 2.0 ** 40).astype(np.int64)

    for i, (n, parents) in enumerate(zip(rows, _trees(case))):
        pr, qr = p[r0:r0 + n].cpu().numpy(), None if q is None else q[r0:r0 + n].cpu().numpy()
        at, path, done = 0, [], False
        while not done:
            a, b, mass, done = np.float32(0), np.float32(1), 1.0, True
            for nth, c in enumerate(c for c in range(1, n) if parents[c] == at):
                x = tokens[r0 + c]
                if qr is None:
                    good = x == int(pr[at].argmax())
                else:
                    if nth:
                        b = np.float32(int(whole(rest(at, a)).sum()) * 2.0 ** -40 / mass)
                    with np.errstate(divide="ignore", invalid="ignore"):
                        good = np.float32(u[r0 + c]) < np.minimum(np.float32(1), rest(at, a)[x] / (b * qr[at, x]))  # (0 / 0 stays what it is)
                    if not good:
                        a = a + b
                        mass = max(mass - float(qr[at, x]), 2.0 ** -24) if case["distinct"] else 1.0
                if good:
                    path.append(c)
                    at, done = c, False
                    break
        if qr is None:
            token = int(pr[at].argmax())
        else:
            w = whole(rest(at, a))
            total = int(w.sum())
            bound = int(u[r0] * 2 ** 24) * total >> 24
            token = int(np.searchsorted(np.cumsum(w), bound, side="right")) if total else int(pr[at].argmax())
        result[i, :2 + len(path)] = [len(path), token] + path
        r0 += n
    return {"result": torch.from_numpy(result).to(_DEVICE)}


def exact(case, seed):
    do = case["do"]
    if do == "attend":
        return {"out": _exact_attend(case, seed, 0)}
    if do == "pass":
        return [_exact_attend(case, seed, layer) for layer in range(case["layers"])]
    if do == "accept":
        return _exact_accept(case, seed)
    # texts that begin as the same one
    context, clients, rows = case["context"], case["clients"], case.get("rows", 0)
    k, v = [], []
    for layer in range(case["layers"]):
        text = _text(case, seed, layer, 0, context + (rows if do == "keep" else 0))
        new = _text(case, seed, layer, 1, clients * rows) if do == "fork" else None
        for into, j in ((k, 0), (v, 1)):
            parts = []
            for c in range(clients):
                parts.append(text[j][:context])
                if do == "fork":
                    parts.append(new[j][c * rows:(c + 1) * rows])
                if do == "keep":
                    parts.append(text[j][context:][_kept(case, c)])
            into.append(torch.cat(parts).double())
    return {"k": torch.stack(k), "v": torch.stack(v)}
