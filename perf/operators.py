"""The operators on a 4-bit cache as cases that can be timed and checked, beside their plain forms.

The 4-bit cache holds keys and values as e2m1 numbers (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with one power of
two per 32 neighbouring channels of a token and head: 4.25 bits a value, where the bf16 cache takes 16.  A server keeps
long contexts, or many clients, in it.  The operators:

  store   new rows of several clients are rounded into the cache, and read back as the values it then holds;
  attend  query rows of several clients attend to their caches (causal, or as many tokens as the caller says), and
          the weight that the rows gave to every cached token is summed where the caller asks for it;
  evict   a client's cache is cut to a budget: the newest tokens and, of the others, those that were given the
          most weight (per layer and head); the kept cache is read back as values.

Rounding.  A block of 32 values with largest magnitude a gets the power 2^e, e the smallest integer with a <= 7 * 2^e, at
least -125 and at most 125; a value x becomes the nearest number to x / 2^e, ties to the even code (0, 1, 2, 4 before
0.5, 1.5, 3, 6), at most 6.

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
        # a step of sixteen clients that generate one token each: latency
        {"name": "store_8b_16x1", "do": "store", "heads": "8b", "dtype": "bf16", "clients": 16, "context": 4096, "rows": 1},
        # a prompt block behind a context that ends inside a cache block
        {"name": "store_8b_2048", "do": "store", "heads": "8b", "dtype": "bf16", "clients": 1, "context": 1531, "rows": 2048},
        # the small fp32 model verifies four drafts
        {"name": "attend_tiny_k4", "do": "attend", "heads": "tiny", "dtype": "f32", "clients": 1, "context": 128, "rows": 5, "limits": False, "mass": False},
        # one token at a time behind a short context, head dim 64
        {"name": "attend_1b_decode", "do": "attend", "heads": "1b", "dtype": "bf16", "clients": 1, "context": 1023, "rows": 1, "limits": False, "mass": False},
        # the headline round: eight drafts behind 2048 tokens
        {"name": "attend_8b_k8", "do": "attend", "heads": "8b", "dtype": "bf16", "clients": 1, "context": 2048, "rows": 9, "limits": False, "mass": False},
        # sixteen clients of all lengths, a number of rows each, some of which see less than their text or nothing
        {"name": "attend_8b_batch16", "do": "attend", "heads": "8b", "dtype": "bf16", "clients": 16, "context": 4096, "rows": 17, "limits": True, "mass": False},
        # one token at a time at the far end of a long context: what the cache is for
        {"name": "attend_8b_long", "do": "attend", "heads": "8b", "dtype": "bf16", "clients": 1, "context": 131071, "rows": 1, "limits": False, "mass": False},
        # four clients with long contexts and long drafts, no shared heads
        {"name": "attend_13b_batch4", "do": "attend", "heads": "13b", "dtype": "bf16", "clients": 4, "context": 8192, "rows": 17, "limits": False, "mass": False},
        # a block of a long prompt behind what is cached of it
        {"name": "attend_8b_prompt", "do": "attend", "heads": "8b", "dtype": "bf16", "clients": 1, "context": 6144, "rows": 2048, "limits": False, "mass": False},
        # a prompt's last rows weigh its tokens, so that a cut can follow
        {"name": "attend_1b_mass", "do": "attend", "heads": "1b", "dtype": "bf16", "clients": 1, "context": 12001, "rows": 32, "limits": False, "mass": True},
        # a short context cut to its budget, all layers
        {"name": "evict_1b_777", "do": "evict", "heads": "1b", "dtype": "bf16", "layers": 16, "context": 777, "keep": 512, "recent": 32},
        # a long one cut to a quarter
        {"name": "evict_8b_8192", "do": "evict", "heads": "8b", "dtype": "bf16", "layers": 32, "context": 8192, "keep": 2048, "recent": 256},
    ]


def draw(rng):
    def spread(low, high):
        return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))

    most = [work(c) for c in listed()]
    most_bytes, most_flops = (max(w[k] for w in most) for k in ("bytes", "flops"))
    while True:
        do = rng.choice(["store", "attend", "attend", "attend", "evict"])
        heads, dtype = rng.choice(sorted(_HEADS)), rng.choice(["bf16", "bf16", "f32"])
        if do == "store":
            clients = spread(1, 16)
            case = {"do": do, "heads": heads, "dtype": dtype, "clients": clients, "context": spread(1, 8192), "rows": spread(1, 2048 // clients)}
        elif do == "evict":
            context = spread(2, 16384)
            keep = max(1, int(context * rng.uniform(0.1, 1.0)))
            case = {"do": do, "heads": heads, "dtype": dtype, "layers": rng.randint(1, 16), "context": context, "keep": keep, "recent": rng.randint(0, keep)}
        else:
            clients = spread(1, 16) if rng.random() < 0.6 else 1
            rows = spread(1, 32) if clients > 1 or rng.random() < 0.7 else spread(33, 2048)
            case = {"do": do, "heads": heads, "dtype": dtype, "clients": clients, "context": spread(1, 131072 // clients), "rows": rows,
                    "limits": rng.random() < 0.3, "mass": rng.random() < 0.3}
        w = work(case)
        if w["bytes"] <= most_bytes and w["flops"] <= most_flops:
            return case


def _lengths(case):
    """(tokens that a client has cached before the pass, its new rows), per client; the first has the most of both."""
    r = random.Random(case["clients"] * 1000003 + case["context"] * 101 + case["rows"])
    before, rows = [case["context"]], [case["rows"]]
    for _ in range(case["clients"] - 1):
        before.append(r.randint(0, case["context"]))
        rows.append(r.randint(1, case["rows"]))
    return before, rows


def work(case):
    nq, nkv, dim = _HEADS[case["heads"]]
    size = 4 if case["dtype"] == "f32" else 2
    token = nkv * 2 * (dim // 2 + dim // 32)  # bytes of a token in the cache of a layer
    values = nkv * 2 * dim * size             # and as numbers
    if case["do"] == "store":
        _, rows = _lengths(case)
        # numbers in, the cache's bytes out; the read back: those in, numbers out
        return {"bytes": 2 * sum(rows) * (values + token), "flops": 0}
    if case["do"] == "evict":
        kept = case["layers"] * case["keep"]
        # weights in and the kept ones out, indices out, the kept bytes in and out; the read back
        return {"bytes": case["layers"] * nkv * 4 * (case["context"] + 2 * case["keep"]) + kept * (3 * token + values), "flops": 0}
    before, rows = _lengths(case)
    total = [b + r for b, r in zip(before, rows)]
    seen = sum(r * b + r * (r + 1) // 2 for b, r in zip(before, rows))
    return {"bytes": sum(total) * token + sum(rows) * nq * dim * 2 * size + (sum(total) * nkv * 4 if case["mass"] else 0),
            "flops": 4 * dim * nq * seen}


# ---- inputs -------------------------------------------------------------------------------------


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _generator(seed, part):
    g = torch.Generator(device=_DEVICE)
    g.manual_seed(seed * 1009 + part)
    return g


def _keys_values(case, seed, layer, tokens):
    """A layer's keys and values [clients][tokens][heads][dim].  A few channels of the keys are several times larger than the
    others, as in trained models."""
    _, nkv, dim = _HEADS[case["heads"]]
    g = _generator(seed, 2 + layer)
    shape = (case.get("clients", 1), tokens, nkv, dim)
    large = 1 + 3 * (torch.rand(nkv, dim, generator=g, device=_DEVICE) < 0.05)
    k = torch.randn(shape, generator=g, device=_DEVICE) * large
    v = torch.randn(shape, generator=g, device=_DEVICE)
    return k.to(_type(case)), v.to(_type(case))


def _queries(case, seed, rows):
    nq, _, dim = _HEADS[case["heads"]]
    return (1.5 * torch.randn((rows, nq, dim), generator=_generator(seed, 0), device=_DEVICE)).to(_type(case))


def _limits(before, rows):
    """Tokens that each row sees: its own position and all before it, but every fifth row nothing, every seventh half, and the
    client's last row more than there are (which is all)."""
    lim = []
    for b, n in zip(before, rows):
        for i in range(n):
            seen = b + i + 1
            lim.append(0 if i % 5 == 3 else seen // 2 if i % 7 == 5 else seen + 100 if i == n - 1 and i > 0 else seen)
    return lim


def _weights(case, seed):
    """Accumulated weights [layers][heads][tokens]: few tokens hold most, many hold next to nothing and some exactly that."""
    _, nkv, _ = _HEADS[case["heads"]]
    g = _generator(seed, 1)
    w = torch.rand((case["layers"], nkv, case["context"]), generator=g, device=_DEVICE).pow(8) * 32
    return torch.where(torch.rand(w.shape, generator=g, device=_DEVICE) < 0.1, 0.0, w)


def _ints(v):
    return torch.tensor(v, dtype=torch.int64, device=_DEVICE)


# ---- plain forms --------------------------------------------------------------------------------


def _round(x):
    """x [..][dim] as codes: two to a byte (the even channel low), and the exponents' bytes (e + 127)."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    frac, power = torch.frexp(top / 7)                         # top / 7 = frac * 2^power, 0.5 <= frac < 1
    # (the quotient is rounded: whether top <= 7 * 2^power is asked of the product, which is exact)
    power = torch.where(top <= torch.ldexp(torch.full_like(top, 7), power - 1), power - 1, power)
    power = torch.where(top > torch.ldexp(torch.full_like(top, 7), power), power + 1, power)
    power = torch.where(top > 0, power, -125).clamp(-125, 125)
    y = torch.ldexp(x, -power.unsqueeze(-1))
    a = y.abs()
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5).int())
    code = (code + 8 * (y < 0).int()).flatten(-2).unflatten(-1, (-1, 2))
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), (power + 127).to(torch.uint8)


def _values(codes, powers):
    """The numbers that codes [..][dim / 2] with exponents [..][dim / 32] stand for, in 32 bits."""
    numbers = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    c = codes.int()
    y = numbers[torch.stack([c & 15, c >> 4], -1)].flatten(-2).unflatten(-1, (-1, 32))
    return (y * torch.exp2(powers.float() - 127).unsqueeze(-1)).flatten(-2)


def _plain_pages(layers, blocks, nkv, dim):
    """Blocks [layer][block][head][token] of codes and exponents, for keys and values."""
    return [torch.zeros((layers, blocks, nkv, _BLOCK, n), dtype=torch.uint8, device=_DEVICE) for n in (dim // 2, dim // 32) * 2]


def _plain_table(case, seed, tokens):
    """Blocks in no order [clients][blocks of a client]."""
    blocks = -(-tokens // _BLOCK)
    clients = case.get("clients", 1)
    return torch.randperm(clients * blocks, generator=_generator(seed, 99), device=_DEVICE).view(clients, blocks)


def _plain_put(pages, layer, block, token, k, v):
    for page, part in zip(pages, (*_round(k), *_round(v))):
        page[layer][block, :, token] = part


def _run_store(s):
    pages, block, token = s["pages"], s["block"], s["token"]
    _plain_put(pages, 0, block, token, s["k"], s["v"])
    kc, ke, vc, ve = (page[0][block, :, token] for page in pages)
    return {"k": _values(kc, ke).to(s["type"]), "v": _values(vc, ve).to(s["type"])}


def _run_attend(s):
    clients, most, nq, nkv, dim = s["sizes"]
    group = nq // nkv
    # [block][head][token][..] -> [client][head][tokens of a client][..]
    kc, ke, vc, ve = (page[0][s["table"]].permute(0, 2, 1, 3, 4).flatten(2, 3) for page in s["pages"])
    k, v = _values(kc, ke), _values(vc, ve)
    q = s["q"].float()[s["row_at"]]                               # [client][most rows][query head][dim]
    q = q.view(clients, most, nkv, group, dim).permute(0, 2, 1, 3, 4).reshape(clients, nkv, most * group, dim)
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(dim)
    sees = torch.arange(k.shape[2], device=score.device) < s["seen"].unsqueeze(-1)   # [client][most rows][token]
    sees = sees.unsqueeze(1).unsqueeze(3).expand(-1, nkv, -1, group, -1).reshape(score.shape)
    score = score.masked_fill(~sees, -torch.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -torch.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = torch.matmul(p, v).view(clients, nkv, most, group, dim).permute(0, 2, 1, 3, 4).reshape(clients * most, nq, dim)
    out = {"out": o[s["row_of"]].to(s["type"])}
    if s["mass"] is not None:
        out["mass"] = p.sum(2)[:, None, :, :s["mass"].shape[-1]]
    return out


def _run_evict(s):
    layers, nkv, context, keep, recent = s["sizes"]
    w = s["weights"]
    order = torch.sort(w[..., :context - recent], dim=-1, descending=True, stable=True).indices[..., :keep - recent]
    newest = torch.arange(context - recent, context, device=w.device).expand(layers, nkv, recent)
    kept = torch.cat([order, newest], -1).sort(-1).values         # [layer][head][kept]
    at = torch.arange(keep, device=w.device)
    from_block, from_token = s["table"][0][kept // _BLOCK], kept % _BLOCK
    to_block, to_token = s["to"][0][at // _BLOCK], at % _BLOCK
    one, two = torch.arange(layers, device=w.device)[:, None, None], torch.arange(nkv, device=w.device)[None, :, None]
    got = []
    for page, new in zip(s["pages"], s["new"]):
        new[one, to_block, two, to_token] = page[one, from_block, two, from_token]
        got.append(new[one, to_block, two, to_token].transpose(1, 2))   # [layer][kept][head][..]
    return {"kept": kept.int()[None], "mass": torch.gather(w, -1, kept)[None], "k": _values(got[0], got[1]).to(s["type"]),
            "v": _values(got[2], got[3]).to(s["type"])}


# ---- what a program has in hand -----------------------------------------------------------------


def _cache(case, layers, clients, tokens):
    """The library's 4-bit cache for `clients` clients of up to `tokens` tokens."""
    from paper_2605_13319_amd import inputs as I
    from paper_2605_13319_amd import nav

    nq, nkv, dim = _HEADS[case["heads"]]
    shape = I.ModelShape(case["heads"], layers, 512, nq, nkv, dim, 512, 512, dtype=I.DTYPE_F32 if case["dtype"] == "f32" else I.DTYPE_BF16)
    return nav.KV4Cache(shape, max_seqs=clients, n_blocks=clients * -(-tokens // _BLOCK))


def _fill(cache, layers, seqs, lengths, rows):
    """Tokens 0 .. length - 1 of every client, in passes of up to 2048 rows; rows(layer, client, first, n) gives a client's keys and values."""
    for c, n in zip(seqs, lengths):
        for first in range(0, n, 2048):
            part = min(2048, n - first)
            cache.extend([c], [part])
            for layer in range(layers):
                cache.append(layer, *rows(layer, c, first, part))


def prepare(case, seed):
    nq, nkv, dim = _HEADS[case["heads"]]
    s = {"do": case["do"], "type": _type(case)}
    if case["do"] == "evict":
        layers, context, keep = case["layers"], case["context"], case["keep"]
        s.update(sizes=(layers, nkv, context, keep, case["recent"]), weights=_weights(case, seed))
        if own:
            s["cache"] = _cache(case, layers, 2, context)
            s["mass"] = torch.zeros((2, layers, nkv, context), device=_DEVICE)
            s["mass"][0] = s["weights"]
        else:
            s["pages"], s["table"] = _plain_pages(layers, -(-context // _BLOCK), nkv, dim), _plain_table(case, seed, context)
            s["new"], s["to"] = _plain_pages(layers, -(-keep // _BLOCK), nkv, dim), _plain_table(case, seed + 1, keep)
        if own:
            s["cache"].extend([0], [context])
        for layer in range(layers):
            k, v = _keys_values(case, seed, layer, context)
            if own:
                s["cache"].append(layer, k[0], v[0])
            else:
                at = torch.arange(context, device=_DEVICE)
                _plain_put(s["pages"], layer, s["table"][0][at // _BLOCK], at % _BLOCK, k[0], v[0])
        return s

    before, rows = _lengths(case)
    clients, tokens, most = case["clients"], max(b + r for b, r in zip(before, rows)), max(rows)
    k, v = _keys_values(case, seed, 0, tokens)
    client = torch.repeat_interleave(torch.arange(clients, device=_DEVICE), _ints(rows))
    row = torch.cat([torch.arange(n, device=_DEVICE) for n in rows])
    pos = _ints(before)[client] + row
    new_k, new_v = k[client, pos].contiguous(), v[client, pos].contiguous()
    if own:
        s["cache"] = _cache(case, 1, clients, tokens)
        _fill(s["cache"], 1, range(clients), before, lambda layer, c, first, n: (k[c, first:first + n], v[c, first:first + n]))
        s["seqs"], s["before"], s["rows"] = list(range(clients)), before, rows
    else:
        s["pages"], s["table"] = _plain_pages(1, clients * -(-tokens // _BLOCK), nkv, dim), _plain_table(case, seed, tokens)
        every = torch.arange(tokens, device=_DEVICE)
        for c in range(clients):
            _plain_put(s["pages"], 0, s["table"][c][every // _BLOCK], every % _BLOCK, k[c], v[c])
        s["block"], s["token"] = s["table"][client, pos // _BLOCK], pos % _BLOCK
    if case["do"] == "store":
        s.update(k=new_k, v=new_v)
        return s
    lim = _ints(_limits(before, rows)) if case["limits"] else None
    s["q"] = _queries(case, seed, sum(rows))
    s["mass"] = torch.zeros((clients, 1, nkv, tokens), device=_DEVICE) if case["mass"] else None
    if own:
        s["cache"].extend(s["seqs"], rows)
        s["cache"].append(0, new_k, new_v)
        s["limits"] = None if lim is None else lim.int()
        s["out"] = torch.empty_like(s["q"])
    else:
        seen = torch.zeros((clients, most), dtype=torch.int64, device=_DEVICE)
        seen[client, row] = torch.minimum(pos + 1 if lim is None else lim, _ints([b + n for b, n in zip(before, rows)])[client])
        row_at = torch.zeros((clients, most), dtype=torch.int64, device=_DEVICE)
        row_at[client, row] = torch.arange(len(client), device=_DEVICE)
        s.update(sizes=(clients, most, nq, nkv, dim), seen=seen, row_at=row_at, row_of=client * most + row)
    return s


def run(s):
    if not own:
        return {"store": _run_store, "attend": _run_attend, "evict": _run_evict}[s["do"]](s)
    cache = s["cache"]
    if s["do"] == "store":
        cache.truncate(s["seqs"], s["before"])
        cache.extend(s["seqs"], s["rows"])
        cache.append(0, s["k"], s["v"])
        k, v = cache.read(s["seqs"], s["before"], s["rows"])
        return {"k": k[0], "v": v[0]}
    if s["do"] == "attend":
        out = {"out": cache.attend(0, s["q"], out=s["out"], limits=s["limits"], mass=s["mass"], decay=0.0)}
        if s["mass"] is not None:
            out["mass"] = s["mass"]
        return out
    layers, nkv, context, keep, recent = s["sizes"]
    kept = cache.evict([0], [1], keep, recent, s["mass"])
    k, v = cache.read([1], [0], [keep])
    return {"kept": kept, "mass": s["mass"][1:, :, :, :keep], "k": k, "v": v}


# ---- the definition in 64 bits ------------------------------------------------------------------


def _exact_values(x):
    """What the cache holds for x [..][dim], in 64 bits."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 7))
    e = torch.where(top > 7 * torch.exp2(e), e + 1, e)
    e = torch.where(top <= 7 * torch.exp2(e - 1), e - 1, e)
    power = torch.exp2(torch.where(top > 0, e, -125.0).clamp(-125, 125))
    a = (x / power).abs().clamp(max=6)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.sign(x) * torch.round(a / step) * step * power).flatten(-2)


def exact(case, seed):
    nq, nkv, dim = _HEADS[case["heads"]]
    if case["do"] == "evict":
        layers, context, keep, recent = case["layers"], case["context"], case["keep"], case["recent"]
        w = _weights(case, seed).double()
        old = w[..., :context - recent]
        # place of a token among the old ones: how many come before it in (weight falling, index rising)
        place = torch.argsort(torch.argsort(-old, dim=-1, stable=True), dim=-1)
        stays = torch.cat([place < keep - recent, torch.ones_like(w[..., :recent], dtype=torch.bool)], -1)
        kept = stays.nonzero()[:, 2].view(layers, nkv, keep)
        got = [[], []]
        for layer in range(layers):
            for into, x in zip(got, _keys_values(case, seed, layer, context)):
                into.append(_exact_values(torch.gather(x[0], 0, kept[layer].T[..., None].expand(-1, -1, dim))))
        return {"kept": kept.int()[None], "mass": w[stays].view(1, layers, nkv, keep), "k": torch.stack(got[0]), "v": torch.stack(got[1])}
    before, rows = _lengths(case)
    k, v = _keys_values(case, seed, 0, max(b + r for b, r in zip(before, rows)))
    if case["do"] == "store":
        return {name: torch.cat([_exact_values(x[c, b:b + n]) for c, (b, n) in enumerate(zip(before, rows))]) for name, x in (("k", k), ("v", v))}
    q, limits, r0, out = _queries(case, seed, sum(rows)).double(), _limits(before, rows), 0, []
    mass = torch.zeros((case["clients"], 1, nkv, k.shape[1]), dtype=torch.float64, device=_DEVICE)
    group = nq // nkv
    for c, (b, n) in enumerate(zip(before, rows)):
        seen = limits[r0:r0 + n] if case["limits"] else [b + i + 1 for i in range(n)]
        seen = _ints(seen).clamp(max=b + n)
        hidden = torch.arange(b + n, device=_DEVICE)[None, None] >= seen[None, :, None]
        o = torch.zeros((n, nq, dim), dtype=torch.float64, device=_DEVICE)
        for h in range(nkv):
            kh, vh = _exact_values(k[c, :b + n, h]), _exact_values(v[c, :b + n, h])
            z = (q[r0:r0 + n, h * group:(h + 1) * group].transpose(0, 1).reshape(group * n, dim) @ kh.T.contiguous() / math.sqrt(dim)).view(group, n, -1)
            p = torch.nan_to_num(torch.softmax(z.masked_fill(hidden, -torch.inf), -1))  # (rows that see nothing have no weights)
            o[:, h * group:(h + 1) * group] = (p.view(group * n, -1) @ vh).view(group, n, dim).transpose(0, 1)
            mass[c, 0, h, :b + n] = p.sum((0, 1))
        out.append(o)
        r0 += n
    return {"out": torch.cat(out), "mass": mass} if case["mass"] else {"out": torch.cat(out)}
