"""Rounds on trees of drafts as a server runs them: a small model's forward over the paged cache, drafts of several continuations, the decision,
the accepted path kept, the next round behind it.  With token matching the text is the model's own greedy text, whatever the drafts; and
whatever was accepted, the cache holds what a forward over the text alone gives."""
import math
import random

import pytest
import torch

from oracle.tree import tree_accept as checker
from paper_2605_13319_amd import inputs as I
from paper_2605_13319_amd import nav

gpu = pytest.mark.gpu
VOCAB, D, NQ, NKV, HD, LAYERS = 61, 128, 4, 2, 64, 2


class Toy:
    """Weights in 64 bits on the host, fp32 on the GPU; positions are added to the embeddings."""

    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
        self.emb, self.pos, self.head = rand(VOCAB, D), 0.3 * rand(400, D), rand(VOCAB, D) / math.sqrt(D)
        self.w = [{n: rand(o, i) / math.sqrt(i) for n, o, i in (("q", NQ * HD, D), ("k", NKV * HD, D), ("v", NKV * HD, D), ("o", D, NQ * HD))} for _ in range(LAYERS)]
        dev = lambda x: x.float().cuda()
        self.gpu = (dev(self.emb), dev(self.pos), dev(self.head), [{n: dev(x) for n, x in w.items()} for w in self.w])

    def text(self, tokens):
        """(logits, [(k, v)] of the layers) of a text alone, in 64 bits."""
        n = len(tokens)
        x, kv = self.emb[tokens] + self.pos[:n], []
        hidden = torch.triu(torch.ones(n, n, dtype=torch.bool), 1)
        for w in self.w:
            h = x / x.pow(2).mean(-1, keepdim=True).sqrt()
            q, k, v = (h @ w[m].T for m in "qkv")
            q, k, v = q.view(n, NKV, NQ // NKV, HD), k.view(n, NKV, HD), v.view(n, NKV, HD)
            kv.append((k, v))
            z = torch.einsum("rhgd,thd->hgrt", q, k) / math.sqrt(HD)
            p = torch.softmax(z.masked_fill(hidden, -torch.inf), -1)
            x = x + torch.einsum("hgrt,thd->rhgd", p, v).reshape(n, NQ * HD) @ w["o"].T
        return x @ self.head.T, kv

    def rows(self, cache, seqs, tokens, depths, parents, counts):
        """Logits of a pass's rows: the model over the cache."""
        emb, pos, head, layers = self.gpu
        cache.extend(seqs, counts, parents)
        x = emb[tokens] + pos[depths]
        for i, w in enumerate(layers):
            h = x / x.pow(2).mean(-1, keepdim=True).sqrt()
            qkv = h @ torch.cat([w[m] for m in "qkv"]).T
            q, k, v = qkv.split([NQ * HD, NKV * HD, NKV * HD], 1)  # (columns of one matrix, as fused projections leave them)
            cache.append(i, k, v)
            x = x + cache.attend(i, q, out=torch.empty_like(x[:, :1].expand(-1, NQ * HD).contiguous())) @ w["o"].T
        return x @ head.T


def greedy(model, prompt, n):
    text, margin = list(prompt), math.inf
    for _ in range(n):
        z = model.text(text)[0][-1]
        two = z.topk(2)
        margin = min(margin, float(two.values[0] - two.values[1]))
        text.append(int(two.indices[0]))
    return text, margin


def make_tree(r, want, depth, width):
    """Rows of a round: the pending token, then drafts, some of them what comes next, in an order in which parents come first."""
    tokens, parents, depths = [None], [-1], [0]
    right = [0]  # rows on the true continuation
    for level in range(1, depth + 1):
        over = [i for i in range(len(tokens)) if depths[i] == level - 1]
        for _ in range(r.randint(1, width)):
            tokens.append(r.randrange(VOCAB))
            parents.append(r.choice(over))
            depths.append(level)
        if right[-1] is not None and depths[right[-1]] == level - 1 and r.random() < 0.75:
            tokens.append(want[level - 1])
            parents.append(right[-1])
            depths.append(level)
            right.append(len(tokens) - 1)
    return tokens, parents, depths


def compare_cache(cache, model, seq, text):
    """fp32 sums over D and the text against 64 bits: 2^-24 times a few hundred operations and the layers' growth, 1e-4 allowed of values of about 1
    to 4."""
    n = cache.length(seq)
    _, kv = model.text(text[:n])
    k, v = cache.read([seq], [0], [n])
    for layer in range(LAYERS):
        for got, want in zip((k[layer], v[layer]), kv[layer]):
            assert float((got.cpu().double() - want).abs().max()) < 1e-4


@gpu
def test_token_matching_gives_the_models_own_text():
    model, r = Toy(1), random.Random(5)
    prompts = [[r.randrange(VOCAB) for _ in range(n)] for n in (1, 37, 16)]
    wants = [greedy(model, p, 60) for p in prompts]
    margin = min(m for _, m in wants)  # of the best logit over the next: their order holds as long as each is off by less than half of it
    cache = nav.PageCache(I.ModelShape("toy", LAYERS, D, NQ, NKV, HD, 512, 512, dtype=I.DTYPE_F32), 3, 60)
    cache.pool.fill_(255)
    texts = [list(p) for p in prompts]  # committed; all but the last are cached
    for c, p in enumerate(prompts):
        if len(p) > 1:
            model.rows(cache, [c], p[:-1], list(range(len(p) - 1)), None, [len(p) - 1])
    accepted = rounds = 0
    while min(len(t) - len(p) for t, p in zip(texts, prompts)) < 50:
        seqs = [c for c in range(3) if len(texts[c]) - len(prompts[c]) < 50]
        trees = [make_tree(r, wants[c][0][len(texts[c]):], 4, 3) for c in seqs]
        before = [cache.length(c) for c in seqs]
        assert before == [len(texts[c]) - 1 for c in seqs]
        tokens = [x for c, (t, _, _) in zip(seqs, trees) for x in [texts[c][-1]] + t[1:]]
        parents = [x for _, p, _ in trees for x in p]
        depths = [b + x for b, (_, _, d) in zip(before, trees) for x in d]
        counts = [len(t) for t, _, _ in trees]
        z = model.rows(cache, seqs, tokens, depths, parents, counts)
        got = nav.tree_accept(torch.softmax(z, -1), None, tokens, parents, None, rows=counts).cpu().tolist()
        paths = [row[2:2 + row[0]] for row in got]
        cache.compact(seqs, before, [[0] + path for path in paths])
        at = 0
        for c, path, row, n in zip(seqs, paths, got, counts):
            texts[c] += [tokens[at + i] for i in path]
            assert float((z[[at] + [at + i for i in path]].cpu().double() - model.text(texts[c])[0][-1 - len(path):]).abs().max()) < margin / 2
            texts[c].append(row[1])
            at += n
            accepted += len(path)
            rounds += 1
    assert accepted > rounds  # (the drafts were worth it)
    for c in range(3):
        n = len(texts[c])
        assert texts[c] == wants[c][0][:n]
        compare_cache(cache, model, c, texts[c])


@gpu
def test_sampling_rounds_keep_the_cache_of_the_text():
    """Drafts drawn without putting back from a noisy target; clients forked from one prompt go their own ways; every decision is the checker's."""
    model, r = Toy(2), random.Random(6)
    g = torch.Generator(device="cuda").manual_seed(3)
    prompt = [r.randrange(VOCAB) for _ in range(45)]
    cache = nav.PageCache(I.ModelShape("toy", LAYERS, D, NQ, NKV, HD, 512, 512, dtype=I.DTYPE_F32), 4, 80)
    cache.pool.fill_(255)
    model.rows(cache, [0], prompt[:-1], list(range(44)), None, [44])
    cache.fork([0, 0, 0], [1, 2, 3])
    texts = [list(prompt) for _ in range(4)]
    parents = [-1, 0, 0, 0, 1, 1, 2, 4, 4]
    depth = [0, 1, 1, 1, 2, 2, 2, 3, 3]
    n = len(parents)
    work = nav.tree_workspace(4, 4 * n)
    accepted = 0
    for _ in range(8):
        before = [cache.length(c) for c in range(4)]
        # the draft model: the target's logits along the tree, noisy (here: from a look at the target, forgotten again)
        tokens = [[t[-1]] + [0] * (n - 1) for t in texts]
        qs = torch.zeros(4, n, VOCAB, device="cuda")
        for level in range(4):
            flat = [x for t in tokens for x in t]
            z = model.rows(cache, [0, 1, 2, 3], flat, [b + x for b in before for x in depth], parents * 4, [n] * 4).view(4, n, VOCAB)
            cache.truncate([0, 1, 2, 3], before)
            for row in [i for i in range(n) if depth[i] == level]:
                children = [i for i in range(n) if parents[i] == row]
                if children:
                    qs[:, row] = torch.softmax(z[:, row] + 0.5 * torch.randn(4, VOCAB, generator=g, device="cuda"), -1)
                    for c, drawn in enumerate(torch.multinomial(qs[:, row], len(children), generator=g).tolist()):
                        for i, x in zip(children, drawn):
                            tokens[c][i] = x
        flat = [x for t in tokens for x in t]
        p = torch.softmax(model.rows(cache, [0, 1, 2, 3], flat, [b + x for b in before for x in depth], parents * 4, [n] * 4), -1)
        u = (torch.randint(0, 1 << 24, (4 * n,), generator=g, device="cuda").float() * 2.0 ** -24).tolist()
        got = nav.tree_accept(p, qs.view(4 * n, VOCAB), flat, parents * 4, u, rows=[n] * 4, distinct=True, workspace=work).cpu().tolist()
        for c in range(4):
            part = slice(c * n, (c + 1) * n)
            path, token = checker(p[part].cpu().numpy(), qs[c].cpu().numpy(), tokens[c], parents, u[part], True)
            assert got[c] == [len(path), token] + path + [-1] * (n - 1 - len(path))
            texts[c] += [tokens[c][i] for i in path] + [token]
            accepted += len(path)
        cache.compact([0, 1, 2, 3], before, [[0] + row[2:2 + row[0]] for row in got])
    assert accepted > 16
    assert len({tuple(t) for t in texts}) == 4
    for c in range(4):
        compare_cache(cache, model, c, texts[c])
