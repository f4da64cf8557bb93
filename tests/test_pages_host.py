"""The paged cache of operators without a GPU: what is refused (and changes nothing), and which blocks clients hold, alone or with
others, through random calls, against a count by hand."""
import ctypes as C
import random

import numpy as np
import pytest
import torch

from paper_2605_13319_amd import inputs as I
from paper_2605_13319_amd import nav


def shape_of(nq=8, nkv=2, dim=64, dtype=I.DTYPE_BF16, layers=2):
    return I.ModelShape("pages", layers, 512, nq, nkv, dim, 512, 512, dtype=dtype)


def cache(max_seqs=4, blocks=8, **kw):
    return nav.PageCache(shape_of(**kw), max_seqs, blocks, on_device=False)


def refused(status, call, *args):
    with pytest.raises(nav.PipesdError) as e:
        call(*args)
    assert e.value.status == status


def state(pg):
    return [(pg.length(s), pg.seq_blocks(s)) for s in range(pg.max_seqs)], pg.free_blocks()


@pytest.mark.parametrize("bad", [dict(nq=3, nkv=2), dict(dim=96), dict(nq=514, nkv=2), dict(layers=0), dict(dtype=5)])
def test_configs_that_are_refused(bad):
    refused(nav.EINVAL, lambda: cache(**bad))


def test_create_refuses():
    cfg, h = nav.config_of(shape_of()), C.c_void_p()
    bb = nav._lib.pipesd_pages_block_bytes(C.byref(cfg), 16)
    assert bb == 2 * 2 * 2 * 64 * 16 * 2
    make = nav._lib.pipesd_pages_create
    assert nav._lib.pipesd_pages_block_bytes(C.byref(cfg), 8) == 0
    for args in ((C.byref(cfg), 0, 16, None, bb), (C.byref(cfg), 1, 8, None, bb), (C.byref(cfg), 1, 16, None, bb - 1), (C.byref(cfg), 1, 16, 257, bb),
                 (C.byref(cfg), 1 << 20, 16, None, bb << 11), (C.byref(cfg), 1, 16, None, bb << 27), (None, 1, 16, None, bb)):
        assert make(*args, C.byref(h)) == nav.EINVAL
    assert make(C.byref(cfg), 1, 16, None, bb, None) == nav.EINVAL
    assert nav._lib.pipesd_pages_destroy(None) == nav.EINVAL


def test_passes_that_are_refused_change_nothing():
    pg = cache()
    pg.extend([0, 1], [20, 3])
    before = state(pg)
    for ids, n, parents in (([4], [1], None), ([-1], [1], None), ([0, 0], [1, 1], None), ([2, 1, 2], [1, 1, 1], None), ([0], [0], None), ([0], [-1], None),
                            ([0], [2], [-1, 1]), ([0], [2], [0, 0]), ([0], [2], [-2, 0]), ([0, 2], [1, 2], [-1, -1, 1]), ([2], [257], list(range(-1, 256))),
                            ([2], [2 ** 30], None)):
        refused(nav.EINVAL, pg.extend, ids, n, parents)
        assert state(pg) == before
    refused(nav.ENOMEM, pg.extend, [2], [16 * 6], None)
    assert state(pg) == before
    with pytest.raises(ValueError):
        pg.extend([0], [1, 2])
    with pytest.raises(ValueError):
        pg.extend([0], [2], [-1])
    refused(nav.ESTATE, pg.truncate, [0], [21])
    refused(nav.ESTATE, pg.truncate, [0], [-1])
    refused(nav.EINVAL, pg.truncate, [0, 0], [1, 1])
    assert state(pg) == before
    pg.extend([2], [16 * 5])
    assert pg.free_blocks() == 0


def test_targets_that_are_refused():
    pg = cache()
    pg.extend([0, 1], [40, 3])
    before = state(pg)
    for call in (pg.fork, pg.copy):
        for ids, into, n in (([0], [0], None), ([0, 1], [2, 1], None), ([0, 0], [2, 2], None), ([0], [4], None), ([5], [2], None)):
            refused(nav.EINVAL, call, ids, into, n)
        refused(nav.ESTATE, call, [0], [2], [41])
        refused(nav.ESTATE, call, [0], [2], [-1])
        with pytest.raises(ValueError):
            call([0], [2, 3])
        with pytest.raises(ValueError):
            call([0], [2], [1, 2])
    refused(nav.ENOMEM, pg.copy, [0, 0], [2, 3], None)  # 6 blocks, 4 free
    assert state(pg) == before
    pg.copy([0], [1])  # (its own block counts)
    assert state(pg) == ([(40, 3), (40, 3), (0, 0), (0, 0)], 2)
    pg.fork([0, 0], [2, 3], [40, 33])
    assert state(pg) == ([(40, 3), (40, 3), (40, 3), (33, 3)], 2)
    refused(nav.ENOMEM, pg.copy, [0], [2])  # what the target holds is not its alone: 3 of 2
    assert state(pg) == ([(40, 3), (40, 3), (40, 3), (33, 3)], 2)


def test_compactions_that_are_refused():
    pg = cache()
    pg.extend([0, 1], [40, 3])
    before = state(pg)
    for first, kept, status in (([41], [[]], nav.ESTATE), ([-1], [[]], nav.EINVAL), ([38], [[2]], nav.ESTATE), ([38], [[0, 0]], nav.EINVAL),
                                ([30], [[5, 3]], nav.EINVAL), ([30], [[-1]], nav.EINVAL)):
        refused(status, pg.compact, [0], first, kept)
    refused(nav.EINVAL, pg.compact, [0, 0], [1, 1], [[], []])
    refused(nav.EINVAL, pg.compact, [0, 7], [1, 1], [[], []])
    with pytest.raises(ValueError):
        pg.compact([0], [1], [[], []])
    assert state(pg) == before
    pg.fork([0, 0], [2, 3])
    pg.extend([1], [16 * 4 + 13])  # no block is left
    assert pg.free_blocks() == 0
    refused(nav.ENOMEM, pg.compact, [0], [20], [[1]])
    pg.compact([0], [20], [[0, 1, 2]])  # (what stays where it is needs no block)
    assert pg.length(0) == 23 and pg.seq_blocks(0) == 2 and pg.free_blocks() == 0


def test_calls_without_a_pool_or_a_pass():
    pg = cache()
    pg.extend([0], [3])
    x = C.c_void_p(4096)
    assert nav._lib.pipesd_pages_append(pg.handle, 0, x, 128, x, 128, None) == nav.ESTATE
    assert nav._lib.pipesd_pages_attend(pg.handle, 0, x, 512, C.c_void_p(1 << 20), 512, None) == nav.ESTATE
    for layer, q, qs, o, os_ in ((2, 4096, 512, 1 << 20, 512), (-1, 4096, 512, 1 << 20, 512), (0, 0, 512, 1 << 20, 512), (0, 4098, 512, 1 << 20, 512),
                                 (0, 4096, 504, 1 << 20, 512), (0, 4096, 516, 1 << 20, 512), (0, 4096, 512, 4096 + 1024, 512), (0, 4096, 512, 4096, 1024)):
        assert nav._lib.pipesd_pages_attend(pg.handle, layer, C.c_void_p(q), qs, C.c_void_p(o), os_, None) == nav.EINVAL, (layer, q, qs, o, os_)
    assert nav._lib.pipesd_pages_append(pg.handle, 0, x, 120, x, 128, None) == nav.EINVAL
    one, zero, n = (C.c_int32 * 1)(1), (C.c_int32 * 1)(0), (C.c_int32 * 1)(4)
    assert nav._lib.pipesd_pages_read(pg.handle, 1, zero, zero, n, 0, 1, x, x, None) == nav.ESTATE
    assert nav._lib.pipesd_pages_read(pg.handle, 1, zero, zero, one, 0, 3, x, x, None) == nav.EINVAL
    assert nav._lib.pipesd_pages_read(pg.handle, 1, zero, zero, one, 0, 1, x, C.c_void_p(4100), None) == nav.EINVAL
    assert nav._lib.pipesd_pages_read(pg.handle, 1, zero, zero, one, 0, 1, x, x, None) == nav.ESTATE  # no pool


class Count:
    """Which blocks clients hold, by name: shared ones are the same name."""

    def __init__(self, max_seqs, blocks):
        self.len, self.held, self.blocks, self.names = [0] * max_seqs, [[] for _ in range(max_seqs)], blocks, 0

    def free(self):
        return self.blocks - len({b for h in self.held for b in h})

    def fresh(self):
        self.names += 1
        return self.names

    def users(self, b):
        return sum(b in h for h in self.held)

    def extend(self, ids, ns):
        was = [list(h) for h in self.held]
        for c, n in zip(ids, ns):
            if n and self.len[c] % 16 and self.users(self.held[c][-1]) > 1:
                self.held[c][-1] = self.fresh()
            while len(self.held[c]) < -(-(self.len[c] + n) // 16):
                self.held[c].append(self.fresh())
        if len({b for h in self.held for b in h}) > self.blocks:
            self.held = was
            return False
        for c, n in zip(ids, ns):
            self.len[c] += n
        return True

    def cut(self, c, n):
        self.len[c] = n
        self.held[c] = self.held[c][:-(-n // 16)]

    def become(self, c, into, n, own):
        self.len[into] = n
        self.held[into] = [self.fresh() if own else b for b in self.held[c][:-(-n // 16)]]

    def compact(self, ids, firsts, kept):
        was = [list(h) for h in self.held]
        for c, f, k in zip(ids, firsts, kept):
            j = next((j for j, x in enumerate(k) if x != j), None)
            if j is not None:
                for b in range((f + j) // 16, -(-(f + len(k)) // 16)):
                    if self.users(self.held[c][b]) > 1:
                        self.held[c][b] = self.fresh()
        if len({b for h in self.held for b in h} | {b for h in was for b in h}) > self.blocks:
            self.held = was
            return False
        for c, f, k in zip(ids, firsts, kept):
            self.cut(c, f + len(k))
        return True


@pytest.mark.parametrize("seed", range(12))
def test_random_calls_hold_the_blocks_that_they_should(seed):
    r = random.Random(seed)
    clients, blocks = 6, 14
    pg, want, failed = cache(clients, blocks), Count(clients, blocks), 0
    for _ in range(400):
        do = r.choice(["extend", "extend", "extend", "cut", "fork", "copy", "compact"])
        ids = r.sample(range(clients), r.randint(1, clients))
        if do == "extend":
            ns = [r.choice([0, 1, 1, 5, 16, 40]) for _ in ids]
            if sum(ns) == 0:
                continue
            if want.extend(ids, ns):
                pg.extend(ids, ns, r.choice([None, [p for n in ns for p in ([-1] + [r.randint(-1, i) for i in range(n - 1)] if n else [])]]))
            else:
                failed += 1
                refused(nav.ENOMEM, pg.extend, ids, ns)
        elif do == "cut":
            ns = [r.randint(0, want.len[c]) for c in ids]
            pg.truncate(ids, ns)
            for c, n in zip(ids, ns):
                want.cut(c, n)
        elif do in ("fork", "copy"):
            into = ids[:r.randint(1, len(ids))]
            rest = [c for c in range(clients) if c not in into]
            if not rest:
                continue
            src = [r.choice(rest) for _ in into]
            ns = [r.choice([want.len[c], r.randint(0, want.len[c])]) for c in src]
            trial = [h for c, h in enumerate(want.held) if c not in into]
            need = sum(-(-n // 16) for n in ns) if do == "copy" else 0
            if len({b for h in trial for b in h}) + need > blocks:
                failed += 1
                refused(nav.ENOMEM, pg.copy, src, into, ns)
                continue
            getattr(pg, do)(src, into, ns)
            for c in into:
                want.cut(c, 0)
            for c, t, n in zip(src, into, ns):
                want.become(c, t, n, do == "copy")
        else:
            firsts = [r.randint(0, want.len[c]) for c in ids]
            kept = [sorted(r.sample(range(want.len[c] - f), r.randint(0, want.len[c] - f))) for c, f in zip(ids, firsts)]
            if want.compact(ids, firsts, kept):
                pg.compact(ids, firsts, kept)
            else:
                failed += 1
                refused(nav.ENOMEM, pg.compact, ids, firsts, kept)
        assert state(pg) == ([(want.len[c], len(want.held[c])) for c in range(clients)], want.free())
    assert failed > 5


def test_decisions_that_are_refused():
    """Checked on the host: no pointer is followed."""
    p = q = result = 4096
    work = 1 << 20
    size = nav._lib.pipesd_tree_accept_workspace()

    def call(rows=(3,), tokens=(0, 1, 2), parents=(-1, 0, 0), u=(0.5, 0.5, 0.5), vocab=10, ps=10, qs=10, stride=4, p=p, q=q, result=result, work=work,
             size=size, n=None):
        keep = [np.ascontiguousarray(x, np.int32) for x in (rows, tokens, parents)]
        uu = None if u is None else np.ascontiguousarray(u, np.float32)
        return nav._lib.pipesd_tree_accept(p, ps, q, qs, vocab, len(rows) if n is None else n, keep[0].ctypes.data, keep[1].ctypes.data, keep[2].ctypes.data,
                                           None if uu is None else uu.ctypes.data, 0, result, stride, work, size, None)

    for bad in (dict(p=None), dict(result=None), dict(work=None), dict(work=(1 << 20) + 8), dict(size=size - 1), dict(vocab=0), dict(vocab=(1 << 22) + 1, ps=1 << 23, qs=1 << 23),
                dict(ps=9), dict(qs=9), dict(stride=3), dict(n=0), dict(rows=(0,)), dict(rows=(257,), stride=300), dict(tokens=(0, 10, 1)), dict(tokens=(0, -1, 1)),
                dict(parents=(0, 0, 0)), dict(parents=(-1, -1, 0)), dict(parents=(-1, 0, 2)), dict(u=None), dict(u=(0.5, 1.0, 0.5)), dict(u=(0.5, -0.1, 0.5)),
                dict(u=(float("nan"), 0.5, 0.5)), dict(p=4098), dict(result=4098)):
        assert call(**bad) == nav.EINVAL, bad
    import torch

    with pytest.raises(ValueError):
        nav.tree_accept(torch.zeros(3, 4), None, [0, 0, 0], [-1, 0, 0], None)
    with pytest.raises(ValueError):
        nav.tree_accept(torch.zeros(3, 4), None, [0, 0], [-1, 0, 0], None)


def test_kept_tokens_of_any_kind_of_integers():
    pg = cache(2, 20)
    for kept in ([1, 4, 7], (1, 4, 7), range(1, 8, 3), np.array([1, 4, 7]), np.array([1, 4, 7], dtype=np.int16), torch.tensor([1, 4, 7])):
        pg.extend([0], [30])
        pg.compact([0], [3], [kept])
        assert pg.length(0) == 6
        pg.truncate([0], [0])
    pg.extend([0], [30])
    for kept in ([1.0, 4.0], np.array([1.0]), ["1"], [2 ** 40]):
        with pytest.raises((TypeError, OverflowError)):
            pg.compact([0], [3], [kept])
    assert pg.length(0) == 30
