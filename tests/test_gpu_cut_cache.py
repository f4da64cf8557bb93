"""The example that verifies drafts over a cut 4-bit cache: every attention of it against the definition in 64 bits over what the
cache holds, every cut against the weights that the attentions gave, lengths and positions against the decisions."""
import math

import pytest
import torch

from examples import cut_cache
from paper_2605_13319_amd import inputs as I
from paper_2605_13319_amd import nav
from tests.test_gpu_kv4 import check_rows

gpu = pytest.mark.gpu


class Checked(nav.KV4Cache):
    """Compares what it does; keeps the weights that each token was given, token by token, in 64 bits."""
    passes = cuts = 0

    def attend(self, layer, q, out=None, limits=None, mass=None, decay=1.0):
        s = self.shape
        n, length = q.shape[0], self.length(0)
        k, v = (x[0].double() for x in self.read([0], [0], [length], layer0=layer, n_layers=1))
        was = None if mass is None else mass[0, layer, :, :length].double()
        got = super().attend(layer, q, out, limits, mass, decay)
        group = s.n_q_heads // s.n_kv_heads
        blind = torch.arange(length, device="cuda")[None] > torch.arange(length - n, length, device="cuda")[:, None]
        for h in range(s.n_kv_heads):
            weight = torch.zeros(length, dtype=torch.float64, device="cuda")
            a_most = 0.0
            for g in range(h * group, (h + 1) * group):
                x = q[:, g].double()
                a = (x.abs() @ k[:, h].abs().T.contiguous()).masked_fill(blind, 0).amax(-1, keepdim=True) / math.sqrt(s.head_dim)
                p = (x @ k[:, h].T.contiguous() / math.sqrt(s.head_dim)).masked_fill(blind, -torch.inf).softmax(-1)
                check_rows(got[:, g], (p @ v[:, h]).cpu(), (p @ v[:, h].abs()).cpu(), a.cpu(), "f32" if s.dtype == I.DTYPE_F32 else "bf16")
                weight += p.sum(0)
                a_most = max(a_most, float(a.max()))
            if mass is not None:
                old = torch.where(torch.arange(length, device="cuda") < length - n, decay * was[h], 0) if decay else 0
                # (the old weights are what the buffer had; a product and a sum of fp32 numbers: 2^-22)
                bound = 2.0 ** -18 * (1 + a_most) * weight + 2.0 ** -22 * (weight + old) + 1e-30
                assert bool(((mass[0, layer, h, :length].double() - old - weight).abs() <= bound).all())
        self.passes += 1
        return got

    def evict(self, seqs, into, keep, recent, mass, kept=None):
        length = self.length(0)
        before = mass[0, :, :, :length].cpu()
        k, v = (x.cpu() for x in self.read([0], [0], [length]))
        kept = super().evict(seqs, into, keep, recent, mass, kept)
        heavy = torch.sort(torch.argsort(-before[..., :length - recent], dim=-1, stable=True)[..., :keep - recent], -1).values
        want = torch.cat([heavy, torch.arange(length - recent, length).expand(*heavy.shape[:2], recent)], -1)
        assert torch.equal(kept[0].cpu().long(), want)
        assert torch.equal(mass[0, :, :, :keep].cpu(), before.gather(-1, want))
        index = want.permute(0, 2, 1)[..., None].expand(-1, -1, -1, self.shape.head_dim)
        for old, new in zip((k, v), self.read([0], [0], [keep])):
            assert torch.equal(new.cpu(), old.gather(1, index))
        self.cuts += 1
        return kept


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_drafts_over_a_cut_cache(dtype):
    shape = I.TINY if dtype == "f32" else I.ModelShape("small", 2, 256, 6, 2, 128, 512, 1000)
    lines = []
    lengths, accepted, model = cut_cache.run(shape, 300, 100, 20, 12, 9, 3, make_cache=Checked, say=lines.append)
    at = 299
    for length, took, line in zip(lengths, accepted, lines[2:]):
        if at > 112:
            assert "(cut)" in line
            at = 100
        at += 1 + took
        assert length == at
    assert model.position == 299 + 9 + sum(accepted)
    assert model.cache.cuts >= 1 and model.cache.passes == shape.n_layers * (2 + 9)
    used = model.cache.seq_blocks(0)
    assert used == -(-at // 16)


@gpu
def test_a_prompt_within_the_budget_is_not_cut():
    lengths, accepted, model = cut_cache.run(I.TINY, 40, 200, 20, 0, 3, 2, make_cache=Checked, say=lambda s: None)
    assert model.cache.cuts == 0 and lengths[-1] == 39 + 3 + sum(accepted)
