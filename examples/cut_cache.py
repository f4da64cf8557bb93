"""Drafts verified over a cache held in 4 bits that is cut to a budget whenever it has grown past it.

    python examples/cut_cache.py [--workload tiny|llama-1b|llama-8b|llama-13b] [--layers N] [--prompt N] [--keep N] [--recent N]
                                 [--slack N] [--rounds N] [--k N]

A Llama-shaped decoder with random weights, its forward in torch, its cache an nav.KV4Cache: every layer of a pass appends its
keys and values and attends, and the attention reports what weight it gave to each cached token.  The prompt goes in by pieces; its last
rows weigh it.  Then rounds of k drafts: a pass over the pending token and the drafts, the accept / resample decision, the
rejected rows forgotten.  When the cache holds more than keep + slack tokens it is cut, per layer and head, to the newest
`recent` and the heaviest others.  Positions go on from the uncut text, as keys are rotated before they are cached."""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2605_13319_amd import inputs as I  # noqa: E402
from paper_2605_13319_amd import nav  # noqa: E402

DEVICE = "cuda:0"


class Decoder:
    """Forward passes of one client over a 4-bit cache."""

    def __init__(self, shape: I.ModelShape, seed: int, cache: nav.KV4Cache, tokens: int):
        self.shape, self.cache = shape, cache
        self.dtype = torch.float32 if shape.dtype == I.DTYPE_F32 else torch.bfloat16

        def tensor(a):
            return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).to(DEVICE).view(self.dtype)

        w = I.make_weights(shape, seed)
        self.emb, self.head = tensor(w["tok_emb"]), tensor(w["lm_head"])
        self.qkv = [torch.cat([tensor(w[n][i]) for n in ("wq", "wk", "wv")]) for i in range(shape.n_layers)]
        self.o, self.down = ([tensor(m) for m in w[n]] for n in ("wo", "w_down"))
        self.gate_up = [torch.cat([tensor(w["w_gate"][i]), tensor(w["w_up"][i])]) for i in range(shape.n_layers)]
        # weights given to the cached tokens, of client 0
        self.mass = torch.zeros(1, shape.n_layers, shape.n_kv_heads, tokens, device=DEVICE)
        self.position = 0  # of the next token in the uncut text

    def norm(self, x):
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.shape.rms_eps)).to(self.dtype)

    def rotate(self, x, positions):
        half = self.shape.head_dim // 2
        angle = positions[:, None] * self.shape.rope_base ** (-torch.arange(half, device=DEVICE) / half)
        cos, sin = angle.cos()[:, None], angle.sin()[:, None]
        a, b = x[..., :half].float(), x[..., half:].float()
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(self.dtype)

    def forward(self, tokens, weigh: bool, decay: float = 1.0):
        """Logits after each of the tokens, which become the cache's last; with `weigh` the cached tokens get their weight."""
        s, n = self.shape, len(tokens)
        self.cache.extend([0], [n])
        positions = torch.arange(self.position, self.position + n, device=DEVICE, dtype=torch.float32)
        x = self.emb[torch.as_tensor(tokens, device=DEVICE, dtype=torch.long)].float()
        for layer in range(s.n_layers):
            q, k, v = (self.norm(x) @ self.qkv[layer].T).split([s.q_dim, s.kv_dim, s.kv_dim], -1)
            q = self.rotate(q.reshape(n, s.n_q_heads, s.head_dim), positions)
            k = self.rotate(k.reshape(n, s.n_kv_heads, s.head_dim), positions)
            self.cache.append(layer, k, v)  # (v: columns of the wider product, as they are)
            o = self.cache.attend(layer, q, mass=self.mass if weigh else None, decay=decay)
            x = x + (o.flatten(1) @ self.o[layer].T).float()
            g, u = (self.norm(x) @ self.gate_up[layer].T).float().chunk(2, -1)
            x = x + ((torch.nn.functional.silu(g) * u).to(self.dtype) @ self.down[layer].T).float()
        self.position += n
        return (self.norm(x) @ self.head.T).float()

    def forget(self, n: int) -> None:
        """Take back the last n tokens."""
        self.cache.truncate([0], [self.cache.length(0) - n])
        self.position -= n


def run(shape, prompt: int, keep: int, recent: int, slack: int, rounds: int, k: int, seed: int = 1, make_cache=nav.KV4Cache, say=print):
    """Returns (lengths of the cache after each round, accepted drafts of each round, the decoder)."""
    most = max(prompt, keep + slack) + k + 1
    blocks = -(-most // 16) + -(-keep // 16)  # (a cut goes to fresh blocks)
    cache = make_cache(shape, 1, blocks)
    say(f"{shape.name}: a block of 16 tokens takes {cache.block_bytes} bytes, {16 * shape.kv_bytes_per_token()} as it is computed")
    model = Decoder(shape, seed + I.SEED_WEIGHTS, cache, blocks * 16)
    text = I.make_tokens(prompt, shape.vocab, seed + I.SEED_PREFIX)
    # The last rows of the prompt weigh all of it; so do, with what was before counting less and less, the rounds.
    last = min(32, prompt - 1)
    start = time.perf_counter()
    for first in range(0, prompt - 1 - last, 1024):
        model.forward(text[first:min(first + 1024, prompt - 1 - last)], weigh=False)
    if last:
        model.forward(text[prompt - 1 - last:prompt - 1], weigh=True, decay=0.0)
    torch.cuda.synchronize()
    say(f"prompt of {prompt} tokens: {1e3 * (time.perf_counter() - start):.1f} ms")
    pending, lengths, accepted = int(text[-1]), [], []
    result = torch.zeros(2, dtype=torch.int32, device=DEVICE)
    for r in range(rounds):
        drafts, probs = I.make_independent_drafts(k, shape.vocab, seed + I.SEED_NOISE + 100 * r, seed + I.SEED_DRAFT_U + 100 * r)
        probs = torch.from_numpy(probs).to(DEVICE)
        torch.cuda.synchronize()
        start = time.perf_counter()
        cut = cache.length(0) > keep + slack
        if cut:
            cache.evict([0], [0], keep, recent, model.mass)
        logits = model.forward([pending, *drafts.tolist()], weigh=True, decay=0.9)
        nav.spec_accept_static(logits.softmax(-1), probs, drafts.tolist(), I.make_uniforms(k + 1, seed + I.SEED_VERIFY_U + r), result)
        took, pending = result.tolist()
        model.forget(k - took)
        lengths.append(cache.length(0))
        accepted.append(took)
        say(f"round {r}: {took} of {k} drafts, {lengths[-1]} tokens cached at position {model.position}"
            f"{' (cut)' if cut else ''}, {1e3 * (time.perf_counter() - start):.2f} ms")
    return lengths, accepted, model


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--workload", default="llama-1b", choices=sorted(I.WORKLOADS))
    for name, default in (("layers", 4), ("prompt", 4096), ("keep", 1024), ("recent", 128), ("slack", 64), ("rounds", 24), ("k", 4)):
        p.add_argument(f"--{name}", type=int, default=default)
    a = p.parse_args()
    model_shape = I.WORKLOADS[a.workload]["shape"]
    run(model_shape.truncated(min(a.layers, model_shape.n_layers)), a.prompt, a.keep, a.recent, a.slack, a.rounds, a.k)
