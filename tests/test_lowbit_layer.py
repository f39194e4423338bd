"""The operators in fewer bits as a decoder layer runs them: norms around the blocks, 8-bit
linears, the 4-bit cache with its append and attention (GPU), against the same layer in plain
float64 torch operations on the quantized weights, and seeded random batches through the cache.

The layer's tolerance: each 8-bit linear adds a relative error of its tokens' codes, half a step
of the largest of K values (max / 254 against their root mean square: about 4 / 254 / sqrt(3)), each
bf16 rounding 2^-8, and the 4-bit rows are shared with the reference, which reads them back; so
the outputs are within 5 % of the residual stream's part that the layer adds, in the 2-norm.
"""

import random

import numpy as np
import pytest
import torch

from oracle import lowbit_ref as low
from oracle import target_ref as ref
from paper_2607_04244_amd import qlin

from test_kv4 import HEAD, Cache, check_append, check_attention, i32, rand, starts

pytestmark = pytest.mark.gpu
WIDTH, HQ, HKV, INNER, EPS = 512, 8, 2, 768, 1e-6


class Layer:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.lin = {}
        for name, n, k in (("qkv", (HQ + 2 * HKV) * HEAD, WIDTH), ("o", WIDTH, HQ * HEAD), ("up", 2 * INNER, WIDTH), ("down", WIDTH, INNER)):
            w = torch.randn((n, k), generator=g) * k ** -0.5
            s = w.abs().amax(1) / 127
            self.lin[name] = (torch.round(w / s[:, None]).to(torch.int8).cuda(), s.cuda())
        self.norms = [(1 + 0.2 * torch.randn(WIDTH, generator=g)).to(torch.bfloat16).cuda() for _ in range(4)]
        self.qk = [(1 + 0.2 * torch.randn(HEAD, generator=g)).to(torch.bfloat16).cuda() for _ in range(2)]
        self.freq = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()

    def linear(self, name, x, gated=False):
        return qlin.linear_i8(*qlin.quantize_tokens(x, gated=gated), *self.lin[name])

    def run(self, h, x, cache, at, length, n):
        """The residual stream and its normed form, before and behind the layer."""
        y = self.linear("qkv", x)
        q, k, v = y[:, :HQ * HEAD], y[:, HQ * HEAD:(HQ + HKV) * HEAD], y[:, (HQ + HKV) * HEAD:]
        q = qlin.norm_rope_append_kv4(q, k, v, cache, at, length, max_new=n, q_norm=self.qk[0], k_norm=self.qk[1], inv_freq=self.freq)
        o = qlin.causal_attention_kv4(q, cache, at, length, max_new=n)
        x, h = qlin.block_norm(self.linear("o", o.view(-1, HQ * HEAD)), h, self.norms[1], post_norm=self.norms[0])
        y = self.linear("down", self.linear("up", x), gated=True)
        return qlin.block_norm(y, h, self.norms[3], post_norm=self.norms[2])

    def plain(self, h, x, cache, new, length):
        """The same in float64; the new tokens' keys and values are those that the cache holds."""
        def norm(x, w):
            return x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w.double()

        def linear(name, x):
            w, s = self.lin[name]
            return x @ (w.double() * s.double()[:, None]).t().contiguous()

        q = linear("qkv", x.double())[:, :HQ * HEAD].reshape(-1, HQ, HEAD)
        q = norm(q, self.qk[0]).cpu().numpy()
        parts, m = [], 0
        for b, (n, L) in enumerate(zip(new, length)):
            rows = [low.row_values(cache[2 * i][b, :, :L].cpu().numpy().view(np.uint32), *[cache[2 * i + 1][b, :, :L, j].cpu().double().numpy() for j in (0, 1)])
                    for i in (0, 1)]
            turned = np.stack([ref.rotate(q[m + i], L - n + i, self.freq.cpu().numpy(), False) for i in range(n)])
            parts.append(ref.causal_attention(turned, rows[0].transpose(1, 0, 2), rows[1].transpose(1, 0, 2), HEAD ** -0.5)[0])
            m += n
        o = torch.from_numpy(np.concatenate(parts)).cuda().reshape(-1, HQ * HEAD)
        h = h.double() + norm(linear("o", o), self.norms[0])
        a, b = linear("up", norm(h, self.norms[1])).chunk(2, 1)
        return h + norm(linear("down", a * torch.sigmoid(a) * b), self.norms[2])


def test_a_layer_of_prompts_blocks_and_single_tokens():
    layer = Layer(0)
    cache = qlin.new_kv4_cache(2, HKV, 260)
    for new, length in [([90, 41], [90, 41]), ([16, 16], [106, 57]), ([16, 16], [101, 60]), ([1, 1], [102, 61])]:
        h = rand(sum(length), (sum(new), WIDTH), 1.0).cuda()
        x, _ = qlin.block_norm(None, h, layer.norms[0])
        before = h.clone()
        out, got = layer.run(h, x, cache, i32(starts(new)), i32(length), max(new))
        torch.cuda.synchronize()
        want = layer.plain(before, x, cache, new, length)
        added = (want - before.double()).norm()
        assert (got.double() - want).norm() < 0.05 * added, float((got.double() - want).norm() / added)
        assert torch.equal(h, before)                       # a new residual stream, not the old one


def test_a_captured_layer_follows_its_lengths():
    layer = Layer(1)
    cache = qlin.new_kv4_cache(3, HKV, 130)
    for part in (1, 3):
        cache[part][..., 0] = 0.1
    h, at, length = rand(1, (3, WIDTH)).cuda(), i32([0, 1, 2, 3]), i32([70, 3, 100])

    def step():
        x, _ = qlin.block_norm(None, h, layer.norms[0])
        return layer.run(h, x, cache, at, length, 1)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, res = step()
    for i in range(4):
        h.copy_(rand(20 + i, (3, WIDTH)))
        length.copy_(i32([71 + i, 4 + i, 101 + i]))
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone(), res.clone()
        again = step()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    rng = random.Random(seed)
    Hkv, G = rng.choice((1, 2, 3)), rng.choice((1, 2, 3, 4, 7))
    n = rng.randint(1, 6)
    new = [rng.choice((0, 1, 1, 5, 16, 33, 70)) for _ in range(n)]
    if not any(new):
        new[0] = 1
    length = [max(0, x + rng.choice((-2, 0, 0, 1, 63, 64, 65, 130, 500))) for x in new]
    layout = rng.choice(("heads", "tokens", "packed"))
    check_append(new, length, layout, Hq=Hkv * G, Hkv=Hkv, rot=rng.choice((128, 64, 0)), interleaved=rng.random() < 0.4, norm=rng.random() < 0.7,
                 pad=rng.choice((0, 3)), seed=seed)
    check_attention(new, length, layout, Hq=Hkv * G, Hkv=Hkv, splits=rng.choice((0, 0, 1, 3)), pad=rng.choice((0, 3)), seed=seed,
                    spread=rng.choice((0.0, 1.0, 2.0)), cache=Cache(layout, length, Hkv, seed + 40, spread=1.0))
