"""GPU test of the operators as a program runs them together: prompts and
decoding turns of several requests through one attention layer over a paged
4-bit cache, with a 4-bit projection and a 4-bit head, and a token sampled each
turn; against the reference of the same steps, and captured into a graph."""

import numpy as np
import pytest

from oracle import attention as ref

pytestmark = pytest.mark.gpu

HQ, HK, D, WIDTH, VOCAB, PAGE = 4, 2, 64, 96, 333, 16


@pytest.fixture(scope="module")
def env():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2606_22768_amd as fgd

    return fgd, torch


class Layer:
    def __init__(self, env, B, pages=40, width=9):
        self.fgd, torch = env
        self.torch = torch
        g = torch.Generator().manual_seed(1)
        gpu = lambda *s: torch.randn(s, generator=g).cuda()  # noqa: E731
        self.embed = gpu(VOCAB, WIDTH)
        self.project = self.fgd.mx4_quantize(gpu((HQ + 2 * HK) * D, WIDTH) * 0.1)
        self.back = self.fgd.mx4_quantize(gpu(VOCAB, HQ * D) * 0.1)
        self.wq, self.wk = 1 + 0.1 * gpu(D), 1 + 0.1 * gpu(D)
        self.freqs = (10.0 ** -torch.arange(D // 2, dtype=torch.float64)).cuda()
        ints = lambda a: torch.as_tensor(a, dtype=torch.int32).cuda()  # noqa: E731
        self.tables, self.lengths = ints(np.full((B, width), -1)), ints([0] * B)
        self.free, self.count = ints(np.random.default_rng(0).permutation(pages)), ints([pages])
        self.cache = self.fgd.Mx4Cache(pages, PAGE, HK, D)
        self.seen = []

    def turn(self, tokens, counts, stream=None):
        """Logits of every token, rows behind the last undefined."""
        fgd = self.fgd
        T = tokens.shape[0]
        starts, positions, slots = fgd.extend_pages(self.tables, self.lengths, counts, self.free, self.count, PAGE, T)
        x = self.embed[tokens]
        qkv = fgd.mx4_linear(x, self.project).unflatten(1, (HQ + 2 * HK, D))
        q, k = fgd.rotate_heads(qkv[:, :HQ], qkv[:, HQ:HQ + HK], positions, self.freqs, self.wq, self.wk)
        fgd.mx4_cache_write(self.cache, k, qkv[:, HQ + HK:], slots)
        o = fgd.mx4_attend(q, self.cache, self.tables, self.lengths, starts, max_q=T)
        return starts, fgd.mx4_linear(o.flatten(1), self.back), qkv, o


def test_turns_against_the_reference(env):
    fgd, torch = env
    B = 5
    layer = Layer(env, B)
    g = torch.Generator().manual_seed(2)
    history = [[] for _ in range(B)]  # each request's projected heads
    for counts in ([7, 1, 0, 33, 16], [1] * 5, [1, 0, 5, 1, 1], [1] * 5):
        total = sum(counts)
        tokens = torch.randint(0, VOCAB, (total + 2,), generator=g).cuda()
        starts, logits, qkv, o = layer.turn(tokens, torch.tensor(counts, dtype=torch.int32).cuda())
        assert starts.tolist() == np.cumsum([0, *counts]).tolist()
        qkv, o = qkv.double().cpu().numpy(), o.double().cpu().numpy()
        for b in range(B):
            history[b] += [qkv[t] for t in range(*starts[b:b + 2].tolist())]
            n, L = counts[b], len(history[b])
            if n == 0:
                continue
            x = np.stack(history[b])
            at = np.arange(L)
            f = layer.freqs.cpu().numpy()
            q, _ = ref.rotate_heads(x[L - n:, :HQ], layer.wq.cpu().numpy(), at[L - n:], f, np.float64(np.float32(1e-6)),
                                    False)
            k, _ = ref.rotate_heads(x[:, HQ:HQ + HK], layer.wk.cpu().numpy(), at, f, np.float64(np.float32(1e-6)), False)
            # The cache holds what float32 keys round to; a key near the middle
            # of two codes may take either, which the last step's test leaves
            # out by taking the cache's own values.
            held = fgd.mx4_cache_read(layer.cache, _slots(torch, layer, b, L))
            kk, vv = (t.double().cpu().numpy() for t in held)
            close = abs(kk - ref.cached(k)) > 0
            assert close.mean() < 1e-3 and np.array_equal(vv, ref.cached(x[:, HQ + HK:]))
            want, tol = ref.attend(q, kk, vv, np.float64(np.float32(D ** -0.5)))
            # q itself is off by 20 2^-24 of terms of at most sqrt(D) 2: the scores by that times |k|.
            slack = 2 * 20 * 2.0 ** -24 * 2 * np.sqrt(D) * abs(kk).sum(-1).max() * D ** -0.5 * abs(vv).max()
            rows = slice(*starts[b:b + 2].tolist())
            assert np.all(abs(o[rows] - want) <= tol + slack + 2.0 ** -23 * abs(want))
        assert torch.isfinite(logits[:total]).all()
        u = torch.rand(total, generator=g).cuda()
        token, p = fgd.sample(logits[:total], u, temperature=0.8, top_k=20)
        assert (token >= 0).all() and (p > 0).all()
    fgd.truncate_pages(layer.tables, layer.lengths, torch.zeros(B, dtype=torch.int32).cuda(), layer.free, layer.count, PAGE)
    assert layer.count.item() == 40 and sorted(layer.free.tolist()) == list(range(40))


def _slots(torch, layer, b, L):
    at = torch.arange(L, device="cuda")
    return layer.tables[b].long()[at // PAGE] * PAGE + at % PAGE


def test_captured_turns_equal_eager_ones(env):
    fgd, torch = env
    B = 6
    a, b = Layer(env, B, 60, 8), Layer(env, B, 60, 8)
    prompt = torch.randint(0, VOCAB, (60,), generator=torch.Generator().manual_seed(3)).cuda()
    counts = torch.tensor([10, 20, 1, 9, 15, 5], dtype=torch.int32).cuda()
    for layer in (a, b):
        layer.turn(prompt, counts)
    tokens = torch.zeros(B, dtype=torch.int64, device="cuda")
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    state = [t.clone() for t in (a.tables, a.lengths, a.free, a.count, a.cache.data)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = a.turn(tokens, one)
    for t, s in zip((a.tables, a.lengths, a.free, a.count, a.cache.data), state):
        t.copy_(s)
    for i in range(20):  # through a page's end
        tokens.copy_(torch.arange(B) * 7 + i)
        graph.replay()
        torch.cuda.synchronize()
        want = b.turn(tokens, one)
        for x, y in zip(out, want):
            assert torch.equal(x, y)
        assert torch.equal(a.tables, b.tables) and torch.equal(a.lengths, b.lengths)
