"""GPU tests of the pages' tables against the rule request by request: whole
numbers, all equal."""

import numpy as np
import pytest

from oracle import attention as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2606_22768_amd as fgd

    return fgd, torch


class Pool:
    """The state on the GPU and the reference's beside it."""

    def __init__(self, env, B, W, page, N, seed, stride=0):
        self.fgd, self.torch = env
        self.rng = np.random.default_rng(seed)
        self.page, self.W, self.N = page, W, N
        wide = self._gpu(np.full((B, W + stride), 99))
        self.tables = wide[:, :W]
        self.tables.fill_(-1)
        self.wide = wide
        self.lengths, self.free = self._gpu(np.zeros(B)), self._gpu(self.rng.permutation(N))
        self.count = self._gpu([N])
        self.state = [[-1] * W for _ in range(B)], [0] * B, self.free.tolist()

    def _gpu(self, a):
        return self.torch.from_numpy(np.asarray(a, np.int32)).cuda()

    def extend(self, counts, tokens):
        made = self.fgd.extend_pages(self.tables, self.lengths, self._gpu(counts), self.free, self.count, self.page,
                                     tokens)
        want = ref.extend_pages(*self.state[:2], list(counts), self.state[2], self.page, tokens)
        self.state = want[:3]
        for got, w in zip(made, want[3:]):
            assert got.tolist() == w
        self.check()
        return made

    def truncate(self, keep):
        self.fgd.truncate_pages(self.tables, self.lengths, self._gpu(keep), self.free, self.count, self.page)
        self.state = ref.truncate_pages(*self.state[:2], list(keep), self.state[2], self.page)
        self.check()

    def check(self):
        assert self.tables.tolist() == self.state[0]
        assert self.lengths.tolist() == self.state[1]
        n = self.count.item()
        assert n == len(self.state[2]) and self.free[:n].tolist() == self.state[2]
        assert (self.wide[:, self.W:] == 99).all()


@pytest.mark.parametrize("B, W, page, N, tokens", [(1, 1, 1, 1, 1), (1, 40, 16, 40, 640), (3, 5, 16, 10, 100),
                                                   (64, 9, 64, 300, 5000), (65, 7, 3, 200, 500), (257, 4, 16, 700, 4097),
                                                   (1025, 3, 32, 2000, 20_000), (2500, 2, 16, 3000, 9000)])
def test_turns(env, B, W, page, N, tokens):
    p = Pool(env, B, W, page, N, B, stride=B % 3)
    for turn in range(6):
        most = [page, 2 * page, W * page][turn % 3]
        p.extend(p.rng.integers(-1, most + 2, B), tokens)
        if turn % 2:
            p.truncate(p.rng.integers(-2, W * page, B) * (p.rng.random(B) < 0.7))
    before = [t.clone() for t in (p.tables, p.lengths, p.free, p.count)]
    lengths = p.lengths.tolist()
    p.extend(p.rng.integers(0, page + 1, B), tokens)
    p.truncate(lengths)  # all given back: the stack is as it was
    for a, b in zip(before, (p.tables, p.lengths, p.free, p.count)):
        assert p.torch.equal(a, b)


def test_one_long_prompt(env):
    p = Pool(env, 2, 9000, 16, 9000, 1)
    p.extend([131_077, 7], 140_000)
    p.extend([1, 1], 2)
    p.truncate([0, 0])


def test_what_does_not_fit(env):
    p = Pool(env, 4, 4, 16, 6, 2)
    p.extend([0, 0, 0, 0], 10)
    p.extend([65, 64, 17, 16], 1000)  # too long for its table; four pages; two; none left for the last
    assert p.lengths.tolist() == [0, 64, 17, 0]
    p.extend([0, 0, 15, 3], 1000)  # no page is needed; none is free
    assert p.lengths.tolist() == [0, 64, 32, 0]
    p.truncate([99, 0, 99, 99])
    p.extend([5, 5, 0, 5], 10)  # the third request of five tokens is past the turn's ten
    assert p.lengths.tolist() == [5, 5, 32, 0]
    p.extend([1, 1, 1, 1], 0)
    assert p.lengths.tolist() == [5, 5, 32, 0]


def test_odd_state(env):
    fgd, torch = env
    gpu = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    # A stack that claims more than it holds, a page that was never given, lengths below 0.
    tables, lengths = gpu([[-1, -1], [-1, -1]]), gpu([-5, 3])
    free, count = gpu([4, 5]), gpu([7])
    starts, positions, slots = fgd.extend_pages(tables, lengths, gpu([1, 1]), free, count, 16, 3)
    assert starts.tolist() == [0, 1, 2] and positions.tolist() == [0, 3, 0] and slots.tolist() == [5 * 16, -1, -1]
    assert lengths.tolist() == [1, 4] and count.tolist() == [1]
    # Pages that would pass the stack's capacity are dropped.
    tables, lengths, free, count = gpu([[1, 2, 3]]), gpu([48]), gpu([9, 9]), gpu([1])
    fgd.truncate_pages(tables, lengths, gpu([0]), free, count, 16)
    assert count.tolist() == [2] and free.tolist() == [9, 3] and tables.tolist() == [[-1, -1, -1]]
    # Lengths past the table, a whole-range count.
    tables, lengths, free, count = gpu([[1, 2]]), gpu([2 ** 31 - 1]), gpu([0] * 4), gpu([0])
    starts = fgd.extend_pages(tables, lengths, gpu([2 ** 31 - 1]), free, count, 16, 5)[0]
    assert starts.tolist() == [0, 0] and lengths.tolist() == [2 ** 31 - 1]
    fgd.truncate_pages(tables, lengths, gpu([16]), free, count, 16)
    assert lengths.tolist() == [16] and tables.tolist() == [[1, -1]] and free.tolist() == [2, 0, 0, 0]


def test_empty(env):
    fgd, torch = env
    gpu = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    none = torch.empty((0, 3), dtype=torch.int32, device="cuda")
    for tokens in (0, 5, 5000):
        starts, positions, slots = fgd.extend_pages(none, gpu([]), gpu([]), gpu([1]), gpu([1]), 16, tokens)
        assert starts.tolist() == [0] and (positions == 0).all() and (slots == -1).all() and len(slots) == tokens
    fgd.truncate_pages(none, gpu([]), gpu([]), gpu([1]), gpu([1]), 16)
    width0 = torch.empty((2, 0), dtype=torch.int32, device="cuda")
    starts, _, slots = fgd.extend_pages(width0, gpu([0, 0]), gpu([3, 0]), gpu([]), gpu([0]), 16, 4)
    assert starts.tolist() == [0, 0, 0] and slots.tolist() == [-1] * 4


def test_captured_turns(env):
    fgd, torch = env
    p, r = Pool(env, 33, 8, 16, 150, 5), Pool(env, 33, 8, 16, 150, 5)
    counts, keep = p._gpu(np.ones(33)), p._gpu(np.full(33, 1000))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = fgd.extend_pages(p.tables, p.lengths, counts, p.free, p.count, 16, 5000)
        fgd.truncate_pages(p.tables, p.lengths, keep, p.free, p.count, 16)
    for i in range(6):
        c, k = p.rng.integers(0, 40, 33), p.rng.integers(0, 128, 33)
        counts.copy_(p._gpu(c))
        keep.copy_(p._gpu(k))
        graph.replay()
        torch.cuda.synchronize()
        want = r.extend(c, 5000)
        r.truncate(k)
        for a, b in zip((*made, p.tables, p.lengths, p.count), (*want, r.tables, r.lengths, r.count)):
            assert torch.equal(a, b)
        n = r.count.item()
        assert torch.equal(p.free[:n], r.free[:n])
