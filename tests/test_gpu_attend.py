"""GPU tests of attention over the paged 4-bit cache against the 64-bit
reference of the values that the cache holds.

Tolerances are the reference's bound of a float32 computation, plus for bf16
outputs what weights in two bf16 parts leave out (2^-17 of each) and half a
step of the rounding (2^-8 of the value).  Where one key is seen the bits have
to be equal, and for f32 outputs where keys are equal: every number is exact.
"""

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


def _np(t):
    return t.detach().double().cpu().numpy()


class Batch:
    """Sequences in a cache that holds garbage wherever nothing was written."""

    def __init__(self, env, lengths, counts, HQ, HK, D, page=16, dtype="f32", seed=0, spare=2, tail=0, keys=None):
        fgd, torch = env
        self.fgd, self.dtype, self.D = fgd, dtype, D
        g = torch.Generator().manual_seed(seed)
        self.lens, self.counts = list(lengths), list(counts)
        B, self.T = len(self.lens), sum(counts)
        held = [-(-max(n, 0) // page) for n in self.lens]
        pages = sum(held) + 3
        self.cache = fgd.Mx4Cache(pages, page, HK, D)
        self.cache.data.copy_(torch.randint(0, 256, (self.cache.nbytes,), generator=g, dtype=torch.uint8))
        width = max(held, default=0) + spare
        order = torch.randperm(pages, generator=g, dtype=torch.int32)
        table = torch.full((B, width + tail), -7, dtype=torch.int32)
        table[:, ::2] = 2 ** 31 - 1  # entries that must not be read
        self.k, self.v, first = [], [], 0
        for b, n in enumerate(self.lens):
            own = order[first:first + held[b]]
            first += held[b]
            table[b, :held[b]] = own
            n = max(n, 0)
            k, v = ((torch.randn((n, HK, D), generator=g) * (1 + torch.arange(HK).view(1, HK, 1))).cuda() for _ in "kv")
            if keys is not None:
                keys(b, k, v)
            at = torch.arange(n)
            slots = own.long()[at // page] * page + at % page if n else at
            fgd.mx4_cache_write(self.cache, k, v, slots.cuda())
            self.k.append(ref.cached(_np(k)))
            self.v.append(ref.cached(_np(v)))
        self.tables = table.cuda()[:, :width]
        self.lengths = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.starts = torch.tensor(np.cumsum([0, *self.counts]), dtype=torch.int32).cuda()
        t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.q = (2 * torch.randn((self.T, HQ, D), generator=g)).to(t).cuda()

    def run(self, window=0, scale=None, starts=True, **kw):
        return self.fgd.mx4_attend(self.q, self.cache, self.tables, self.lengths, self.starts if starts else None,
                                   window=window, scale=scale, **kw)

    def check(self, window=0, scale=None, **kw):
        got = _np(self.run(window, scale, **kw))
        s = np.float64(np.float32(self.D ** -0.5 if scale is None else scale))
        first = 0
        for b, n in enumerate(self.counts):
            rows, first = slice(first, first + n), first + n
            q = _np(self.q[rows])
            want, tol = ref.attend(q, self.k[b], self.v[b], s, window)
            if self.dtype == "bf16":
                tol = tol + ref.weight_error(q, self.k[b], self.v[b], s, window)
                tol = tol + 2.0 ** -8 * (abs(want) + tol)
            else:
                tol = tol + 2.0 ** -23 * abs(want)
            assert got[rows].shape == want.shape and np.isfinite(got[rows]).all()
            assert np.all(abs(got[rows] - want) <= tol), (b, np.max(abs(got[rows] - want) / tol))
        return got


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 257]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
def test_one_query_each(env, D, dtype):
    Batch(env, LENGTHS, [1] * len(LENGTHS), 6, 2, D, dtype=dtype, seed=D).check(starts=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("HQ, HK, page", [(1, 1, 16), (8, 1, 32), (3, 3, 64), (16, 1, 16), (34, 2, 128), (8, 8, 16),
                                          (40, 1, 256)])
def test_head_layouts_and_pages(env, HQ, HK, page, dtype):
    b = Batch(env, [1, 40, 77, 300], [1] * 4, HQ, HK, 64, page, dtype, seed=HQ)
    b.check(starts=False)
    b.check(window=33)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [0, 1, 7, 16, 50, 10_000, 2 ** 31 - 1])
def test_several_queries(env, window, dtype):
    lengths = [5, 33, 64, 100, 7, 0, 3, 90]
    counts = [5, 3, 20, 41, 0, 2, 9, 1]  # more queries than keys: the first see nothing
    for D, HQ, HK in ((64, 4, 2), (96, 7, 1), (256, 2, 1)):
        got = Batch(env, lengths, counts, HQ, HK, D, 16, dtype, seed=window % 1000).check(window)
        assert (got[69:71] == 0).all() and (got[71:77] == 0).all() and (got[77:80] != 0).any(-1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128, 160, 192, 224, 256])
def test_rows_enough_to_fill_the_card(env, D, dtype):
    # 70 sequences x 16 heads: waves have rows of their own.
    rng = np.random.default_rng(D)
    lengths = rng.integers(0, 60, 70)
    counts = np.minimum(rng.integers(0, 4, 70), 3)
    b = Batch(env, lengths.tolist(), counts.tolist(), 16, 16, D, 16, dtype, seed=D)
    b.check(max_q=40)
    b.check(window=9, max_q=40)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_hint_changes_no_result_beyond_rounding(env, dtype):
    b = Batch(env, [200, 70, 300], [60, 1, 33], 8, 2, 64, 32, dtype, seed=4)
    for most in (0, 1, 2, 61, 5000, None):
        b.check(max_q=most)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_long_sequences_are_split(env, D, dtype):
    b = Batch(env, [4000, 1, 0, 2777], [1] * 4, 4, 2, D, 64, dtype, seed=3, spare=200)
    b.check(starts=False)
    b.check(starts=False, window=1500)
    Batch(env, [3000, 2500], [5, 2], 4, 1, D, 16, dtype, seed=3, spare=90).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_sequences_and_pages(env, dtype):
    # More sequences than a wave has lanes, and tables of more pages.
    rng = np.random.default_rng(7)
    b = Batch(env, rng.integers(0, 90, 150).tolist(), [1] * 150, 2, 1, 32, 16, dtype, seed=3)
    b.check(starts=False)
    b = Batch(env, rng.integers(0, 60, 140).tolist(), rng.integers(0, 3, 140).tolist(), 2, 1, 64, 16, dtype, seed=3)
    b.check()
    for most in (1, 50_000):
        Batch(env, [2500, 1040], [30, 17], 4, 2, 64, 16, dtype, seed=5).check(max_q=most)
        Batch(env, [1030] * 3, [9] * 3, 4, 2, 96, 16, dtype, seed=6).check(window=900, max_q=most)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("most", [1, 50_000])
@pytest.mark.parametrize("power", [-100, -118, -121, 100, 120])
def test_values_of_any_size(env, power, most, dtype):
    # One key is seen: its value comes out as it is held, down to 2^-126.
    def keys(_, k, v):
        v *= 2.0 ** power
    b = Batch(env, [20, 33], [2, 3], 2, 1, 64, 16, dtype, seed=power, keys=keys)
    got = _np(b.run(window=1, max_q=most))
    want = np.concatenate([np.repeat(b.v[0][18:], 2, 1), np.repeat(b.v[1][30:], 2, 1)])
    assert abs(want).max() > 0
    small = abs(want) < 2.0 ** -126  # numbers that a float32 sum may flush
    assert np.array_equal(np.where(small, 0, got), np.where(small, 0, want))
    assert np.all(abs(got[small] - want[small]) < 2.0 ** -126)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
def test_items_that_are_cut(env, D, dtype):
    # Long tables: items of 16 rows and of 32, cut between blocks.
    Batch(env, [700, 0, 1, 333], [1] * 4, 4, 2, D, 16, dtype, seed=D, spare=120).check()
    b = Batch(env, [150, 40, 7, 500], [6, 1, 9, 13], 6, 2, D, 32, dtype, seed=D, spare=120)
    for most in (13, 300):  # few items by the hint, and many
        b.check(max_q=most)
        b.check(window=60, max_q=most)


def test_large_scores_and_scales(env):
    def keys(b, k, v):
        k *= 30

    for scale in (1e-6, 0.3, 5.0):
        Batch(env, [50, 300], [3, 1], 4, 2, 64, seed=1, keys=keys).check(scale=scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shared", [True, False])
def test_exact_where_one_key_is_seen(env, shared, dtype):
    fgd, torch = env
    n = 3 if shared else 70
    b = Batch(env, [40] * n, [5] * n, 16, 16, 96, 16, dtype, seed=9)
    got = _np(b.run(window=1, max_q=5 if shared else 40))
    for i in range(n):
        assert np.array_equal(got[5 * i:5 * i + 5], b.v[i][35:])

    # All keys equal: the mean of values that are whole numbers.
    def keys(_, k, v):
        k[:] = k[:1]
        v[:] = torch.randint(-2, 3, v.shape).float().cuda() * 2
    b = Batch(env, [64] * n, [1] * n, 16, 16, 96, 16, dtype, seed=9, keys=keys)
    got = _np(b.run(max_q=1 if shared else 40))
    for i in range(n):
        want, size = b.v[i].mean(0), abs(b.v[i]).mean(0)
        if dtype == "f32":  # every weight is 1
            assert np.array_equal(got[i], _round(torch, want, dtype))
            continue
        # bf16: every weight is one number near 1, held in two parts to 2^-17 of itself. The sum of 2 x 64 exact terms is
        # off by 2^-23 of the terms' at each addition, 2^-16 of it in all; and then the result's half step.
        tol = 2.0 ** -16 * (size + abs(want))
        assert np.all(abs(got[i] - want) <= tol + 2.0 ** -8 * (abs(want) + tol))


def _round(torch, a, dtype):
    t = torch.from_numpy(a).float()
    return (t.bfloat16() if dtype == "bf16" else t).double().numpy()


def test_float32_queries_keep_all_their_bits(env):
    # One product per score: q's last bits decide between two keys' weights.
    fgd, torch = env
    def keys(_, k, v):
        k.zero_()
        v.zero_()
        k[0, :, 0] = 4.0
        v[0] = 1.0
    b = Batch(env, [2], [1], 1, 1, 32, keys=keys)
    for x in (1.0 + 2.0 ** -23, -1.2345678, 0.3333333):
        b.q.zero_()
        b.q[..., 0] = x
        got = _np(b.run(scale=1.0))[0, 0, 0]
        x = float(np.float32(x))
        want = 1 / (1 + np.exp(-4 * x))
        assert abs(got - want) < 2.0 ** -22  # a dozen float32 operations on numbers of 1 at most, and 4 x 2^-24
        # the part of x below its first 16 bits alone moves the result further
    b.check(scale=1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("shared", [True, False])
def test_what_is_hidden_never_shows(env, shared, bad, dtype):
    fgd, torch = env
    def keys(b, k, v):
        if b == 0:
            k[90, 0, 3] = v[90, 0, 40] = bad  # seen by the last 10 queries, and by none with a window of 1 but one
            v[4, 1, 70] = bad
    n = 2 if shared else 70
    batch = Batch(env, [100] * n, [30] * n, 16, 16, 96, 32, dtype, seed=2, keys=keys)
    most = 30 if shared else 64  # of a wave's own rows
    got = _np(batch.run(max_q=most)).reshape(n, 30, 16, 96)
    assert np.isfinite(got[1:]).all()
    assert np.isfinite(got[0, :20, 0]).all() and np.isnan(got[0, 20:, 0]).all()
    assert np.isnan(got[0, :, 1, 64:]).all() and np.isfinite(got[0, :, 1, :64]).all()
    assert np.isfinite(got[0, :, 2:]).all()
    got = _np(batch.run(window=20, max_q=most)).reshape(n, 30, 16, 96)
    assert np.isfinite(got[0, :, 1]).all() and np.isnan(got[0, 20:, 0]).all() and np.isfinite(got[0, :20]).all()
    # A value alone: only its block, in queries that see it.
    def keys(b, k, v):
        if b == 0:
            v[90, 0, 40] = bad
    batch = Batch(env, [100] * n, [30] * n, 16, 16, 96, 32, dtype, seed=2, keys=keys)
    got = _np(batch.run(max_q=most, window=5)).reshape(n, 30, 16, 96)
    seen = np.zeros((n, 30, 16, 96), bool)
    seen[0, 20:25, 0, 32:64] = True
    assert np.array_equal(np.isnan(got), seen)


def test_queries_of_nan_and_infinity(env):
    fgd, torch = env
    b = Batch(env, [50] * 4, [1] * 4, 4, 4, 64, seed=5)
    b.q[1, 2, 7] = float("nan")
    b.q[2, 1, 9] = float("inf")
    got = _np(b.run(starts=False))
    bad = np.zeros((4, 4), bool)
    bad[1, 2] = bad[2, 1] = True
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    b.q[2, 1, 9] = 3e38  # finite: the scores are infinite or not, the rows beside it are not touched
    assert np.isfinite(_np(b.run(starts=False))[~bad]).all()


@pytest.mark.parametrize("bad", [0, 1, 62, 63, 64, 65, 127, 128])
def test_a_bad_page_of_many_rows(env, bad):
    # Every page that rows see, wherever a program's 64 of them begin: by waves of their own, and in items.
    fgd, torch = env
    b = Batch(env, [129 * 16 - 3] * 2, [160, 160], 256, 16, 32, 16, "bf16", seed=bad)
    for most in (None, 1):
        assert np.isfinite(_np(b.run(max_q=most))).all()
    b.tables[1, bad] = b.cache.pages
    for most in (None, 1):
        got = _np(b.run(max_q=most))
        assert np.isfinite(got[:160]).all()
        seen = [i for i in range(160, 320) if b.lens[1] - 160 + (i - 160) >= 16 * bad]
        assert seen and np.isnan(got[seen]).any(-1).all()


@pytest.mark.parametrize("shared", [True, False])
def test_bad_pages_and_lengths(env, shared):
    fgd, torch = env
    n = 4 if shared else 70
    b = Batch(env, [50] * n, [1] * n, 16, 16, 64, 16, seed=6, spare=1)
    most = 1 if shared else 40
    want = _np(b.run(max_q=most))
    b.tables[1, 2] = -1
    b.tables[2, 0] = b.cache.pages
    b.lengths[3] = 5 * 16 + 1  # past its table
    got = _np(b.run(max_q=most))
    assert np.isnan(got[1:4]).all()
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[4:], want[4:])
    assert np.isfinite(_np(b.run(max_q=most, window=2))[1:3]).all()  # the bad page is not among those it needs
    b.lengths[3] = -3
    assert (_np(b.run(max_q=most))[3] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("many", [False, True])
def test_rows_of_no_sequence_stay(env, many, dtype):
    fgd, torch = env
    n = 70 if many else 3
    for spare in (1, 300):
        b = Batch(env, [200, 20, 0][:3] + [5] * (n - 3), [3, 2, 1] + [1] * (n - 3), 16, 16, 64, 16, dtype, spare=spare)
        want = b.run()
        q = torch.cat((b.q, torch.full((5, 16, 64), float("nan"), dtype=b.q.dtype, device="cuda")))
        out = torch.full(q.shape, 3.0, dtype=q.dtype, device="cuda")
        fgd.mx4_attend(q, b.cache, b.tables, b.lengths, b.starts, out=out, max_q=40 if many else 3)
        assert torch.equal(out[b.T:], torch.full_like(out[b.T:], 3.0))
        tol = 2.0 ** -7 if dtype == "bf16" else 1e-4
        assert (out[:b.T].float() - want.float()).abs().max() <= tol * want.abs().max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(env, dtype):
    fgd, torch = env
    b = Batch(env, [90, 33, 4], [2, 1, 3], 6, 2, 96, 16, dtype, tail=5)
    want = b.check()
    wide = torch.zeros((b.T, 6 * 96 + 1), dtype=b.q.dtype, device="cuda")
    wide[:, 1:] = b.q.flatten(1)
    out = torch.full((6, b.T + 2, 101), 5.0, dtype=b.q.dtype, device="cuda")
    view = out[:, 1:-1, 3:99].transpose(0, 1)
    fgd.mx4_attend(wide[:, 1:].unflatten(1, (6, 96)), b.cache, b.tables, b.lengths, b.starts, out=view)
    assert np.array_equal(_np(view), want)
    out[:, 1:-1, 3:99] = 5.0
    assert (out == 5.0).all()


def test_empty(env):
    fgd, torch = env
    cache = fgd.Mx4Cache(2, 16, 2, 64)
    none = torch.empty((0, 4, 64), device="cuda")
    tables = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    assert fgd.mx4_attend(none, cache, tables, ints()).shape == (0, 4, 64)
    assert fgd.mx4_attend(none, cache, tables, ints(), ints(0)).shape == (0, 4, 64)
    q = torch.ones((2, 4, 64), device="cuda")
    width0 = torch.zeros((2, 0), dtype=torch.int32, device="cuda")
    assert (fgd.mx4_attend(q, cache, width0, ints(0, 0)) == 0).all()
    assert torch.isnan(fgd.mx4_attend(q, cache, width0, ints(1, 5))).all()
    no_pages = fgd.Mx4Cache(0, 16, 2, 64)
    assert (fgd.mx4_attend(q, no_pages, width0, ints(0, 0)) == 0).all()


def test_equal_calls_streams_and_graphs(env):
    fgd, torch = env
    b = Batch(env, [3000, 40, 900], [1] * 3, 8, 2, 128, 64, "bf16", seed=8, spare=50)
    c = Batch(env, [500, 700], [40, 9], 8, 2, 128, 16, "bf16", seed=9)
    want = b.run(starts=False), c.run()
    assert torch.equal(b.run(starts=False), want[0]) and torch.equal(c.run(), want[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = b.run(starts=False, stream=s), c.run(stream=s)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    # Two calls at once, on streams and workspaces of their own.
    t = torch.cuda.Stream()
    for _ in range(5):
        for x in (s, t):
            x.wait_stream(torch.cuda.current_stream())
        got = [(b.run(starts=False, stream=x), c.run(stream=x)) for x in (s, t, s, t)]
        torch.cuda.synchronize()
        assert all(torch.equal(w, g) for pair in got for w, g in zip(want, pair))
    # Two graphs that share a workspace, replayed one after the other.
    need = max(fgd.fgd_mx4_attend_workspace_size(x.cache._c, fgd.fgd_attention(
        "bf16", x.tables.shape[0], x.tables.shape[1], 8, 0, x.T, 64, 1.0)) for x in (b, c))
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    graphs = []
    for x, kw in ((b, dict(starts=False)), (c, dict(max_q=40))):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = x.run(**kw, workspace=work)
        graphs.append((g, out, x, kw))
    for i in range(4):
        for g, out, x, kw in graphs:
            x.q.copy_(torch.randn(x.q.shape, device="cuda"))
            x.lengths.sub_(i)
            g.replay()
        torch.cuda.synchronize()
        for g, out, x, kw in graphs:
            assert torch.equal(out, x.run(**kw))


def _route(route):
    """(sequences, query heads, key heads, queries each, hint, spare pages) of a call that goes this way."""
    return {"items": (3, 4, 2, 5, 5, 2), "cut items": (3, 4, 2, 5, 5, 120), "items of 32": (40, 16, 4, 8, 8, 2),
            "cut items of 32": (40, 16, 4, 8, 8, 120), "own rows": (70, 16, 16, 5, 40, 2)}[route]


ROUTES = ["items", "cut items", "items of 32", "cut items of 32", "own rows"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.125, 0.69, 0.7, 4.0, 1e30])
@pytest.mark.parametrize("sign", ["both", "negative"])
@pytest.mark.parametrize("route", ROUTES)
def test_scores_far_from_zero(env, route, sign, scale, dtype):
    # Exact scores q.k of 2^10 to 2^127.2 with 2^9 between any two: finite, while scale log2(e) times them may not be.
    # The largest that a query sees has the weight 1, the others together at most 2^-92 of it, times values of 2^7 at most
    # and 100 keys less than 2^-78.  A float32 sum is off by 2^-23 of itself at each of its 3 x 100 additions at most, which
    # a bf16 output does not show.
    fgd, torch = env
    n, HQ, HK, count, most, spare = _route(route)
    rng = np.random.default_rng(ROUTES.index(route))

    def keys(b, k, v):
        k.zero_()
        for h in range(HK):
            i = rng.permutation(106)[:len(k)]
            size = 2.0 ** (10 + i % 53) * np.where(i < 53, 1.0, 1.5)
            size *= rng.choice([-1, 1], len(k)) if sign == "both" else 1
            k[:, h, 0] = torch.from_numpy(size).float().cuda()

    b = Batch(env, [100 - b % 60 for b in range(n)], [count] * n, HQ, HK, 64, 16, dtype, seed=3, spare=spare, keys=keys)
    b.q.zero_()
    by = rng.choice([1.0, 1.5], (b.T, HQ)) * 2.0 ** rng.choice([0, 3, 64], (b.T, HQ)) * (-1 if sign == "negative" else 1)
    b.q[..., 0] = torch.from_numpy(by).to(b.q.dtype).cuda()
    for window in (0, 37):
        got = _np(b.run(window, scale, max_q=most)).reshape(n, count, HQ, 64)
        for i in range(n):
            s = np.einsum("thd,khd->thk", _np(b.q[count * i:count * i + count]), np.repeat(b.k[i], HQ // HK, 1))
            at = b.lens[i] - count + np.arange(count)[:, None, None]
            key = np.arange(b.lens[i])
            s = np.where((key <= at) & (key > at - (window or 1000)), s, -np.inf)
            want = np.stack([b.v[i][s[:, h].argmax(-1), h // (HQ // HK)] for h in range(HQ)], 1)
            assert abs(b.v[i]).max() <= 128
            assert np.all(abs(got[i] - want) <= 300 * 2.0 ** -23 * abs(want) + 2.0 ** -78)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("route", ROUTES)
def test_scales_above_one(env, route, dtype):
    def keys(b, k, v):
        k *= 5

    n, HQ, HK, count, most, spare = _route(route)
    b = Batch(env, [100 - b % 60 for b in range(n)], [count] * n, HQ, HK, 64, 16, dtype, seed=4, spare=spare, keys=keys)
    for scale in (0.69, 0.7, 5.0):
        b.check(scale=scale, max_q=most)
    b.check(33, 1.5, max_q=most)


def test_large_scores_and_scales_bf16(env):
    def keys(b, k, v):
        k *= 30

    for scale in (1e-6, 0.3, 5.0):
        Batch(env, [50, 300], [3, 1], 4, 2, 64, dtype="bf16", seed=1, keys=keys).check(scale=scale)


@pytest.mark.parametrize("scale", [0.125, 3.0])
@pytest.mark.parametrize("route", ROUTES)
def test_bf16_queries_of_nan_and_infinity(env, route, scale):
    fgd, torch = env
    n, HQ, HK, count, most, spare = _route(route)
    b = Batch(env, [50] * n, [count] * n, HQ, HK, 64, 16, "bf16", seed=5, spare=spare)
    b.q[1, 2, 7] = float("nan")
    b.q[2, 1, 9] = float("inf")
    got = _np(b.run(scale=scale, max_q=most))
    bad = np.zeros((b.T, HQ), bool)
    bad[1, 2] = bad[2, 1] = True
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    b.q[2, 1, 9] = 3e38  # finite: its scores may pass every number, the rows beside it are not touched
    assert np.isfinite(_np(b.run(scale=scale, max_q=most))[~bad]).all()


@pytest.mark.parametrize("D, dtype", [(32, "f32"), (64, "f32"), (96, "f32"), (32, "bf16"), (64, "bf16"), (96, "bf16"),
                                      (128, "bf16")])
@pytest.mark.parametrize("cut", [False, True])
def test_items_of_32_rows(env, D, dtype, cut):
    # 8 queries of 4 heads a key head: items for 40 sequences of 4 key heads, some without a row or with one tile of
    # two, some sequences of two items; whole, and cut between blocks where the tables are long.
    fgd, torch = env
    rng = np.random.default_rng(D + cut)
    lengths = rng.integers(0, 500 if cut else 300, 40)
    counts = rng.integers(0, 9, 40)
    lengths[:6], counts[:6] = [1, 0, 33, 297, 64, 150], [8, 3, 1, 8, 4, 12]
    b = Batch(env, lengths.tolist(), counts.tolist(), 16, 4, D, 16, dtype, seed=D, spare=120 if cut else 2)
    b.check(max_q=8)
    b.check(window=41, max_q=8)

    def need(most):
        return fgd.fgd_mx4_attend_workspace_size(b.cache._c, fgd.fgd_attention(
            dtype, 40, b.tables.shape[1], 16, 0, b.T, most, 1.0))
    # Whole items leave no parts; of cut ones 32 rows have their place, or 16 of them by a hint of one query. Where two
    # blocks are launched for each one of twice the rows, both need as much.
    if not cut:
        assert need(8) == need(1) == 0
    elif (D, dtype) in ((64, "f32"), (96, "bf16")):
        assert need(8) == need(1) > 0
    else:
        assert need(8) > need(1) > 0


@pytest.mark.parametrize("D, dtype", [(32, "bf16"), (128, "bf16"), (96, "f32")])
def test_items_of_32_rows_of_long_sequences(env, D, dtype):
    # Items of many blocks each, of one block, and blocks of several items.
    lengths = [3000, 1, 2047, 20, 700, 2500] + [60] * 26
    counts = [8, 1, 7, 8, 2, 5] + [6] * 26
    b = Batch(env, lengths, counts, 16, 4, D, 16, dtype, seed=D)
    b.check(max_q=8)
    b.check(window=1100, max_q=8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 256])
def test_own_rows_of_long_sequences(env, D, dtype):
    # Rows of their own in all four waves and both of their tiles, blocks of a sequence one after the other, 4 heads a
    # key head; steps enough for every buffer to be used again, and pages past the first 64.
    lengths = [1500, 260, 64, 1, 0, 700] + [30] * 58
    counts = [200, 130, 33, 1, 4, 17] + [2] * 58
    b = Batch(env, lengths, counts, 16, 4, D, 16, dtype, seed=D)
    b.check(max_q=200)
    b.check(window=300, max_q=200)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("HQ, HK", [(7, 1), (6, 2)])
def test_own_rows_of_many_sequences(env, HQ, HK, dtype):
    # Over 64 sequences, which keep their order; groups that do not divide a tile.
    rng = np.random.default_rng(HQ)
    lengths = rng.integers(100, 250, 100)
    counts = rng.integers(0, 40, 100)
    counts[::9] = 100
    b = Batch(env, lengths.tolist(), counts.tolist(), HQ, HK, 64, 32, dtype, seed=HQ)
    for window in (0, 50):
        b.check(window, max_q=400)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power", [-122, -123, -124, -125, -126])
@pytest.mark.parametrize("route", ROUTES)
def test_values_of_the_smallest_scales(env, route, power, dtype):
    # Blocks of scale byte 0 (largest magnitude below 2^-124): one key is seen, its value comes out as it is held.
    n, HQ, HK, count, most, spare = _route(route)

    def keys(_, k, v):
        v *= 2.0 ** power
    b = Batch(env, [40] * n, [count] * n, HQ, HK, 96, 16, dtype, seed=-power, keys=keys, spare=spare)
    got = _np(b.run(window=1, max_q=most))
    want = np.concatenate([np.repeat(v[40 - count:], HQ // HK, 1) for v in b.v])
    small = abs(want) < 2.0 ** -126  # numbers that a float32 sum may flush
    assert (~small).any() and (abs(want) < 2.0 ** -124).any()
    assert np.array_equal(np.where(small, 0, got), np.where(small, 0, want))
    assert np.all(abs(got[small] - want[small]) < 2.0 ** -126)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("route", ROUTES)
def test_keys_of_the_smallest_scales(env, route, dtype):
    # Keys of 2^-126 to 2^-124 in blocks of scale byte 0 and queries of 2^123: scores of ordinary size.
    fgd, torch = env
    n, HQ, HK, count, most, spare = _route(route)

    def keys(_, k, v):
        k[:] = torch.where(k < 0, -1.0, 1.0) * (2.0 ** -126 * (1 + (abs(k) > 1).float() + (abs(k) > 2).float()))
    b = Batch(env, [40] * n, [count] * n, HQ, HK, 96, 16, dtype, seed=8, keys=keys, spare=spare)
    for k in b.k:
        assert abs(k).min() == 2.0 ** -126 and abs(k).max() == 3 * 2.0 ** -126
    b.q.mul_(2.0 ** 123)
    b.check(scale=0.3, max_q=most)
