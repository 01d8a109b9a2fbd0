"""GPU tests of sampling against a 64-bit reference of the whole-number
definition.

With T chosen so that the scaled logits are the logits' own whole-number
differences, every weight is a power of two, the masses are exact on both
sides, and the token must be equal.  With ordinary logits the two sides'
powers of two differ by up to 1.5 float32 ulps (3 2^-24 relative) and a mass by
one unit from its rounding, so a sum of n masses differs by at most
3 2^-24 of it plus n units; the drawn token must be one whose span of the
reference's mass, widened by four such errors, holds the reference's target,
and its probability must agree within the same error.
"""

import numpy as np
import pytest

from oracle import operators as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2606_22768_amd as fgd

    return fgd, torch


def _unit_temperature():
    """A float32 T with (1 / T) log2(e) = 1 exactly."""
    t = np.float32(np.log2(np.e))
    for _ in range(8):
        for s in (-np.inf, np.inf):
            v = t
            for _ in range(4):
                if (np.float32(1) / v) * np.float32(np.log2(np.e)) == np.float32(1):
                    return float(v)
                v = np.nextafter(v, np.float32(s))
    raise AssertionError("no such temperature")


UNIT_T = _unit_temperature()


def _cuda(torch, a, dtype="f32"):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _rows(torch, v, dtype=np.float32):
    return torch.from_numpy(np.asarray(v, dtype)).cuda()


def _run(env, z, u, dtype="f32", **kw):
    fgd, torch = env
    t, p = fgd.sample(_cuda(torch, z, dtype), _rows(torch, u), **kw)
    return t.cpu().numpy(), p.cpu().numpy()


SIZES = [1, 2, 3, 63, 64, 65, 255, 1000, 1025, 4099, 8192, 32000, 50257, 128256, 152064]
SETTINGS = [dict(), dict(top_k=1), dict(top_k=7), dict(top_k=300), dict(top_k=5000), dict(top_p=0.5),
            dict(top_p=0.95), dict(top_p=1e-9), dict(min_p=0.25), dict(min_p=2.0 ** -20), dict(min_p=3.0),
            dict(top_k=40, top_p=0.8), dict(top_k=1000, top_p=0.99, min_p=0.01), dict(top_p=0.0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_exact_weights_give_equal_tokens(env, V, dtype):
    """Whole-number logits (many ties), several rows and settings at once,
    some tokens masked."""
    rng = np.random.default_rng(V)
    n = len(SETTINGS)
    z = np.minimum(rng.geometric(0.2, (n, V)), 40).astype(np.float32)
    z[rng.random((n, V)) < 0.2] = -np.inf
    z[:, rng.integers(V)] = 3.0
    u = rng.random(n).astype(np.float32)
    print(f"[sample] exact V={V} {dtype}", flush=True)
    fgd, torch = env
    get = lambda k, d: _rows(torch, [s.get(k, d) for s in SETTINGS],  # noqa: E731
                             np.int32 if k == "top_k" else np.float32)
    tok, prob = _run(env, z, u, dtype, temperature=UNIT_T, top_k=get("top_k", 0), top_p=get("top_p", 1.0),
                     min_p=get("min_p", 0.0))
    for i, s in enumerate(SETTINGS):
        t, mass, total, _, _, _ = ref.sample(z[i], u[i], UNIT_T, **s)
        assert tok[i] == t, (s, u[i])
        assert prob[i] == np.float32(np.float32(mass) / np.float32(total)), s
        one, p1 = _run(env, z[i:i + 1], u[i:i + 1], dtype, temperature=UNIT_T, **s)  # a row alone, scalar settings
        assert one[0] == t and p1[0] == prob[i], s


@pytest.mark.parametrize("V", [5, 1000, 32001])
def test_every_draw_of_a_tied_row(env, V):
    """All logits equal: the draw walks the indices in order."""
    n = 64
    u = (np.arange(n) / n).astype(np.float32)
    z = np.full((n, V), -7.25, np.float32)
    tok, prob = _run(env, z, u)
    total = V << 31
    assert np.array_equal(tok, [int(np.float64(x) * total) >> 31 for x in u])
    assert (prob == np.float32(2.0 ** 31) / np.float32(total)).all()
    k = V // 2 + 1
    tok, _ = _run(env, z, u, top_k=k)
    assert np.array_equal(tok, [int(np.float64(x) * (k << 31)) >> 31 for x in u])


def _check_row(z, u, tok, prob, temperature, s):
    t, mass, total, before, idx, keep = ref.sample(z, u, temperature, **s)
    if t < 0 or not temperature > 0:
        assert tok == t
        return
    m, _ = ref.sample_masses(z, temperature)
    m = m[idx]
    # A cut may fall a few tokens away where masses lie within the error of
    # it; the tokens there are equally likely to within that error.
    err = 4 * (3 * 2.0 ** -24 * float(m.sum()) + z.size)
    at = int(np.nonzero(idx == tok)[0][0])
    lo = float(m[:at].sum())
    target = float(np.float64(np.float32(u))) * total
    assert lo - err <= target <= lo + float(m[at]) + err, (s, tok, t)
    assert abs(prob - float(m[at]) / total) <= err / total + 2.0 ** -22, s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [17, 777, 5000, 50257, 128256])
def test_ordinary_logits(env, V, dtype):
    fgd, torch = env
    rng = np.random.default_rng(V + 1)
    temps = [0.3, 0.7, 1.0, 1.5, 5.0]
    cases = [(t, s) for t in temps for s in SETTINGS]
    print(f"[sample] ordinary V={V} {dtype}", flush=True)
    z = (rng.standard_normal((len(cases), V)) * 2.5).astype(np.float32)
    z[np.arange(len(cases)), rng.integers(0, V, len(cases))] += 8
    z = _cuda(torch, z, dtype)
    u = rng.random(len(cases)).astype(np.float32)
    get = lambda k, d: _rows(torch, [s.get(k, d) for _, s in cases],  # noqa: E731
                             np.int32 if k == "top_k" else np.float32)
    tok, prob = fgd.sample(z, _rows(torch, u), _rows(torch, [t for t, _ in cases]), get("top_k", 0),
                           get("top_p", 1.0), get("min_p", 0.0))
    tok, prob, h = tok.cpu().numpy(), prob.cpu().numpy(), z.float().cpu().numpy()
    for i, (t, s) in enumerate(cases):
        _check_row(h[i], u[i], tok[i], prob[i], t, s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [6, 1000, 40000])
def test_rows_with_little_left(env, V, dtype):
    """Masked rows, infinities, NaN, the type's lowest value, extreme
    settings."""
    inf, low = np.inf, float(np.finfo(np.float32).min) if dtype == "f32" else -3.3895313892515355e38
    z = np.zeros((14, V), np.float32)
    z[0] = -inf
    z[1] = -inf
    z[1, V - 1] = -3.0                       # one token left
    z[2, 3] = np.nan
    z[3, 2] = inf                            # all the mass on one
    z[4, 1] = z[4, V - 1] = inf              # ... on two
    z[5] = low                               # nothing masked: all equal
    z[6] = low
    z[6, 4] = 0.0
    z[7, 5] = -inf
    z[8], z[8, 0] = -inf, np.nan
    z[9], z[9, 5] = 0.0, -0.0                # the zeros are equal
    z[10], z[10, 4] = 1.0, 2.0
    z[11], z[11, 4] = 1.0, 2.0
    z[12], z[12, 4] = 1.0, 2.0
    z[13] = 3.0e38 if dtype == "f32" else 2.9e38
    z[13, 2] = low
    u = np.array([0.5, 0.99, 0.5, 0.9, 0.75, 0.0, 0.999, 0.0, 0.1, 0.0, np.nan, -1.0, 2.0, 0.0], np.float32)
    tok, prob = _run(env, z, u, dtype)
    assert tok[0] == -1 and prob[0] == 0
    assert tok[1] == V - 1 and prob[1] == 1
    assert tok[2] == -1 and np.isnan(prob[2])
    assert tok[3] == 2 and prob[3] == 1
    assert tok[4] == V - 1 and prob[4] == 0.5
    assert tok[5] == 0 and prob[5] == np.float32(2.0 ** 31) / np.float32(V << 31)
    assert tok[6] == 4 and prob[6] == 1
    assert tok[7] == 0
    assert tok[8] == -1 and np.isnan(prob[8])
    assert tok[9] == 0
    assert tok[10] == 4 and tok[11] == 4     # NaN and negative: as 0
    last = [i for i in range(V) if i != 4][-1]
    assert tok[12] == last                   # above 1: as just below
    assert tok[13] == 0
    for t in (0.0, -1.0, float("nan"), 1e-45, 1e-39):  # greedy: the first of the largest
        tok, prob = _run(env, z, u, dtype, temperature=t)
        assert list(tok) == [-1, V - 1, -1, 2, 1, 0, 4, 0, -1, 0, 4, 4, 4, 0]
        ok = tok >= 0
        assert (prob[ok] == 1).all()
    tok, prob = _run(env, z[10:13], np.zeros(3, np.float32), dtype, temperature=float("inf"))
    assert (tok == 4).all() and (prob == np.float32(2.0 ** 31) / np.float32(V << 31)).all()


def test_long_tail_of_ties_and_padding(env):
    """bf16 logits tie by the thousand; a padded row's tail is never used,
    whatever it holds; rows may start off any boundary."""
    fgd, torch = env
    rng = np.random.default_rng(2)
    for V, ld in ((9001, 9001), (9001, 9013), (777, 1000)):
        z = np.round(rng.standard_normal((5, V)) * 4).astype(np.float32)
        u = rng.random(5).astype(np.float32)
        for dtype in ("f32", "bf16"):
            pool = torch.full((5, ld + 3), float("nan"), device="cuda",
                              dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
            pool[:, 3:3 + V] = _cuda(torch, z, dtype)
            for s in SETTINGS:
                tok, _ = fgd.sample(pool[:, 3:], _rows(torch, u), UNIT_T, vocab=V, **s)
                assert tok.tolist() == [ref.sample(z[i], u[i], UNIT_T, **s)[0] for i in range(5)], s


def test_rows_do_not_depend_on_their_batch(env):
    fgd, torch = env
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    U, V = 700, 30011
    z = torch.randn((U, V), generator=g, device="cuda") * 3
    u = torch.rand(U, generator=g, device="cuda")
    kw = dict(temperature=1.1, top_k=2000, top_p=0.97, min_p=1e-4)
    tok, prob = fgd.sample(z, u, **kw)
    for n in (1, 2, 9, 100, 257):
        t, p = fgd.sample(z[:n], u[:n], **kw)
        assert torch.equal(t, tok[:n]) and torch.equal(p, prob[:n])
    t, p = fgd.sample(z, u, **kw)
    assert torch.equal(t, tok) and torch.equal(p, prob)


def test_draws_follow_the_distribution(env):
    """20 000 draws of one row at evenly spaced random numbers: each token is
    drawn its share, to one draw at each end of its span."""
    fgd, torch = env
    rng = np.random.default_rng(8)
    V, n = 300, 20000
    z = (rng.standard_normal(V) * 2).astype(np.float32)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    tok, _ = fgd.sample(_cuda(torch, z[None]).expand(n, V).contiguous(), _rows(torch, u), temperature=0.8)
    got = np.bincount(tok.cpu().numpy(), minlength=V)
    p = np.exp(z.astype(np.float64) / 0.8)
    p /= p.sum()
    assert np.all(np.abs(got - n * p) <= 2)


def test_far_rows(env):
    """Rows that start past 2^32 bytes."""
    fgd, torch = env
    ld = 1_500_000_000
    V = 1003
    rng = np.random.default_rng(6)
    z = np.minimum(rng.geometric(0.3, (3, V)), 30).astype(np.float32)
    print("[sample] far rows", flush=True)
    pool = torch.zeros(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    view = pool.as_strided((3, V), (ld, 1))
    view.copy_(_cuda(torch, z, "bf16"))
    u = np.array([0.2, 0.6, 0.9], np.float32)
    tok, _ = fgd.sample(view, _rows(torch, u), UNIT_T)
    assert tok.tolist() == [ref.sample(z[i], u[i], UNIT_T)[0] for i in range(3)]


def test_other_stream_and_graph(env):
    fgd, torch = env
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    for U, V in ((2, 128256), (300, 5000)):
        z = torch.randn((U, V), generator=g, device="cuda") * 3
        u = torch.rand(U, generator=g, device="cuda")
        tok = torch.zeros(U, dtype=torch.int32, device="cuda")
        prob = torch.zeros(U, device="cuda")
        need = fgd.fgd_sample_workspace_size("f32", U, V)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        kw = dict(temperature=0.9, top_k=50, top_p=0.9, tokens_out=tok, probs_out=prob, workspace=ws)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        want = fgd.sample(z, u, 0.9, 50, 0.9)
        fgd.sample(z, u, stream=side, **kw)
        side.synchronize()
        assert torch.equal(tok, want[0]) and torch.equal(prob, want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            fgd.sample(z, u, **kw)
        torch.cuda.synchronize()
        for rep in range(3):
            u.copy_(torch.rand(U, generator=g, device="cuda"))
            ws.fill_(0x5A + rep)
            tok.zero_()
            want = fgd.sample(z, u, 0.9, 50, 0.9)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(tok, want[0]) and torch.equal(prob, want[1])


def test_many_long_bf16_rows(env):
    """Rows whose 16-bit values are counted, beside each of the reasons that
    send a row another way: values without a counter (tiny, huge), more of a
    value than half a counter holds, infinities, NaN, rows of masks alone."""
    fgd, torch = env
    n, V = 40, 70001
    rng = np.random.default_rng(11)
    z = rng.integers(-24, 9, (n, V)).astype(np.float32)
    z[rng.random((n, V)) < 0.1] = -np.inf
    lowest = -float(torch.finfo(torch.bfloat16).max)
    z[1] = -np.inf
    z[2, 5::2] = lowest
    z[3] = lowest
    z[4] = 0.0
    z[4, ::3] = -0.0
    z[5] = np.where(rng.random(V) < 0.5, 0.0, -0.0)
    z[6] = 4.0  # 70001 tokens of one value
    z[7] = -3.0
    z[8, 100] = np.nan
    z[9, 60000] = z[9, 61000] = np.inf
    z[10, :] = -5.0
    z[10, 69999] = 2.0 ** -40
    z[11, 17] = 2.0 ** 40
    z[12] = -np.inf
    z[12, 70000] = -1.0
    z[13] = -np.inf
    z[13, 0] = 2.0
    z[14] = -(2.0 ** 33)
    z[15, 1:] = -np.inf
    u = rng.random(n).astype(np.float32)
    settings = [SETTINGS[i % len(SETTINGS)] if i < 20 else SETTINGS[-(i % len(SETTINGS)) - 1] for i in range(n)]
    get = lambda k, d: _rows(torch, [s.get(k, d) for s in settings],  # noqa: E731
                             np.int32 if k == "top_k" else np.float32)
    kw = dict(top_k=get("top_k", 0), top_p=get("top_p", 1.0), min_p=get("min_p", 0.0))
    dense = _cuda(torch, z, "bf16")
    wide = torch.full((n, V + 6), 9.0, dtype=torch.bfloat16, device="cuda")
    for shift in (0, 1, 3):  # rows that start on no boundary of 16 bytes
        wide.fill_(9.0)
        wide[:, shift:shift + V] = dense
        for T in (UNIT_T, 0.0):
            print(f"[sample] counted rows, shift {shift}, T {T}", flush=True)
            tok, prob = fgd.sample(wide[:, shift:shift + V], _rows(torch, u), T, **kw)
            tok, prob = tok.cpu().numpy(), prob.cpu().numpy()
            for i, s in enumerate(settings):
                t, mass, total, _, _, _ = ref.sample(z[i], u[i], T, **s)
                assert tok[i] == t, (i, s, u[i])
                if i == 8:
                    assert np.isnan(prob[i])
                elif t < 0:
                    assert prob[i] == 0
                elif T:
                    assert prob[i] == np.float32(np.float32(mass) / np.float32(total)), (i, s)
    # Few rows take another form: the same tokens and probabilities.
    got = fgd.sample(dense, _rows(torch, u), 0.7, **kw)
    for lo in range(0, n, 8):
        few = fgd.sample(dense[lo:lo + 8], _rows(torch, u[lo:lo + 8]), 0.7,
                         **{k: v[lo:lo + 8] for k, v in kw.items()})
        for a, b in zip(got, few):
            assert torch.equal(torch.nan_to_num(a[lo:lo + 8], nan=-9.0), torch.nan_to_num(b, nan=-9.0))


def test_top_k_of_any_size(env):
    """A Python number past 32 bits keeps all tokens, whatever its lower bits."""
    fgd, torch = env
    V = 1000
    z = torch.zeros((8, V), device="cuda")
    u = torch.full((8,), 0.875, device="cuda")
    for k in (0, -1, -2 ** 31, -2 ** 31 - 5, 2 ** 31 - 1, 2 ** 31 + 5, 2 ** 32 + 5, 2 ** 70, np.int64(2 ** 32 + 5)):
        tok, prob = fgd.sample(z, u, top_k=k)
        assert (tok == 875).all() and (prob == float(np.float32(1 / V))).all(), k


def _time(torch, f, calls=10):
    """The least time of a call, in us, of five runs of `calls`."""
    f()
    best = float("inf")
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        a.record()
        for _ in range(calls):
            f()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) / calls * 1e3)
    return best


def _masked(torch, U, V, value, seed=1):
    """(bf16 logits of which 60% are masked with `value`, the same with -inf)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((U, V), generator=g, device="cuda") * 2
    forbidden = torch.rand((U, V), generator=g, device="cuda") < 0.6
    return [z.masked_fill(forbidden, v).bfloat16() for v in (value, -float("inf"))]


def test_more_of_a_value_than_a_counter_holds(env):
    """Long bf16 rows in which over 65535 tokens share a value without mass:
    the tokens are those of rows masked with -inf, and such rows are read four
    times for two (with atomics on one address beside that), not by the dozen."""
    fgd, torch = env
    U, V = 64, 128256
    z, plain = _masked(torch, U, V, -100.0)
    u = torch.rand(U, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    settings = (dict(top_p=0.9), dict(top_k=50, top_p=0.9), dict(temperature=0.7), dict(min_p=0.05),
                dict(top_k=1000, top_p=0.95, min_p=0.001))
    for kw in settings:
        print(f"[sample] over 65535 of a value {kw}", flush=True)
        for a, b in zip(fgd.sample(z, u, **kw), fgd.sample(plain, u, **kw)):
            assert torch.equal(a, b), kw
    for kw in settings[:2]:
        t, t_plain = (_time(torch, lambda: fgd.sample(v, u, **kw)) for v in (z, plain))
        assert t < 5 * t_plain, (t, t_plain)


def test_finite_masks(env):
    """Long bf16 rows masked with the usual finite values, also far more
    tokens than a counter holds: the tokens and, to a factor of two (measured:
    one), the time of rows masked with -inf."""
    fgd, torch = env
    U, V = 64, 128256
    u = torch.rand(U, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    for value in (-1e3, -1e4, -65504.0, -1e9, -1e30, -float(torch.finfo(torch.bfloat16).max)):
        z, plain = _masked(torch, U, V, value, 4)
        print(f"[sample] masked with {value}", flush=True)
        for kw in (dict(top_p=0.9), dict(top_k=50, top_p=0.9), dict(temperature=1.3, min_p=0.01), dict()):
            for a, b in zip(fgd.sample(z, u, **kw), fgd.sample(plain, u, **kw)):
                assert torch.equal(a, b), (value, kw)
        t, t_plain = (_time(torch, lambda: fgd.sample(v, u, top_p=0.9)) for v in (z, plain))
        assert t < 2 * t_plain, (value, t, t_plain)


def test_large_logits_that_have_mass(env):
    """Long bf16 rows at a temperature so high that logits of hundreds and
    thousands, tiny ones and masks weigh alike: c = 2^-8, logits of multiples
    of 2^8, so that every weight is a power of two."""
    fgd, torch = env
    n, V = 40, 70001
    rng = np.random.default_rng(21)
    T = float(np.float32(UNIT_T * 256))
    assert (np.float32(1) / np.float32(T)) * np.float32(np.log2(np.e)) == np.float32(2.0 ** -8)
    z = (rng.integers(-12, 2, (n, V)) * 256).astype(np.float32)  # down to -12 2^8, up to 2^8
    z[1] = np.where(rng.random(V) < 0.95, -1024.0, z[1])
    z[2, 77] = 512.0
    z[3, 65000] = 4096.0
    z[4] = np.where(rng.random(V) < 0.5, -np.inf, np.minimum(z[4], 0))
    z[5] = -512.0
    z[6] = -768.0
    z[6, 5] = -512.0
    z[7] = -np.inf
    z[7, ::9] = -2.0 ** 20
    z[8] = -256.0
    z[9] = 256.0
    z[10, 3] = 2.0 ** -60  # as good as zero, but before it in the order
    z[10] = np.minimum(z[10], 2.0 ** -60)
    u = rng.random(n).astype(np.float32)
    print("[sample] large logits", flush=True)
    settings = [SETTINGS[i % len(SETTINGS)] for i in range(n)]
    get = lambda k, d: _rows(torch, [s.get(k, d) for s in settings],  # noqa: E731
                             np.int32 if k == "top_k" else np.float32)
    kw = dict(top_k=get("top_k", 0), top_p=get("top_p", 1.0), min_p=get("min_p", 0.0))
    tok, prob = _run(env, z, u, "bf16", temperature=T, **kw)
    z = _host_of_bf16(torch, z)
    for i, s in enumerate(settings):
        t, mass, total, _, _, _ = ref.sample(z[i], u[i], T, **s)
        assert tok[i] == t, (i, s, u[i])
        assert prob[i] == np.float32(np.float32(mass) / np.float32(total)), (i, s)


def test_flat_rows_at_no_temperature(env):
    """1 / T = 0: every token that is not masked by -inf weighs the same."""
    fgd, torch = env
    rng = np.random.default_rng(22)
    for U, V, dtype in ((3, 5000, "f32"), (40, 40000, "bf16"), (2, 70001, "f32")):
        z = (rng.standard_normal((U, V)) * 3).astype(np.float32)
        z[rng.random((U, V)) < 0.3] = -np.inf
        u = rng.random(U).astype(np.float32)
        z = _host_of_bf16(torch, z) if dtype == "bf16" else z
        for s in (dict(), dict(top_k=100), dict(top_p=0.25), dict(min_p=1.0)):
            tok, prob = _run(env, z, u, dtype, temperature=float("inf"), **s)
            for i in range(U):
                t, mass, total, _, _, _ = ref.sample(z[i], u[i], float("inf"), **s)
                assert tok[i] == t, (U, i, s)
                assert prob[i] == np.float32(np.float32(mass) / np.float32(total))


def _host_of_bf16(torch, a):
    return torch.from_numpy(a).bfloat16().float().numpy()


def test_masses_bit_by_bit(env):
    """Rows of two tokens whose logits differ by -t at c = 1.  The second is
    kept up to min_p = w, which gives the kernel's own weight w = 2^t to the bit;
    its probability is then that of the mass that the definition gives w, also
    where w 2^31 is a whole number and w 2^31 + 1/2 a tie."""
    fgd, torch = env
    rng = np.random.default_rng(31)
    t = np.concatenate([-7 - rng.random(500), -20 * rng.random(300)]).astype(np.float32)
    near = np.exp2(t.astype(np.float64)).astype(np.float32)
    steps = np.arange(-6, 7, dtype=np.int32)
    cand = (near.view(np.int32)[:, None] + steps).view(np.float32)  # neighbouring float32 values
    z = np.zeros((t.size, 2), np.float32)
    z[:, 1] = t
    below_1 = np.nextafter(np.float32(1), np.float32(0))
    tok, _ = _run(env, np.repeat(z, steps.size, 0), np.full(cand.size, below_1), temperature=UNIT_T,
                  min_p=_rows(torch, cand.reshape(-1)))
    kept = tok.reshape(cand.shape) == 1
    assert kept[:, 0].all() and not kept[:, -1].any() and (kept[:, :-1] >= kept[:, 1:]).all()
    w = cand[np.arange(t.size), kept.sum(1) - 1]
    m = ref.mass_of(w)
    tok, prob = _run(env, z, np.full(t.size, below_1), temperature=UNIT_T)
    assert (tok == 1).all()
    f32 = np.float32
    assert np.array_equal(prob, (m.astype(f32) / (m + 2 ** 31).astype(f32)).astype(f32))
    whole = (w.astype(np.float64) * 2 ** 31).astype(np.int64)
    tie = (whole >= 2 ** 23) & (whole < 2 ** 24) & (whole % 2 == 1)
    other = (whole.astype(f32) / (whole + 2 ** 31).astype(f32)).astype(f32)
    assert (tie & (prob != other)).sum() > 50  # the two can be told apart


@pytest.mark.parametrize("V", [28671, 28672, 28679, 262143, 262144, 262145])
def test_counted_rows_at_the_ends_of_their_range(env, V):
    """bf16 rows on both sides of the shortest and of the longest that are
    counted (and of the last word of their matches' bits), starting on and off
    16 bytes; the token drawn lies in the head, the first and the last vectors,
    the last word, and the tail."""
    fgd, torch = env
    n = 40
    rng = np.random.default_rng(V)
    z = rng.integers(-24, -12, (n, V)).astype(np.float32)
    places = [0, 1, 7, 8, 9, 255, V // 2, V - 264, V - 256, V - 33, V - 17, V - 16, V - 10, V - 9, V - 8, V - 7, V - 2, V - 1]
    for i in range(n):  # rows of one heavy token, then of two alike
        z[i, places[i % len(places)]] = 8.0
        z[i, places[(i + i // len(places)) % len(places)]] = 8.0
    z[n - 1] = -2.0  # more of a value than a counter holds, where the row is long
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    want = [ref.sample(z[i], u[i], UNIT_T, top_p=0.99) for i in range(n)]
    full = [ref.sample(z[i], u[i], UNIT_T) for i in range(n)]
    wide = torch.full((n, V + 9), 9.0, dtype=torch.bfloat16, device="cuda")
    for shift in (0, 1, 7):
        print(f"[sample] ends of the counted range V={V} shift {shift}", flush=True)
        wide.fill_(9.0)
        rows = wide[:, shift:shift + V]
        rows.copy_(_cuda(torch, z, "bf16"))
        for refs, kw in ((want, dict(top_p=0.99)), (full, dict())):
            tok, prob = fgd.sample(rows, _rows(torch, u), UNIT_T, **kw)
            tok, prob = tok.tolist(), prob.cpu().numpy()
            for i, r in enumerate(refs):
                assert tok[i] == r[0], (i, kw)
                assert prob[i] == np.float32(np.float32(r[1]) / np.float32(r[2])), (i, kw)


@pytest.mark.parametrize("U, V, dtype", [(3, 70001, "f32"), (3, 70001, "bf16"), (40, 30001, "bf16")], ids=str)
def test_far_long_rows(env, U, V, dtype):
    """Rows that start past 2^32 bytes, split over blocks and counted."""
    fgd, torch = env
    es = 4 if dtype == "f32" else 2
    ld = (9 * 2 ** 30 // es // (U - 1)) | 1
    rng = np.random.default_rng(V)
    z = np.minimum(rng.geometric(0.3, (U, V)), 30).astype(np.float32)
    print(f"[sample] far rows {U} x {V} {dtype}", flush=True)
    pool = torch.zeros((U - 1) * ld + V, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    view = pool.as_strided((U, V), (ld, 1))
    view.copy_(_cuda(torch, z, dtype))
    u = rng.random(U).astype(np.float32)
    for kw in (dict(), dict(top_k=50, top_p=0.9)):
        tok, _ = fgd.sample(view, _rows(torch, u), UNIT_T, **kw)
        assert tok.tolist() == [ref.sample(z[i], u[i], UNIT_T, **kw)[0] for i in range(U)]


def test_every_binade_of_counted_logits(env):
    """Long bf16 rows with logits of every binade and either sign, on both
    sides of the ranges that are counted, below a top beside which the small
    ones vanish: c = 2^-8, so that every weight is a power of two."""
    fgd, torch = env
    V = 30011
    rng = np.random.default_rng(41)
    T = float(np.float32(UNIT_T * 256))
    ends = [2.0 ** e for e in (-133, -126, -56, -55, -54, -33, -32, -31)]
    large = [2.0 ** e for e in range(8, 13)]
    rows = []
    for top in (256.0, 4096.0, 2.0 ** 20, 2.0 ** 31, 2.0 ** 33):
        small = rng.choice(ends + [2.0 ** e for e in range(-60, -20)] + [0.0], V) * rng.choice([-1.0, 1.0], V)
        z = np.where(rng.random(V) < 0.3, -rng.choice(large, V), small)
        z[rng.integers(0, V, 5)] = top
        rows.append(z)                             # some above, masks among them
        rows.append(np.where(z > 0, -z, z))        # none above zero
        rows.append(np.where(np.abs(z) < 1, z, -np.inf))
        rows.append(np.where(z == 0, top, -np.abs(z)))
    z = np.stack(rows * 2).astype(np.float32)      # 40 rows
    z = _host_of_bf16(torch, z)
    n = z.shape[0]
    u = rng.random(n).astype(np.float32)
    settings = [SETTINGS[(i + i // 20) % len(SETTINGS)] for i in range(n)]
    get = lambda k, d: _rows(torch, [s.get(k, d) for s in settings],  # noqa: E731
                             np.int32 if k == "top_k" else np.float32)
    print("[sample] every binade", flush=True)
    tok, prob = _run(env, z, u, "bf16", temperature=T, top_k=get("top_k", 0), top_p=get("top_p", 1.0),
                     min_p=get("min_p", 0.0))
    for i, s in enumerate(settings):
        t, mass, total, _, _, _ = ref.sample(z[i], u[i], T, **s)
        assert tok[i] == t, (i, s, u[i])
        assert prob[i] == np.float32(np.float32(mass) / np.float32(total)), (i, s)
