"""GPU tests of the 4-bit operators against 64-bit references.

Quantisation is exact: the scale is a power of two and the rounding is to a
grid that both sides know, so values and scale bytes must agree bit for bit.

Products of 4-bit values are exact in float32; what the kernels round are
the sums of up to K of them.  A sum of n float32 terms in any order is off by
at most n eps sum|terms| (eps = 2^-24); the instruction adds 128 of them per
step, so the bar is (K / 128 + 128) eps sum|a b|.  A bf16 output is the float32
one rounded once, bit for bit.
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


def _t(torch, dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _host(t):
    return t.detach().to("cpu").double().numpy()


def _values(shape, seed, spread=3.0):
    """Normal values whose blocks differ in size by a few binades."""
    rng = np.random.default_rng(seed)
    return (rng.standard_normal(shape) * np.exp2(rng.uniform(-spread, spread, shape[:-1] + (1,)))).astype(np.float32)


def _tensor(torch, a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(_t(torch, dtype))


SHAPES = [(1, 1), (1, 32), (1, 33), (3, 31), (16, 128), (17, 129), (64, 127), (65, 256), (5, 1000), (200, 96),
          (1, 4097), (130, 513)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_round_trip_along_rows_and_columns(env, shape, dtype):
    fgd, torch = env
    print(f"[mx4] round trip {shape} {dtype}", flush=True)
    x = _tensor(torch, _values(shape, 1 + shape[0] * shape[1]), dtype)
    for view in (x, x.mT):
        q = fgd.mx4_quantize(view)
        assert q.shape == tuple(view.shape)
        want = ref.mx4_values(_host(view))
        for out in ("f32", "bf16"):
            got = _host(fgd.mx4_dequantize(q, out))
            assert np.array_equal(got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_round_trip_of_batches_and_strides(env, dtype):
    """Batches of padded rows, rows that start off any 16-byte boundary, a
    broadcast batch, and the columns of the same storage."""
    fgd, torch = env
    rng = np.random.default_rng(3)
    pool = _tensor(torch, rng.standard_normal(3 * 70 * 211 + 5).astype(np.float32), dtype)
    for off in (0, 1, 3):
        base = pool[off:off + 3 * 70 * 211].view(3, 70, 211)
        for x in (base, base[:, :, 1:200], base[:, 3:68, :], base[1:2].expand(3, 70, 211), base.mT, base[:, 2:].mT):
            got = _host(fgd.mx4_dequantize(fgd.mx4_quantize(x)))
            assert np.array_equal(got, ref.mx4_values(_host(x)))
    out = torch.full((3, 70, 300), 7.0, dtype=_t(torch, dtype), device="cuda")
    q = fgd.mx4_quantize(base)
    fgd.mx4_dequantize(q, out=out[:, :, 5:216])
    assert np.array_equal(_host(out[:, :, 5:216]), ref.mx4_values(_host(base)))
    assert (out[:, :, :5] == 7).all() and (out[:, :, 216:] == 7).all()  # nothing beside the view


def test_every_binade_and_tie(env):
    """Blocks whose largest magnitude runs through every float32 binade,
    denormals included, with elements on, just below and just above every
    rounding boundary; scale bytes as the header lays them out."""
    fgd, torch = env
    edges = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], np.float64)
    rows = []
    for e in range(-149, 128):
        unit = 2.0 ** (e - 2)
        v = np.concatenate([edges, edges * (1 - 2 ** -20), edges * (1 + 2 ** -20), -edges]) * unit
        with np.errstate(over="ignore"):
            v = v.astype(np.float32)
        v[np.abs(v) >= 2.0 ** min(e + 1, 127)] = 0
        v[31] = np.float32(2.0 ** e)
        rows.append(v)
    x = np.stack(rows)
    q = fgd.mx4_quantize(_tensor(torch, x, "f32"))
    assert np.array_equal(_host(fgd.mx4_dequantize(q)), ref.mx4_values(x))
    s = q.scales.cpu().numpy().reshape(-1, 64, 4)  # [row tile][lane][fragment]: one column tile
    got = np.array([s[r // 64, r % 32, 2 * (r % 64 // 32)] for r in range(x.shape[0])])
    assert np.array_equal(got, ref.mx4_scale_bytes(x)[:, 0])


def test_zero_signs_infinities_and_nan(env):
    fgd, torch = env
    x = np.zeros((6, 96), np.float32)
    x[0, 3] = -0.0
    x[1, 40] = np.inf
    x[2, 70] = -np.inf
    x[3, 5] = np.nan
    x[4, 33] = np.finfo(np.float32).max
    x[5] = -np.finfo(np.float32).max
    for dtype in ("f32", "bf16"):
        t = _tensor(torch, x, dtype)
        got = _host(fgd.mx4_dequantize(fgd.mx4_quantize(t)))
        want = ref.mx4_values(_host(t))
        assert np.array_equal(got, want, equal_nan=True)
        assert np.signbit(got[0, 3]) and np.isnan(got[1, 32:64]).all() and not np.isnan(got[1, :32]).any()


def _check_product(got, a, w):
    """The float32 output `got` against the 64-bit product of the quantised
    values a, w."""
    want = a @ np.swapaxes(w, -1, -2)
    size = np.abs(a) @ np.swapaxes(np.abs(w), -1, -2)
    K = a.shape[-1]
    bar = (K / 128 + 128) * 2.0 ** -24 * size
    bad = ~(np.abs(got - want) <= bar)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / (size + 1e-300))}"


PRODUCTS = [(1, 1, 1), (1, 5, 33), (1, 128, 256), (2, 64, 1000), (3, 257, 129), (16, 300, 96), (17, 65, 640),
            (31, 1000, 224), (64, 64, 128), (65, 33, 300), (100, 513, 2048), (129, 255, 1024), (256, 256, 256),
            (257, 300, 520), (300, 1030, 385), (1, 700, 9000), (40, 90, 8200),
            (1, 9000, 2048), (4, 9000, 2048), (5, 9000, 2048), (30, 9000, 100), (2, 9000, 8192), (48, 8200, 300),
            (70, 4200, 1100), (300, 2100, 700), (520, 2049, 1153)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mnk", PRODUCTS, ids=str)
def test_product(env, mnk, dtype):
    fgd, torch = env
    m, n, k = mnk
    print(f"[mx4] product {mnk} {dtype}", flush=True)
    x, w = _tensor(torch, _values((m, k), m + k), dtype), _tensor(torch, _values((n, k), n + k, 1.0), dtype)
    a4, w4 = fgd.mx4_quantize(x), fgd.mx4_quantize(w)
    a, b = ref.mx4_values(_host(x)), ref.mx4_values(_host(w))
    y = fgd.mx4_matmul(a4, w4, "f32")
    assert y.dtype == torch.float32
    _check_product(_host(y), a, b)
    assert torch.equal(fgd.mx4_matmul(a4, w4), y.to(torch.bfloat16))
    for out_dtype in ("f32", "bf16"):  # the same bits from one call
        assert torch.equal(fgd.mx4_linear(x, w4, out_dtype), y.to(_t(torch, out_dtype)))
    assert torch.equal(fgd.mx4_linear(x, w4), fgd.mx4_linear(x, w4, dtype))


@pytest.mark.parametrize("T", [1, 3, 20, 70, 200])
@pytest.mark.parametrize("M", [2, 9])
def test_product_of_workers(env, M, T):
    """A batch gives each worker's own product, also from strided rows and
    into a strided output."""
    fgd, torch = env
    N, K = 333, 420
    print(f"[mx4] batch M={M} T={T}", flush=True)
    x = _tensor(torch, _values((M, T, K + 13), 7), "bf16")[:, :, 3:3 + K]
    w = _tensor(torch, _values((M, N, K), 8), "bf16")
    w4 = fgd.mx4_quantize(w)
    pool = torch.full((M, T + 2, N + 9), 3.0, dtype=torch.float32, device="cuda")
    y = fgd.mx4_linear(x, w4, out=pool[:, 1:T + 1, 2:N + 2])
    for i in range(M):
        a, b = ref.mx4_values(_host(x[i])), ref.mx4_values(_host(w[i]))
        _check_product(_host(y[i]), a, b)
        _check_product(_host(fgd.mx4_linear(x[i], fgd.mx4_quantize(w[i]), "f32")), a, b)
    pool[:, 1:T + 1, 2:N + 2] = 3.0
    assert (pool == 3.0).all()


def test_every_number_of_tokens(env):
    """The first n tokens of a batch, for n on both sides of every tile."""
    fgd, torch = env
    x = _tensor(torch, _values((300, 1500), 5), "bf16")
    w = _tensor(torch, _values((700, 1500), 6), "bf16")
    w4 = fgd.mx4_quantize(w)
    a, b = ref.mx4_values(_host(x)), ref.mx4_values(_host(w))
    for n in (1, 2, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 191, 192, 193, 256, 257):
        y = fgd.mx4_linear(x[:n], w4, "f32")
        _check_product(_host(y), a[:n], b)
        assert torch.equal(y, fgd.mx4_linear(x[:n], w4, "f32"))


def test_nan_blocks_reach_only_their_row_and_column(env):
    fgd, torch = env
    for T in (4, 300):
        x = _tensor(torch, _values((T, 256), 1), "f32")
        w = _tensor(torch, _values((300, 256), 2), "f32")
        x[2, 100] = float("inf")
        w[77, 3] = float("nan")
        y = fgd.mx4_linear(x, fgd.mx4_quantize(w))
        nan = torch.zeros((T, 300), dtype=torch.bool, device="cuda")
        nan[2], nan[:, 77] = True, True
        assert torch.equal(torch.isnan(y), nan)


def test_sizes_of_zero(env):
    fgd, torch = env
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    assert fgd.mx4_dequantize(fgd.mx4_quantize(z(0, 5))).shape == (0, 5)
    assert fgd.mx4_dequantize(fgd.mx4_quantize(z(0, 3, 5))).shape == (0, 3, 5)
    assert fgd.mx4_linear(z(0, 64), fgd.mx4_quantize(z(7, 64))).shape == (0, 7)
    assert fgd.mx4_linear(z(3, 64), fgd.mx4_quantize(z(0, 64))).shape == (3, 0)
    out = torch.full((3, 7), 5.0, device="cuda")
    fgd.mx4_linear(z(3, 0), fgd.mx4_quantize(z(7, 0)), out=out)
    assert (out == 0).all()  # a product over nothing


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mtnk", [(None, 1, 40, 64), (None, 130, 200, 96), (2, 77, 100, 210), (None, 300, 513, 290)],
                         ids=str)
def test_gradients_against_their_formula(env, mtnk, dtype):
    fgd, torch = env
    M, T, N, K = mtnk
    lead = () if M is None else (M,)
    print(f"[mx4] grads {mtnk} {dtype}", flush=True)
    x, w = _tensor(torch, _values((*lead, T, K), 1), dtype), _tensor(torch, _values((*lead, N, K), 2), dtype)
    dy = _tensor(torch, _values((*lead, T, N), 3), dtype)
    w_t = fgd.mx4_quantize(w.mT)
    dx, dw = fgd.mx4_linear_grads(dy, x, w_t)
    assert dx.dtype == dy.dtype and dw.dtype == torch.float32
    sw = lambda a: np.swapaxes(a, -1, -2)  # noqa: E731
    hx, hw, hdy = _host(x), _host(w), _host(dy)
    _check_product(_host(dw), ref.mx4_values(sw(hdy)), ref.mx4_values(sw(hx)))
    kept = fgd.mx4_linear_grads(dy, fgd.mx4_quantize(x.mT), w_t, dx_dtype="f32", dw_dtype="bf16")
    _check_product(_host(kept[0]), ref.mx4_values(hdy), ref.mx4_values(sw(hw)))
    assert kept[0].dtype == torch.float32 and torch.equal(kept[0].to(dx.dtype), dx)
    assert torch.equal(kept[1], dw.to(torch.bfloat16))


def test_gradients_against_differences(env):
    """Where every operand stands on the 4-bit grid along both axes, rounding
    is the identity, so the layer is bilinear and differences of its loss
    sum(dy y) are exact: moving one x or w by 1 (which stays on the grid) moves
    the loss by that element's gradient."""
    fgd, torch = env
    rng = np.random.default_rng(4)
    T, N, K = 64, 96, 64

    def grid(shape):
        """Whole numbers of {-2..2}, with a 4 in every block of 32 of both
        axes, so that every block's scale is 1 and +1 moves stay on it."""
        a = rng.integers(-2, 3, shape).astype(np.float32)
        for i in range(0, shape[0], 32):
            for j in range(0, shape[1], 32):
                d = rng.permutation(32)
                a[i + np.arange(32), j + d] = 4.0
        return a

    x, w, dy = grid((T, K)), grid((N, K)), grid((T, N))
    t = lambda a: _tensor(torch, a, "f32")  # noqa: E731
    dx, dw = (_host(g) for g in fgd.mx4_linear_grads(t(dy), t(x), fgd.mx4_quantize(t(w).mT)))

    def loss(x, w):
        return float((_host(fgd.mx4_linear(t(x), fgd.mx4_quantize(t(w)))) * dy).sum())

    base = loss(x, w)
    for _ in range(12):
        i, j = int(rng.integers(T)), int(rng.integers(K))
        if x[i, j] < 2:
            moved = x.copy()
            moved[i, j] += 1
            assert loss(moved, w) - base == dx[i, j]
        i = int(rng.integers(N))
        if w[i, j] < 2:
            moved = w.copy()
            moved[i, j] += 1
            assert loss(x, moved) - base == dw[i, j]


def test_offsets_past_32_bits(env):
    """A matrix whose source and output elements lie past 2^31 elements and
    2^32 bytes: the last rows of a large strided array."""
    fgd, torch = env
    rows, ld = 3, 1_500_000_000
    print("[mx4] far rows", flush=True)
    pool = torch.zeros(2 * ld + 300, dtype=torch.bfloat16, device="cuda")
    x = pool.as_strided((rows, 300), (ld, 1))
    x.copy_(_tensor(torch, _values((rows, 300), 9), "bf16"))
    q = fgd.mx4_quantize(x)
    want = ref.mx4_values(_host(x))
    assert np.array_equal(_host(fgd.mx4_dequantize(q)), want)
    w = _tensor(torch, _values((300, 300), 10), "bf16")
    near = fgd.mx4_linear(x, fgd.mx4_quantize(w))
    fgd.mx4_linear(x.clone(), fgd.mx4_quantize(w), out=x)
    assert torch.equal(x, near)


def test_other_stream_and_graph(env):
    """The calls run on the stream they are given, and may be captured; a
    replay reads what the inputs hold then."""
    fgd, torch = env
    x = _tensor(torch, _values((40, 512), 1), "bf16")
    w = _tensor(torch, _values((300, 512), 2), "bf16")
    w4 = fgd.mx4_quantize(w)
    want = fgd.mx4_linear(x, w4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = torch.empty_like(want)
    ws = torch.empty(fgd.fgd_mx4_linear_workspace_size(1, 40, 512), dtype=torch.uint8, device="cuda")
    fgd.mx4_linear(x, w4, out=y, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    q = fgd.mx4_quantize(w)
    back = torch.empty_like(w)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        fgd.mx4_linear(x, w4, out=y, workspace=ws)
        fgd.mx4_dequantize(q, out=back)
    torch.cuda.synchronize()
    for rep in range(3):
        x.copy_(_tensor(torch, _values((40, 512), 20 + rep), "bf16"))
        y.zero_()
        back.zero_()
        ws.fill_(0xA5)
        want = fgd.mx4_linear(x, w4)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), rep
        assert np.array_equal(_host(back), ref.mx4_values(_host(w)))


def test_what_a_call_allocates_belongs_to_its_stream(env):
    """The calls' own workspaces, temporaries and outputs are not handed to
    the current stream while the stream that they were given is still to run."""
    fgd, torch = env
    x = _tensor(torch, _values((1000, 512), 3), "bf16")
    w = _tensor(torch, _values((600, 512), 4), "bf16")
    dy = _tensor(torch, _values((1000, 600), 5), "bf16")
    z = _tensor(torch, _values((2, 200000), 6), "f32")
    u = torch.full((2,), 0.5, device="cuda")
    w4, w_t4 = fgd.mx4_quantize(w), fgd.mx4_quantize(w.mT)

    def calls(stream):
        return [fgd.mx4_linear(x, w4, stream=stream), *fgd.mx4_linear_grads(dy, x, w_t4, stream=stream),
                fgd.mx4_dequantize(fgd.mx4_quantize(x, stream), stream=stream), *fgd.sample(z, u, stream=stream)]

    want = calls(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)  # about 10 ms
        got = calls(stream)
        mine = [torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")
                for n in [2 ** k for k in range(9, 22)] for _ in range(4)]
        torch.cuda.synchronize()
        assert all(bool((t == 0xA5).all()) for t in mine)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("bmnk", [(1, 7, 17001, 300), (1, 30, 17001, 1300), (1, 2, 40000, 2048), (1, 1, 40001, 96),
                                  (1, 1100, 17000, 300), (1, 1100, 17000, 640), (1, 2100, 33000, 100),
                                  (1, 2100, 33000, 300), (1, 2100, 33000, 385), (3, 300, 9000, 200),
                                  (2, 130, 40000, 129)], ids=str)
def test_products_of_many_blocks(env, bmnk):
    """More blocks of the result than the card holds at once, whole ones and
    the matrix's edges, over even and odd numbers of column tiles."""
    fgd, torch = env
    b, m, n, k = bmnk
    print(f"[mx4] many blocks {bmnk}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(sum(bmnk))
    x = torch.randn(b, m, k, device="cuda", generator=g).bfloat16()
    w = torch.randn(b, n, k, device="cuda", generator=g).bfloat16()
    a4, w4 = fgd.mx4_quantize(x), fgd.mx4_quantize(w)
    y, y16 = fgd.mx4_matmul(a4, w4, "f32"), fgd.mx4_matmul(a4, w4)
    assert torch.equal(y16, y.bfloat16())
    lines = torch.full((b, m, n + 3), 7.0, dtype=torch.float32, device="cuda")
    assert torch.equal(fgd.mx4_linear(x, w4, out=lines[:, :, 1:n + 1]), y)
    lines[:, :, 1:n + 1] = 7.0
    assert bool((lines == 7.0).all())
    for i in range(b):
        p = torch.from_numpy(ref.mx4_values(_host(x[i]))).cuda()
        q = torch.from_numpy(ref.mx4_values(_host(w[i]))).cuda().T.contiguous()
        off = (y[i].double() - p @ q).abs_()
        assert bool((off <= (k / 128 + 128) * 2.0 ** -24 * (p.abs() @ q.abs())).all())


def test_more_matrices_than_a_grid_holds(env):
    """A batch of 70000 tiny matrices: quantised, read back, multiplied."""
    fgd, torch = env
    b, m, n, k = 70000, 2, 3, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(b, m, k, device="cuda", generator=g)
    w = torch.randn(b, n, k, device="cuda", generator=g)
    x4, w4 = fgd.mx4_quantize(x), fgd.mx4_quantize(w)
    p, q = fgd.mx4_dequantize(x4), fgd.mx4_dequantize(w4)
    for i in (0, 1, 65534, 65535, 65536, b - 1):
        assert np.array_equal(_host(p[i]), ref.mx4_values(_host(x[i])))
        assert np.array_equal(_host(q[i]), ref.mx4_values(_host(w[i])))
    y, p, q = fgd.mx4_matmul(x4, w4, "f32"), p.double(), q.double()
    assert torch.equal(fgd.mx4_linear(x, w4), y)
    terms = p[:, :, None, :] * q[:, None, :, :]
    off = (y.double() - terms.sum(-1)).abs()
    assert bool((off <= (k / 128 + 128) * 2.0 ** -24 * terms.abs().sum(-1)).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_both_axes_in_one_reading(env, dtype):
    """The codes and scales of the two calls, byte for byte."""
    fgd, torch = env

    def same(x):
        q, t = fgd.mx4_quantize_both(x)
        for got, want in ((q, fgd.mx4_quantize(x)), (t, fgd.mx4_quantize(x.mT))):
            assert got.shape == want.shape
            assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales), tuple(x.shape)

    for shape in SHAPES + [(63, 64), (128, 128), (129, 65), (300, 1000), (4097, 3), (2, 77, 200), (3, 1, 129),
                           (5, 130, 33)]:
        print(f"[mx4] both {shape} {dtype}", flush=True)
        x = _tensor(torch, _values(shape, sum(shape)), dtype)
        same(x)
        same(x.mT)
    wide = _tensor(torch, _values((3, 90, 207), 1), dtype)
    same(wide[:, 1:, 3:200])
    odd = wide[0].clone()
    odd[3, 5], odd[70, 6], odd[71, 7], odd[8] = float("nan"), float("inf"), -0.0, 0.0
    odd[:, 40] = 1e-39
    same(odd)
    for shape in ((0, 5), (5, 0), (0, 0), (2, 0, 3)):
        q, t = fgd.mx4_quantize_both(torch.empty(shape, device="cuda"))
        assert q.shape == shape and t.shape == (*shape[:-2], shape[-1], shape[-2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mtnk", [(None, 1, 1, 1), (None, 1, 40, 64), (None, 257, 130, 1), (2, 77, 100, 210),
                                  (None, 300, 513, 290), (None, 0, 5, 7), (3, 4, 0, 7), (None, 4, 5, 0), (0, 4, 5, 6)],
                         ids=str)
def test_gradients_in_one_call_are_those_of_its_parts(env, mtnk, dtype):
    """The same bits, also from padded rows, from operands stored by columns
    and from a kept transpose."""
    fgd, torch = env
    M, T, N, K = mtnk
    lead = () if M is None else (M,)
    print(f"[mx4] gradients in one call {mtnk} {dtype}", flush=True)
    dy, x = _tensor(torch, _values((*lead, T, N), 3), dtype), _tensor(torch, _values((*lead, T, K), 4), dtype)
    w_t = fgd.mx4_quantize(_tensor(torch, _values((*lead, K, N), 5), dtype))
    want = (fgd.mx4_matmul(fgd.mx4_quantize(dy), w_t, dy.dtype),
            fgd.mx4_matmul(fgd.mx4_quantize(dy.mT), fgd.mx4_quantize(x.mT), "f32"))

    def padded(t):
        wide = torch.full((*t.shape[:-1], t.shape[-1] + 5), 9.0, dtype=t.dtype, device="cuda")
        wide[..., 2:2 + t.shape[-1]] = t
        return wide[..., 2:2 + t.shape[-1]]

    by_columns = lambda t: t.mT.contiguous().mT  # noqa: E731
    for a, b in ((dy, x), (padded(dy), padded(x)), (by_columns(dy), x), (dy, by_columns(x)),
                 (dy, fgd.mx4_quantize(x.mT))):
        got = fgd.mx4_linear_grads(a, b, w_t)
        for g, v in zip(got, want):
            assert g.dtype == v.dtype and torch.equal(g, v)
    got = fgd.mx4_linear_grads(dy, x, w_t, dx_dtype="f32", dw_dtype="bf16")
    assert torch.equal(got[0].to(dy.dtype), want[0]) and torch.equal(got[1], want[1].bfloat16())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_row_of_strided_columns(env, dtype):
    """A matrix of one row (or column) has no other to be apart from: every
    call that takes it contiguous takes it with any stride."""
    fgd, torch = env
    pool = _tensor(torch, _values((3, 5, 600), 2), dtype)
    for x in (pool[0, :1, ::3], pool[0, 1:2, 1::2], pool[:, 2:3, ::3], pool[:, :, 7:8], pool[1, :, 5:6],
              pool[0, :1, ::3].mT, pool[:, 1:2, 1::2].mT):
        q, t = fgd.mx4_quantize_both(x)
        plain = x.contiguous()
        for got, want in ((q, fgd.mx4_quantize(plain)), (t, fgd.mx4_quantize(plain.mT.contiguous())),
                          (fgd.mx4_quantize(x), q), (fgd.mx4_quantize(x.mT), t)):
            assert got.shape == want.shape
            assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales)
    dy, x = pool[0, :1, ::3], pool[1, :1, 1::2]  # the gradients of one token
    w_t = fgd.mx4_quantize(_tensor(torch, _values((300, 200), 3), dtype))
    for got, want in zip(fgd.mx4_linear_grads(dy, x, w_t), fgd.mx4_linear_grads(dy.contiguous(), x.contiguous(), w_t)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("mnk", PRODUCTS + [(2100, 2100, 200), (1100, 17000, 385)], ids=str)
def test_products_whose_sums_are_exact(env, mnk):
    """Operands on the grid with scales of 1: products are multiples of 1/4 and
    sums of up to 9000 of them stay below 2^24 quarters, so that every order of
    float32 additions gives the exact result."""
    fgd, torch = env
    m, n, k = mnk
    print(f"[mx4] exact sums {mnk}", flush=True)

    def grid(rows, seed):
        rng = np.random.default_rng(seed)
        a = rng.choice(ref.GRID, (rows, k)) * rng.choice([-1.0, 1.0], (rows, k))
        for j in range(0, k, 32):  # one of the largest binade in every block
            a[np.arange(rows), j + rng.integers(0, min(32, k - j), rows)] = rng.choice([4.0, 6.0, -6.0], rows)
        return torch.from_numpy(a).cuda()

    x, w = grid(m, m + k), grid(n, n + k + 1)
    assert 36 * k * 4 < 2 ** 24
    want = x @ w.T.contiguous()
    w4 = fgd.mx4_quantize(w.float())
    assert torch.equal(fgd.mx4_linear(x.float(), w4).double(), want)
    assert torch.equal(fgd.mx4_matmul(fgd.mx4_quantize(x.float()), w4, "f32").double(), want)


@pytest.mark.parametrize("mnk", PRODUCTS + [(2100, 2100, 200), (1100, 17000, 385)], ids=str)
def test_products_within_their_instructions_rounding(env, mnk):
    """The matrix instruction sums 64 terms and adds them to what it holds: K /
    64 additions over the steps, 64 within one, and 8 of the waves' sums."""
    fgd, torch = env
    m, n, k = mnk
    print(f"[mx4] rounding {mnk}", flush=True)
    x, w = _tensor(torch, _values((m, k), m + k + 5), "f32"), _tensor(torch, _values((n, k), n + k + 6, 1.0), "f32")
    x4, w4 = fgd.mx4_quantize(x), fgd.mx4_quantize(w)
    p, q = fgd.mx4_dequantize(x4).double(), fgd.mx4_dequantize(w4).double().T.contiguous()
    off = (fgd.mx4_matmul(x4, w4, "f32").double() - p @ q).abs_()
    assert bool((off <= (k / 64 + 64 + 8) * 2.0 ** -24 * (p.abs() @ q.abs())).all())
