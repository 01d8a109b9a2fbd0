"""CPU tests of the operators' entry points: sizes, and every refusal before
anything is launched (no call here reaches a kernel)."""

import ctypes

import pytest
import torch

import paper_2606_22768_amd as fgd

BAD = fgd.FGD_ERR_INVALID_ARG
A = 1 << 20  # addresses far apart that nothing reads
B, C, D, E, F = (A + (i << 40) for i in range(1, 6))


def refused(call, text):
    with pytest.raises(fgd.FgdError, match=text) as e:
        call()
    assert e.value.status == BAD


@pytest.mark.parametrize("batch, rows, cols, tiles", [(1, 1, 1, 1), (1, 64, 128, 1), (1, 65, 128, 2), (1, 64, 129, 2),
                                                      (3, 130, 300, 27), (0, 5, 5, 0), (2, 0, 5, 0), (2, 5, 0, 0),
                                                      (1, 128_256, 8192, 128_256)])
def test_mx4_sizes(batch, rows, cols, tiles):
    assert fgd.fgd_mx4_size(batch, rows, cols) == (tiles * 4096, tiles * 256)
    assert fgd.fgd_mx4_linear_workspace_size(batch, rows, cols) == tiles * 4352


@pytest.mark.parametrize("sizes", [(-1, 1, 1), (1, -1, 1), (1, 1, -1), (1, 1 << 40, 1 << 40), (1 << 30, 1 << 30, 1 << 30)])
def test_mx4_size_refusals(sizes):
    refused(lambda: fgd.fgd_mx4_size(*sizes), "negative|too large")
    refused(lambda: fgd.fgd_mx4_linear_workspace_size(*sizes), "negative|too large")


def test_mx4_quantize_refusals():
    def q(x=A, dtype="f32", batch=2, rows=70, cols=130, bs=70 * 130, rs=130, cs=1, codes=B, scales=C):
        fgd.fgd_mx4_quantize(x, dtype, batch, rows, cols, bs, rs, cs, codes, scales, 0)

    refused(lambda: q(dtype=2), "dtype")
    refused(lambda: q(x=None), "NULL")
    refused(lambda: q(codes=None), "NULL")
    refused(lambda: q(scales=None), "NULL")
    refused(lambda: q(x=A + 2), "aligned")
    refused(lambda: q(x=A + 1, dtype="bf16"), "aligned")
    refused(lambda: q(codes=B + 8), "aligned")
    refused(lambda: q(scales=C + 4), "aligned")
    refused(lambda: q(rows=-1), "negative")
    refused(lambda: q(bs=-1), "negative")
    refused(lambda: q(rs=260, cs=2), "contiguous")
    refused(lambda: q(rs=1 << 59), "too large")
    refused(lambda: q(codes=A), "overlap")
    refused(lambda: q(scales=A + 4096), "overlap")
    refused(lambda: q(scales=B + 4096), "overlap")
    q(x=None, rows=0, codes=None, scales=None)  # nothing to do, nothing needed


def test_mx4_dequantize_refusals():
    def d(codes=A, scales=B, batch=2, rows=70, cols=130, out=C, dtype="f32", bs=70 * 130, rs=130):
        fgd.fgd_mx4_dequantize(codes, scales, batch, rows, cols, out, dtype, bs, rs, 0)

    refused(lambda: d(dtype=7), "dtype")
    refused(lambda: d(out=None), "NULL")
    refused(lambda: d(codes=None), "NULL")
    refused(lambda: d(codes=A + 8), "aligned")
    refused(lambda: d(out=C + 2), "aligned")
    refused(lambda: d(rs=129), "row_stride")
    refused(lambda: d(bs=70 * 130 - 1), "batch_stride")
    refused(lambda: d(out=A), "overlap")
    refused(lambda: d(out=B), "overlap")
    d(out=None, cols=0, codes=None, scales=None)


def test_mx4_matmul_refusals():
    def p(ac=A, as_=B, wc=C, ws=D, batch=2, m=70, n=100, k=200, out=E, dtype="f32", bs=7000, rs=100):
        fgd.fgd_mx4_matmul(ac, as_, wc, ws, batch, m, n, k, out, dtype, bs, rs, 0)

    refused(lambda: p(dtype=3), "dtype")
    for name in ("ac", "as_", "wc", "ws", "out"):
        refused(lambda: p(**{name: None}), "NULL")
    for name in ("ac", "as_", "wc", "ws"):
        refused(lambda: p(**{name: A + 8}), "aligned")
        refused(lambda: p(**{name: E}), "overlap")
    refused(lambda: p(out=E + 1), "aligned")
    refused(lambda: p(rs=99), "row_stride")
    refused(lambda: p(bs=6999), "batch_stride")
    refused(lambda: p(m=-1), "negative")
    refused(lambda: p(n=-1), "negative")
    p(m=0, ac=None, as_=None, out=None)
    p(batch=0, ac=None, as_=None, wc=None, ws=None, out=None)


def test_mx4_linear_refusals():
    need = fgd.fgd_mx4_linear_workspace_size(2, 70, 200)

    def f(x=A, dtype="bf16", xbs=14000, xrs=200, wc=B, ws=C, batch=2, t=70, n=100, k=200, out=D, odt="f32", bs=7000,
          rs=100, work=E, size=need):
        fgd.fgd_mx4_linear(x, dtype, xbs, xrs, wc, ws, batch, t, n, k, out, odt, bs, rs, work, size, 0)

    refused(lambda: f(dtype=3), "dtype")
    refused(lambda: f(odt=3), "dtype")
    for name in ("x", "wc", "ws", "out", "work"):
        refused(lambda: f(**{name: None}), "NULL")
    refused(lambda: f(work=E + 8), "aligned")
    refused(lambda: f(size=need - 1), "below")
    refused(lambda: f(work=A), "overlap")
    refused(lambda: f(work=B), "overlap")
    refused(lambda: f(work=D), "overlap")
    refused(lambda: f(out=A), "overlap")
    refused(lambda: f(out=B), "overlap")
    f(t=0, x=None, out=None, work=None, size=0)


def settings(**kw):
    return fgd.fgd_sampling(ctypes.sizeof(fgd.fgd_sampling), **kw)


def test_sample_refusals():
    need = fgd.fgd_sample_workspace_size("f32", 5, 1000)

    def s(z=A, dtype="f32", rows=5, vocab=1000, ld=1000, u=B, st=None, tok=C, prob=D, work=E, size=None):
        fgd.fgd_sample(z, dtype, rows, vocab, ld, u, settings() if st is None else st, tok, prob, work,
                       need if size is None else size, 0)

    refused(lambda: s(dtype=2), "dtype")
    refused(lambda: s(rows=-1), "num_rows")
    refused(lambda: s(rows=1 << 31), "num_rows")
    refused(lambda: s(vocab=0), "vocab")
    refused(lambda: s(vocab=fgd.FGD_MAX_SAMPLE_VOCAB + 1, ld=1 << 23), "vocab")
    refused(lambda: s(ld=999), "ldk")
    for name in ("z", "u", "tok"):
        refused(lambda: s(**{name: None}), "NULL")
        refused(lambda: s(**{name: A + 2}), "aligned")
    refused(lambda: s(prob=D + 1), "aligned")
    refused(lambda: s(z=A + 1, dtype="bf16"), "aligned")
    refused(lambda: s(work=E + 8), "aligned")
    refused(lambda: s(st=fgd.fgd_sampling(8)), "settings")
    refused(lambda: s(st=settings(reserved=1)), "reserved")
    refused(lambda: s(st=settings(top_k_rows=A + 1)), "aligned")
    refused(lambda: s(tok=A + 400), "overlap")
    refused(lambda: s(prob=B), "overlap")
    refused(lambda: s(prob=C), "overlap")
    refused(lambda: s(st=settings(top_p_rows=C)), "overlap")
    with pytest.raises(fgd.FgdError):
        fgd.fgd_sample(A, "f32", 5, 1000, 1000, B, None, C, D, E, need, 0)
    s(rows=0, z=None, u=None, tok=None, prob=None)


@pytest.mark.parametrize("sizes", [(2, 1, 10), ("f32", -1, 10), ("f32", 1, 0), ("f32", 1, 1 << 23)])
def test_sample_size_refusals(sizes):
    refused(lambda: fgd.fgd_sample_workspace_size(*sizes), "dtype|num_rows|vocab")


# ------------------------------------------------------------ tensor level

def fake(rows, cols, batch=None):
    c, s = fgd.fgd_mx4_size(batch or 1, rows, cols)
    return fgd.Mx4(torch.zeros(c, dtype=torch.uint8), torch.zeros(s, dtype=torch.uint8), batch, rows, cols)


def test_mx4_tensors_are_checked_before_any_launch():
    x = torch.zeros(4, 64)
    w = fake(10, 64)
    with pytest.raises(TypeError, match="torch tensor"):
        fgd.mx4_quantize([1.0])
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        fgd.mx4_quantize(x.double())
    with pytest.raises(ValueError, match="shape"):
        fgd.mx4_quantize(torch.zeros(4))
    with pytest.raises(ValueError, match="contiguous"):
        fgd.mx4_quantize(torch.zeros(8, 64)[::2, ::2])
    with pytest.raises(ValueError, match="GPU"):
        fgd.mx4_quantize(x)
    with pytest.raises(TypeError, match="Mx4"):
        fgd.mx4_dequantize(x)
    with pytest.raises(TypeError, match="dtype"):
        fgd.mx4_dequantize(w, "f16")
    with pytest.raises(TypeError, match="Mx4"):
        fgd.mx4_matmul(w, x)
    with pytest.raises(ValueError, match="share"):
        fgd.mx4_matmul(w, fake(10, 65))
    with pytest.raises(ValueError, match="share"):
        fgd.mx4_matmul(w, fake(10, 64, 2))
    with pytest.raises(ValueError, match="share"):
        fgd.mx4_linear(torch.zeros(4, 63), w)
    with pytest.raises(ValueError, match="contiguous"):
        fgd.mx4_linear(torch.zeros(64, 4).mT, w)
    with pytest.raises(ValueError, match="expected a tensor on"):
        fgd.mx4_linear(x, w.__class__(w.codes.to("meta"), w.scales, None, 10, 64))
    with pytest.raises(ValueError, match="shape"):
        fgd.mx4_dequantize(w, out=torch.zeros(10, 63))
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        fgd.mx4_dequantize(w, out=torch.zeros(10, 64, dtype=torch.float16))
    with pytest.raises(ValueError, match="expected a tensor on"):
        fgd.mx4_dequantize(w, out=torch.zeros(10, 64))
    with pytest.raises(TypeError, match="Mx4"):
        fgd.mx4_linear_grads(x, x, x)
    with pytest.raises(ValueError, match="x: expected shape"):
        fgd.mx4_linear_grads(torch.zeros(4, 10), torch.zeros(5, 64), fake(64, 10))


def test_sample_tensors_are_checked_before_any_launch():
    z, u = torch.zeros(3, 50), torch.zeros(3)
    for bad, error, text in ((dict(logits=[0.0]), TypeError, "torch tensor"),
                             (dict(logits=z.double()), TypeError, "float32 or bfloat16"),
                             (dict(logits=z[0]), ValueError, "shape"),
                             (dict(logits=torch.zeros(50, 3).mT), ValueError, "contiguous"),
                             (dict(logits=z[:1].expand(3, 50)), ValueError, "overlap"),
                             (dict(vocab=51), ValueError, "vocab"),
                             (dict(uniform=u.double()), TypeError, "float32"),
                             (dict(uniform=u[:2]), ValueError, "shape"),
                             (dict(uniform=torch.zeros(6)[::2]), ValueError, "contiguous"),
                             (dict(uniform=0.5), TypeError, "torch tensor"),
                             (dict(temperature=torch.zeros(2)), ValueError, "temperature"),
                             (dict(top_k=torch.zeros(3)), TypeError, "int32"),
                             (dict(top_p=torch.zeros(3, 1)), ValueError, "top_p"),
                             (dict(min_p=torch.zeros(3, dtype=torch.int32)), TypeError, "min_p"),
                             (dict(tokens_out=torch.zeros(3)), TypeError, "int32"),
                             (dict(probs_out=torch.zeros(4)), ValueError, "probs_out"),
                             (dict(), ValueError, "GPU")):
        args = {"logits": z, "uniform": u, **bad}
        with pytest.raises(error, match=text):
            fgd.sample(**args)


def test_gradients_check_a_kept_transpose():
    import torch

    import paper_2606_22768_amd as fgd

    def packed(rows, cols):
        c, n = fgd.fgd_mx4_size(1, rows, cols)
        return fgd.Mx4(torch.zeros(c, dtype=torch.uint8), torch.zeros(n, dtype=torch.uint8), None, rows, cols)

    with pytest.raises(ValueError, match="rows of its transpose"):
        fgd.mx4_linear_grads(torch.zeros(8, 16), packed(40, 8), packed(32, 16))


def test_quantising_both_axes_checks_its_arrays():
    import paper_2606_22768_amd as fgd

    at = [1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20]  # never touched: every call is refused

    def call(arrays=at, dtype="f32", rows=64, cols=128, row_stride=128):
        fgd.fgd_mx4_quantize_both(arrays[0], dtype, 1, rows, cols, 0, row_stride, *arrays[1:], stream=0)

    for i in range(5):
        with pytest.raises(fgd.FgdError, match="NULL"):
            call(at[:i] + [None] + at[i + 1:])
        for j in range(i):
            with pytest.raises(fgd.FgdError, match="overlap"):
                call(at[:i] + [at[j]] + at[i + 1:])
    for i in range(1, 5):
        with pytest.raises(fgd.FgdError, match="aligned"):
            call(at[:i] + [at[i] + 8] + at[i + 1:])
    with pytest.raises(fgd.FgdError, match="aligned to its element"):
        call([at[0] + 1] + at[1:])
    with pytest.raises(fgd.FgdError, match="dtype"):
        call(dtype=7)
    with pytest.raises(fgd.FgdError, match="negative"):
        call(rows=-1)
    with pytest.raises(fgd.FgdError, match="negative stride"):
        call(row_stride=-128)


def test_mx4_linear_grads_refusals():
    need = fgd.fgd_mx4_linear_grads_workspace_size(2, 70, 100, 200)
    assert need == fgd.fgd_mx4_linear_workspace_size(2, 70, 100) + fgd.fgd_mx4_linear_workspace_size(2, 100, 70) + \
        fgd.fgd_mx4_linear_workspace_size(2, 200, 70)
    at = [i << 24 for i in range(1, 8)]

    def f(dy=at[0], dt="bf16", dyrs=100, x=at[1], xt="f32", xrs=200, wc=at[2], ws=at[3], batch=2, t=70, n=100, k=200,
          dx=at[4], dxt="bf16", dxrs=200, dw=at[5], dwt="f32", dwrs=200, dwbs=20000, work=at[6], size=need):
        fgd.fgd_mx4_linear_grads(dy, dt, 7000, dyrs, x, xt, 14000, xrs, wc, ws, batch, t, n, k, dx, dxt, 14000, dxrs,
                                 dw, dwt, dwbs, dwrs, work, size, 0)

    for name in ("dt", "xt", "dxt", "dwt"):
        refused(lambda: f(**{name: 3}), "dtype")
    names = ("dy", "x", "wc", "ws", "dx", "dw", "work")
    for name in names:
        refused(lambda: f(**{name: None}), "NULL")
    for name in ("wc", "ws", "work"):
        refused(lambda: f(**{name: at[names.index(name)] + 8}), "aligned")
    for out in ("dx", "dw", "work"):
        for i, name in enumerate(names):
            if name != out:
                refused(lambda: f(**{out: at[i]}), "overlap")
    for name in ("dyrs", "xrs"):
        refused(lambda: f(**{name: -1}), "negative")
    for name in ("batch", "t", "n", "k"):
        refused(lambda: f(**{name: -1}), "negative")
        refused(lambda: fgd.fgd_mx4_linear_grads_workspace_size(*(-1 if v == name else 2
                                                                  for v in ("batch", "t", "n", "k"))), "negative")
    refused(lambda: f(dxrs=199), "row_stride")
    refused(lambda: f(dwrs=199), "row_stride")
    refused(lambda: f(dwbs=19999), "batch_stride")
    refused(lambda: f(size=need - 1), "below")
    f(batch=0, dy=None, x=None, wc=None, ws=None, dx=None, dw=None, work=None, size=0)


def test_an_empty_batch_may_have_any_strides():
    fgd.fgd_mx4_quantize(None, "f32", 0, 4, 5, 0, 0, 0, None, None, 0)
    fgd.fgd_mx4_quantize(None, "f32", 0, 4, 5, 7, 9, 3, None, None, 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_refuses_spans_past_every_address(dtype):
    """(num_rows - 1) * ldk elements in full: neither a wrapped nor a negative
    span may hide an overlap."""
    def s(rows, ld, tok=C):
        fgd.fgd_sample(A, dtype, rows, 1000, ld, B, settings(), tok, D, E, 1 << 40, 0)

    for rows, ld in (((1 << 31) - 1, 1 << 40), ((1 << 23) + 1, 1 << 40), ((1 << 22) + 1, 1 << 40),
                     ((1 << 31) - 1, 1 << 33)):
        refused(lambda: s(rows, ld), "too large")
    refused(lambda: s(1 << 20, 1 << 36, A + (1 << 50)), "overlap")  # in range: the tokens lie among the rows


def test_kept_codes_and_scales_are_checked():
    """The kernels read what the sizes say: arrays that are shorter, of
    another type, strided or apart are refused where they become a matrix."""
    c, s = fgd.fgd_mx4_size(2, 70, 200)
    codes, scales = torch.zeros(c, dtype=torch.uint8), torch.zeros(s, dtype=torch.uint8)
    q = fgd.Mx4(codes, scales, 2, 70, 200)
    assert q.shape == (2, 70, 200) and q.nbytes == c + s and q.codes is codes and q.scales is scales
    assert fgd.Mx4(codes[:c // 2], scales[:s // 2], None, 70, 200).shape == (70, 200)
    for args, error, text in (((codes[:-1], scales), ValueError, "codes: expected"),
                              ((codes, scales[1:]), ValueError, "scales: expected"),
                              ((scales, codes), ValueError, "codes: expected"),
                              ((codes.char(), scales), TypeError, "codes: expected uint8"),
                              ((codes, scales.float()), TypeError, "scales: expected uint8"),
                              ((None, scales), TypeError, "codes: expected a torch tensor"),
                              ((codes, b"0" * s), TypeError, "scales: expected a torch tensor"),
                              ((torch.zeros(2 * c, dtype=torch.uint8)[::2], scales), ValueError, "contiguous"),
                              ((codes, scales.to("meta")), ValueError, "scales: expected a tensor on cpu")):
        with pytest.raises(error, match=text):
            fgd.Mx4(*args, 2, 70, 200)
    for sizes in ((3, 70, 200), (2, 129, 200), (2, 70, 257), (None, 70, 200)):
        with pytest.raises(ValueError, match="codes: expected"):
            fgd.Mx4(codes, scales, *sizes)
    with pytest.raises(fgd.FgdError, match="negative"):
        fgd.Mx4(codes, scales, 2, -70, 200)


def test_a_batch_past_32_bits_is_refused():
    """A broadcast tensor can have one; its lower bits must not stand for it."""
    for n in (1 << 31, (1 << 32) + 1):
        with pytest.raises(ValueError, match="batch"):
            fgd.fgd_mx4_size(n, 1, 1)
        with pytest.raises(ValueError, match="batch"):
            fgd.Mx4(torch.zeros(4096, dtype=torch.uint8), torch.zeros(256, dtype=torch.uint8), n, 1, 1)
    assert fgd.fgd_mx4_size((1 << 31) - 1, 1, 1) == (((1 << 31) - 1) * 4096, ((1 << 31) - 1) * 256)


def test_sampled_rows_are_split_where_that_pays():
    """Only rows that are split over blocks need a workspace: those that
    measure faster so, not those that a block each takes in less time."""
    size = fgd.fgd_sample_workspace_size
    for rows, vocab in ((1, 16384), (4, 16384), (64, 24000), (64, 32000), (85, 32000), (128, 33000), (128, 40000),
                        (129, 128256), (2048, 128256), (0, 128256)):
        assert size("f32", rows, vocab) == 0, (rows, vocab)
    for rows, vocab in ((1, 32000), (1, 128256), (16, 32000), (16, 50257), (64, 50257), (64, 128256), (128, 80000),
                        (128, 128256)):
        assert size("f32", rows, vocab) > 0, (rows, vocab)
