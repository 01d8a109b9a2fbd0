"""CPU tests of the entry points of heads, caches, attention and pages: sizes,
and every refusal before anything is launched (no call here reaches a
kernel)."""

import numpy as np
import pytest
import torch

import paper_2606_22768_amd as fgd

BAD = fgd.FGD_ERR_INVALID_ARG
A = 1 << 20  # addresses far apart that nothing reads
B, C, D, E, F, G, H, I, J, K = (A + (i << 40) for i in range(1, 11))


def refused(call, text):
    with pytest.raises(fgd.FgdError, match=text) as e:
        call()
    assert e.value.status == BAD


# ------------------------------------------------------------------ heads

def sizes(**kw):
    return fgd.fgd_heads(**{**dict(dtype="f32", batch=2, q_heads=4, k_heads=2, head_dim=64, rot_dim=64, tokens=10,
                                   eps=1e-6), **kw})


SQ, SK = (2560, 256, 64), (1280, 128, 64)


def rotate(s=None, q=A, qs=SQ, k=B, ks=SK, positions=C, freqs=D, wq=E, wk=F, qo=G, qos=SQ, ko=H, kos=SK, **kw):
    fgd.fgd_rotate_heads(sizes(**kw) if s is None else s, q, qs, k, ks, positions, freqs, wq, wk, qo, qos, ko, kos, 0)


def grads(dq=A, dk=B, q=I, k=J, positions=C, freqs=D, wq=E, wk=F, gq=G, gk=H, gwq=K, gwk=K + (1 << 20), work=K + (1 << 30),
          n=1 << 24, gqs=SQ, gks=SK, **kw):
    fgd.fgd_rotate_heads_grads(sizes(**kw), dq, SQ, dk, SK, q, SQ, k, SK, positions, freqs, wq, wk, gq, gqs, gk, gks, gwq,
                               gwk, work, n, 0)


@pytest.mark.parametrize("kw, text", [
    (dict(dtype=2), "dtype"), (dict(weight_dtype=5), "dtype"), (dict(batch=-1), "negative"),
    (dict(tokens=-1), "negative"), (dict(q_heads=-1), "negative"), (dict(head_dim=63), "even"),
    (dict(head_dim=0), "even"), (dict(head_dim=514), "even"), (dict(rot_dim=66), "rot_dim"),
    (dict(rot_dim=3), "rot_dim"), (dict(rot_dim=-2), "rot_dim"), (dict(interleaved=2), "interleaved"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(position_stride=9), "position_stride"), (dict(weight_stride=63), "weight_stride"),
    (dict(q_heads=60_000, k_heads=6000), "too large"), (dict(tokens=1 << 55), "too large"),
    (dict(position_stride=1 << 60), "too large"), (dict(weight_stride=1 << 60), "too large")])
def test_heads_sizes(kw, text):
    refused(lambda: rotate(**kw), text)
    refused(lambda: grads(**kw), text)
    refused(lambda: fgd.fgd_rotate_heads_grads_workspace_size(sizes(**kw)), text)


def test_heads_arrays():
    s = sizes()
    s.struct_size -= 4
    refused(lambda: rotate(s), "another size")
    for name in ("q", "k", "qo", "ko", "positions", "freqs"):
        refused(lambda: rotate(**{name: None}), "NULL")
    for name in ("qs", "ks", "qos", "kos"):
        refused(lambda: rotate(**{name: None}), "NULL strides")
    for name in ("q", "k", "qo", "ko", "wq", "wk", "positions", "freqs"):
        refused(lambda: rotate(**{name: A + (15 << 41) + 2}), "aligned")
    refused(lambda: rotate(qs=(2560, -256, 64)), "negative stride")
    refused(lambda: rotate(qs=(2560, 1 << 59, 64)), "too large")
    refused(lambda: rotate(qos=(2560, 255, 64)), "elements overlap")
    refused(lambda: rotate(qos=(2559, 256, 64)), "elements overlap")
    refused(lambda: rotate(qos=(0, 256, 64)), "elements overlap")
    refused(lambda: rotate(qo=A + 64), "overlap")
    refused(lambda: rotate(qo=A, qos=(2560, 64, 640)), "overlap")  # in place means the same strides
    refused(lambda: rotate(ko=A), "overlap")
    refused(lambda: rotate(ko=G), "overlap")
    refused(lambda: rotate(qo=E), "overlap")
    refused(lambda: rotate(qo=A, positions=A + 256), "overlap")
    refused(lambda: rotate(qo=A, ks=SQ, k=A, k_heads=4, kos=SQ), "share elements")
    rotate(q=None, k=None, qo=None, ko=None, positions=None, freqs=None, tokens=0)
    rotate(q=None, qs=None, k=None, ks=None, qo=None, qos=None, ko=None, kos=None, q_heads=0, k_heads=0)


@pytest.mark.parametrize("qh, kh, at, strides, batch, tokens, text", [
    (4, 2, 256, (3840, 384, 64), 2, 10, None), (4, 2, 255, (3840, 384, 64), 2, 10, "share elements"),
    (4, 2, 193, (3840, 384, 64), 2, 10, "share elements"), (4, 2, 0, (3840, 384, 64), 2, 10, "share elements"),
    (4, 4, 64, (5120, 512, 128), 2, 10, None), (4, 4, 65, (5120, 512, 128), 2, 10, "share elements"),
    (4, 2, 256 + 384, (3840, 384, 64), 2, 10, None), (4, 2, 257 + 384, (3840, 384, 64), 2, 10, "share elements"),
    (4, 2, 256 + 3840, (7680, 384, 64), 2, 10, None), (4, 2, 320 - 384, (3840, 384, 64), 2, 10, "share elements"),
    (2, 3, 1280, (3200, 64, 640), 2, 10, None), (2, 3, 1279, (3200, 64, 640), 2, 10, "share elements"),
    (2, 1, 256, (192, 384, 64), 2, 10, "share elements"), (2, 1, 128, (192, 384, 64), 2, 10, None),
    (1, 1, 64, (128, 128, 64), 1, 10, None), (1, 1, 32, (128, 128, 64), 1, 10, "share elements")])
def test_heads_in_place_apart(qh, kh, at, strides, batch, tokens, text):
    # k begins `at` elements after q: by hand, which elements the two have.
    def elements(first, heads):
        return {first + b * strides[0] + t * strides[1] + h * strides[2] + d
                for b in range(batch) for t in range(tokens) for h in range(heads) for d in range(64)}
    assert bool(elements(0, qh) & elements(at, kh)) == (text is not None)
    # The positions refuse what passes the check, so that nothing is launched.
    refused(lambda: rotate(q=B, qo=B, k=B + 4 * at, ko=B + 4 * at, qs=strides, qos=strides, ks=strides, kos=strides,
                           q_heads=qh, k_heads=kh, batch=batch, tokens=tokens, positions=B + 64), text or "inputs")
    refused(lambda: rotate(q=B, qo=B, k=B + 4 * at, ko=H, qs=strides, qos=strides, ks=strides, kos=(1 << 20, 1 << 14, 64),
                           q_heads=qh, k_heads=kh, batch=batch, tokens=tokens, positions=B + 64), text or "inputs")


@pytest.mark.parametrize("at, apart", [(256, True), (255, False), (257, False), (0, False), (320, False), (256 + 384, True),
                                       (-128, True), (-127, False), (256 + 3840, True)])
def test_gradients_between_each_other(at, apart):
    # Gradients of 4 and 2 heads of 64 as views of one array of 6: their spans meet, their elements do or do not.
    s = (3840, 384, 64)
    q = {b * 3840 + t * 384 + d for b in range(2) for t in range(10) for d in range(256)}
    k = {at + b * 3840 + t * 384 + d for b in range(2) for t in range(10) for d in range(128)}
    assert bool(q & k) != apart
    # A weight's gradient in place of a weight refuses what passes, so that nothing is launched.
    refused(lambda: grads(gq=G, gk=G + 4 * at, gqs=s, gks=s, gwq=E), "the inputs" if apart else "each other")
    refused(lambda: grads(gq=G, gk=G + 4 * at, gqs=s, gks=s, positions=G + 64), "the inputs")
    # Of other strides they count as meeting where their spans do.
    if abs(at) < 3840:
        refused(lambda: grads(gq=G, gk=G + 4 * at, gqs=s, gks=(3840, 384, 128), gwq=E), "each other")
    refused(lambda: rotate(qo=G, ko=G + 4 * at, qos=s, kos=s, positions=G + 64), "the inputs")
    if not apart:
        refused(lambda: rotate(qo=G, ko=G + 4 * at, qos=s, kos=s), "each other")


def test_heads_in_place_strides():
    refused(lambda: rotate(q=B, qo=B, k=B + 1024, ko=B + 1024, qs=(3840, 384, 64), qos=(3840, 384, 64),
                           ks=(3840, 192, 64), kos=(3840, 192, 64)), "share elements")
    refused(lambda: rotate(q=A, qo=A, positions=A), "inputs")


def test_heads_gradients():
    for name in ("dq", "dk", "q", "k", "gq", "gk"):
        refused(lambda: grads(**{name: None}), "NULL")
    refused(lambda: grads(gwq=None), "together")
    refused(lambda: grads(wk=None), "together")
    refused(lambda: grads(gwk=K + (1 << 20) + 2), "aligned")
    refused(lambda: grads(work=K + (1 << 30) + 8), "aligned")
    refused(lambda: grads(n=100), "workspace")
    refused(lambda: grads(work=None), "workspace")
    refused(lambda: grads(gq=A), "overlap")
    refused(lambda: grads(gk=J), "overlap")
    refused(lambda: grads(gwq=E), "overlap")
    refused(lambda: grads(gwk=K), "overlap")
    refused(lambda: grads(work=A), "overlap")
    refused(lambda: grads(gqs=(2560, 64, 64)), "elements overlap")
    assert fgd.fgd_rotate_heads_grads_workspace_size(sizes(batch=0)) == 0
    assert fgd.fgd_rotate_heads_grads_workspace_size(sizes(tokens=1 << 20)) <= 1024 * 2 * 64 * 4
    refused(lambda: fgd._check(fgd.lib.fgd_rotate_heads_grads_workspace_size(None, None), "x"), "NULL")


def test_rotate_heads_tensors():
    q, k = torch.zeros(5, 4, 64), torch.zeros(5, 2, 64)
    p, f, w = torch.zeros(5, dtype=torch.int32), torch.ones(32, dtype=torch.float64), torch.ones(64)
    run = lambda q=q, k=k, p=p, f=f, wq=w, wk=w, **kw: fgd.rotate_heads(q, k, p, f, wq, wk, **kw)  # noqa: E731
    for bad, error, text in [
            (dict(q=None), TypeError, "q: expected a torch"), (dict(q=q.half()), TypeError, "float32 or bfloat16"),
            (dict(q=q[0]), ValueError, "tokens"), (dict(q=q[..., ::2]), ValueError, "contiguous"),
            (dict(k=k.bfloat16()), TypeError, "k: expected"), (dict(k=k[:3]), ValueError, "k: expected shape"),
            (dict(k=k[..., :32]), ValueError, "k: expected shape"), (dict(k=None), ValueError, "no keys"),
            (dict(p=p.long()), TypeError, "positions"), (dict(p=p[:3]), ValueError, "positions"),
            (dict(p=None), TypeError, "positions"), (dict(f=f.float()), TypeError, "freqs"),
            (dict(f=f[None]), ValueError, "freqs"), (dict(wq=w[:3]), ValueError, "q_weight"),
            (dict(wq=w.half()), TypeError, "q_weight"), (dict(wq=w.bfloat16()), ValueError, "one type"),
            (dict(wk=w[None]), ValueError, "k_weight"), (dict(), ValueError, "on a GPU")]:
        with pytest.raises(error, match=text):
            run(**bad)
    with pytest.raises(fgd.FgdError, match="rot_dim"):
        fgd.rotate_heads_grads(q, k, q, k, p, torch.ones(33, dtype=torch.float64), w, w)
    with pytest.raises(TypeError, match="q: expected"):
        fgd.rotate_heads_grads(q, k, None, k, p, f, w, w)
    with pytest.raises(ValueError, match="k: expected shape"):
        fgd.rotate_heads_grads(q, k, q, q, p, f, w, w)
    with pytest.raises(ValueError, match="workspace"):
        fgd.rotate_heads_grads(q, k, q, k, p, f, w, w, workspace=torch.empty(5, dtype=torch.uint8))


# ------------------------------------------------------------------ cache

def cache(page=64, heads=2, head_dim=64, pages=10, data=A):
    return fgd.fgd_mx4_cache(page, heads, head_dim, pages, data)


@pytest.mark.parametrize("kw, size", [(dict(), 10 * 2 * 4 * 17 * 64), (dict(pages=0), 0),
                                      (dict(page=16, heads=1, head_dim=32, pages=3), 3 * 17 * 32),
                                      (dict(page=256, heads=8, head_dim=256, pages=10 ** 6), 10 ** 6 * 8 * 16 * 17 * 256)])
def test_cache_sizes(kw, size):
    assert fgd.fgd_mx4_cache_size(cache(**kw)) == size


def attention(**kw):
    return fgd.fgd_attention(**{**dict(dtype="f32", sequences=3, table_width=4, q_heads=8, tokens=3, most_queries=1,
                                       scale=0.1), **kw})


def attend(c=None, s=None, q=B, qt=512, qh=64, tables=C, ts=4, lengths=D, starts=E, out=F, ot=512, oh=64, work=G,
           n=1 << 30, **kw):
    fgd.fgd_mx4_attend(cache() if c is None else c, attention(**kw) if s is None else s, q, qt, qh, tables, ts, lengths,
                       starts, out, ot, oh, work, n, 0)


def write(c=None, k=B, kt=128, kh=64, v=C, vt=128, vh=64, dtype="f32", tokens=7, slots=D):
    fgd.fgd_mx4_cache_write(cache() if c is None else c, k, kt, kh, v, vt, vh, dtype, tokens, slots, 0)


def read(c=None, k=B, kt=128, kh=64, v=C, vt=128, vh=64, dtype="f32", tokens=7, slots=D):
    fgd.fgd_mx4_cache_read(cache() if c is None else c, slots, tokens, k, kt, kh, v, vt, vh, dtype, 0)


@pytest.mark.parametrize("kw, text", [
    (dict(page=8), "page"), (dict(page=48), "page"), (dict(page=1 << 17), "page"), (dict(heads=0), "heads"),
    (dict(heads=70_000), "heads"), (dict(head_dim=48), "head_dim"), (dict(head_dim=0), "head_dim"),
    (dict(head_dim=288), "head_dim"), (dict(pages=-1), "negative"), (dict(pages=1 << 31), "too large"),
    (dict(pages=(1 << 31) - 1, page=65536, heads=60_000), "too large")])
def test_cache_refusals(kw, text):
    c = cache(**kw)
    for call in (lambda: fgd.fgd_mx4_cache_size(c), lambda: write(c), lambda: read(c), lambda: attend(c),
                 lambda: fgd.fgd_mx4_attend_workspace_size(c, attention())):
        refused(call, text)


def test_write_and_read_refusals():
    c = cache()
    c.struct_size += 8
    r = cache()
    r.reserved = 1
    for call in (write, read):
        refused(lambda: call(c), "another size")
        refused(lambda: call(r), "reserved")
        refused(lambda: call(cache(data=None)), "NULL")
        refused(lambda: call(cache(data=A + 8)), "aligned")
        for name in ("k", "v", "slots"):
            refused(lambda: call(**{name: None}), "NULL")
        refused(lambda: call(k=B + 2), "aligned")
        refused(lambda: call(slots=D + 4), "aligned")
        refused(lambda: call(dtype=9), "dtype")
        refused(lambda: call(tokens=-1), "tokens")
        refused(lambda: call(tokens=1 << 31), "tokens")
        refused(lambda: call(kt=-128), "negative stride")
        refused(lambda: call(vh=1 << 59), "too large")
        for name in ("k", "v", "slots"):
            refused(lambda: call(**{name: A + 4096}), "overlap")
        call(tokens=0, k=None, v=None, slots=None)
    refused(lambda: read(kt=100), "elements overlap")
    refused(lambda: read(v=B + 64), "overlap")
    refused(lambda: read(slots=B), "overlap")
    write(cache(pages=0, data=None))


@pytest.mark.parametrize("most", [1 << 20, (1 << 31) - 1, 1 << 31, (1 << 32) + 1, (1 << 63) - 1])
def test_most_queries_above_the_tokens(most):
    # No sequence has more queries than there are: the same launch, so the same workspace.
    def size(n):
        return fgd.fgd_mx4_attend_workspace_size(cache(), attention(most_queries=n, table_width=4096, tokens=40, sequences=300))
    assert size(40) != size(1)  # rows of 40 queries go another way than those of one
    assert size(most) == size(40)


def test_attend_refusals():
    s = attention()
    s.struct_size = 0
    refused(lambda: attend(s=s), "another size")
    s = attention()
    s.reserved = 3
    refused(lambda: attend(s=s), "reserved")
    for kw, text in [(dict(dtype=4), "dtype"), (dict(tokens=-1), "tokens"), (dict(sequences=-1), "negative"),
                     (dict(table_width=-1), "negative"), (dict(q_heads=3), "multiple"), (dict(q_heads=0), "multiple"),
                     (dict(q_heads=65_536), "multiple"), (dict(most_queries=-1), "most_queries"),
                     (dict(window=-1), "window"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"),
                     (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"),
                     (dict(table_width=1 << 25), "at most 2\\^31"), (dict(tokens=1 << 28), "at most 2\\^31")]:
        refused(lambda: attend(**kw), text)
        refused(lambda: fgd.fgd_mx4_attend_workspace_size(cache(), attention(**kw)), text)
    refused(lambda: attend(cache(pages=0)), "width 0")
    refused(lambda: attend(cache(data=None)), "NULL")
    for name in ("q", "tables", "lengths", "out"):
        refused(lambda: attend(**{name: None}), "NULL")
        refused(lambda: attend(**{name: A + (15 << 41) + 2}), "aligned")
    refused(lambda: attend(starts=E + 1), "aligned")
    refused(lambda: attend(starts=None, tokens=4), "one query per sequence")
    refused(lambda: attend(ts=3), "table_stride")
    refused(lambda: attend(ts=1 << 60), "too large")
    refused(lambda: attend(qt=-1), "negative stride")
    refused(lambda: attend(ot=500), "elements overlap")
    refused(lambda: attend(work=G + 8), "16-byte")
    need = fgd.fgd_mx4_attend_workspace_size(cache(pages=9000), attention(table_width=2000))
    assert need > 0
    refused(lambda: attend(cache(pages=9000), table_width=2000, ts=2000, n=need - 1), "workspace")
    refused(lambda: attend(cache(pages=9000), table_width=2000, ts=2000, n=need, work=None), "workspace")
    for at in (A + 4096, B, C, D, E):
        refused(lambda: attend(out=at), "overlap")
        refused(lambda: attend(cache(pages=9000), table_width=2000, ts=2000, work=at), "overlap")
    refused(lambda: attend(cache(pages=9000), table_width=2000, ts=2000, work=F), "overlap")
    attend(tokens=0, q=None, out=None, work=None, n=1 << 20)
    attend(sequences=0, tokens=0, q=None, out=None, tables=None, lengths=None, work=None, n=1 << 20)


def test_cache_tensors():
    with pytest.raises(ValueError, match="pages"):
        fgd.Mx4Cache(1 << 31, 16, 1, 32, device="cpu")
    with pytest.raises(ValueError, match="page:"):
        fgd.Mx4Cache(1, 1 << 33, 1, 32, device="cpu")
    with pytest.raises(fgd.FgdError, match="head_dim"):
        fgd.Mx4Cache(1, 16, 1, 40, device="cpu")
    with pytest.raises(ValueError, match="data: expected 544 bytes"):
        fgd.Mx4Cache(1, 16, 1, 32, data=torch.zeros(543, dtype=torch.uint8))
    with pytest.raises(TypeError, match="data"):
        fgd.Mx4Cache(1, 16, 1, 32, data=torch.zeros(544, dtype=torch.int8))
    c = fgd.Mx4Cache(3, 16, 2, 64, device="cpu")
    assert c.nbytes == 3 * 2 * 17 * 64 and "pages=3" in repr(c)
    k, s = torch.zeros(5, 2, 64), torch.zeros(5, dtype=torch.int64)
    ints = lambda *a: torch.zeros(a, dtype=torch.int32)  # noqa: E731
    put = lambda k=k, v=k, s=s, c=c: fgd.mx4_cache_write(c, k, v, s)  # noqa: E731
    for bad, error, text in [
            (dict(c=k), TypeError, "Mx4Cache"), (dict(k=None), TypeError, "k: expected a torch"),
            (dict(k=k.half()), TypeError, "float32 or bfloat16"), (dict(k=k[0]), ValueError, "k: expected"),
            (dict(k=k[None]), ValueError, "k: expected"), (dict(k=k[..., :32], v=k[..., :32]), ValueError, "64 elements"),
            (dict(k=k[:, :1]), ValueError, "2 heads"), (dict(v=k[:, :1]), ValueError, "2 heads"),
            (dict(v=k.bfloat16()), TypeError, "v: expected"), (dict(v=k[:4]), ValueError, "v: expected"),
            (dict(), ValueError, "on a GPU")]:
        with pytest.raises(error, match=text):
            put(**bad)
    with pytest.raises(TypeError, match="dtype"):
        fgd.mx4_cache_read(c, s, "f16")
    with pytest.raises(TypeError, match="slots"):
        fgd.mx4_cache_read(c, s.int())
    with pytest.raises(ValueError, match="slots"):
        fgd.mx4_cache_read(c, s[None])
    with pytest.raises(ValueError, match="on a GPU"):
        fgd.mx4_cache_read(c, s)
    q = torch.zeros(3, 4, 64)
    run = lambda q=q, c=c, t=ints(3, 2), n=ints(3), starts=None, **kw: fgd.mx4_attend(q, c, t, n, starts, **kw)  # noqa: E731
    for bad, error, text in [
            (dict(q=torch.zeros(3, 3, 64)), ValueError, "multiple of 2"), (dict(q=q[:, :0]), ValueError, "multiple"),
            (dict(q=q[..., :32]), ValueError, "64 elements"), (dict(t=None), TypeError, "tables"),
            (dict(t=ints(3, 2).long()), TypeError, "tables"), (dict(t=ints(3)), ValueError, "tables"),
            (dict(t=ints(3, 4)[:, ::2]), ValueError, "contiguous"),
            (dict(t=ints(1, 2).expand(3, 2)), ValueError, "overlap"), (dict(n=ints(4)), ValueError, "lengths"),
            (dict(n=ints(3).long()), TypeError, "lengths"), (dict(starts=ints(3)), ValueError, "starts"),
            (dict(q=torch.zeros(4, 4, 64)), ValueError, "several need starts"),
            (dict(out=torch.zeros(3, 2, 64)), ValueError, "out: expected"),
            (dict(out=q.bfloat16()), TypeError, "out: expected"), (dict(), ValueError, "on a GPU")]:
        with pytest.raises(error, match=text):
            run(**bad)


def test_cache_of_given_data_on_a_named_device():
    data = torch.zeros(544, dtype=torch.uint8)
    for device in (None, "cpu", data.device):
        c = fgd.Mx4Cache(1, 16, 1, 32, device=device, data=data)
        assert c.data is data and c.device == data.device
    for device in ("meta", "cuda", "cuda:0"):
        with pytest.raises(ValueError, match="data: expected a tensor on"):
            fgd.Mx4Cache(1, 16, 1, 32, device=device, data=data)


BROKEN = [0.5, 2.9, 16.7, float("nan"), float("inf")]


@pytest.mark.parametrize("bad", BROKEN)
def test_sizes_that_are_no_whole_numbers(bad):
    for at in range(4):
        with pytest.raises(ValueError, match="whole number"):
            fgd.Mx4Cache(*(bad if i == at else 32 for i in range(4)), device="cpu")
    c = fgd.Mx4Cache(3, 16, 2, 64, device="cpu")
    q, t, n = torch.zeros(3, 4, 64), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    starts = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="window: expected a whole number"):
        fgd.mx4_attend(q, c, t, n, window=bad)
    with pytest.raises(ValueError, match="max_q: expected a whole number"):
        fgd.mx4_attend(q, c, t, n, starts, max_q=bad)
    free, count = torch.zeros(9, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="page: expected a whole number"):
        fgd.extend_pages(t, n, n, free, count, bad, 5)
    with pytest.raises(ValueError, match="tokens: expected a whole number"):
        fgd.extend_pages(t, n, n, free, count, 16, bad)
    with pytest.raises(ValueError, match="page: expected a whole number"):
        fgd.truncate_pages(t, n, n, free, count, bad)


def test_whole_numbers_of_other_types():
    for kind in (float, np.int64, np.float32, torch.tensor):
        c = fgd.Mx4Cache(*map(kind, (3, 16, 2, 64)), device="cpu")
        assert (c.pages, c.page, c.heads, c.dim) == (3, 16, 2, 64) and type(c.pages) is int
        q, t, n = torch.zeros(3, 4, 64), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
        for window in (5, 2 ** 40):  # the checks after that of the window refuse what is not on a GPU
            with pytest.raises(ValueError, match="on a GPU"):
                fgd.mx4_attend(q, c, t, n, window=kind(window))
        with pytest.raises(ValueError, match="window"):
            fgd.mx4_attend(q, c, t, n, window=kind(-1))


# ------------------------------------------------------------------ pages

def pages(page=16, requests=3, table_width=4, table_stride=4, tables=A, lengths=B, free=C, free_count=D, capacity=9):
    return fgd.fgd_pages(page, requests, table_width, table_stride, tables, lengths, free, free_count, capacity)


def extend(p=None, counts=E, tokens=20, starts=F, positions=G, slots=H):
    fgd.fgd_extend_pages(pages() if p is None else p, counts, tokens, starts, positions, slots, 0)


@pytest.mark.parametrize("requests, width", [(1 << 11, 1 << 20), (2, 1 << 30), ((1 << 31) - 1, 2)])
def test_tables_past_2_to_31_entries(requests, width):
    p = pages(requests=requests, table_width=width, table_stride=width, page=1, tables=A, lengths=A + (1 << 44),
              free=A + (1 << 45), free_count=A + (1 << 46))
    refused(lambda: extend(p), "too large")
    refused(lambda: fgd.fgd_truncate_pages(p, A + (1 << 47), 0), "too large")


def test_pages_refusals():
    for call in (extend, lambda p: fgd.fgd_truncate_pages(p, E, 0)):
        p = pages()
        p.struct_size = 1
        refused(lambda: call(p), "another size")
        p = pages()
        p.reserved = 1
        refused(lambda: call(p), "reserved")
        for kw, text in [(dict(requests=-1), "negative"), (dict(table_width=-1), "negative"),
                         (dict(capacity=-1), "negative"), (dict(page=0), "page"), (dict(page=65537), "page"),
                         (dict(table_stride=3), "table_stride"), (dict(table_stride=1 << 60), "too large"),
                         (dict(tables=None), "NULL"), (dict(lengths=None), "NULL"), (dict(free=None), "NULL"),
                         (dict(free_count=None), "NULL"), (dict(tables=A + 2), "aligned"),
                         (dict(free_count=D + 1), "aligned"), (dict(lengths=A + 8), "overlap"),
                         (dict(free=B), "overlap"), (dict(free_count=C + 4), "overlap"), (dict(tables=E), "overlap")]:
            refused(lambda: call(pages(**kw)), text)
    for name in ("counts", "starts", "positions", "slots"):
        refused(lambda: extend(**{name: None}), "NULL")
        refused(lambda: extend(**{name: A + (15 << 41) + 2}), "aligned")
        refused(lambda: extend(**{name: A}), "overlap")
    refused(lambda: extend(positions=F + 8), "overlap")
    refused(lambda: extend(slots=H + 4), "aligned")
    refused(lambda: extend(tokens=-1), "tokens")
    refused(lambda: extend(tokens=1 << 31), "tokens")
    refused(lambda: fgd.fgd_truncate_pages(pages(), None, 0), "NULL")


def test_pages_tensors():
    ints = lambda *a: torch.zeros(a, dtype=torch.int32)  # noqa: E731
    t, n, f, c = ints(3, 2), ints(3), ints(9), ints(1)
    run = lambda t=t, n=n, counts=n, f=f, c=c, page=16, tokens=5: fgd.extend_pages(t, n, counts, f, c, page, tokens)  # noqa: E731
    for bad, error, text in [
            (dict(t=t.long()), TypeError, "tables"), (dict(n=None), TypeError, "lengths"),
            (dict(n=ints(2)), ValueError, "lengths"), (dict(counts=ints(4)), ValueError, "counts"),
            (dict(counts=n.long()), TypeError, "counts"), (dict(f=ints(3, 3)), ValueError, "free"),
            (dict(f=f.long()), TypeError, "free"), (dict(c=ints(2)), ValueError, "free_count"),
            (dict(page=0), ValueError, "page"), (dict(page=1 << 40), ValueError, "page"),
            (dict(tokens=-1), ValueError, "tokens"), (dict(tokens=1 << 40), ValueError, "tokens"),
            (dict(), ValueError, "on a GPU")]:
        with pytest.raises(error, match=text):
            run(**bad)
    with pytest.raises(ValueError, match="keep"):
        fgd.truncate_pages(t, n, ints(2), f, c, 16)
    with pytest.raises(ValueError, match="on a GPU"):
        fgd.truncate_pages(t, n, n, f, c, 16)
