"""GPU tests of rotate_heads and its gradients against the 64-bit reference.

Tolerances, with u = 2^-24: a head's mean of squares is a sum of positive
terms, 8 in a lane and up to 6 steps over lanes, so its root's inverse is off by
at most (14 + 2) u / 2 + 2 u; a normed and weighted element by 12 u + 2 u, its
cosine and sine by u each, and the two products and their sum by 2 u: 17 u of
the terms' magnitudes, held against 20 u.  A gradient has the same factors, a
mean of 14 u and four more operations on it: 64 u of its terms' magnitudes.  A
weight's gradient is a sum of such terms of 16 u each, of which a lane adds at
most 16 + 4 rounds in float32, a block one for each of its groups of lanes,
and the rest is float64.  bf16 outputs are off by 2^-8 of the value besides.
"""

import numpy as np
import pytest

from oracle import attention as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2606_22768_amd as fgd

    return fgd, torch


def _np(t):
    return t.detach().double().cpu().numpy()


def _check(got, want, bound, u, dtype):
    got = _np(got)
    tol = u * U * bound + 1e-37
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (abs(want) + tol) + 2.0 ** -134
    worst = np.max(abs(got - want) / tol) if want.size else 0
    assert np.all(abs(got - want) <= tol), worst


def _groups(D):
    lanes = 1
    while 8 * lanes < D:
        lanes *= 2
    return 256 // lanes


class Case:
    def __init__(self, env, M, T, HQ, HK, D, rot, dtype, weights="own", far=1000, seed=0, spread=1):
        self.fgd, torch = env
        self.torch, self.dtype = torch, dtype
        g = torch.Generator().manual_seed(seed)
        t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        lead = (T,) if M is None else (M, T)
        mk = lambda h: (torch.randn((*lead, h, D), generator=g) * spread).to(t).cuda()  # noqa: E731
        self.q, self.k, self.dq, self.dk = mk(HQ), mk(HK), mk(HQ), mk(HK)
        self.positions = torch.randint(-far, far + 1, (T,), generator=g, dtype=torch.int32).cuda()
        self.freqs = torch.pow(torch.tensor(10000.0, dtype=torch.float64),
                               -torch.arange(rot // 2, dtype=torch.float64) * 2 / max(rot, 1)).cuda()
        shape = (D,) if M is None or weights == "shared" else (M, D)
        self.w = [None, None] if weights is None else [(1 + torch.randn(shape, generator=g)).cuda() for _ in range(2)]

    def forward(self, **kw):
        return self.fgd.rotate_heads(self.q, self.k, self.positions, self.freqs, *self.w, **kw)

    def check(self, eps=1e-6, interleaved=False):
        got = self.forward(eps=eps, interleaved=interleaved)
        args = (_np(self.positions), _np(self.freqs), np.float32(eps).astype(np.float64), interleaved)
        for y, x, w in zip(got, (self.q, self.k), self.w):
            _check(y, *ref.rotate_heads(_np(x), None if w is None else _np(w), *args), 20, self.dtype)
        got = self.fgd.rotate_heads_grads(self.dq, self.dk, self.q, self.k, self.positions, self.freqs, *self.w,
                                          eps=eps, interleaved=interleaved)
        for i, (dy, x, w) in enumerate(zip((self.dq, self.dk), (self.q, self.k), self.w)):
            dx, dw, bx, bw = ref.rotate_heads_grads(_np(dy), _np(x), None if w is None else _np(w), *args)
            _check(got[i], dx, bx, 64, self.dtype)
            if w is None:
                assert got[2 + i] is None
            else:
                assert got[2 + i].dtype == self.torch.float32
                _check(got[2 + i], dw, bw, 16 + 20 + _groups(x.shape[-1]) + 1, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("M, T, HQ, HK, D, rot", [
    (None, 1, 1, 1, 2, 2), (None, 3, 5, 2, 6, 4), (None, 17, 3, 1, 40, 10), (None, 5, 7, 1, 80, 20),
    (None, 33, 4, 4, 64, 64), (2, 9, 8, 2, 128, 128), (3, 21, 2, 1, 96, 32), (1, 7, 2, 2, 256, 128),
    (2, 5, 1, 3, 512, 512), (None, 11, 3, 2, 128, 0), (None, 130, 6, 1, 34, 34)])
def test_heads_and_gradients(env, M, T, HQ, HK, D, rot, interleaved, dtype):
    Case(env, M, T, HQ, HK, D, rot, dtype, seed=T).check(interleaved=interleaved)


@pytest.mark.parametrize("weights", [None, "shared", "own"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weights_of_a_batch(env, weights, dtype):
    Case(env, 4, 50, 4, 2, 64, 64, dtype, weights=weights).check()


def test_many_tokens(env):
    # More tokens than the gradients' blocks take at once.
    Case(env, 2, 3000, 7, 2, 64, 32, "bf16").check()


def test_far_positions(env):
    c = Case(env, None, 64, 2, 1, 128, 128, "f32", far=2 ** 31 - 1)
    c.positions[:2] = c.torch.tensor([2 ** 31 - 1, -2 ** 31 + 1])
    # The angle itself is a float64 product: 2^31 radians to 2^-22 / 2^31 of a turn.
    got = c.forward()
    args = (_np(c.positions), _np(c.freqs), 1e-6, False)
    for y, x, w in zip(got, (c.q, c.k), c.w):
        want, bound = ref.rotate_heads(_np(x), _np(w), *args)
        _check(y, want, bound, 20 + 2 * 2 ** 31 * 3 * 2.0 ** -53 / U, "f32")


def test_bf16_weights_and_one_input(env):
    fgd, torch = env
    c = Case(env, None, 19, 4, 2, 96, 48, "bf16")
    c.w = [w.bfloat16() for w in c.w]
    c.check()
    q, none = fgd.rotate_heads(c.q, None, c.positions, c.freqs, c.w[0])
    assert none is None and torch.equal(q, c.forward()[0])
    dq, dk, wq, wk = fgd.rotate_heads_grads(c.dq, None, c.q, None, c.positions, c.freqs, c.w[0])
    assert dk is None and wk is None and torch.isfinite(dq).all() and torch.isfinite(wq).all()
    c.w = [c.w[0], None]  # a norm on queries alone
    c.check()
    only = fgd.rotate_heads_grads(c.dq, c.dk, None, None, c.positions, c.freqs)
    assert only[2] is None and torch.isfinite(only[1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 34])
def test_views_of_a_projection_and_in_place(env, D, dtype):
    fgd, torch = env
    c = Case(env, 2, 13, 6, 2, D, D, dtype)
    want = c.forward()
    for pad in (0, 1, 4):  # aligned and not
        qkv = torch.randn((2, 13, 10 * D + pad), device="cuda").to(c.q.dtype)
        qkv[..., :6 * D] = c.q.flatten(-2)
        qkv[..., 6 * D:8 * D] = c.k.flatten(-2)
        before = qkv.clone()
        q, k = qkv[..., :6 * D].unflatten(-1, (6, D)), qkv[..., 6 * D:8 * D].unflatten(-1, (2, D))
        for a, b in zip(want, fgd.rotate_heads(q, k, c.positions, c.freqs, *c.w)):
            assert torch.equal(a, b)
        got = fgd.rotate_heads_grads(c.dq, c.dk, q, k, c.positions, c.freqs, *c.w)
        base = fgd.rotate_heads_grads(c.dq, c.dk, c.q, c.k, c.positions, c.freqs, *c.w)
        assert all(torch.equal(a, b) for a, b in zip(got, base))
        fgd.rotate_heads(q, k, c.positions, c.freqs, *c.w, q_out=q, k_out=k)
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])
        assert torch.equal(qkv[..., 8 * D:], before[..., 8 * D:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_that_are_views_of_one_array(env, dtype):
    fgd, torch = env
    D = 64
    c = Case(env, 2, 13, 6, 2, D, D, dtype)
    want = c.forward()
    both = torch.full((2, 13, 10 * D), 3.0, dtype=c.q.dtype, device="cuda")
    q, k = both[..., :6 * D].unflatten(-1, (6, D)), both[..., 6 * D:8 * D].unflatten(-1, (2, D))
    fgd.rotate_heads(c.q, c.k, c.positions, c.freqs, *c.w, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and (both[..., 8 * D:] == 3).all()
    with pytest.raises(fgd.FgdError, match="each other"):
        fgd.rotate_heads(c.q, c.k, c.positions, c.freqs, *c.w, q_out=q, k_out=both[..., 1 + 5 * D:1 + 7 * D].unflatten(-1, (2, D)))
    # The gradients too, by the C call.
    want = fgd.rotate_heads_grads(c.dq, c.dk, c.q, c.k, c.positions, c.freqs, *c.w)
    sizes = fgd.fgd_heads(dtype, 2, 6, 2, D, D, 0, 13, 0, D, 1e-6)
    work = torch.empty(fgd.fgd_rotate_heads_grads_workspace_size(sizes), dtype=torch.uint8, device="cuda")
    wq, wk = torch.empty((2, 2, D), device="cuda").unbind()
    axes = lambda t: tuple(t.stride()[:3])  # noqa: E731
    fgd.fgd_rotate_heads_grads(sizes, c.dq, axes(c.dq), c.dk, axes(c.dk), c.q, axes(c.q), c.k, axes(c.k), c.positions,
                               c.freqs, *c.w, q, axes(q), k, axes(k), wq, wk, work, work.numel(),
                               torch.cuda.current_stream().cuda_stream)
    assert all(torch.equal(a, b) for a, b in zip((q, k, wq, wk), want)) and (both[..., 8 * D:] == 3).all()


def test_positions_of_every_batch_entry(env):
    fgd, torch = env
    c = Case(env, 3, 8, 2, 1, 64, 64, "f32")
    c.positions = torch.randint(0, 999, (3, 8), dtype=torch.int32, device="cuda")
    c.check()
    per = [fgd.rotate_heads(c.q[m], c.k[m], c.positions[m], c.freqs, c.w[0][m], c.w[1][m]) for m in range(3)]
    whole = c.forward()
    for i in range(2):
        assert torch.equal(torch.stack([p[i] for p in per]), whole[i])


def test_extreme_rows(env):
    fgd, torch = env
    c = Case(env, None, 6, 1, 1, 64, 64, "f32")
    c.q[0] = 0
    c.q[1, 0, 3] = float("inf")
    c.q[2, 0, 5] = float("nan")
    c.q[3] *= 1e-30
    q, _ = c.forward()
    assert (q[0] == 0).all() and torch.isnan(q[2]).all()
    assert torch.isnan(q[1]).any() and torch.isfinite(q[[0, 3, 4, 5]]).all()
    g = fgd.rotate_heads_grads(c.dq, c.dk, c.q, c.k, c.positions, c.freqs, *c.w)
    assert torch.isfinite(g[0][[0, 3, 4, 5]]).all() and torch.isnan(g[0][2]).all()


def test_gradients_against_differences(env):
    fgd, torch = env
    c = Case(env, 2, 6, 3, 2, 64, 32, "f32", weights="shared")
    args = (c.positions, c.freqs)
    dq, dk, wq, wk = fgd.rotate_heads_grads(c.dq, c.dk, c.q, c.k, *args, *c.w)

    def f(q, k, a, b):
        y, z = fgd.rotate_heads(q, k, *args, a, b)
        return (y.double() * c.dq.double()).sum() + (z.double() * c.dk.double()).sum()

    # Steps of 2^-6: the second difference's error is about h^2 / 6 of the third
    # derivative, and 20 u of 2 10^3 terms over 2 h of rounding: 2e-3 is held.
    h = 2.0 ** -6
    for i, g in enumerate((dq, dk, wq, wk)):
        at = [c.q, c.k, *c.w]
        d = torch.randn(g.shape, device="cuda")
        d /= d.norm()
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * d, at[i] - h * d
        slope = ((f(*up) - f(*down)) / (2 * h)).item()
        assert abs(slope - (g.double() * d.double()).sum().item()) < 2e-3 * max(1, g.norm().item())


@pytest.mark.parametrize("shape", [(0, 2, 64), (5, 0, 64)])
def test_empty(env, shape):
    fgd, torch = env
    q = torch.empty(shape, device="cuda")
    k = torch.empty((shape[0], 0, 64), device="cuda")
    p = torch.zeros(shape[0], dtype=torch.int32, device="cuda")
    f = torch.ones(32, dtype=torch.float64, device="cuda")
    w = torch.ones(64, device="cuda")
    assert fgd.rotate_heads(q, k, p, f, w, w)[0].shape == shape
    dq, dk, wq, wk = fgd.rotate_heads_grads(q, k, q, k, p, f, w, w)
    assert (wq == 0).all() and (wk == 0).all()


def test_stream_graph_and_equal_bits(env):
    fgd, torch = env
    c = Case(env, 2, 40, 4, 2, 128, 128, "bf16")
    want = (*c.forward(), *fgd.rotate_heads_grads(c.dq, c.dk, c.q, c.k, c.positions, c.freqs, *c.w))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = (*c.forward(stream=s),
           *fgd.rotate_heads_grads(c.dq, c.dk, c.q, c.k, c.positions, c.freqs, *c.w, stream=s))
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = (*c.forward(), *fgd.rotate_heads_grads(c.dq, c.dk, c.q, c.k, c.positions, c.freqs, *c.w))
    for i in range(4):
        c.q.copy_(torch.randn(c.q.shape, device="cuda"))
        c.positions.add_(i)
        graph.replay()
        torch.cuda.synchronize()
        want = (*c.forward(), *fgd.rotate_heads_grads(c.dq, c.dk, c.q, c.k, c.positions, c.freqs, *c.w))
        assert all(torch.equal(a, b) for a, b in zip(want, out))
