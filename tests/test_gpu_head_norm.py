"""Normalised and turned heads on the GPU against the float64 definition.

Tolerances, from the arithmetic.  u = 2^-24 and w = 2^-8 are half a unit of fp32 and of bfloat16.  A sum over a head's d values passes no value through
more than n = 2 sqrt(d) + 16 additions.  Sines and cosines are off by at most 4 u (series, roundings of the angle to the nearest quarter of a turn, 2^-32 turns of its whole
number).  With the pair's magnitudes |u| + |v| an output is off by at most (n + 16) u of them; dx by (2 n + 24) u of rstd (|w| m + |xh| mean(|w| m |xh|)) with m the
magnitudes of a pair of gradients; the weights' gradients, sums of N terms, each through at most 2 sqrt(N) + 200 additions, by (2 sqrt(N) + n + 216) u of
the sums of magnitudes.  One rounding on the way out to bfloat16: w |ref|.  The errors are independent: their root mean square is asserted to be 2^-20 of the
root mean square of the terms that a result is the difference or sum of (dx: of rstd |w| m.  Its two terms are equal but for eps where a head has one value: the result is then no
measure of the roundings), plus w of the results' in bfloat16.
"""
import ctypes as C

import numpy as np
import pytest

from oracle import memory as om

pytestmark = pytest.mark.gpu

U, W = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def torch():
    import torch as _torch
    assert _torch.cuda.is_available(), "these tests need the MI355X"
    return _torch


@pytest.fixture(scope="module")
def pxr():
    from paper_2502_00021_amd import pxr as _pxr
    _pxr.lib()
    return _pxr


def f64(x):
    return x.detach().double().cpu().numpy()


def gpu(torch, x, dtype="f32"):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def close(got, ref, bound, bf16, what, terms=None):
    if not ref.size:
        return
    terms = ref if terms is None else terms
    bound = bound + (W * np.abs(ref) if bf16 else 0.0) + 1e-37
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {ref[bad][0]}, bound {bound[bad][0]}"
    if ref.size >= 64:
        assert np.sqrt(((got - ref) ** 2).mean()) <= (W if bf16 else 0.0) * np.sqrt((ref ** 2).mean()) + 2.0 ** -20 * np.sqrt((terms ** 2).mean()), what


def frequencies(r, base=10000.0):
    return [base ** (-2 * i / r) for i in range(r // 2)]


def pairs(m, r):
    """Magnitudes [.., d]: for values that are turned, those of both of the pair."""
    m = np.array(m)
    both = m[..., :r // 2] + m[..., r // 2:r]
    m[..., :r // 2], m[..., r // 2:r] = both, both
    return m


def check(torch, pxr, layer, q, k, qw, kw, at, dq, dk, f, backward=True, first=0):
    """Tensors [B,T,H,d]; at: positions on the GPU, or None."""
    some = q if q is not None else k
    bf16, d, r = some.dtype == torch.bfloat16, some.shape[-1], layer.rotary
    B, T = some.shape[:2]
    P = np.broadcast_to(np.arange(T) + first, (B, T)) if at is None else at.cpu().numpy()
    args = dict(positions=at, first=first)
    n = 2 * np.sqrt(d) + 16
    outs = layer.forward(q, k, qw, kw, **args)
    for x, w, y in ((q, qw, outs[0]), (k, kw, outs[1])):
        if x is None:
            assert y is None
            continue
        assert y.dtype == x.dtype and y.shape == x.shape
        X, Wt = f64(x), None if w is None else f64(w)
        plain = om.head_norm(X, Wt, P, [], layer.eps)
        close(f64(y), om.head_norm(X, Wt, P, f, layer.eps), (n + 16) * U * pairs(np.abs(plain), r), bf16, "y")
    if not backward:
        return outs
    got = layer.backward(dq, dk, q, k, qw, kw, **args)
    for i, (x, w, dy) in enumerate(((q, qw, dq), (k, kw, dk))):
        dx, dw = got[i], got[2 + i]
        if x is None:
            assert dx is None and dw is None
            continue
        X, Wt, D = f64(x), None if w is None else f64(w), f64(dy)
        rx, rw = om.head_norm_backward(D, X, Wt, P, f, layer.eps)
        rstd = 1 / np.sqrt((X ** 2).mean(-1, keepdims=True) + layer.eps)
        m, xh = pairs(np.abs(D), r), np.abs(X * rstd)
        wm = m * (1.0 if Wt is None else np.abs(Wt))
        close(f64(dx), rx, (2 * n + 24) * U * rstd * (wm + xh * (wm * xh).mean(-1, keepdims=True)), bf16, "dx", rstd * wm)
        N = X.size // max(d, 1)
        close(f64(dw), rw, (2 * np.sqrt(N) + n + 216) * U * (m * xh).sum((0, 1, 2)), dw.dtype == torch.bfloat16, "dweight")
        assert dx.dtype == x.dtype and dw.dtype == (torch.float32 if w is None else w.dtype)
    return (*outs, *got)


def inputs(torch, rng, B, T, H, Hk, d, dtype, params="f32", layout="bthd", far=1000):
    def make(h):
        x = rng.standard_normal((B, T, h, d)) * (0.2 + rng.random((B, T, h, 1)))
        if layout == "bhtd":
            return gpu(torch, x.transpose(0, 2, 1, 3).copy(), dtype).transpose(1, 2)
        return gpu(torch, x, dtype)
    if layout == "fused":
        qkv = gpu(torch, rng.standard_normal((B, T, (H + 2 * Hk) * d)), dtype)
        q, k, _ = qkv.split([H * d, Hk * d, Hk * d], -1)
        q, k = q.unflatten(-1, (H, d)), k.unflatten(-1, (Hk, d))
    else:
        q, k = make(H), make(Hk)
    qw, kw = (gpu(torch, 1 + 0.3 * rng.standard_normal(d), params) for _ in range(2))
    at = torch.from_numpy(rng.integers(0, far, (B, T))).cuda()
    return q, k, qw, kw, at, make(H), make(Hk)


@pytest.mark.parametrize("dtype,params", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("d,r", [(1, 0), (2, 2), (3, 2), (8, 8), (8, 0), (16, 16), (24, 16), (31, 30), (33, 8), (48, 48), (64, 64), (64, 32), (64, 6), (96, 96), (100, 100), (127, 64), (128, 128),
                                 (200, 128), (130, 130), (255, 254), (255, 1 + 1), (256, 256), (256, 0)])
def test_sizes_of_heads(torch, pxr, d, r, dtype, params):
    rng = np.random.default_rng(d * 300 + r)
    f = frequencies(r)
    layer = pxr.HeadNorm(d, r)
    check(torch, pxr, layer, *inputs(torch, rng, 3, 11, 5, 2, d, dtype, params), f)
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,r", [(4, 0), (5, 0), (6, 0), (7, 0), (9, 0), (17, 0), (9, 8), (10, 10), (11, 10), (13, 8), (15, 8), (16, 10), (17, 8), (18, 10), (23, 10), (37, 20), (50, 26), (64, 30), (70, 70),
                                 (83, 40), (100, 50), (101, 58), (157, 156), (160, 154), (199, 90), (253, 250), (255, 8), (256, 246)])
def test_heads_that_are_no_whole_vectors(torch, pxr, d, r, dtype):
    rng = np.random.default_rng(d * 300 + r)
    layer = pxr.HeadNorm(d, r, frequencies(r))
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, 3, 11, 3, 2, d, dtype)
    check(torch, pxr, layer, q, k, qw, kw, at, dq, dk, frequencies(r))
    # in place: the vectors share values
    want = layer.forward(q, k, qw, kw, positions=at)
    a, b = q.clone(), k.clone()
    layer.forward(a, b, qw, kw, positions=at, q_out=a, k_out=b)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,Hk", [(1, 1, 1, 1), (1, 1, 16, 4), (16, 1, 4, 4), (5, 3, 7, 7), (2, 50, 9, 3), (300, 7, 4, 1), (1, 4000, 2, 1), (64, 128, 8, 8), (1, 1, 100, 33)])
def test_numbers_of_tokens_and_heads(torch, pxr, B, T, H, Hk, dtype):
    rng = np.random.default_rng(B + T)
    layer = pxr.HeadNorm(64)
    check(torch, pxr, layer, *inputs(torch, rng, B, T, H, Hk, 64, dtype), frequencies(64))
    layer.close()
    layer = pxr.HeadNorm(18, 12, base=100.0)
    check(torch, pxr, layer, *inputs(torch, rng, B, T, H, Hk, 18, dtype), frequencies(12, 100.0))
    layer.close()


def test_many_tokens(torch, pxr):
    rng = np.random.default_rng(1)
    layer = pxr.HeadNorm(32)
    check(torch, pxr, layer, *inputs(torch, rng, 100, 701, 3, 1, 32, "bf16"), frequencies(32))
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bthd", "bhtd", "fused"])
@pytest.mark.parametrize("d", [64, 20, 9])
def test_layouts(torch, pxr, layout, d, dtype):
    rng = np.random.default_rng(d)
    layer = pxr.HeadNorm(d)
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, 3, 40, 4, 2, d, dtype, layout=layout)
    f = frequencies(d // 2 * 2)
    got = check(torch, pxr, layer, q, k, qw, kw, at, dq, dk, f)
    # positions in other types and strides, of all environments together, or by the step's number
    again = check(torch, pxr, layer, q, k, qw, kw, at.int().t().contiguous().t(), dq, dk, f)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    check(torch, pxr, layer, q, k, qw, kw, at[:1].expand(3, -1), dq, dk, f)
    check(torch, pxr, layer, q, k, None, kw, None, dq, dk, f, first=-7)
    check(torch, pxr, layer, q, k, None, None, None, dq, dk, f, first=2 ** 33)
    # heads that share, environments that share
    check(torch, pxr, layer, q[:1].expand(3, -1, -1, -1), k[:, :, :1].expand(-1, -1, 2, -1), qw, kw, at, dq[:, :1].expand(-1, 40, -1, -1), dk, f)
    # queries alone, keys alone
    assert torch.equal(check(torch, pxr, layer, q, None, qw, None, at, dq, None, f)[0], got[0])
    assert torch.equal(check(torch, pxr, layer, None, k, None, kw, at, None, dk, f)[1], got[1])
    # single steps
    for t in (0, 17):
        q1, k1 = layer.forward(q[:, t], k[:, t], qw, kw, positions=at[:, t])
        assert q1.shape == (3, 4, d) and torch.equal(q1, got[0][:, t]) and torch.equal(k1, got[1][:, t])
        g = layer.backward(dq[:, t], dk[:, t], q[:, t], k[:, t], qw, kw, positions=at[:, t])
        assert torch.equal(g[0], got[2][:, t]) and torch.equal(g[1], got[3][:, t])
    layer.close()


@pytest.mark.parametrize("wide", [True, False])
def test_far_positions(torch, pxr, wide):
    """Angles of millions of turns: their sines from whole numbers of 64 bits, against the definition's in long double."""
    rng = np.random.default_rng(2)
    d = 64
    f = np.array(frequencies(d))
    layer = pxr.HeadNorm(d)
    x = gpu(torch, rng.standard_normal((1, 400, 1, d)))
    most = 2 ** 31 - 1
    at = rng.integers(-most, most, (1, 400))
    at[0, :4] = most, -most - 1, 0, -1
    y, _ = layer.forward(x, None, positions=torch.from_numpy(at if wide else at.astype(np.int32)).cuda())
    X = f64(x)
    n = om.head_norm(X, None, np.zeros((1, 400)), [], layer.eps)
    angle = np.fmod(at[0, :, None].astype(np.longdouble) * f.astype(np.longdouble), 2 * np.longdouble("3.14159265358979323846264338327950288"))
    c, s = (fn(angle).astype(np.float64)[None, :, None] for fn in (np.cos, np.sin))
    lo, hi = n[..., :32], n[..., 32:]
    ref = np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)
    # the angle itself: 2^31 positions of a fraction rounded to 2^-63 turns, and the definition's own remainder of 2^-64 of the angle
    close(f64(y), ref, ((2 * 8 + 32) * U + 2 * np.pi * 2.0 ** -30) * pairs(np.abs(n), d), False, "y")
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 33])
def test_in_place(torch, pxr, d, dtype):
    rng = np.random.default_rng(d)
    layer = pxr.HeadNorm(d)
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, 4, 30, 6, 5, d, dtype)
    want = layer.forward(q, k, qw, kw, positions=at)
    q2, k2 = q.clone(), k.clone()
    layer.forward(q2, k2, qw, kw, positions=at, q_out=q2, k_out=k2)
    assert torch.equal(q2, want[0]) and torch.equal(k2, want[1])
    # gradients: in the place of the inputs, or of the outputs' gradients
    want = layer.backward(dq, dk, q, k, qw, kw, positions=at)
    at32 = at.int()
    for alias in (0, 1):
        t = [x.clone() for x in (q, k, dq, dk)]
        views = [pxr.Tokens(x.data_ptr(), *x.stride()[:3]) for x in t]
        r = pxr.Heads(1 if dtype == "bf16" else 0, 0, 4, 30, 6, 5, views[0], views[1], qw.data_ptr(), kw.data_ptr(), at32.data_ptr(), 32, 30, 1, 0)
        into = [C.byref(v) for v in (views[:2] if alias else views[2:])]
        assert pxr.lib().pxr_head_norm_backward(layer._h, C.byref(r), C.byref(views[2]), C.byref(views[3]), *into, None, None, None, 0,
                                                torch.cuda.current_stream().cuda_stream) == pxr.OK
        got = t[:2] if alias else t[2:]
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    layer.close()


def test_of_no_tokens_or_heads(torch, pxr):
    layer = pxr.HeadNorm(16)
    for shape in ((0, 5, 3, 16), (5, 0, 3, 16), (0, 3, 16), (2, 3, 0, 16)):
        x = torch.empty(shape, device="cuda")
        y, none = layer.forward(x, None)
        assert y.shape == shape and none is None
        dq, dk, dqw, dkw = layer.backward(x, x, x, x)
        assert dq.shape == shape and (dqw == 0).all() and (dkw == 0).all()
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,H", [(64, 6), (33, 3), (256, 2), (8, 9)])
def test_heads_do_not_reach_each_other(torch, pxr, d, H, dtype):
    """A NaN or an infinity stays in its head; equal rows of zeros are zeros."""
    rng = np.random.default_rng(d)
    layer = pxr.HeadNorm(d)
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, 3, 9, H, H, d, dtype)
    want, grads = layer.forward(q, k, qw, kw, positions=at), layer.backward(dq, dk, q, k, qw, kw, positions=at)
    for value in (float("nan"), float("inf")):
        bad = q.clone()
        bad[1, 4, H - 1, d // 2] = value
        got = layer.forward(bad, k, qw, kw, positions=at)
        keep = torch.ones(q.shape[:3], dtype=torch.bool, device="cuda")
        keep[1, 4, H - 1] = False
        assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1], want[1]) and got[0][1, 4, H - 1].isnan().any()
        g = layer.backward(dq, dk, bad, k, qw, kw, positions=at)
        assert torch.equal(g[0][keep], grads[0][keep]) and torch.equal(g[1], grads[1]) and torch.equal(g[3], grads[3])
        bad = dk.clone()
        bad[1, 4, H - 1, d // 2] = value
        g = layer.backward(dq, bad, q, k, qw, kw, positions=at)
        assert torch.equal(g[1][keep], grads[1][keep]) and torch.equal(g[0], grads[0]) and torch.equal(g[2], grads[2])
    q.zero_()
    assert (layer.forward(q, None, qw, positions=at)[0] == 0).all()
    g = layer.backward(dq, None, q, None, qw, positions=at)
    assert g[0].isfinite().all() and (g[2] == 0).all()
    layer.close()


def test_gradients_by_differences(torch, pxr):
    """The kernels' own forward pass, moved along a direction."""
    rng = np.random.default_rng(3)
    layer = pxr.HeadNorm(32, 24)
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, 4, 20, 3, 2, 32, "f32")
    q, k = q + 0.5, k + 0.5
    got = layer.backward(dq, dk, q, k, qw, kw, positions=at)
    h = 2.0 ** -8

    def f(*x):
        a, b = layer.forward(*x, positions=at)
        return float((a.double() * dq.double()).sum() + (b.double() * dk.double()).sum())
    for i, grad in enumerate(got):
        d = gpu(torch, rng.standard_normal(tuple(grad.shape)))
        up, down = [q, k, qw, kw], [q, k, qw, kw]
        up[i], down[i] = up[i] + h * d, down[i] - h * d
        want = float((grad.double() * d.double()).sum())
        size = float((grad.double() * d.double()).square().sum().sqrt())
        # h^2 times third derivatives (order 10 a value: heads of a root mean square of a half), and 12800 roundings, in the root of their number, over h
        assert abs((f(*up) - f(*down)) / (2 * h) - want) < 30 * h * h * size + 16 * U * np.sqrt(12800.0) / h, i
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,Hk,d,r", [(3, 7, 5, 2, 33, 30), (2, 300, 8, 1, 64, 64), (40, 1, 3, 3, 24, 16), (1, 5, 2, 1, 255, 100)])
def test_writes_nothing_else_and_gives_equal_bits(torch, pxr, B, T, H, Hk, d, r, dtype):
    rng = np.random.default_rng(d)
    layer = pxr.HeadNorm(d, r)
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, B, T, H, Hk, d, dtype)
    want = layer.forward(q, k, qw, kw, positions=at)
    wide = torch.full((B + 2, T + 2, H + Hk + 1, d + 3), 7.0, device="cuda", dtype=q.dtype)
    into = [wide[1:-1, 1:-1, :H, 1:1 + d], wide[1:-1, 1:-1, H:H + Hk, 2:2 + d]]
    got = layer.forward(q, k, qw, kw, positions=at, q_out=into[0], k_out=into[1])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for t in into:
        t.fill_(7.0)
    assert (wide == 7).all()
    first = layer.backward(dq, dk, q, k, qw, kw, positions=at)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, layer.backward(dq, dk, q, k, qw, kw, positions=at)))
    layer.close()


def test_offsets_past_32_bits(torch, pxr):
    rng = np.random.default_rng(4)
    layer = pxr.HeadNorm(64)
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, 2, 6, 3, 2, 64, "bf16")
    apart = 2 ** 31 + 64
    big = torch.empty(apart + 6 * 3 * 64 + 64, device="cuda", dtype=torch.bfloat16)
    view = big.as_strided(q.shape, (apart, 3 * 64, 64, 1), 8)
    view.copy_(q)
    want, grads = layer.forward(q, k, qw, kw, positions=at), layer.backward(dq, dk, q, k, qw, kw, positions=at)
    got = layer.forward(view, k, qw, kw, positions=at)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all(torch.equal(a, b) for a, b in zip(grads, layer.backward(dq, dk, view, k, qw, kw, positions=at)))
    layer.forward(view, k, qw, kw, positions=at, q_out=view)
    assert torch.equal(view, want[0])
    layer.close()


def test_streams_and_graphs(torch, pxr):
    """On a stream of the caller's, and captured twice and replayed with new values, with eager calls between."""
    rng = np.random.default_rng(5)
    layer = pxr.HeadNorm(48, 32)
    for B, T in ((4, 60), (700, 1)):
        sets = [inputs(torch, rng, B, T, 4, 2, 48, "bf16") for _ in range(4)]
        static = [t.clone() for t in sets[0]]

        def both(q, k, qw, kw, at, dq, dk, **stream):
            return (*layer.forward(q, k, qw, kw, positions=at, **stream), *layer.backward(dq, dk, q, k, qw, kw, positions=at, **stream))
        want = [both(*t) for t in sets]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = both(*sets[1], stream=side.cuda_stream)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want[1]))
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                graphs.append((g, both(*static)))
        for i in (1, 2, 3, 0, 2):
            for t, new in zip(static, sets[i]):
                t.copy_(new)
            for g, got in graphs:
                g.replay()
                eager = both(*sets[(i + 1) % 4])
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want[i])) and all(torch.equal(a, b) for a, b in zip(eager, want[(i + 1) % 4]))
    layer.close()


def test_refusals(torch, pxr):
    rng = np.random.default_rng(6)
    layer = pxr.HeadNorm(16)
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, 2, 10, 3, 2, 16, "f32")
    for bad in (dict(q=q.half()), dict(k=k.bfloat16()), dict(k=k[:, :9]), dict(q=q.cpu()), dict(q=q[..., :15]), dict(q=q.transpose(2, 3)), dict(q_weight=qw[:15]), dict(q_weight=qw.half()),
                dict(k_weight=kw.bfloat16()), dict(positions=at[:, :9]), dict(positions=at.float()), dict(positions=at, first=1), dict(q=None, k=None), dict(q=q[:, 0]),
                dict(q_out=q[:, :9]), dict(q=None, q_weight=None, q_out=q)):
        a = dict(dict(q=q, k=k, q_weight=qw, k_weight=kw, positions=at), **bad)
        with pytest.raises(AssertionError):
            layer.forward(a.pop("q"), a.pop("k"), **a)
    with pytest.raises(AssertionError):
        layer.backward(dq[:, 1:], dk, q, k)
    # at the library itself, before anything is launched
    view = pxr.Tokens(q.data_ptr(), *q.stride()[:3])
    off = pxr.Tokens(q.data_ptr() + 2, *q.stride()[:3])
    L, n = pxr.lib(), C.c_size_t()

    def heads(**change):
        r = pxr.Heads(0, 0, 2, 10, 3, 2, view, view, None, None, None, 32, 0, 0, 0)
        for name, value in change.items():
            setattr(r, name, value)
        return C.byref(r)
    v = C.byref(view)
    for change in (dict(dtype=2), dict(param_dtype=1), dict(position_bits=16), dict(n_envs=2 ** 31, n_steps=1), dict(n_envs=2 ** 16, n_steps=2 ** 16), dict(n_heads=65536), dict(n_key_heads=65536)):
        assert L.pxr_head_norm_forward(layer._h, heads(**change), v, v, None) == pxr.ERR_INVALID_ARG
        assert L.pxr_head_norm_workspace(layer._h, heads(**change), C.byref(n)) == pxr.ERR_INVALID_ARG
        assert L.pxr_head_norm_backward(layer._h, heads(**change), v, v, v, v, None, None, None, 0, None) == pxr.ERR_INVALID_ARG
    for change in (dict(q=off), dict(k=off), dict(q=pxr.Tokens()), dict(d_q_weight=66), dict(d_k_weight=66), dict(d_positions=66)):
        assert L.pxr_head_norm_forward(layer._h, heads(**change), v, v, None) == pxr.ERR_INVALID_ARG
        assert L.pxr_head_norm_backward(layer._h, heads(**change), v, v, v, v, None, None, None, 0, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_head_norm_workspace(layer._h, heads(), None) == pxr.ERR_INVALID_ARG
    for outs in ((None, v), (v, None), (C.byref(off), v), (v, C.byref(off))):
        assert L.pxr_head_norm_forward(layer._h, heads(), *outs, None) == pxr.ERR_INVALID_ARG
        assert L.pxr_head_norm_backward(layer._h, heads(), *outs, v, v, None, None, None, 0, None) == pxr.ERR_INVALID_ARG
        assert L.pxr_head_norm_backward(layer._h, heads(), v, v, *outs, None, None, None, 0, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_head_norm_workspace(layer._h, heads(), C.byref(n)) == pxr.OK and n.value
    sums = torch.empty(16, device="cuda")
    ws = torch.empty(n.value + 16, dtype=torch.uint8, device="cuda")
    for at_ws, size in ((None, n.value), (ws.data_ptr() + 8, n.value), (ws.data_ptr(), n.value - 1)):
        assert L.pxr_head_norm_backward(layer._h, heads(), v, v, v, v, sums.data_ptr(), None, at_ws, size, None) == pxr.ERR_INVALID_ARG
    layer.close()


@pytest.mark.parametrize("d,r", [(32, 32), (64, 64), (100, 50)])
def test_is_as_exact_as_elementary_operations(torch, pxr, d, r):
    """Root mean square of the errors of a million values and more against those of the same formula in PyTorch's fp32 operations, which has sines of angles in 64 bits, rounded once.  There a turned value has
    five roundings of its own besides its terms' (two sines, two products, a sum); here four, and sines that are off by some more than a rounding, 1.7e-8 for 1.45e-8 of values around 0.7: that
    is 2 (1.7^2 - 1.45^2) = 1.6 of 1e-16, and the rounding of a product that is not there, of values around 0.5, 1.2 of them, in a sum of more than 25.  So no more than 2 % in the root; the sample's share is 0.1 %."""
    rng = np.random.default_rng(d)
    layer = pxr.HeadNorm(d, r)
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, 32, 100, 8, 6, d, "f32", far=100000)
    angle = at.double()[:, :, None, None] * torch.tensor(frequencies(r), dtype=torch.float64, device="cuda")

    def turned(y, cos, sin):
        lo, hi, rest = y.split([r // 2, r // 2, d - r], -1)
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin, rest], -1)

    def formula(to, x, w, dy):
        x, w, dy, cos, sin = x.to(to), w.to(to), dy.to(to), angle.cos().to(to), angle.sin().to(to)
        rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + layer.eps)
        g = turned(dy, cos, -sin)
        return turned(x * rstd * w, cos, sin), rstd * (g * w - x * rstd * (g * w * x * rstd).mean(-1, keepdim=True))
    got = (*layer.forward(q, k, qw, kw, positions=at), *layer.backward(dq, dk, q, k, qw, kw, positions=at)[:2])
    for y, dx, x, w, dy in ((got[0], got[2], q, qw, dq), (got[1], got[3], k, kw, dk)):
        for ours, plain, ref in zip((y, dx), formula(torch.float32, x, w, dy), formula(torch.float64, x, w, dy)):
            ours, plain = ((t.double() - ref).square().mean().sqrt() for t in (ours, plain))
            assert float(ours) <= 1.02 * float(plain)
    layer.close()


def test_outputs_in_the_place_of_other_heads(torch, pxr):
    """Of the other kind, of the other output, a step or a head on: refused.  Parts of one buffer side by side are none of these."""
    rng = np.random.default_rng(10)
    B, T, d = 3, 20, 16
    layer = pxr.HeadNorm(d)
    q, k, qw, kw, at, dq, dk = inputs(torch, rng, B, T, 4, 2, d, "f32")
    args = dict(positions=at)
    want = layer.forward(q, k, qw, kw, **args)
    wide = torch.cat([q, k, torch.zeros_like(q), torch.zeros_like(k)], 2)
    a, b, c, e = wide.split([4, 2, 4, 2], 2)
    got = layer.forward(a, b, qw, kw, **args, q_out=c, k_out=e)
    assert torch.equal(c, want[0]) and torch.equal(e, want[1]) and torch.equal(a, q) and torch.equal(b, k)
    for outs in (dict(q_out=wide[:, :, 1:5]), dict(q_out=wide[:, :, 5:9]), dict(k_out=wide[:, :, 3:5]), dict(k_out=wide[:, :, 5:7]), dict(q_out=c, k_out=wide[:, :, 9:11]), dict(q_out=wide[:, :, 2:6], k_out=b)):
        with pytest.raises(pxr.PxrError, match="overlaps"):
            layer.forward(a, b, qw, kw, **args, **outs)
    one = k.clone()
    for outs in (dict(q_out=one), dict(k_out=one)):  # queries that are the keys: neither can take their place
        with pytest.raises(pxr.PxrError, match="overlaps"):
            layer.forward(one, one, qw, kw, **args, **outs)
    longer = torch.zeros((B, T + 1, 4, d), device="cuda")
    with pytest.raises(pxr.PxrError, match="overlaps"):
        layer.forward(longer[:, 1:], k, qw, kw, **args, q_out=longer[:, :-1])
    # gradients, by the C call
    L, at32 = pxr.lib(), at.int()
    t = dict(q=q.clone(), k=k.clone(), dq=dq.clone(), dk=dk.clone())
    v = {name: pxr.Tokens(x.data_ptr(), *x.stride()[:3]) for name, x in t.items()}
    r = pxr.Heads(0, 0, B, T, 4, 2, v["q"], v["k"], qw.data_ptr(), kw.data_ptr(), at32.data_ptr(), 32, T, 1, 0)
    moved = lambda name, by: pxr.Tokens(v[name].data + 4 * by, v[name].env, v[name].step, v[name].head)
    for to_q, to_k in ((v["k"], v["dk"]), (v["dk"], v["k"]), (v["q"], v["q"]), (v["dq"], v["dq"]), (v["q"], v["dq"]), (moved("q", d), v["k"]), (v["q"], moved("dk", 1))):
        assert L.pxr_head_norm_backward(layer._h, C.byref(r), C.byref(v["dq"]), C.byref(v["dk"]), C.byref(to_q), C.byref(to_k), None, None, None, 0, None) == pxr.ERR_INVALID_ARG
        assert "overlaps" in L.pxr_last_error().decode()
    layer.close()
