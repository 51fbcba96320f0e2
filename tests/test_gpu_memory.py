"""A policy's memory on the GPU (layer norm, linear attention with a decay for each head) against the float64 definitions.

Tolerances, from the arithmetic.  u = 2^-24 and w = 2^-8 are half a unit of fp32 and of bfloat16 (8 significant bits).

Layer norm: a row's sums are fp32 over at least sqrt(D) / 2 lanes, so no value passes through more than n = 2 sqrt(D) + 16
additions.  With a = the mean of |x|: the mean is off by at most n u a; the variance by n u of itself (and by the square of
the mean's error), so xh by n u (|xh| + a rstd), and a few operations more.  dx: the two sums are off by n u of the
sums of magnitudes.  dw, db: sums over N rows in at most n' = 2 sqrt(N) + 64 additions a value.  One rounding to bfloat16
on the way out: w |ref|.

Linear attention: with A = the result for the magnitudes of all inputs, products and sums in fp32 give at most (64 + d + T) u A
(no term passes through more additions than a head has values and the rollout steps).  From bfloat16 inputs the
probabilities and the state may be rounded to bfloat16 once before they are multiplied, each term having one of the two: w A;
the rounding on the way out: w |ref|.  A worst case has all roundings in one direction; they are independent, so the root
mean square of the error is asserted as well: at most w of the results' (three roundings of w / sqrt(3) or less each, sqrt(3)
in all), and in fp32 and for states 2^-20.
"""
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
    return torch.from_numpy(np.asarray(x, np.float32)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def within(got, ref, bound, what):
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {ref[bad][0]}, bound {np.broadcast_to(bound, ref.shape)[bad][0]}"


# ------------------------------------------------------------------ layer norm

def check_norm(torch, pxr, x, w, b, dy, eps=1e-5):
    """Forward and backward of GPU tensors x [N,D], dy, weight and bias (or None) against the definition."""
    N, D = x.shape
    X, Wt, Bs = f64(x), None if w is None else f64(w), None if b is None else f64(b)
    out_w = W if x.dtype == torch.bfloat16 else 0.0
    par_w = W if w is not None and w.dtype == torch.bfloat16 else 0.0
    y, mean, rstd = pxr.layer_norm(x, w, b, eps=eps)
    ref, rm, rr = om.layer_norm(X, Wt, Bs, eps)
    n, a = 2 * np.sqrt(D) + 16, np.abs(X).mean(1) if D else 0
    within(f64(mean), rm, n * U * a + 1e-37, "mean")
    far = n * U * (1 + a * rr) ** 2  # (a row far from zero: the mean's error against the spread)
    within(f64(rstd), rr, far * rr, "rstd")
    aw = 1.0 if Wt is None else np.abs(Wt)
    xh = np.abs((X - rm[:, None]) * rr[:, None])
    within(f64(y), ref, out_w * np.abs(ref) + far[:, None] * aw * (xh + 1) + 4 * U * (np.abs(ref) + (0 if Bs is None else np.abs(Bs))) + 1e-37, "y")
    if dy is None:
        return
    G = f64(dy)
    dx, dw, db = pxr.layer_norm_backward(dy, x, mean, rstd, w)
    m, r = f64(mean), f64(rstd)  # what the backward pass is given
    rdx, rdw, rdb = om.layer_norm_backward(G, X, m, r, Wt)
    xh = np.abs((X - m[:, None]) * r[:, None])
    g = np.abs(G) * aw
    slack = g + g.mean(1, keepdims=True) + xh * (g * xh).mean(1, keepdims=True)
    within(f64(dx), rdx, out_w * np.abs(rdx) + (n + 8) * U * r[:, None] * slack + 1e-37, "dx")
    k = 2 * np.sqrt(N) + 64
    within(f64(dw), rdw, par_w * np.abs(rdw) + k * U * (np.abs(G) * (xh + 1)).sum(0) + 1e-37, "dweight")
    within(f64(db), rdb, par_w * np.abs(rdb) + k * U * np.abs(G).sum(0) + 1e-37, "dbias")
    assert dw.dtype == db.dtype == (torch.float32 if w is None else w.dtype)


@pytest.mark.parametrize("dtype,params", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("N,D", [(1, 1), (5, 1), (1, 7), (3, 64), (300, 8), (129, 50), (64, 63), (65, 65), (1000, 24), (31, 257), (17, 512), (9, 1000),
                                 (40, 1024), (7, 2049), (5, 4104), (3, 8191), (4, 30752), (2, 53792), (2, 70001), (2, 131088)])
def test_layer_norm(torch, pxr, N, D, dtype, params):
    rng = np.random.default_rng(N * 1000 + D)
    x = gpu(torch, rng.standard_normal((N, D)) * 1.5 + 0.4, dtype)
    w, b = gpu(torch, 1 + 0.2 * rng.standard_normal(D), params), gpu(torch, 0.3 * rng.standard_normal(D), params)
    check_norm(torch, pxr, x, w, b, gpu(torch, rng.standard_normal((N, D)), dtype))


@pytest.mark.parametrize("N,D", [(70000, 8), (20011, 64), (4099, 130), (2050, 777)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_of_many_rows(torch, pxr, N, D, dtype):
    rng = np.random.default_rng(D)
    check_norm(torch, pxr, gpu(torch, rng.standard_normal((N, D)), dtype), gpu(torch, 1 + 0.2 * rng.standard_normal(D)), None,
               gpu(torch, rng.standard_normal((N, D)), dtype))


@pytest.mark.parametrize("N,D,dtype", [(1500, 1299, "f32"), (1031, 2601, "bf16"), (1025, 4095, "f32"), (1024, 8000, "bf16"), (1030, 7777, "f32"),
                                       (1027, 12345, "bf16"), (1100, 9000, "f32"), (1033, 20002, "bf16"), (3, 160001, "f32"), (2, 300007, "bf16")])
def test_layer_norm_of_many_long_rows(torch, pxr, N, D, dtype):
    """Rows of a workgroup's, several at a time, and rows that no workgroup holds."""
    rng = np.random.default_rng(N + D)
    check_norm(torch, pxr, gpu(torch, rng.standard_normal((N, D), dtype=np.float32), dtype), gpu(torch, 1 + 0.2 * rng.standard_normal(D)),
               gpu(torch, rng.standard_normal(D)), gpu(torch, rng.standard_normal((N, D), dtype=np.float32), dtype))


@pytest.mark.parametrize("D,dtype", [(34001, "f32"), (70003, "f32"), (140003, "bf16")])
def test_layer_norm_of_the_longest_rows_in_place(torch, pxr, D, dtype):
    rng = np.random.default_rng(D)
    x, dy, w = gpu(torch, rng.standard_normal((7, D)), dtype), gpu(torch, rng.standard_normal((7, D)), dtype), gpu(torch, rng.standard_normal(D))
    y, mean, rstd = pxr.layer_norm(x, w)
    z = x.clone()
    pxr.layer_norm(z, w, out=z)
    assert torch.equal(z, y)
    got = pxr.layer_norm_backward(dy, x, mean, rstd, w)
    for alias in (0, 1):
        t = [dy.clone(), x.clone()]
        assert all(torch.equal(a, b) for a, b in zip(got, pxr.layer_norm_backward(t[0], t[1], mean, rstd, w, dx=t[alias])))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_without_parameters_and_of_any_leading_shape(torch, pxr, dtype):
    rng = np.random.default_rng(3)
    x, dy = gpu(torch, rng.standard_normal((5, 7, 48)), dtype), gpu(torch, rng.standard_normal((5, 7, 48)), dtype)
    check_norm(torch, pxr, x.view(35, 48), None, None, dy.view(35, 48))
    y, mean, rstd = pxr.layer_norm(x)
    assert y.shape == x.shape and mean.shape == rstd.shape == (5, 7)
    assert torch.equal(y.view(35, 48), pxr.layer_norm(x.view(35, 48))[0])
    assert torch.equal(pxr.layer_norm_backward(dy, x, mean, rstd)[0].view(35, 48),
                       pxr.layer_norm_backward(dy.view(35, 48), x.view(35, 48), mean.view(35), rstd.view(35))[0])
    one = pxr.layer_norm(x[0, 0])
    assert one[0].shape == (48,) and one[1].shape == () and torch.equal(one[0], y[0, 0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,pitch,first", [(64, 96, 0), (64, 96, 32), (64, 67, 1), (40, 48, 8), (333, 400, 3), (2048, 2056, 8), (30752, 30753, 1)])
def test_layer_norm_of_slices(torch, pxr, D, pitch, first, dtype):
    """Rows a stride apart, at any alignment: inputs and outputs, and nothing between the rows is written."""
    rng = np.random.default_rng(D + pitch)
    N = 23
    wide = [gpu(torch, rng.standard_normal((N, pitch)), dtype) for _ in range(4)]
    x, dy, y, dx = (t[:, first:first + D] for t in wide)
    w, b = gpu(torch, 1 + 0.2 * rng.standard_normal(D)), gpu(torch, rng.standard_normal(D))
    before = [t.clone() for t in wide]
    check_norm(torch, pxr, x, w, b, dy)
    _, mean, rstd = pxr.layer_norm(x, w, b, out=y)
    pxr.layer_norm_backward(dy, x, mean, rstd, w, dx=dx)
    assert torch.equal(y, pxr.layer_norm(x.contiguous(), w, b)[0])
    assert torch.equal(dx, pxr.layer_norm_backward(dy.contiguous(), x.contiguous(), mean, rstd, w)[0])
    for i, (t, o) in enumerate(zip(wide, before)):
        keep = torch.ones(pitch, dtype=torch.bool, device="cuda")
        if i >= 2:
            keep[first:first + D] = False
        assert torch.equal(t[:, keep], o[:, keep])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 333, 5000, 30752])
def test_layer_norm_in_place(torch, pxr, D, dtype):
    rng = np.random.default_rng(D)
    x, dy, w = gpu(torch, rng.standard_normal((50, D)), dtype), gpu(torch, rng.standard_normal((50, D)), dtype), gpu(torch, rng.standard_normal(D))
    y, mean, rstd = pxr.layer_norm(x, w)
    z = x.clone()
    pxr.layer_norm(z, w, out=z)
    assert torch.equal(z, y)
    dx, dw, db = pxr.layer_norm_backward(dy, x, mean, rstd, w)
    for alias in (0, 1):
        t = [dy.clone(), x.clone()]
        got = pxr.layer_norm_backward(t[0], t[1], mean, rstd, w, dx=t[alias])
        assert all(torch.equal(a, b) for a, b in zip(got, (dx, dw, db)))


@pytest.mark.parametrize("D", [50, 64, 512, 4096, 30752])
def test_layer_norm_far_from_zero_and_of_equal_values(torch, pxr, D):
    """The variance of a row that lies far from zero; a row of equal values, whose variance is nothing but eps."""
    rng = np.random.default_rng(D)
    x = rng.standard_normal((6, D)) + np.array([0, 1e2, -1e3, 1e4, 0, 0])[:, None]
    x[4], x[5] = 3.0, 0.0
    check_norm(torch, pxr, gpu(torch, x), None, None, None)
    y, _, rstd = pxr.layer_norm(gpu(torch, x))
    assert (y[4:] == 0).all() and (rstd[4:] - 1e-5 ** -0.5).abs().max() < 1e-3
    check_norm(torch, pxr, gpu(torch, x[:1]), None, None, None, eps=0.0)


@pytest.mark.parametrize("D", [8, 64, 300, 2048, 30752, 70000])
def test_layer_norm_rows_do_not_reach_each_other(torch, pxr, D):
    """A NaN or an infinity makes its own row NaN and no other."""
    rng = np.random.default_rng(D)
    x = gpu(torch, rng.standard_normal((12, D)))
    y, mean, rstd = pxr.layer_norm(x)
    bad = x.clone()
    bad[3, D // 2], bad[7, 0] = float("nan"), float("inf")
    yb, mb, rb = pxr.layer_norm(bad)
    keep = [i for i in range(12) if i not in (3, 7)]
    assert torch.equal(yb[keep], y[keep]) and torch.equal(mb[keep], mean[keep]) and torch.equal(rb[keep], rstd[keep])
    assert yb[3].isnan().all() and yb[7].isnan().all()
    dx = pxr.layer_norm_backward(x, x, mean, rstd)[0]
    assert torch.equal(pxr.layer_norm_backward(x, bad, mean, rstd)[0][keep], dx[keep])


def test_layer_norm_of_no_rows(torch, pxr):
    x, w = torch.empty((0, 40), device="cuda"), torch.ones(40, device="cuda")
    y, mean, rstd = pxr.layer_norm(x, w)
    assert y.shape == (0, 40) and mean.shape == (0,)
    dx, dw, db = pxr.layer_norm_backward(x, x, mean, rstd, w)
    assert dx.shape == (0, 40) and (dw == 0).all() and (db == 0).all()


def test_layer_norm_gradient_by_differences(torch, pxr):
    """The kernels' own forward pass, moved along a direction: third differences of the normalisation are of order h^2."""
    rng = np.random.default_rng(6)
    x, w, b, dy = (gpu(torch, rng.standard_normal(s)) for s in ((40, 200), 200, 200, (40, 200)))
    _, mean, rstd = pxr.layer_norm(x, w, b)
    dx, dw, db = pxr.layer_norm_backward(dy, x, mean, rstd, w)
    h = 1e-2

    def f(x_, w_, b_):
        return float((pxr.layer_norm(x_, w_, b_)[0].double() * dy.double()).sum())
    for grad, move in ((dx, lambda d: (x + d, w, b)), (dw, lambda d: (x, w + d, b)), (db, lambda d: (x, w, b + d))):
        d = gpu(torch, rng.standard_normal(tuple(grad.shape)))
        want = float((grad.double() * d.double()).sum())
        size = float((grad.double() * d.double()).square().sum().sqrt())
        # h^2 times third derivatives (order 1 a value), and 8000 roundings of y, in the root of their number, over h
        assert abs((f(*move(h * d)) - f(*move(-h * d))) / (2 * h) - want) < 3 * h * h * size + 8 * U * np.sqrt(8000.0) / h


@pytest.mark.parametrize("N,D", [(1, 100), (16, 256), (60, 64), (3, 1300), (2, 8000), (1, 30000), (500, 64), (40, 5000), (5, 40000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_sums_of_one_kind(torch, pxr, N, D, dtype):
    """dweight without dbias, dbias without dweight, neither: the same as of both, and what is not asked for is not written."""
    import ctypes as C
    rng = np.random.default_rng(N + D)
    x, dy = gpu(torch, rng.standard_normal((N, D)), dtype), gpu(torch, rng.standard_normal((N, D)), dtype)
    w = gpu(torch, rng.standard_normal(D))
    _, mean, rstd = pxr.layer_norm(x, w)
    both = pxr.layer_norm_backward(dy, x, mean, rstd, w)
    code = 1 if dtype == "bf16" else 0
    d = pxr.LayerNormDesc(code, 0, N, D, 0.0, D, D, D)
    need = C.c_size_t()
    assert pxr.lib().pxr_layer_norm_workspace(C.byref(d), C.byref(need)) == pxr.OK
    ws = torch.empty(max(16, need.value), dtype=torch.uint8, device="cuda")
    for want in ((1, 0), (0, 1), (0, 0)):
        dx = torch.empty_like(x)
        sums = [torch.full((D + 2,), 7.0, device="cuda") for _ in want]
        at = [s[1:].data_ptr() if k else None for s, k in zip(sums, want)]
        assert pxr.lib().pxr_layer_norm_backward(C.byref(d), dy.data_ptr(), x.data_ptr(), mean.data_ptr(), rstd.data_ptr(), w.data_ptr(), dx.data_ptr(),
                                                 *at, ws.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream) == pxr.OK
        assert torch.equal(dx, both[0])
        for s, k, ref in zip(sums, want, both[1:]):
            assert s[0] == 7 and s[-1] == 7
            assert torch.equal(s[1:-1], ref) if k else bool((s == 7).all())


def test_layer_norm_sums_have_one_order(torch, pxr):
    rng = np.random.default_rng(8)
    for N, D in ((5000, 64), (300, 30752), (70000, 33)):
        x, dy = gpu(torch, rng.standard_normal((N, D))), gpu(torch, rng.standard_normal((N, D)))
        _, mean, rstd = pxr.layer_norm(x)
        first = pxr.layer_norm_backward(dy, x, mean, rstd)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, pxr.layer_norm_backward(dy, x, mean, rstd)))


def test_layer_norm_sums_of_the_widest_rows(torch, pxr):
    """More columns than a launch that gives 32 threads to each could count in 32 bits."""
    D = 2 ** 27 + 1000
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, dy = (torch.randn((1, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    mean, rstd = torch.tensor([0.25], device="cuda"), torch.tensor([0.5], device="cuda")
    dx, dw, db = pxr.layer_norm_backward(dy, x, mean, rstd)
    assert torch.equal(db, dy[0].float())
    # (one product, rounded once: a power of two scales it, and x - 0.25 has at most 16 bits where it is not rounded itself)
    want = dy[0].double() * ((x[0].float() - 0.25) * 0.5).double()
    assert ((dw.double() - want).abs() <= U * want.abs()).all()
    assert dx.isfinite().all()


# ------------------------------------------------------------------ linear attention

def inputs(torch, rng, B, T, H, dk, dv, dtype, resets=0.05, state=True, layout="bthd"):
    """GPU tensors in one of the layouts that programs have, and their decays."""
    def make(d):
        x = rng.standard_normal((B, T, H, d))
        if layout == "bhtd":
            return gpu(torch, x.transpose(0, 2, 1, 3).copy(), dtype).transpose(1, 2)
        if layout == "tbhd":
            return gpu(torch, x.transpose(1, 0, 2, 3).copy(), dtype).transpose(0, 1)
        return gpu(torch, x, dtype)
    if layout == "fused":
        qkv = gpu(torch, rng.standard_normal((B, T, H * (2 * dk + dv))), dtype)
        q, k, v = (p.unflatten(-1, (H, -1)) for p in qkv.split([H * dk, H * dk, H * dv], -1))
    else:
        q, k, v = make(dk), make(dk), make(dv)
    r = torch.from_numpy(rng.random((B, T)) < resets).cuda() if resets else None
    s = gpu(torch, rng.standard_normal((B, H, dk, dv))) if state else None
    ld = np.float32(np.log1p(-0.5 ** np.linspace(1, 7, H)))
    return q, k, v, r, s, ld, make(dv) if layout != "fused" else gpu(torch, rng.standard_normal((B, T, H, dv)), dtype), gpu(torch, rng.standard_normal((B, H, dk, dv)))


def close(got, ref, mag, depth, bf16, what):
    if not ref.size:
        return
    bound = depth * U * mag + (W * mag + W * np.abs(ref) if bf16 else 0.0) + 1e-37
    within(got, ref, bound, what)
    rms = np.sqrt((ref ** 2).mean())
    if ref.size >= 64 and rms > 0:
        assert np.sqrt(((got - ref) ** 2).mean()) <= (W if bf16 else 2.0 ** -20) * rms, what


def check_attention(torch, pxr, q, k, v, r, s, ld, dout, ds, scale=None, backward=True):
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    bf16 = q.dtype == torch.bfloat16
    layer = pxr.LinearAttention(H, dk, dv, ld, scale=scale)
    Q, K, V = f64(q), f64(k), f64(v)
    R, S = None if r is None else r.cpu().numpy(), None if s is None else f64(s)
    out, last = layer.forward(q, k, v, resets=r, state=s)
    ref, rlast = om.linear_attention(Q, K, V, ld, layer.scale, R, S)
    mag, mlast = om.linear_attention(abs(Q), abs(K), abs(V), ld, abs(layer.scale), R, None if S is None else abs(S))
    close(f64(out), ref, mag, 64 + dk + T, bf16, "out")
    close(f64(last), rlast, mlast, 64 + T, False, "state")
    if backward:
        got = layer.backward(dout, q, k, v, resets=r, state=s, dstate=ds)
        args = (f64(dout), Q, K, V)
        D = None if ds is None else f64(ds)
        ref = om.linear_attention_backward(*args, ld, layer.scale, R, S, D)
        mag = om.linear_attention_backward(*(abs(a) for a in args), ld, abs(layer.scale), R, None if S is None else abs(S), None if D is None else abs(D))
        for name, g, rf, m in zip(("dq", "dk", "dv"), got, ref, mag):
            assert g.dtype == q.dtype
            close(f64(g), rf, m, 64 + max(dk, dv) + T, bf16, name)
        if s is None:
            assert got[3] is None
        else:
            close(f64(got[3]), ref[3], mag[3], 64 + T, False, "dstate")
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [128, 200, 330, 500, 580, 1100, 2300])
def test_attention_of_few_long_rollouts(torch, pxr, T, dtype):
    """Cut into 2 to 35 segments, whose states are joined a few at a time."""
    rng = np.random.default_rng(T)
    check_attention(torch, pxr, *inputs(torch, rng, 1, T, 1, 24, 16, dtype, resets=0.003))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,dk,dv", [(1, 700, 1, 64, 128), (2, 40, 3, 128, 64), (1, 900, 2, 16, 100), (3, 70, 2, 100, 33), (1, 600, 1, 200, 40), (2, 65, 1, 40, 250),
                                         (2, 33, 2, 32, 64), (1, 300, 2, 60, 30)])
def test_attention_of_keys_and_values_of_different_widths(torch, pxr, B, T, H, dk, dv, dtype):
    """Their gradients take kernels of their own; states whose last block of 32 rows is not whole, columns too."""
    rng = np.random.default_rng(T + dk)
    check_attention(torch, pxr, *inputs(torch, rng, B, T, H, dk, dv, dtype, resets=0.01))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 31, 32, 33, 63, 64, 65, 96, 127, 129, 200, 333])
def test_attention_lengths(torch, pxr, T, dtype):
    rng = np.random.default_rng(T)
    check_attention(torch, pxr, *inputs(torch, rng, 3, T, 2, 64, 64, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(1, 1), (1, 40), (8, 8), (16, 32), (32, 16), (31, 33), (33, 31), (48, 40), (64, 128), (128, 64), (96, 96), (100, 7), (128, 128), (255, 3), (5, 256),
                                   (256, 256)])
def test_attention_sizes_of_heads(torch, pxr, dk, dv, dtype):
    rng = np.random.default_rng(dk * 300 + dv)
    check_attention(torch, pxr, *inputs(torch, rng, 2, 75, 3, dk, dv, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bthd", "bhtd", "tbhd", "fused"])
@pytest.mark.parametrize("dk,dv", [(32, 64), (20, 12), (9, 11)])
def test_attention_layouts(torch, pxr, layout, dk, dv, dtype):
    rng = np.random.default_rng(dk)
    check_attention(torch, pxr, *inputs(torch, rng, 3, 70, 2, dk, dv, dtype, layout=layout))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("resets", [0.0, 0.02, 0.3, 1.0])
@pytest.mark.parametrize("state", [True, False])
def test_attention_resets_and_states(torch, pxr, resets, state, dtype):
    rng = np.random.default_rng(int(resets * 100))
    q, k, v, r, s, ld, dout, ds = inputs(torch, rng, 4, 150, 2, 32, 32, dtype, resets=resets, state=state)
    check_attention(torch, pxr, q, k, v, r, s, ld, dout, ds if state else None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_resets_at_the_edges_of_tiles(torch, pxr, dtype):
    rng = np.random.default_rng(1)
    q, k, v, r, s, ld, dout, ds = inputs(torch, rng, 8, 130, 1, 32, 32, dtype)
    r.zero_()
    for b, at in enumerate(([0], [1], [31, 32], [63], [64], [65, 128], [129], list(range(60, 70)))):
        r[b, at] = True
    check_attention(torch, pxr, q, k, v, r, s, ld, dout, ds)
    check_attention(torch, pxr, q, k, v, r.to(torch.uint8) * 255, s, ld, dout, ds)
    check_attention(torch, pxr, q, k, v, r.t().contiguous().t(), s, ld, dout, ds)
    check_attention(torch, pxr, q, k, v, r[:1].expand(8, -1), s, ld, dout, ds)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,dk,dv", [(1, 3000, 1, 32, 32), (1, 2500, 2, 64, 100), (2, 1111, 3, 40, 48), (1, 1500, 1, 200, 64)])
def test_attention_along_a_long_axis(torch, pxr, B, T, H, dk, dv, dtype):
    """Few rows: the axis of steps is what the work can be cut along."""
    rng = np.random.default_rng(T)
    check_attention(torch, pxr, *inputs(torch, rng, B, T, H, dk, dv, dtype, resets=0.002))
    check_attention(torch, pxr, *inputs(torch, rng, B, T, H, dk, dv, dtype, resets=0.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_decays(torch, pxr, dtype):
    """No decay at all, one that forgets within a step, one that underflows, one over thousands of steps."""
    rng = np.random.default_rng(2)
    q, k, v, r, s, _, dout, ds = inputs(torch, rng, 2, 200, 4, 32, 32, dtype, resets=0.01)
    check_attention(torch, pxr, q, k, v, r, s, np.float32([0.0, -1e-4, -3.0, -200.0]), dout, ds)
    check_attention(torch, pxr, q, k, v, None, s, np.float32([-0.0, -1e30, -0.7, -1e-30]), dout, ds, scale=-2.5)
    check_attention(torch, pxr, q, k, v, None, s, np.float32([-0.1] * 4), dout, ds, scale=0.0)


def test_attention_many_rows(torch, pxr):
    rng = np.random.default_rng(3)
    check_attention(torch, pxr, *inputs(torch, rng, 300, 20, 4, 32, 32, "bf16"))
    check_attention(torch, pxr, *inputs(torch, rng, 100, 70, 8, 16, 16, "f32"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_shared_heads_and_broadcast_inputs(torch, pxr, dtype):
    """Strides of zero: heads that share keys and values, environments that share everything.  The gradients of what is shared
    are the sums over those that share it, which a caller forms from the gradients of each."""
    rng = np.random.default_rng(4)
    q, k, v, r, s, ld, dout, ds = inputs(torch, rng, 3, 40, 4, 32, 16, dtype)
    check_attention(torch, pxr, q, k[:, :, :1].expand(-1, -1, 4, -1), v[:, :, 1:2].expand(-1, -1, 4, -1), r, s, ld, dout, ds)
    check_attention(torch, pxr, q[:1].expand(3, -1, -1, -1), k[:1].expand(3, -1, -1, -1), v, r, s, ld, dout[:, :1].expand(-1, 40, -1, -1), ds)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_without_steps(torch, pxr, dtype):
    rng = np.random.default_rng(5)
    q, k, v, r, s, ld, dout, ds = inputs(torch, rng, 3, 0, 2, 8, 12, dtype, resets=0.0)
    layer = pxr.LinearAttention(2, 8, 12, ld)
    out, last = layer.forward(q, k, v, state=s)
    assert out.shape == (3, 0, 2, 12) and torch.equal(last, s)
    assert (layer.forward(q, k, v)[1] == 0).all()
    dq, dk, dv, dfirst = layer.backward(dout, q, k, v, state=s, dstate=ds)
    assert dq.shape == dk.shape == (3, 0, 2, 8) and dv.shape == (3, 0, 2, 12) and torch.equal(dfirst, ds)
    assert (layer.backward(dout, q, k, v, state=s)[3] == 0).all()
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_attention_what_is_not_finite_reaches_only_later_steps_of_its_episode(torch, pxr, bad, dtype):
    rng = np.random.default_rng(6)
    q, k, v, r, s, ld, dout, ds = inputs(torch, rng, 2, 200, 2, 32, 32, dtype)
    r.zero_()
    r[0, 100] = True
    layer = pxr.LinearAttention(2, 32, 32, ld)
    out, last = layer.forward(q, k, v, resets=r, state=s)
    for which in ("k", "v"):
        x = dict(q=q, k=k.clone(), v=v.clone())
        x[which][0, 77, 1, 5] = bad
        o, e = layer.forward(x["q"], x["k"], x["v"], resets=r, state=s)
        keep = torch.ones(out.shape[:3], dtype=torch.bool, device="cuda")
        keep[0, 77:100, 1] = False
        # (a tile that holds such a value may be summed in another order)
        assert o[keep].isfinite().all() and (o[keep].float() - out[keep].float()).abs().max() <= 2 * W * out.float().abs().max()
        assert e.isfinite().all() and (e - last).abs().max() <= 2.0 ** -18 * last.abs().max()
        reached = o[0, 77:100, 1]  # (a value in v reaches its own column, one in k reaches them all)
        assert not (reached[:, 5] if which == "v" else reached).isfinite().any()
    # a state that is no number, cut off by an episode that begins
    broken = s.clone()
    broken[0, 0] = bad
    o, e = layer.forward(q, k, v, resets=r, state=broken)
    assert not o[0, :100, 0].isfinite().any() and o[0, 100:].isfinite().all() and o[0, :, 1].isfinite().all() and e.isfinite().all()
    # gradients: what reaches a step comes from the later steps of its episode
    d = dout.clone()
    d[0, 50, 1, 3] = bad
    dq, dk, dv, dfirst = layer.backward(d, q, k, v, resets=r, state=s, dstate=ds)
    for g in (dk, dv):
        assert g[0, 51:, 1].isfinite().all() and g[0, :, 0].isfinite().all() and g[1].isfinite().all()
    assert dq[0, :50, 1].isfinite().all() and dq[0, 51:, 1].isfinite().all() and not dq[0, 50, 1].isfinite().any()
    assert not dv[0, :51, 1, 3].isfinite().any() and not dk[0, :51, 1].isfinite().any()
    assert dfirst[0, 0].isfinite().all() and dfirst[1].isfinite().all() and not dfirst[0, 1, :, 3].isfinite().any()
    d = ds.clone()
    d[0, 0] = bad
    dq, dk, dv, dfirst = layer.backward(dout, q, k, v, resets=r, state=s, dstate=d)
    assert dk[0, :100].isfinite().all() and not dk[0, 100:, 0].isfinite().any() and dq.isfinite().all() and dfirst.isfinite().all()
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("B,T,at", [(2, 20, 0), (2, 20, 7), (2, 63, 32), (2, 200, 100), (2, 200, 0), (1, 1500, 640), (1, 1500, 701)])
def test_attention_what_is_not_finite_in_a_step_that_begins_an_episode_stays_in_it(torch, pxr, B, T, at, bad, dtype):
    """Nothing passes an episode's beginning, forward or backward, whole rollouts and such that are cut into segments: what is
    before it is as near to the definition as it is without that value."""
    rng = np.random.default_rng(T + at)
    q, k, v, r, s, ld, dout, ds = inputs(torch, rng, B, T, 2, 32, 32, dtype)
    r.zero_()
    r[0, at] = True
    if at:
        r[0, at - 1] = True  # an episode of one step before it
    layer = pxr.LinearAttention(2, 32, 32, ld)
    args = [f64(x) for x in (dout, q, k, v)]
    R, S, D = r.cpu().numpy(), f64(s), f64(ds)
    ref = om.linear_attention_backward(*args, ld, layer.scale, R, S, D)
    mag = om.linear_attention_backward(*(abs(a) for a in args), ld, abs(layer.scale), R, abs(S), abs(D))
    bf16 = dtype == "bf16"
    for which in range(4):
        x = [t.clone() for t in (dout, q, k, v)]
        x[which][0, at, 1, 5] = bad
        got = layer.backward(*x, resets=r, state=s, dstate=ds)
        for name, g, rf, m in zip(("dq", "dk", "dv"), got, ref, mag):
            keep = np.ones((B, T, 2), bool)
            # the step itself; q and dout reach no other step's dq, k and v reach those of later steps of the episode
            keep[0, at if which < 2 or name != "dq" else slice(at, None), 1] = False
            close(f64(g)[keep], rf[keep], m[keep], 64 + 32 + T, bf16, (which, name))
        close(f64(got[3]), ref[3], mag[3], 64 + T, False, (which, "dstate"))
        if at == 0:
            assert (got[3][0] == 0).all(), which
    layer.close()


@pytest.mark.parametrize("B,T,H,dk,dv", [(3, 90, 2, 32, 32), (1, 640, 1, 64, 64), (2, 33, 2, 24, 100), (2, 70, 1, 128, 96), (1, 40, 1, 100, 40)])
@pytest.mark.parametrize("large", ["probabilities", "states"])
def test_attention_of_whole_numbers_is_exact_up_to_the_outputs_rounding(torch, pxr, large, B, T, H, dk, dv):
    """bfloat16 inputs that are whole numbers, no decay: every sum stays below 2^24, so that fp32 holds it, and an output is the
    definition's, rounded once.  Probabilities and states of 17 bits and more nearly cancel in it, so that less than all of their
    bits would not do: keys and queries of 8 bits come in pairs that differ by one, with values and gradients of opposite sign; or the
    states are one large odd number and a few more or less, and what they are multiplied with adds up to nothing."""
    rng = np.random.default_rng(dk + T)

    def whole(*shape, most):
        return rng.integers(-most, most + 1, shape).astype(np.float64)
    r = np.zeros((B, T), bool)
    r[:, 2 * rng.integers(1, T // 2, B)] = True
    if large == "probabilities":
        q, k, v, dout = (np.zeros((B, T, H, d)) for d in (dk, dk, dv, dv))
        at = rng.choice(dk, 4, replace=False)
        for x, y in ((k, v), (q, dout)):
            x[:, ::2, :, at] = 255 - rng.integers(0, 9, x[:, ::2, :, at].shape)
            y[:, ::2] = whole(*y[:, ::2].shape, most=1) * (rng.random(y[:, ::2].shape) < 8 / T)
            pairs = T // 2
            x[:, 1:2 * pairs:2], y[:, 1:2 * pairs:2] = x[:, :2 * pairs:2], -y[:, :2 * pairs:2]
            x[:, 1:2 * pairs:2, :, at[0]] -= 1
        s, ds = whole(B, H, dk, dv, most=3), whole(B, H, dk, dv, most=3)
    else:
        def paired(d):
            x, at = np.zeros((B, T, H, d)), 2 * rng.choice(d // 2, 4, replace=False)
            x[..., at] = whole(B, T, H, 4, most=1)
            x[..., at + 1] = -x[..., at]
            return x
        q, k, v, dout = paired(dk), paired(dk), paired(dv), paired(dv)
        big = 2 ** 20 - 2 ** 13 + 2411
        s, ds = big + whole(B, H, dk, dv, most=9), big + whole(B, H, dk, dv, most=9)
    ld = np.zeros(H, np.float32)
    ref = (*om.linear_attention(q, k, v, ld, 1.0, r, s), *om.linear_attention_backward(dout, q, k, v, ld, 1.0, r, s, ds))
    mags = [abs(x) for x in (q, k, v)]
    most = (*om.linear_attention(*mags, ld, 1.0, r, abs(s)), *om.linear_attention_backward(abs(dout), *mags, ld, 1.0, r, abs(s), abs(ds)))
    assert max(m.max() for m in most) < 2 ** 24
    if large == "probabilities":
        assert np.einsum("bihd,bjhd->bhij", q[:, :9], k[:, :9]).max() > 2 ** 17
    else:
        assert np.abs(s).min() > 2 ** 19
    Q, K, V, DO = (gpu(torch, x, "bf16") for x in (q, k, v, dout))
    layer, R = pxr.LinearAttention(H, dk, dv, ld, scale=1.0), torch.from_numpy(r).cuda()
    got = (*layer.forward(Q, K, V, resets=R, state=gpu(torch, s)), *layer.backward(DO, Q, K, V, resets=R, state=gpu(torch, s), dstate=gpu(torch, ds)))
    for name, g, rf in zip(("out", "state", "dq", "dk", "dv", "dstate"), got, ref):
        assert torch.equal(g, torch.from_numpy(rf).cuda().float().to(g.dtype)), name
    layer.close()


def test_attention_gradients_by_differences(torch, pxr):
    """The kernels' own forward pass, moved along a direction.  It is linear in each input alone, so the difference over any
    distance is the derivative; the directions are small, so that roundings are those of the results themselves."""
    rng = np.random.default_rng(7)
    q, k, v, r, s, ld, dout, ds = inputs(torch, rng, 2, 90, 2, 24, 40, "f32")
    layer = pxr.LinearAttention(2, 24, 40, ld)
    grads = layer.backward(dout, q, k, v, resets=r, state=s, dstate=ds)

    def f(*x):
        out, last = layer.forward(*x[:3], resets=r, state=x[3])
        return float((out.double() * dout.double()).sum() + (last.double() * ds.double()).sum())
    for i, g in enumerate(grads):
        d = gpu(torch, rng.standard_normal(tuple(g.shape)))
        up, down = [q, k, v, s], [q, k, v, s]
        up[i], down[i] = up[i] + d, down[i] - d
        want = float((g.double() * d.double()).sum())
        size = float((g.double() * d.double()).square().sum().sqrt())
        assert abs((f(*up) - f(*down)) / 2 - want) <= 2.0 ** -14 * size
    layer.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,dk,dv", [(1, 1, 1, 1), (3, 2, 64, 64), (5, 3, 33, 31), (2, 4, 128, 100), (300, 4, 32, 32), (2, 1, 256, 256), (7, 2, 16, 8), (1, 16, 128, 128), (2, 2, 3, 130)])
def test_step_equals_a_rollout(torch, pxr, B, H, dk, dv, dtype):
    """Acting step by step, the state updated in place, against the definition of the whole rollout."""
    rng = np.random.default_rng(B + dk)
    T = 6
    q, k, v, r, s, ld, _, _ = inputs(torch, rng, B, T, H, dk, dv, dtype, resets=0.2)
    layer = pxr.LinearAttention(H, dk, dv, ld)
    state = s.clone()
    out = torch.stack([layer.step(q[:, t], k[:, t], v[:, t], state, resets=r[:, t]) for t in range(T)], 1)
    args = (f64(q), f64(k), f64(v))
    ref, rlast = om.linear_attention(*args, ld, layer.scale, r.cpu().numpy(), f64(s))
    mag, mlast = om.linear_attention(*(abs(a) for a in args), ld, layer.scale, r.cpu().numpy(), abs(f64(s)))
    close(f64(out), ref, mag, 64 + dk + T, dtype == "bf16", "out")
    close(f64(state), rlast, mlast, 64 + T, False, "state")
    one, last = layer.forward(q, k, v, resets=r, state=s)
    close(f64(one), ref, mag, 64 + dk + T, dtype == "bf16", "rollout")
    alone = s.clone()
    assert torch.equal(layer.step(q[:, 0], k[:, 0], v[:, 0], alone), layer.step(q[:, 0], k[:, 0], v[:, 0], s.clone(), resets=torch.zeros_like(r[:, 0])))
    layer.close()


def test_step_a_reset_drops_whatever_the_state_held(torch, pxr):
    rng = np.random.default_rng(9)
    q, k, v, _, s, ld, _, _ = inputs(torch, rng, 3, 1, 2, 40, 24, "f32")
    layer = pxr.LinearAttention(2, 40, 24, ld)
    s[1] = float("nan")
    s[2, 0, 3] = float("inf")
    r = torch.tensor([False, True, True], device="cuda")
    out = layer.step(q[:, 0], k[:, 0], v[:, 0], s, resets=r)
    assert out.isfinite().all() and s.isfinite().all()
    assert torch.equal(s[1:], k[1:, 0, :, :, None] * v[1:, 0, :, None, :])
    layer.close()


def test_attention_looks_back_over_thousands_of_steps_alike_in_both_forms(torch, pxr):
    """The decay's own rounding would add up (u a step): both forms stay with the definition."""
    rng = np.random.default_rng(10)
    T = 4000
    q, k, v, _, s, _, _, _ = inputs(torch, rng, 1, T, 1, 16, 16, "f32", resets=0.0)
    ld = np.float32([np.log1p(-1 / 5000)])
    layer = pxr.LinearAttention(1, 16, 16, ld)
    s *= 100.0
    state = s.clone()
    for t in range(T):
        layer.step(q[:, t], k[:, t], v[:, t], state)
    ref, rlast = om.linear_attention(f64(q), f64(k), f64(v), ld, layer.scale, None, f64(s))
    size = np.sqrt((rlast ** 2).mean())
    # T roundings of u / sqrt(3) each, independent: sqrt(T / 3) u = 2.2e-6
    assert np.sqrt(((f64(state) - rlast) ** 2).mean()) < 3e-6 * size
    assert np.sqrt(((f64(layer.forward(q, k, v, state=s)[1]) - rlast) ** 2).mean()) < 3e-6 * size
    layer.close()


# ------------------------------------------------------------------ how it is called

def test_memory_on_another_stream_and_in_a_graph(torch, pxr):
    """Outputs and workspaces on a stream of the caller's; the calls recorded in a graph, replayed with eager work between."""
    rng = np.random.default_rng(11)
    q, k, v, r, s, ld, dout, ds = inputs(torch, rng, 2, 700, 2, 64, 64, "bf16", resets=0.01)
    layer = pxr.LinearAttention(2, 64, 64, ld)
    w = gpu(torch, rng.standard_normal(64))

    def all_of_it(stream=None):
        out, last = layer.forward(q, k, v, resets=r, state=s, stream=stream)
        y, mean, rstd = pxr.layer_norm(out, w, stream=stream)
        dy, dw, db = pxr.layer_norm_backward(dout, out, mean, rstd, w, stream=stream)
        return [out, last, y, mean, rstd, dy, dw, db, *layer.backward(dy, q, k, v, resets=r, state=s, dstate=ds, stream=stream)]

    want = [t.clone() for t in all_of_it()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = all_of_it(side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    other = torch.from_numpy(rng.standard_normal(tuple(q.shape)).astype(np.float32)).cuda().to(q.dtype)
    first = q.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of_it()
    for trial in range(6):
        q.copy_(first if trial % 2 == 0 else other)
        for t in got:
            t.fill_(1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = all_of_it()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), trial
    layer.close()


def test_attention_gives_equal_bits_for_equal_inputs(torch, pxr):
    rng = np.random.default_rng(12)
    for B, T in ((1, 2000), (40, 100)):
        q, k, v, r, s, ld, dout, ds = inputs(torch, rng, B, T, 2, 64, 64, "bf16")
        layer = pxr.LinearAttention(2, 64, 64, ld)
        first = (*layer.forward(q, k, v, resets=r, state=s), *layer.backward(dout, q, k, v, resets=r, state=s, dstate=ds))
        for _ in range(3):
            again = (*layer.forward(q, k, v, resets=r, state=s), *layer.backward(dout, q, k, v, resets=r, state=s, dstate=ds))
            assert all(torch.equal(a, b) for a, b in zip(first, again))
        layer.close()


def test_attention_refusals(torch, pxr):
    rng = np.random.default_rng(13)
    q, k, v, r, s, ld, dout, ds = inputs(torch, rng, 2, 600, 2, 16, 24, "f32")
    layer = pxr.LinearAttention(2, 16, 24, ld)
    for wrong in (lambda: layer.forward(q[..., :8], k, v), lambda: layer.forward(q, k, v.to(torch.bfloat16)), lambda: layer.forward(q, k, v, state=s.double()),
                  lambda: layer.forward(q, k, v, resets=r.float()), lambda: layer.forward(q, k, v, resets=r[:1]), lambda: layer.forward(q.half(), k.half(), v.half()),
                  lambda: layer.forward(q, k, v, state=s.transpose(0, 1)), lambda: layer.forward(q.transpose(2, 3), k, v), lambda: layer.step(q[:, 0], k[:, 0], v, s),
                  lambda: layer.forward(q[:, :, :1], k, v), lambda: layer.forward(q.cpu(), k, v)):
        with pytest.raises((AssertionError, RuntimeError)):
            wrong()
    with pytest.raises(pxr.PxrError) as e:
        layer.forward(q, k, v, state=s, state_out=s)
    assert e.value.code == pxr.ERR_INVALID_ARG and "overlap" in str(e.value)
    # the C calls themselves
    import ctypes as C
    L = pxr.lib()
    packed = layer._rollout(torch, q, k, v, r, s)[0]
    assert len(packed) == C.sizeof(pxr.Rollout)
    roll = pxr.Rollout.from_buffer_copy(packed)
    assert (roll.n_envs, roll.n_steps, roll.q.data, roll.v.head, roll.resets_step, roll.d_state) == (2, 600, q.data_ptr(), 24, 1, s.data_ptr())
    out = torch.empty_like(v)
    view = pxr.Tokens(out.data_ptr(), *out.stride()[:3])
    need = C.c_size_t()
    assert L.pxr_linear_attention_workspace(layer._h, 0, 2, 600, 1, C.byref(need)) == 0
    ws = torch.empty(need.value + 16, dtype=torch.uint8, device="cuda")

    def forward(h=layer._h, roll=roll, view=view, ws=ws.data_ptr(), n=need.value):
        return L.pxr_linear_attention_forward(h, C.byref(roll) if roll is not None else None, C.byref(view) if view is not None else None, None, ws, n, None)
    assert forward() == 0
    assert forward(h=None) == forward(roll=None) == forward(view=None) == pxr.ERR_INVALID_ARG
    for field, value in (("dtype", 2), ("n_envs", 0), ("n_envs", 2 ** 31), ("n_steps", 2 ** 31), ("q", pxr.Tokens()), ("v", pxr.Tokens(v.data_ptr() + 2, 0, 0, 0)), ("d_state", s.data_ptr() + 2)):
        other = pxr.Rollout.from_buffer_copy(roll)
        setattr(other, field, value)
        assert forward(roll=other) == pxr.ERR_INVALID_ARG, field
    if need.value:
        assert L.pxr_linear_attention_backward(layer._h, C.byref(roll), C.byref(view), None, *[C.byref(view)] * 3, None, ws.data_ptr() + 1, need.value, None) == pxr.ERR_INVALID_ARG
        assert L.pxr_linear_attention_backward(layer._h, C.byref(roll), C.byref(view), None, *[C.byref(view)] * 3, None, ws.data_ptr(), need.value - 1, None) == pxr.ERR_INVALID_ARG
        assert L.pxr_linear_attention_backward(layer._h, C.byref(roll), C.byref(view), None, *[C.byref(view)] * 3, None, None, need.value, None) == pxr.ERR_INVALID_ARG
    assert L.pxr_linear_attention_step(layer._h, C.byref(roll), s.data_ptr(), C.byref(view), None) == pxr.ERR_INVALID_ARG  # 600 steps
    torch.cuda.synchronize()
    layer.close()
