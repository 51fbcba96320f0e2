"""A learner's update on the GPU against the float64 definition.

Tolerances, from the arithmetic.  u = 2^-24, w = 2^-8 half a unit of fp32 and bfloat16.  How much an error of a step grows up to the last one goes by the matrix and the
coefficients; what the same steps in plain fp32 are off by on the same matrix, e, measures it: fp32 rounds every value and every sum once, by u.  Here a value is held to
2 u (two fp16 parts), a product leaves out up to 4 u (lo lo), and a sum of K products is 3 K / 16 instructions long, whose roundings add up like their root.  So the result may be off by
(8 + sqrt(3 K / 16)) max(e, 2 u), K the longer side, relative in the Frobenius norm; and w more in bfloat16.
"""
import numpy as np
import pytest

from oracle import learner

pytestmark = pytest.mark.gpu

U, W = 2.0 ** -24, 2.0 ** -8
QUINTIC = (3.4445, -4.7750, 2.0315)
FIVE = [tuple(float(np.float32(c)) for c in QUINTIC)] * 5


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


def plain(torch, x, coefficients, eps, dtype):
    """The definition by PyTorch's products in `dtype`."""
    x = x.to(dtype)
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    x = x / (x.double().square().sum().sqrt().to(dtype) + eps)
    for a, b, c in coefficients:
        gram = x @ x.t().contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if tall else x


def check(torch, pxr, x, coefficients=FIVE, eps=1e-7, out=None, got=None):
    """x [m,n] or [B,m,n] on the GPU."""
    y = pxr.orthogonalise(x, coefficients=coefficients, eps=eps, out=out) if got is None else got
    assert y.shape == x.shape and y.dtype == x.dtype
    for m, g in zip(x if x.dim() == 3 else [x], y if x.dim() == 3 else [y]):
        if m.numel() <= 1 << 16:
            ref = torch.from_numpy(learner.orthogonalise(m.double().cpu().numpy(), coefficients, eps)).cuda()
        else:
            ref = plain(torch, m, coefficients, eps, torch.float64)
        norm = float(ref.norm())
        e = float((plain(torch, m, coefficients, eps, torch.float32).double() - ref).norm()) / norm
        off = float((g.double() - ref).norm()) / norm
        allowed = (8 + np.sqrt(3 * max(m.shape) / 16)) * max(e, 2 * U) + (W if x.dtype == torch.bfloat16 else 0)
        assert off <= allowed, (tuple(x.shape), off, allowed, e)
    return y


def normal(torch, seed, *shape, dtype="f32", scale=1e-3):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 7), (9, 1), (2, 2), (5, 3), (31, 33), (64, 64), (65, 63), (64, 96), (96, 64), (127, 129), (128, 128), (130, 200), (256, 64), (48, 1000), (300, 301),
                                 (500, 257), (513, 700)])
def test_sizes(torch, pxr, m, n, dtype):
    check(torch, pxr, normal(torch, m * 1000 + n, m, n, dtype=dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,m,n", [(3, 64, 96), (5, 17, 9), (2, 200, 1500), (9, 130, 128), (2, 5, 20000), (8, 1000, 1030), (300, 33, 20)])
def test_batches(torch, pxr, B, m, n, dtype):
    x = normal(torch, B, B, m, n, dtype=dtype) * torch.linspace(0.5, 100, B, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)[:, None, None]
    y = check(torch, pxr, x[:12])
    assert torch.equal(y[0], pxr.orthogonalise(x[:12])[0])
    whole = pxr.orthogonalise(x)
    check(torch, pxr, x[-3:], got=whole[-3:])


@pytest.mark.parametrize("m,n,dtype", [(64, 30000, "f32"), (20011, 256, "f32"), (30752, 256, "bf16"), (1500, 4000, "f32"), (2050, 2100, "bf16"), (3001, 3000, "f32"), (4, 200000, "f32")])
def test_large(torch, pxr, m, n, dtype):
    check(torch, pxr, normal(torch, n, m, n, dtype=dtype))


@pytest.mark.parametrize("B,m,n,dtype", [(1, 3601, 3590, "f32"), (1, 3600, 5003, "bf16"), (28, 1020, 1030, "f32"), (4, 2050, 2060, "bf16")])
def test_tiles_of_both_sizes(torch, pxr, B, m, n, dtype):
    """Around the numbers of tiles from which on symmetric products take larger ones."""
    x = normal(torch, n, B, m, n, dtype=dtype)
    got = pxr.orthogonalise(x)
    check(torch, pxr, x[:2], got=got[:2])
    check(torch, pxr, x[-2:], got=got[-2:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,m,n", [(1, 1, 3000), (2, 2001, 1), (1, 5, 30000), (4, 14982, 5), (1, 16, 2500), (3, 17, 4097), (1, 28196, 31), (1, 32, 1300), (2, 1301, 32), (1, 32, 100000), (70, 20, 1500), (1, 33, 2000), (2, 20, 320), (2, 321, 20),
                                   (3000, 3, 1300)])
def test_long_matrices_of_few_rows(torch, pxr, B, m, n, dtype):
    x = normal(torch, m + n, B, m, n, dtype=dtype)
    got = pxr.orthogonalise(x)
    check(torch, pxr, x[:3], got=got[:3])
    check(torch, pxr, x[-1], got=got[-1])
    again = x.clone()
    pxr.orthogonalise(again, out=again)
    assert torch.equal(again, got)
    assert (pxr.orthogonalise(torch.zeros_like(x[:2])) == 0).all()


def test_long_matrices_as_updates_have_them(torch, pxr):
    """Singular values that lie far apart, a rank of one, rows of zeros, any scale, other steps, and what is not finite."""
    m, n = 24, 5000
    u, v = torch.linalg.qr(normal(torch, 2, m, m).double())[0], torch.linalg.qr(normal(torch, 3, n, m).double())[0]
    apart = ((u * torch.logspace(0, -4, m, device="cuda", dtype=torch.float64)) @ v.t().contiguous()).float()
    one = (u[:, :1] @ v[:, :1].t().contiguous()).float()
    rows = normal(torch, 4, m, n)
    rows[::3] = 0
    for x in (apart, one, rows, apart * 1e-30, apart * 1e30, rows * 1e-20):
        check(torch, pxr, x, eps=0.0)
        check(torch, pxr, x.t().contiguous(), eps=0.0)
        for c in ([QUINTIC], [(1.5, -0.5, 0.0)] * 12, [(3.0, -3.2, 1.2), (2.5, -2.0, 0.5), (1.5, -0.5, 0.0)], [(0.5, 0.0, 0.0)]):
            check(torch, pxr, x, [tuple(float(np.float32(v)) for v in t) for t in c], eps=0.0)
    x = torch.stack([rows, apart, one])
    want = pxr.orthogonalise(x)
    for value in (float("nan"), float("inf"), -float("inf")):
        bad = x.clone()
        bad[1, m // 2, n // 3] = value
        for c in ([QUINTIC] * 2, [(1.5, -0.5, 0.0)], [(0.5, 0.0, 0.0)]):
            got = pxr.orthogonalise(bad, coefficients=c)
            assert got[1].isnan().all() and got[0].isfinite().all() and got[2].isfinite().all()
        got = pxr.orthogonalise(bad)
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("m,n", [(60, 90), (300, 200)])
def test_coefficients(torch, pxr, m, n):
    """Cubic and quintic steps, few and many, of factors far from one, and another triple in every step."""
    x = normal(torch, 1, m, n)
    for c in ([QUINTIC], [QUINTIC] * 2, [(1.5, -0.5, 0.0)] * 12, [(15 / 8, -10 / 8, 3 / 8)] * 8, [(3.0, -3.2, 1.2), (2.5, -2.0, 0.5), (1.5, -0.5, 0.0)], [(0.5, 0.0, 0.0)], [(100.0, 0.0, 0.0)],
              [(0.0, 1.0, 0.0)], [(-2.0, 1.0, 0.5)] * 2, [(1e-3, 0.0, 0.0), (1e3, 0.0, 0.0)]):
        check(torch, pxr, x, [tuple(float(np.float32(v)) for v in t) for t in c])
    assert torch.equal(pxr.orthogonalise(x), pxr.orthogonalise(x, coefficients=[QUINTIC] * 5))
    assert torch.equal(pxr.orthogonalise(x, steps=3), pxr.orthogonalise(x, 3, list(QUINTIC)))
    assert (pxr.orthogonalise(x, coefficients=[(0.0, 0.0, 0.0)] * 3) == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(96, 64), (140, 300)])
def test_matrices_as_updates_have_them(torch, pxr, m, n, dtype):
    """Singular values that lie far apart, a rank of one, rows of zeros, values far from each other, any scale."""
    r = min(m, n)
    u, v = torch.linalg.qr(normal(torch, 2, m, r).double())[0], torch.linalg.qr(normal(torch, 3, n, r).double())[0]
    to = torch.bfloat16 if dtype == "bf16" else torch.float32
    apart = (u * torch.logspace(0, -4, r, device="cuda", dtype=torch.float64)) @ v.t().contiguous()
    check(torch, pxr, apart.to(to))
    check(torch, pxr, (u[:, :1] @ v[:, :1].t().contiguous()).to(to))
    check(torch, pxr, torch.eye(m, n, device="cuda").to(to))
    x = normal(torch, 4, m, n, dtype=dtype)
    x[::3] = 0
    check(torch, pxr, x)
    x = normal(torch, 4, m, n, dtype=dtype)
    x[:, ::2] *= 2.0 ** -10
    check(torch, pxr, x)
    for scale in (1e-30, 1e-18, 1e18, 1e30):
        check(torch, pxr, normal(torch, 5, m, n, dtype=dtype, scale=scale), eps=0.0)
    assert (pxr.orthogonalise(torch.zeros((m, n), device="cuda", dtype=to)) == 0).all()
    assert (pxr.orthogonalise(normal(torch, 5, m, n, dtype=dtype, scale=1e-30)).abs() < 1e-12).all()  # eps is what it is divided by


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,m,n,pitch", [(3, 40, 30, 33), (2, 130, 257, 300), (1, 300, 64, 65)])
def test_strides_in_place_and_nothing_else_written(torch, pxr, B, m, n, pitch, dtype):
    wide = normal(torch, m, B, m + 2, pitch, dtype=dtype)
    x = wide[:, 1:-1, 2:2 + n]
    if x.shape[-1] < n:
        x = wide[:, 1:-1, 1:1 + n]
    want = check(torch, pxr, x.contiguous())
    assert torch.equal(pxr.orthogonalise(x), want)
    into = torch.full((B + 1, m + 3, pitch + 1), 7.0, device="cuda", dtype=x.dtype)
    view = into[:B, 2:2 + m, 1:1 + n]
    assert torch.equal(pxr.orthogonalise(x, out=view), want)
    view.fill_(7.0)
    assert (into == 7).all()
    before = wide.clone()
    pxr.orthogonalise(x, out=x)
    assert torch.equal(x, want)
    x.copy_(before[:, 1:-1, x.storage_offset() % pitch:][..., :n])
    assert torch.equal(wide, before)
    # a batch that shares its input
    shared = before[:1, 1:-1, :n].expand(3, -1, -1)
    y = pxr.orthogonalise(shared)
    assert torch.equal(y[0], y[2]) and torch.equal(y[0], pxr.orthogonalise(before[0, 1:-1, :n]))


@pytest.mark.parametrize("m,n", [(30, 50), (200, 140), (40, 9000)])
def test_what_is_not_finite_stays_in_its_matrix(torch, pxr, m, n):
    x = normal(torch, m, 3, m, n)
    want = pxr.orthogonalise(x)
    for value in (float("nan"), float("inf"), -float("inf")):
        bad = x.clone()
        bad[1, m // 2, n // 3] = value
        y = pxr.orthogonalise(bad)
        assert torch.equal(y[0], want[0]) and torch.equal(y[2], want[2]) and y[1].isnan().all()


def test_offsets_past_32_bits(torch, pxr):
    x = normal(torch, 6, 2, 70, 50, dtype="bf16")
    want = pxr.orthogonalise(x)
    apart, row = 2 ** 31 + 64, 2 ** 24
    big = torch.empty(apart + 69 * row + 64, device="cuda", dtype=torch.bfloat16)
    view = big.as_strided(x.shape, (apart, row, 1), 5)
    view.copy_(x)
    assert torch.equal(pxr.orthogonalise(view), want)
    pxr.orthogonalise(x, out=view)
    assert torch.equal(view, want)


def test_streams_graphs_and_equal_bits(torch, pxr):
    for shape in ((3, 64, 96), (700, 300), (40, 9000)):
        sets = [normal(torch, i, *shape) for i in range(4)]
        want = [pxr.orthogonalise(x) for x in sets]
        for _ in range(3):
            assert torch.equal(pxr.orthogonalise(sets[0]), want[0])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = pxr.orthogonalise(sets[1], stream=side.cuda_stream)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want[1])
        static = sets[0].clone()
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                graphs.append((g, pxr.orthogonalise(static)))
        for i in (1, 2, 3, 0, 2):
            static.copy_(sets[i])
            for g, y in graphs:
                g.replay()
                eager = pxr.orthogonalise(sets[(i + 1) % 4])
                torch.cuda.synchronize()
                assert torch.equal(y, want[i]) and torch.equal(eager, want[(i + 1) % 4])


def test_refusals(torch, pxr):
    x = normal(torch, 7, 20, 30)
    for bad in (dict(x=x.half()), dict(x=x.cpu()), dict(x=x[0]), dict(x=x.t()), dict(x=x[None, None]), dict(x=x[:0]), dict(out=torch.empty_like(x)[:19]), dict(out=torch.empty_like(x).bfloat16()),
                dict(coefficients=(1.0, 2.0)), dict(coefficients=[QUINTIC] * 3, steps=4), dict(out=torch.empty((30, 20), device="cuda").t())):
        a = dict(dict(x=x), **bad)
        with pytest.raises(AssertionError):
            pxr.orthogonalise(a.pop("x"), **a)
    for bad, why in ((dict(steps=0), "n_steps"), (dict(steps=65), "n_steps"), (dict(eps=-1.0), "eps"), (dict(coefficients=(100.0, 0.0, 0.0)), "2\\^20"), (dict(coefficients=(float("nan"), 0.0, 0.0)), "finite")):
        with pytest.raises(pxr.PxrError, match=why):
            pxr.orthogonalise(x, **bad)
    with pytest.raises(pxr.PxrError, match="overlap"):
        pxr.orthogonalise(x[None].expand(2, -1, -1), out=x[None].expand(2, -1, -1))
    assert pxr.orthogonalise(torch.empty((0, 5, 6), device="cuda")).shape == (0, 5, 6)


def _of_rank(rng, m, n, rank, whole):
    """[m,n] of this rank but for fp32's rounding, or of whole numbers small enough for bfloat16, and of this rank exactly."""
    if whole:
        return (rng.integers(-1, 2, (m, rank)) @ rng.integers(-4, 5, (rank, n))).astype(np.float32)
    return (rng.standard_normal((m, rank)) @ rng.standard_normal((rank, n))).astype(np.float32)


def _in_80_bits(x, coefficients):
    x = x.astype(np.longdouble)
    x = x / np.sqrt((x ** 2).sum())
    for a, b, c in coefficients:
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.astype(np.float64)


@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("step,n_steps", [(QUINTIC, 6), (QUINTIC, 7), (QUINTIC, 14), (QUINTIC, 16), (QUINTIC, 24), (QUINTIC, 64), ((1.5, -0.5, 0.0), 24), ((1.5, -0.5, 0.0), 40), ((1.5, -0.5, 0.0), 64)])
def test_long_matrices_of_lower_rank_take_many_steps(torch, pxr, step, n_steps, tall):
    """As where a batch had fewer examples than the matrix has rows.  In every step that a singular value is far below one it is multiplied by 3.4 (1.5), and the definition's own roundings in 64 bits with
    it: e, what those steps in fp64 are off by from the same ones in 80 bits.  Here A is formed from X again before the steps have multiplied it by 1024 and the next step's factor, and is off by that, squared, of the roundings of its sums, s of
    2^-53; the result by 8 e for other orders, that, and its own rounding.  Where e leaves nothing to compare with, singular values have the bound that the steps have: the quintic's is 1.2025, the cubic's 1, from their
    values at most 1, and a chain of roundings beside it."""
    rng = np.random.default_rng(n_steps)
    five = tuple(float(np.float32(c)) for c in step)
    sets = [(_of_rank(rng, 32, 400, 5, False), "f32"), (_of_rank(rng, 32, 400, 5, True), "f32"), (_of_rank(rng, 7, 3000, 3, True), "bf16"), (_of_rank(rng, 20, 1000, 1, False), "f32")]
    for x, dtype in sets:
        t = torch.from_numpy(x.T.copy() if tall else x).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        got = pxr.orthogonalise(t, coefficients=[five] * n_steps, eps=0.0)
        assert got.dtype == t.dtype and bool(got.isfinite().all())
        out = got.double().cpu().numpy()
        out = out.T if tall else out
        assert np.linalg.norm(out, 2) <= (1.2025 if step == QUINTIC else 1.0) * (1 + 2.0 ** -10) + (W if dtype == "bf16" else 0) * np.linalg.norm(out)
        ref = _in_80_bits(x, [five] * n_steps)
        e = np.linalg.norm(learner.orthogonalise(x, [five] * n_steps, 0.0) - ref) / np.linalg.norm(ref)
        allowed = U + len(x) * 2.0 ** -53 * (1024 * step[0]) ** 2 + 8 * e + (W if dtype == "bf16" else 0)
        if e <= 0.01:
            assert np.linalg.norm(out - ref) <= allowed * np.linalg.norm(ref), (x.shape, dtype, e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rounds_of_steps_of_several_long_matrices(torch, pxr, dtype):
    """Each matrix by itself, in place, with rows apart, beside one that is not finite, in a graph; nothing else is written."""
    many = dict(steps=20)
    for B, m, n in ((3, 9, 2000), (2, 1500, 30)):
        x = normal(torch, n, B, m, n, dtype=dtype)
        want = pxr.orthogonalise(x, **many)
        for i in range(B):
            assert torch.equal(pxr.orthogonalise(x[i], **many), want[i])
        wide = torch.full((B + 1, m + 2, n + 5), 7.0, device="cuda", dtype=x.dtype)
        view = wide[:B, 1:-1, 3:3 + n]
        view.copy_(x)
        pxr.orthogonalise(view, out=view, **many)
        assert torch.equal(view, want)
        view.fill_(7.0)
        assert (wide == 7).all()
        bad = x.clone()
        bad[0, m // 2, n // 3] = float("inf")
        got = pxr.orthogonalise(bad, **many)
        assert got[0].isnan().all() and torch.equal(got[1:], want[1:])
        assert (pxr.orthogonalise(torch.zeros_like(x), **many) == 0).all()
        # the workspace goes by the steps as well: fewer and more of them in turn
        for steps in (5, 20, 6, 7):
            assert bool(pxr.orthogonalise(x, steps=steps).isfinite().all())
        static, g = x.clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = pxr.orthogonalise(static, **many)
        for i in (1, 2, 1):
            static.copy_(x * i)
            g.replay()
            eager = pxr.orthogonalise(x * i, **many)
            torch.cuda.synchronize()
            assert torch.equal(y, eager)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(32, 300), (100, 90), (40, 3000), (300, 200)])
def test_other_matrices_of_lower_rank_take_many_steps(torch, pxr, m, n, dtype):
    """Directions that a matrix does not have are made of the parts' roundings, 2^-23, after some 13 steps, as they are of fp32's: they stay below the bound of the singular values that it has."""
    x = torch.from_numpy(_of_rank(np.random.default_rng(m), m, n, 5, True)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    for step, most in ((QUINTIC, 1.2025), ((1.5, -0.5, 0.0), 1.0)):
        for n_steps in (16, 24, 64):
            got = pxr.orthogonalise(x, n_steps, step, eps=0.0)
            assert bool(got.isfinite().all())
            assert float(torch.linalg.matrix_norm(got.double().cpu(), 2)) <= most * 1.01 + (W if dtype == "bf16" else 0) * float(got.double().norm())


@pytest.mark.parametrize("m,n", [(64, 30000), (20011, 256), (513, 700), (700, 9000), (1500, 4000), (3001, 3000)])
def test_errors_do_not_grow_with_the_long_side(torch, pxr, m, n):
    """Sums go in chains of 512 values, 96 matrix instructions of three products, and the chains' results, K / 512 of them, are added up, K the longer side: (8 + sqrt(96) + sqrt(K / 512)) max(e, 2 u), where one chain of everything
    would have sqrt(3 K / 16).  Without the low parts in the first product 20011 x 256 would be off by 8.5e-5, and 4.5e-5 are allowed; 513 x 700 by 5e-4, of 3.6e-5."""
    x = normal(torch, n, m, n)
    ref = plain(torch, x, FIVE, 1e-7, torch.float64)
    e = float((plain(torch, x, FIVE, 1e-7, torch.float32).double() - ref).norm() / ref.norm())
    assert float((pxr.orthogonalise(x).double() - ref).norm() / ref.norm()) <= (8 + np.sqrt(96) + np.sqrt(max(m, n) / 512)) * max(e, 2 * U)


@pytest.mark.parametrize("m,n", [(90, 100), (64, 30000), (20011, 256), (700, 900), (1500, 2000), (30011, 40)])
def test_a_step_of_one_direction_keeps_all_bits(torch, pxr, m, n):
    """Signs, of rank one: every value is the same but for its sign, and what its second part leaves out has one direction too.  One step makes a + b + c of each.  What it is off by, relative: A 16 u (two values of 2 u, 4 u of
    products left out, as much again for its own two parts and the squares') and its sums' roundings, sqrt(96) + sqrt(K / 512) u; of that |a| + |b| + 2 |c| times, over |a + b + c| = 0.70.  The low parts left out of one
    product are 2^-12 of each value, over the same: 8e-5 to 2e-3 for most of these sizes in each of the three products, where 2.7e-5 to 3.5e-5 are allowed."""
    rng = np.random.default_rng(m)
    signs = np.outer(rng.choice([-1.0, 1.0], m), rng.choice([-1.0, 1.0], n))
    a, b, c = (float(np.float32(v)) for v in QUINTIC)
    got = pxr.orthogonalise(torch.from_numpy(signs.astype(np.float32)).cuda(), steps=1, eps=0.0).double().cpu().numpy()
    want = (a + b + c) / np.sqrt(m * n)
    off = np.linalg.norm(got * signs - want) / np.sqrt(m * n) / abs(want)
    assert off <= (abs(a) + abs(b) + 2 * abs(c)) / abs(a + b + c) * (16 + np.sqrt(96) + np.sqrt(max(m, n) / 512)) * U, off
