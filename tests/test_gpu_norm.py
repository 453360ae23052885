"""Group norm with an activation, channels last: forward and backward against the 64-bit definitions."""
import numpy as np
import pytest

from dense_util import HALF, back_bounds, f64, flags_of, norm_bound, types
from oracle import dense

pytestmark = pytest.mark.gpu

# n, h, w, c, groups: one pixel; one channel per group; odd everything; a group of 3 x 8 bytes; one group; more pixels than a block,
# than a cluster; more channels per group than threads; rows of pixels that are not whole 16 bytes, nor 8
SHAPES = [(1, 1, 1, 64, 16), (1, 1, 1, 5, 1), (2, 5, 5, 7, 7), (1, 7, 7, 512, 32), (3, 17, 23, 150, 30), (2, 9, 11, 36, 3), (2, 14, 14, 128, 8), (2, 9, 9, 640, 20),
          (1, 9, 9, 2048, 1), (1, 3, 3, 4100, 1), (1, 5, 4, 3001, 1), (1, 64, 70, 66, 2), (2, 56, 56, 64, 32), (1, 112, 112, 32, 8), (1, 200, 150, 24, 3),
          (1, 130, 90, 1031, 1), (5, 3, 2, 96, 12), (67, 2, 2, 32, 4), (1, 2, 2, 8192, 1), (2, 2, 3, 8200, 2), (3, 11, 13, 70, 35), (2, 40, 33, 50, 5)]


def _inputs(seed, n, hw, c, dtype, alcs, mean=0.5, spread=1.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    t = types(alcs)[dtype][1]
    x = (rnd(n, hw, c) * spread + mean * rnd(c)).to(t)
    return x, rnd(n, hw, c).to(t), 1 + 0.3 * rnd(c), 0.3 * rnd(c)


# Calls large enough to read x twice from L2: images of several runs and of one, more images than stay in L2, loads of 16, 8 and 2 or 4 bytes, threads without
# channels, one row of pixels at a time, one image
LARGE = [(16, 56, 56, 256, 32, "bf16", "silu"), (16, 56, 56, 256, 32, "f16", "relu"), (40, 62, 63, 100, 10, "f16", "none"), (24, 50, 56, 150, 30, "f32", "silu"),
         (8, 28, 28, 2048, 32, "bf16", "silu"), (1, 448, 448, 64, 8, "f32", "silu"), (600, 9, 16, 320, 64, "bf16", "none"), (90, 20, 20, 380, 76, "f16", "silu"),
         (50, 64, 64, 31, 31, "f32", "relu")]


class Norm:
    """Buffers of one shape and the calls on them, every output filled with NaN first."""

    def __init__(self, alcs, x, shape, dtype, act="none", eps=1e-5, gamma=None, beta=None):
        import torch
        self.alcs, self.x, self.shape, self.act, self.eps, self.gamma, self.beta = alcs, x, shape, act, eps, gamma, beta
        n, c, groups = shape[0], shape[3], shape[4]
        self.dt = types(alcs)[dtype][0]
        nan = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
        self.mean, self.rstd, self.dgamma, self.dbeta = nan(n, groups), nan(n, groups), nan(c), nan(c)
        self.bytes = alcs.alcs_group_norm_workspace(*shape, self.dt)
        self.ws = torch.full((max(1, self.bytes),), 255, dtype=torch.uint8, device="cuda")

    def forward(self, y=None, stats=True, stream=None):
        import torch
        y = torch.full_like(self.x, float("nan")) if y is None else y
        self.alcs.alcs_group_norm(self.x, y, *self.shape, self.gamma, self.beta, self.eps, flags_of(self.alcs, self.act), self.dt, self.mean if stats else None,
                                  self.rstd if stats else None, self.ws, self.bytes, stream or torch.cuda.current_stream())
        return y

    def backward(self, dy, dx=None, stream=None):
        import torch
        dx = torch.full_like(self.x, float("nan")) if dx is None else dx
        self.alcs.alcs_group_norm_backward(self.x, dy, dx, *self.shape, self.mean, self.rstd, self.gamma, self.beta, self.dgamma, self.dbeta,
                                           flags_of(self.alcs, self.act), self.dt, self.ws, self.bytes, stream or torch.cuda.current_stream())
        return dx


def _within(got, ref, bound):
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bound).all(), float((np.abs(got - ref) / bound).max())


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,act", [("f32", "silu"), ("f16", "none"), ("bf16", "relu"), ("bf16", "silu")])
def test_forward_and_backward(alcs, shape, dtype, act):
    n, h, w, c, groups = shape
    x, dy, gamma, beta = _inputs(sum(shape), n, h * w, c, dtype, alcs)
    k = Norm(alcs, x, shape, dtype, act, 1e-5, gamma, beta)
    y, dx = k.forward(), k.backward(dy)
    ref = dense.group_norm_backward(f64(x), f64(dy), groups, f64(gamma), f64(beta), 1e-5, act)
    _within(f64(y), ref["y"], norm_bound(ref, f64(x), f64(gamma), f64(beta), groups, dtype))
    bx, bg, bb = back_bounds(ref, f64(x), f64(dy), f64(gamma), f64(beta), groups, dtype)
    if act == "relu":      # where z is nearer to 0 than its error, either slope is right: then the whole group may move
        near = np.abs(ref["z"]) <= norm_bound(dict(ref, y=0 * ref["y"]), f64(x), f64(gamma), f64(beta), groups, "f32")
        jump = np.where(near, np.abs(f64(gamma) * f64(dy)), 0.0)
        s = jump.reshape(n, h * w, groups, -1).sum((1, 3))[:, None, :]
        r = np.repeat(ref["rstd"], c // groups, axis=1)[:, None, :]
        bx = bx + r * (jump + np.repeat(s, c // groups, axis=2) * (1 + np.abs(ref["xh"]) * np.abs(ref["xh"]).max()) / (h * w * c // groups))
        bg, bb = bg + (np.where(near, np.abs(f64(dy) * ref["xh"]), 0)).sum((0, 1)), bb + np.where(near, np.abs(f64(dy)), 0).sum((0, 1))
    _within(f64(dx), ref["dx"], bx)
    _within(f64(k.dgamma), ref["dgamma"], bg)
    _within(f64(k.dbeta), ref["dbeta"], bb)
    xa = np.abs(f64(x)).reshape(n, h * w, groups, -1)
    _within(f64(k.mean), ref["mean"], 64 * 2.0 ** -24 * xa.mean((1, 3)) + 1e-30)
    _within(f64(k.rstd), ref["rstd"], 128 * 2.0 ** -24 * ref["rstd"] * (1 + xa.max((1, 3)) * ref["rstd"] * 1e-3))


@pytest.mark.parametrize("case", LARGE, ids=lambda s: "x".join(map(str, s)))
def test_large_calls(alcs, case):
    """Every image against the definition for the first and last ones, the others by what the sums over all of them are."""
    import torch
    *shape, dtype, act = case
    n, h, w, c, groups = shape
    x, dy, gamma, beta = _inputs(sum(shape), n, h * w, c, dtype, alcs)
    k = Norm(alcs, x, tuple(shape), dtype, act, 1e-5, gamma, beta)
    y, dx = k.forward(), k.backward(dy)
    xd, g64, b64 = x.double().view(n, h * w, groups, -1), gamma.double(), beta.double()
    mean = xd.mean((1, 3), keepdim=True)
    rstd = 1 / ((xd - mean).square().mean((1, 3), keepdim=True) + 1e-5).sqrt()
    xh = ((xd - mean) * rstd).view(n, h * w, c)
    z = xh * g64 + b64
    s = torch.sigmoid(z)
    slope = s + z * s * (1 - s) if act == "silu" else (z > 0).double() if act == "relu" else torch.ones_like(z)
    ref_y = z * s if act == "silu" else z.clamp(min=0) if act == "relu" else z
    dz = dy.double() * slope
    t = (dz * g64).view(n, h * w, groups, -1)
    xg = xh.view(n, h * w, groups, -1)
    ref_dx = (rstd * (t - t.mean((1, 3), keepdim=True) - xg * (t * xg).mean((1, 3), keepdim=True))).view(n, h * w, c)
    # the bounds of dense_util, image by image
    for i in sorted({0, 1 % n, n // 2, n - 1}):
        ref = dense.group_norm_backward(f64(x[i:i + 1]), f64(dy[i:i + 1]), groups, f64(gamma), f64(beta), 1e-5, act)
        assert np.abs(f64(ref_dx[i:i + 1]) - ref["dx"]).max() < 1e-9 and np.abs(f64(ref_y[i:i + 1]) - ref["y"]).max() < 1e-9
        _within(f64(y[i:i + 1]), ref["y"], norm_bound(ref, f64(x[i:i + 1]), f64(gamma), f64(beta), groups, dtype))
        if act != "relu":
            _within(f64(dx[i:i + 1]), ref["dx"], back_bounds(ref, f64(x[i:i + 1]), f64(dy[i:i + 1]), f64(gamma), f64(beta), groups, dtype)[0])
    # all of them, by the sum of squared differences: each is at most the bound, which is a few units of the type in the mean
    for got, ref in ((y, ref_y), (dx, ref_dx)):
        d = (got.double() - ref).norm() / ref.norm()
        # relu: a slope of the wrong side where z is within 64 u (1 + M) of 0, at most one value in 10^4, each off by less than 10 of them
        assert d < HALF[dtype] + 256 * 2.0 ** -24 + (0.02 if act == "relu" and got is dx else 0), d.item()
    # sums of n h w values: 64 u of their magnitudes, and what dz and xh themselves are off by (1e-5, with M of 10 or less)
    for got, term in ((k.dgamma, dz * xh), (k.dbeta, dz)):
        ref, scale = term.sum((0, 1)), term.abs().sum((0, 1))
        assert ((got.double() - ref).abs() <= 2e-5 * scale + (1e-4 * dy.double().abs().sum((0, 1)) if act == "relu" else 0)).all()
    # the same bits again
    assert (k.forward() == y).all() and (k.backward(dy) == dx).all()


# Several rounds of blocks that an SM has room for few of, and fewer blocks than SMs: twice the threads; loads of 16, 8 and 4 bytes, groups that are not whole loads
@pytest.mark.parametrize("case", [(1, 224, 224, 64, 32, "bf16", "silu"), (64, 28, 28, 256, 32, "f32", "relu"), (20, 112, 112, 120, 30, "bf16", "relu"),
                                  (1, 224, 221, 66, 22, "f16", "none"), (70, 28, 27, 250, 25, "f32", "silu"), (128, 28, 28, 160, 20, "f16", "silu")],
                         ids=lambda s: "x".join(map(str, s)))
def test_blocks_of_twice_the_threads(alcs, case):
    test_large_calls(alcs, case)


@pytest.mark.parametrize("shape", [(2, 14, 14, 128, 8), (1, 130, 120, 64, 2)])
def test_without_parameters_and_statistics(alcs, shape):
    n, h, w, c, groups = shape
    x, dy, _, _ = _inputs(1, n, h * w, c, "f32", alcs)
    k = Norm(alcs, x, shape, "f32")
    y = k.forward(stats=False)
    assert k.mean.isnan().all()
    one, zero = np.ones(c), np.zeros(c)
    ref = dense.group_norm_backward(f64(x), f64(dy), groups)
    _within(f64(y), ref["y"], norm_bound(ref, f64(x), one, zero, groups, "f32"))
    k.forward()
    k.dgamma, k.dbeta = None, None
    _within(f64(k.backward(dy)), ref["dx"], back_bounds(ref, f64(x), f64(dy), one, zero, groups, "f32")[0])


@pytest.mark.parametrize("shape", [(2, 30, 30, 64, 8), (1, 150, 120, 64, 2)])
def test_a_mean_far_from_zero(alcs, shape):
    """Values of spread 1 around 1000: their squares' mean less the square of their mean would be off by 2^-24 10^6, several per cent of the variance."""
    n, h, w, c, groups = shape
    x, dy, gamma, beta = _inputs(2, n, h * w, c, "f32", alcs, 0.0)
    x += 1000
    k = Norm(alcs, x, shape, "f32", "none", 1e-5, gamma, beta)
    y = f64(k.forward())
    ref = dense.group_norm(f64(x), groups, f64(gamma), f64(beta))
    _within(y, ref["y"], norm_bound(ref, f64(x), f64(gamma), f64(beta), groups, "f32"))
    # rstd comes from differences: 2 D u, and the square of the mean's own error, (D u 1000)^2
    assert np.abs(f64(k.rstd) / ref["rstd"] - 1).max() <= 128 * 2.0 ** -24 + (64 * 2.0 ** -24 * 1001) ** 2


@pytest.mark.parametrize("shape", [(1, 30, 30, 64, 8), (2, 41, 37, 35, 5), (1, 150, 120, 64, 2), (1, 60, 50, 1031, 1), (1, 120, 120, 31, 31)])
def test_an_outlier_where_a_thread_or_a_block_starts(alcs, shape):
    """10^4 among values of order 1, at the first and at some other pixel: the variance is theirs, to the rounding of its sums."""
    n, h, w, c, groups = shape
    x, dy, gamma, beta = _inputs(7, n, h * w, c, "f32", alcs)
    x[:, 0] += 1e4
    x[:, 57] -= 2e4
    k = Norm(alcs, x, shape, "f32", "none", 1e-5, gamma, beta)
    y = f64(k.forward())
    ref = dense.group_norm(f64(x), groups, f64(gamma), f64(beta))
    _within(y, ref["y"], norm_bound(ref, f64(x), f64(gamma), f64(beta), groups, "f32"))
    # A sum of squared distances is rounded once at each of a thread's values (at most 32 loads of 5 vectors), twice at each of some 15 unions, and a term of
    # it has 6 roundings of its own: 196 x 2^-24, half of that in rstd.
    assert np.abs(f64(k.rstd) / ref["rstd"] - 1).max() <= 98 * 2.0 ** -24


@pytest.mark.parametrize("spread", [0.0, 2.0 ** -10])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 64, 16), (2, 1, 3, 7, 7), (2, 5, 5, 96, 12), (3, 7, 7, 150, 30), (1, 150, 121, 64, 2), (1, 5, 4, 3001, 1)])
def test_values_whose_squares_are_beyond_fp32(alcs, shape, dtype, spread):
    """Around 2^66, apart by up to 2^56 or so: what is squared is distances between them, also where a thread has no value of its own."""
    import torch
    n, h, w, c, groups = shape
    x, _, gamma, beta = _inputs(8, n, h * w, c, "f32", alcs, 0.0)
    x = ((1 + spread * x) * 2.0 ** 66).to(types(alcs)[dtype][1])
    k = Norm(alcs, x, shape, dtype, "none", 1e-5, gamma, beta)
    y = f64(k.forward())
    ref = dense.group_norm(f64(x), groups, f64(gamma), f64(beta))
    _within(y, ref["y"], norm_bound(ref, f64(x), f64(gamma), f64(beta), groups, dtype))
    assert np.abs(f64(k.mean) / 2.0 ** 66 - 1).max() <= 2.0 ** -8 and torch.isfinite(k.rstd).all()      # (means of a few values off by up to 5 x 2^-10)


def test_constant_groups_and_eps(alcs):
    import torch
    x = torch.full((1, 25, 32), 7.0, device="cuda")
    gamma, beta = torch.full((32,), 3.0, device="cuda"), torch.arange(32.0, device="cuda")
    y = Norm(alcs, x, (1, 5, 5, 32, 4), "f32", gamma=gamma, beta=beta).forward()
    assert (y == beta).all()
    # eps = 0 and no spread: 0 / 0
    assert Norm(alcs, x, (1, 5, 5, 32, 4), "f32", eps=0.0).forward().isnan().all()
    x = torch.randn(1, 25, 32, device="cuda") * 1e-3
    ref = dense.group_norm(f64(x), 4, eps=0.5)
    _within(f64(Norm(alcs, x, (1, 5, 5, 32, 4), "f32", eps=0.5).forward()), ref["y"], norm_bound(ref, f64(x), np.ones(32), np.zeros(32), 4, "f32"))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("shape", [(2, 9, 9, 32, 4), (2, 130, 120, 64, 2)])
def test_what_is_not_finite_stays_in_its_group(alcs, bad, shape):
    n, h, w, c, groups = shape
    x, dy, gamma, beta = _inputs(3, n, h * w, c, "bf16", alcs)
    clean = Norm(alcs, x, shape, "bf16", "silu", 1e-5, gamma, beta)
    y, dx = clean.forward(), clean.backward(dy)
    x2 = x.clone()
    k = c // groups
    x2[1, 5, k + 1] = bad
    dirty = Norm(alcs, x2, shape, "bf16", "silu", 1e-5, gamma, beta)
    y2, dx2 = dirty.forward(), dirty.backward(dy)
    for a, b in ((y, y2), (dx, dx2)):
        assert b[1, :, k:2 * k].isnan().all()
        b[1, :, k:2 * k] = a[1, :, k:2 * k]
        assert (a == b).all()
    dirty.act = "relu"
    assert (dirty.forward()[1, :, k:2 * k] == 0).all()


def test_nothing_to_sum_gives_zero_gradients(alcs):
    import torch
    k = Norm(alcs, torch.empty(0, 16, 8, device="cuda"), (0, 4, 4, 8, 2), "f32")
    k.backward(k.x, k.x)
    assert (k.dgamma == 0).all() and (k.dbeta == 0).all()


@pytest.mark.parametrize("shape", [(2, 14, 14, 128, 8), (1, 150, 120, 64, 2)])
def test_in_place(alcs, shape):
    n, h, w, c, groups = shape
    x, dy, gamma, beta = _inputs(4, n, h * w, c, "bf16", alcs)
    k = Norm(alcs, x.clone(), shape, "bf16", "silu", 1e-5, gamma, beta)
    y, dx = k.forward(), k.backward(dy)
    other = dy.clone()
    assert (k.backward(other, other) == dx).all()
    assert (k.backward(dy, k.x) == dx).all()
    k.x = x.clone()
    assert (k.forward(k.x) == y).all()


@pytest.mark.parametrize("dtype,offset", [("bf16", 1), ("bf16", 4), ("f16", 2), ("f32", 1), ("f32", 2)])
@pytest.mark.parametrize("shape", [(2, 14, 14, 64, 8), (1, 100, 120, 64, 2)])
def test_buffers_that_start_anywhere(alcs, dtype, offset, shape):
    import torch
    n, h, w, c, groups = shape
    x, dy, gamma, beta = _inputs(5, n, h * w, c, dtype, alcs)

    def moved(t):
        m = torch.full((t.numel() + 2 * offset + 8,), 77.0, dtype=t.dtype, device="cuda")
        v = m[offset:offset + t.numel()].view(t.shape)
        v.copy_(t)
        return m, v

    (_, xm), (_, dym), (ym, y), (dxm, dx) = moved(x), moved(dy), moved(x), moved(x)
    k = Norm(alcs, xm, shape, dtype, "silu", 1e-5, gamma, beta)
    k.forward(y)
    k.backward(dym, dx)
    ref = dense.group_norm_backward(f64(x), f64(dy), groups, f64(gamma), f64(beta), 1e-5, "silu")
    _within(f64(y), ref["y"], norm_bound(ref, f64(x), f64(gamma), f64(beta), groups, dtype))
    _within(f64(dx), ref["dx"], back_bounds(ref, f64(x), f64(dy), f64(gamma), f64(beta), groups, dtype)[0])
    for m in (ym, dxm):
        assert (m[:offset] == 77).all() and (m[offset + x.numel():] == 77).all()


@pytest.mark.parametrize("shape", [(3, 14, 14, 128, 8), (2, 150, 120, 64, 2)])
def test_streams_graphs_and_the_same_bits(alcs, shape):
    """Eager calls, two captured graphs with workspaces of their own that run side by side, replays on new data: the same bits."""
    import torch
    n, h, w, c, groups = shape
    sets = [_inputs(10 + i, n, h * w, c, "bf16", alcs) for i in range(2)]
    want = []
    for x, dy, gamma, beta in sets:
        k = Norm(alcs, x, shape, "bf16", "silu", 1e-5, gamma, beta)
        want.append((k.forward(), k.backward(dy), k.dgamma, k.dbeta))
    nets, graphs, outs, streams = [], [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for i, (x, dy, gamma, beta) in enumerate(sets):
        k = Norm(alcs, x.clone(), shape, "bf16", "silu", 1e-5, gamma, beta)
        y, dx, d = torch.empty_like(x), torch.empty_like(x), dy.clone()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[i]):
            k.forward(y, stream=streams[i])
            k.backward(d, dx, stream=streams[i])
        nets.append((k, d)), graphs.append(g), outs.append((y, dx))
    for rep in range(3):
        for (k, _), (y, dx) in zip(nets, outs):
            for t in (y, dx, k.dgamma, k.dbeta, k.mean, k.rstd):
                t.fill_(float("nan"))
            k.ws.fill_(255)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (k, _), (y, dx), w in zip(nets, outs, want):
            for a, b in zip((y, dx, k.dgamma, k.dbeta), w):
                assert (a == b).all()
    # the other set's data through the first graph
    k, d = nets[0]
    k.x.copy_(sets[1][0]), d.copy_(sets[1][1]), k.gamma.copy_(sets[1][2]), k.beta.copy_(sets[1][3])
    graphs[0].replay()
    torch.cuda.synchronize()
    for a, b in zip((*outs[0], k.dgamma, k.dbeta), want[1]):
        assert (a == b).all()


def test_more_elements_than_32_bits_count(alcs):
    """33 images of 2^27 elements: the last one comes out as it does alone."""
    import torch
    hw, c, groups = 1 << 20, 128, 32
    x = torch.empty(33, hw, c, dtype=torch.bfloat16, device="cuda")
    one, dy, gamma, beta = _inputs(6, 1, hw, c, "bf16", alcs)
    x[:32] = 0
    x[32] = one[0]
    k = Norm(alcs, one, (1, 1024, 1024, c, groups), "bf16", "silu", 1e-5, gamma, beta)
    y, dx = k.forward(), k.backward(dy)
    many = Norm(alcs, x, (33, 1024, 1024, c, groups), "bf16", "silu", 1e-5, gamma, beta)
    many.forward(stats=True)
    dys = torch.zeros_like(x)
    dys[32] = dy[0]
    many.backward(dys, dys)
    # (how an image is cut into chunks depends on how many there are: sums in another order, then one rounding)
    for a, b in ((many.mean[32], k.mean[0]), (many.rstd[32], k.rstd[0])):
        assert ((a - b).abs() <= 1e-5 * (1 + b.abs())).all()
    # dx is of order 1: 1e-5 of that, and a unit of bf16 where a sum falls on the other side of a rounding
    assert ((dys[32].float() - dx[0].float()).abs() <= 2.0 ** -7 * dx[0].float().abs() + 1e-4).all()
    assert (dys[0] == 0).all()
    many.forward(x)
    assert ((x[32].float() - y[0].float()).abs() <= 2.0 ** -7 * y[0].float().abs() + 1e-4).all()


def test_host_memory_is_refused(alcs):
    import torch
    x = torch.randn(1, 16, 32)
    y = torch.empty(1, 16, 32, device="cuda")
    for a, b in ((x, y), (y, x), (x.pin_memory(), y)):
        with pytest.raises(alcs.AlcsError) as e:
            alcs.alcs_group_norm(a, b, 1, 4, 4, 32, 4, stream=torch.cuda.current_stream())
        assert e.value.status == alcs.ALCS_ERR_INVALID_ARG
