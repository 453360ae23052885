"""Group norm at the edges of its ranges: clusters with blocks that have no pixels; chains of calls through the same buffers; SiLU far below 0; the most
channels; values near the end of fp32."""
import numpy as np
import pytest

import test_gpu_norm as norm
from dense_util import D, HALF, TINY, U, back_bounds, f64, norm_bound, types
from oracle import dense

pytestmark = pytest.mark.gpu


# 49 and 25 pixels in clusters of 8 blocks of 7 and 4: the last block has none (all but the fp32 one of one group of 1024 channels, which takes two passes)
@pytest.mark.parametrize("dtype,act", [("f32", "none"), ("f32", "silu"), ("f16", "relu"), ("bf16", "silu")])
@pytest.mark.parametrize("shape", [(1, 7, 7, 512, 1), (2, 7, 7, 1024, 1), (1, 7, 7, 1024, 4), (3, 7, 7, 2048, 8), (1, 5, 5, 2048, 2), (5, 5, 5, 512, 1)],
                         ids=lambda s: "x".join(map(str, s)))
def test_blocks_without_pixels(alcs, shape, dtype, act):
    norm.test_forward_and_backward(alcs, shape, dtype, act)


def test_a_chain_whose_buffers_are_used_again(alcs):
    """Norm in place, quantisation, its inverse and the product, 40 times over in one captured graph, all through the same buffers: every kernel starts while the
    one before it still writes what it reads, and what it read the time before.  Each link's results are those of calls that have the GPU to themselves."""
    import torch
    n, h, w, c, cout, groups, links = 4, 14, 14, 256, 64, 32, 40
    rows, dt, t = n * h * w, alcs.ALCS_BF16, torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    xs, gammas, weights = rnd(links, rows, c).to(t), 1 + 0.3 * rnd(links, c), rnd(cout, c)
    bytes_of = lambda r: [torch.empty(b, dtype=torch.uint8, device="cuda") for b in alcs.alcs_mx4_bytes(r, c)]  # noqa: E731
    x, gamma, q, wq = torch.empty(rows, c, dtype=t, device="cuda"), torch.empty(c, device="cuda"), bytes_of(rows), bytes_of(cout)
    ws = torch.empty(alcs.alcs_group_norm_workspace(n, h, w, c, groups, dt), dtype=torch.uint8, device="cuda")
    alcs.alcs_mx4_quantize(weights, cout, c, c, alcs.ALCS_F32, *wq, torch.cuda.current_stream())
    values, ys = torch.empty(links, rows, c, dtype=t, device="cuda"), torch.empty(links, rows, cout, dtype=t, device="cuda")

    def run(stream, wait):
        for i in range(links):
            x.copy_(xs[i])
            gamma.copy_(gammas[i])
            for call in (lambda: alcs.alcs_group_norm(x, x, n, h, w, c, groups, gamma, None, 1e-5, alcs.ALCS_SILU, dt, None, None, ws, ws.numel(), stream),
                         lambda: alcs.alcs_mx4_quantize(x, rows, c, c, dt, *q, stream),
                         lambda: alcs.alcs_mx4_dequantize(*q, rows, c, x, c, dt, stream),
                         lambda: alcs.alcs_group_norm(x, x, n, h, w, c, groups, gamma, None, 1e-5, 0, dt, None, None, ws, ws.numel(), stream),
                         lambda: alcs.alcs_mx4_quantize(x, rows, c, c, dt, *q, stream),
                         lambda: alcs.alcs_mx4_product(*q, rows, *wq, cout, c, ys[i], gamma[:cout], None, 0, dt, stream),
                         lambda: alcs.alcs_mx4_dequantize(*q, rows, c, values[i], c, dt, stream)):
                call()
                if wait:
                    torch.cuda.synchronize()

    run(torch.cuda.current_stream(), True)
    want = values.clone(), ys.clone()
    assert not want[0].isnan().any() and not want[1].isnan().any()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        run(stream, False)
    for _ in range(10):
        values.fill_(float("nan")), ys.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(values, want[0]) and torch.equal(ys, want[1])


# loads of 8, 2 and 1 elements; a group that is not whole loads; two passes
@pytest.mark.parametrize("shape", [(2, 9, 9, 96, 12), (3, 7, 5, 150, 30), (2, 11, 9, 35, 5), (3, 13, 11, 66, 22), (1, 448, 448, 32, 8), (70, 56, 56, 64, 8)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_silu_far_below_zero(alcs, shape, dtype):
    """Group 0 has a beta of -30 to -105, group 1 the lowest number, group 2 minus infinity (a channel that is masked out).

    y: a relative error is what z is off by, q = D u |gamma| (|xh| + M) + 2 u |z| with M = max|x| rstd, as in norm_bound, and (8 + 2 |z|) u of exp and the
    quotient; below -43 y stays what it is there, 43 x 2^-62 = 9.33e-18 and less than 1e-17 with that error, instead of going to 0.  The slope s + z s (1 - s) is
    between z exp(z) and half of it there, so that it is off by twice the relative error, and by less than 1e-17 below -43.  dx: every term is off by that of dz and by 2 D u (1 + M)
    of xh, rstd and the sums, as in back_bounds."""
    import torch
    n, h, w, c, groups = shape
    x, dy, gamma, beta = norm._inputs(sum(shape), n, h * w, c, dtype, alcs)
    k, far = c // groups, 1e-17
    beta[:k] = -torch.linspace(30, 105, k, device="cuda")
    beta[k:2 * k], beta[2 * k:3 * k] = float(np.finfo(np.float32).min), float("-inf")
    call = norm.Norm(alcs, x, shape, dtype, "silu", 1e-5, gamma, beta)
    y, dx = f64(call.forward()), f64(call.backward(dy))
    dgamma, dbeta = f64(call.dgamma), f64(call.dbeta)
    # the other groups are what they are
    rest = slice(3 * k, c)
    args = f64(x[..., rest]), f64(gamma[rest]), f64(beta[rest])
    ref = dense.group_norm_backward(args[0], f64(dy[..., rest]), groups - 3, *args[1:], 1e-5, "silu")
    assert (np.abs(y[..., rest] - ref["y"]) <= norm_bound(ref, *args, groups - 3, dtype)).all()
    assert (np.abs(dx[..., rest] - ref["dx"]) <= back_bounds(ref, args[0], f64(dy[..., rest]), *args[1:], groups - 3, dtype)[0]).all()
    for g in range(3):
        at = slice(g * k, (g + 1) * k)
        xg, dyg, gg = f64(x[..., at]), f64(dy[..., at]), np.abs(f64(gamma[at]))
        ref = dense.group_norm_backward(xg, dyg, 1, f64(gamma[at]), f64(beta[at]) if g == 0 else None, 1e-5, "silu" if g == 0 else "none")
        xh, r = np.abs(ref["xh"]), ref["rstd"][:, :, None]
        m = np.abs(xg).max((1, 2), keepdims=True) * r
        if g == 0:
            z = np.abs(ref["z"])
            q, want, dz, want_dx = D * U * gg * (xh + m) + U * (8 + 4 * z), ref["y"], dyg * dense.activation_slope(ref["z"], "silu"), ref["dx"]
        else:      # masked out: z is -3e38 or minus infinity
            q, want, dz, want_dx = 0 * xh, 0 * xh, 0 * xh, 0 * xh
        bound = q * np.abs(want) + far
        assert (np.abs(y[..., at] - want) <= bound + HALF[dtype] * (np.abs(want) + bound) + TINY[dtype]).all()
        off = 2 * q.max() * np.abs(dz) + far * np.abs(dyg)      # of dz
        e = 2 * D * U * (1 + m)
        t, o = np.abs(gg * dz), gg * off
        mean = lambda v: v.mean((1, 2), keepdims=True)  # noqa: E731
        bound = r * (o + mean(o) + xh * mean(o * xh) + e * (t + mean(t) * (1 + xh) + (1 + xh) * mean(t * xh)))
        assert (np.abs(dx[..., at] - want_dx) <= bound + HALF[dtype] * (np.abs(want_dx) + bound) + TINY[dtype]).all()
        for got, f in ((dgamma[at], ref["xh"]), (dbeta[at], 1 + 0 * xh)):
            assert (np.abs(got - (dz * f).sum((0, 1))) <= (off * np.abs(f) + e * np.abs(dz) * (1 + xh)).sum((0, 1))).all()


@pytest.mark.parametrize("shape", [(1, 2, 2, 65536, 8), (2, 1, 3, 65536, 65536), (1, 3, 3, 65528, 8), (1, 5, 5, 65535, 1285), (1, 12, 11, 65536, 1024)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,act", [("f32", "none"), ("bf16", "silu")])
def test_the_most_channels(alcs, shape, dtype, act):
    norm.test_forward_and_backward(alcs, shape, dtype, act)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 30, 30, 64, 8), (2, 3, 3, 35, 5), (2, 56, 56, 64, 2), (1, 448, 448, 32, 8), (1, 5, 4, 3001, 1), (2, 7, 7, 512, 1), (1, 1, 1, 64, 16),
                                   (3, 17, 23, 150, 30), (1, 130, 90, 1031, 1)], ids=lambda s: "x".join(map(str, s)))
def test_values_whose_sums_are_beyond_fp32(alcs, shape, dtype):
    """All values of an image 2^100, 10^36 or 2^126: y is act(beta), the mean the value.  Then both signs of them: squared distances are no numbers of fp32, rstd is 0."""
    import torch
    n, h, w, c, groups = shape
    _, dy, gamma, beta = norm._inputs(9, n, h * w, c, dtype, alcs)
    t = dy.dtype
    for value in (2.0 ** 100, 1e36, 2.0 ** 126):
        x = torch.full_like(dy, value)
        k = norm.Norm(alcs, x, shape, dtype, "none", 1e-5, gamma, beta)
        assert torch.equal(k.forward(), beta.to(t).expand_as(x))
        v = x.flatten()[0].double()
        assert ((k.mean.double() / v - 1).abs() <= D * U).all() and torch.isfinite(k.rstd).all()
        if h * w * c // groups < 2:
            continue
        sign = torch.where(torch.arange(x.numel(), device="cuda") % 2 == 0, 1, -1).view(x.shape)
        k = norm.Norm(alcs, x * sign, shape, dtype, "none", 1e-5, gamma, beta)
        assert torch.equal(k.forward(), beta.to(t).expand_as(x)) and (k.rstd == 0).all()
        assert (k.backward(dy) == 0).all() and (k.dgamma == 0).all() and torch.isfinite(k.dbeta).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,c", [(600, 250), (600, 256), (3, 96)])
def test_a_pruned_layer_behind_a_norm_in_place(alcs, n, c, dtype):
    """Images of one pixel are channels last and channels first at once: a norm in place and the pruned layer that reads it, 30 times over in one captured graph through the
    same buffer, against calls that have the GPU to themselves."""
    import torch
    cout, g, groups, links = 64, 4, 2, 30
    dt, t = types(alcs)[dtype]
    r = np.random.default_rng(n + c)
    mask = (r.random((cout // g, c)) < 0.3).astype(np.uint8)
    w = torch.from_numpy(r.normal(size=(cout, c)).astype(np.float32) / 8).to(t)
    host = w.view(torch.uint16).numpy() if dtype == "bf16" else w.numpy()
    packed = alcs.alcs_packed_upload(alcs.alcs_pack(host, mask, g, bf16=dtype == "bf16"), 0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    xs = torch.randn(links, n, 1, c, generator=gen, device="cuda").to(t)
    gamma, x = 1 + 0.3 * torch.randn(c, generator=gen, device="cuda"), torch.empty(n, 1, c, device="cuda", dtype=t)
    size = alcs.alcs_group_norm_workspace(n, 1, 1, c, groups, dt)
    ws, ys = torch.empty(size, device="cuda", dtype=torch.uint8), torch.empty(links, n, cout, 1, device="cuda", dtype=t)

    def run(stream, wait):
        for i in range(links):
            x.copy_(xs[i])
            for k in range(2):
                alcs.alcs_group_norm(x, x, n, 1, 1, c, groups, gamma, None, 1e-5, alcs.ALCS_RELU if k else 0, dt, None, None, ws, size, stream)
                if wait:
                    torch.cuda.synchronize()
                alcs.alcs_spconv1x1(packed, x, ys[i], n, 1, 1, None, 0, stream)
                if wait:
                    torch.cuda.synchronize()

    run(torch.cuda.current_stream(), True)
    want = ys.clone()
    assert torch.isfinite(want).all() and want.abs().max() > 0
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        run(stream, False)
    for _ in range(10):
        ys.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ys, want)
    last = dense.group_norm(f64(xs[-1]), groups, f64(gamma))["y"].reshape(n, 1, c)
    if dtype == "f32":
        # The last link against the definitions.  A norm is off by D u |gamma| (|xh| + M), 64 x 2^-24 x 2 x 10 = 8e-5 with gamma below 2 and values below 5; the first one's
        # error goes through the second, whose rstd is about 1; a sum of 128 products by 128 u |W| |z|, 8e-6: less than 4e-4 (1 + |z|) |W|.
        z = dense.group_norm(last, groups, f64(gamma), act="relu")["y"].reshape(n, c)
        full = f64(w) * np.repeat(mask, g, 0)
        assert (np.abs(f64(ys[-1])[:, :, 0] - z @ full.T) <= 4e-4 * (1 + np.abs(z)) @ np.abs(full).T).all()
