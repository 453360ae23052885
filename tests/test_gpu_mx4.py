"""Microscaled 4-bit floating point: quantisation to the bit, the product on the tensor cores against 64 bits, and a layer of all of it."""
import numpy as np
import pytest

from dense_util import f64, norm_bound, product_bound, types
from oracle import dense

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _quantize(alcs, x, cols, ldx, dtype, stream=None):
    torch = _torch()
    rows = x.shape[0]
    db, sb = alcs.alcs_mx4_bytes(rows, cols)
    data, scales = torch.full((db,), 0xA5, dtype=torch.uint8, device="cuda"), torch.full((sb,), 0x5A, dtype=torch.uint8, device="cuda")
    alcs.alcs_mx4_quantize(x, rows, cols, ldx, types(alcs)[dtype][0], data, scales, stream or torch.cuda.current_stream())
    return data, scales


def _check_quantized(alcs, x, cols, ldx, dtype):
    """Every byte of both arrays, what has to be left alone included."""
    data, scales = _quantize(alcs, x, cols, ldx, dtype)
    codes, sc = dense.mx4_quantize(f64(x)[:, :cols])
    d, s = dense.mx4_store(codes, sc, cols)
    free = dense.mx4_store(0 * codes, 0 * sc, cols, fill=1)[0] == 1
    free_s = dense.mx4_store(0 * codes, 0 * sc, cols, fill=1)[1] == 1
    d[free], s[free_s] = 0xA5, 0x5A
    assert (data.cpu().numpy() == d).all()
    assert (scales.cpu().numpy() == s).all()
    return data, scales, codes, sc


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (1, 4096), (3, 33), (7, 31), (49, 512), (128, 64), (129, 97), (200, 100), (300, 8), (1000, 130)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_quantize_and_back(alcs, rows, cols, dtype):
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(rows * 7 + cols)
    t = types(alcs)[dtype][1]
    x = (torch.randn(rows, cols, generator=g, device="cuda") * (0.3 + torch.randn(cols, generator=g, device="cuda").abs())).clamp(min=-0.2).to(t)
    data, scales, codes, sc = _check_quantized(alcs, x, cols, cols, dtype)
    y = torch.full_like(x, float("nan"))
    alcs.alcs_mx4_dequantize(data, scales, rows, cols, y, cols, types(alcs)[dtype][0], torch.cuda.current_stream())
    # (values of two bits by a power of two: exact in every type at this size)
    assert (f64(y) == dense.mx4_values(codes, sc)[:, :cols]).all()


def test_every_tie_and_its_neighbours(alcs):
    """A block's largest value fixes the scale to 1; the others stand on, just below and just above every border, both signs."""
    torch = _torch()
    q = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0], np.float32)
    q = np.concatenate([q, np.nextafter(q, np.float32(0)), np.nextafter(q, np.float32(9)), [0.0, 1e-30]]).astype(np.float32)
    v = np.concatenate([q, -q])
    v = np.concatenate([v, np.zeros(-len(v) % 31, np.float32)]).reshape(-1, 31)
    x = np.concatenate([np.full((len(v), 1), 4.0, np.float32), v], 1)
    for scale in (2.0 ** -120, 1.0, 2.0 ** 90):
        _check_quantized(alcs, torch.from_numpy((x * np.float32(scale)).astype(np.float32)).cuda(), 32, 32, "f32")


def test_smallest_largest_and_not_finite(alcs):
    torch = _torch()
    x = torch.zeros(12, 96)
    x[0, 0], x[1, 0], x[2, 0] = 2.0 ** -149, 3.4e38, -2.0 ** -126
    x[3, 40], x[4, 40], x[5, 95] = float("inf"), float("nan"), float("-inf")
    x[6] = -0.0
    x[7, :32], x[8] = 2.0 ** -130, 2.0 ** -127
    x[9, :3] = torch.tensor([2.0 ** -125, 2.0 ** -126, 2.0 ** -127])
    data, scales, codes, sc = _check_quantized(alcs, x.cuda(), 96, 96, "f32")
    assert sc[3, 1] == 255 and sc[3, 0] == 0 and sc[4, 1] == 255 and sc[5, 2] == 255 and (codes[6] == 8).all()
    y = torch.empty(12, 96, device="cuda")
    alcs.alcs_mx4_dequantize(data, scales, 12, 96, y, 96, alcs.ALCS_F32, torch.cuda.current_stream())
    v = dense.mx4_values(codes, sc)
    assert np.array_equal(f64(y), v, equal_nan=True)
    y16 = torch.empty(12, 96, device="cuda", dtype=torch.float16)
    alcs.alcs_mx4_dequantize(data, scales, 12, 96, y16, 96, alcs.ALCS_F16, torch.cuda.current_stream())
    assert torch.equal(y16.isnan(), y.isnan()) and y16[1, 0] == float("inf") and y16[0, 0] == 0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols,ld,offset", [(64, 72, 0), (64, 65, 0), (100, 104, 0), (96, 96, 1), (40, 48, 3), (33, 40, 2)])
def test_rows_apart_and_buffers_that_start_anywhere(alcs, dtype, cols, ld, offset):
    torch = _torch()
    t = types(alcs)[dtype][1]
    rows = 37
    m = torch.randn(offset + rows * ld + 8, device="cuda").to(t)
    x = m[offset:offset + rows * ld].view(rows, ld)
    data, scales, codes, sc = _check_quantized(alcs, x, cols, ld, dtype)
    out = torch.full((offset + rows * ld + 8,), 77.0, device="cuda", dtype=t)
    y = out[offset:offset + rows * ld].view(rows, ld)
    alcs.alcs_mx4_dequantize(data, scales, rows, cols, y, ld, types(alcs)[dtype][0], torch.cuda.current_stream())
    assert (f64(y)[:, :cols] == dense.mx4_values(codes, sc)[:, :cols]).all()
    assert (y[:, cols:] == 77).all() and (out[:offset] == 77).all() and (out[offset + rows * ld:] == 77).all()


def _matrix(seed, rows, cols, positive=False, spread=3):
    """Codes and scales as they come: any code, scales of 2^-spread to 2^spread."""
    r = np.random.default_rng(seed)
    nb = -(-cols // 32)
    codes = r.integers(0, 8 if positive else 16, (rows, nb * 32), dtype=np.uint8)
    codes[:, cols:] = 0
    return codes, r.integers(127 - spread, 128 + spread, (rows, nb), dtype=np.uint8)


def _device(codes, scales, cols, fill=0xFF):
    """The storage format on the device; rows behind the last hold NaN scales and codes of 6."""
    torch = _torch()
    return tuple(torch.from_numpy(a).cuda() for a in dense.mx4_store(codes, scales, cols, fill))


class Product:
    def __init__(self, alcs, rows, cin, cout, dtype, bias=True, residual=False, relu=False, seed=0):
        torch = _torch()
        self.alcs, self.rows, self.cin, self.cout, self.dtype, self.relu = alcs, rows, cin, cout, dtype, relu
        self.dt, t = types(alcs)[dtype]
        self.cx, self.cw = _matrix(seed + 1, rows, cin), _matrix(seed + 2, cout, cin)
        self.x, self.w = _device(*self.cx, cin), _device(*self.cw, cin)
        r = np.random.default_rng(seed + 3)
        self.bias = torch.from_numpy(r.normal(size=cout).astype(np.float32)).cuda() if bias else None
        self.res = torch.from_numpy(r.normal(size=(rows, cout)).astype(np.float32)).cuda().to(t) if residual else None
        self.y = torch.full((rows, cout), float("nan"), dtype=t, device="cuda")

    def run(self, stream=None, y=None, res=None):
        y = self.y if y is None else y
        self.alcs.alcs_mx4_product(*self.x, self.rows, *self.w, self.cout, self.cin, y, self.bias, self.res if res is None else res,
                                   self.alcs.ALCS_RELU if self.relu else 0, self.dt, stream or _torch().cuda.current_stream())
        return y

    def expected(self):
        xv, wv = dense.mx4_values(*self.cx)[:, :self.cin], dense.mx4_values(*self.cw)[:, :self.cin]
        ref, scale = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
        for t in (self.bias, self.res):
            if t is not None:
                ref, scale = ref + f64(t), scale + np.abs(f64(t))
        bound = product_bound(scale, ref, self.cin, self.dtype)
        return (np.maximum(ref, 0) if self.relu else ref), bound

    def check(self):
        ref, bound = self.expected()
        got = f64(self.y)
        assert np.isfinite(got).all()
        assert (np.abs(got - ref) <= bound).all(), float((np.abs(got - ref) / bound).max())
        assert self.alcs.alcs_mx4_status() == 0


# rows, cin, cout: single rows; one block, half a step, part of a stage; tiles of 128 rows and their borders; tiles of 64 .. 256 channels; columns shared by
# clusters of 2, 4, 8, with pixels as rows of the tiles and as columns (up to 64); more tiles than SMs; a long sum
SIZES = [(1, 32, 16), (1, 1, 1), (1, 1024, 1000), (2, 100, 7), (16, 64, 128), (17, 96, 130), (49, 512, 512), (64, 320, 64), (65, 320, 64), (127, 64, 129),
         (128, 128, 128), (129, 160, 257), (300, 1000, 300), (196, 4096, 64), (1955, 100, 150), (700, 96, 1031), (2500, 224, 192), (5000, 64, 200),
         (9000, 128, 256), (9500, 40, 64), (6000, 130, 520), (33, 8192, 100), (3, 2048, 4096), (40000, 32, 24),
         (1, 1500, 40), (64, 1600, 300), (130, 3500, 70), (250, 3200, 120), (17, 2600, 999),
         (4900, 800, 2200), (6400, 1025, 2304), (2600, 2100, 4100)]


@pytest.mark.parametrize("rows,cin,cout", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_product(alcs, rows, cin, cout, dtype):
    k = Product(alcs, rows, cin, cout, dtype, residual=rows % 2 == 1, relu=cout % 3 == 0)
    k.run()
    k.check()


@pytest.mark.parametrize("rows,cin,cout", [(5, 200, 40), (200, 512, 72), (3000, 128, 72), (5, 2000, 40), (200, 4000, 72)])
def test_residual_is_the_output_and_odd_starts(alcs, rows, cin, cout):
    torch = _torch()
    k = Product(alcs, rows, cin, cout, "bf16", residual=True, relu=True)
    k.run()
    k.check()
    y = k.res.clone()
    assert (k.run(y=y, res=y) == k.y).all()
    # outputs that do not start on 16 bytes: stored one by one
    m = torch.full((rows * cout + 9,), 77.0, dtype=torch.bfloat16, device="cuda")
    v = m[3:3 + rows * cout].view(rows, cout)
    assert (k.run(y=v) == k.y).all() and (m[:3] == 77).all() and (m[3 + rows * cout:] == 77).all()


@pytest.mark.parametrize("rows,cout", [(3, 5), (200, 33)])
def test_no_columns(alcs, rows, cout):
    torch = _torch()
    bias = torch.randn(cout, device="cuda")
    y = torch.full((rows, cout), float("nan"), device="cuda")
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    alcs.alcs_mx4_product(none, none, rows, none, none, cout, 0, y, bias, None, alcs.ALCS_RELU, alcs.ALCS_F32, torch.cuda.current_stream())
    assert (y == bias.clamp(min=0)).all()


@pytest.mark.parametrize("rows,cin,cout", [(4, 256, 70), (300, 256, 70), (4, 2048, 70), (300, 3200, 70)])
def test_nan_blocks_take_their_row_and_column_alone(alcs, rows, cin, cout):
    k = Product(alcs, rows, cin, cout, "f32")
    clean = k.run().clone()
    for which, at in (("cx", (rows - 1, 5)), ("cw", (66, 0))):
        codes, sc = getattr(k, which)
        sc = sc.copy()
        sc[at] = 255
        saved = k.x, k.w
        k.x, k.w = (_device(codes, sc, cin), k.w) if which == "cx" else (k.x, _device(codes, sc, cin))
        y = k.run().clone()
        nan = np.zeros((rows, cout), bool)
        nan[(at[0], slice(None)) if which == "cx" else (slice(None), at[0])] = True
        assert (y.isnan().cpu().numpy() == nan).all()
        assert (y.cpu().numpy()[~nan] == clean.cpu().numpy()[~nan]).all()
        k.x, k.w = saved


def test_scales_at_the_ends_of_their_range(alcs):
    """2^-100 times 2^100, 2^-127 times 2^127; products below fp32's range vanish, above it are infinite."""
    torch = _torch()
    for sx, sw, want in ((27, 227, 1.0), (0, 254, 1.0), (0, 0, 0.0), (254, 254, float("inf"))):
        cx, cw = np.full((4, 32), 2, np.uint8), np.full((16, 32), 2, np.uint8)      # ones
        x, w = _device(cx, np.full((4, 1), sx, np.uint8), 32), _device(cw, np.full((16, 1), sw, np.uint8), 32)
        y = torch.empty(4, 16, device="cuda")
        alcs.alcs_mx4_product(*x, 4, *w, 16, 32, y, None, None, 0, alcs.ALCS_F32, torch.cuda.current_stream())
        assert (y == 32 * want).all(), (sx, sw, y[0, 0].item())


def test_streams_graphs_and_the_same_bits(alcs):
    torch = _torch()
    sizes = [(3, 2048, 512), (300, 1024, 300), (5000, 128, 200)]
    want = [Product(alcs, *s, "bf16", residual=True).run().clone() for s in sizes]
    work = [Product(alcs, *s, "bf16", residual=True) for s in sizes]
    streams = [torch.cuda.Stream() for _ in sizes]
    torch.cuda.synchronize()
    graphs = []
    for k, s in zip(work, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            k.run(s)
        graphs.append(g)
    for _ in range(4):
        for k in work:
            k.y.fill_(float("nan"))
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        for k, s in zip(work, streams):      # an eager call behind the replay, on its stream
            k.run(s)
        torch.cuda.synchronize()
        for k, w in zip(work, want):
            assert (k.y == w).all()
    assert alcs.alcs_mx4_status() == 0


def test_outputs_and_inputs_beyond_32_bits(alcs):
    """2^20 + 200 rows of 4096 channels: more than 2^32 outputs.  And rows 2^31 elements apart."""
    torch = _torch()
    rows, cin, cout = (1 << 20) + 200, 64, 4096
    x = torch.randn(rows, cin, device="cuda").to(torch.bfloat16)
    w = torch.randn(cout, cin, device="cuda").to(torch.bfloat16)
    xq, wq = _quantize(alcs, x, cin, cin, "bf16"), _quantize(alcs, w, cin, cin, "bf16")
    y = torch.empty(rows, cout, dtype=torch.bfloat16, device="cuda")
    st = torch.cuda.current_stream()
    alcs.alcs_mx4_product(*xq, rows, *wq, cout, cin, y, None, None, 0, alcs.ALCS_BF16, st)
    tail = _quantize(alcs, x[-300:].contiguous(), cin, cin, "bf16")
    part = torch.empty(300, cout, dtype=torch.bfloat16, device="cuda")
    alcs.alcs_mx4_product(*tail, 300, *wq, cout, cin, part, None, None, 0, alcs.ALCS_BF16, st)
    assert (y[-300:] == part).all()
    del y
    far = torch.empty(2, (1 << 31) + 8, dtype=torch.bfloat16, device="cuda")
    far[:, :64] = x[:2]
    q = _quantize(alcs, far, 64, far.shape[1], "bf16")
    near = _quantize(alcs, x[:2].contiguous(), 64, 64, "bf16")
    assert (q[0] == near[0]).all() and (q[1] == near[1]).all()


def test_a_pruned_layer_in_four_bits_behind_a_norm(alcs):
    """What a user runs together: norm with SiLU, its output to 4 bits, the pruned weights (unpacked) in 4 bits, the product with bias,
    shortcut and ReLU.  Every stage against its definition on what the stage before it gave."""
    torch = _torch()
    n, h, wd, c, cout, groups, g = 4, 14, 14, 256, 192, 32, 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    st = torch.cuda.current_stream()
    x, gamma, beta = rnd(n, h * wd, c).to(torch.bfloat16), 1 + 0.2 * rnd(c), 0.2 * rnd(c)
    z = torch.empty_like(x)
    alcs.alcs_group_norm(x, z, n, h, wd, c, groups, gamma, beta, 1e-5, alcs.ALCS_SILU, alcs.ALCS_BF16, stream=st)
    ref = dense.group_norm(f64(x), groups, f64(gamma), f64(beta), 1e-5, "silu")
    assert (np.abs(f64(z) - ref["y"]) <= norm_bound(ref, f64(x), f64(gamma), f64(beta), groups, "bf16")).all()
    r = np.random.default_rng(9)
    mask = (r.random((cout // g, c)) < 0.3).astype(np.uint8)
    weights, _ = alcs.alcs_unpack(alcs.alcs_pack((r.normal(size=(cout, c)) / 8).astype(np.float32), mask, g))
    assert ((weights == 0) == (np.repeat(mask, g, 0) == 0)).all()
    zq = _quantize(alcs, z.view(n * h * wd, c), c, c, "bf16")
    wt = torch.from_numpy(weights).cuda()
    wq = _quantize(alcs, wt, c, c, "f32")
    bias, short = rnd(cout), rnd(n * h * wd, cout).to(torch.bfloat16)
    y = torch.empty_like(short)
    alcs.alcs_mx4_product(*zq, n * h * wd, *wq, cout, c, y, bias, short, alcs.ALCS_RELU, alcs.ALCS_BF16, st)
    zv = dense.mx4_values(*dense.mx4_quantize(f64(z).reshape(-1, c)))
    wv = dense.mx4_values(*dense.mx4_quantize(f64(wt)))
    out = zv @ wv.T + f64(bias) + f64(short)
    bound = product_bound(np.abs(zv) @ np.abs(wv).T + np.abs(f64(bias)) + np.abs(f64(short)), out, c, "bf16")
    assert (np.abs(f64(y) - np.maximum(out, 0)) <= bound).all()


def test_host_memory_is_refused(alcs):
    torch = _torch()
    k = Product(alcs, 4, 64, 32, "f32")
    for args in ((k.x[0].cpu(), k.x[1]), (k.x[0], k.x[1].cpu())):
        with pytest.raises(alcs.AlcsError) as e:
            alcs.alcs_mx4_product(*args, 4, *k.w, 32, 64, k.y, stream=torch.cuda.current_stream())
        assert e.value.status == alcs.ALCS_ERR_INVALID_ARG
    with pytest.raises(alcs.AlcsError):
        alcs.alcs_mx4_quantize(torch.randn(4, 64), 4, 64, 64, alcs.ALCS_F32, *k.x, torch.cuda.current_stream())
