"""What group norm and the 4-bit operators refuse, and the sizes they report: decided on the host before anything touches a device."""
import pytest

U8 = 0x10000       # an address that no check before the device's looks behind


def _status(alcs, f, *args, **kw):
    try:
        f(*args, **kw)
    except alcs.AlcsError as e:
        return e.status
    return 0


NORM = dict(x=U8, y=1 << 30, n=2, h=4, wd=4, c=64, groups=8, gamma=1 << 33, beta=(1 << 33) + 4096, eps=1e-5, flags=0, dt=2, mean=1 << 34,
            rstd=(1 << 34) + 4096, workspace=None, workspace_bytes=0)
BACK = dict(x=U8, dy=1 << 29, dx=1 << 30, n=2, h=4, wd=4, c=64, groups=8, mean=1 << 34, rstd=(1 << 34) + 4096, gamma=1 << 33, beta=(1 << 33) + 4096,
            dgamma=1 << 35, dbeta=(1 << 35) + 4096, flags=0, dt=2, workspace=1 << 36, workspace_bytes=1 << 20)
PRODUCT = dict(x=U8, x_scales=1 << 28, rows=4, w=1 << 29, w_scales=(1 << 29) + (1 << 20), cout=64, cin=64, y=1 << 30, bias=1 << 33, residual=1 << 31,
               flags=0, dt=2)
QUANTIZE = dict(x=U8, rows=4, cols=64, ldx=64, dt=2, data=1 << 30, scales=1 << 31)
DEQUANTIZE = dict(data=1 << 30, scales=1 << 31, rows=4, cols=64, y=U8, ldy=64, dt=2)

INVALID, SHAPE = -1, -2
REFUSED = [
    ("alcs_group_norm", NORM, dict(x=None), INVALID), ("alcs_group_norm", NORM, dict(y=None), INVALID),
    ("alcs_group_norm", NORM, dict(x=U8 + 1), INVALID), ("alcs_group_norm", NORM, dict(gamma=2), INVALID),
    ("alcs_group_norm", NORM, dict(y=U8 + 2), INVALID), ("alcs_group_norm", NORM, dict(mean=U8 + 64), INVALID),
    ("alcs_group_norm", NORM, dict(mean=1 << 34, rstd=1 << 34), INVALID), ("alcs_group_norm", NORM, dict(beta=1 << 30), INVALID),
    ("alcs_group_norm", NORM, dict(n=-1), INVALID), ("alcs_group_norm", NORM, dict(h=-1), INVALID), ("alcs_group_norm", NORM, dict(c=-8), INVALID),
    ("alcs_group_norm", NORM, dict(groups=0), INVALID), ("alcs_group_norm", NORM, dict(groups=7), SHAPE),
    ("alcs_group_norm", NORM, dict(c=1 << 17, groups=1 << 10), SHAPE), ("alcs_group_norm", NORM, dict(h=1 << 15, wd=1 << 15), SHAPE),
    ("alcs_group_norm", NORM, dict(c=8256, groups=1), -3), ("alcs_group_norm_backward", BACK, dict(c=16400, groups=2), -3),
    ("alcs_group_norm", NORM, dict(n=1 << 24), SHAPE), ("alcs_group_norm", NORM, dict(eps=-1.0), INVALID),
    ("alcs_group_norm", NORM, dict(eps=float("nan")), INVALID), ("alcs_group_norm", NORM, dict(eps=float("inf")), INVALID),
    ("alcs_group_norm", NORM, dict(flags=2), INVALID), ("alcs_group_norm", NORM, dict(flags=5), INVALID), ("alcs_group_norm", NORM, dict(flags=8), INVALID),
    ("alcs_group_norm", NORM, dict(dt=3), INVALID), ("alcs_group_norm", NORM, dict(dt=-1), INVALID),
    # a shape of two passes without its workspace
    ("alcs_group_norm", NORM, dict(h=512, wd=512, y=1 << 32, gamma=None, beta=None), INVALID),
    ("alcs_group_norm_backward", BACK, dict(dy=None), INVALID), ("alcs_group_norm_backward", BACK, dict(dx=None), INVALID),
    ("alcs_group_norm_backward", BACK, dict(mean=None), INVALID), ("alcs_group_norm_backward", BACK, dict(rstd=None), INVALID),
    ("alcs_group_norm_backward", BACK, dict(workspace=None), INVALID), ("alcs_group_norm_backward", BACK, dict(workspace_bytes=1023), INVALID),
    ("alcs_group_norm_backward", BACK, dict(workspace=(1 << 36) + 8), INVALID), ("alcs_group_norm_backward", BACK, dict(workspace=1 << 30), INVALID),
    ("alcs_group_norm_backward", BACK, dict(dgamma=(1 << 35) + 4096), INVALID), ("alcs_group_norm_backward", BACK, dict(dx=U8 + 2), INVALID),
    ("alcs_group_norm_backward", BACK, dict(dbeta=1 << 34), INVALID), ("alcs_group_norm_backward", BACK, dict(flags=5), INVALID),
    ("alcs_group_norm_backward", BACK, dict(groups=5), SHAPE), ("alcs_group_norm_backward", BACK, dict(dt=7), INVALID),
    ("alcs_mx4_quantize", QUANTIZE, dict(x=None), INVALID), ("alcs_mx4_quantize", QUANTIZE, dict(data=None), INVALID),
    ("alcs_mx4_quantize", QUANTIZE, dict(scales=None), INVALID), ("alcs_mx4_quantize", QUANTIZE, dict(data=(1 << 30) + 8), INVALID),
    ("alcs_mx4_quantize", QUANTIZE, dict(scales=(1 << 31) + 4), INVALID), ("alcs_mx4_quantize", QUANTIZE, dict(x=U8 + 1), INVALID),
    ("alcs_mx4_quantize", QUANTIZE, dict(ldx=63), INVALID), ("alcs_mx4_quantize", QUANTIZE, dict(rows=-1), INVALID),
    ("alcs_mx4_quantize", QUANTIZE, dict(cols=-1, ldx=0), INVALID), ("alcs_mx4_quantize", QUANTIZE, dict(dt=3), INVALID),
    ("alcs_mx4_quantize", QUANTIZE, dict(data=U8), INVALID), ("alcs_mx4_quantize", QUANTIZE, dict(scales=1 << 30), INVALID),
    ("alcs_mx4_quantize", QUANTIZE, dict(cols=(1 << 24) + 1, ldx=1 << 25), SHAPE), ("alcs_mx4_quantize", QUANTIZE, dict(rows=(1 << 30) + 1), SHAPE),
    ("alcs_mx4_quantize", QUANTIZE, dict(ldx=1 << 50), SHAPE),
    ("alcs_mx4_dequantize", DEQUANTIZE, dict(y=None), INVALID), ("alcs_mx4_dequantize", DEQUANTIZE, dict(y=1 << 30), INVALID),
    ("alcs_mx4_dequantize", DEQUANTIZE, dict(ldy=1), INVALID), ("alcs_mx4_dequantize", DEQUANTIZE, dict(data=1), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(x=None), INVALID), ("alcs_mx4_product", PRODUCT, dict(x_scales=None), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(w=None), INVALID), ("alcs_mx4_product", PRODUCT, dict(w_scales=None), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(y=None), INVALID), ("alcs_mx4_product", PRODUCT, dict(x=U8 + 8), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(w_scales=(1 << 29) + 8), INVALID), ("alcs_mx4_product", PRODUCT, dict(y=(1 << 30) + 1), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(bias=(1 << 33) + 2), INVALID), ("alcs_mx4_product", PRODUCT, dict(residual=(1 << 31) + 1), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(residual=(1 << 30) + 2), INVALID), ("alcs_mx4_product", PRODUCT, dict(y=U8), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(y=1 << 29), INVALID), ("alcs_mx4_product", PRODUCT, dict(flags=2), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(flags=4), INVALID), ("alcs_mx4_product", PRODUCT, dict(dt=9), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(rows=-4), INVALID), ("alcs_mx4_product", PRODUCT, dict(cout=-1), INVALID),
    ("alcs_mx4_product", PRODUCT, dict(cin=-1), INVALID), ("alcs_mx4_product", PRODUCT, dict(cin=(1 << 24) + 1), SHAPE),
    ("alcs_mx4_product", PRODUCT, dict(rows=(1 << 30) + 1), SHAPE), ("alcs_mx4_product", PRODUCT, dict(cout=(1 << 24) + 1), SHAPE),
]


@pytest.mark.parametrize("name,args,wrong,status", REFUSED, ids=[f"{n[5:]}-{w}" for n, _, w, _ in REFUSED])
def test_refused_before_the_device(alcs, name, args, wrong, status):
    assert _status(alcs, getattr(alcs, name), **{**args, **wrong}) == status


@pytest.mark.parametrize("name,args,empty", [("alcs_group_norm", NORM, dict(n=0)), ("alcs_group_norm", NORM, dict(h=0)),
                                             ("alcs_group_norm", NORM, dict(c=0, x=None, y=None)),
                                             ("alcs_group_norm_backward", BACK, dict(c=0)),
                                             ("alcs_mx4_quantize", QUANTIZE, dict(rows=0, x=None)), ("alcs_mx4_quantize", QUANTIZE, dict(cols=0)),
                                             ("alcs_mx4_dequantize", DEQUANTIZE, dict(rows=0)), ("alcs_mx4_product", PRODUCT, dict(rows=0, y=None)),
                                             ("alcs_mx4_product", PRODUCT, dict(cout=0, w=None))])
def test_nothing_to_do(alcs, name, args, empty):
    assert _status(alcs, getattr(alcs, name), **{**args, **empty}) == 0


def test_without_a_device_or_its_memory(alcs):
    """Addresses that are no device memory: no device at all, or not its memory."""
    for name, args in (("alcs_group_norm", NORM), ("alcs_group_norm_backward", BACK), ("alcs_mx4_quantize", QUANTIZE),
                       ("alcs_mx4_dequantize", DEQUANTIZE), ("alcs_mx4_product", PRODUCT)):
        assert _status(alcs, getattr(alcs, name), **args) in (alcs.ALCS_ERR_CUDA, alcs.ALCS_ERR_INVALID_ARG)


def test_sizes(alcs):
    assert alcs.alcs_mx4_bytes(0, 64) == (0, 0) and alcs.alcs_mx4_bytes(5, 0) == (0, 0)
    assert alcs.alcs_mx4_bytes(1, 1) == (2 * 2048, 512) and alcs.alcs_mx4_bytes(128, 64) == (2 * 2048, 512)
    assert alcs.alcs_mx4_bytes(129, 65) == (2 * 4 * 2048, 2 * 512) and alcs.alcs_mx4_bytes(128, 129) == (6 * 2048, 2 * 512)
    assert alcs.alcs_mx4_bytes(1 << 30, 1 << 24) == (1 << 53, 1 << 49)
    for rows, cols in ((-1, 1), (1, -1), ((1 << 30) + 1, 1), (1, (1 << 24) + 1)):
        with pytest.raises(alcs.AlcsError):
            alcs.alcs_mx4_bytes(rows, cols)


def test_workspace_of_group_norm(alcs):
    """At least two sums per channel and image; more where an image is spread over blocks; nothing for nothing."""
    assert alcs.alcs_group_norm_workspace(2, 7, 7, 64, 8, alcs.ALCS_BF16) >= 2 * 2 * 64 * 4
    assert alcs.alcs_group_norm_workspace(1, 512, 512, 64, 8, alcs.ALCS_F32) > 2 * 64 * 4
    for args in ((0, 7, 7, 64, 8, 0), (2, 0, 7, 64, 8, 0), (2, 7, 7, 0, 8, 0), (2, 7, 7, 64, 0, 0), (2, 7, 7, 64, 7, 0), (2, 7, 7, 64, 8, 5), (-2, 7, 7, 64, 8, 0)):
        assert alcs.alcs_group_norm_workspace(*args) == 0
