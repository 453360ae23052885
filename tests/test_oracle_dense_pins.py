"""The 64-bit definitions of group norm and of microscaled 4-bit floating point against what they have to be: closed forms,
differences, brute force over all codes."""
import numpy as np
import pytest

from oracle import dense


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_group_norm_gradients_are_the_differences(act):
    r = np.random.default_rng(3)
    n, hw, c, groups = 2, 5, 6, 3
    x, dy = r.normal(size=(n, hw, c)) * 2 + 1, r.normal(size=(n, hw, c))
    gamma, beta = r.normal(size=c) + 1, r.normal(size=c)
    b = dense.group_norm_backward(x, dy, groups, gamma, beta, act=act)
    assert act != "relu" or np.abs(b["z"]).min() > 1e-4       # (no kink within the step)
    loss = lambda x, gamma, beta: (dense.group_norm(x, groups, gamma, beta, act=act)["y"] * dy).sum()  # noqa: E731
    h = 1e-6
    for which, grad in ((0, b["dx"]), (1, b["dgamma"]), (2, b["dbeta"])):
        args = [x, gamma, beta]
        flat = np.empty(grad.size)
        for i in range(grad.size):
            d = np.zeros(grad.size)
            d[i] = h
            up, down = list(args), list(args)
            up[which], down[which] = args[which] + d.reshape(grad.shape), args[which] - d.reshape(grad.shape)
            flat[i] = (loss(*up) - loss(*down)) / (2 * h)
        # central differences: h^2 times a third derivative of order 1, and 2^-53 |loss| / h
        assert np.abs(flat.reshape(grad.shape) - grad).max() < 1e-7


def test_group_norm_of_a_library():
    torch = pytest.importorskip("torch")
    r = np.random.default_rng(4)
    x, gamma, beta = r.normal(size=(3, 7, 12)), r.normal(size=12), r.normal(size=12)
    ref = torch.nn.functional.group_norm(torch.from_numpy(x).permute(0, 2, 1), 4, torch.from_numpy(gamma), torch.from_numpy(beta), 1e-3)
    assert np.abs(dense.group_norm(x, 4, gamma, beta, 1e-3)["y"] - ref.permute(0, 2, 1).numpy()).max() < 1e-13


def test_group_norm_of_a_constant_is_beta():
    f = dense.group_norm(np.full((1, 4, 6), 3.0), 2, np.arange(6.0), np.arange(6.0) - 2)
    assert (f["xh"] == 0).all() and (f["y"] == np.arange(6.0) - 2).all()


def test_mx4_rounding_is_the_nearest_code_with_ties_to_even():
    q = np.concatenate([np.arange(-9, 9, 1 / 64), [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 1e9], [np.nextafter(0.25, 1), np.nextafter(5, 0)]])
    codes = dense.mx4_round(q)
    for v, c in zip(q, codes):
        d = np.abs(dense.MX4_VALUES - min(abs(v), 6.0))
        best = np.flatnonzero(d == d.min())
        assert c % 8 == (best[0] if best.size == 1 else next(b for b in best if b % 2 == 0))
        assert c // 8 == np.signbit(v)
    assert [int(c) for c in dense.mx4_round(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]))] == [0, 2, 2, 4, 4, 6, 6]


@pytest.mark.parametrize("top,byte", [(0.0, 0), (1.0, 125), (1.999, 125), (2.0, 126), (6.0, 127), (7.9, 127), (8.0, 128), (3e38, 252),
                                      (2.0 ** -126, 0), (2.0 ** -125, 0), (2.0 ** -124, 1), (2.0 ** -149, 0)])
def test_mx4_scale_is_the_exponent_of_the_largest_less_two(top, byte):
    x = np.zeros((1, 32))
    x[0, 5] = top
    codes, scales = dense.mx4_quantize(x)
    assert scales[0, 0] == byte
    v = dense.mx4_values(codes, scales)[0, 5]
    # half a step of the codes from 4 on (1 of 4), or the clamp at 6 of a value below 8
    assert top < 2.0 ** -126 or abs(v - top) <= top / 4


def test_mx4_storage_holds_every_block_once():
    r = np.random.default_rng(5)
    for rows, cols in ((1, 1), (3, 33), (130, 100), (257, 320)):
        nb = -(-cols // 32)
        codes, scales = r.integers(0, 16, (rows, nb * 32), dtype=np.uint8), r.integers(0, 255, (rows, nb), dtype=np.uint8)
        data, sc = dense.mx4_store(codes, scales, cols)
        c, s = dense.mx4_load(data, sc, rows, cols)
        assert (c == codes).all() and (s == scales).all()
        rr, bb = np.meshgrid(np.arange(rows), np.arange(nb), indexing="ij")
        assert np.unique(dense.mx4_data_index(rr, bb, cols)).size == rows * nb and dense.mx4_data_index(rr, bb, cols).max() + 16 <= data.size
        assert np.unique(dense.mx4_scale_index(rr, bb, cols)).size == rows * nb and dense.mx4_scale_index(rr, bb, cols).max() < sc.size


def test_mx4_blocks_that_are_not_finite_are_nan():
    x = np.ones((2, 40))
    x[0, 3], x[1, 39] = np.inf, np.nan
    v = dense.mx4_values(*dense.mx4_quantize(x))
    assert np.isnan(v[0, :32]).all() and (v[0, 32:40] == 1).all() and (v[1, :32] == 1).all() and np.isnan(v[1, 32:40]).all()
