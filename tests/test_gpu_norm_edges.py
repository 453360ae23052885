"""Group norm at the edges of its ranges: clusters with blocks that have no pixels; chains of calls through the same buffers."""
import pytest

import test_gpu_norm as norm

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
