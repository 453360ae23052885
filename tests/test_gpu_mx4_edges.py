"""The 4-bit product at the ends of its ranges."""
import pytest

pytestmark = pytest.mark.gpu


def _values(data, rows, first, last):
    """The values of blocks first .. last of the first rows, scales 1, as float64 on the device: the storage order undone."""
    import torch
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda", dtype=torch.float64)
    table = torch.cat([table, -table])
    b = data[:, first:last, :min(rows, 128)].permute(0, 2, 1, 3).reshape(-1, (last - first) * 16)[:rows].int()
    return table[torch.stack([b & 15, b >> 4], 2).view(rows, -1)]


# one row in a cluster, as columns of the tiles; tiles shared by clusters; a block per tile: each up to the longest rows that memory or time allow
@pytest.mark.parametrize("rows,cin,cout", [(1, 1 << 24, 16), (65, 1 << 24, 8), (200, 1 << 21, 300), (9600, 1 << 17, 256), (130, (1 << 20) + 64, 72)])
def test_long_rows(alcs, rows, cin, cout):
    """Random codes, scales of 1.  Every product is a multiple of 1/4 of at most 36 and sums of them are random walks, of cin = 2^24 some 12 x 2^12 and far below
    2^22: they are numbers of fp32, and so are all partial sums, in whatever order.  The result has to be equal."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    tiles = lambda r: -(-r // 128)  # noqa: E731
    blocks, quads = cin // 32, -(-cin // 128)
    x, w = (torch.randint(0, 256, (tiles(r), blocks, 128, 16), generator=g, device="cuda", dtype=torch.uint8) for r in (rows, cout))
    sx, sw = (torch.full((tiles(r) * quads * 512,), 127, device="cuda", dtype=torch.uint8) for r in (rows, cout))
    assert (x.numel(), sx.numel()) == alcs.alcs_mx4_bytes(rows, cin)
    y = torch.full((rows, cout), float("nan"), device="cuda")
    alcs.alcs_mx4_product(x, sx, rows, w, sw, cout, cin, y, None, None, 0, alcs.ALCS_F32, torch.cuda.current_stream())
    assert alcs.alcs_mx4_status() == 0
    want = torch.zeros(rows, cout, device="cuda", dtype=torch.float64)
    step = max(1, (1 << 26) // (32 * max(rows, cout)))
    for b in range(0, blocks, step):
        want += _values(x, rows, b, min(blocks, b + step)) @ _values(w, cout, b, min(blocks, b + step)).T
    assert want.abs().max() < 2 ** 21
    assert (y == want).all()
