"""A 4-bit weight made from its tiles: their number is checked before any kernel
reads them."""
import pytest

pytestmark = pytest.mark.gpu


def test_tiles_have_to_be_all_there():
    import torch
    from paper_2609_09240_gb300 import tq
    W = torch.randn((40, 256), device="cuda").half()
    a = tq.quantize_w4(W)
    b = tq.W4Weight(40, 256, a.tiles.clone())
    x = torch.randn((2, 256), device="cuda").half()
    assert torch.equal(tq.tq_w4_linear(x, a), tq.tq_w4_linear(x, b))
    n = a.tiles.numel()
    for bad in (a.tiles[:n - 1], a.tiles[:n // 2], torch.cat([a.tiles, a.tiles]), a.tiles.view(torch.int16),
                a.tiles.cpu(), a.tiles.view(-1, 16)):
        with pytest.raises(ValueError):
            tq.W4Weight(40, 256, bad)
    with pytest.raises(tq.TQError):
        tq.W4Weight(40, 200, a.tiles)
    with pytest.raises(TypeError):
        tq.W4Weight(40, 256, None)
