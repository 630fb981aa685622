"""The calls for 8-bit layers and of what stands around a layer, together, as the example has them."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,n,f,experts", [(1, 512, 768, 4), (5, 1024, 2048, 8), (40, 768, 1536, 6), (64, 1024, 512, 16)])
def test_blocks_around_layers(tokens, n, f, experts):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2406_11235_amd import example_layers
    assert len(example_layers.main(tokens, n, f, experts, seed=tokens)) == 7
