"""The table gradient of a group has the same bits whatever other groups are in the call, and whatever columns stand beside its own."""
import pytest
import torch

from test_gpu_language import BF16, F32, b, randn, tokens          # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("G,T,V,D", [(4, 8192, 500, 2048), (32, 4096, 40, 1000), (9, 20000, 3000, 520), (16, 300, 30, 72)])
def test_gradient_of_a_shard(b, G, T, V, D, dtype, accumulate):
    dout, ids = randn(300, G, T, D, dtype=dtype), tokens(301, G, T, V)
    before = randn(302, G, V, D)
    whole = b.prsgd_embed_grad(dout, ids, before.clone(), accumulate=accumulate)
    for g in range(G):
        one = slice(g, g + 1)
        assert torch.equal(b.prsgd_embed_grad(dout[one], ids[one], before[one].clone(), accumulate=accumulate), whole[one]), g
    part = b.prsgd_embed_grad(dout[..., 8:40], ids, before[..., 8:40].contiguous(), accumulate=accumulate)
    assert torch.equal(part, whole[..., 8:40])
