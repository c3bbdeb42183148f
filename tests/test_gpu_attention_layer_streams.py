"""A served layer that is built while torch is on a side stream, behind work that is still running there, is the one that is built on the default stream."""
import pytest
import torch

from paper_2311_03285_amd.attention_layer import AttentionLayer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,wide", [(4, 0), (8, 200)])
def test_built_on_a_side_stream(bits, wide):
    sizes = dict(H=512, n_heads=8, layers=1, pool_pages=1000, max_seqs=2, max_tokens=60, budget=20, recent=4, ranks={0: 8, 1: 20}, seed=3, bits=bits, wide=wide)
    x = torch.randn(26, 512, device="cuda").half()
    ahead, side = torch.randn(4096, 4096, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            ahead = (ahead @ ahead).clamp_(-1, 1)
        m = AttentionLayer(**sizes)
    with m, AttentionLayer(**sizes) as want:
        if bits == 8:
            assert all(torch.equal(a, b) for a, b in zip(m.packed, want.packed))
        assert all(torch.equal(m.adapters[a], want.adapters[a]) for a in m.adapters)
        got, ref = (layer.step([0, 1], [15, 11], [0, 1], x)[0] for layer in (m, want))
        torch.cuda.synchronize()
        assert torch.equal(got, ref)
