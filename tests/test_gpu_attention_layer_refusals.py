"""Steps that a served layer refuses: before anything is launched, and with its sequences as they were."""
import pytest
import torch

from paper_2311_03285_amd import slora
from paper_2311_03285_amd.attention_layer import AttentionLayer

pytestmark = pytest.mark.gpu


def test_a_refused_step_changes_nothing():
    with AttentionLayer(H=512, n_heads=8, layers=1, pool_pages=1000, max_seqs=2, max_tokens=60, budget=20, recent=4, ranks={0: 8}, seed=3) as m:
        x = torch.randn(26, 512, device="cuda").to(m.dtype)
        m.step([0, 1], [15, 11], [0, 0], x)
        free = slora.pool_free_pages(m.pool)
        for bad in (x[:2], x.float(), x[:, :256], x.cpu(), torch.empty((512, 26), dtype=m.dtype, device="cuda").t(), torch.cat([x, x[:1]])):
            with pytest.raises(ValueError):
                m.step([0, 1], [15, 11], [0, 0], bad)
        with pytest.raises(ValueError):
            m.step([0, 1], [15, 11], [0], x)
        for seqs, adapters, code in (([0, 1], [0, 5], slora.ENOENT), ([0, 0], [0, 0], slora.EBUSY), ([0, 2], [0, 0], slora.ERANGE)):
            with pytest.raises(slora.SloraError) as e:
                m.step(seqs, [15, 11], adapters, x)
            assert e.value.code == code
        with pytest.raises(slora.SloraError) as e:
            m.step([0, 1], [1, 50], [0, 0], torch.randn(51, 512, device="cuda").to(m.dtype))  # beyond max_tokens
        assert e.value.code == slora.ERANGE
        assert slora.kv8_lengths(m.cache, [0, 1]).tolist() == [15, 11] and slora.pool_free_pages(m.pool) == free
        out = m.step([0, 1], [15, 11], [0, 0], x)
        torch.cuda.synchronize()
        assert torch.isfinite(out[0]).all() and slora.kv8_lengths(m.cache, [0, 1]).tolist() == [20, 20]
