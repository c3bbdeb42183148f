"""Arguments that the calls on a cache with device memory refuse: with their code, before any launch, and with nothing changed."""
import pytest
import torch

from kv8_util import Twin
from paper_2311_03285_amd import slora
from test_host_kv8 import refused

pytestmark = pytest.mark.gpu


def test_what_is_refused():
    with Twin(512, 64, 2, 2, max_seqs=2, max_tokens=100) as t:
        t.step([0, 1], [40, 9])
        batch = t.step([0, 1], [1, 3])
        keeps = t.plan([0, 1], [0, 0], [30, 5])
        short = t.plan([0, 1], [100, 3])
        w, w_out, pos = t.weight_arrays()
        q = torch.zeros((4, 256), dtype=t.dtype, device="cuda")
        out = torch.full_like(q, 5.0)
        torch.cuda.synchronize()
        p, o, a, b, c = (x.data_ptr() for x in (q, out, w, w_out, pos))
        for layer in (-1, 1):
            refused(slora.ERANGE, slora.kv8_append, batch, layer, p, 256, p, 256)
            refused(slora.ERANGE, slora.kv8_attend, batch, layer, p, 256, o, 256, 0.1)
            refused(slora.ERANGE, slora.kv8_evict, keeps, layer, 1, a, b, c, c)
        for bad in ((0, 256, p, 256), (p, 256, 0, 256), (p + 8, 256, p, 256), (p, 256, p + 2, 256), (p, 120, p, 256), (p, 256, p, 132)):
            refused(slora.EINVAL, slora.kv8_append, batch, 0, *bad)
        refused(slora.EINVAL, slora.kv8_append, short, 0, p, 256, p, 256)
        for bad in ((0, 256, o, 256), (p, 256, 0, 256), (p + 8, 256, o, 256), (p, 256, o + 4, 256), (p, 248, o, 256), (p, 256, o, 260)):
            refused(slora.EINVAL, slora.kv8_attend, batch, 0, *bad, 0.1)
        for scale in (float("inf"), float("nan"), -float("inf"), 3e38):  # (times log2 e, in which scores are taken, the last is infinite as well)
            refused(slora.EINVAL, slora.kv8_attend, batch, 0, p, 256, o, 256, scale)
        for bad in ((a, b, None), (a, None, c), (None, b, c), (a, None, None), (a + 2, b, c), (a, b + 1, c), (a, b, c + 2)):
            refused(slora.EINVAL, slora.kv8_attend, batch, 0, p, 256, o, 256, 0.1, True, bad)
        refused(slora.EINVAL, slora.kv8_evict, batch, 0, 1, a, b, c, c)  # planned without keep
        refused(slora.EINVAL, slora.kv8_evict, keeps, 0, -1, a, b, c, c)
        for bad in ((0, b, c, c), (a, 0, c, c), (a, b, 0, c), (a, b, c, 0), (a + 1, b, c, c), (a, b, c, c + 2)):
            refused(slora.EINVAL, slora.kv8_evict, keeps, 0, 1, *bad)
        torch.cuda.synchronize()
        assert (out == 5.0).all() and (w_out == -1.0).all() and (pos == -1).all()
        t.check_contents()
        refused(slora.EINVAL, slora.kv8_init, t.lib_pool, 1, 4, 2, 64, 2, 100, None)
