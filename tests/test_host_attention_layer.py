"""What a served layer does with the library when it is built, without a GPU: the library's calls are recorded, not made."""
import pytest
import torch

from paper_2311_03285_amd import attention_layer, slora
from paper_2311_03285_amd.attention_layer import AttentionLayer

SIZES = dict(H=64, n_heads=8, layers=2, pool_pages=64, max_seqs=1, max_tokens=16, budget=8, recent=2, ranks={0: 8, 2: 3}, device="cpu")


class Stream:
    cuda_stream = 0x77


@pytest.fixture
def calls(monkeypatch):
    """(name, stream) of each call that is enqueued, and "wait" where the host waits for the device"""
    made = []

    def enqueued(name, at):
        def call(*args, stream=None):
            made.append((name, args[at] if len(args) > at else stream))
            return name
        return call

    for name, at in (("w4_pack", 8), ("w8_pack", 6), ("adapter_upload", 3)):
        monkeypatch.setattr(slora, name, enqueued(name, at))
    for name in ("pool_init", "kv8_init", "adapter_alloc", "norm_init"):
        monkeypatch.setattr(slora, name, lambda *args, **kw: None)
    monkeypatch.setattr(slora, "w4_bytes", lambda *args: 16)
    monkeypatch.setattr(slora, "w8_bytes", lambda *args: 16)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *args: Stream)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *args: made.append(("wait", None)))
    return made


@pytest.mark.parametrize("bits,wide,matrices", [(4, 0, 8), (8, 0, 8), (8, 96, 14)])
def test_weights_are_laid_out_behind_the_operations_that_make_them(calls, bits, wide, matrices):
    """packing and uploads are on the stream that torch is on: side streams do not wait for the default stream, nor it for them"""
    AttentionLayer(**SIZES, bits=bits, wide=wide)
    enqueued = [c for c in calls if c[0] != "wait"]
    assert [name for name, _ in enqueued] == [f"w{bits}_pack"] * matrices + ["adapter_upload"] * 2
    assert all(stream is Stream for _, stream in enqueued)
    assert calls[-1][0] == "wait"  # what a step on another stream reads is there


@pytest.mark.parametrize("kw", [dict(wide=65537), dict(wide=70000), dict(wide=131071), dict(H=32832, n_heads=8), dict(H=65536, n_heads=8)])
def test_layers_that_no_step_could_run_are_refused_when_built(calls, kw):
    """rows of the gated product and of the norms are wider than those operators take; products alone would take them, so that a step would fail midway"""
    with pytest.raises(ValueError, match="wide"):
        AttentionLayer(**{**SIZES, **kw}, bits=8)
    assert not calls


def test_the_widest_rows_are_those_that_the_operators_take():
    for width, refused in ((slora.W8_MAX_WIDTH, False), (slora.W8_MAX_WIDTH + 1, True)):
        if refused:
            with pytest.raises(slora.SloraError, match="width"):
                slora.w8_quantize(0, width, slora.F16, slora.ACT_NONE, 0, 0)
        else:
            slora.w8_quantize(0, width, slora.F16, slora.ACT_NONE, 0, 0)
    with pytest.raises(slora.SloraError, match="width"):
        slora.norm_init(slora.NORM_MAX_WIDTH + 1, slora.F16)
    with pytest.raises(slora.SloraError) as e:  # (without a GPU it is the device that is missed)
        slora.norm_apply(slora.norm_init(slora.NORM_MAX_WIDTH, slora.F16), -1, 0, 0)
    assert e.value.code in (slora.EHIP, slora.EINVAL) and "width" not in str(e.value)
