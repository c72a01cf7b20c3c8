"""What the denoiser block refuses before any device call: these run without a device."""
import types

import pytest
import torch

from paper_2604_10103_b200 import binding as hf, block as bl, inputs as gen

HIGH, WIDE = 4, 8
W = gen.Workload("refusals", batch=2, heads=2, head_dim=64, tokens_per_frame=HIGH * WIDE, chunk_frames=2, window_frames=4, block=16, topk=2, keep_permille=0)


def build(w=W, **kw):
    context = types.SimpleNamespace(cfg=hf.make_config(W, merge=hf.HF_MERGE_IDENTITY), device=0)
    return bl.DenoiserBlock(w, HIGH, WIDE, context, device="cpu", **kw)


def chunk(dtype=torch.bfloat16, batch=W.batch, tokens=W.chunk_tokens, width=128, frames=W.chunk_frames):
    return torch.zeros(batch, tokens, width, dtype=dtype), torch.zeros(batch, frames, 6, width, dtype=dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_types_that_the_attention_does_not_take(dtype):
    """The attention reads bfloat16 through bare pointers."""
    with pytest.raises(ValueError, match="bfloat16"):
        build(dtype=dtype)
    b = build()
    x, mod = chunk(dtype)
    for call in (b.forward, b.commit):
        with pytest.raises(ValueError, match="bfloat16"):
            call(x, mod, b.positions(0))


@pytest.mark.parametrize("kw", [dict(batch=1), dict(batch=3), dict(tokens=W.chunk_tokens - 32), dict(tokens=W.chunk_tokens + 32), dict(tokens=1), dict(width=64),
                                dict(width=192)])
def test_chunks_of_other_sizes_than_the_context(kw):
    """The attention reads and writes batch x heads x tokens of its context, whatever lies behind the pointers."""
    b = build()
    x, mod = chunk(**{k: v for k, v in kw.items() if k != "tokens"}, tokens=kw.get("tokens", W.chunk_tokens))
    for call in (b.forward, b.commit):
        with pytest.raises(ValueError, match=r"x is \[.*\]: \[2, 64, 128\] is taken"):
            call(x, mod, b.positions(0))
    for bad in (x[0], x[None]):
        with pytest.raises(ValueError, match="is taken"):
            b(bad, mod, b.positions(0))


@pytest.mark.parametrize("kw", [dict(batch=1), dict(heads=3), dict(heads=1, head_dim=128), dict(tokens_per_frame=2 * HIGH * WIDE), dict(chunk_frames=4)])
def test_a_context_of_another_workload(kw):
    context = types.SimpleNamespace(cfg=hf.make_config(W.with_(**kw)), device=0)
    with pytest.raises(ValueError, match="context"):
        bl.DenoiserBlock(W, HIGH, WIDE, context, device="cpu")


def test_tensors_on_another_device_than_the_context():
    b = build()
    x, mod = chunk()
    with pytest.raises(ValueError, match="x is on cpu"):
        b(x, mod, b.positions(0))


def test_frames_outside_the_time_table():
    """On the device a position outside its table is taken as 0; where the frame is a Python number it is refused."""
    b = build(last_frame=20)
    assert b.positions(0)[:, 0].max() == 1 and b.positions(19)[:, 0].max() == 20
    for first in (-1, 20, 21, 255, 2 ** 40):
        with pytest.raises(ValueError, match="last_frame"):
            b.positions(first)
    assert build(last_frame=70000).positions(69999)[:, 0].max() == 70000
