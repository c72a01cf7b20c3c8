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
