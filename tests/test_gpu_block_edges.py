"""The denoiser block where it can go wrong without an error: types, selections made in between, chunks that follow one another."""
import pytest
import torch

pytestmark = pytest.mark.gpu
HIGH, WIDE = 8, 12


def build(keep=500, batch=1, window=2, **kw):
    from paper_2604_10103_b200 import binding as hf, block as bl, inputs as gen
    w = gen.Workload("edges", batch=batch, heads=3, head_dim=64, tokens_per_frame=HIGH * WIDE, chunk_frames=4, window_frames=4 * window,
                     block=128, topk=0, keep_permille=keep, seed=3)
    ctx = hf.Context(hf.make_config(w, merge=hf.HF_MERGE_IDENTITY))
    torch.manual_seed(5)
    return w, ctx, bl.DenoiserBlock(w, HIGH, WIDE, ctx, **kw)


def chunk(w, seed):
    g = torch.Generator().manual_seed(seed)
    width = w.heads * w.head_dim
    return (torch.randn(w.batch, w.chunk_tokens, width, generator=g).bfloat16().cuda(),
            (0.3 * torch.randn(w.batch, w.chunk_frames, 6, width, generator=g)).bfloat16().cuda())


def test_autocast_to_another_type_is_refused():
    w, ctx, b = build()
    x, mod = chunk(w, 1)
    ref = b(x, mod, b.positions(0))
    for call in (b.forward, b.commit):
        with torch.autocast("cuda", dtype=torch.float16), pytest.raises(ValueError, match="projection is torch.float16"):
            call(x, mod, b.positions(0))
    with torch.autocast("cuda", dtype=torch.bfloat16):
        assert torch.equal(b(x, mod, b.positions(0)), ref)
