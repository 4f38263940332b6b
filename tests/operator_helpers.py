"""Contexts without a model for the tests of cache reordering, shared-prefix attention and token log probabilities."""
import torch

from paper_2403_18647_amd import binding as B
from paper_2403_18647_amd import synth


def context(heads=2, head_dim=64, dtype="fp32", layers=1, batch=1, slots=64, q=1, vocab=64):
    """A context of zero weights (these calls read none)."""
    sh = synth.small_shape(n_layers=layers, d_model=heads * head_dim, n_heads=heads, head_dim=head_dim, d_ffn=64,
                           vocab=vocab, n_adaptive=0, dtype=dtype)
    w = [torch.zeros(synth.tensor_shape(sh, n), device="cuda",
                     dtype=torch.float32 if synth.is_gain(n) or dtype == "fp32" else torch.bfloat16)
         for n in synth.tensor_names(sh)]
    return B.Context(B.make_config(sh, batch, slots, q), w)


def device_error(ctx):
    """The device's error flags, as the next synchronous call reports them (no token is generated): its code or 0."""
    import numpy as np
    torch.cuda.synchronize()
    try:
        B.sdsat_generate(ctx.handle, np.zeros((1, 1), np.int32), 0, 0, [])
    except B.SdsatError as e:
        return e.code
    return 0
