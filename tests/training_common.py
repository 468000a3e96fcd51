"""What the GPU tests of the training side share."""
import numpy as np
import torch

from oracle import fp_formats as ff

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_ULP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # of a value rounded to the type (8 and 24 significant bits), relative
F32 = 2.0 ** -24


def keep(type):
    """v as an array of the type holds it, coming from an fp32 result"""
    if type == "f32":
        return lambda v: v.astype(np.float32).astype(np.float64)
    return lambda v: ff.bf16_bits_to_f64(ff.f64_to_bf16_bits(v.astype(np.float32).astype(np.float64)))


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def randn(shape, type, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(TYPES[type])


def guarded(shape, dtype, fill=37.0):
    """A tensor of `shape` inside a larger allocation, and a check that nothing around it was written."""
    n = int(np.prod(shape))
    pad = 1024
    whole = torch.full((n + 2 * pad,), 0, dtype=dtype, device="cuda").fill_(fill)
    inner = whole[pad:pad + n].view(shape)
    mark = torch.full((pad,), 0, dtype=dtype, device="cuda").fill_(fill)

    def check():
        assert torch.equal(whole[:pad], mark) and torch.equal(whole[pad + n:], mark), "written outside the tensor"
    return inner, check


class Context:
    """A context with the gradients' workspace."""

    def __init__(self, moe, T=0, d=128, E=1, k=1, reserve=True):
        self.moe = moe
        self.ctx = moe.moe_create(T, d, E, k, 128)
        if reserve:
            moe.moe_reserve_gradients(self.ctx)

    def __enter__(self):
        return self.ctx

    def __exit__(self, *_):
        torch.cuda.synchronize()
        self.moe.moe_destroy(self.ctx)
