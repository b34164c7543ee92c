"""Helpers of the tests of training the refiner's last layer: tensors inside
canary-filled buffers, and the roundings that the tolerances count."""
from __future__ import annotations

import numpy as np
import torch

U32 = 2.0 ** -24                                         # half a step of fp32, relative
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}   # half a step of the type, relative
CANARY = 0x5A


def dev():
    return torch.device("cuda", 0)


def host(t):
    """fp64 copy of a tensor's values."""
    return t.detach().float().cpu().numpy().astype(np.float64)


class Guarded:
    """Output tensors as views in buffers filled with a canary; check() says whether
    a byte outside a view has changed."""

    def __init__(self):
        self.held = []

    def empty(self, *shape, dtype=torch.float32, offset=0, row=None):
        """A tensor of `shape` whose rows are `row` elements apart (default: dense),
        starting `offset` elements into its buffer (which is 16-byte aligned)."""
        esz = torch.empty(0, dtype=dtype).element_size()
        row = shape[-1] if row is None else row
        rows = int(np.prod(shape[:-1])) if len(shape) > 1 else 1
        lead = 1024 // esz + offset
        n = lead + rows * row + 1024 // esz
        raw = torch.full((n * esz,), CANARY, dtype=torch.uint8, device=dev())
        strides = [1]
        for k in range(len(shape) - 1, 0, -1):
            strides.insert(0, row if len(strides) == 1 else strides[0] * shape[k])
        view = raw.view(dtype).as_strided(shape, strides, lead)
        inside = torch.zeros(n, dtype=torch.bool, device=dev())
        inside.as_strided(shape, strides, lead).fill_(True)
        self.held.append((raw, inside, esz))
        return view

    def like(self, t, offset=0, row=None):
        v = self.empty(*t.shape, dtype=t.dtype, offset=offset, row=row)
        v.copy_(t)
        return v

    def check(self):
        torch.cuda.synchronize()
        for raw, inside, esz in self.held:
            outside = raw.view(-1, esz)[~inside]
            assert bool((outside == CANARY).all()), "a byte outside a tensor changed"


def within(got, want, bound, where=""):
    """|got - want| <= bound, element by element (NaN and infinities in the same places)."""
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    bound = np.broadcast_to(np.asarray(bound, dtype=np.float64), want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{where}: NaN in other places"
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), f"{where}: infinities differ"
    over = np.abs(got - want)[fine] - bound[fine]
    assert over.size == 0 or over.max() <= 0, \
        f"{where}: off by up to {np.abs(got - want)[fine].max():.3g}, {over.max():.3g} over the bound"
