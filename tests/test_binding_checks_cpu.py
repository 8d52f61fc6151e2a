"""What the binding looks at before it hands pointers on: no tensor that a kernel would read or write beyond."""
import math

import torch

from paper_2605_12471_b200 import binding


class OnGpu:
    """As much of a CUDA tensor as the checks look at."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=0, contiguous=True):
        self.shape, self.dtype, self.device, self.contiguous = shape, dtype, device, contiguous

    def numel(self):
        return math.prod(self.shape)

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.contiguous


def test_tensors_of_a_scored_call():
    cfg = binding.make_config(8, 2, 128, "bf16", 100, 10)
    bf, f32 = torch.bfloat16, torch.float32
    q, k = OnGpu(5, 8, 128), OnGpu(5, 2, 128)

    def fits(q=q, k=k, v=k, out=None, lse=None, out_dtype=bf):
        return binding._fits(cfg, 5, bf, out_dtype, q, k, v, out, lse)

    assert fits() and fits(k=None, v=None) and fits(out=OnGpu(5, 8, 128), lse=OnGpu(5, 8, dtype=f32))
    assert fits(out=OnGpu(10, 8, 128)) and fits(lse=OnGpu(80, dtype=f32)) and fits(q=OnGpu(5, 1024))          # room to spare, other shapes
    assert fits(out=OnGpu(5, 8, 128, dtype=f32), out_dtype=f32)
    for bad in (OnGpu(5, 4, 128), OnGpu(5, 8, 64), OnGpu(4, 8, 128), OnGpu(6, 8, 128), OnGpu(5, 8, 128, dtype=f32), OnGpu(5, 8, 128, device=-1),
                OnGpu(5, 8, 128, contiguous=False)):
        assert not fits(q=bad)
    for bad in (OnGpu(5, 1, 128), OnGpu(4, 2, 128), OnGpu(5, 2, 128, dtype=f32), OnGpu(5, 2, 128, device=1), OnGpu(5, 2, 128, contiguous=False)):
        assert not fits(k=bad) and not fits(v=bad)
    for bad in (OnGpu(5, 4, 128), OnGpu(5, 8, 128, dtype=f32), OnGpu(5, 8, 128, device=-1), OnGpu(5, 8, 128, contiguous=False)):
        assert not fits(out=bad)
    for bad in (OnGpu(4, 8, dtype=f32), OnGpu(5, 8), OnGpu(5, 8, dtype=f32, device=1), OnGpu(5, 8, dtype=f32, contiguous=False)):
        assert not fits(lse=bad)
