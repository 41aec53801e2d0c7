"""spconv_attention at the ends of what it accepts: caps, strides, rows outside of the call's
documents, values and lengths far from the ordinary."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV, say
from tests.test_gpu_attention import Batch, ints

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", [1e-40, 1e-3, 0.5, 64.0, 65.0, 200.0, 1e3, 1e4, 1e6, 1e12, 1e30])
def test_caps_of_all_sizes(cap, dtype):
    """A cap far above the scores leaves them as they are: its error must not grow with the cap."""
    say(f"attention with a cap of {cap} {dtype}")
    for ql, kl, d in (([150, 40], [150, 333], 64), ([1, 3], [700, 90], 128), ([130], [200], 256)):
        for spread in (1.0, 12.0, 100.0):
            b = Batch(ql, kl, 4, 2, d, dtype, spread=spread, seed=21)
            for bias in ("none", "position", "voxel"):
                got = b.run(causal=True, cap=cap, bias=bias)
                want, mag = ref.attention(b.q, b.k, b.v, b.q_lens, b.k_lens, causal=True, cap=cap, **b.bias(bias))
                u = ref.UNIT[dtype]  # float32 errors of the scores grow with them, and end at the cap
                bound = mag * (2 * u + 4e-5 * max(1.0, min(spread, cap))) + want.abs() * u + ref.TINY[dtype]
                off = (got.double() - want).abs()
                assert bool((off <= bound).all()), f"{bias}, scores of {spread}: {float((off / bound).max()):.2f} of the bound"
