"""GPU tests of the operators at the far end of what their descriptors allow."""
import numpy as np
import pytest
import torch

import paper_2510_04008_amd as ra
from oracle import rotary

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,d,rot", [((1 << 26) + 5, 72, 4), ((1 << 29) + 5, 16, 2)])
def test_rotary_forward_of_more_tokens_than_one_grid(N, d, rot):
    """A thread per element and token would be more than a grid's 2^32 threads.  The rows as given repeat (a stride of zero), the positions do not."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    row = torch.randn((1, 1, 1, d), generator=gen, device="cuda").bfloat16()
    w = 1 + 0.3 * torch.randn(d, generator=gen, device="cuda")
    desc = ra.make_rotary_desc(1, N, 1, 0, d, rot, ra.RACE_BF16, pos0=7)
    freq = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
    Q, _ = ra.race_qk_rotary_fwd(desc, row.expand(1, N, 1, d), None, w, None, freq)
    for at in (0, (1 << 24) - 3, (1 << 26) - 60, N - 40):
        places = np.arange(at, at + 40)[None] + 7
        x = row.double().cpu().numpy().repeat(40, 1)
        want = rotary.forward(x, w.double().cpu().numpy(), places, freq, rot, "rms", np.float64(np.float32(1e-6)), False)
        got = Q[:, :, at:at + 40].double().cpu().numpy()
        # one rounding to bf16, and a dozen of fp32
        assert (np.abs(got - want) <= 2.0**-8 * np.abs(want) + 2.0**-20 * np.abs(want).max()).all(), at
