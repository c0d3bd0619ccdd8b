"""GPU tests of the segments' join, one after the other and in groups, at the lengths where the one takes over from the other, against the fp64 recurrence.
Tolerances as in tests/test_gpu_delta.py."""
import numpy as np
import pytest
import torch

import paper_2510_04008_amd as ra
from oracle import delta as oracle

pytestmark = pytest.mark.gpu

ROUNDED = ("O", "dQ", "dK", "dV")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,segments,dk,dv", [(2, 24, 16, 16), (2, 25, 72, 24), (2, 26, 16, 16), (1, 50, 128, 128), (8, 32, 16, 40), (8, 33, 16, 16), (10, 51, 8, 8), (17, 60, 8, 8)])
def test_segments_of_one_chunk(H, segments, dk, dv, dtype):
    N = 64 * segments - 5
    r = np.random.RandomState(segments)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
    x = {"Q": unit(r.randn(1, H, N, dk)), "K": unit(r.randn(1, H, N, dk)), "V": r.randn(1, H, N, dv), "dO": r.randn(1, H, N, dv)}
    x = {n: torch.from_numpy(v).to(t) for n, v in x.items()}
    # decays of a few hundred tokens: states and cotangents cross several segments
    x["g"], x["beta"] = torch.from_numpy(-0.01 * r.rand(1, H, N)).float(), torch.from_numpy(r.rand(1, H, N)).float()
    x["state"], x["dstate"] = (torch.from_numpy(r.randn(1, H, dk, dv)).float() for _ in range(2))
    y = {n: v.cuda() for n, v in x.items()}
    d = ra.make_delta_desc(1, H, H, N, dk, dv, dk**-0.5, ra.RACE_F32 if dtype == "f32" else ra.RACE_BF16, 64)
    a = [y[n] for n in ("Q", "K", "V", "g", "beta")]
    O, out = ra.race_delta_fwd(d, *a, state_in=y["state"], want_state=True)
    grads = ra.race_delta_bwd(d, *a, y["dO"], state_in=y["state"], dstate_out=y["dstate"], want_dstate=True)
    names = ("dQ", "dK", "dV", "dg", "dbeta", "dstate")
    got = dict(zip(names, grads), O=O, state=out)
    h = [x[n].double().numpy() for n in ("Q", "K", "V", "g", "beta")]
    S, dS, dO = (x[n].double().numpy() for n in ("state", "dstate", "dO"))
    want = dict(zip(names, oracle.backward(*h, dk**-0.5, dO, S, dS)))
    want["O"], want["state"] = oracle.forward(*h, dk**-0.5, S)
    for n, w in want.items():
        tol = 2.0**-8 if dtype == "bf16" and n in ROUNDED else 2.0**-16
        off = np.linalg.norm(got[n].double().cpu().numpy() - w) / np.linalg.norm(w)
        print("%s %.2e of %.2e" % (n, off, tol), flush=True)
        assert off <= tol, (n, off)
