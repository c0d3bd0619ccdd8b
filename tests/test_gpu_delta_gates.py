"""GPU tests of the gates' gradient where decays are strong: dg of a token is of the size of its decay, and keeps its digits head by head.

Tolerance: 2^-16, that of the operator's fp32 outputs (tests/test_gpu_delta.py): fewer than 256 roundings of 2^-24.  A decay of e^-20 is off by the rounding of its
exponent, 29 * 2^-24, within that."""
import numpy as np
import pytest
import torch

import paper_2510_04008_amd as ra
from oracle import delta as oracle

pytestmark = pytest.mark.gpu

TOL = 2.0**-16
MEANS = (-0.05, -1.0, -3.0, -5.0, -8.0, -12.0, -20.0)


def _inputs(H, Hk, N, dk, dv, dtype, seed):
    r = np.random.RandomState(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
    x = {"Q": unit(r.randn(1, Hk, N, dk)), "K": unit(r.randn(1, Hk, N, dk)), "V": r.randn(1, H, N, dv), "dO": r.randn(1, H, N, dv)}
    x = {n: torch.from_numpy(v).to(t) for n, v in x.items()}
    x["beta"] = torch.from_numpy(0.05 + 0.95 * r.rand(1, H, N)).float()
    x["state"], x["dstate"] = (torch.from_numpy(r.randn(1, H, dk, dv)).float() for _ in range(2))
    return x, r


def _dg(x, chunk=0):
    y = {n: v.cuda() for n, v in x.items()}
    (_, Hk, N, dk), (_, H, _, dv) = x["Q"].shape, x["V"].shape
    d = ra.make_delta_desc(1, H, Hk, N, dk, dv, dk**-0.5, ra.RACE_F32 if x["Q"].dtype == torch.float32 else ra.RACE_BF16, chunk)
    grads = ra.race_delta_bwd(d, *(y[n] for n in ("Q", "K", "V", "g", "beta")), y["dO"], state_in=y["state"], dstate_out=y["dstate"])
    a = [x[n].double().numpy() for n in ("Q", "K", "V", "g", "beta")]
    want = oracle.backward(*a, dk**-0.5, *(x[n].double().numpy() for n in ("dO", "state", "dstate")))[3]
    return grads[3].double().cpu().numpy()[0], want[0]


def _near(got, want, label):
    off = np.linalg.norm(got - want) / np.linalg.norm(want)
    print("%s: %.2e" % (label, off), flush=True)
    assert off <= TOL, (label, off)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,dk,dv,Hk,chunk", [(256, 128, 128, 7, 0), (200, 64, 64, 1, 64), (77, 24, 40, 7, 0), (2, 8, 8, 7, 0)])
def test_every_head_has_its_own_decay(N, dk, dv, Hk, chunk, dtype):
    H = len(MEANS)
    x, r = _inputs(H, Hk, N, dk, dv, dtype, seed=N)
    x["g"] = torch.from_numpy(np.array(MEANS)[None, :, None] * r.uniform(0.8, 1.2, (1, H, N))).float()
    got, want = _dg(x, chunk)
    for h in range(H):
        _near(got[h], want[h], "mean gate %g" % MEANS[h])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", [(128, 128), (64, 64)])
def test_strong_decays_among_slow_ones(dk, dv, dtype):
    """Single tokens of strong decay, whose dg is a small part of its head's norm, and resets, whose dg is nothing."""
    H, N = 4, 300
    x, r = _inputs(H, 2, N, dk, dv, dtype, seed=dk)
    g = -0.05 * r.rand(1, H, N)
    kinds = r.choice(4, (1, H, N), p=(0.7, 0.1, 0.1, 0.1))
    kinds[:, 3][kinds[:, 3] == 3] = 0       # one head without resets: what is behind them does not depend on what is before
    g[kinds == 1], g[kinds == 2], g[kinds == 3] = -8.0, -16.0, -np.inf
    x["g"] = torch.from_numpy(g).float()
    got, want = _dg(x, 64)
    for h in range(H):
        for kind, name in ((0, "slow"), (1, "e^-8"), (2, "e^-16")):
            at = kinds[0, h] == kind
            _near(got[h][at], want[h][at], "head %d, %s" % (h, name))
    assert not got[kinds[0] == 3].any()
