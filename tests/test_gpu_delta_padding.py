"""GPU tests of tokens of strength zero: padding whose rows hold any finite numbers is not there for the rest of the sequence.

Tolerances are those of the operator (tests/test_gpu_delta.py): fewer than 256 roundings of 2^-24, and the one to bf16 of O, dQ, dK and dV."""
import numpy as np
import pytest
import torch

import paper_2510_04008_amd as ra
from oracle import delta as oracle

pytestmark = pytest.mark.gpu

TOKENS = ("Q", "K", "V", "dO", "g", "beta")
ROUNDED = ("O", "dQ", "dK", "dV")


def _sequence(B, H, Hk, N, dk, dv, dtype, seed):
    r = np.random.RandomState(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
    x = {n: torch.from_numpy(v).to(t) for n, v in (("Q", unit(r.randn(B, Hk, N, dk))), ("K", unit(r.randn(B, Hk, N, dk))), ("V", r.randn(B, H, N, dv)),
                                                  ("dO", r.randn(B, H, N, dv)))}
    x["g"] = torch.from_numpy(-np.exp(r.uniform(-6, 0, (B, H, 1))) * r.rand(B, H, N)).float()
    x["beta"] = torch.from_numpy(0.05 + r.rand(B, H, N)).float()
    x["state"], x["dstate"] = (torch.from_numpy(r.randn(B, H, dk, dv)).float() for _ in range(2))
    return x, r


def _run(x, chunk):
    y = {n: v.cuda() for n, v in x.items()}
    (B, Hk, N, dk), (_, H, _, dv) = x["Q"].shape, x["V"].shape
    d = ra.make_delta_desc(B, H, Hk, N, dk, dv, dk**-0.5, ra.RACE_F32 if x["Q"].dtype == torch.float32 else ra.RACE_BF16, chunk)
    a = [y[n] for n in ("Q", "K", "V", "g", "beta")]
    O, out = ra.race_delta_fwd(d, *a, state_in=y["state"], want_state=True)
    grads = ra.race_delta_bwd(d, *a, y["dO"], state_in=y["state"], dstate_out=y["dstate"], want_dstate=True)
    torch.cuda.synchronize()
    got = dict(zip(("dQ", "dK", "dV", "dg", "dbeta", "dstate"), grads), O=O, state=out)
    return {n: v.double().cpu().numpy() for n, v in got.items()}


def _want(x):
    a = [x[n].double().numpy() for n in ("Q", "K", "V", "g", "beta")]
    scale, S, dS, dO = x["Q"].shape[-1]**-0.5, *(x[n].double().numpy() for n in ("state", "dstate", "dO"))
    O, out = oracle.forward(*a, scale, S)
    return dict(zip(("dQ", "dK", "dV", "dg", "dbeta", "dstate"), oracle.backward(*a, scale, dO, S, dS)), O=O, state=out)


def _near(got, want, name, dtype):
    tol = 2.0**-8 if dtype == "bf16" and name in ROUNDED else 2.0**-16
    off = np.linalg.norm(got - want) / np.linalg.norm(want)
    print("%s %.2e of %.2e" % (name, off, tol), flush=True)
    assert np.isfinite(got).all() and off <= tol, (name, off)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e10, 1e20, 3e38])
@pytest.mark.parametrize("B,H,Hk,N,dk,dv,chunk", [(2, 4, 2, 200, 64, 64, 64), (1, 2, 2, 150, 128, 128, 0), (1, 2, 1, 90, 40, 72, 0)])
def test_padding_rows_of_any_size(B, H, Hk, N, dk, dv, chunk, size, dtype):
    """Between the tokens, a whole chunk of them, and behind the last.  Keys whose squares leave fp32 among them; queries stay within 1e20, so that their products with
    keys and states do not leave it."""
    x, r = _sequence(B, H, Hk, N, dk, dv, dtype, seed=N)
    places = np.sort(r.choice(N + 200, N + 100, replace=False))
    places[places >= 70] += 64                          # nobody in 70 .. 133
    places = np.delete(places, slice(N, None))
    total = N + 300
    y = {n: x[n] for n in ("state", "dstate")}
    for n in TOKENS:
        shape = list(x[n].shape)
        shape[2] = total
        fill = np.zeros(shape)
        if n in ("Q", "K", "V"):
            fill = r.uniform(-1, 1, shape) * (min(size, 1e20) if n == "Q" else size)
        y[n] = torch.from_numpy(fill).to(x[n].dtype)
        y[n][:, :, places] = x[n]
    got, want = _run(y, chunk), _want(x)
    idle = np.setdiff1d(np.arange(total), places)
    assert not got["dK"][:, :, idle].any() and not got["dV"][:, :, idle].any() and not got["dQ"][:, :, idle].any()
    for n in want:
        _near(got[n] if "state" in n else got[n][:, :, places], want[n], n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", [(128, 128), (64, 64), (24, 16)])
@pytest.mark.parametrize("strength", [0.0, -0.0, 1e-38, 2.0**-101])
def test_gradient_of_a_strength_of_zero(dk, dv, strength, dtype):
    """Reading tokens that write nothing: their own gradients, with decays and cotangents of their own."""
    x, r = _sequence(2, 2, 1, 170, dk, dv, dtype, seed=dk)
    idle = r.rand(2, 2, 170) < 0.3
    x["beta"][torch.from_numpy(idle)] = strength
    x["beta"][1, 1] = strength                          # a head that never writes
    idle[1, 1] = True
    got, want = _run(x, 64), _want(x)
    for n in want:
        _near(got[n], want[n], n, dtype)
    _near(got["dbeta"][idle], want["dbeta"][idle], "dbeta of idle tokens", dtype)
    assert not got["dV"][idle].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1.0, 1e20, 3e38])
def test_a_step_of_padding_leaves_the_state(size, dtype):
    B, H, Hk, dk, dv = 3, 4, 2, 40, 72
    r = np.random.RandomState(0)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, v = (torch.from_numpy(r.uniform(-1, 1, s) * m).to(t).cuda() for s, m in (((B, Hk, dk), 1.0), ((B, Hk, dk), size), ((B, H, dv), size)))
    state = torch.from_numpy(r.randn(B, H, dk, dv)).float().cuda()
    zero, before = torch.zeros((B, H), device="cuda"), state.clone()
    d = ra.make_delta_desc(B, H, Hk, 1, dk, dv, 1.0, ra.RACE_F32 if dtype == "f32" else ra.RACE_BF16)
    o = ra.race_delta_step(d, q, k, v, zero, zero, state)
    assert torch.equal(state, before)
    want = (before.double() * q.double().repeat_interleave(H // Hk, 1)[..., None]).sum(-2)
    # one rounding to the element type, and 40 of fp32
    assert ((o.double() - want).abs() <= 2.0**-8 * want.abs() + 2.0**-18 * want.abs().max()).all()
