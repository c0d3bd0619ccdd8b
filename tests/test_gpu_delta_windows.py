"""GPU tests of the gated delta rule over windows of its workspace and over tensors beyond 2^31 elements, against the fp64 recurrence of some of the heads (heads do not
meet).  Tolerances as in tests/test_gpu_delta.py."""
import numpy as np
import pytest
import torch

import paper_2510_04008_amd as ra
from oracle import delta as oracle

pytestmark = pytest.mark.gpu

ROUNDED = ("O", "dQ", "dK", "dV")


def _near(got, want, name):
    got = got.double().cpu().numpy()
    tol = 2.0**-8 if name in ROUNDED else 2.0**-16
    off = np.linalg.norm(got - want) / np.linalg.norm(want)
    print("%s %.2e of %.2e" % (name, off, tol), flush=True)
    assert np.isfinite(got).all() and off <= tol, (name, off)


def _inputs(B, H, N, dk, dv, gate, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    x = {"Q": torch.nn.functional.normalize(rand(B, H, N, dk), dim=-1), "K": torch.nn.functional.normalize(rand(B, H, N, dk), dim=-1), "V": rand(B, H, N, dv),
         "dO": rand(B, H, N, dv)}
    x["g"], x["beta"] = -gate * torch.rand((B, H, N), generator=gen, device="cuda"), torch.rand((B, H, N), generator=gen, device="cuda")
    x["state"], x["dstate"] = (torch.randn((B, H, dk, dv), generator=gen, device="cuda") for _ in range(2))
    return x


def _host(x, b, h, tokens=slice(None)):
    cut = lambda v: v[b:b + 1, h:h + 1, tokens].double().cpu().numpy()  # noqa: E731
    return {n: cut(v) if n not in ("state", "dstate") else v[b:b + 1, h:h + 1].double().cpu().numpy() for n, v in x.items()}


@pytest.mark.parametrize("B,H,N,chunk,heads", [
    (8, 128, 64 * 100 + 5, 256, ((0, 0), (3, 77), (7, 127))),       # windows of ten segments, the last of five
    (8, 128, 64 * 90, 0, ((0, 0), (7, 127))),                       # one segment a window
    (1, 128, 64 * 420 - 7, 0, ((0, 0), (0, 127)))])                 # windows of two segments
def test_windows_against_the_recurrence(B, H, N, chunk, heads):
    dk = 8
    x = _inputs(B, H, N, dk, dk, 0.05, seed=N)
    d = ra.make_delta_desc(B, H, H, N, dk, dk, 0.3, ra.RACE_BF16, chunk)
    half = ra.make_delta_desc(B, H, H, N // 2, dk, dk, 0.3, ra.RACE_BF16, chunk)
    assert ra.race_delta_bwd_workspace_bytes(d) < 1.6 * ra.race_delta_bwd_workspace_bytes(half)       # more than one window
    a = [x[n] for n in ("Q", "K", "V", "g", "beta")]
    O, out = ra.race_delta_fwd(d, *a, state_in=x["state"], want_state=True)
    grads = ra.race_delta_bwd(d, *a, x["dO"], state_in=x["state"], dstate_out=x["dstate"], want_dstate=True)
    got = dict(zip(("dQ", "dK", "dV", "dg", "dbeta", "dstate"), grads), O=O, state=out)
    for b, h in heads:
        y = _host(x, b, h)
        a = [y[n] for n in ("Q", "K", "V", "g", "beta")]
        want = dict(zip(("dQ", "dK", "dV", "dg", "dbeta", "dstate"), oracle.backward(*a, 0.3, y["dO"], y["state"], y["dstate"])))
        want["O"], want["state"] = oracle.forward(*a, 0.3, y["state"])
        for n, w in want.items():
            _near(got[n][b:b + 1, h:h + 1], w, n)


def test_backward_beyond_two_to_the_31_elements():
    """Gates of up to -0.5 a token: 600 tokens away nothing is left (e^-150) of a state or of its cotangent."""
    H, N, dk, dv, part = 64, 262144 + 17, 64, 128, 200
    x = _inputs(1, H, N, dk, dv, 0.5, seed=0)
    assert x["V"].numel() > 1 << 31 and x["Q"].numel() * 2 > 1 << 31
    d = ra.make_delta_desc(1, H, H, N, dk, dv, 0.125, ra.RACE_BF16)
    grads = ra.race_delta_bwd(d, *(x[n] for n in ("Q", "K", "V", "g", "beta")), x["dO"], state_in=x["state"], dstate_out=x["dstate"], want_dstate=True)
    names = ("dQ", "dK", "dV", "dg", "dbeta")
    for h in (0, H - 1):
        for tokens, mine, first in ((slice(0, 800), slice(0, part), True), (slice(N - 800, N), slice(800 - part, 800), False)):
            y = _host(x, 0, h, tokens)
            want = oracle.backward(*(y[n] for n in ("Q", "K", "V", "g", "beta")), 0.125, y["dO"], y["state"] if first else None, None if first else y["dstate"])
            for n, got, w in zip(names, grads, want):
                _near(got[:, h:h + 1, tokens][:, :, mine], w[:, :, mine], n)
            if first:
                _near(grads[5][:, h:h + 1], want[5], "dstate")


def test_images_of_the_way_back_are_formed_once():
    """A window's M^T, T^T and A^T: by the launch that its gradients read, not by the one before for its states alone."""
    B, H, N, dk = 8, 128, 64 * 100 + 5, 8
    x = _inputs(B, H, N, dk, dk, 0.05, seed=1)
    d = ra.make_delta_desc(B, H, H, N, dk, dk, 0.3, ra.RACE_BF16, 256)
    ra.race_attn_profile_enable(True)
    ra.race_delta_bwd(d, *(x[n] for n in ("Q", "K", "V", "g", "beta")), x["dO"], state_in=x["state"])
    torch.cuda.synchronize()
    launches = {n: count for n, (_, count) in ra.race_attn_profile_read().items()}
    ra.race_attn_profile_enable(False)
    windows = launches["delta_scan_back"]
    assert windows > 2 and launches["delta_prep_back"] == windows and launches["delta_prep"] == windows - 1
