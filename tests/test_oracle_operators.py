"""The fp64 oracles of the gated delta rule and of the rotated rows: gradients against differences of the forward pass, and
what the definitions say of special inputs."""
import numpy as np
import pytest

from oracle import delta, rotary


def _delta_inputs(seed, B=1, H=4, Hk=2, N=7, dk=8, dv=16):
    r = np.random.RandomState(seed)
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
    return dict(Q=unit(r.randn(B, Hk, N, dk)), K=unit(r.randn(B, Hk, N, dk)), V=r.randn(B, H, N, dv), g=-r.rand(B, H, N), beta=r.rand(B, H, N),
                state=r.randn(B, H, dk, dv)), r


def test_delta_gradients_against_differences():
    x, r = _delta_inputs(0)
    dO, dS = r.randn(*x["V"].shape), r.randn(*x["state"].shape)
    loss = lambda x: sum((a * b).sum() for a, b in zip(delta.forward(x["Q"], x["K"], x["V"], x["g"], x["beta"], 0.3, x["state"]), (dO, dS)))  # noqa: E731
    got = delta.backward(x["Q"], x["K"], x["V"], x["g"], x["beta"], 0.3, dO, x["state"], dS)
    for name, grad in zip(("Q", "K", "V", "g", "beta", "state"), got):
        for _ in range(6):
            at = tuple(r.randint(0, n) for n in x[name].shape)
            h, both = 1e-6, []
            for sign in (1, -1):
                y = {n: v.copy() for n, v in x.items()}
                y[name][at] += sign * h
                both.append(loss(y))
            assert abs((both[0] - both[1]) / (2 * h) - grad[at]) < 1e-7 * max(1, abs(grad[at])), (name, at)


def test_delta_special_tokens():
    x, _ = _delta_inputs(1)
    O, S = delta.forward(x["Q"], x["K"], x["V"], x["g"], x["beta"], 1.0, x["state"])
    # a padding token leaves the state alone, a decay of zero empties it, strength one writes its value exactly
    x["g"][..., -1] = 0.0
    x["beta"][..., -1] = 0.0
    before = delta.forward(*(x[n][:, :, :-1] for n in ("Q", "K", "V", "g", "beta")), 1.0, x["state"])[1]
    assert np.allclose(delta.forward(x["Q"], x["K"], x["V"], x["g"], x["beta"], 1.0, x["state"])[1], before)
    x["g"][..., -1] = -np.inf
    x["beta"][..., -1] = 1.0
    k, v = np.repeat(x["K"], 2, 1)[:, :, -1], x["V"][:, :, -1]
    assert np.allclose(delta.forward(x["Q"], x["K"], x["V"], x["g"], x["beta"], 1.0, x["state"])[1], k[..., None] * v[..., None, :])


@pytest.mark.parametrize("norm", ["rms", "l2", "none"])
@pytest.mark.parametrize("neighbours", [False, True])
def test_rotary_gradients_against_differences(norm, neighbours):
    r = np.random.RandomState(3)
    x, w, pos, freq = r.randn(2, 3, 2, 16), 1 + 0.1 * r.randn(16), r.randint(0, 1000, (2, 3)), r.rand(5)
    dy = r.randn(2, 2, 3, 16)
    args = (pos, freq, 10, norm, 1e-2, neighbours)
    dx, dw = rotary.backward(x, w, *args, dy)
    for name, arr, grad in (("x", x, dx), ("w", w, dw)):
        for _ in range(8):
            at = tuple(r.randint(0, n) for n in arr.shape)
            both = []
            for sign in (1, -1):
                y = arr.copy()
                y[at] += sign * 1e-6
                both.append((rotary.forward(y if name == "x" else x, y if name == "w" else w, *args) * dy).sum())
            assert abs((both[0] - both[1]) / 2e-6 - grad[at]) < 1e-7 * max(1, abs(grad[at]))


def test_rotary_depends_on_the_distance_alone():
    r = np.random.RandomState(4)
    q, k, freq = r.randn(1, 1, 1, 32), r.randn(1, 1, 1, 32), 10000.0 ** (-np.arange(16) / 16)
    dot = lambda m, n: (rotary.forward(q, None, [[m]], freq, 32, "rms", 0.0, False) * rotary.forward(k, None, [[n]], freq, 32, "rms", 0.0, False)).sum()  # noqa: E731
    assert abs(dot(5, 3) - dot(1005, 1003)) < 1e-9
    assert abs(np.linalg.norm(rotary.forward(q, None, [[77]], freq, 32, "l2", 0.0, True)) - 1) < 1e-12
