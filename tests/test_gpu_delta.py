"""GPU tests of the gated delta rule against the fp64 recurrence.

Tolerances count roundings.  Sums, states and decays are fp32 or better in both types: products summed over at most 128 elements and 64 tokens, fewer than 256
roundings of 2^-24 one after another.  O, dQ, dK and dV of the bf16 type are rounded to it once, at the end: half a step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

import paper_2510_04008_amd as ra
from oracle import delta as oracle

pytestmark = pytest.mark.gpu

F32 = {n: 2.0**-16 for n in ("O", "dQ", "dK", "dV", "state", "dg", "dbeta", "dstate")}
BF16 = dict(F32, **{n: 2.0**-8 for n in ("O", "dQ", "dK", "dV")})
TOL = {"bf16": BF16, "f32": F32}


def _inputs(B, H, Hk, N, dk, dv, dtype, seed=0, gates="usual"):
    r = np.random.RandomState(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
    x = {"Q": unit(r.randn(B, Hk, N, dk)), "K": unit(r.randn(B, Hk, N, dk)), "V": r.randn(B, H, N, dv), "dO": r.randn(B, H, N, dv)}
    x = {n: torch.from_numpy(v).to(t) for n, v in x.items()}
    g = -np.exp(r.uniform(-6, 0.5, (B, H, 1))) * r.rand(B, H, N)
    beta = r.rand(B, H, N)
    if gates == "hard":         # resets, gates of nothing, padding, strengths of nothing and beyond one
        g[r.rand(B, H, N) < 0.05] = -np.inf
        g[r.rand(B, H, N) < 0.1] = 0.0
        g[r.rand(B, H, N) < 0.05] = -30.0
        beta[r.rand(B, H, N) < 0.2] = 0.0
        beta[r.rand(B, H, N) < 0.1] = 1.9
        pad = r.rand(B, H, N) < 0.1
        g[pad], beta[pad] = 0.0, 0.0
    x["g"], x["beta"] = (torch.from_numpy(v).float() for v in (g, beta))
    x["state"], x["dstate"] = (torch.from_numpy(r.randn(B, H, dk, dv)).float() for _ in range(2))
    return x


def _desc(x, chunk=0):
    (B, Hk, N, dk), (_, H, _, dv) = x["Q"].shape, x["V"].shape
    return ra.make_delta_desc(B, H, Hk, N, dk, dv, dk**-0.5, ra.RACE_F32 if x["Q"].dtype == torch.float32 else ra.RACE_BF16, chunk)


def _device(x):
    return {n: v.cuda() for n, v in x.items()}


def _want(x, state=True):
    a = [x[n].double().numpy() for n in ("Q", "K", "V", "g", "beta")]
    scale, S, dS = x["Q"].shape[-1]**-0.5, *(x[n].double().numpy() if state else None for n in ("state", "dstate"))
    O, out = oracle.forward(*a, scale, S)
    dQ, dK, dV, dg, db, din = oracle.backward(*a, scale, x["dO"].double().numpy(), S, dS)
    return {"O": O, "state": out, "dQ": dQ, "dK": dK, "dV": dV, "dg": dg, "dbeta": db, "dstate": din}


def _got(x, chunk=0, state=True, stream=None):
    d, y = _desc(x, chunk), _device(x)
    S, dS = (y["state"], y["dstate"]) if state else (None, None)
    a = [y[n] for n in ("Q", "K", "V", "g", "beta")]
    O, out = ra.race_delta_fwd(d, *a, state_in=S, want_state=True, stream=stream)
    dQ, dK, dV, dg, db, din = ra.race_delta_bwd(d, *a, y["dO"], state_in=S, dstate_out=dS, want_dstate=True, stream=stream)
    return {"O": O, "state": out, "dQ": dQ, "dK": dK, "dV": dV, "dg": dg, "dbeta": db, "dstate": din}


def _check(got, want, dtype, label="", tol=None):
    torch.cuda.synchronize()
    tol = tol or TOL[dtype]
    for n, w in want.items():
        x = got[n].double().cpu().numpy()
        assert np.isfinite(x).all(), (label, n)
        norm = np.linalg.norm(w)
        off, big = np.linalg.norm(x - w), np.abs(x - w).max()
        print("%s %s: rel %.2e of %.2e, max %.2e" % (label, n, off / max(norm, 1e-30), tol[n], big / max(np.abs(w).max(), 1e-30)), flush=True)
        assert off <= tol[n] * norm + 1e-30, (label, n, off / norm)
        assert big <= 8 * tol[n] * np.abs(w).max() + 1e-30, (label, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk,N,dk,dv,chunk", [
    (1, 1, 1, 1, 8, 8, 0), (2, 2, 1, 2, 16, 24, 0), (1, 2, 2, 31, 40, 72, 0), (1, 1, 1, 63, 64, 64, 0), (2, 3, 3, 64, 72, 40, 0),
    (1, 4, 2, 65, 128, 128, 0), (1, 2, 1, 127, 128, 8, 0), (1, 1, 1, 128, 8, 128, 0), (1, 6, 2, 129, 96, 96, 64), (2, 2, 2, 200, 64, 128, 64),
    (1, 2, 1, 500, 128, 64, 64), (1, 1, 1, 449, 128, 128, 128), (1, 2, 2, 700, 56, 104, 256), (1, 4, 1, 300, 32, 32, 1000)])
def test_passes(B, H, Hk, N, dk, dv, chunk, dtype):
    x = _inputs(B, H, Hk, N, dk, dv, dtype, seed=N + dk)
    _check(_got(x, chunk), _want(x), dtype, "B%d H%d/%d N%d %dx%d" % (B, H, Hk, N, dk, dv))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_states(dtype):
    x = _inputs(1, 2, 1, 150, 64, 64, dtype)
    got, want = _got(x, 64, state=False), _want(x, state=False)
    _check(got, want, dtype)
    d, y = _desc(x), _device(x)
    O, none = ra.race_delta_fwd(d, *(y[n] for n in ("Q", "K", "V", "g", "beta")))
    assert none is None
    _check({"O": O}, {"O": want["O"]}, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("chunk", [0, 64])
def test_gates_of_all_kinds(dtype, chunk):
    x = _inputs(2, 4, 2, 400, 64, 64, dtype, seed=5, gates="hard")
    _check(_got(x, chunk), _want(x), dtype, "hard")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_alike(dtype):
    """Every key the same and strengths of one: I + A has ones all over its lower triangle, powers of A reach 10^18."""
    x = _inputs(1, 2, 2, 200, 64, 64, dtype, seed=7)
    x["K"][:] = x["K"][:, :, :1]
    x["g"][:] = 0.0
    x["beta"][:] = 1.0
    # |k|^2 = 1 up to the rounding of its elements: the recurrence is stable, but dK and dbeta are sums over all later tokens
    _check(_got(x), _want(x), dtype, "alike")


def test_more_than_one_window():
    """So many heads that the backward pass uses its workspace for one part of the sequence after another."""
    B, H, Hk, N, dk = 64, 128, 64, 450, 8
    x = _inputs(B, H, Hk, N, dk, dk, "bf16", seed=1)
    assert ra.race_delta_segment_tokens(_desc(x)) == 512 and _windows(_desc(x)) > 1
    _check(_got(x), _want(x), "bf16", "windows")


def _windows(d):
    """Whether a sequence twice as long takes less than twice the workspace: the backward pass goes by windows."""
    twice = ra.make_delta_desc(d.B, d.H, d.Hk, 2 * d.N, d.dk, d.dv, d.scale, d.dtype, d.chunk)
    return 2 if ra.race_delta_bwd_workspace_bytes(twice) < 1.5 * ra.race_delta_bwd_workspace_bytes(d) else 1


@pytest.mark.parametrize("B,H,N,cut", [(1, 128, 64 * 420 - 7, 64 * 200), (255, 257, 64 * 5, 64 * 2)])
def test_windows_against_parts(B, H, N, cut):
    """Windows of several segments each, and windows of the forward pass: the sequence in one call against its two parts, the state and its cotangent carried."""
    dk = 8
    gen = torch.Generator(device="cuda").manual_seed(0)
    t = torch.bfloat16
    Q, K = (torch.nn.functional.normalize(torch.randn((B, H, N, dk), generator=gen, device="cuda"), dim=-1).to(t) for _ in range(2))
    V, dO = (torch.randn((B, H, N, dk), generator=gen, device="cuda").to(t) for _ in range(2))
    g, beta = -0.05 * torch.rand((B, H, N), generator=gen, device="cuda"), torch.rand((B, H, N), generator=gen, device="cuda")
    S, dS = (torch.randn((B, H, dk, dk), generator=gen, device="cuda") for _ in range(2))
    desc = lambda n: ra.make_delta_desc(B, H, H, n, dk, dk, 0.3, ra.RACE_BF16)  # noqa: E731
    assert _windows(desc(N)) == 2
    x = (Q, K, V, g, beta)
    O, end = ra.race_delta_fwd(desc(N), *x, state_in=S, want_state=True)
    grads = ra.race_delta_bwd(desc(N), *x, dO, state_in=S, dstate_out=dS, want_dstate=True)
    head, tail = ([v[:, :, sl].contiguous() for v in x + (dO,)] for sl in (slice(0, cut), slice(cut, N)))
    Oh, mid = ra.race_delta_fwd(desc(cut), *head[:5], state_in=S, want_state=True)
    Ot, out = ra.race_delta_fwd(desc(N - cut), *tail[:5], state_in=mid, want_state=True)
    gt = ra.race_delta_bwd(desc(N - cut), *tail, state_in=mid, dstate_out=dS, want_dstate=True)
    gh = ra.race_delta_bwd(desc(cut), *head, state_in=S, dstate_out=gt[5], want_dstate=True)
    names = ("dQ", "dK", "dV", "dg", "dbeta")
    got = dict({"O": O, "state": end, "dstate": grads[5]}, **dict(zip(names, grads)))
    want = dict({"O": torch.cat((Oh, Ot), 2), "state": out, "dstate": gh[5]}, **{n: torch.cat((a, b), 2) for n, a, b in zip(names, gh, gt)})
    for n in want:      # both sides are off by what the tolerances say
        a, b = got[n].double(), want[n].double()
        off = ((a - b).norm() / b.norm()).item()
        print("%s %.2e" % (n, off), flush=True)
        assert off <= 2 * BF16[n], n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_and_parts_continue_a_state(dtype):
    """A prompt in two calls and single tokens behind it, the state carried in place, are the sequence in one call."""
    B, H, Hk, N, dk, dv = 2, 4, 2, 150, 48, 80
    x = _inputs(B, H, Hk, N, dk, dv, dtype, seed=3)
    want = _want(x)
    y = _device(x)
    state, parts = y["state"].clone(), []
    cut = lambda a, b: [y[n][:, :, a:b].contiguous() for n in ("Q", "K", "V", "g", "beta")]  # noqa: E731
    for a, b in ((0, 65), (65, 140)):
        z = cut(a, b)
        d = ra.make_delta_desc(B, H, Hk, b - a, dk, dv, dk**-0.5, _desc(x).dtype, 64)
        O, out = ra.race_delta_fwd(d, *z, state_in=state, state_out=state)
        assert out is state
        parts.append(O)
    for t in range(140, N):
        z = [v[:, :, 0].contiguous() for v in cut(t, t + 1)]
        parts.append(ra.race_delta_step(_desc(x), *z, state)[:, :, None])
    _check({"O": torch.cat(parts, 2), "state": state}, {n: want[n] for n in ("O", "state")}, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk,dk,dv", [(1, 1, 1, 8, 8), (3, 4, 2, 40, 72), (2, 8, 1, 128, 128), (70, 16, 16, 64, 96)])
def test_step(B, H, Hk, dk, dv, dtype):
    x = _inputs(B, H, Hk, 1, dk, dv, dtype, seed=dk, gates="hard" if B == 70 else "usual")
    want = _want(x)
    y = _device(x)
    z = [y[n][:, :, 0].contiguous() for n in ("Q", "K", "V", "g", "beta")]
    o = ra.race_delta_step(_desc(x), *z, y["state"])
    # fp32 arithmetic throughout: the state of either type, and before its rounding the output
    _check({"O": o[:, :, None], "state": y["state"]}, {n: want[n] for n in ("O", "state")}, dtype, tol={"O": 2.0**-8 if dtype == "bf16" else 2.0**-16, "state": 2.0**-16})


def test_empty_sequence_hands_the_state_on():
    x = _device(_inputs(1, 2, 1, 1, 16, 16, "f32"))
    y = {n: (v[:, :, :0].contiguous() if n not in ("state", "dstate") else v) for n, v in x.items()}
    d = ra.make_delta_desc(1, 2, 1, 0, 16, 16, 1.0, ra.RACE_F32)
    a = [y[n] for n in ("Q", "K", "V", "g", "beta")]
    assert torch.equal(ra.race_delta_fwd(d, *a, state_in=y["state"], want_state=True)[1], y["state"])
    assert ra.race_delta_fwd(d, *a, want_state=True)[1].abs().max().item() == 0
    assert torch.equal(ra.race_delta_bwd(d, *a, y["dO"], dstate_out=y["dstate"], want_dstate=True)[5], y["dstate"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_any_element(dtype):
    """Tensors that begin one element behind an aligned address."""
    x = _inputs(1, 2, 1, 100, 40, 24, dtype, seed=9)
    d, y = _desc(x), _device(x)
    z = {n: torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda")[1:].view(v.shape).copy_(v) for n, v in y.items()}
    outs = []
    for v in (y, z):
        a = [v[n] for n in ("Q", "K", "V", "g", "beta")]
        new = lambda n: torch.empty(v[n].numel() + 1, dtype=v[n].dtype, device="cuda")[v is z:][:v[n].numel()].view(v[n].shape)  # noqa: E731,B023
        O, S = ra.race_delta_fwd(d, *a, state_in=v["state"], O=new("V"), state_out=new("state"))
        grads = ra.race_delta_bwd(d, *a, v["dO"], state_in=v["state"], dstate_out=v["dstate"], dQ=new("Q"), dK=new("K"), dV=new("V"), dg=new("g"),
                                  dbeta=new("beta"), dstate_in=new("state"))
        step, state = [v[n][:, :, 3].clone() for n in ("Q", "K", "V", "g", "beta")], new("state").copy_(v["state"])
        o = ra.race_delta_step(d, *step, state)
        outs.append([O, S, *grads, o, state])
    torch.cuda.synchronize()
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_other_heads_and_rows_behind_are_left_alone():
    """What a call writes is its outputs: guard bands around every one of them stay; a NaN of one head stays in it."""
    x = _inputs(1, 4, 2, 90, 24, 40, "bf16", seed=2)
    y = _device(x)
    clean = _got(x)
    y["V"][:, 2] = float("nan")
    d = _desc(x)
    a = [y[n] for n in ("Q", "K", "V", "g", "beta")]
    bands = {}

    def guarded(v):
        buf = torch.full((v.numel() + 512,), 7.0, dtype=v.dtype, device="cuda")
        bands[id(buf)] = buf
        return buf[256:256 + v.numel()].view(v.shape)

    O, S = ra.race_delta_fwd(d, *a, state_in=y["state"], O=guarded(y["V"]), state_out=guarded(y["state"]))
    dQ, dK, dV, dg, db, dS = ra.race_delta_bwd(d, *a, y["dO"], state_in=y["state"], dstate_out=y["dstate"], dQ=guarded(y["Q"]), dK=guarded(y["K"]),
                                               dV=guarded(y["V"]), dg=guarded(y["g"]), dbeta=guarded(y["beta"]), dstate_in=guarded(y["state"]))
    torch.cuda.synchronize()
    for buf in bands.values():
        assert (buf[:256] == 7).all() and (buf[-256:] == 7).all()
    for n, v in (("O", O), ("state", S), ("dV", dV), ("dg", dg), ("dbeta", db), ("dstate", dS)):
        for h in (0, 1, 3):
            assert torch.equal(v[:, h], clean[n][:, h]), (n, h)
    assert torch.equal(dQ[:, 0], clean["dQ"][:, 0]) and torch.equal(dK[:, 0], clean["dK"][:, 0])
    assert torch.isnan(O[:, 2].float()).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_bits_on_another_stream_and_beside_another_call(dtype):
    x = _inputs(1, 4, 2, 333, 64, 64, dtype, seed=4)
    want = _got(x, 64)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(_got(x, 64))
    got.append(_got(x, 64, stream=streams[0]))
    torch.cuda.synchronize()
    for g in got:
        for n in want:
            assert torch.equal(g[n], want[n]), n


@pytest.mark.parametrize("dtype,H,Hk,N,chunk", [("bf16", 4, 2, 333, 64), ("f32", 2, 2, 100, 0)])
def test_replayed_from_a_graph(dtype, H, Hk, N, chunk):
    """Forward, backward and a step with the state in place, captured once; replays with eager work between them give the eager bits.  Two graphs on one workspace,
    one after the other, do too."""
    x = _device(_inputs(1, H, Hk, N, 64, 64, dtype, seed=6))
    d = _desc(x, chunk)
    a = [x[n] for n in ("Q", "K", "V", "g", "beta")]
    tok = [v[:, :, 5].contiguous() for v in a]
    ws = torch.empty(ra.race_delta_bwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    outs = {n: torch.empty_like(x[m]) for n, m in (("O", "V"), ("dQ", "Q"), ("dK", "K"), ("dV", "V"), ("dg", "g"), ("dbeta", "beta"), ("S", "state"), ("dS", "state"))}
    outs["o"] = torch.empty_like(tok[2])

    def run():
        ra.race_delta_fwd(d, *a, state_in=x["state"], O=outs["O"], state_out=outs["S"], workspace=ws)
        ra.race_delta_step(d, *tok, outs["S"], o=outs["o"])
        ra.race_delta_bwd(d, *a, x["dO"], state_in=x["state"], dstate_out=x["dstate"], dQ=outs["dQ"], dK=outs["dK"], dV=outs["dV"], dg=outs["dg"],
                          dbeta=outs["dbeta"], dstate_in=outs["dS"], workspace=ws)

    run()
    torch.cuda.synchronize()
    want = {n: v.clone() for n, v in outs.items()}
    side, graphs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            run()
    for rep in range(3):
        for graph in graphs:
            for v in outs.values():
                v.zero_()
            ws.fill_(0xFF)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for n in want:
                assert torch.equal(outs[n], want[n]), (rep, n)
        run()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(outs[n], want[n]), (rep, n)


def test_long_offsets():
    """Rows beyond 2^31 bytes and 2^31 elements of a tensor: the last tokens of a long sequence of many heads against the same
    tokens continued from the state before them."""
    B, H, N, dk, dv, cut = 1, 64, 262144 + 17, 64, 128, 262144 - 64
    gen = torch.Generator(device="cuda").manual_seed(0)
    Q, K = (torch.nn.functional.normalize(torch.randn((B, H, N, dk), generator=gen, device="cuda", dtype=torch.bfloat16), dim=-1) for _ in range(2))
    V = torch.randn((B, H, N, dv), generator=gen, device="cuda", dtype=torch.bfloat16)
    assert V.numel() > 1 << 31 and Q.numel() * 2 > 1 << 31
    g = -0.1 * torch.rand((B, H, N), generator=gen, device="cuda")
    beta = torch.rand((B, H, N), generator=gen, device="cuda")
    O, S = ra.race_delta_fwd(ra.make_delta_desc(B, H, H, N, dk, dv, 0.125, ra.RACE_BF16), Q, K, V, g, beta, want_state=True)
    head = [x[:, :, :cut].contiguous() for x in (Q, K, V, g, beta)]
    state = ra.race_delta_fwd(ra.make_delta_desc(B, H, H, cut, dk, dv, 0.125, ra.RACE_BF16), *head, want_state=True)[1]
    tail = [x[:, :, cut:].contiguous().cpu() for x in (Q, K, V, g, beta)]
    want = oracle.forward(*(x.double().numpy() for x in tail), 0.125, state.double().cpu().numpy())
    _check({"O": O[:, :, cut:], "state": S}, {"O": want[0], "state": want[1]}, "bf16")


def test_every_tensor_is_checked():
    x = _device(_inputs(1, 4, 2, 20, 16, 24, "f32"))
    d = _desc(x)
    names = ("Q", "K", "V", "g", "beta")
    wrong = [lambda t: t[..., :-1], lambda t: t.to(torch.float16), lambda t: t.cpu(), lambda t: t.transpose(-1, -2), lambda t: t.unsqueeze(0)]
    for w in wrong:
        for n in names + ("state",):
            y = dict(x)
            y[n] = w(x[n])
            with pytest.raises(ValueError):
                ra.race_delta_fwd(d, *(y[m] for m in names), state_in=y["state"])
            with pytest.raises(ValueError):
                z = {m: (v[:, :, 0].contiguous() if m != "state" else v) for m, v in x.items()}
                z[n] = w(z[n])
                ra.race_delta_step(d, *(z[m] for m in names), z["state"])
        for n in ("dO", "dstate"):
            y = dict(x)
            y[n] = w(x[n])
            with pytest.raises(ValueError):
                ra.race_delta_bwd(d, *(y[m] for m in names), y["dO"], dstate_out=y["dstate"])
    with pytest.raises(ValueError):
        ra.race_delta_fwd(d, *(x[m] for m in names), workspace=torch.empty(1 << 20, dtype=torch.uint8))
    with pytest.raises(ra.RaceAttnError) as e:
        ra.race_delta_fwd(d, *(x[m] for m in names), workspace=torch.empty(1024, dtype=torch.uint8, device="cuda"))
    assert e.value.status == ra.RACE_ERR_WORKSPACE
    with pytest.raises(TypeError):
        ra.race_delta_fwd(ra.make_desc(1, 1, 1, 8, 1, 1, 1.0, True, 0), *(x[m] for m in names), workspace=torch.empty(1024, dtype=torch.uint8, device="cuda"),
                          O=x["V"], state_out=x["state"])
