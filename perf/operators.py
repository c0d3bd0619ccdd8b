"""What the operators around the layer are measured on: the calls a user's program makes, over the sizes it makes them with.

Two operators, each in the forms that training and serving call:
  delta    the gated delta rule, the linear-time layer with a carried (dk, dv) state beside RACE attention.  Per value head
           S_t = a_t S_{t-1} + k_t b_t (v_t - a_t S_{t-1}^T k_t)^T,  a_t = exp(g_t),  o_t = scale S_t^T q_t:
             train    race_delta_fwd, then race_delta_bwd of the same inputs;
             prefill  race_delta_fwd from a carried state, with the state behind the sequence;
             step     race_delta_step, one token per sequence on the carried state (updated in place).
  rotary   norms of queries and keys for each head with the position rotation in the same pass, from the (batch, token, head)
           rows of a fused projection to the (batch, head, token) tensors that the attention layers take:
             train    race_qk_rotary_fwd, then race_qk_rotary_bwd;
             prefill  race_qk_rotary_fwd over a sequence (decoding: over one token per sequence, at positions of its own).
A delta case's values: op, kind, B, H (value heads), Hk (heads of queries and keys), N, dk, dv, dtype, pad (the last tokens of
every sequence but the first are padding: g = 0 and beta = 0).  A rotary case's: op, kind, B, N, H, Hk, d, rot (rotated
elements), norm ("rms", "l2", "none"), pairs ("halves", "neighbours"), at (position of the first token), dtype.
"""
import math

import torch

own = False             # set from outside: run() calls the framework's operators instead of their plain forms

_CHUNK = 64             # tokens that the plain form of the delta rule takes at a time
_BASE = 10000.0         # frequencies of the rotation: _BASE ** (-2 i / rot)
_EPS = 1e-6


def _delta(name, kind, B, H, Hk, N, dk, dv, dtype, pad=False):
    return {"name": name, "op": "delta", "kind": kind, "B": B, "H": H, "Hk": Hk, "N": N, "dk": dk, "dv": dv, "dtype": dtype, "pad": pad}


def _rotary(name, kind, B, N, H, Hk, d, rot, norm, pairs, dtype, at=0):
    return {"name": name, "op": "rotary", "kind": kind, "B": B, "N": N, "H": H, "Hk": Hk, "d": d, "rot": rot, "norm": norm,
            "pairs": pairs, "dtype": dtype, "at": at}


def listed():
    return [
        # one sequence being generated: the smallest call there is, once per token and layer
        _delta("step-1x4", "step", 1, 4, 4, 1, 128, 128, "bf16"),
        # a serving batch, two value heads to a key head: every state is read and written once per token
        _delta("step-64x32", "step", 64, 32, 16, 1, 128, 128, "bf16"),
        # a small fp32 layer, ragged length: research code and gradient checks
        _delta("train-f32-2k", "train", 2, 4, 4, 2003, 64, 64, "f32"),
        # short ragged sequences, padded at their ends: a small training batch
        _delta("train-short-1k", "train", 4, 4, 4, 1000, 128, 128, "bf16", pad=True),
        # heads of queries and keys shared by value heads, narrow keys, odd length
        _delta("train-shared-10k", "train", 2, 8, 4, 10007, 64, 128, "bf16"),
        # the benchmark's causal 64K configuration: few heads, one long sequence
        _delta("train-64k", "train", 1, 4, 4, 65536, 128, 128, "bf16"),
        # a prompt of odd length: outputs and the state decoding goes on from
        _delta("prefill-30k", "prefill", 1, 4, 4, 30011, 128, 128, "bf16"),
        # long context: 2^20 tokens, the shape of the scaling grid
        _delta("prefill-1m", "prefill", 1, 4, 4, 1048576, 128, 128, "bf16"),
        # one token of every sequence of a serving batch, each at its own far position
        _rotary("rotary-decode-64x32", "prefill", 64, 1, 32, 16, 128, 128, "rms", "halves", "bf16", at=4000000),
        # a prompt of odd length behind a context
        _rotary("rotary-prefill-30k", "prefill", 1, 30011, 8, 4, 128, 128, "rms", "halves", "bf16", at=4096),
        # a small fp32 layer: part of every row rotated, neighbouring elements paired, rows of length one
        _rotary("rotary-train-f32-2k", "train", 2, 2003, 4, 4, 96, 64, "l2", "neighbours", "f32"),
        # one long training sequence with eight heads of each
        _rotary("rotary-train-256k", "train", 1, 262144, 8, 8, 128, 128, "rms", "halves", "bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges above: sizes over their logarithm, odd ones among them."""
    if rng.random() < 0.4:
        kind = rng.choice(["train", "train", "prefill", "decode"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256])
        rot = rng.choice([d, d, d, d // 2, d // 4])
        Hk = rng.choice([1, 2, 3, 4, 8])
        H = Hk * rng.choice([1, 1, 2, 4])
        B = _log_uniform(rng, 1, 64) if kind == "decode" else rng.choice([1, 1, 2, 4])
        N = 1 if kind == "decode" else _log_uniform(rng, 64, 32768)
        c = _rotary("", "prefill" if kind == "decode" else kind, B, N, H, Hk, d, rot, rng.choice(["rms", "rms", "l2", "none"]),
                    rng.choice(["halves", "halves", "neighbours"]), dtype, at=rng.choice([0, 0, _log_uniform(rng, 1, 10000000)]))
    else:
        kind = rng.choice(["step", "train", "train", "train", "prefill", "prefill"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        dk, dv = rng.choice([(128, 128), (128, 128), (64, 64), (64, 128), (128, 64), (96, 96), (40, 72), (16, 32)])
        Hk = rng.choice([1, 2, 3, 4])
        H = Hk * rng.choice([1, 1, 2, 4])
        B = _log_uniform(rng, 1, 64) if kind == "step" else rng.choice([1, 1, 2, 4])
        N = 1 if kind == "step" else _log_uniform(rng, 1, 8192 if dtype == "f32" else 32768)
        c = _delta("", kind, B, H, Hk, N, dk, dv, dtype, pad=kind == "train" and B > 1 and rng.random() < 0.5)
    del c["name"]
    return c


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _unit(x):
    return x / x.norm(dim=-1, keepdim=True).clamp_min(1e-12)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = _type(case)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    B, H, Hk, N = case["B"], case["H"], case["Hk"], case["N"]
    s = dict(case)
    if case["op"] == "rotary":
        d = case["d"]
        # the rows of a fused projection of a token: its queries, keys and values behind one another
        s["rows"] = normal(B, N, (H + 2 * Hk) * d).to(t)
        s["q"] = s["rows"][..., :H * d].unflatten(-1, (H, d))
        s["k"] = s["rows"][..., H * d:(H + Hk) * d].unflatten(-1, (Hk, d))
        s["wq"], s["wk"] = 1 + 0.1 * normal(d), 1 + 0.1 * normal(d)
        if N == 1:      # decoding: every sequence is at a place of its own
            s["positions"] = case["at"] + torch.randint(0, 4096, (B, 1), generator=gen, device="cuda")
        else:
            s["positions"] = None
        s["inv_freq"] = [_BASE ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)]
        if case["kind"] == "train":
            s["dQ"], s["dK"] = normal(B, H, N, d).to(t), normal(B, Hk, N, d).to(t)
        return s
    dk, dv = case["dk"], case["dv"]
    row = () if case["kind"] == "step" else (N,)
    # rows of length one, gates as a trained layer has them: decays of a few to a few thousand tokens, another scale for each head
    s["Q"], s["K"] = _unit(normal(B, Hk, *row, dk)).to(t), _unit(normal(B, Hk, *row, dk)).to(t)
    s["V"] = normal(B, H, *row, dv).to(t)
    rate = torch.exp(-7.0 * torch.rand((B, H) + (1,) * len(row), generator=gen, device="cuda"))
    s["g"] = -rate * torch.nn.functional.softplus(normal(B, H, *row))
    s["beta"] = torch.sigmoid(normal(B, H, *row))
    if case["pad"]:
        for b in range(1, B):
            behind = N - (b * N) // (2 * B)
            s["g"][b, :, behind:] = 0.0
            s["beta"][b, :, behind:] = 0.0
    if case["kind"] != "train":
        s["state"] = 0.3 * normal(B, H, dk, dv)
    else:
        s["dO"] = normal(B, H, N, dv).to(t)
    return s


# ---- plain forms

def _inverse(A):
    """(I + A)^-1 of strictly lower triangular A (..., n, n), n a power of two: inverses of diagonal blocks, doubled."""
    n = A.shape[-1]
    T = torch.ones(A.shape[:-2] + (n, 1, 1), dtype=A.dtype, device=A.device)
    size = 1
    while size < n:
        blocks = A.unflatten(-2, (n // (2 * size), 2 * size)).unflatten(-1, (n // (2 * size), 2 * size))
        low = torch.diagonal(blocks[..., size:, :, :size], dim1=-4, dim2=-2).movedim(-1, -3)
        first, second = T[..., 0::2, :, :], T[..., 1::2, :, :]
        corner = -(second @ (low @ first))
        T = torch.cat((torch.cat((first, torch.zeros_like(corner)), -1), torch.cat((corner, second), -1)), -2)
        size *= 2
    return T.squeeze(-3)


def _plain_delta(Q, K, V, g, beta, state, scale):
    """Chunks of _CHUNK tokens: what lies within a chunk at once for all of them, the states one after another."""
    H, N = V.shape[1], V.shape[2]
    C = _CHUNK
    pad = -N % C
    Q, K = (x.float().repeat_interleave(H // x.shape[1], 1) for x in (Q, K))
    Q, K, V = (torch.nn.functional.pad(x.float(), (0, 0, 0, pad)).unflatten(2, (-1, C)) for x in (Q, K, V))
    g, beta = (torch.nn.functional.pad(x, (0, pad)).unflatten(2, (-1, C)) for x in (g, beta))
    G = g.double().cumsum(-1)
    lower = torch.ones((C, C), dtype=torch.bool, device=V.device).tril()
    D = torch.where(lower, G[..., :, None] - G[..., None, :], -math.inf).exp().float()
    start, end, whole = G.exp().float()[..., None], (G[..., -1:] - G).exp().float()[..., None], G[..., -1].exp().float()[..., None, None]
    beta = beta[..., None]
    T = _inverse(beta * (K @ K.transpose(-1, -2) * D).tril(-1))
    U, W = T @ (beta * V), T @ (beta * start * K)
    Kend = (end * K).transpose(-1, -2)
    S = torch.zeros(V.shape[:2] + (K.shape[-1], V.shape[-1]), device=V.device) if state is None else state
    states, updates = [], []
    for c in range(V.shape[2]):
        u = U[:, :, c] - W[:, :, c] @ S
        states.append(S)
        updates.append(u)
        S = whole[:, :, c] * S + Kend[:, :, c] @ u
    O = (start * Q) @ torch.stack(states, 2) + (Q @ K.transpose(-1, -2) * D) @ torch.stack(updates, 2)
    return (scale * O).flatten(2, 3)[:, :, :N], S


def _plain_rotary(x, w, case, positions, inv_freq):
    rot = case["rot"]
    x = x.float()
    if case["norm"] == "rms":
        x = x / (x.square().mean(-1, keepdim=True) + _EPS).sqrt()
    elif case["norm"] == "l2":
        x = x / (x.square().sum(-1, keepdim=True) + _EPS).sqrt()
    x = x * w
    turn = positions.double()[:, :, None, None] * torch.tensor(inv_freq, dtype=torch.float64, device=x.device)
    cos, sin = turn.cos().float(), turn.sin().float()
    part, rest = x[..., :rot], x[..., rot:]
    if case["pairs"] == "halves":
        a, b = part[..., :rot // 2], part[..., rot // 2:]
        part = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((part, rest), -1).transpose(1, 2)


def _places(s):
    if s["positions"] is not None:
        return s["positions"]
    return (s["at"] + torch.arange(s["N"], device=s["q"].device)).expand(s["B"], s["N"])


def _run_plain(s):
    t = _type(s)
    if s["op"] == "rotary":
        at = _places(s)
        if s["kind"] == "prefill":
            return {"Q": _plain_rotary(s["q"], s["wq"], s, at, s["inv_freq"]).to(t).contiguous(),
                    "K": _plain_rotary(s["k"], s["wk"], s, at, s["inv_freq"]).to(t).contiguous()}
        q, k, wq, wk = (s[n].detach().float().requires_grad_(True) for n in ("q", "k", "wq", "wk"))
        Q, K = _plain_rotary(q, wq, s, at, s["inv_freq"]), _plain_rotary(k, wk, s, at, s["inv_freq"])
        dq, dk, dwq, dwk = torch.autograd.grad((Q, K), (q, k, wq, wk), (s["dQ"].float(), s["dK"].float()))
        return {"Q": Q.detach().to(t).contiguous(), "K": K.detach().to(t).contiguous(), "dq": dq.to(t), "dk": dk.to(t), "dwq": dwq, "dwk": dwk}
    scale = s["dk"] ** -0.5
    if s["kind"] == "step":
        H, S = s["H"], s["state"]
        q, k = (s[n].float().repeat_interleave(H // s["Hk"], 1) for n in ("Q", "K"))
        S.mul_(s["g"].exp()[..., None, None])
        u = s["beta"][..., None] * (s["V"].float() - (S * k[..., None]).sum(-2))
        S.add_(k[..., None] * u[..., None, :])
        return {"O": (scale * (S * q[..., None]).sum(-2)).to(t), "state": S}
    if s["kind"] == "prefill":
        O, state = _plain_delta(s["Q"], s["K"], s["V"], s["g"], s["beta"], s["state"], scale)
        return {"O": O.to(t), "state": state}
    leaves = [s[n].detach().float().requires_grad_(True) for n in ("Q", "K", "V", "g", "beta")]
    O, _ = _plain_delta(*leaves, None, scale)
    dQ, dK, dV, dg, dbeta = torch.autograd.grad(O, leaves, s["dO"].float())
    return {"O": O.detach().to(t), "dQ": dQ.to(t), "dK": dK.to(t), "dV": dV.to(t), "dg": dg, "dbeta": dbeta}


# ---- the framework's operators

def _handle(s):
    """What a program keeps from call to call: the descriptor, the workspace and the output buffers."""
    import paper_2510_04008_amd as ra
    kind = ra.RACE_F32 if s["dtype"] == "f32" else ra.RACE_BF16
    like = lambda x: torch.empty(x.shape, dtype=x.dtype, device=x.device)  # noqa: E731
    if s["op"] == "rotary":
        d = ra.make_rotary_desc(s["B"], s["N"], s["H"], s["Hk"], s["d"], s["rot"], kind, norm=s["norm"], pairs=s["pairs"], eps=_EPS, pos0=s["at"])
        t, h = _type(s), {"ra": ra, "desc": d}
        h["Q"] = torch.empty((s["B"], s["H"], s["N"], s["d"]), dtype=t, device="cuda")
        h["K"] = torch.empty((s["B"], s["Hk"], s["N"], s["d"]), dtype=t, device="cuda")
        if s["kind"] == "train":
            h["rows"] = like(s["rows"])             # the cotangent of the fused projection, whose values' part is another's to write
            n, m = s["H"] * s["d"], s["Hk"] * s["d"]
            h["dq"], h["dk"] = h["rows"][..., :n].unflatten(-1, (s["H"], s["d"])), h["rows"][..., n:n + m].unflatten(-1, (s["Hk"], s["d"]))
            h["dwq"], h["dwk"] = like(s["wq"]), like(s["wk"])
            h["ws"] = torch.empty(max(256, ra.race_qk_rotary_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
        return h
    d = ra.make_delta_desc(s["B"], s["H"], s["Hk"], s["N"], s["dk"], s["dv"], s["dk"] ** -0.5, kind)
    h = {"ra": ra, "desc": d, "O": like(s["V"])}
    if s["kind"] == "prefill":
        h["state"] = like(s["state"])
    if s["kind"] != "step":
        need = ra.race_delta_workspace_bytes(d)
        if s["kind"] == "train":
            need = max(need, ra.race_delta_bwd_workspace_bytes(d))
            h["grads"] = [like(s[n]) for n in ("Q", "K", "V", "g", "beta")]
        h["ws"] = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    return h


def _run_own(s):
    if "handle" not in s:
        s["handle"] = _handle(s)
    h = s["handle"]
    ra, d = h["ra"], h["desc"]
    if s["op"] == "rotary":
        ra.race_qk_rotary_fwd(d, s["q"], s["k"], s["wq"], s["wk"], s["inv_freq"], s["positions"], Q=h["Q"], K=h["K"])
        if s["kind"] == "prefill":
            return {"Q": h["Q"], "K": h["K"]}
        ra.race_qk_rotary_bwd(d, s["q"], s["k"], s["wq"], s["wk"], s["inv_freq"], s["positions"], s["dQ"], s["dK"], dq=h["dq"], dk=h["dk"],
                              dwq=h["dwq"], dwk=h["dwk"], workspace=h["ws"])
        return {n: h[n] for n in ("Q", "K", "dq", "dk", "dwq", "dwk")}
    if s["kind"] == "step":
        ra.race_delta_step(d, s["Q"], s["K"], s["V"], s["g"], s["beta"], s["state"], o=h["O"])
        return {"O": h["O"], "state": s["state"]}
    if s["kind"] == "prefill":
        ra.race_delta_fwd(d, s["Q"], s["K"], s["V"], s["g"], s["beta"], state_in=s["state"], O=h["O"], state_out=h["state"], workspace=h["ws"])
        return {"O": h["O"], "state": h["state"]}
    ra.race_delta_fwd(d, s["Q"], s["K"], s["V"], s["g"], s["beta"], O=h["O"], workspace=h["ws"])
    dQ, dK, dV, dg, dbeta = h["grads"]
    ra.race_delta_bwd(d, s["Q"], s["K"], s["V"], s["g"], s["beta"], s["dO"], dQ=dQ, dK=dK, dV=dV, dg=dg, dbeta=dbeta, workspace=h["ws"])
    return {"O": h["O"], "dQ": dQ, "dK": dK, "dV": dV, "dg": dg, "dbeta": dbeta}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without

def work(case):
    B, H, Hk, N = case["B"], case["H"], case["Hk"], case["N"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rotary":
        rows, d = B * N * (H + Hk), case["d"]
        train = case["kind"] == "train"
        # forward: rows in and out; backward: rows and cotangents in, cotangents out
        return {"bytes": e * rows * d * (5 if train else 2), "flops": rows * d * (24 if train else 8)}
    dk, dv = case["dk"], case["dv"]
    rows = B * N
    qk, v, gates = e * rows * Hk * 2 * dk, e * rows * H * dv, 8 * rows * H
    state = 4 * B * H * dk * dv
    recurrence = rows * H * dk * dv
    if case["kind"] == "step":      # S^T k, the update and S^T q
        return {"bytes": qk + 2 * v + gates + 2 * state, "flops": 7 * recurrence}
    if case["kind"] == "prefill":
        return {"bytes": qk + 2 * v + gates + 2 * state, "flops": 7 * recurrence}
    # forward; backward: inputs and dO in, five gradients out, the states once more and their cotangents (five products a token)
    return {"bytes": (qk + 2 * v + gates) + (2 * qk + 3 * v + 2 * gates), "flops": (7 + 7 + 12) * recurrence}


# ---- 64 bits, from the definitions

def _exact_delta(s):
    """One token after another."""
    group, N, scale = s["H"] // s["Hk"], s["N"], s["dk"] ** -0.5
    Q, K = (s[n].double().unsqueeze(2).expand(-1, -1, group, *s[n].shape[2:]).flatten(1, 2) for n in ("Q", "K"))
    V, g, beta = s["V"].double(), s["g"].double(), s["beta"].double()
    if s["kind"] == "step":
        Q, K, V, g, beta = (x.unsqueeze(2) for x in (Q, K, V, g, beta))
    a = g.exp()

    def token(S, t):
        """The decayed state, the error and the new state."""
        Sd = a[:, :, t, None, None] * S
        e = V[:, :, t] - torch.matmul(K[:, :, t, None, :], Sd)[:, :, 0]
        return Sd, e, Sd + K[:, :, t, :, None] * (beta[:, :, t, None] * e)[:, :, None, :]

    S = s["state"].double() if "state" in s else torch.zeros(V.shape[:2] + (s["dk"], s["dv"]), dtype=torch.float64, device=V.device)
    O = torch.empty_like(V)
    block, marks = 64, []
    for t in range(N):
        if t % block == 0:
            marks.append(S)
        S = token(S, t)[2]
        O[:, :, t] = scale * torch.matmul(Q[:, :, t, None, :], S)[:, :, 0]
    if s["kind"] == "step":
        return {"O": O[:, :, 0], "state": S}
    if s["kind"] == "prefill":
        return {"O": O, "state": S}
    dO = s["dO"].double()
    dQ, dK, dV, dg, db = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V), torch.empty_like(g), torch.empty_like(g)
    dS = torch.zeros_like(S)
    for c in range(len(marks) - 1, -1, -1):
        kept, S = [], marks[c]
        for t in range(c * block, min(N, (c + 1) * block)):
            kept.append(token(S, t))
            S = kept[-1][2]
        for t in range(min(N, (c + 1) * block) - 1, c * block - 1, -1):
            Sd, e, S = kept[t - c * block]
            q, k, do, b = Q[:, :, t], K[:, :, t], dO[:, :, t], beta[:, :, t, None]
            dQ[:, :, t] = scale * torch.matmul(S, do[..., None])[..., 0]
            dS = dS + scale * q[..., None] * do[:, :, None, :]
            du = torch.matmul(k[:, :, None, :], dS)[:, :, 0]
            de = b * du
            dV[:, :, t] = de
            db[:, :, t] = (e * du).sum(-1)
            dK[:, :, t] = torch.matmul(dS, (b * e)[..., None])[..., 0] - torch.matmul(Sd, de[..., None])[..., 0]
            dS = dS - k[..., None] * de[:, :, None, :]
            dg[:, :, t] = (Sd * dS).sum((-1, -2))
            dS = a[:, :, t, None, None] * dS
    dQ, dK = (x.unflatten(1, (s["Hk"], group)).sum(2) for x in (dQ, dK))
    return {"O": O, "dQ": dQ, "dK": dK, "dV": dV, "dg": dg, "dbeta": db}


def _exact_rotary(s):
    """The rotation as a product of complex numbers, its gradient as the product with the conjugate."""
    d, rot = s["d"], s["rot"]
    freq = torch.tensor(s["inv_freq"], dtype=torch.float64, device=s["q"].device)
    angle = _places(s).double()[:, None, :, None] * freq
    turn = torch.complex(angle.cos(), angle.sin())
    order = torch.arange(rot, device=s["q"].device)
    order = order.view(2, -1).t() if s["pairs"] == "halves" else order.view(-1, 2)          # (pair, member)

    def rotate(x, by):
        z = torch.view_as_complex(x[..., order].contiguous()) * by
        y = x.clone()
        y[..., order] = torch.view_as_real(z)
        return y

    out = {}
    for x, w, name, grad in ((s["q"], s["wq"], "Q", "q"), (s["k"], s["wk"], "K", "k")):
        x, w = x.double().transpose(1, 2), w.double()
        n = {"rms": (x * x).sum(-1, keepdim=True) / d, "l2": (x * x).sum(-1, keepdim=True), "none": None}[s["norm"]]
        r = (n + _EPS) ** -0.5 if n is not None else torch.ones_like(x[..., :1])
        out[name] = rotate(x * r * w, turn)
        if s["kind"] == "train":
            dy = rotate(s["d" + name].double(), turn.conj())
            out["dw" + grad] = (dy * x * r).sum((0, 1, 2))
            dx = dy * w * r
            if n is not None:
                dx = dx - x * (dx * x).sum(-1, keepdim=True) * r * r / (d if s["norm"] == "rms" else 1)
            out["d" + grad] = dx.transpose(1, 2)
    return out


def exact(case, seed):
    tokens = case["N"] if case["op"] == "delta" else 0
    if tokens > 32768 or (case["kind"] == "train" and tokens > 12000):
        return None             # one token after another would take too long
    s = prepare(case, seed)
    return _exact_rotary(s) if case["op"] == "rotary" else _exact_delta(s)
