"""GPU tests of outputs that are small differences: values that overwrite much larger ones, read back by their keys.

Keys and queries are unit vectors e_i, so products with them are exact, strengths one and decays none.  O_t is the value just written, the sum of the state's row before and the
update; its terms are up to max |S|, each held in fp32 or as 24 bits (half a step: 2^-24), and at most eight of them are not zeros: 8 * 2^-24 max |S| = 2^-21 max |S|, and the
rounding to bf16, 2^-8 of the value.  An element of dQ_t is a sum of dv products of such a row with dO_t: dv * 2^-21 max |S| max |dO|."""
import numpy as np
import pytest
import torch

import paper_2510_04008_amd as ra

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv,chunk", [(16, 16, 0), (32, 64, 0), (64, 64, 0), (64, 128, 64), (128, 128, 0), (128, 128, 64)])
def test_small_values_over_large_ones(dk, dv, chunk, dtype):
    H, rounds = 2, 2
    N = rounds * dk
    r = np.random.RandomState(dk + dv)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    rows = np.tile(np.eye(dk), (rounds, 1))[None, None].repeat(H, 1)
    Q, K, V, dO = (torch.from_numpy(x).to(t) for x in (rows, rows, r.randn(1, H, N, dv), r.randn(1, H, N, dv)))
    state = torch.from_numpy(4096.0 * r.randn(1, H, dk, dv)).float()
    g, beta = torch.zeros((1, H, N)), torch.ones((1, H, N))
    d = ra.make_delta_desc(1, H, H, N, dk, dv, 1.0, ra.RACE_F32 if dtype == "f32" else ra.RACE_BF16, chunk)
    a, S = [x.cuda() for x in (Q, K, V, g, beta)], state.cuda()
    O, out = ra.race_delta_fwd(d, *a, state_in=S, want_state=True)
    dQ = ra.race_delta_bwd(d, *a, dO.cuda(), state_in=S)[0]
    torch.cuda.synchronize()
    big, step = state.abs().max().item(), 2.0**-8 if dtype == "bf16" else 2.0**-24
    O, dQ, V, dO = (x.double().cpu().numpy() for x in (O, dQ, V, dO))
    # the rows of the state are the values written last
    assert np.abs(out.double().cpu().numpy() - V[:, :, N - dk:]).max() <= 2.0**-21 * big
    off = np.abs(O - V)
    print("O: %.2e of %.2e" % (off.max(), 2.0**-21 * big), flush=True)
    assert (off <= step * np.abs(V) + 2.0**-21 * big).all()
    for i in range(N):              # elements whose row has been overwritten
        last = [i - (i - j) % dk for j in range(min(i + 1, dk))]
        want = np.einsum("bhkv,bhv->bhk", V[:, :, last], dO[:, :, i])
        got = dQ[:, :, i, :len(last)]
        assert (np.abs(got - want) <= step * np.abs(want) + dv * 2.0**-21 * big * np.abs(dO).max()).all(), i
