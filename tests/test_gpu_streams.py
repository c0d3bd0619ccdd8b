"""GPU test of calls on streams of their own without a workspace: their scratch is nobody else's while they run."""
import pytest
import torch

import paper_2510_04008_amd as ra
from paper_2510_04008_amd import binding

pytestmark = pytest.mark.gpu


class Watch:
    """The binding's extension module, noting the workspace's bytes of every call."""

    def __init__(self, module, at):
        self.module, self.at, self.spans = module, at, []

    def __getattr__(self, name):
        def call(*args):
            w = args[self.at[name]]
            self.spans.append((w.data_ptr(), w.data_ptr() + w.numel()))
            return getattr(self.module, name)(*args)
        return call


def _overlap(a, b):
    return a[0] < b[1] and b[0] < a[1]


def test_scratch_of_two_streams_and_of_the_current_one(monkeypatch):
    B, H, N, D = 2, 4, 1500, 64
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    d = ra.make_delta_desc(B, H, H, N, D, D, 0.125, ra.RACE_BF16)
    r = ra.make_rotary_desc(B, N, H, H, D, D, ra.RACE_BF16)
    freq = [10000.0 ** (-2.0 * i / D) for i in range(D // 2)]
    sets = []
    for _ in range(2):
        Q, K = (torch.nn.functional.normalize(rand(B, H, N, D), dim=-1).bfloat16() for _ in range(2))
        V, dO = rand(B, H, N, D).bfloat16(), rand(B, H, N, D).bfloat16()
        g, beta = -torch.rand((B, H, N), generator=gen, device="cuda"), torch.rand((B, H, N), generator=gen, device="cuda")
        q, k, w = rand(B, N, H, D).bfloat16(), rand(B, N, H, D).bfloat16(), 1 + 0.1 * rand(D)
        sets.append((Q, K, V, g, beta, dO, q, k, w))

    def run(x, stream):
        Q, K, V, g, beta, dO, q, k, w = x
        return [*ra.race_delta_fwd(d, Q, K, V, g, beta, want_state=True, stream=stream), *ra.race_delta_bwd(d, Q, K, V, g, beta, dO, want_dstate=True, stream=stream),
                *ra.race_qk_rotary_bwd(r, q, k, w, w, freq, None, dO, dO, stream=stream)]

    want = [run(x, None) for x in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    watch = Watch(binding._native(), {"delta_fwd": 9, "delta_bwd": 15, "rotary_bwd": 13})
    monkeypatch.setattr(binding, "_native_module", watch)
    got, spans = [], []
    for x, s in zip(sets, streams):
        with torch.cuda.stream(s):
            torch.cuda._sleep(2_000_000)        # the calls wait behind it
        watch.spans.clear()
        got.append(run(x, s))
        spans.append(list(watch.spans))
    # what the current stream is given now is none of it
    mine = [torch.empty(b - a, dtype=torch.uint8, device="cuda") for span in spans for a, b in span]
    spans.append([(t.data_ptr(), t.data_ptr() + t.numel()) for t in mine])
    for i in range(len(spans)):
        for j in range(i):
            assert not any(_overlap(a, b) for a in spans[i] for b in spans[j])
    for t in mine:
        t.fill_(0xFF)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
