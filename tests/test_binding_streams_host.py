"""CPU checks of what the binding allocates for a call on another stream: scratch and outputs belong to that stream (the allocator hands a block on behind the
work of the stream that it was allocated for, so scratch of the current stream could be another tensor's while the call still runs)."""
import contextlib
import types

import pytest

import paper_2510_04008_amd as ra
from paper_2510_04008_amd import binding


class Stream:
    def __init__(self, raw):
        self.cuda_stream = raw


class Tensor:
    is_cuda, device = True, "cuda:0"

    def __init__(self, shape, dtype, made_on=None):
        self.shape, self.dtype, self.made_on, self.users = tuple(shape), dtype, made_on, []

    def is_contiguous(self):
        return True

    def numel(self):
        return 1 << 40

    def data_ptr(self):
        return 1 << 20

    def record_stream(self, stream):
        self.users.append(stream)


class Torch:
    """The part of torch that the binding calls; `made` holds every tensor that it allocates."""
    uint8, float32, bfloat16 = "uint8", "float32", "bfloat16"

    def __init__(self):
        self.made, self.here, self.outer = [], None, Stream(7)
        self.cuda = types.SimpleNamespace(Stream=Stream, ExternalStream=Stream, stream=self._on, current_stream=lambda: self.here or self.outer,
                                          default_stream=lambda: Stream(0))

    @contextlib.contextmanager
    def _on(self, stream):
        before, self.here = self.here, stream
        yield
        self.here = before

    def empty(self, shape, dtype, device):
        self.made.append(Tensor(shape if isinstance(shape, tuple) else (shape,), dtype, self.here))
        return self.made[-1]

    def empty_like(self, x):
        return self.empty(x.shape, x.dtype, x.device)


class Native:
    def __getattr__(self, name):
        return lambda *args: ra.RACE_OK


B, H, N, D = 2, 4, 70, 64
FREQ = [1.0] * (D // 2)


def _calls():
    ad, dd, rd = ra.make_desc(B, H, N, D, 4, 4, 4.0, True, ra.RACE_F32), ra.make_delta_desc(B, H, H, N, D, D, 1.0, ra.RACE_F32), ra.make_rotary_desc(B, N, H, H, D, D, ra.RACE_F32)
    full, rows, row = Tensor((B, H, N, D), "float32"), Tensor((B, N, H, D), "float32"), Tensor((B, H, D), "float32")
    gates, gate, state, w = Tensor((B, H, N), "float32"), Tensor((B, H), "float32"), Tensor((B, H, D, D), "float32"), Tensor((D,), "float32")
    seeds = [1, 2, 3, 4]
    return {
        "race_attn_fwd": lambda **s: ra.race_attn_fwd(ad, full, full, full, seeds, **s),
        "race_attn_bwd": lambda **s: ra.race_attn_bwd(ad, full, full, full, full, gates, full, seeds, **s),
        "race_attn_bwd_beta": lambda **s: ra.race_attn_bwd_beta(ad, full, full, full, full, gates, full, seeds, **s),
        "race_attn_bwd_saved": lambda **s: ra.race_attn_bwd_saved(ad, full, full, full, full, gates, full, seeds, full, want_dbeta=True, **s),
        "race_attn_state_init": lambda **s: ra.race_attn_state_init(ad, full, full, seeds, **s),
        "race_attn_step": lambda **s: ra.race_attn_step(ad, row, row, row, seeds, full, **s),
        "race_delta_fwd": lambda **s: ra.race_delta_fwd(dd, full, full, full, gates, gates, want_state=True, **s),
        "race_delta_bwd": lambda **s: ra.race_delta_bwd(dd, full, full, full, gates, gates, full, want_dstate=True, **s),
        "race_delta_step": lambda **s: ra.race_delta_step(dd, row, row, row, gate, gate, state, **s),
        "race_qk_rotary_fwd": lambda **s: ra.race_qk_rotary_fwd(rd, rows, rows, w, w, FREQ, **s),
        "race_qk_rotary_bwd": lambda **s: ra.race_qk_rotary_bwd(rd, rows, rows, w, w, FREQ, None, full, full, **s),
    }


@pytest.fixture
def torch_(monkeypatch):
    t = Torch()
    monkeypatch.setattr(binding, "_torch", lambda: t)
    monkeypatch.setattr(binding, "_native_module", Native())
    return t


@pytest.mark.parametrize("name", list(_calls()))
def test_what_a_call_allocates_belongs_to_its_stream(torch_, name):
    stream = Stream(123456)
    out = _calls()[name](stream=stream)
    out = out if isinstance(out, tuple) else (out,)
    assert torch_.made and all(t.made_on is stream for t in torch_.made)
    assert torch_.here is None
    for t in torch_.made:           # what the caller gets is used on the current stream next
        assert t.users == ([torch_.outer] if any(t is o for o in out) else [])


def test_raw_handles_and_the_current_stream(torch_):
    for raw, want in ((4711, 4711), (0, 0)):        # the null handle is the default stream
        torch_.made.clear()
        _calls()["race_delta_fwd"](stream=raw)
        assert torch_.made and all(t.made_on.cuda_stream == want for t in torch_.made)
    torch_.made.clear()
    _calls()["race_delta_fwd"]()
    assert torch_.made and all(t.made_on is None and t.users == [] for t in torch_.made)
