"""CPU checks of how the gated delta rule's workspace grows."""
import pytest

import paper_2510_04008_amd as ra


def _desc(N, B=1, H=4, Hk=4, chunk=0):
    return ra.make_delta_desc(B, H, Hk, N, 128, 128, 1.0, ra.RACE_BF16, chunk)


@pytest.mark.parametrize("chunk", [0, 4096, 65536])
@pytest.mark.parametrize("N", [1 << 24, 1 << 26])
def test_what_windows_leave_of_a_segment(N, chunk):
    """Of every segment behind the first window a state, and backward its transposed transition (of a state's size here): not what only its window needs."""
    d, twice = _desc(N, chunk=chunk), _desc(2 * N, chunk=chunk)
    segment, state = ra.race_delta_segment_tokens(d), ra.race_delta_state_bytes(d)
    assert ra.race_delta_segment_tokens(twice) == segment
    assert ra.race_delta_workspace_bytes(twice) - ra.race_delta_workspace_bytes(d) <= (N // segment + 1) * state + 4096
    # (a backward pass that chooses its segments takes shorter ones: 60 chunks)
    assert ra.race_delta_bwd_workspace_bytes(twice) - ra.race_delta_bwd_workspace_bytes(d) <= (N // (chunk or 3000) + 1) * 2 * state + 4096


def test_workspace_of_a_caller_s_segment():
    """Chunks of 64 tokens of a segment that is the whole sequence: the figures of the header."""
    for N in (1 << 16, 1 << 20):
        chunks = 4 * N // 64
        for need, Hk, lo, hi in ((ra.race_delta_workspace_bytes, 4, 17e3, 18e3), (ra.race_delta_bwd_workspace_bytes, 4, 0.25e6, 0.27e6), (ra.race_delta_bwd_workspace_bytes, 2, 0.31e6, 0.34e6)):
            assert lo < need(_desc(N, Hk=Hk, chunk=N)) / chunks < hi
