// Plan of a gated delta rule call: what the host side (operators_api.cpp) derives from a validated descriptor and the launches
// (delta_kernels.hip) follow.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace race {
namespace delta {

// Whether `steps` transitions of BH heads are joined in groups (delta_combine_kernel) and not one after the other.  In groups there are three short chains for a long
// one, but every group's transitions are multiplied with one another, which fills the chip from some eight heads on.  Measured, us, one after the other / in groups,
// 128 x 128, bf16:  4 heads: 16 steps 31 / 37, 20: 37 / 38, 24: 44 / 41, 64: 106 / 59;  8 heads: 24: 43 / 49, 32: 56 / 59, 48: 81 / 67;  16 heads: 64: 108 / 129,
// 128: 324 / 308;  32 heads: 128: 359 / 566.  64 x 64: 4 heads: 24: 23 / 26, 32: 30 / 29;  16 heads: 32: 29 / 32, 48: 41 / 36.
inline bool joined_in_groups(int steps, int BH) { return BH <= 16 && steps >= 24 && 2 * steps >= BH * BH; }

struct DeltaPlan {
    int B, H, Hk, BH, dk, dv, dvp, dtype;       // dvp: dv rounded up to 32
    int64_t N;
    float scale;
    int chunks;                     // of 64 tokens
    int seg_chunks, nseg;           // chunks per segment (the last may be short), segments
    int win_segs, windows;          // segments per window (the last may hold fewer), windows: a window's workspace is the next one's too
    // workspace, byte offsets (multiples of 256).  Per chunk of a window: T, decays and, backward, M^T, T^T, A^T, states, U, cotangents, dR
    size_t off_T, off_dec, off_MT, off_TT, off_AT, off_S, off_U, off_dS, off_dR, off_pq, off_pk;
    // per segment of a window: states (cotangents) from zero, transitions and, backward, cotangents at the ends; per segment of the sequence: states at the
    // starts and, backward, transposed transitions (the windows are gone through from the last to the first once all starts are known)
    size_t off_add, off_P, off_end, off_start, off_PT;
    int join_groups;                // at most, of a window's segments (delta_combine_kernel); their transitions, states from zero and starts
    size_t off_group_P, off_group_add, off_group_start;
    size_t off_carry;               // one state a head between windows
    size_t total;
};

struct DeltaIo {
    const void *Q, *K, *V, *dO;
    const float *g, *beta, *state_in, *dstate_out;
    void *O, *dQ, *dK, *dV;
    float *state_out, *dg, *dbeta, *dstate_in;
};

hipError_t forward(const DeltaPlan &p, const DeltaIo &io, char *ws, hipStream_t st);
hipError_t backward(const DeltaPlan &p, const DeltaIo &io, char *ws, hipStream_t st);
hipError_t step(const DeltaPlan &p, const DeltaIo &io, hipStream_t st);        // io.state_out is the state, updated in place
hipError_t copy_state(const DeltaPlan &p, const float *from, float *to, hipStream_t st);       // from null: zeros

}  // namespace delta
}  // namespace race
