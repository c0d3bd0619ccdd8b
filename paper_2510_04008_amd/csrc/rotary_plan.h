// Arguments of the per-head norms with the position rotation: what the host side (operators_api.cpp) hands to the launches
// (rotary_kernels.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace race {
namespace rotary {

constexpr int kMaxPairs = 128;      // of a row
constexpr int kMaxParts = 1024;     // partial sums of the weights' cotangents

struct Rows {
    const void *x;                  // the rows as given
    const float *w;                 // null: ones
    void *y;                        // forward: (B, heads, N, d) out; backward: its cotangent, in
    void *dx;                       // backward, out
    int heads;
    int64_t batch, token, head;     // strides of x, elements
    int64_t dbatch, dtoken, dhead;  // strides of dx
};
struct RotaryPlan {
    int B, d, rot, norm, neighbours, dtype;
    int64_t N, pos0;
    float eps;
    const int64_t *positions;       // (B, N), null: pos0 + index
    Rows q, k;
    double turns[kMaxPairs];        // of a pair, per position
};

size_t workspace_bytes(const RotaryPlan &p);            // backward
hipError_t forward(const RotaryPlan &p, hipStream_t st);
hipError_t backward(const RotaryPlan &p, float *dwq, float *dwk, char *ws, hipStream_t st);

}  // namespace rotary
}  // namespace race
