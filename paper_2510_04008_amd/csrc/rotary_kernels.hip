// Norms of queries and keys for each head with the position rotation in the same pass.
//
// A row x (d elements of one token and head) becomes y = rotate(x r w) with r = 1 / sqrt(mean x^2 + eps) ("rms"), 1 / sqrt(sum x^2 + eps) ("l2")
// or 1, and rotate turning pair i of the first rot elements by the angle position * frequency_i.  Backward, with u the cotangent of y turned
// back: dw = sum over rows of u x r, dx = r w u - x r^3 <w u, x> / d (l2: without the d).
//
// Every row is read and written once and that is what bounds it.  A group of lanes holds a row: a lane has W elements of each
// side of W pairs, so that a pair never leaves its lane.  The sines and cosines of a token are the same for all heads: a group
// makes them once and takes several heads.  Angles are counted in turns in fp64 (position times turns per position, less the nearest
// whole number) and only then rounded to fp32: at position 10^7 an fp32 angle would be off by half a radian.
//
// 262144 tokens of 8 + 8 heads, d = 128, bf16: forward 452 us (2.1 GB, 4.8 TB/s), backward with the weights' sums 690 us (3.2 GB, 4.7 TB/s); a copy of 2 GiB
// reaches 4.9 TB/s.  64 tokens of 32 + 16 heads: 4.5 us, one launch; there a workgroup takes few heads of a token, for there are not tokens enough to fill the chip.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "rotary_plan.h"

namespace race {
namespace rotary {
namespace {

constexpr int kThreads = 256;
// Workgroups of a launch of the forward pass: a grid's dimension has to stay below 2^32 threads, so more tokens take several launches.  (A loop over tokens
// in the kernel instead cost a tenth of its time: 262144 tokens of 8 + 8 heads, d = 128, 491 us against 446.)
constexpr int64_t kMaxBlocks = 1 << 23;

template <class E, int W> struct Run;       // W elements as they lie in memory; a caller's rows are aligned to their elements only
template <> struct Run<uint16_t, 4> { typedef __attribute__((ext_vector_type(4), aligned(2))) uint16_t T; };
template <> struct Run<float, 4> { typedef __attribute__((ext_vector_type(4), aligned(4))) float T; };
template <> struct Run<uint16_t, 1> { typedef __attribute__((ext_vector_type(1))) uint16_t T; };
template <> struct Run<float, 1> { typedef __attribute__((ext_vector_type(1))) float T; };

__device__ __forceinline__ float value(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ void put(uint16_t &to, float x) { to = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }
__device__ __forceinline__ void put(float &to, float x) { to = x; }

template <int W, class E>
__device__ __forceinline__ void load(const E *p, float *x)
{
    const typename Run<E, W>::T v = *reinterpret_cast<const typename Run<E, W>::T *>(p);
#pragma unroll
    for (int e = 0; e < W; ++e) x[e] = value(static_cast<E>(v[e]));
}
template <int W, class E>
__device__ __forceinline__ void store(E *p, const float *x)
{
    typename Run<E, W>::T v;
#pragma unroll
    for (int e = 0; e < W; ++e) {
        E t;
        put(t, x[e]);
        v[e] = t;
    }
    *reinterpret_cast<typename Run<E, W>::T *>(p) = v;
}

// the lane's place in a row, and the turns of its pairs
template <int W, int NU>
struct Lane {
    bool there[NU], turned[NU];
    int a[NU], b[NU];               // first elements of its two runs
    float c[NU][W], s[NU][W];

    __device__ __forceinline__ void place(const RotaryPlan &p, int lane, int lanes)
    {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int unit = lane + u * lanes;
            there[u] = 2 * W * unit < p.d;
            turned[u] = there[u] && 2 * W * unit < p.rot;
            const bool halves = turned[u] && !p.neighbours;
            a[u] = halves ? W * unit : 2 * W * unit;
            b[u] = halves ? p.rot / 2 + W * unit : 2 * W * unit + W;
        }
    }
    __device__ __forceinline__ void turn(const RotaryPlan &p, int lane, int lanes, int64_t position)
    {
#pragma unroll
        for (int u = 0; u < NU; ++u)
            if (turned[u])
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const double t = static_cast<double>(position) * p.turns[W * (lane + u * lanes) + e];
                    sincospif(2.f * static_cast<float>(t - rint(t)), &s[u][e], &c[u][e]);
                }
    }
    // members of pair e among the 2 W values of unit u (two runs behind one another)
    static __device__ __forceinline__ void rotate(bool neighbours, float *x, const float *c, const float *s, float sign)
    {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            float &m = neighbours ? x[2 * e] : x[e], &n = neighbours ? x[2 * e + 1] : x[W + e];
            const float y = m * c[e] - sign * n * s[e];
            n = n * c[e] + sign * m * s[e];
            m = y;
        }
    }
    // a loop over constants for each order, so that the values stay in registers
    __device__ __forceinline__ void rotate(const RotaryPlan &p, float (&x)[NU][2 * W], float sign) const
    {
#pragma unroll
        for (int u = 0; u < NU; ++u)
            if (turned[u]) {
                if (p.neighbours) rotate(true, x[u], c[u], s[u], sign);
                else rotate(false, x[u], c[u], s[u], sign);
            }
    }
    template <class E>
    __device__ __forceinline__ void row(const E *p, float (&x)[NU][2 * W]) const
    {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
#pragma unroll
            for (int e = 0; e < 2 * W; ++e) x[u][e] = 0.f;
            if (there[u]) {
                load<W>(p + a[u], x[u]);
                load<W>(p + b[u], x[u] + W);
            }
        }
    }
    template <class E>
    __device__ __forceinline__ void put_row(E *p, const float (&x)[NU][2 * W]) const
    {
#pragma unroll
        for (int u = 0; u < NU; ++u)
            if (there[u]) {
                store<W>(p + a[u], x[u]);
                store<W>(p + b[u], x[u] + W);
            }
    }
};

__device__ __forceinline__ float over_group(float x, int lanes)
{
    for (int m = 1; m < lanes; m *= 2) x += __shfl_xor(x, m);
    return x;
}
__device__ __forceinline__ float scale_of(const RotaryPlan &p, float squares)
{
    if (p.norm == 0) return 1.f;
    return 1.f / sqrtf((p.norm == 1 ? squares / static_cast<float>(p.d) : squares) + p.eps);
}

template <class E, int W, int NU>
__global__ __launch_bounds__(kThreads) void rotary_fwd_kernel(RotaryPlan p, int lanes, int heads_each, int64_t token0)
{
    const int lane = threadIdx.x & (lanes - 1), groups = kThreads / lanes;
    const int64_t tokens = static_cast<int64_t>(p.B) * p.N;
    const int64_t token = token0 + static_cast<int64_t>(blockIdx.x) * groups + threadIdx.x / lanes;
    if (token >= tokens) return;            // whole groups: the sums over a group's lanes stay complete
    const int64_t b = token / p.N, n = token - b * p.N;
    Lane<W, NU> l;
    l.place(p, lane, lanes);
    l.turn(p, lane, lanes, p.positions ? p.positions[token] : p.pos0 + n);
    const int first = blockIdx.y * heads_each, last = min(first + heads_each, p.q.heads + p.k.heads);
    for (int hh = first; hh < last; ++hh) {
        const bool isq = hh < p.q.heads;
        const Rows &r = isq ? p.q : p.k;
        const int h = isq ? hh : hh - p.q.heads;
        float x[NU][2 * W], w[NU][2 * W];
        l.row(static_cast<const E *>(r.x) + b * r.batch + n * r.token + h * r.head, x);
        float ss = 0.f;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int e = 0; e < 2 * W; ++e) ss += x[u][e] * x[u][e];
        const float scale = scale_of(p, p.norm ? over_group(ss, lanes) : 0.f);
        if (r.w) l.row(r.w, w);
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int e = 0; e < 2 * W; ++e) x[u][e] *= r.w ? scale * w[u][e] : scale;
        l.rotate(p, x, 1.f);
        l.put_row(static_cast<E *>(r.y) + ((b * r.heads + h) * p.N + n) * p.d, x);
    }
}

// Sums for the weights: a lane adds up over the rows that it meets, the groups of a workgroup are added in order in LDS, and the
// workgroups' sums by the kernel below, in order: the same bits every time.
template <class E, int W, int NU>
__global__ __launch_bounds__(kThreads) void rotary_bwd_kernel(RotaryPlan p, int lanes, float *parts)
{
    extern __shared__ float sums[];         // (groups, d)
    const int lane = threadIdx.x & (lanes - 1), groups = kThreads / lanes, group = threadIdx.x / lanes;
    const int64_t tokens = static_cast<int64_t>(p.B) * p.N;
    Lane<W, NU> l;
    l.place(p, lane, lanes);
    float dw[2][NU][2 * W];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int e = 0; e < 2 * W; ++e) dw[i][u][e] = 0.f;
    for (int64_t token = static_cast<int64_t>(blockIdx.x) * groups + group; token < tokens; token += static_cast<int64_t>(gridDim.x) * groups) {
        const int64_t b = token / p.N, n = token - b * p.N;
        l.turn(p, lane, lanes, p.positions ? p.positions[token] : p.pos0 + n);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const Rows &r = i == 0 ? p.q : p.k;
            float w[NU][2 * W];
            if (r.w) l.row(r.w, w);
            for (int h = 0; h < r.heads; ++h) {
                float x[NU][2 * W], u[NU][2 * W];
                l.row(static_cast<const E *>(r.x) + b * r.batch + n * r.token + h * r.head, x);
                l.row(static_cast<const E *>(r.y) + ((b * r.heads + h) * p.N + n) * p.d, u);
                l.rotate(p, u, -1.f);
                float ss = 0.f, dot = 0.f;
#pragma unroll
                for (int j = 0; j < NU; ++j)
#pragma unroll
                    for (int e = 0; e < 2 * W; ++e) {
                        ss += x[j][e] * x[j][e];
                        dot += (r.w ? w[j][e] * u[j][e] : u[j][e]) * x[j][e];
                    }
                float scale = 1.f, back = 0.f;
                if (p.norm) {
                    scale = scale_of(p, over_group(ss, lanes));
                    back = over_group(dot, lanes) * scale * scale * scale;
                    if (p.norm == 1) back /= static_cast<float>(p.d);
                }
#pragma unroll
                for (int j = 0; j < NU; ++j)
#pragma unroll
                    for (int e = 0; e < 2 * W; ++e) {
                        dw[i][j][e] += u[j][e] * x[j][e] * scale;
                        u[j][e] = scale * (r.w ? w[j][e] * u[j][e] : u[j][e]) - x[j][e] * back;
                    }
                l.put_row(static_cast<E *>(r.dx) + b * r.dbatch + n * r.dtoken + h * r.dhead, u);
            }
        }
    }
    if (!parts) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        __syncthreads();
        l.put_row(sums + group * p.d, dw[i]);
        __syncthreads();
        for (int e = threadIdx.x; e < p.d; e += kThreads) {
            float s = 0.f;
            for (int g = 0; g < groups; ++g) s += sums[g * p.d + e];
            parts[(static_cast<size_t>(blockIdx.x) * 2 + i) * p.d + e] = s;
        }
    }
}

// one workgroup per 8 elements: 32 threads add every 32nd part each, in order, then the 32 sums in order
__global__ __launch_bounds__(kThreads) void rotary_weights_kernel(const float *parts, int count, int d, float *dwq, float *dwk)
{
    __shared__ float sums[32][8];
    const int e = threadIdx.x & 7, g = threadIdx.x >> 3, at = blockIdx.x * 8 + e;
    float s = 0.f;
    for (int i = g; i < count; i += 32) s += parts[static_cast<size_t>(i) * 2 * d + at];
    sums[g][e] = s;
    __syncthreads();
    if (threadIdx.x < 8) {
        s = 0.f;
        for (int i = 0; i < 32; ++i) s += sums[i][e];
        float *to = at < d ? dwq : dwk;
        if (to) to[at < d ? at : at - d] = s;
    }
}

// runs of four elements where pairs allow it, single elements otherwise
bool by_fours(const RotaryPlan &p) { return p.rot % 8 == 0; }
int lanes_of(const RotaryPlan &p, int w)
{
    int lanes = 4;
    while (lanes < 64 && 2 * w * lanes < p.d) lanes *= 2;
    return lanes;
}
int parts_of(const RotaryPlan &p)
{
    const int groups = kThreads / lanes_of(p, by_fours(p) ? 4 : 1);
    const int64_t tokens = static_cast<int64_t>(p.B) * p.N;
    return static_cast<int>(std::min<int64_t>(kMaxParts, (tokens + groups - 1) / groups));
}

template <class E, int W, int NU>
hipError_t launch_fwd(const RotaryPlan &p, hipStream_t st)
{
    const int lanes = lanes_of(p, W), groups = kThreads / lanes, heads = p.q.heads + p.k.heads;
    const int64_t blocks = (static_cast<int64_t>(p.B) * p.N + groups - 1) / groups;
    int each = heads;       // fewer heads a group where there are few tokens
    while (each > 1 && blocks * ((heads + each - 1) / each) < 1024) each = (each + 1) / 2;
    for (int64_t first = 0; first < blocks; first += kMaxBlocks) {
        const dim3 grid(static_cast<unsigned>(std::min(kMaxBlocks, blocks - first)), (heads + each - 1) / each);
        ProfileScope scope("rotary_fwd", st);
        rotary_fwd_kernel<E, W, NU><<<grid, kThreads, 0, st>>>(p, lanes, each, first * groups);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <class E, int W, int NU>
hipError_t launch_bwd(const RotaryPlan &p, float *parts, hipStream_t st)
{
    const int lanes = lanes_of(p, W), groups = kThreads / lanes;
    ProfileScope scope("rotary_bwd", st);
    rotary_bwd_kernel<E, W, NU><<<parts_of(p), kThreads, groups * p.d * sizeof(float), st>>>(p, lanes, parts);
    return hipGetLastError();
}

}  // namespace

size_t workspace_bytes(const RotaryPlan &p) { return static_cast<size_t>(parts_of(p)) * 2 * p.d * sizeof(float); }

hipError_t forward(const RotaryPlan &p, hipStream_t st)
{
    if (p.dtype == RACE_BF16) {
        if (by_fours(p)) return launch_fwd<uint16_t, 4, 1>(p, st);
        return p.d > 128 ? launch_fwd<uint16_t, 1, 2>(p, st) : launch_fwd<uint16_t, 1, 1>(p, st);
    }
    if (by_fours(p)) return launch_fwd<float, 4, 1>(p, st);
    return p.d > 128 ? launch_fwd<float, 1, 2>(p, st) : launch_fwd<float, 1, 1>(p, st);
}

hipError_t backward(const RotaryPlan &p, float *dwq, float *dwk, char *ws, hipStream_t st)
{
    float *parts = dwq || dwk ? reinterpret_cast<float *>(ws) : nullptr;
    hipError_t e;
    if (p.dtype == RACE_BF16) {
        if (by_fours(p)) e = launch_bwd<uint16_t, 4, 1>(p, parts, st);
        else e = p.d > 128 ? launch_bwd<uint16_t, 1, 2>(p, parts, st) : launch_bwd<uint16_t, 1, 1>(p, parts, st);
    } else {
        if (by_fours(p)) e = launch_bwd<float, 4, 1>(p, parts, st);
        else e = p.d > 128 ? launch_bwd<float, 1, 2>(p, parts, st) : launch_bwd<float, 1, 1>(p, parts, st);
    }
    if (e != hipSuccess || !parts) return e;
    ProfileScope scope("rotary_weights", st);
    rotary_weights_kernel<<<2 * p.d / 8, kThreads, 0, st>>>(parts, parts_of(p), p.d, dwq, dwk);
    return hipGetLastError();
}

}  // namespace rotary
}  // namespace race
