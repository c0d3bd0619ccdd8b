// The gated delta rule: forward and backward pass over chunks of 64 tokens, and the decoding step.  The mathematics and the
// operand layouts stand in delta_common.h.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "delta_common.h"
#include "delta_plan.h"
#include "internal.h"

namespace race {
namespace delta {
namespace {

struct Sizes {
    int64_t N;
    int H, Hk, dk, dv, dvp;         // dvp: dv rounded up to 32
    float scale;
    int seg_chunks, nseg, win_segs; // chunks per segment, segments of the sequence, of a window (the last may hold fewer)
    int seg0, segs;                 // the window: first segment, segments
    int chunk0, chunks;             // first chunk, chunks
};

__device__ __forceinline__ int64_t qk_row(const Sizes &z, int bh, int64_t t)
{
    const int b = bh / z.H, h = bh - b * z.H;
    return (static_cast<int64_t>(b) * z.Hk + h / (z.H / z.Hk)) * z.N + t;
}
__device__ __forceinline__ int tokens_of(const Sizes &z, int chunk) { return static_cast<int>(min(static_cast<int64_t>(C), z.N - static_cast<int64_t>(chunk) * C)); }

// one 32-row operand of caller's rows: row0 + lane % 32, elements k0 .. k0 + 7
template <class X>
__device__ __forceinline__ typename X::Exact rows8(const typename X::E *p, int row, int rows, int width, int k0)
{
    return load8(p + static_cast<int64_t>(row) * width + k0, row < rows && k0 < width);
}

// 8 values of an fp32 image
__device__ __forceinline__ void kept8(const float *p, float *x)
{
    const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
}

// ------------------------------------------------------------------ what a chunk needs besides the states
// T and the decays of one chunk of one head, and for the backward pass M^T, T^T and A^T.  T: the four 16 x 16 diagonal blocks by substitution (one wavefront, a lane
// per column), then [[T1, 0], [-T2 A21 T1, T2]] twice on the fp32 matrix instructions, each block in A's place.  Substitution and not powers of A: with keys
// alike the powers reach thousands where T stays near one.
// Images are written in the order in which the scans' operands lie in LDS (rows in spread order), in fp32: half of the bytes of a Split.
// One workgroup of four wavefronts per chunk and head, several on a CU, so that one's substitution (16 steps of one wavefront) runs beside another's loads.  65536 chunks
// of dk = 128, bf16 (2^20 tokens, four heads): 658 us, 34 KB a chunk and 3.4 TB/s; wavefronts wait 75 % of their time, for loads and
// at the barriers between the steps.  With what the way back needs, 80 KB a chunk, 4096 chunks take 88 us.
template <int SIZE>
struct MergeBlocks {
    static constexpr int NT = SIZE / 16;
    f32x4 R[NT];
    // -T2 A21 T1 for 16 columns of the pair of blocks that begins at row `base`
    __device__ __forceinline__ void form(float (*A)[68], int base, int slab, int lane)
    {
        const int r16 = lane & 15, q = lane >> 4;
        f32x4 P[NT];
#pragma unroll
        for (int ti = 0; ti < NT; ++ti) {
            P[ti] = zero4();
#pragma unroll
            for (int k = 0; k < SIZE / 4; ++k)
                P[ti] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[base + SIZE + 16 * ti + r16][base + 4 * k + q], A[base + 4 * k + q][base + 16 * slab + r16], P[ti], 0, 0, 0);
        }
#pragma unroll
        for (int ti = 0; ti < NT; ++ti) {
            R[ti] = zero4();
#pragma unroll
            for (int tk = 0; tk < NT; ++tk)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    R[ti] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[base + SIZE + 16 * ti + r16][base + SIZE + 16 * tk + 4 * q + r], P[tk][r], R[ti], 0, 0, 0);
        }
    }
    __device__ __forceinline__ void put(float (*A)[68], int base, int slab, int lane) const
    {
#pragma unroll
        for (int ti = 0; ti < NT; ++ti)
#pragma unroll
            for (int r = 0; r < 4; ++r) A[base + SIZE + 16 * ti + 4 * (lane >> 4) + r][base + 16 * slab + (lane & 15)] = -R[ti][r];
    }
};

struct PrepArgs {
    Sizes z;
    const void *Q, *K;
    const float *g, *beta;
    float *T, *MT, *TT, *AT;        // 64 x 64 images, rows in spread order: T - I; backward also M^T, T^T - I and, on and below A's diagonal, A^T
    float *dec;             // per chunk (kDec): e^G, e^{G_C - G}, beta, and G as the sum of two floats
};

template <class X, int DK, bool BWD>
__global__ __launch_bounds__(256) void delta_prep_kernel(PrepArgs a)
{
    typedef typename X::E E;
    __shared__ __attribute__((aligned(16))) float B[C], hi_of[C], lo_of[C];
    __shared__ __attribute__((aligned(16))) float A[C][68];     // then T
    const Sizes &z = a.z;
    const int tid = threadIdx.x, wave = wave_index(), lane = tid & 63, h = lane >> 5, col = lane & 31;
    const int bh = blockIdx.y, n = tokens_of(z, z.chunk0 + blockIdx.x);
    const int64_t t0 = static_cast<int64_t>(z.chunk0 + blockIdx.x) * C;
    const size_t at = static_cast<size_t>(bh) * z.chunks + blockIdx.x;
    const int ti = wave > 0 ? 1 : 0, tj = wave == 2 ? 1 : 0;
    f32x16 kk = zero16(), qk = zero16();
    if (wave == 3) {
        const int64_t t = static_cast<int64_t>(bh) * z.N + t0 + lane;
        const double g = prefix64(lane < n ? static_cast<double>(gate(a.g[t])) : 0.0, lane);
        const float b = lane < n ? strength(a.beta[t]) : 0.f, hi = static_cast<float>(g);
        hi_of[lane] = hi;
        lo_of[lane] = static_cast<float>(g - hi);
        B[lane] = b;
        float *dec = a.dec + at * kDec;
        dec[lane] = expf(hi);
        dec[C + lane] = expf(static_cast<float>(__shfl(g, 63) - g));
        dec[2 * C + lane] = b;
        dec[3 * C + lane] = hi;
        dec[4 * C + lane] = static_cast<float>(g - hi);
#pragma unroll
        for (int i = 0; i < 16; ++i) A[2 * i + (lane >> 5)][32 + (lane & 31)] = 0.f;
    } else {
        const E *Q = static_cast<const E *>(a.Q) + qk_row(z, bh, t0) * z.dk, *K = static_cast<const E *>(a.K) + qk_row(z, bh, t0) * z.dk;
#pragma unroll
        for (int kb = 0; kb < DK / 16; ++kb) {
            const int k0 = 16 * kb + 8 * h;
            const typename X::Exact ki = rows8<X>(K, 32 * ti + col, n, z.dk, k0), kj = rows8<X>(K, 32 * tj + col, n, z.dk, k0);
            kk = mma(ki, kj, kk);
            if (BWD) qk = mma(rows8<X>(Q, 32 * ti + col, n, z.dk, k0), kj, qk);
        }
    }
    __syncthreads();
    if (wave < 3) {
        const size_t to = at * C * C + (32 * tj + col) * C + 32 * ti;
        const int j = 32 * tj + col;
        const float hj = hi_of[j], lj = lo_of[j];
        const bool idle_j = B[j] == 0.f;
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const int i0 = 32 * ti + acc_row(4 * e4, h);
            const f32x4 hi = *reinterpret_cast<const f32x4 *>(hi_of + i0), lo = *reinterpret_cast<const f32x4 *>(lo_of + i0), b = *reinterpret_cast<const f32x4 *>(B + i0);
            f32x4 m, y4;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float D = decay(hi[e], lo[e], hj, lj), x = z.scale * D * qk[4 * e4 + e], y = b[e] * D * kk[4 * e4 + e];
                m[e] = j <= i0 + e ? (idle_j ? idle(x) : x) : 0.f;
                // (the column of a token of strength zero meets its zeros; only its own cotangent reads it)
                A[i0 + e][j] = y4[e] = j < i0 + e && b[e] != 0.f ? (idle_j ? (BWD ? idle(y) : 0.f) : y) : 0.f;
            }
            if (BWD) {
                *reinterpret_cast<f32x4 *>(a.MT + to + spread(acc_row(4 * e4, h))) = m;
                *reinterpret_cast<f32x4 *>(a.AT + to + spread(acc_row(4 * e4, h))) = y4;
            }
        }
    }
    __syncthreads();
    if (wave == 0) {
        const int b0 = (lane >> 4) * 16, c16 = lane & 15;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == c16 ? 1.f : 0.f;
#pragma unroll
            for (int j = 0; j < i; ++j) s -= A[b0 + i][b0 + j] * x[j];
            x[i] = s;
        }
        // (all of the wavefront has read its block)
#pragma unroll
        for (int i = 0; i < 16; ++i) A[b0 + i][b0 + c16] = x[i];
    }
    __syncthreads();
    if (wave < 2) {
        MergeBlocks<16> m;
        m.form(A, 32 * wave, 0, lane);
        m.put(A, 32 * wave, 0, lane);
    }
    __syncthreads();
    MergeBlocks<32> m;
    if (wave < 2) m.form(A, 0, wave, lane);
    __syncthreads();            // both halves have been read
    if (wave < 2) m.put(A, 0, wave, lane);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int task = tid + 256 * i, row = task >> 4, k = 4 * (task & 15);
        f32x4 v = *reinterpret_cast<const f32x4 *>(&A[row][k]), w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (k + e == row) v[e] = 0.f;
            w[e] = k + e == row || !BWD ? 0.f : A[k + e][row];
        }
        *reinterpret_cast<f32x4 *>(a.T + at * C * C + row * C + spread(k)) = v;
        if (BWD) *reinterpret_cast<f32x4 *>(a.TT + at * C * C + row * C + spread(k)) = w;
    }
}

// ------------------------------------------------------------------ tiles in LDS
template <class X, int DK>
struct Lds {
    typedef typename X::E E;
    static constexpr int kRow = DK + X::kPad;       // a token's row
    static constexpr int kTok = C + X::kPad;        // a row over tokens, in spread order
    static constexpr int kByTokens = C * kRow, kByRows = DK * kTok, kSquare = C * kTok;
};

// 64 rows of a caller's tensor on their way into LDS, as they are, or transposed, or both.  Loads are asked for a chunk ahead (take) and
// written when the tiles are free (put): with two wavefronts per SIMD nothing else hides their latency.  2 DK tasks of four tokens by eight elements.
// The rows of the transposed tile are stored in the order of the state's rows in the accumulators (row_place).
__device__ __forceinline__ int row_place(int k) { return (k & ~31) | ((k & 4) << 2) | ((k & 24) >> 1) | (k & 3); }
template <class X, int DK>
struct RowsStage {
    typedef typename X::E E;
    typedef Lds<X, DK> L;
    typename X::Exact x[4];
    // sixteen lanes take four by four: neither way of writing meets one bank more than twice
    static __device__ __forceinline__ int quad(int task) { return (task & 3) | (task >> 2 & 12); }
    static __device__ __forceinline__ int octet(int task) { return (task >> 2 & 3) | (task >> 4 & ~3); }
    __device__ __forceinline__ void take(const E *src, int n, int dk, int task)
    {
        const int tq = quad(task), o = octet(task);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = load8(src + static_cast<int64_t>(min(4 * tq + r, n - 1)) * dk + (8 * o < dk ? 8 * o : 0), true);
    }
    template <bool ROWS, bool COLS, bool PLACED = true>
    __device__ __forceinline__ void put(int n, int dk, E *rows, E *cols, int task)
    {
        const int tq = quad(task), o = octet(task);
        if (n < C || dk < DK) {
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = or_zero(x[r], 4 * tq + r < n && 8 * o < dk);
        }
        if (ROWS) {
#pragma unroll
            for (int r = 0; r < 4; ++r) put8(rows + (4 * tq + r) * L::kRow + 8 * o, x[r]);
        }
        if (COLS) {
            E e[4][8];
#pragma unroll
            for (int r = 0; r < 4; ++r) __builtin_memcpy(e[r], &x[r], sizeof e[r]);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                E v[4] = {e[0][k], e[1][k], e[2][k], e[3][k]};
                E *to = cols + (PLACED ? row_place(8 * o + k) : 8 * o + k) * L::kTok + spread(4 * tq);
                __builtin_memcpy(__builtin_assume_aligned(to, 4 * sizeof(E)), v, 4 * sizeof(E));
            }
        }
    }
};

// a 64 x 64 fp32 image of the workspace on its way into LDS as an operand in planes, by 512 threads or 256
template <int THREADS>
struct ImageStage {
    static constexpr int kEach = 512 / THREADS;
    float x[kEach][8];
    __device__ __forceinline__ void take(const float *src, int tid)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) kept8(src + (tid + THREADS * i) * 8, x[i]);
    }
    template <class X, class OPERAND>
    __device__ __forceinline__ void put(typename X::E *dst, int tid) const
    {
        constexpr int kTok = C + X::kPad;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int task = tid + THREADS * i;
            OPERAND s;
            split8(x[i], s);
            put8(dst + (task >> 3) * kTok + (task & 7) * 8, C * kTok, s);
        }
    }
};

// left operand from a tile in LDS: rows row0 + lane % 16, 32 places from k0
template <class X, int STRIDE>
__device__ __forceinline__ typename X::Exact tile8(const typename X::E *t, int row0, int k0, int lane)
{
    return get8(t + (row0 + (lane & 15)) * STRIDE + k0 + 8 * (lane >> 4));
}
template <class OPERAND, int STRIDE, class E>
__device__ __forceinline__ OPERAND tile8s(const E *t, int row0, int k0, int lane)
{
    OPERAND x;
    get8(t + (row0 + (lane & 15)) * STRIDE + k0 + 8 * (lane >> 4), C * STRIDE, x);
    return x;
}

// The compiler would ask for the operands of later products long before it has registers for them.
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// two accumulators on top of one another as a right operand
template <class OPERAND>
__device__ __forceinline__ OPERAND operand(const f32x4 &first, const f32x4 &second)
{
    const float x[8] = {first[0], first[1], first[2], first[3], second[0], second[1], second[2], second[3]};
    OPERAND s;
    split8(x, s);
    return s;
}
template <class X>
__device__ __forceinline__ typename X::Exact rounded(const f32x4 &first, const f32x4 &second)
{
    const float x[8] = {first[0], first[1], first[2], first[3], second[0], second[1], second[2], second[3]};
    typename X::Exact s;
    round8(x, s);
    return s;
}

// 64 rows by 16 columns of a caller's tensor on their way into accumulators (rows in registers, columns in lanes)
template <class X>
struct ColumnsStage {
    typename X::Exact x[4];
    __device__ __forceinline__ void take(const typename X::E *p, int n, int width, int k0, int lane)
    {
        const int k = k0 + 8 * ((lane >> 4) & 1);
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) x[ti] = load8(p + static_cast<int64_t>(min(16 * ti + (lane & 15), n - 1)) * width + (k < width ? k : 0), true);
    }
    // Rows behind the last token repeat it: their strengths, keys and queries are zero.  Columns that there are not are zeros of `unit`.
    static __device__ __forceinline__ typename X::Exact unit(int width, int k0, int lane)
    {
        return or_zero(unit8<X, false>(0, lane), k0 + 8 * ((lane >> 4) & 1) < width);
    }
    __device__ __forceinline__ f32x4 tile(int ti, const typename X::Exact &unit) const { return mma(x[ti], unit, zero4()); }
};
// the way back, rounded to the element type: two accumulators on top of one another, 32 rows from row0
template <class X>
__device__ __forceinline__ void store_rows(typename X::E *p, int row0, int rows, int width, int k0, const f32x4 &first, const f32x4 &second, int lane)
{
    const typename X::Exact x = rounded<X>(first, second);
    const int k = k0 + 4 * (lane >> 4);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const f32x4 t = mma(x, unit8<X, true>(b, lane), zero4());
        const int row = row0 + 16 * b + (lane & 15);
        const float y[4] = {t[0], t[1], t[2], t[3]};
        if (row < rows && k < width) store4(p + static_cast<int64_t>(row) * width + k, y);
    }
}
// Two accumulators on top of one another, as the operand that they are, into the workspace.  Tokens (U, dR): rows row0 .. + 31 of a 64 x dvp image, columns
// k0 .. k0 + 15 in spread order.
template <class X>
__device__ __forceinline__ void keep_tokens(float *p, int row0, int width, int k0, const typename X::Split &x, int lane)
{
    const buffer_t image = buffer(p, static_cast<size_t>(C) * width);
    const int to = 4 * ((lane & 15) * width + spread(k0 + 4 * (lane >> 4)));
#pragma unroll
    for (int b = 0; b < 2; ++b) put_buffer(image, to + 4 * (row0 + 16 * b) * width, mma(x, unit8<X, true>(b, lane), zero4()));
}
// States: in the order in which they are read as right operands, of dk, 256 floats together (16 rows, half of a step of 32 columns)
__device__ __forceinline__ int state_place(int tile, int step, int half, int steps) { return ((tile * steps + step) * 2 + half) * 256; }
template <class X, int DK>
__device__ __forceinline__ void keep_state(float *p, int tile0, int width, int k0, const typename X::Split &x, int lane)
{
    const buffer_t image = buffer(p, static_cast<size_t>(DK) * width);
#pragma unroll
    for (int b = 0; b < 2; ++b)
        put_buffer(image, 4 * (state_place(tile0 + b, k0 >> 5, k0 >> 4 & 1, width / 32) + 4 * lane), mma(x, unit8<X, false>(b, lane), zero4()));
}

// A wavefront's 16 columns of a (dk, dv) fp32 state; rows and columns that it has not are zero, and are not written.  Rows are
// dealt to the accumulators so that two of them, as an operand, hold rows 8 q .. 8 q + 7 of 32 (the order of K's rows in memory).
__device__ __forceinline__ int state_row(int tile, int q, int e) { return 32 * (tile >> 1) + 8 * q + 4 * (tile & 1) + e; }
__device__ __forceinline__ int state_offset(int row, int dv, int col) { return col < dv ? 4 * (row * dv + col) : kNowhere; }
// A transition, a DK x DK fp32 matrix, lies in the order in which it is read as a left operand: 512 values together for 16 rows (dealt as above) by 32
// columns.
constexpr int kOperand = 512;
template <int DK>
__device__ __forceinline__ int transition_place(int row, int k)
{
    const int tile = 2 * (row >> 5) + (row >> 2 & 1), m = (row >> 3 & 3) * 4 + (row & 3);
    return (tile * (DK / 32) + (k >> 5)) * kOperand + ((k >> 3 & 3) * 16 + m) * 8 + (k & 7);
}
template <int TILES>
__device__ __forceinline__ void get_state(f32x4 (&S)[TILES], const float *state, int dk, int dv, int tile0, int col, int lane)
{
    const buffer_t b = buffer(state, static_cast<size_t>(dk) * dv);
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[t][e] = get_buffer(b, state_offset(state_row(tile0 + t, lane >> 4, e), dv, col));
}
template <int TILES>
__device__ __forceinline__ void put_state(const f32x4 (&S)[TILES], float *state, int dk, int dv, int tile0, int col, int lane)
{
    const buffer_t b = buffer(state, static_cast<size_t>(dk) * dv);
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) put_buffer(b, state_offset(state_row(tile0 + t, lane >> 4, e), dv, col), S[t][e]);
}

// ------------------------------------------------------------------ the states, chunk after chunk
// One workgroup per segment, head and up to eight (four) tiles of 16 columns of the state; a wavefront keeps its columns of the state in
// accumulators from chunk to chunk (DK x 16 fp32), where they are at once the right operand of the products with K and Q.
// Columns never meet, so wavefronts share the tiles in LDS and nothing else.
//
// A chunk is a chain of products, each of which needs the one before it, and no unit is saturated: at dk = dv = 128, bf16, the matrix units are busy 41 to 47 % of the time, the
// vector ALU, which splits states, R and U into bf16 for the next product, 49 to 61 % (the issue of matrix instructions included), LDS 32 to 48 % (bank conflicts 14 to 21),
// and wavefronts wait 22 to 32 %; the state's columns in registers (up to 248 a lane) leave room for two wavefronts a SIMD to fill the gaps.  (fp32, 64 x 64: matrix units 43
// to 49 %, vector ALU 17, waiting 28 to 38.)  Sixteen columns a wavefront and eight wavefronts beat 32 columns and four (one wavefront a SIMD: nothing
// to fill its waits).  Tried without gain: operands asked for before the split of the state, and priorities for the matrix phases or for half of the wavefronts.  2^20 tokens, four heads, 64 segments, so a workgroup
// on every CU: 2.02 ms, 7.9 us a chunk; the pre-pass, two workgroups a segment: 2.21 ms; kKeep, 96 KB a chunk more to write, takes 7.2 us a chunk.
enum ScanMode { kOut, kPre, kKeep };        // the pass proper; a segment's transition and state from zero; states and U for the backward pass

struct ScanArgs {
    Sizes z;
    const void *Q, *K, *V;
    const float *T, *dec;
    const float *start;             // state at the start of a segment, (dk, dv) fp32: start + bh * start_head + segment * dk * dv; null: zero
    size_t start_head;
    float *final_state;             // state behind the window's last segment (null: not wanted); kPre: behind every segment
    size_t final_head;
    void *O;
    float *P, *PT;                  // kPre: the transition, per segment of the window, and its transpose, per segment of the sequence (null: not wanted)
    int transitions;                // kPre
    float *S, *U;                   // kKeep: states at the chunks' starts, and U, rows in spread order
};

template <class X, int DK, int THREADS, int MODE>
__global__ __launch_bounds__(THREADS) void delta_scan_kernel(ScanArgs a)
{
    typedef typename X::E E;
    typedef typename X::Split Split;
    typedef Lds<X, DK> L;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    E *Ks = reinterpret_cast<E *>(lds_raw), *Kt = Ks + L::kByTokens, *Ts = Kt + L::kByRows, *Qs = Ts + X::kPlanes * L::kSquare;
    E *Ms = Qs + L::kByTokens;
    float *dec = reinterpret_cast<float *>(MODE == kOut ? Ms + X::kPlanes * L::kSquare : Qs);
    const Sizes &z = a.z;
    const int tid = threadIdx.x, wave = wave_index(), lane = tid & 63, q = lane >> 4, col = lane & 15;
    const int bh = blockIdx.z, seg = blockIdx.y;
    const int vtiles = z.dvp / 16, tile = blockIdx.x * (THREADS / 64) + wave;
    const bool trans = MODE == kPre && tile >= vtiles;
    const bool active = MODE == kPre ? tile < vtiles + (a.transitions ? DK / 16 : 0) : tile < vtiles;
    const int vcol = 16 * tile + col;                   // column of V (or, less the tiles of V, of the transition)
    const int c0 = (z.seg0 + seg) * z.seg_chunks - z.chunk0, c1 = min(c0 + z.seg_chunks, z.chunks);
    static_assert(THREADS >= 4 * DK, "a thread stages rows of K or of Q");
    const bool has_k = tid < 2 * DK, has_q = MODE == kOut && tid >= 2 * DK && tid < 4 * DK;
    const int task = has_k ? tid : tid - 2 * DK;

    f32x4 S[DK / 16];
#pragma unroll
    for (int t = 0; t < DK / 16; ++t) S[t] = zero4();
    if (trans) {
#pragma unroll
        for (int t = 0; t < DK / 16; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) S[t][e] = state_row(t, q, e) == vcol - z.dvp ? 1.f : 0.f;
    } else if (a.start && active) {
        get_state(S, a.start + bh * a.start_head + static_cast<size_t>(seg) * z.dk * z.dv, z.dk, z.dv, 0, vcol, lane);
    }
    constexpr bool kAhead = sizeof(E) == 2;         // fp32 operands leave no registers for the images
    RowsStage<X, DK> rows;
    ImageStage<THREADS> is;
    ColumnsStage<X> vs;
    const typename X::Exact unit = ColumnsStage<X>::unit(z.dv, 16 * tile, lane);
    float ds[(kDec + THREADS - 1) / THREADS];
    auto take = [&](int c) {
        const int64_t t0 = static_cast<int64_t>(z.chunk0 + c) * C;
        const int n = tokens_of(z, z.chunk0 + c);
        const size_t at = static_cast<size_t>(bh) * z.chunks + c;
        if (has_k || has_q) rows.take(static_cast<const E *>(has_k ? a.K : a.Q) + qk_row(z, bh, t0) * z.dk, n, z.dk, task);
        if (kAhead) {
            is.take(a.T + at * C * C, tid);
        }
#pragma unroll
        for (int i = 0; i < (kDec + THREADS - 1) / THREADS; ++i)
            if (tid + THREADS * i < kDec) ds[i] = a.dec[at * kDec + tid + THREADS * i];
    };
    auto take_columns = [&](int c) {
        const int64_t t0 = static_cast<int64_t>(z.chunk0 + c) * C;
        if (!trans) vs.take(static_cast<const E *>(a.V) + (static_cast<int64_t>(bh) * z.N + t0) * z.dv, tokens_of(z, z.chunk0 + c), z.dv, 16 * tile, lane);
    };
    if (c0 < c1) {
        take(c0);
        if (active) take_columns(c0);
    }
    if (MODE == kOut && tid < 128) {        // what M's tiles leave out of the steps of 32 tokens on the diagonal
        const int t = 2 * (tid >> 6), row = 16 * t + (tid >> 2 & 15);
        put4(Ms + row * L::kTok + spread(16 * t + 16 + 4 * (tid & 3)), L::kSquare, zero4());
    }
    for (int c = c0; c < c1; ++c) {
        const int64_t t0 = static_cast<int64_t>(z.chunk0 + c) * C;
        const int n = tokens_of(z, z.chunk0 + c);
        const size_t at = static_cast<size_t>(bh) * z.chunks + c;
        __syncthreads();
        if (has_k) rows.template put<true, true>(n, z.dk, Ks, Kt, task);
        if (has_q) rows.template put<true, false>(n, z.dk, Qs, nullptr, task);
        if (!kAhead) is.take(a.T + at * C * C, tid);
        is.template put<X, Split>(Ts, tid);
#pragma unroll
        for (int i = 0; i < (kDec + THREADS - 1) / THREADS; ++i)
            if (tid + THREADS * i < kDec) dec[tid + THREADS * i] = ds[i];
        __syncthreads();
        if (c + 1 < c1) take(c + 1);
        const float *eG = dec, *eEnd = dec + C, *beta = dec + 2 * C;
        if (MODE == kOut) {         // M, a tile on or below the diagonal after the other: rows j, columns i
            for (int t = wave; t < 10; t += THREADS / 64) {
                const int ti = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3, tj = t - ti * (ti + 1) / 2, i = 16 * ti + col, j0 = 16 * tj + 4 * q;
                f32x4 m = zero4();
#pragma unroll
                for (int kb = 0; kb < DK / 32; ++kb) m = mma(tile8<X, L::kRow>(Ks, 16 * tj, 32 * kb, lane), tile8<X, L::kRow>(Qs, 16 * ti, 32 * kb, lane), m);
                const float hi = dec[3 * C + i], lo = dec[4 * C + i];
                const f32x4 hj = *reinterpret_cast<const f32x4 *>(dec + 3 * C + j0), lj = *reinterpret_cast<const f32x4 *>(dec + 4 * C + j0);
                const f32x4 bj = *reinterpret_cast<const f32x4 *>(beta + j0);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = z.scale * decay(hi, lo, hj[e], lj[e]) * m[e];
                    m[e] = j0 + e <= i && bj[e] != 0.f ? x : 0.f;
                }
                put4(Ms + i * L::kTok + spread(j0), L::kSquare, m);
            }
            fence();
        }
        if (!active && MODE != kOut) continue;
        fence();
        // K S, and Q S for the outputs
        f32x4 R[4], O[4];
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) R[ti] = O[ti] = zero4();
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) {
            const Split s = operand<Split>(S[2 * kb], S[2 * kb + 1]);
            if (sizeof(E) == 4) fence();
            if (MODE == kKeep) keep_state<X, DK>(a.S + at * DK * z.dvp, 2 * kb, z.dvp, 16 * tile, s, lane);
#pragma unroll
            for (int ti = 0; ti < 4; ++ti) {
                R[ti] = mma(tile8<X, L::kRow>(Ks, 16 * ti, 32 * kb, lane), s, R[ti]);
                if (MODE == kOut) O[ti] = mma(tile8<X, L::kRow>(Qs, 16 * ti, 32 * kb, lane), s, O[ti]);
            }
        }
        fence();
        // b (V - e^G K S)
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) {
            f32x4 v = zero4();
            if (MODE != kPre || !trans) v = vs.tile(ti, unit);
            const f32x4 g = *reinterpret_cast<const f32x4 *>(eG + 16 * ti + 4 * q), b = *reinterpret_cast<const f32x4 *>(beta + 16 * ti + 4 * q);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                R[ti][e] = b[e] != 0.f ? b[e] * (v[e] - g[e] * R[ti][e]) : 0.f;
                if (MODE == kOut) O[ti][e] *= z.scale * g[e];
            }
        }
        if (active && c + 1 < c1) take_columns(c + 1);
        fence();
        // U = T R = R + (T - I) R, and the outputs' M U
        f32x4 U[4];
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) U[ti] = R[ti];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const Split r = operand<Split>(R[2 * kb], R[2 * kb + 1]);
            if (sizeof(E) == 4) fence();
#pragma unroll
            for (int ti = 2 * kb; ti < 4; ++ti) U[ti] = mma(tile8s<Split, L::kTok>(Ts, 16 * ti, 32 * kb, lane), r, U[ti]);
        }
        if (MODE == kOut) {
            __syncthreads();
            if (!active) continue;
            E *out = static_cast<E *>(a.O) + (static_cast<int64_t>(bh) * z.N + t0) * z.dv;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const Split u = operand<Split>(U[2 * kb], U[2 * kb + 1]);
#pragma unroll
                for (int ti = 2 * kb; ti < 4; ++ti) O[ti] = mma(tile8s<Split, L::kTok>(Ms, 16 * ti, 32 * kb, lane), u, O[ti]);
                store_rows<X>(out, 32 * kb, n, z.dv, 16 * tile, O[2 * kb], O[2 * kb + 1], lane);
            }
        }
        if (MODE == kKeep) {
            float *keep = a.U + at * C * z.dvp;
#pragma unroll
            for (int ti = 0; ti < 4; ti += 2) keep_tokens<X>(keep, 16 * ti, z.dvp, 16 * tile, operand<Split>(U[ti], U[ti + 1]), lane);
        }
        fence();
        // the state behind the chunk
        const float whole = eG[C - 1];
#pragma unroll
        for (int t = 0; t < DK / 16; ++t) S[t] *= whole;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const f32x4 e0 = *reinterpret_cast<const f32x4 *>(eEnd + 32 * kb + 4 * q), e1 = *reinterpret_cast<const f32x4 *>(eEnd + 32 * kb + 16 + 4 * q);
            const Split u = operand<Split>(U[2 * kb] * e0, U[2 * kb + 1] * e1);
            if (sizeof(E) == 4) fence();
#pragma unroll
            for (int t = 0; t < DK / 16; ++t) S[t] = mma(tile8<X, L::kTok>(Kt, 16 * t, 32 * kb, lane), u, S[t]);
        }
    }
    if (!active) return;
    if (trans) {
        // P row by row; P^T: its columns, of which a lane holds eight rows that lie together
        float *P = a.P + (static_cast<size_t>(bh) * z.win_segs + seg) * DK * DK, *PT = a.PT + (static_cast<size_t>(bh) * z.nseg + z.seg0 + seg) * DK * DK;
        const int k0 = 16 * tile - z.dvp;
#pragma unroll
        for (int t = 0; t < DK / 16; t += 2) {
            const Split x = operand<Split>(S[t], S[t + 1]);
            if (a.PT) {
                f32x4 *to = reinterpret_cast<f32x4 *>(PT + transition_place<DK>(k0 + col, 16 * t + 8 * q));
                to[0] = S[t];
                to[1] = S[t + 1];
            }
#pragma unroll
            for (int b = 0; b < 2; ++b)
                *reinterpret_cast<f32x4 *>(P + transition_place<DK>(16 * t + 16 * b + col, k0 + 4 * q)) = mma(x, unit8<X, false>(b, lane), zero4());
        }
        return;
    }
    if (a.final_state && (MODE == kPre || seg == z.segs - 1))
        put_state(S, a.final_state + bh * a.final_head + (MODE == kPre ? static_cast<size_t>(seg) * z.dk * z.dv : 0), z.dk, z.dv, 0, vcol, lane);
}

// ------------------------------------------------------------------ states at the segments' starts
// S <- P_s S + B_s, segment after segment (REV: from the last to the first, with P_s^T).  One workgroup per head and 16 COLS columns, a
// wavefront per 16 rows; the new rows reach the other wavefronts as operands through LDS, one barrier a step (two buffers), and P and B are
// asked for two steps ahead (three: no faster).  A step takes 1.6 us all the same (dk = 64: 0.8), a chain of LDS, barrier and products one after the other, so many segments
// of few heads (joined_in_groups) are joined in groups of about the root of their number: the transitions of the groups side by side (compose), the groups one after the other,
// then the segments of all groups side by side.  64 transitions of four heads, dk = dv = 128, bf16: 59 us in the three launches, 106 one after the other.
struct CombineArgs {
    Sizes z;
    int heads, groups, each;        // transitions of a group: each; the last group's may be fewer
    int steps;                      // transitions in all: segments first, first + 1, .. of the window (REV: first, first - 1, ..)
    int first;
    const float *P, *add;           // P_s: image bh * p_head + s; B_s: add + (bh * add_head + s) * dk * dv
    size_t p_head, add_head;
    const float *carry;             // state to start from (null: zero): carry + bh * carry_head + group * carry_group
    size_t carry_head, carry_group;
    float *at;                      // states at the segments' starts (REV: cotangents at their ends): at + bh * at_head + s * dk * dv; null: not wanted
    size_t at_head;
    float *out_P;                   // compose: the groups' transitions and states from zero, image bh * out_head + group
    float *out_add;
    size_t out_head;
};

constexpr int kAheadSteps = 2;

template <class X, int DK, int COLS, bool REV>
__global__ __launch_bounds__(4 * DK) void delta_combine_kernel(CombineArgs a)
{
    typedef typename X::E E;
    typedef typename X::Split Split;
    __shared__ __attribute__((aligned(16))) E ops[2][COLS][X::kPlanes][DK / 32][64 * 8];
    const Sizes &z = a.z;
    // workgroups go to the eight XCDs in turn: those of one head and group to the same one, whose L2 then fetches P once
    const int vtiles = z.dvp / 16 / COLS, tiles = vtiles + (a.out_P ? DK / 16 / COLS : 0), slot = blockIdx.x >> 3, unit = slot / tiles * 8 + (blockIdx.x & 7);
    if (unit >= a.heads * a.groups) return;
    const int bh = unit / a.groups, group = unit - bh * a.groups, tile = slot % tiles;
    const int begin = group * a.each, end = min(begin + a.each, a.steps);
    const int wave = wave_index(), lane = threadIdx.x & 63, q = lane >> 4, col0 = 16 * COLS * tile + (lane & 15);
    const bool trans = tile >= vtiles;
    const size_t one = static_cast<size_t>(z.dk) * z.dv;
    auto segment = [&](int i) { return REV ? a.first - i : a.first + i; };
    struct Step {
        float P[DK / 32][8];
        f32x4 B[COLS];
    } ahead[kAheadSteps];
    f32x4 S[COLS];
#pragma unroll
    for (int n = 0; n < COLS; ++n) S[n] = zero4();
    auto get = [&](f32x4 (&to)[COLS], const float *state) {
#pragma unroll
        for (int n = 0; n < COLS; ++n) get_state(reinterpret_cast<f32x4 (&)[1]>(to[n]), state, z.dk, z.dv, wave, col0 + 16 * n, lane);
    };
    auto put_to = [&](float *state) {
#pragma unroll
        for (int n = 0; n < COLS; ++n) put_state(reinterpret_cast<f32x4 (&)[1]>(S[n]), state, z.dk, z.dv, wave, col0 + 16 * n, lane);
    };
    auto take = [&](int i, Step &to) {
        const float *p = a.P + (bh * a.p_head + segment(i)) * DK * DK + wave * (DK / 32) * kOperand + lane * 8;
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) kept8(p + kb * kOperand, to.P[kb]);
#pragma unroll
        for (int n = 0; n < COLS; ++n) to.B[n] = zero4();
        if (!trans) get(to.B, a.add + (bh * a.add_head + segment(i)) * one);
    };
    auto put = [&](int i) {
        if (a.at) put_to(a.at + bh * a.at_head + segment(i) * one);
    };
    auto step = [&](int i, Step &my, E (*op)[X::kPlanes][DK / 32][64 * 8]) {
        put(i);
        // the lane's four rows are half of its eight places in the operand of 32 rows
#pragma unroll
        for (int n = 0; n < COLS; ++n) put4(&op[n][0][wave >> 1][lane * 8 + 4 * (wave & 1)], DK / 32 * 64 * 8, S[n]);
        f32x4 sums[COLS][2];
#pragma unroll
        for (int n = 0; n < COLS; ++n) sums[n][0] = my.B[n], sums[n][1] = zero4();
        Split P[DK / 32];
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) split8(my.P[kb], P[kb]);
        __syncthreads();
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb)
#pragma unroll
            for (int n = 0; n < COLS; ++n) {
                Split s;
                get8(&op[n][0][kb][lane * 8], DK / 32 * 64 * 8, s);
                sums[n][kb & 1] = mma(P[kb], s, sums[n][kb & 1]);
            }
#pragma unroll
        for (int n = 0; n < COLS; ++n) S[n] = sums[n][0] + sums[n][1];
        if (i + kAheadSteps < end) take(i + kAheadSteps, my);
    };
    if (trans) {
#pragma unroll
        for (int n = 0; n < COLS; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) S[n][e] = state_row(wave, q, e) == col0 + 16 * n - z.dvp ? 1.f : 0.f;
    } else if (a.carry) {
        get(S, a.carry + bh * a.carry_head + group * a.carry_group);
    }
#pragma unroll
    for (int k = 0; k < kAheadSteps; ++k)
        if (begin + k < end) take(begin + k, ahead[k]);
    for (int i = begin; i < end; i += kAheadSteps)
#pragma unroll
        for (int k = 0; k < kAheadSteps; ++k)
            if (i + k < end) step(i + k, ahead[k], ops[(i + k) & 1]);
    if (a.out_P) {
        const size_t g = static_cast<size_t>(bh) * a.out_head + group;
        if (trans) {
            float *P = a.out_P + g * DK * DK;
#pragma unroll
            for (int n = 0; n < COLS; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) P[transition_place<DK>(state_row(wave, q, e), col0 + 16 * n - z.dvp)] = S[n][e];
        } else {
            put_to(a.out_add + g * one);
        }
    } else if (group == a.groups - 1) {
        put(a.steps);
    }
}

// ------------------------------------------------------------------ cotangents of the states, last chunk first
// The scan's mirror image: the same split of the work, as little saturated (matrix units busy 31 to 36 %, vector ALU 37 to 45 %, waiting 31 to 33 %, two wavefronts a SIMD, and more to
// stage and to write), 11.8 us a chunk with dV and what the gradients read (FULL: 96 KB a chunk), 8.5 us without, at dk = dv = 128, bf16.
struct RevArgs {
    Sizes z;
    const void *Q, *K, *dO;
    const float *TT, *MT, *dec;
    const float *end;               // cotangent at the end of a segment: end + bh * end_head + segment * dk * dv (segment from the window's first); null: zero
    size_t end_head;
    float *final_state;             // cotangent of the state before the window's first segment; without FULL: before every segment (null: not wanted)
    size_t final_head;
    int seg_skip;                   // without FULL: segments of the window passed over
    void *dV;
    float *dS, *dR;                 // FULL: cotangents at the chunks' ends, and dR, rows in spread order
};

template <class X, int DK, int THREADS, bool FULL>
__global__ __launch_bounds__(THREADS) void delta_rev_kernel(RevArgs a)
{
    typedef typename X::E E;
    typedef typename X::Split Split;
    typedef Lds<X, DK> L;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    E *Ks = reinterpret_cast<E *>(lds_raw), *Kt = Ks + L::kByTokens, *Qt = Kt + L::kByRows, *Ts = Qt + L::kByRows, *Ms = Ts + X::kPlanes * L::kSquare;
    float *dec = reinterpret_cast<float *>(Ms + X::kPlanes * L::kSquare);
    const Sizes &z = a.z;
    const int tid = threadIdx.x, wave = wave_index(), lane = tid & 63, q = lane >> 4;
    const int bh = blockIdx.z, seg = blockIdx.y + a.seg_skip;
    const int tile = blockIdx.x * (THREADS / 64) + wave, vcol = 16 * tile + (lane & 15);
    const bool active = tile < z.dvp / 16;
    const int c0 = (z.seg0 + seg) * z.seg_chunks - z.chunk0, c1 = min(c0 + z.seg_chunks, z.chunks);
    static_assert(THREADS >= 4 * DK, "a thread stages rows of K or of Q");
    const bool has_k = tid < 2 * DK, has_q = tid >= 2 * DK && tid < 4 * DK;
    const int task = has_k ? tid : tid - 2 * DK;

    f32x4 S[DK / 16];
#pragma unroll
    for (int t = 0; t < DK / 16; ++t) S[t] = zero4();
    if (a.end && active) get_state(S, a.end + bh * a.end_head + static_cast<size_t>(seg) * z.dk * z.dv, z.dk, z.dv, 0, vcol, lane);
    constexpr bool kAhead = sizeof(E) == 2;         // fp32 operands leave no registers for the images, at dk > 64 not for rows either
    constexpr bool kAheadRows = kAhead || DK <= 64;
    RowsStage<X, DK> rows;
    ImageStage<THREADS> is, ms;
    ColumnsStage<X> os;
    const typename X::Exact unit = ColumnsStage<X>::unit(z.dv, 16 * tile, lane);
    float ds = 0.f;
    auto take = [&](int c) {
        const int64_t t0 = static_cast<int64_t>(z.chunk0 + c) * C;
        const int n = tokens_of(z, z.chunk0 + c);
        const size_t at = static_cast<size_t>(bh) * z.chunks + c;
        if (kAheadRows && (has_k || has_q)) rows.take(static_cast<const E *>(has_k ? a.K : a.Q) + qk_row(z, bh, t0) * z.dk, n, z.dk, task);
        if (kAhead) {
            is.take(a.TT + at * C * C, tid);
            ms.take(a.MT + at * C * C, tid);
        }
        if (tid < 3 * C) ds = a.dec[at * kDec + tid];
    };
    auto take_columns = [&](int c) {
        const int64_t t0 = static_cast<int64_t>(z.chunk0 + c) * C;
        os.take(static_cast<const E *>(a.dO) + (static_cast<int64_t>(bh) * z.N + t0) * z.dv, tokens_of(z, z.chunk0 + c), z.dv, 16 * tile, lane);
    };
    if (c0 < c1) {
        take(c1 - 1);
        if (active) take_columns(c1 - 1);
    }
    for (int c = c1 - 1; c >= c0; --c) {
        const int64_t t0 = static_cast<int64_t>(z.chunk0 + c) * C;
        const int n = tokens_of(z, z.chunk0 + c);
        const size_t at = static_cast<size_t>(bh) * z.chunks + c;
        __syncthreads();
        if (!kAheadRows && (has_k || has_q)) rows.take(static_cast<const E *>(has_k ? a.K : a.Q) + qk_row(z, bh, t0) * z.dk, n, z.dk, task);
        if (has_k) rows.template put<true, true>(n, z.dk, Ks, Kt, task);
        if (has_q) rows.template put<false, true>(n, z.dk, nullptr, Qt, task);
        if (!kAhead) is.take(a.TT + at * C * C, tid);
        is.template put<X, Split>(Ts, tid);
        if (!kAhead) ms.take(a.MT + at * C * C, tid);
        ms.template put<X, Split>(Ms, tid);
        if (tid < 3 * C) dec[tid] = ds;
        __syncthreads();
        if (c > c0) take(c - 1);
        if (!active) continue;
        const float *eG = dec, *eEnd = dec + C, *beta = dec + 2 * C;
        f32x4 d[4];
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) d[ti] = os.tile(ti, unit);
        if (kAhead && c > c0) take_columns(c - 1);
        fence();
        // dU = M^T dO + e^{G_C - G} K dS
        f32x4 U[4];
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) U[ti] = zero4();
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) {
            const Split s = operand<Split>(S[2 * kb], S[2 * kb + 1]);
            if (sizeof(E) == 4) fence();
            if (FULL) keep_state<X, DK>(a.dS + at * DK * z.dvp, 2 * kb, z.dvp, 16 * tile, s, lane);
#pragma unroll
            for (int ti = 0; ti < 4; ++ti) U[ti] = mma(tile8<X, L::kRow>(Ks, 16 * ti, 32 * kb, lane), s, U[ti]);
        }
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) U[ti] *= *reinterpret_cast<const f32x4 *>(eEnd + 16 * ti + 4 * q);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const typename X::Exact o = rounded<X>(d[2 * kb], d[2 * kb + 1]);      // (exact: elements of dO)
#pragma unroll
            for (int ti = 0; ti < 2 * kb + 2; ++ti) U[ti] = mma(tile8s<Split, L::kTok>(Ms, 16 * ti, 32 * kb, lane), o, U[ti]);
        }
        auto strengths = [&](int ti) { return *reinterpret_cast<const f32x4 *>(beta + 16 * ti + 4 * q); };
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) {
            const f32x4 b = strengths(ti);
#pragma unroll
            for (int e = 0; e < 4; ++e) U[ti][e] = b[e] != 0.f ? U[ti][e] : idle(U[ti][e]);
        }
        fence();
        // dR = T^T dU = dU + (T^T - I) dU
        f32x4 R[4];
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) R[ti] = U[ti];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const Split u = operand<Split>(U[2 * kb], U[2 * kb + 1]);
            if (sizeof(E) == 4) fence();
#pragma unroll
            for (int ti = 0; ti < 2 * kb + 2; ++ti) R[ti] = mma(tile8s<Split, L::kTok>(Ts, 16 * ti, 32 * kb, lane), u, R[ti]);
        }
        if (FULL) {
            float *keep = a.dR + at * C * z.dvp;
            E *dV = static_cast<E *>(a.dV) + (static_cast<int64_t>(bh) * z.N + t0) * z.dv;
#pragma unroll
            for (int ti = 0; ti < 4; ti += 2) {
                keep_tokens<X>(keep, 16 * ti, z.dvp, 16 * tile, operand<Split>(R[ti], R[ti + 1]), lane);
                store_rows<X>(dV, 16 * ti, n, z.dv, 16 * tile, strengths(ti) * R[ti], strengths(ti + 1) * R[ti + 1], lane);
            }
        }
        fence();
        // the cotangent before the chunk
        const float whole = eG[C - 1];
#pragma unroll
        for (int t = 0; t < DK / 16; ++t) S[t] *= whole;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            f32x4 g[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) g[i] = *reinterpret_cast<const f32x4 *>(eG + 32 * kb + 16 * i + 4 * q);
            const Split o = operand<Split>(d[2 * kb] * (z.scale * g[0]), d[2 * kb + 1] * (z.scale * g[1]));
#pragma unroll
            for (int t = 0; t < DK / 16; ++t) S[t] = mma(tile8<X, L::kTok>(Qt, 16 * t, 32 * kb, lane), o, S[t]);
            if (FULL) fence();
            const Split r = operand<Split>(R[2 * kb] * (-strengths(2 * kb) * g[0]), R[2 * kb + 1] * (-strengths(2 * kb + 1) * g[1]));
#pragma unroll
            for (int t = 0; t < DK / 16; ++t) S[t] = mma(tile8<X, L::kTok>(Kt, 16 * t, 32 * kb, lane), r, S[t]);
            if (FULL) fence();
        }
        if (!kAhead && c > c0) take_columns(c - 1);
    }
    if (active && a.final_state && (!FULL || seg == 0))
        put_state(S, a.final_state + bh * a.final_head + (FULL ? 0 : static_cast<size_t>(seg) * z.dk * z.dv), z.dk, z.dv, 0, vcol, lane);
}

// ------------------------------------------------------------------ gradients of a chunk
struct GradArgs {
    Sizes z;
    const void *Q, *K, *V, *dO;
    const float *dec, *MT, *AT, *S, *U, *dS, *dR;
    void *dQ, *dK;                  // the caller's tensors, or with `shared` fp32 (BH, 64 chunks, dk) parts
    int shared;
    float *dg, *dbeta;
    int each;                       // chunks of a workgroup
};

// the elements of a caller's row at eight places of the spread order, from place p (a multiple of 8)
template <class X>
__device__ __forceinline__ typename X::Exact rows8_spread(const typename X::E *t, int row, int rows, int width, int p)
{
    const int k = (p & ~31) + ((p & 31) >> 1);
    return load8_spread(t + static_cast<int64_t>(row) * width + k, row < rows && k < width, row < rows && k + 16 < width);
}
// Sums over 16 lanes of N values a lane: afterwards lane l holds the sum of value l % N.  M lanes apart, half of the values are handed over at a time.  (A template
// and not a loop over M: the compiler left such a loop standing and chose each value by sixteen comparisons, half of the kernel's instructions.)
template <int M, int N>
__device__ __forceinline__ void fold_lanes(float (&v)[N], int lane)
{
    if constexpr (M >= N) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], M);
    } else {
        const bool up = lane & M;
#pragma unroll
        for (int k = 0; k < M; ++k) {
            const float keep = up ? v[k + M] : v[k], give = up ? v[k] : v[k + M];
            v[k] = keep + __shfl_xor(give, M);
        }
    }
    if constexpr (M > 1) fold_lanes<M / 2>(v, lane);
}
template <int N>
__device__ __forceinline__ float sum_lanes(float (&v)[N], int lane)
{
    fold_lanes<8>(v, lane);
    return v[0];
}
// within each 16 lanes: the value N lanes above (below with N < 0), zero beyond the ends; the sum over this lane and those above it; the sum over those below it
template <int N>
__device__ __forceinline__ float lanes_off(float x)
{
    constexpr int kRowShl = 0x100, kRowShr = 0x110;
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), N > 0 ? kRowShl + N : kRowShr - N, 0xf, 0xf, true));
}
__device__ __forceinline__ float suffix16(float x)
{
    x += lanes_off<1>(x);
    x += lanes_off<2>(x);
    x += lanes_off<4>(x);
    return x + lanes_off<8>(x);
}
__device__ __forceinline__ float prefix16(float x)
{
    x = lanes_off<-1>(x);
    x += lanes_off<-1>(x);
    x += lanes_off<-2>(x);
    x += lanes_off<-4>(x);
    return x + lanes_off<-8>(x);
}

// One workgroup of eight wavefronts per chunk.  U, dR and dO are read once, into LDS, as operands; a wavefront then has 16 columns of dQ and dK
// (and with dk <= 64 half of the tokens), for which it reads its rows of S and dS once, as right operands: dO S^T, dR S^T and U dS^T.  F and E are
// formed from the same tiles before these are overwritten with F, F^T and E + E^T, whose products with K and Q end the kernel.  A workgroup goes on to the
// chunk before it, whose states it has asked for by then.
// dg: W = M o (dO U^T) - A o (dR U^T) lies in the same 16 x 16 tiles as F and E, rows j in registers and columns i in lanes.  A tile's sums over i >= t are four
// steps over the lanes; below the diagonal they and the sums of its rows j are all that dg needs of it (kPairs), and one wavefront adds up a chunk's.
// 4096 chunks of dk = dv = 128, bf16: 425 us for 1.32 GB, 3.1 TB/s; matrix units busy 19 % of the time, vector ALU 34 %, LDS 35 %, waiting 31 %.  LDS holds one workgroup of
// a CU, which waits for its own reading at the chunk's start and for tiles in LDS after that.  (dR and dS as three
// bf16 and not two cost 12 % of the kernel, the sums for dg another 12.)
constexpr int kGradThreads = 512;

template <class X, int DK>
struct GradLds {
    typedef typename X::E E;
    typedef Lds<X, DK> L;
    static constexpr int kWide = 128 + X::kPad;                         // a token's row over columns of the state, in spread order
    static constexpr bool kHasO = sizeof(E) == 2;                       // dO has no room beside fp32 tiles: its operands come from memory
    static constexpr int kPairs = 20 * 32;                              // of a tile of W's two products: sums over i >= t and j, and over i for each j
    static constexpr int kFloats = kDec + kPairs + C + 8;               // decays and strengths, sums of W, v.dR, partial sums
    static constexpr int kDots = 3 * 8 * C;                             // p, s and k.X of eight wavefronts
    static constexpr int kTiles = C * kWide * (2 * X::kPlanes + (kHasO ? 1 : 0));
    static constexpr size_t kBytes = kFloats * sizeof(float) + sizeof(E) * (2 * L::kByRows + kTiles);
    static_assert(3 * X::kPlanes * L::kSquare * sizeof(E) + kDots * sizeof(float) <= kTiles * sizeof(E), "F, F^T, E + E^T and these sums lie where U, dR and dO were");
};

template <class X, int DK>
__global__ __launch_bounds__(kGradThreads) void delta_grad_kernel(GradArgs a)
{
    typedef typename X::E E;
    typedef typename X::Exact Exact;
    typedef typename X::Split Split;
    typedef Lds<X, DK> L;
    typedef GradLds<X, DK> G;
    constexpr int kWide = G::kWide, kTok = L::kTok, TI = DK / 32;       // TI: 16-token tiles of a wavefront
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    float *eG = reinterpret_cast<float *>(lds_raw), *eEnd = eG + C, *bs = eEnd + C, *hi_of = bs + C, *lo_of = hi_of + C, *pairs = lo_of + C, *vd = pairs + G::kPairs, *part = vd + C;
    E *Kt = reinterpret_cast<E *>(part + 8), *Qt = Kt + L::kByRows, *Us = Qt + L::kByRows, *Rs = Us + X::kPlanes * C * kWide, *Os = Rs + X::kPlanes * C * kWide;
    E *F = Us, *Ft = F + X::kPlanes * L::kSquare, *Es = Ft + X::kPlanes * L::kSquare;
    float *pd = reinterpret_cast<float *>(Es + X::kPlanes * L::kSquare), *sd = pd + 8 * C, *kd = sd + 8 * C;
    const Sizes &z = a.z;
    const int wave = wave_index();
    int tid = threadIdx.x;
    int lane = tid & 63, q = lane >> 4, col = lane & 15;
    const int bh = blockIdx.y, c_low = blockIdx.x * a.each, c_high = min(c_low + a.each, z.chunks);
    const int deep = z.dvp / 32;            // steps of a product over the state's columns
    int dcol = 16 * (wave % (DK / 16)) + col;
    const int ti0 = DK == 128 ? 0 : wave / (DK / 16) * TI;
    constexpr bool kNext = DK == 128;       // a tile's operands are asked for while the one before is multiplied; with dk <= 64 there are only two, and branches

    // what a chunk reads: asked for at once, and while the products of the chunk before are formed
    RowsStage<X, DK> rows;
    float u[2][8], r[2][8], s[4][8], d[4][8], decs = 0.f;
    f32x4 ma[3];                    // of M and A, what the wavefront's tiles of F and E are multiplied with
    Exact v[2], o[2];
    auto take_state = [&](const float *from, float (&to)[4][8]) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
            if (kb < deep) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(from + state_place(dcol >> 4, kb, half, deep) + 4 * lane);
#pragma unroll
                    for (int e = 0; e < 4; ++e) to[kb][4 * half + e] = x[e];
                }
            }
    };
    auto take = [&](int c) {
        const bool has_k = tid < 2 * DK, has_q = tid >= kGradThreads - 2 * DK;
        const int task = has_k ? tid : tid - (kGradThreads - 2 * DK), p0 = 8 * (tid & 15);          // 16 lanes a token, eight places each
        const int n = tokens_of(z, z.chunk0 + c);
        const int64_t t0 = static_cast<int64_t>(z.chunk0 + c) * C, row0 = static_cast<int64_t>(bh) * z.N + t0;
        const size_t at = static_cast<size_t>(bh) * z.chunks + c;
        if (has_k || has_q) rows.take(static_cast<const E *>(has_k ? a.K : a.Q) + qk_row(z, bh, t0) * z.dk, n, z.dk, task);
        if (tid < kDec) decs = a.dec[at * kDec + tid];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = (tid >> 4) + 32 * half;
#pragma unroll
            for (int e = 0; e < 8; ++e) u[half][e] = r[half][e] = 0.f;
            if (p0 < z.dvp) {
                kept8(a.U + (at * C + i) * z.dvp + p0, u[half]);
                kept8(a.dR + (at * C + i) * z.dvp + p0, r[half]);
            }
            v[half] = rows8_spread<X>(static_cast<const E *>(a.V) + row0 * z.dv, i, p0 < z.dvp ? n : 0, z.dv, p0);
            o[half] = rows8_spread<X>(static_cast<const E *>(a.dO) + row0 * z.dv, i, p0 < z.dvp ? n : 0, z.dv, p0);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int job = wave + 8 * k, t = job < 10 ? job : job - 10;
            if (job >= 20) continue;
            const int ti = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3, tj = t - ti * (ti + 1) / 2;
            const float *from = (job < 10 ? a.MT : a.AT) + at * C * C + (16 * tj + 4 * q) * C + spread(16 * ti + col);
#pragma unroll
            for (int e = 0; e < 4; ++e) ma[k][e] = from[e * C];
        }
    };
    auto take_states = [&](int c) {
        const size_t at = static_cast<size_t>(bh) * z.chunks + c;
        take_state(a.S + at * DK * z.dvp, s);
        take_state(a.dS + at * DK * z.dvp, d);
    };
    if (c_low < c_high) take_states(c_high - 1);
    for (int c = c_high - 1; c >= c_low; --c) {
        // (what follows from the lane is formed anew for each chunk, not kept in registers)
        asm volatile("" : "+v"(tid));
        lane = tid & 63, q = lane >> 4, col = lane & 15, dcol = 16 * (wave % (DK / 16)) + col;
        const int n = tokens_of(z, z.chunk0 + c);
        const int64_t t0 = static_cast<int64_t>(z.chunk0 + c) * C, row0 = static_cast<int64_t>(bh) * z.N + t0;
        const size_t at = static_cast<size_t>(bh) * z.chunks + c;
        const E *dO = static_cast<const E *>(a.dO) + row0 * z.dv;
        const bool has_k = tid < 2 * DK, has_q = tid >= kGradThreads - 2 * DK;
        const int task = has_k ? tid : tid - (kGradThreads - 2 * DK), p0 = 8 * (tid & 15);
        take(c);
        __syncthreads();                        // the chunk before is done with the tiles
        if (tid < kDec) eG[tid] = decs;
        if (has_k || has_q) rows.template put<false, true, false>(n, z.dk, nullptr, has_k ? Kt : Qt, task);
        __syncthreads();                        // the strengths
        const bool idle_tokens = __any(lane < n && bs[lane] == 0.f);
        // the tiles, and on the way u.dR and v.dR of every token; over the states <S, dS>
        float dot = 0.f;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
            if (kb < deep) {
#pragma unroll
                for (int e = 0; e < 8; ++e) dot += s[kb][e] * d[kb][e];
            }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = (tid >> 4) + 32 * half;
            fence();
            Split us, rs;
            split8(u[half], us);
            split8(r[half], rs);
            put8(Us + i * kWide + p0, C * kWide, us);
            put8(Rs + i * kWide + p0, C * kWide, rs);
            if (G::kHasO) put8(Os + i * kWide + p0, o[half]);
            float x[8], ud = 0.f, vr = 0.f;
            values8(v[half], x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ud += u[half][e] * r[half][e];
                vr += x[e] * r[half][e];
            }
#pragma unroll
            for (int m = 1; m < 16; m *= 2) {
                ud += __shfl_xor(ud, m);
                vr += __shfl_xor(vr, m);
            }
            if ((tid & 15) == 0) {
                vd[i] = vr;
                if (i < n && bs[i] != 0.f) a.dbeta[row0 + i] = ud / bs[i];
            }
        }
        __syncthreads();
        // rows of the left operands: 16 tokens of a tile, 32 places from p
        auto tokens_o = [&](int row, int p) -> Exact {
            if (G::kHasO) return get8(Os + (row + col) * kWide + p + 8 * q);
            return rows8_spread<X>(dO, row + col, n, z.dv, p + 8 * q);
        };

        fence();
        // F (jobs 0 .. 9) and E (10 .. 19): 16 x 16 tiles on and below the diagonal; rows j, columns i
        f32x4 jobs[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            jobs[k] = zero4();
            const int job = wave + 8 * k, t = job < 10 ? job : job - 10;
            if (job >= 20) continue;
            const int ti = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3, tj = t - ti * (ti + 1) / 2;
#pragma unroll 1
            for (int kb = 0; kb < deep; ++kb) {
                const int p = 32 * kb;
                if (job < 10) {
                    Split u;
                    get8(Us + (16 * tj + col) * kWide + p + 8 * q, C * kWide, u);
                    jobs[k] = mma(u, tokens_o(16 * ti, p), jobs[k]);
                } else {
                    Split u, r;
                    get8(Us + (16 * tj + col) * kWide + p + 8 * q, C * kWide, u);
                    get8(Rs + (16 * ti + col) * kWide + p + 8 * q, C * kWide, r);
                    jobs[k] = mma(u, r, jobs[k]);
                }
            }
            // the tile of W: sums over i' >= i, of them those over j < i and, below the diagonal, the whole rows j
            f32x4 w;
            float over_j = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = job < 10 ? ma[k][e] * jobs[k][e] : -ma[k][e] * jobs[k][e];
                w[e] = suffix16(ti > tj || 4 * q + e < col ? w[e] : 0.f);
                over_j += ti > tj || 4 * q + e < col ? w[e] : 0.f;
            }
            over_j += __shfl_xor(over_j, 16);
            over_j += __shfl_xor(over_j, 32);
            if (q == 0) pairs[32 * job + col] = over_j;
            if (col == 0) *reinterpret_cast<f32x4 *>(pairs + 32 * job + 16 + 4 * q) = w;
        }
        // dQ = scale e^G dO S^T, and of dK: e^{G_C - G} U dS^T - b e^G dR S^T (b = 0: X's part)
        f32x4 dq[TI], dk[TI], y[TI];
#pragma unroll
        for (int t = 0; t < TI; ++t) dq[t] = dk[t] = y[t] = zero4();
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            if (kb >= deep) continue;
            const int p = 32 * kb;
            fence();
            Split ss, ds;
            split8(s[kb], ss);
            split8(d[kb], ds);
            Split u[2], r[2];
            Exact o[2];
            auto get = [&](int t) {
                const int row = 16 * (ti0 + t);
                get8(Us + (row + col) * kWide + p + 8 * q, C * kWide, u[t & 1]);
                get8(Rs + (row + col) * kWide + p + 8 * q, C * kWide, r[t & 1]);
                o[t & 1] = tokens_o(row, p);
            };
            if (kNext) get(0);
#pragma unroll
            for (int t = 0; t < TI; ++t) {
                if (!kNext) get(t);
                else if (t + 1 < TI) get(t + 1);
                fence();
                dq[t] = mma(o[t & 1], ss, dq[t]);
                y[t] = mma(r[t & 1], ss, y[t]);
                dk[t] = mma(u[t & 1], ds, dk[t]);
                if (kNext) fence();
            }
        }
        if (ti0 > 0) dot = 0.f;         // with dk <= 64 two wavefronts have met the same rows
#pragma unroll
        for (int m = 1; m < 64; m *= 2) dot += __shfl_xor(dot, m);
        if (lane == 0) part[wave] = dot;
        // p, s (and further down k.X): sums over the wavefront's columns, of which a lane has one token's
        float ps[4 * TI], ss[4 * TI];
#pragma unroll
        for (int t = 0; t < TI; ++t) {
            const int i = 16 * (ti0 + t) + 4 * q;
            const f32x4 g = *reinterpret_cast<const f32x4 *>(eG + i), b = *reinterpret_cast<const f32x4 *>(bs + i);
            float xq[4], xk[4];
            get4(Qt + dcol * kTok + spread(i), xq);
            get4(Kt + dcol * kTok + spread(i), xk);
            dq[t] *= z.scale * g;
            dk[t] *= *reinterpret_cast<const f32x4 *>(eEnd + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float gy = g[e] * y[t][e];
                ps[4 * t + e] = xq[e] * dq[t][e] - xk[e] * (b[e] * gy);
                ss[4 * t + e] = xk[e] * dk[t][e];
                dk[t][e] -= (b[e] != 0.f ? b[e] : 1.f) * gy;
            }
        }
        const float p_sum = sum_lanes(ps, lane), s_sum = sum_lanes(ss, lane);
        const int sum_at = wave * C + 16 * (ti0 + (col % (4 * TI) >> 2)) + 4 * q + (col & 3);
        __syncthreads();
        // F, its transpose, and E + E^T (b = 0: the row of X, and nothing in E^T)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int job = wave + 8 * k, t = job < 10 ? job : job - 10;
            if (job >= 20) continue;
            const int ti = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3, tj = t - ti * (ti + 1) / 2;
            const int i = 16 * ti + col, j0 = 16 * tj + 4 * q;
            const float hi = hi_of[i], lo = lo_of[i];
            const f32x4 hj = *reinterpret_cast<const f32x4 *>(hi_of + j0), lj = *reinterpret_cast<const f32x4 *>(lo_of + j0);
            f32x4 D;
#pragma unroll
            for (int e = 0; e < 4; ++e) D[e] = decay(hi, lo, hj[e], lj[e]);
            if (job < 10) {
                const f32x4 f = z.scale * D * jobs[k];
                f32x4 f0;
#pragma unroll
                for (int e = 0; e < 4; ++e) f0[e] = j0 + e <= i ? f[e] : 0.f;
                put4(F + i * kTok + spread(j0), L::kSquare, f0);
#pragma unroll
                for (int e = 0; e < 4; ++e) put1(Ft + (j0 + e) * kTok + spread(i), L::kSquare, f0[e]);
            } else {
                const bool idle_i = bs[i] == 0.f;
                const f32x4 x = (idle_i ? -1.f : -bs[i]) * D * jobs[k];
                f32x4 x0;
#pragma unroll
                for (int e = 0; e < 4; ++e) x0[e] = j0 + e < i ? x[e] : 0.f;
                put4(Es + i * kTok + spread(j0), L::kSquare, x0);
                // after the rows: in a diagonal tile these places hold its zeros
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j0 + e < i) put1(Es + (j0 + e) * kTok + spread(i), L::kSquare, idle_i ? 0.f : x[e]);
            }
        }
        if (col < 4 * TI) pd[sum_at] = p_sum, sd[sum_at] = s_sum;
        fence();
        if (c > c_low) take_states(c - 1);
        fence();
        // what F and F^T have not: half of the steps of 32 tokens on the diagonal
        if (wave >= 4) {
            const int t = 2 * (wave & 1);
            E *to = wave < 6 ? F + (16 * t + col) * kTok + spread(16 * t + 16 + 4 * q) : Ft + (16 * t + 16 + col) * kTok + spread(16 * t + 4 * q);
            if (wave < 6) put4(to, L::kSquare, zero4());
            else put4(to, L::kSquare, zero4());
        }
        __syncthreads();
        // dQ += F K, dK += F^T Q + (E + E^T) K
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const int p = 32 * kb + 8 * q;
            const Exact k = get8(Kt + dcol * kTok + p), qq = get8(Qt + dcol * kTok + p);
            Split e[2], ft[2];
            Split f[2];
            auto get = [&](int t) {
                const int ti = ti0 + t, place = (16 * ti + col) * kTok + p;
                get8(Es + place, L::kSquare, e[t & 1]);
                if (ti >= 2 * kb) get8(F + place, L::kSquare, f[t & 1]);           // F is lower triangular
                if (ti < 2 * kb + 2) get8(Ft + place, L::kSquare, ft[t & 1]);
            };
            if (kNext) get(0);
#pragma unroll
            for (int t = 0; t < TI; ++t) {
                const int ti = ti0 + t;
                if (!kNext) get(t);
                else if (t + 1 < TI) get(t + 1);
                if (kNext) fence();
                dk[t] = mma(e[t & 1], k, dk[t]);
                if (ti >= 2 * kb) dq[t] = mma(f[t & 1], k, dq[t]);
                if (ti < 2 * kb + 2) dk[t] = mma(ft[t & 1], qq, dk[t]);
                if (kNext) fence();
            }
        }
        if (idle_tokens) {
            float ks[4 * TI];
#pragma unroll
            for (int t = 0; t < TI; ++t) {
                const int i = 16 * (ti0 + t) + 4 * q;
                const f32x4 b = *reinterpret_cast<const f32x4 *>(bs + i);
                float x[4];
                get4(Kt + dcol * kTok + spread(i), x);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ks[4 * t + e] = x[e] * dk[t][e];
                    dk[t][e] = b[e] != 0.f ? dk[t][e] : 0.f;
                }
            }
            const float k_sum = sum_lanes(ks, lane);
            if (col < 4 * TI) kd[sum_at] = k_sum;
        }
        const int d0 = dcol - col;
        if (a.shared) {
            const buffer_t outq = buffer(static_cast<float *>(a.dQ) + at * C * z.dk, static_cast<size_t>(C) * z.dk);
            const buffer_t outk = buffer(static_cast<float *>(a.dK) + at * C * z.dk, static_cast<size_t>(C) * z.dk);
#pragma unroll
            for (int t = 0; t < TI; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int to = state_offset(16 * (ti0 + t) + 4 * q + e, z.dk, dcol);
                    put_buffer(outq, to, dq[t][e]);
                    put_buffer(outk, to, dk[t][e]);
                }
        } else {
            E *outq = static_cast<E *>(a.dQ) + qk_row(z, bh, t0) * z.dk, *outk = static_cast<E *>(a.dK) + qk_row(z, bh, t0) * z.dk;
#pragma unroll
            for (int t = 0; t < TI; t += 2) {
                store_rows<X>(outq, 16 * (ti0 + t), n, z.dk, d0, dq[t], dq[t + 1], lane);
                store_rows<X>(outk, 16 * (ti0 + t), n, z.dk, d0, dk[t], dk[t + 1], lane);
            }
        }
        __syncthreads();
        if (wave == 0) {
            auto over_wavefronts = [&](const float *x) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < 8; ++w)
                    if (DK == 128 || w / (DK / 16) == lane / 32) s += x[w * C + lane];       // (with dk <= 64 a wavefront has half of the tokens)
                return s;
            };
            // across the token's tile of 16: from tiles before it, to tiles behind it, within it, and past the whole of it
            float sum = 0.f, rows_j = 0.f;
            const int x = lane >> 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int ti = max(x, k), tile = 32 * (ti * (ti + 1) / 2 + min(x, k));
                if (k <= x) sum += pairs[tile + col] + pairs[tile + 320 + col];
                else rows_j += pairs[tile + 16 + col] + pairs[tile + 336 + col];
            }
            sum += prefix16(rows_j);
            // (the first of a tile's sums over i' >= i is the whole tile's: of tiles 3 = (2, 0), 6 = (3, 0), 7 = (3, 1))
            const float past20 = pairs[96] + pairs[416], past30 = pairs[192] + pairs[512], past31 = pairs[224] + pairs[544];
            if (x == 1) sum += past20 + past30;
            if (x == 2) sum += past30 + past31;
            float tail = 0.f, p = over_wavefronts(pd), s = __shfl_up(over_wavefronts(sd), 1);
            s = lane > 0 ? s : 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) tail += part[w];
            // p of this token and those behind it, s of those before it
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const float y = __shfl_down(p, d), z = __shfl_up(s, d);
                if (lane + d < 64) p += y;
                if (lane >= d) s += z;
            }
            s += p + sum + eG[C - 1] * tail;
            if (lane < n && bs[lane] == 0.f) a.dbeta[row0 + lane] = vd[lane] + over_wavefronts(kd);
            if (lane < n) a.dg[row0 + lane] = s;
        }
    }
}

// dQ and dK of heads that value heads share: the parts in order
template <class X>
__global__ __launch_bounds__(256) void delta_shared_heads_kernel(Sizes z, int rows, const float *pq, const float *pk, void *dQ, void *dK)
{
    typedef typename X::E E;
    const int bhk = blockIdx.y, group = z.H / z.Hk;
    const int b = bhk / z.Hk, hk = bhk - b * z.Hk;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= static_cast<int64_t>(rows) * z.dk) return;
    const size_t head = static_cast<size_t>(z.chunks) * C * z.dk;
    const size_t from = (static_cast<size_t>(b) * z.H + static_cast<size_t>(hk) * group) * head + i;
    float q = 0.f, k = 0.f;
    for (int j = 0; j < group; ++j) {
        q += pq[from + j * head];
        k += pk[from + j * head];
    }
    const size_t to = (static_cast<size_t>(bhk) * z.N + static_cast<int64_t>(z.chunk0) * C) * z.dk + i;
    put1(static_cast<E *>(dQ) + to, q);
    put1(static_cast<E *>(dK) + to, k);
}

// ------------------------------------------------------------------ one token
// The state is read and written once and everything else is small.  A workgroup owns 32 columns of one head's state: 8 lanes of four
// columns by 32 groups of rows, four rows a lane (dk = 128), all held in registers between the two sums over rows.  Memory bounds it: 2048 states of
// 128 x 128 (268 MB read and written) take 45 us, 5.9 TB/s, above the 4.9 TB/s of a copy of 2 GiB because part of the states stays in the last-level cache.
// Four states take 4 us, which is one launch.
template <class E>
__global__ __launch_bounds__(256) void delta_step_kernel(Sizes z, const E *q, const E *k, const E *v, const float *g, const float *beta, float *state, E *o)
{
    __shared__ float ks[128], qs[128];
    __shared__ f32x4 sum[4][8];
    const int tid = threadIdx.x, bh = blockIdx.y, c4 = tid & 7, rg = tid >> 3;
    const int c0 = blockIdx.x * 32 + 4 * c4;
    const bool there = c0 < z.dv;
    const int64_t row = qk_row(z, bh, 0) * z.dk;
    float *S = state + static_cast<size_t>(bh) * z.dk * z.dv + c0;
    f32x4 s[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = rg + 32 * r;
        s[r] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (there && i < z.dk) s[r] = *reinterpret_cast<const f32x4_any4 *>(S + static_cast<size_t>(i) * z.dv);
    }
    if (tid < 128) {
        ks[tid] = tid < z.dk ? value(k[row + tid]) : 0.f;
        qs[tid] = tid < z.dk ? value(q[row + tid]) : 0.f;
    }
    const float a = expf(gate(g[bh])), b = strength(beta[bh]);
    __syncthreads();
    // sum over rows: the eight row groups of a wavefront, then the four wavefronts
    auto over_rows = [&](const float *w) {
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 4; ++r) t += s[r] * w[rg + 32 * r];
#pragma unroll
        for (int m = 8; m < 64; m *= 2)
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] += __shfl_xor(t[e], m);
        __syncthreads();
        if ((tid & 63) < 8) sum[tid >> 6][c4] = t;
        __syncthreads();
        return sum[0][c4] + sum[1][c4] + sum[2][c4] + sum[3][c4];
    };
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] *= a;
    f32x4 u = over_rows(ks);
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = there && b != 0.f ? b * (value(v[static_cast<size_t>(bh) * z.dv + c0 + e]) - u[e]) : 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = rg + 32 * r;
        s[r] += u * ks[i];
        if (there && i < z.dk) *reinterpret_cast<f32x4_any4 *>(S + static_cast<size_t>(i) * z.dv) = s[r];
    }
    const f32x4 out = over_rows(qs);
    if (there && rg == 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) put1(o + static_cast<size_t>(bh) * z.dv + c0 + e, z.scale * out[e]);
}

// ------------------------------------------------------------------ launches
template <class X, int DK>
constexpr size_t scan_lds(bool out)
{
    typedef Lds<X, DK> L;
    return sizeof(typename X::E) * (L::kByTokens + L::kByRows + X::kPlanes * L::kSquare + (out ? L::kByTokens + X::kPlanes * L::kSquare : 0)) + kDec * sizeof(float);
}
template <class X, int DK>
constexpr size_t rev_lds()
{
    typedef Lds<X, DK> L;
    return sizeof(typename X::E) * (L::kByTokens + 2 * L::kByRows + 2 * X::kPlanes * L::kSquare) + 3 * C * sizeof(float);
}
float *floats(char *ws, size_t at) { return reinterpret_cast<float *>(ws + at); }

Sizes sizes_of(const DeltaPlan &p)
{
    Sizes z{};
    z.N = p.N;
    z.H = p.H;
    z.Hk = p.Hk;
    z.dk = p.dk;
    z.dv = p.dv;
    z.dvp = p.dvp;
    z.scale = p.scale;
    z.seg_chunks = p.seg_chunks;
    z.nseg = p.nseg;
    z.win_segs = p.win_segs;
    return z;
}
void set_window(const DeltaPlan &p, int w, Sizes *z)
{
    z->seg0 = w * p.win_segs;
    z->segs = std::min(p.win_segs, p.nseg - z->seg0);
    z->chunk0 = z->seg0 * p.seg_chunks;
    z->chunks = std::min(z->segs * p.seg_chunks, p.chunks - z->chunk0);
}

#define DELTA_LAUNCH(name, kernel, grid, block, lds, st, ...)                                   \
    do {                                                                                        \
        ProfileScope scope(name, st);                                                           \
        if (hipError_t e = allow_lds(kernel, lds); e != hipSuccess) return e;                   \
        kernel<<<grid, block, lds, st>>>(__VA_ARGS__);                                          \
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;                        \
    } while (0)

template <class X, int DK, int THREADS>
struct Passes {
    static constexpr int kTiles = THREADS / 64;
    static hipError_t prep(const DeltaPlan &p, const Sizes &z, const DeltaIo &io, char *ws, bool bwd, hipStream_t st)
    {
        PrepArgs a{z, io.Q, io.K, io.g, io.beta, floats(ws, p.off_T), bwd ? floats(ws, p.off_MT) : nullptr, bwd ? floats(ws, p.off_TT) : nullptr,
                   bwd ? floats(ws, p.off_AT) : nullptr, floats(ws, p.off_dec)};
        const dim3 grid(z.chunks, p.BH);
        if (bwd) DELTA_LAUNCH("delta_prep_back", (delta_prep_kernel<X, DK, true>), grid, 256, 0, st, a);
        else DELTA_LAUNCH("delta_prep", (delta_prep_kernel<X, DK, false>), grid, 256, 0, st, a);
        return hipSuccess;
    }
    static ScanArgs scan_args(const DeltaPlan &p, const Sizes &z, const DeltaIo &io, char *ws)
    {
        ScanArgs a{};
        a.z = z;
        a.Q = io.Q;
        a.K = io.K;
        a.V = io.V;
        a.T = floats(ws, p.off_T);
        a.dec = floats(ws, p.off_dec);
        return a;
    }
    // transitions and states from zero of `segs` segments of the window
    static hipError_t pre(const DeltaPlan &p, const Sizes &z, const DeltaIo &io, char *ws, int segs, bool bwd, hipStream_t st)
    {
        if (segs <= 0) return hipSuccess;
        ScanArgs a = scan_args(p, z, io, ws);
        const size_t one = static_cast<size_t>(p.dk) * p.dv;
        a.final_state = floats(ws, p.off_add);
        a.final_head = one * p.win_segs;
        a.transitions = 1;
        a.P = floats(ws, p.off_P);
        a.PT = bwd ? floats(ws, p.off_PT) : nullptr;
        const dim3 grid((p.dvp / 16 + DK / 16 + kTiles - 1) / kTiles, segs, p.BH);
        DELTA_LAUNCH("delta_segments", (delta_scan_kernel<X, DK, THREADS, kPre>), grid, THREADS, (scan_lds<X, DK>(false)), st, a);
        return hipSuccess;
    }
    // states at the starts of the window's segments (rev: cotangents at their ends), `steps` transitions from the first (last) on
    static hipError_t combine(const DeltaPlan &p, const Sizes &z, const float *carry, size_t carry_head, char *ws, int steps, bool rev, hipStream_t st)
    {
        const size_t one = static_cast<size_t>(p.dk) * p.dv;
        CombineArgs a{};
        a.z = z;
        a.heads = p.BH;
        a.groups = 1;
        a.each = a.steps = steps;
        a.first = rev ? z.segs - 1 : 0;
        a.P = rev ? floats(ws, p.off_PT) + static_cast<size_t>(z.seg0) * DK * DK : floats(ws, p.off_P);
        a.p_head = rev ? p.nseg : p.win_segs;
        a.add = floats(ws, p.off_add);
        a.add_head = p.win_segs;
        a.carry = carry;
        a.carry_head = carry_head;
        a.at = rev ? floats(ws, p.off_end) : floats(ws, p.off_start) + z.seg0 * one;
        a.at_head = one * (rev ? p.win_segs : p.nseg + 1);
        if (joined_in_groups(steps, p.BH)) {
            const int each = (steps + p.join_groups - 1) / p.join_groups, groups = (steps + each - 1) / each;
            // the groups' transitions; the last group's is nobody's
            CombineArgs c = a;
            c.groups = groups;
            c.each = each;
            c.carry = nullptr;
            c.at = nullptr;
            c.out_P = floats(ws, p.off_group_P);
            c.out_add = floats(ws, p.off_group_add);
            c.out_head = p.join_groups;
            if (hipError_t e = launch_combine(c, rev, st); e != hipSuccess) return e;
            CombineArgs g = a;
            g.steps = g.each = groups - 1;
            g.first = 0;
            g.P = c.out_P;
            g.p_head = g.add_head = p.join_groups;
            g.add = c.out_add;
            g.at = floats(ws, p.off_group_start);
            g.at_head = one * p.join_groups;
            if (hipError_t e = launch_combine(g, false, st); e != hipSuccess) return e;
            a.groups = groups;
            a.each = each;
            a.carry = g.at;
            a.carry_head = g.at_head;
            a.carry_group = one;
        }
        return launch_combine(a, rev, st);
    }
    static hipError_t launch_combine(const CombineArgs &a, bool rev, hipStream_t st)
    {
        // one chain of steps: as few columns as there are workgroups for; several side by side: P read half as often
        return a.groups == 1 && !a.out_P ? launch_columns<1>(a, rev, st) : launch_columns<2>(a, rev, st);
    }
    template <int COLS>
    static hipError_t launch_columns(const CombineArgs &a, bool rev, hipStream_t st)
    {
        const int tiles = (a.z.dvp / 16 + (a.out_P ? DK / 16 : 0)) / COLS, grid = (a.heads * a.groups + 7) / 8 * 8 * tiles;
        if (rev) DELTA_LAUNCH("delta_join", (delta_combine_kernel<X, DK, COLS, true>), grid, 4 * DK, 0, st, a);
        else DELTA_LAUNCH("delta_join", (delta_combine_kernel<X, DK, COLS, false>), grid, 4 * DK, 0, st, a);
        return hipSuccess;
    }

    static hipError_t forward(const DeltaPlan &p, const DeltaIo &io, char *ws, hipStream_t st)
    {
        Sizes z = sizes_of(p);
        const size_t one = static_cast<size_t>(p.dk) * p.dv;
        const float *carry = io.state_in;
        float *kept = floats(ws, p.off_carry);
        for (int w = 0; w < p.windows; ++w) {
            set_window(p, w, &z);
            if (hipError_t e = prep(p, z, io, ws, false, st); e != hipSuccess) return e;
            ScanArgs a = scan_args(p, z, io, ws);
            a.O = io.O;
            a.start = carry;
            a.start_head = one;
            if (z.segs > 1) {
                if (hipError_t e = pre(p, z, io, ws, z.segs - 1, false, st); e != hipSuccess) return e;
                if (hipError_t e = combine(p, z, carry, one, ws, z.segs - 1, false, st); e != hipSuccess) return e;
                a.start = floats(ws, p.off_start) + z.seg0 * one;
                a.start_head = one * (p.nseg + 1);
            }
            a.final_state = w + 1 < p.windows ? kept : io.state_out;
            a.final_head = one;
            carry = kept;
            const dim3 grid((p.dvp / 16 + kTiles - 1) / kTiles, z.segs, p.BH);
            DELTA_LAUNCH("delta_scan", (delta_scan_kernel<X, DK, THREADS, kOut>), grid, THREADS, (scan_lds<X, DK>(true)), st, a);
        }
        return hipSuccess;
    }

    static hipError_t backward(const DeltaPlan &p, const DeltaIo &io, char *ws, hipStream_t st)
    {
        Sizes z = sizes_of(p);
        const size_t one = static_cast<size_t>(p.dk) * p.dv;
        float *start = floats(ws, p.off_start);
        const bool joined = p.win_segs > 1;
        // states at the segments' starts.  What the way back needs of a window's chunks is formed here for the last one alone, whose images stay.
        const float *carry = io.state_in;
        for (int w = 0; w < p.windows; ++w) {
            set_window(p, w, &z);
            if (hipError_t e = prep(p, z, io, ws, w + 1 == p.windows, st); e != hipSuccess) return e;
            if (joined) {
                if (hipError_t e = pre(p, z, io, ws, z.segs, true, st); e != hipSuccess) return e;
                // the windows' starts follow one another in `start`, so the next window's carry is read there
                if (hipError_t e = combine(p, z, w == 0 ? io.state_in : start + z.seg0 * one, w == 0 ? one : one * (p.nseg + 1), ws, z.segs, false, st); e != hipSuccess)
                    return e;
            } else {
                ScanArgs a = scan_args(p, z, io, ws);
                a.start = carry;
                a.start_head = w == 0 ? one : one * (p.nseg + 1);
                a.final_state = start + (w + 1) * one;
                a.final_head = one * (p.nseg + 1);
                carry = a.final_state;
                if (w + 1 < p.windows) {
                    const dim3 grid((p.dvp / 16 + kTiles - 1) / kTiles, 1, p.BH);
                    DELTA_LAUNCH("delta_states", (delta_scan_kernel<X, DK, THREADS, kPre>), grid, THREADS, (scan_lds<X, DK>(false)), st, a);
                }
            }
        }
        const float *dcarry = io.dstate_out;
        float *kept = floats(ws, p.off_carry);
        for (int w = p.windows - 1; w >= 0; --w) {
            set_window(p, w, &z);
            if (w != p.windows - 1)
                if (hipError_t e = prep(p, z, io, ws, true, st); e != hipSuccess) return e;
            {
                ScanArgs a = scan_args(p, z, io, ws);
                const bool own_start = joined || w > 0;
                a.start = own_start ? start + z.seg0 * one : io.state_in;
                a.start_head = own_start ? one * (p.nseg + 1) : one;
                a.S = floats(ws, p.off_S);
                a.U = floats(ws, p.off_U);
                const dim3 grid((p.dvp / 16 + kTiles - 1) / kTiles, z.segs, p.BH);
                DELTA_LAUNCH("delta_states", (delta_scan_kernel<X, DK, THREADS, kKeep>), grid, THREADS, (scan_lds<X, DK>(false)), st, a);
            }
            RevArgs r{};
            r.z = z;
            r.Q = io.Q;
            r.K = io.K;
            r.dO = io.dO;
            r.TT = floats(ws, p.off_TT);
            r.MT = floats(ws, p.off_MT);
            r.dec = floats(ws, p.off_dec);
            RevArgs full = r;
            full.end = dcarry;
            full.end_head = one;
            if (z.segs > 1) {
                r.final_state = floats(ws, p.off_add);
                r.final_head = one * p.win_segs;
                r.seg_skip = 1;
                const dim3 grid((p.dvp / 16 + kTiles - 1) / kTiles, z.segs - 1, p.BH);
                DELTA_LAUNCH("delta_segments_back", (delta_rev_kernel<X, DK, THREADS, false>), grid, THREADS, (rev_lds<X, DK>()), st, r);
                if (hipError_t e = combine(p, z, dcarry, one, ws, z.segs - 1, true, st); e != hipSuccess) return e;
                full.end = floats(ws, p.off_end);
                full.end_head = one * p.win_segs;
            }
            full.final_state = w > 0 ? kept : io.dstate_in;
            full.final_head = one;
            full.dV = io.dV;
            full.dS = floats(ws, p.off_dS);
            full.dR = floats(ws, p.off_dR);
            dcarry = kept;
            {
                const dim3 grid((p.dvp / 16 + kTiles - 1) / kTiles, z.segs, p.BH);
                DELTA_LAUNCH("delta_scan_back", (delta_rev_kernel<X, DK, THREADS, true>), grid, THREADS, (rev_lds<X, DK>()), st, full);
            }
            const float *a_S = floats(ws, p.off_S), *a_U = floats(ws, p.off_U);
            const bool shared = p.H != p.Hk;
            GradArgs g{z, io.Q, io.K, io.V, io.dO, r.dec, r.MT, floats(ws, p.off_AT), a_S, a_U, full.dS, full.dR,
                       shared ? ws + p.off_pq : io.dQ, shared ? ws + p.off_pk : io.dK, shared ? 1 : 0, io.dg, io.dbeta,
                       std::max(1, (z.chunks * p.BH + 255) / 256)};
            DELTA_LAUNCH("delta_gradients", (delta_grad_kernel<X, DK>), dim3((z.chunks + g.each - 1) / g.each, p.BH), kGradThreads, (GradLds<X, DK>::kBytes), st, g);
            if (shared) {
                const int rows = static_cast<int>(std::min<int64_t>(static_cast<int64_t>(z.chunks) * C, p.N - static_cast<int64_t>(z.chunk0) * C));
                const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(rows) * p.dk + 255) / 256), p.BH / p.H * p.Hk);
                DELTA_LAUNCH("delta_shared_heads", (delta_shared_heads_kernel<X>), grid, 256, 0, st, z, rows, floats(ws, p.off_pq),
                             floats(ws, p.off_pk), io.dQ, io.dK);
            }
        }
        return hipSuccess;
    }
};

// Eight wavefronts, also where four would hold all columns of the state and the others only stage rows and images; fp32 takes four then.  Training, 64 x 64, us with eight /
// with four:  bf16, 4 heads x 65536 tokens: 910 / 939 (a prompt: 199 / 214), 32 x 8192: 804 / 848;  fp32, 32 x 8192: 1400 / 1393, 8 x 2003: 240 / 230.
template <class X, class F>
hipError_t for_width(const DeltaPlan &p, F f)
{
    if (p.dk > 64) return f(Passes<X, 128, 512>());
    if constexpr (sizeof(typename X::E) == 4)
        if (p.dvp <= 64) return f(Passes<X, 64, 256>());
    return f(Passes<X, 64, 512>());
}
template <class F>
hipError_t for_shape(const DeltaPlan &p, F f) { return p.dtype == RACE_BF16 ? for_width<Bf>(p, f) : for_width<Fp>(p, f); }

__global__ __launch_bounds__(256) void delta_copy_state_kernel(const float *from, float *to, size_t n)
{
    const size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i < n) to[i] = from ? from[i] : 0.f;
}

}  // namespace

hipError_t forward(const DeltaPlan &p, const DeltaIo &io, char *ws, hipStream_t st)
{
    return for_shape(p, [&](auto passes) { return passes.forward(p, io, ws, st); });
}
hipError_t backward(const DeltaPlan &p, const DeltaIo &io, char *ws, hipStream_t st)
{
    return for_shape(p, [&](auto passes) { return passes.backward(p, io, ws, st); });
}
hipError_t copy_state(const DeltaPlan &p, const float *from, float *to, hipStream_t st)
{
    if (from == to) return hipSuccess;
    const size_t n = static_cast<size_t>(p.BH) * p.dk * p.dv;
    delta_copy_state_kernel<<<static_cast<unsigned>((n + 255) / 256), 256, 0, st>>>(from, to, n);
    return hipGetLastError();
}
hipError_t step(const DeltaPlan &p, const DeltaIo &io, hipStream_t st)
{
    Sizes z = sizes_of(p);
    z.N = 1;
    const dim3 grid(p.dvp / 32, p.BH);
    if (p.dtype == RACE_BF16)
        DELTA_LAUNCH("delta_step", delta_step_kernel<uint16_t>, grid, 256, 0, st, z, static_cast<const uint16_t *>(io.Q), static_cast<const uint16_t *>(io.K),
                     static_cast<const uint16_t *>(io.V), io.g, io.beta, io.state_out, static_cast<uint16_t *>(io.O));
    else
        DELTA_LAUNCH("delta_step", delta_step_kernel<float>, grid, 256, 0, st, z, static_cast<const float *>(io.Q), static_cast<const float *>(io.K),
                     static_cast<const float *>(io.V), io.g, io.beta, io.state_out, static_cast<float *>(io.O));
    return hipSuccess;
}

}  // namespace delta
}  // namespace race
