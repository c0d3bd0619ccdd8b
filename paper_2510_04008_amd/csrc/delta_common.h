// What the kernels of the gated delta rule share: operands of the matrix instructions for both element types, the layouts of
// tiles in LDS and in the workspace, and the arguments of the kernels.
//
// Mathematics.  Per value head, with decay a_t = exp(g_t) and write strength b_t,
//     S_t = a_t S_{t-1} + k_t u_t^T,   u_t = b_t (v_t - a_t S_{t-1}^T k_t),   o_t = scale S_t^T q_t.
// A chunk of C = 64 tokens that starts from S, with G_i the running sum of g inside the chunk and D_ij = exp(G_i - G_j), is
//     (I + A) U = b (V - e^G K S),  A_ij = b_i D_ij k_i.k_j (j < i):   U = T b (V - e^G K S),  T = (I + A)^-1
//     O = scale e^G Q S + M U,      M_ij = scale D_ij q_i.k_j (j <= i)
//     S' = e^{G_C} S + (e^{G_C - G} K)^T U.
// T, M and the decays of all chunks are formed at once (prep); only the products with S are one after the other.  S' is affine
// in S, so a long sequence is cut into segments whose transition P and state from zero B are formed side by side (pre-pass),
// joined (combine), and the pass proper then runs over all segments at once from their true states.
//
// Gradients, with dS the cotangent of the state behind the chunk:
//     dU = M^T dO + e^{G_C - G} K dS,   dR = T^T dU,   dV = b dR,   dS' = e^{G_C} dS + (scale e^G Q)^T dO - (b e^G K)^T dR
//     F_ij = scale D_ij dO_i.u_j (j <= i),   E_ij = -b_i D_ij dR_i.u_j (j < i)
//     dQ = F K + scale e^G dO S^T
//     dK = F^T Q + (E + E^T) K + e^{G_C - G} U dS^T - b e^G dR S^T
//     db_i = u_i.dR_i / b_i
//     dg_t = sum_{j < t <= i} W_ij + sum_{i >= t} p_i + sum_{j < t} s_j + e^{G_C} <S, dS>,   over the chunk, with
//         W_ij = M_ij dO_i.u_j - A_ij dR_i.u_j,   p_i = q_i.(scale e^{G_i} S dO_i) - k_i.(b_i e^{G_i} S dR_i),   s_j = k_j.(e^{G_C - G_j} dS u_j)
// The last: e^{g_t} is a factor of what passes t and of nothing else, from a token before it (or the chunk's start) to one at or behind it (or the chunk's
// end).  Every term of the sum holds that factor, so dg_t keeps its digits however small it is.  (The cotangent of G_i is q_i.dQ_i - v_i.dV_i, and dg
// its sum from the end; but both of these hold terms without any decay, and with g = -8 their difference has lost 3 of 7 digits.)
// Tokens of strength zero (padding; |b| below 2^-100 counts as that) write nothing, whatever finite values their rows hold: their rows of A and of
// b (V - e^G K S) are zeros, not products with zero.  db divides by b; for them it is v_i.dR_i + k_i.X_i with
//     X_i = -sum_j D_ij (dR_i.u_j) k_j - e^{G_i} S dR_i,
// which is their row of (E K - b e^G dR S^T) for b = 1, and not part of dK.  dR_i hangs on their keys alone; what these make of A's and M's columns and
// of dR is kept within 2^60, so that it stays finite where it meets a zero.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace race {
namespace delta {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
// a caller's rows need be aligned to their elements only; global memory takes wide accesses at any address
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t u32x4_any2;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any4;

constexpr int C = 64;               // tokens per chunk
constexpr int kDec = 5 * C;         // decays and strengths of a chunk
constexpr float kBetaFloor = 0x1p-100f, kIdleMax = 0x1p60f;
constexpr float kGateFloor = -1e5f; // log decays below act as this one: exp is 0 either way, and -infinity would make differences NaN

// Element types.  The passes over the states multiply 16 x 16 tiles, 32 deep: lane l holds row (of a left operand) or column (of a right one)
// l % 16 and, with q = l / 16, eight of the 32 k: 8 q + 0..7 ("natural") or 16 a + 4 q + r, a = 0, 1, r = 0..3 ("spread": the rows of two
// accumulators that lie on top of one another, so that a product's result is the next product's operand without leaving the registers).  Any
// order will do, as long as both operands have it; tiles and images whose rows run over tokens or over columns of the state are stored in spread order.
// K K^T and Q K^T of prep are 32 x 32 tiles, 16 deep, half as many operands to a product: lane l holds row l % 32 and the elements 8 h + 0..7, h = l / 32.
//
// bf16: the elements of Q, K, V and dO are exact as they are.  Values that are fp32 by their nature enter as
// sums of three bf16 (Split: all 24 bits) in every product.  Two (2^-16) would do for outputs that are rounded to bf16 at the end, were there no cancellation in them; but
// a value that overwrites a thousand times larger one is read back as the difference of the two.
// fp32: eight fp32 matrix instructions a product, one for each of a lane's k.
struct Bf {
    typedef uint16_t E;
    typedef bf16x8 Exact;
    struct Split { bf16x8 hi, mid, lo; };
    static constexpr int kPlanes = 3;       // of E for a value kept as a Split
    static constexpr int kPad = 8;          // elements behind a row of a tile in LDS: 16 bytes, so that 8 rows lie in 8 places
};
struct Fp {
    typedef float E;
    struct Exact { float v[8]; };
    typedef Exact Split;
    static constexpr int kPlanes = 1;
    static constexpr int kPad = 4;
};

// The wavefront's number as a scalar.  Branches on it have to be scalar branches: matrix instructions do not look at EXEC, and
// in a region that the compiler takes for divergent they are also run by wavefronts that have no lane in it.
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6)); }

__device__ __forceinline__ f32x16 zero16()
{
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}

__device__ __forceinline__ f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
// the smallest terms first; terms below 2^-24 of the product are left out
template <class A> __device__ __forceinline__ A mma(const Bf::Exact &a, const Bf::Exact &b, A c) { return mfma(a, b, c); }
template <class A> __device__ __forceinline__ A mma(const Bf::Exact &a, const Bf::Split &b, A c) { return mfma(a, b.hi, mfma(a, b.mid, mfma(a, b.lo, c))); }
template <class A> __device__ __forceinline__ A mma(const Bf::Split &a, const Bf::Exact &b, A c) { return mfma(a.hi, b, mfma(a.mid, b, mfma(a.lo, b, c))); }
template <class A> __device__ __forceinline__ A mma(const Bf::Split &a, const Bf::Split &b, A c)
{
    return mfma(a.hi, b.hi, mfma(a.hi, b.mid, mfma(a.mid, b.hi, mfma(a.mid, b.mid, mfma(a.hi, b.lo, mfma(a.lo, b.hi, c))))));
}
__device__ __forceinline__ f32x4 mma(const Fp::Exact &a, const Fp::Exact &b, f32x4 c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x16 mma(const Fp::Exact &a, const Fp::Exact &b, f32x16 c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}

// 8 fp32 values as an operand: pairs, so that two values take one conversion
__device__ __forceinline__ uint32_t round2(float a, float b)
{
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
__device__ __forceinline__ float low2(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high2(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ void split8(const float *x, Bf::Split &s)
{
    u32x4 hi, mid, lo;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float a = x[2 * j], b = x[2 * j + 1];
        hi[j] = round2(a, b);
        a -= low2(hi[j]);
        b -= high2(hi[j]);
        mid[j] = round2(a, b);
        lo[j] = round2(a - low2(mid[j]), b - high2(mid[j]));
    }
    s = Bf::Split{__builtin_bit_cast(bf16x8, hi), __builtin_bit_cast(bf16x8, mid), __builtin_bit_cast(bf16x8, lo)};
}
__device__ __forceinline__ void split8(const float *x, Fp::Exact &s)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) s.v[j] = x[j];
}
__device__ __forceinline__ void round8(const float *x, Bf::Exact &s)
{
    s = __builtin_bit_cast(bf16x8, u32x4{round2(x[0], x[1]), round2(x[2], x[3]), round2(x[4], x[5]), round2(x[6], x[7])});
}
__device__ __forceinline__ void round8(const float *x, Fp::Exact &s) { split8(x, s); }

// an operand from / to 8 elements that lie together, 16-byte aligned (LDS, workspace)
__device__ __forceinline__ Bf::Exact get8(const uint16_t *p) { return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p)); }
__device__ __forceinline__ Fp::Exact get8(const float *p)
{
    const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
    return Fp::Exact{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
__device__ __forceinline__ void put8(uint16_t *p, const Bf::Exact &x) { *reinterpret_cast<u32x4 *>(p) = __builtin_bit_cast(u32x4, x); }
__device__ __forceinline__ void put8(float *p, const Fp::Exact &x)
{
    reinterpret_cast<f32x4 *>(p)[0] = f32x4{x.v[0], x.v[1], x.v[2], x.v[3]};
    reinterpret_cast<f32x4 *>(p)[1] = f32x4{x.v[4], x.v[5], x.v[6], x.v[7]};
}
// a Split lies in planes that are `plane` elements apart
__device__ __forceinline__ void get8(const uint16_t *p, int plane, Bf::Split &x) { x = Bf::Split{get8(p), get8(p + plane), get8(p + 2 * plane)}; }
__device__ __forceinline__ void get8(const float *p, int, Fp::Exact &x) { x = get8(p); }
__device__ __forceinline__ void put8(uint16_t *p, int plane, const Bf::Split &x) { put8(p, x.hi); put8(p + plane, x.mid); put8(p + 2 * plane, x.lo); }
__device__ __forceinline__ void put8(float *p, int, const Fp::Exact &x) { put8(p, x); }

// four fp32 values into planes, and four elements
__device__ __forceinline__ void put4(uint16_t *p, int plane, const f32x4 &x)
{
    u32x2 hi, mid, lo;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        float a = x[2 * j], b = x[2 * j + 1];
        hi[j] = round2(a, b);
        a -= low2(hi[j]);
        b -= high2(hi[j]);
        mid[j] = round2(a, b);
        lo[j] = round2(a - low2(mid[j]), b - high2(mid[j]));
    }
    *reinterpret_cast<u32x2 *>(p) = hi;
    *reinterpret_cast<u32x2 *>(p + plane) = mid;
    *reinterpret_cast<u32x2 *>(p + 2 * plane) = lo;
}
__device__ __forceinline__ void put4(float *p, int, const f32x4 &x) { *reinterpret_cast<f32x4 *>(p) = x; }
__device__ __forceinline__ void get4(const uint16_t *p, float *x)
{
    const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
#pragma unroll
    for (int j = 0; j < 2; ++j) x[2 * j] = low2(w[j]), x[2 * j + 1] = high2(w[j]);
}
__device__ __forceinline__ void get4(const float *p, float *x)
{
    const f32x4 w = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = w[j];
}

// one value
__device__ __forceinline__ float value(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ void put1(uint16_t *p, float x) { *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }
__device__ __forceinline__ void put1(float *p, float x) { *p = x; }
__device__ __forceinline__ void put1(uint16_t *p, int plane, float x)
{
    const uint32_t hi = round2(x, 0.f), mid = round2(x - low2(hi), 0.f);
    p[0] = static_cast<uint16_t>(hi);
    p[plane] = static_cast<uint16_t>(mid);
    p[2 * plane] = static_cast<uint16_t>(round2(x - low2(hi) - low2(mid), 0.f));
}
__device__ __forceinline__ void put1(float *p, int, float x) { *p = x; }
__device__ __forceinline__ void values8(const Bf::Exact &x, float *f)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = static_cast<float>(x[j]);
}
__device__ __forceinline__ void values8(const Fp::Exact &x, float *f)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = x.v[j];
}

// 8 elements of a caller's row; zeros where there is none
__device__ __forceinline__ Bf::Exact load8(const uint16_t *p, bool there)
{
    u32x4 v = {0, 0, 0, 0};
    if (there) v = *reinterpret_cast<const u32x4_any2 *>(p);
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ Fp::Exact load8(const float *p, bool there)
{
    Fp::Exact x = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
    if (there) {
        const f32x4 a = reinterpret_cast<const f32x4_any4 *>(p)[0], b = reinterpret_cast<const f32x4_any4 *>(p)[1];
        x = Fp::Exact{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
    }
    return x;
}

// The unit matrix as a right operand, its row 16 b + n in column n (16 columns, natural or spread).  A product with it turns an
// operand whose lanes hold rows into an accumulator whose lanes hold columns, exactly (every value times one, plus zeros): rows that lie together in memory become
// accumulators, and accumulators rows that are stored 8 or 16 bytes at a time, without a way through LDS.
template <class X, bool SPREAD>
__device__ __forceinline__ typename X::Exact unit8(int b, int lane)
{
    float x[8];
    typename X::Exact u;
    if (sizeof(u) == 32) asm volatile("" : "+v"(lane));     // fp32: made anew each time, not kept in registers
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int q = lane >> 4, k = SPREAD ? 16 * (j >> 2) + 4 * q + (j & 3) : 8 * q + j;
        x[j] = k - 16 * b == (lane & 15) ? 1.f : 0.f;
    }
    round8(x, u);
    return u;
}

// fp32 values at 4-byte aligned addresses; out of range (an offset of kNowhere too): zero, and not written
typedef __amdgpu_buffer_rsrc_t buffer_t;
constexpr int kNowhere = -2147483647 - 1;
__device__ __forceinline__ buffer_t buffer(const float *p, size_t floats)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(p), 0, static_cast<int>(floats * sizeof(float)), 0x00020000);
}
__device__ __forceinline__ float get_buffer(buffer_t b, int offset) { return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, offset, 0, 0)); }
__device__ __forceinline__ void put_buffer(buffer_t b, int offset, float x) { __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), b, offset, 0, 0); }

__device__ __forceinline__ void put_buffer(buffer_t b, int offset, const f32x4 &x) { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), b, offset, 0, 0); }

// four elements of a caller's row
__device__ __forceinline__ void store4(uint16_t *p, const float *x)
{
    typedef __attribute__((ext_vector_type(2), aligned(2))) uint32_t u32x2_any2;
    *reinterpret_cast<u32x2_any2 *>(p) = u32x2_any2{round2(x[0], x[1]), round2(x[2], x[3])};
}
__device__ __forceinline__ void store4(float *p, const float *x) { *reinterpret_cast<f32x4_any4 *>(p) = f32x4_any4{x[0], x[1], x[2], x[3]}; }

// 8 elements of a caller's row of which a lane takes two runs of four, 16 elements apart (spread order)
__device__ __forceinline__ Bf::Exact load8_spread(const uint16_t *p, bool first, bool second)
{
    typedef __attribute__((ext_vector_type(2), aligned(2))) uint32_t u32x2_any2;
    u32x2 a = {0, 0}, b = {0, 0};
    if (first) a = *reinterpret_cast<const u32x2_any2 *>(p);
    if (second) b = *reinterpret_cast<const u32x2_any2 *>(p + 16);
    return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
}
__device__ __forceinline__ Fp::Exact load8_spread(const float *p, bool first, bool second)
{
    f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = {0.f, 0.f, 0.f, 0.f};
    if (first) a = *reinterpret_cast<const f32x4_any4 *>(p);
    if (second) b = *reinterpret_cast<const f32x4_any4 *>(p + 16);
    return Fp::Exact{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}

__device__ __forceinline__ Bf::Exact or_zero(const Bf::Exact &x, bool there)
{
    u32x4 v = __builtin_bit_cast(u32x4, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = there ? v[i] : 0;
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ Fp::Exact or_zero(const Fp::Exact &x, bool there)
{
    Fp::Exact y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y.v[i] = there ? x.v[i] : 0.f;
    return y;
}

// place of k within a row that is stored in spread order; of the quad of k that begins at 16 a + 4 q of a group of 32
__device__ __forceinline__ int spread(int k) { return (k & ~31) | ((k & 12) << 1) | ((k & 16) >> 2) | (k & 3); }
// row of accumulator register i (32 x 32), within the tile
__device__ __forceinline__ int acc_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

__device__ __forceinline__ float gate(float g) { return g < kGateFloor ? kGateFloor : g; }       // NaN stays
__device__ __forceinline__ float strength(float b) { return fabsf(b) < kBetaFloor ? 0.f : b; }       // NaN stays
// what hangs on the rows of a token of strength zero
__device__ __forceinline__ float idle(float x) { return fminf(fmaxf(x, -kIdleMax), kIdleMax); }

// exp(G_i - G_j) of sums that are held as two floats each: their difference is exact to fp32 however large they are
__device__ __forceinline__ float decay(float hi_i, float lo_i, float hi_j, float lo_j)
{
    return __builtin_amdgcn_exp2f(((hi_i - hi_j) + (lo_i - lo_j)) * 1.44269504088896f);
}

// running sum over the 64 lanes
__device__ __forceinline__ double prefix64(double x, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

}  // namespace delta
}  // namespace race
