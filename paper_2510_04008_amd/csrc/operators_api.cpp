// Host side of the gated delta rule and of the rows of queries and keys: argument checks, the plan of segments and windows, the workspace.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>

#include "delta_plan.h"
#include "internal.h"
#include "rotary_plan.h"

namespace race {
namespace {

using delta::joined_in_groups;

constexpr int kChunk = 64;
constexpr int kMaxHeads = 65535;            // B H: a grid dimension
constexpr int64_t kMaxTokens = int64_t(1) << 36;       // of all sequences and heads (rows of queries and keys: of a sequence)

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

race_status_t check_workspace(const void *ws, size_t bytes, size_t need)
{
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || bytes < need) return RACE_ERR_WORKSPACE;
    return RACE_OK;
}

// ---------------------------------------------------------------- gated delta rule
// What a window's chunks may take of the workspace.  A window holds a segment of every head at least, so a caller's segment length, or more heads than this holds
// chunks of, take more.
constexpr size_t kWindowBytes = size_t(4) << 30;

race_status_t check_delta(const race_delta_desc_t *d)
{
    if (!d || d->B < 1 || d->H < 1 || d->Hk < 1 || d->N < 0 || d->dk < 1 || d->dv < 1 || d->chunk < 0 || !std::isfinite(d->scale)) return RACE_ERR_INVALID_ARG;
    if ((d->dtype != RACE_F32 && d->dtype != RACE_BF16) || d->H % d->Hk != 0) return RACE_ERR_INVALID_ARG;
    if (d->dk % 8 || d->dv % 8 || d->dk > 128 || d->dv > 128) return RACE_ERR_UNSUPPORTED;
    const int64_t heads = static_cast<int64_t>(d->B) * d->H;
    if (heads > kMaxHeads || d->N > kMaxTokens / heads) return RACE_ERR_UNSUPPORTED;
    return RACE_OK;
}

// Segments that run side by side, by the time of a forward pass, in us, at dk = dv = 128, bf16: a chunk takes 7.9 in the pass proper, with a workgroup per segment and
// head, and 4.3 in the pre-pass, with two; the CUs hold 256 workgroups at once; the join takes 5 + 1.6 a segment one after the other, 30 + 0.45 in groups.
// Sweeps of training steps and prompts over 1 to 128 segments, us, the rule's choice first:  training, 4 heads x 65536 tokens: 64 segments 1584, 47: 1792, 74 (a
// second round): 1996;  16 x 10007, 64 x 128: 16: 799, 14: 810, 32: 823;  4 x 8192, fp32: 64: 671, 32: 766, 128: 875;  8 x 2003, 64 x 64, fp32: 16: 220, 8: 294, 32: 227.
// Prompts, 4 x 30011: 59: 249, 47: 247;  8 x 16384, 128 x 64: 32: 215, 24: 234, 43: 251;  32 x 8192: 8: 350, 6: 403, 13: 359;  64 x 4096: 4: 320, 3: 321;  128 x 2048:
// 2: 296, 1: 276.
int choose_segments(int chunks, int BH)
{
    int best = 1;
    double cost = 7.9 * chunks;
    for (int n = 2; n <= 256 / BH && n <= chunks; ++n) {
        const int m = (chunks + n - 1) / n, rounds = (2 * (n - 1) * BH + 255) / 256;
        const double c = (7.9 + 4.3 * rounds) * m + (joined_in_groups(n - 1, BH) ? 30.0 + 0.45 * n : 5.0 + 1.6 * n) + 12.0;
        if (c < cost) {
            cost = c;
            best = n;
        }
    }
    return best;
}

race_status_t plan_delta(const race_delta_desc_t *d, bool backward, delta::DeltaPlan *pl)
{
    if (race_status_t s = check_delta(d); s != RACE_OK) return s;
    delta::DeltaPlan p{};
    p.B = d->B;
    p.H = d->H;
    p.Hk = d->Hk;
    p.BH = d->B * d->H;
    p.dk = d->dk;
    p.dv = d->dv;
    p.dvp = (d->dv + 31) / 32 * 32;
    p.dtype = d->dtype;
    p.N = d->N;
    p.scale = d->scale;
    p.chunks = static_cast<int>((d->N + kChunk - 1) / kChunk);
    if (p.chunks == 0) {
        *pl = p;
        return RACE_OK;
    }
    const size_t dkp = d->dk <= 64 ? 64 : 128, one = sizeof(float) * p.dk * p.dv, square = kChunk * kChunk;
    const size_t per_chunk = square * 4 + 5 * kChunk * 4 + (backward ? square * 12 + 8 * p.dvp * (dkp + kChunk) + (p.H != p.Hk ? 8 * kChunk * p.dk : 0) : 0);
    const int window = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(p.chunks, kWindowBytes / (per_chunk * p.BH))));
    if (d->chunk > 0) {
        p.seg_chunks = static_cast<int>((std::min(d->chunk, d->N) + kChunk - 1) / kChunk);
        p.win_segs = std::max(1, window < p.chunks ? window / p.seg_chunks : (p.chunks + p.seg_chunks - 1) / p.seg_chunks);
    } else {
        p.win_segs = choose_segments(window, p.BH);
        p.seg_chunks = (window + p.win_segs - 1) / p.win_segs;
    }
    p.nseg = (p.chunks + p.seg_chunks - 1) / p.seg_chunks;
    p.win_segs = std::min({p.win_segs, p.nseg, 65535});
    p.windows = (p.nseg + p.win_segs - 1) / p.win_segs;

    const size_t n = static_cast<size_t>(p.BH) * std::min<int64_t>(static_cast<int64_t>(p.win_segs) * p.seg_chunks, p.chunks);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += align256(bytes);
        return was;
    };
    p.off_T = take(n * square * 4);
    p.off_dec = take(n * 5 * kChunk * sizeof(float));
    const size_t segs = static_cast<size_t>(p.BH) * p.win_segs;
    if (p.win_segs > 1) {
        p.off_add = take(segs * one);
        p.off_P = take(segs * dkp * dkp * 4);
    }
    if (joined_in_groups(p.win_segs, p.BH)) {
        p.join_groups = static_cast<int>(std::lround(std::sqrt(static_cast<double>(p.win_segs))));
        p.off_group_P = take(static_cast<size_t>(p.BH) * p.join_groups * dkp * dkp * 4);
        p.off_group_add = take(static_cast<size_t>(p.BH) * p.join_groups * one);
        p.off_group_start = take(static_cast<size_t>(p.BH) * p.join_groups * one);
    }
    if (p.nseg > 1) p.off_start = take(static_cast<size_t>(p.BH) * (p.nseg + 1) * one);
    if (p.windows > 1) p.off_carry = take(p.BH * one);
    if (backward) {
        if (p.win_segs > 1) {
            p.off_PT = take(static_cast<size_t>(p.BH) * p.nseg * dkp * dkp * 4);
            p.off_end = take(segs * one);
        }
        p.off_MT = take(n * square * 4);
        p.off_TT = take(n * square * 4);
        p.off_AT = take(n * square * 4);
        p.off_S = take(n * dkp * p.dvp * 4);
        p.off_U = take(n * kChunk * p.dvp * 4);
        p.off_dS = take(n * dkp * p.dvp * 4);
        p.off_dR = take(n * kChunk * p.dvp * 4);
        if (p.H != p.Hk) {
            p.off_pq = take(n * kChunk * p.dk * 4);
            p.off_pk = take(n * kChunk * p.dk * 4);
        }
    }
    p.total = at;
    *pl = p;
    return RACE_OK;
}

// ---------------------------------------------------------------- rows of queries and keys
race_status_t plan_rotary(const race_rotary_desc_t *d, rotary::RotaryPlan *pl)
{
    if (!d || d->B < 1 || d->Hq < 1 || d->Hk < 0 || d->N < 0 || d->d < 1 || d->rot < 0 || d->rot % 2 || d->rot > d->d) return RACE_ERR_INVALID_ARG;
    if (d->norm < RACE_NORM_NONE || d->norm > RACE_NORM_L2 || (d->neighbours != 0 && d->neighbours != 1) || !(d->eps >= 0.f) || std::isinf(d->eps))
        return RACE_ERR_INVALID_ARG;
    if (d->dtype != RACE_F32 && d->dtype != RACE_BF16) return RACE_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (d->q_strides[i] < 0 || d->k_strides[i] < 0 || d->dq_strides[i] < 0 || d->dk_strides[i] < 0) return RACE_ERR_INVALID_ARG;
    if (d->d % 8 || d->d > 256 || d->N > kMaxTokens || static_cast<int64_t>(d->Hq) + d->Hk > 65535) return RACE_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(d->B) * d->N > (int64_t(1) << 31)) return RACE_ERR_UNSUPPORTED;
    rotary::RotaryPlan p{};
    p.B = d->B;
    p.d = d->d;
    p.rot = d->rot;
    p.norm = d->norm;
    p.neighbours = d->neighbours;
    p.dtype = d->dtype;
    p.N = d->N;
    p.pos0 = d->pos0;
    p.eps = d->eps;
    p.q.heads = d->Hq;
    p.k.heads = d->Hk;
    p.q.batch = d->q_strides[0], p.q.token = d->q_strides[1], p.q.head = d->q_strides[2];
    p.k.batch = d->k_strides[0], p.k.token = d->k_strides[1], p.k.head = d->k_strides[2];
    p.q.dbatch = d->dq_strides[0], p.q.dtoken = d->dq_strides[1], p.q.dhead = d->dq_strides[2];
    p.k.dbatch = d->dk_strides[0], p.k.dtoken = d->dk_strides[1], p.k.dhead = d->dk_strides[2];
    *pl = p;
    return RACE_OK;
}

struct Axis { int64_t n, stride; };
// whether the last row, if there are any, ends within the bytes that 64 bits can count
bool rows_in_range(const race_rotary_desc_t *d, int heads, const int64_t *s)
{
    if (heads == 0) return true;
    int64_t reach = d->d, step;
    for (const Axis &a : {Axis{d->B, s[0]}, Axis{d->N, s[1]}, Axis{heads, s[2]}})
        if (a.n > 1 && (__builtin_mul_overflow(a.n - 1, a.stride, &step) || __builtin_add_overflow(reach, step, &reach))) return false;
    return reach <= INT64_MAX / static_cast<int64_t>(sizeof(float));
}
// rows (in range) that would be written over one another
bool rows_overlap(const race_rotary_desc_t *d, int heads, const int64_t *s)
{
    Axis axes[3] = {{d->B, s[0]}, {d->N, s[1]}, {heads, s[2]}};
    std::sort(axes, axes + 3, [](const Axis &a, const Axis &b) { return a.stride < b.stride; });
    int64_t reach = d->d;                   // elements from a row's first to behind the last that the axes so far can lead to
    for (const Axis &a : axes)
        if (a.n > 1) {
            if (a.stride < reach) return true;
            reach += (a.n - 1) * a.stride;
        }
    return false;
}

race_status_t read_turns(const race_rotary_desc_t *d, const double *inv_freq, const int64_t *positions, rotary::RotaryPlan *p)
{
    if (!positions && d->pos0 > INT64_MAX - d->N) return RACE_ERR_INVALID_ARG;
    if (d->rot > 0 && !inv_freq) return RACE_ERR_INVALID_ARG;
    for (int i = 0; i < d->rot / 2; ++i) {
        if (!std::isfinite(inv_freq[i])) return RACE_ERR_INVALID_ARG;
        p->turns[i] = inv_freq[i] / (2.0 * 3.14159265358979323846);
    }
    return RACE_OK;
}

}  // namespace
}  // namespace race

using namespace race;

extern "C" {

size_t race_delta_workspace_bytes(const race_delta_desc_t *desc)
{
    delta::DeltaPlan p;
    return plan_delta(desc, false, &p) == RACE_OK ? p.total : 0;
}

size_t race_delta_bwd_workspace_bytes(const race_delta_desc_t *desc)
{
    delta::DeltaPlan p;
    return plan_delta(desc, true, &p) == RACE_OK ? p.total : 0;
}

size_t race_delta_state_bytes(const race_delta_desc_t *desc)
{
    if (!desc) return 0;
    race_delta_desc_t one = *desc;
    one.N = 1;                              // the state does not depend on the context length
    one.chunk = 0;
    if (check_delta(&one) != RACE_OK) return 0;
    return sizeof(float) * one.B * one.H * one.dk * one.dv;
}

int64_t race_delta_segment_tokens(const race_delta_desc_t *desc)
{
    delta::DeltaPlan p;
    if (plan_delta(desc, false, &p) != RACE_OK) return 0;
    return static_cast<int64_t>(p.seg_chunks) * kChunk;
}

race_status_t race_delta_fwd(const race_delta_desc_t *desc, const void *Q, const void *K, const void *V, const float *g, const float *beta,
                             const float *state_in, void *O, float *state_out, void *workspace, size_t workspace_bytes, race_stream_t stream)
{
    delta::DeltaPlan p;
    race_status_t s = plan_delta(desc, false, &p);
    if (s != RACE_OK) return s;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (p.N == 0) {
        hipError_t e = state_out ? delta::copy_state(p, state_in, state_out, st) : hipSuccess;
        return e == hipSuccess ? RACE_OK : hip_failed(e, "race_delta_fwd launch");
    }
    if (!Q || !K || !V || !g || !beta || !O) return RACE_ERR_INVALID_ARG;
    if (any_equal({O}, {Q, K, V, g, beta, state_in, O, state_out})) return RACE_ERR_INVALID_ARG;
    if (state_out && any_equal({state_out}, {Q, K, V, g, beta, O, state_out})) return RACE_ERR_INVALID_ARG;
    if ((s = check_workspace(workspace, workspace_bytes, p.total)) != RACE_OK) return s;
    delta::DeltaIo io{};
    io.Q = Q;
    io.K = K;
    io.V = V;
    io.g = g;
    io.beta = beta;
    io.state_in = state_in;
    io.O = O;
    io.state_out = state_out;
    hipError_t e = delta::forward(p, io, static_cast<char *>(workspace), st);
    return e == hipSuccess ? RACE_OK : hip_failed(e, "race_delta_fwd launch");
}

race_status_t race_delta_bwd(const race_delta_desc_t *desc, const void *Q, const void *K, const void *V, const float *g, const float *beta,
                             const float *state_in, const void *dO, const float *dstate_out, void *dQ, void *dK, void *dV, float *dg, float *dbeta,
                             float *dstate_in, void *workspace, size_t workspace_bytes, race_stream_t stream)
{
    delta::DeltaPlan p;
    race_status_t s = plan_delta(desc, true, &p);
    if (s != RACE_OK) return s;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (p.N == 0) {
        hipError_t e = dstate_in ? delta::copy_state(p, dstate_out, dstate_in, st) : hipSuccess;
        return e == hipSuccess ? RACE_OK : hip_failed(e, "race_delta_bwd launch");
    }
    if (!Q || !K || !V || !g || !beta || !dO || !dQ || !dK || !dV || !dg || !dbeta) return RACE_ERR_INVALID_ARG;
    if (any_equal({dQ, dK, dV, dg, dbeta}, {Q, K, V, g, beta, state_in, dO, dstate_out, dQ, dK, dV, dg, dbeta, dstate_in})) return RACE_ERR_INVALID_ARG;
    if (dstate_in && any_equal({dstate_in}, {Q, K, V, g, beta, state_in, dO, dQ, dK, dV, dg, dbeta, dstate_in})) return RACE_ERR_INVALID_ARG;
    if ((s = check_workspace(workspace, workspace_bytes, p.total)) != RACE_OK) return s;
    delta::DeltaIo io{};
    io.Q = Q;
    io.K = K;
    io.V = V;
    io.g = g;
    io.beta = beta;
    io.state_in = state_in;
    io.dO = dO;
    io.dstate_out = dstate_out;
    io.dQ = dQ;
    io.dK = dK;
    io.dV = dV;
    io.dg = dg;
    io.dbeta = dbeta;
    io.dstate_in = dstate_in;
    hipError_t e = delta::backward(p, io, static_cast<char *>(workspace), st);
    return e == hipSuccess ? RACE_OK : hip_failed(e, "race_delta_bwd launch");
}

race_status_t race_delta_step(const race_delta_desc_t *desc, const void *q, const void *k, const void *v, const float *g, const float *beta,
                              float *state, void *o, race_stream_t stream)
{
    if (!desc) return RACE_ERR_INVALID_ARG;
    race_delta_desc_t one = *desc;
    one.N = 1;
    one.chunk = 0;
    delta::DeltaPlan p;
    race_status_t s = plan_delta(&one, false, &p);
    if (s != RACE_OK) return s;
    if (!q || !k || !v || !g || !beta || !state || !o) return RACE_ERR_INVALID_ARG;
    if (any_equal({state, o}, {q, k, v, g, beta, state, o})) return RACE_ERR_INVALID_ARG;
    delta::DeltaIo io{};
    io.Q = q;
    io.K = k;
    io.V = v;
    io.g = g;
    io.beta = beta;
    io.state_out = state;
    io.O = o;
    hipError_t e = delta::step(p, io, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? RACE_OK : hip_failed(e, "race_delta_step launch");
}

size_t race_qk_rotary_workspace_bytes(const race_rotary_desc_t *desc)
{
    rotary::RotaryPlan p;
    if (plan_rotary(desc, &p) != RACE_OK || p.N == 0) return 0;
    return rotary::workspace_bytes(p);
}

race_status_t race_qk_rotary_fwd(const race_rotary_desc_t *desc, const void *q, const void *k, const float *wq, const float *wk, const double *inv_freq,
                                 const int64_t *positions, void *Q, void *K, race_stream_t stream)
{
    rotary::RotaryPlan p;
    race_status_t s = plan_rotary(desc, &p);
    if (s != RACE_OK) return s;
    if (p.N == 0) return RACE_OK;           // nothing to do, pointers may be null
    if (!q || !Q || (p.k.heads > 0 && (!k || !K))) return RACE_ERR_INVALID_ARG;
    if (!rows_in_range(desc, desc->Hq, desc->q_strides) || !rows_in_range(desc, desc->Hk, desc->k_strides)) return RACE_ERR_INVALID_ARG;
    if ((s = read_turns(desc, inv_freq, positions, &p)) != RACE_OK) return s;
    if (any_equal({Q}, {q, k, wq, wk, positions, Q, K}) || (p.k.heads > 0 && any_equal({K}, {q, k, wq, wk, positions, Q, K}))) return RACE_ERR_INVALID_ARG;
    p.positions = positions;
    p.q.x = q, p.q.w = wq, p.q.y = Q;
    p.k.x = k, p.k.w = wk, p.k.y = K;
    hipError_t e = rotary::forward(p, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? RACE_OK : hip_failed(e, "race_qk_rotary_fwd launch");
}

race_status_t race_qk_rotary_bwd(const race_rotary_desc_t *desc, const void *q, const void *k, const float *wq, const float *wk, const double *inv_freq,
                                 const int64_t *positions, const void *dQ, const void *dK, void *dq, void *dk, float *dwq, float *dwk, void *workspace,
                                 size_t workspace_bytes, race_stream_t stream)
{
    rotary::RotaryPlan p;
    race_status_t s = plan_rotary(desc, &p);
    if (s != RACE_OK) return s;
    const bool keys = p.k.heads > 0;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (!rows_in_range(desc, desc->Hq, desc->q_strides) || !rows_in_range(desc, desc->Hk, desc->k_strides)) return RACE_ERR_INVALID_ARG;
    if (!rows_in_range(desc, desc->Hq, desc->dq_strides) || !rows_in_range(desc, desc->Hk, desc->dk_strides)) return RACE_ERR_INVALID_ARG;
    if (rows_overlap(desc, desc->Hq, desc->dq_strides) || (keys && rows_overlap(desc, desc->Hk, desc->dk_strides))) return RACE_ERR_INVALID_ARG;
    if (p.N == 0) {                         // no rows, other pointers may be null; the sums over them are zero
        hipError_t e = dwq ? zero_floats(dwq, p.d, st) : hipSuccess;
        if (e == hipSuccess && dwk && keys) e = zero_floats(dwk, p.d, st);
        return e == hipSuccess ? RACE_OK : hip_failed(e, "race_qk_rotary_bwd launch");
    }
    if (!q || !dQ || !dq || (keys && (!k || !dK || !dk)) || (!keys && dwk)) return RACE_ERR_INVALID_ARG;
    if ((s = read_turns(desc, inv_freq, positions, &p)) != RACE_OK) return s;
    if (any_equal({dq}, {q, k, wq, wk, positions, dQ, dK, dq, dk, dwq, dwk}) || (keys && any_equal({dk}, {q, k, wq, wk, positions, dQ, dK, dq, dk, dwq, dwk})))
        return RACE_ERR_INVALID_ARG;
    if ((dwq && any_equal({dwq}, {q, k, wq, wk, positions, dQ, dK, dq, dk, dwq, dwk})) ||
        (dwk && any_equal({dwk}, {q, k, wq, wk, positions, dQ, dK, dq, dk, dwq, dwk})))
        return RACE_ERR_INVALID_ARG;
    if ((dwq || dwk) && (s = check_workspace(workspace, workspace_bytes, rotary::workspace_bytes(p))) != RACE_OK) return s;
    p.positions = positions;
    p.q.x = q, p.q.w = wq, p.q.y = const_cast<void *>(dQ), p.q.dx = dq;
    p.k.x = k, p.k.w = wk, p.k.y = const_cast<void *>(dK), p.k.dx = dk;
    hipError_t e = rotary::backward(p, dwq, dwk, static_cast<char *>(workspace), st);
    return e == hipSuccess ? RACE_OK : hip_failed(e, "race_qk_rotary_bwd launch");
}

}  // extern "C"
