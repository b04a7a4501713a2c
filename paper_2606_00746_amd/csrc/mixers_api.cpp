// C ABI of the token mixers beside the scan: the norm of query and key heads
// with the position rotation, windowed attention, and the gated delta rule.
// Argument checks (host only, before any HIP call), workspaces, launches.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/gspn.h"
#include "attn.hpp"
#include "call_args.hpp"
#include "delta.hpp"
#include "launch.hpp"
#include "qk_norm.hpp"

namespace gspn {

template <>
struct requires_reserve<DeltaProblem> : std::true_type {};

namespace {

// Positions stay below 2^30, so that a position and a window add up in 32 bits.
constexpr int64_t kMostTokens = (int64_t)1 << 28;
constexpr int kMostWindow = 1 << 30;

int check_sizes(int64_t B, int64_t T, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D, int most, int dtype)
{
    if (dtype != GSPN_F32 && dtype != GSPN_BF16)
        return GSPN_ERR_DTYPE;
    if (B < 1 || T < 1 || Tk < 1 || Hq < 1 || Hkv < 1 || D < 1)
        return GSPN_ERR_DIM;
    if (D % 8 != 0 || D > most || T > kMostTokens || Tk > kMostTokens || B > kMostTokens || Hq > 65536 || Hkv > 65536 ||
        B * Hq > kMostTokens || B * Hkv > kMostTokens || T > GSPN_MAX_ELEMS / (B * Hq) / D ||
        Tk > GSPN_MAX_ELEMS / (B * Hkv) / D)
        return GSPN_ERR_UNSUPPORTED;
    return GSPN_OK;
}

// Sizes, window and scale of an attention call.
int make_attn(AttnProblem &p, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left, int right, int sinks, int offset,
              float scale, int dtype)
{
    const int st = check_sizes(B, Tq, Tk, Hq, Hkv, D, kAttnMaxHead, dtype);
    if (st != GSPN_OK)
        return st;
    if (Hq % Hkv != 0 || sinks < 0 || offset < 0 || !(scale > 0.f) || !isfinite(scale))
        return GSPN_ERR_DIM;
    if (offset > kMostTokens)
        return GSPN_ERR_UNSUPPORTED;
    p = AttnProblem{};
    p.B = B, p.Tq = Tq, p.Tk = Tk, p.Hq = Hq, p.Hkv = Hkv, p.D = D;
    p.left = left < 0 ? -1 : std::min(left, kMostWindow);
    p.right = right < 0 ? -1 : std::min(right, kMostWindow);
    p.sinks = std::min(sinks, Tk);
    p.offset = offset;
    p.scale = scale;
    p.dtype = dtype;
    return GSPN_OK;
}

const int64_t *at(const int64_t *strides, int i) { return strides ? strides + 3 * i : nullptr; }

int make_norm(NormProblem &p, int B, int T, int Hq, int Hk, int D, int R, int rows, int first, int pairs, float eps,
              int dtype, bool table, bool positions)
{
    const int st = check_sizes(B, T, 1, Hq, Hk, D, kNormMaxHead, dtype);
    if (st != GSPN_OK)
        return st;
    if (R < 0 || R > D || R % 2 != 0 || !(eps >= 0.f) || !isfinite(eps) ||
        (pairs != GSPN_PAIRS_HALF && pairs != GSPN_PAIRS_ADJACENT))
        return GSPN_ERR_DIM;
    if (R > 0 && (rows < 1 || (!positions && (first < 0 || (int64_t)first + T > rows))))
        return GSPN_ERR_DIM;
    if (R > 0 && !table)
        return GSPN_ERR_NULL;
    p = NormProblem{};
    p.B = B, p.T = T, p.Hq = Hq, p.Hk = Hk, p.D = D, p.R = R;
    p.rows = rows, p.first = first;
    p.adjacent = pairs == GSPN_PAIRS_ADJACENT;
    p.eps = eps;
    p.dtype = dtype;
    return GSPN_OK;
}

int make_delta(DeltaProblem &p, int B, int T, int Hq, int Hv, int Dk, int Dv, float scale, int dtype)
{
    int st = check_sizes(B, T, 1, Hq, Hv, Dk, kDeltaMaxHead, dtype);
    if (st == GSPN_OK)
        st = check_sizes(B, T, 1, Hv, Hq, Dv, kDeltaMaxHead, dtype);
    if (st != GSPN_OK)
        return st;
    if (Hv % Hq != 0 || !isfinite(scale))
        return GSPN_ERR_DIM;
    p = DeltaProblem{};
    p.B = B, p.T = T, p.Hq = Hq, p.Hv = Hv, p.Dk = Dk, p.Dv = Dv;
    p.scale = scale;
    p.dtype = dtype;
    return GSPN_OK;
}

// Bytes of the training pair's reserve.
int64_t delta_reserve(const DeltaProblem &p)
{
    Workspace rs;
    rs.counting = true;
    DeltaKept kept;
    DeltaProblem q = p;
    q.rs = &rs;
    if (p.dtype == GSPN_F32)
        take_delta_kept(q, &rs, &kept);
    else
        delta16_reserve(q);
    return (int64_t)rs.used;
}

// The inputs that both passes of the delta rule read.
void delta_inputs(DeltaProblem &p, Buffers &bufs, const void *q, const void *k, const void *v, const void *g,
                  const void *beta, const int32_t *lens, const int64_t *strides)
{
    const int64_t gates = (int64_t)p.B * p.T * p.Hv * storage(p.dtype);
    p.q = bufs.heads(q, at(strides, 0), p.B, p.T, p.Hq, p.Dk, p.dtype, false);
    p.k = bufs.heads(k, at(strides, 1), p.B, p.T, p.Hq, p.Dk, p.dtype, false);
    p.v = bufs.heads(v, at(strides, 2), p.B, p.T, p.Hv, p.Dv, p.dtype, false);
    bufs.buffer(g, gates, (int)storage(p.dtype), false);
    bufs.buffer(beta, gates, (int)storage(p.dtype), false);
    bufs.buffer(lens, (int64_t)p.B * 4, 4, false, true);
    p.g = g, p.beta = beta, p.lens = lens;
}

int delta_fwd(const void *q, const void *k, const void *v, const void *g, const void *beta, const float *state,
              const int32_t *lens, void *o, float *state_out, const int64_t *strides, int B, int T, int Hq, int Hv, int Dk,
              int Dv, float scale, int dtype, void *reserve, int64_t reserve_bytes, bool train, void *workspace,
              int64_t workspace_bytes, void *stream)
{
    DeltaProblem p;
    const int st = make_delta(p, B, T, Hq, Hv, Dk, Dv, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    delta_inputs(p, bufs, q, k, v, g, beta, lens, strides);
    const int64_t states = (int64_t)B * Hv * Dk * Dv * 4;
    if (state != state_out)   // a state may be continued in place
        bufs.buffer(state, states, 16, false, true);
    p.o = bufs.heads(o, at(strides, 3), B, T, Hv, Dv, dtype, true);
    bufs.buffer(state_out, states, 16, true, true);
    p.state = state, p.state_out = state_out;
    Workspace rs;
    if (train) {
        const int64_t need = delta_reserve(p);
        if (bufs.status == GSPN_OK && (reserve == nullptr || reserve_bytes < need))
            return GSPN_ERR_WORKSPACE;
        bufs.buffer(reserve, need, 16, true);
        rs.base = static_cast<char *>(reserve);
        rs.size = (size_t)need;
        p.rs = &rs;
    }
    if (bufs.status != GSPN_OK)
        return bufs.status;
    return run(p, launch_delta_fwd, bufs, workspace, workspace_bytes, stream);
}

// The weights and tables that both passes of the norm read.
void norm_inputs(NormProblem &p, Buffers &bufs, const void *wq, const void *wk, const float *cos_t, const float *sin_t,
                 const int32_t *positions)
{
    const int64_t es = storage(p.dtype), table = (int64_t)p.rows * (p.R / 2) * 4;
    bufs.buffer(wq, p.D * es, 16, false, true);
    bufs.buffer(wk, p.D * es, 16, false, true);
    if (p.R > 0) {
        bufs.buffer(cos_t, table, 16, false);
        bufs.buffer(sin_t, table, 16, false);
        bufs.buffer(positions, (int64_t)p.B * p.T * 4, 4, false, true);
        p.cos = cos_t, p.sin = sin_t, p.positions = positions;
    }
    p.wq = wq, p.wk = wk;
}

}  // namespace
}  // namespace gspn

using namespace gspn;

extern "C" int gspn_qk_norm_rotate_fwd(const void *q, const void *k, const void *wq, const void *wk, const float *cos_t,
                                       const float *sin_t, const int32_t *positions, void *yq, void *yk,
                                       const int64_t *strides, int B, int T, int Hq, int Hk, int D, int R, int table_rows,
                                       int first, int pairs, float eps, int dtype, void *stream)
{
    NormProblem p;
    const int st = make_norm(p, B, T, Hq, Hk, D, R, table_rows, first, pairs, eps, dtype, cos_t && sin_t, positions);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, T, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, T, Hk, D, dtype, false);
    norm_inputs(p, bufs, wq, wk, cos_t, sin_t, positions);
    p.yq = bufs.heads(yq, at(strides, 2), B, T, Hq, D, dtype, true, 0);
    p.yk = bufs.heads(yk, at(strides, 3), B, T, Hk, D, dtype, true, 1);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    return run(p, launch_norm_rotate_fwd, bufs, nullptr, 0, stream);
}

extern "C" int gspn_qk_norm_rotate_workspace_size(int B, int T, int Hq, int Hk, int D, int R, int pairs, int dtype,
                                                  int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    NormProblem p;
    const int st = make_norm(p, B, T, Hq, Hk, D, R, T, 0, pairs, 0.f, dtype, true, false);
    if (st != GSPN_OK)
        return st;
    p.wq = p.wk = bytes;   // counted as if both were there
    return count(p, launch_norm_rotate_bwd, bytes);
}

extern "C" int gspn_qk_norm_rotate_bwd(const void *q, const void *k, const void *wq, const void *wk, const float *cos_t,
                                       const float *sin_t, const int32_t *positions, const void *dyq, const void *dyk,
                                       void *dq, void *dk, void *dwq, void *dwk, const int64_t *strides, int B, int T,
                                       int Hq, int Hk, int D, int R, int table_rows, int first, int pairs, float eps,
                                       int dtype, void *workspace, int64_t workspace_bytes, void *stream)
{
    NormProblem p;
    const int st = make_norm(p, B, T, Hq, Hk, D, R, table_rows, first, pairs, eps, dtype, cos_t && sin_t, positions);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, T, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, T, Hk, D, dtype, false);
    norm_inputs(p, bufs, wq, wk, cos_t, sin_t, positions);
    p.dyq = bufs.heads(dyq, at(strides, 2), B, T, Hq, D, dtype, false);
    p.dyk = bufs.heads(dyk, at(strides, 3), B, T, Hk, D, dtype, false);
    p.dq = bufs.heads(dq, at(strides, 4), B, T, Hq, D, dtype, true);
    p.dk = bufs.heads(dk, at(strides, 5), B, T, Hk, D, dtype, true);
    // a weight that was given has a gradient
    if (wq)
        bufs.buffer(dwq, D * storage(dtype), 16, true);
    if (wk)
        bufs.buffer(dwk, D * storage(dtype), 16, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.dwq = wq ? dwq : nullptr;
    p.dwk = wk ? dwk : nullptr;
    return run(p, launch_norm_rotate_bwd, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_window_attn_workspace_size(int op, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left, int right,
                                               int sinks, int offset, int dtype, int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    if (op != GSPN_ATTN_FWD && op != GSPN_ATTN_BWD && op != GSPN_ATTN_DECODE)
        return GSPN_ERR_UNSUPPORTED;
    AttnProblem p;
    const int st = make_attn(p, B, Tq, Tk, Hq, Hkv, D, left, op == GSPN_ATTN_DECODE ? 0 : right, sinks,
                             op == GSPN_ATTN_DECODE ? 0 : offset, 1.f, dtype);
    if (st != GSPN_OK)
        return st;
    return count(p, op == GSPN_ATTN_FWD ? launch_attn_fwd : op == GSPN_ATTN_BWD ? launch_attn_bwd : launch_attn_split, bytes);
}

extern "C" int gspn_window_attn_fwd(const void *q, const void *k, const void *v, const int32_t *lens, void *o, float *lse,
                                    const int64_t *strides, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left,
                                    int right, int sinks, int offset, float scale, int dtype, void *workspace,
                                    int64_t workspace_bytes, void *stream)
{
    AttnProblem p;
    const int st = make_attn(p, B, Tq, Tk, Hq, Hkv, D, left, right, sinks, offset, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, Tq, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, Tk, Hkv, D, dtype, false);
    p.v = bufs.heads(v, at(strides, 2), B, Tk, Hkv, D, dtype, false);
    bufs.buffer(lens, (int64_t)B * 4, 4, false, true);
    p.o = bufs.heads(o, at(strides, 3), B, Tq, Hq, D, dtype, true);
    bufs.buffer(lse, (int64_t)B * Hq * Tq * 4, 4, true, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.lens = lens;
    p.lse = lse;
    return run(p, launch_attn_fwd, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_window_attn_bwd(const void *q, const void *k, const void *v, const void *o, const float *lse,
                                    const void *dout, const int32_t *lens, void *dq, void *dk, void *dv,
                                    const int64_t *strides, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left,
                                    int right, int sinks, int offset, float scale, int dtype, void *workspace,
                                    int64_t workspace_bytes, void *stream)
{
    AttnProblem p;
    const int st = make_attn(p, B, Tq, Tk, Hq, Hkv, D, left, right, sinks, offset, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, Tq, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, Tk, Hkv, D, dtype, false);
    p.v = bufs.heads(v, at(strides, 2), B, Tk, Hkv, D, dtype, false);
    p.o = bufs.heads(o, at(strides, 3), B, Tq, Hq, D, dtype, false);
    p.dout = bufs.heads(dout, at(strides, 4), B, Tq, Hq, D, dtype, false);
    bufs.buffer(lse, (int64_t)B * Hq * Tq * 4, 4, false);
    bufs.buffer(lens, (int64_t)B * 4, 4, false, true);
    p.dq = bufs.heads(dq, at(strides, 5), B, Tq, Hq, D, dtype, true);
    p.dk = bufs.heads(dk, at(strides, 6), B, Tk, Hkv, D, dtype, true);
    p.dv = bufs.heads(dv, at(strides, 7), B, Tk, Hkv, D, dtype, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.lens = lens;
    p.lse = const_cast<float *>(lse);
    return run(p, launch_attn_bwd, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_window_attn_decode(const void *q, const void *k, const void *v, const int32_t *lens, void *o,
                                       const int64_t *strides, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left,
                                       int sinks, float scale, int dtype, void *workspace, int64_t workspace_bytes,
                                       void *stream)
{
    AttnProblem p;
    const int st = make_attn(p, B, Tq, Tk, Hq, Hkv, D, left, 0, sinks, 0, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, Tq, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, Tk, Hkv, D, dtype, false);
    p.v = bufs.heads(v, at(strides, 2), B, Tk, Hkv, D, dtype, false);
    bufs.buffer(lens, (int64_t)B * 4, 4, false, true);
    p.o = bufs.heads(o, at(strides, 3), B, Tq, Hq, D, dtype, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.lens = lens;
    p.tail = true;
    return run(p, launch_attn_split, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_delta_rule_reserve_size(int B, int T, int Hq, int Hv, int Dk, int Dv, int dtype, int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    DeltaProblem p;
    const int st = make_delta(p, B, T, Hq, Hv, Dk, Dv, 1.f, dtype);
    if (st == GSPN_OK)
        *bytes = delta_reserve(p);
    return st;
}

extern "C" int gspn_delta_rule_workspace_size(int op, int B, int T, int Hq, int Hv, int Dk, int Dv, int dtype,
                                              int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    if (op != GSPN_DELTA_FWD && op != GSPN_DELTA_FWD_TRAIN && op != GSPN_DELTA_BWD_RESERVE)
        return GSPN_ERR_UNSUPPORTED;
    DeltaProblem p;
    const int st = make_delta(p, B, T, Hq, Hv, Dk, Dv, 1.f, dtype);
    if (st != GSPN_OK)
        return st;
    Workspace rs;
    rs.counting = true;
    if (op != GSPN_DELTA_FWD)
        p.rs = &rs;
    return count(p, op == GSPN_DELTA_BWD_RESERVE ? launch_delta_bwd : launch_delta_fwd, bytes);
}

extern "C" int gspn_delta_rule_fwd(const void *q, const void *k, const void *v, const void *g, const void *beta,
                                   const float *state, const int32_t *lens, void *o, float *state_out,
                                   const int64_t *strides, int B, int T, int Hq, int Hv, int Dk, int Dv, float scale,
                                   int dtype, void *workspace, int64_t workspace_bytes, void *stream)
{
    return delta_fwd(q, k, v, g, beta, state, lens, o, state_out, strides, B, T, Hq, Hv, Dk, Dv, scale, dtype, nullptr, 0,
                     false, workspace, workspace_bytes, stream);
}

extern "C" int gspn_delta_rule_fwd_train(const void *q, const void *k, const void *v, const void *g, const void *beta,
                                         const float *state, const int32_t *lens, void *o, float *state_out,
                                         const int64_t *strides, int B, int T, int Hq, int Hv, int Dk, int Dv, float scale,
                                         int dtype, void *reserve, int64_t reserve_bytes, void *workspace,
                                         int64_t workspace_bytes, void *stream)
{
    return delta_fwd(q, k, v, g, beta, state, lens, o, state_out, strides, B, T, Hq, Hv, Dk, Dv, scale, dtype, reserve,
                     reserve_bytes, true, workspace, workspace_bytes, stream);
}

extern "C" int gspn_delta_rule_bwd_reserve(const void *q, const void *k, const void *v, const void *g, const void *beta,
                                           const void *dout, const float *dstate_out, const int32_t *lens, void *dq,
                                           void *dk, void *dv, void *dg, void *dbeta, float *dstate, const int64_t *strides,
                                           int B, int T, int Hq, int Hv, int Dk, int Dv, float scale, int dtype,
                                           void *reserve, int64_t reserve_bytes, void *workspace, int64_t workspace_bytes,
                                           void *stream)
{
    DeltaProblem p;
    const int st = make_delta(p, B, T, Hq, Hv, Dk, Dv, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    delta_inputs(p, bufs, q, k, v, g, beta, lens, strides);
    const int64_t states = (int64_t)B * Hv * Dk * Dv * 4, gates = (int64_t)B * T * Hv * storage(dtype);
    p.dout = bufs.heads(dout, at(strides, 3), B, T, Hv, Dv, dtype, false);
    bufs.buffer(dstate_out, states, 16, false, true);
    p.dq = bufs.heads(dq, at(strides, 4), B, T, Hq, Dk, dtype, true);
    p.dk = bufs.heads(dk, at(strides, 5), B, T, Hq, Dk, dtype, true);
    p.dv = bufs.heads(dv, at(strides, 6), B, T, Hv, Dv, dtype, true);
    bufs.buffer(dg, gates, (int)storage(dtype), true);
    bufs.buffer(dbeta, gates, (int)storage(dtype), true);
    bufs.buffer(dstate, states, 16, true, true);
    p.dg = dg, p.dbeta = dbeta, p.dstate = dstate_out, p.dstate_in = dstate;
    const int64_t need = delta_reserve(p);
    if (bufs.status == GSPN_OK && (reserve == nullptr || reserve_bytes < need))
        return GSPN_ERR_WORKSPACE;
    bufs.buffer(reserve, need, 16, false);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    Workspace rs;
    rs.base = static_cast<char *>(reserve);
    rs.size = (size_t)need;
    p.rs = &rs;
    return run(p, launch_delta_bwd, bufs, workspace, workspace_bytes, stream);
}
