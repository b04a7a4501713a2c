// C ABI of the state space sublayer: the short causal convolution, the selective scan, and
// the joint between two sublayers (norms, gate, residual scale).  Argument checks (host
// only, before any HIP call), workspaces, launches.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "../../include/gspn.h"
#include "call_args.hpp"
#include "launch.hpp"
#include "residual_norm.hpp"
#include "selective.hpp"
#include "short_conv.hpp"

namespace gspn {

template <>
struct requires_reserve<SelectiveProblem> : std::true_type {};

namespace {

constexpr int64_t kMostTokens = (int64_t)1 << 28, kMostChannels = (int64_t)1 << 20;

int check_rows(int64_t B, int64_t T, int64_t C, int dtype)
{
    if (dtype != GSPN_F32 && dtype != GSPN_BF16)
        return GSPN_ERR_DTYPE;
    if (B < 1 || T < 1 || C < 1)
        return GSPN_ERR_DIM;
    if (C % 8 != 0 || C > kMostChannels || T > kMostTokens || B > kMostTokens || B * C > GSPN_MAX_ELEMS / T)
        return GSPN_ERR_UNSUPPORTED;
    return GSPN_OK;
}

// Strides of tensor i (batch, token, head), null: contiguous.
const int64_t *at(const int64_t *strides, int i) { return strides ? strides + 3 * i : nullptr; }

// ---------------------------------------------------------------------------
// short convolution
// ---------------------------------------------------------------------------

int make_conv(ConvProblem &p, int B, int T, int C, int K, int act, int dtype)
{
    const int st = check_rows(B, T, C, dtype);
    if (st != GSPN_OK)
        return st;
    if (K < 1 || (act != GSPN_ACT_NONE && act != GSPN_ACT_SILU))
        return GSPN_ERR_DIM;
    if (K < 2 || K > kConvMaxTaps)
        return GSPN_ERR_UNSUPPORTED;
    p = ConvProblem{};
    p.B = B, p.T = T, p.C = C, p.K = K;
    p.silu = act == GSPN_ACT_SILU;
    p.dtype = dtype;
    return GSPN_OK;
}

// ---------------------------------------------------------------------------
// selective scan
// ---------------------------------------------------------------------------

int make_selective(SelectiveProblem &p, int B, int T, int C, int G, int N, int softplus, int dtype)
{
    const int st = check_rows(B, T, C, dtype);
    if (st != GSPN_OK)
        return st;
    if (G < 1 || N < 1 || C % G != 0 || (softplus != 0 && softplus != 1))
        return GSPN_ERR_DIM;
    if (C / G % 8 != 0 || N > kSelMaxStates || (int64_t)B * C > GSPN_MAX_ELEMS / N / T)
        return GSPN_ERR_UNSUPPORTED;
    p = SelectiveProblem{};
    p.B = B, p.T = T, p.C = C, p.G = G, p.N = N;
    p.softplus = softplus != 0;
    p.dtype = dtype;
    return GSPN_OK;
}

// Bytes of the training pair's reserve.
int64_t selective_reserve(const SelectiveProblem &p)
{
    Workspace rs;
    rs.counting = true;
    SelectiveProblem q = p;
    q.rs = &rs;
    void *kept, *bc;
    (void)take_sel_kept(q, &rs, &kept, &bc);
    return (int64_t)rs.used;
}

// The inputs that both passes read.
void selective_inputs(SelectiveProblem &p, Buffers &bufs, const void *x, const void *dt, const float *A, const void *Bm,
                      const void *Cm, const float *D, const void *z, const float *dt_bias, const int32_t *lens,
                      const int64_t *strides)
{
    const int es = (int)storage(p.dtype);
    p.x = bufs.rows(x, at(strides, 0), p.B, p.T, p.C, p.dtype, false);
    p.dt = bufs.rows(dt, at(strides, 1), p.B, p.T, p.C, p.dtype, false);
    p.Bm = bufs.heads(Bm, at(strides, 2), p.B, p.T, p.G, p.N, p.dtype, false, -1, es);
    p.Cm = bufs.heads(Cm, at(strides, 3), p.B, p.T, p.G, p.N, p.dtype, false, -1, es);
    if (z)
        p.z = bufs.rows(z, at(strides, 4), p.B, p.T, p.C, p.dtype, false);
    bufs.buffer(A, (int64_t)p.C * p.N * 4, 16, false);
    bufs.buffer(D, (int64_t)p.C * 4, 16, false, true);
    bufs.buffer(dt_bias, (int64_t)p.C * 4, 16, false, true);
    bufs.buffer(lens, (int64_t)p.B * 4, 4, false, true);
    p.A = A, p.D = D, p.dt_bias = dt_bias, p.lens = lens;
}

int selective_fwd(const void *x, const void *dt, const float *A, const void *Bm, const void *Cm, const float *D,
                  const void *z, const float *dt_bias, const float *state, const int32_t *lens, void *y, float *state_out,
                  const int64_t *strides, int B, int T, int C, int G, int N, int softplus, int dtype, void *reserve,
                  int64_t reserve_bytes, bool train, void *workspace, int64_t workspace_bytes, void *stream)
{
    SelectiveProblem p;
    const int st = make_selective(p, B, T, C, G, N, softplus, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    selective_inputs(p, bufs, x, dt, A, Bm, Cm, D, z, dt_bias, lens, strides);
    const int64_t states = (int64_t)B * C * N * 4;
    if (state != state_out)   // a state may be continued in place
        bufs.buffer(state, states, 16, false, true);
    p.y = bufs.rows(y, at(strides, 5), B, T, C, dtype, true);
    bufs.buffer(state_out, states, 16, true, true);
    p.state = state, p.state_out = state_out;
    Workspace rs;
    if (train) {
        const int64_t need = selective_reserve(p);
        if (bufs.status == GSPN_OK && (reserve == nullptr || reserve_bytes < need))
            return GSPN_ERR_WORKSPACE;
        bufs.buffer(reserve, need, 16, true);
        rs.base = static_cast<char *>(reserve);
        rs.size = (size_t)need;
        p.rs = &rs;
    }
    if (bufs.status != GSPN_OK)
        return bufs.status;
    return run(p, launch_selective_fwd, bufs, workspace, workspace_bytes, stream);
}

// ---------------------------------------------------------------------------
// the joint between two sublayers
// ---------------------------------------------------------------------------

int make_join(JoinProblem &p, int B, int T, int C, float eps, int dtype, int rdtype)
{
    const int st = check_rows(B, T, C, dtype);
    if (st != GSPN_OK)
        return st;
    if (rdtype != dtype && rdtype != GSPN_F32)
        return GSPN_ERR_DTYPE;
    if (!(eps >= 0.f) || !isfinite(eps))
        return GSPN_ERR_DIM;
    if (C > kJoinMaxRow)
        return GSPN_ERR_UNSUPPORTED;
    p = JoinProblem{};
    p.B = B, p.T = T, p.C = C;
    p.eps = eps;
    p.dtype = dtype, p.rdtype = rdtype;
    return GSPN_OK;
}

// The vectors that both passes read; those of the block's output need one.
void join_vectors(JoinProblem &p, Buffers &bufs, const void *w, const void *w_post, const void *scale, const void *gate)
{
    const int64_t es = storage(p.dtype);
    if (!p.f.p && (w_post || scale || gate))
        bufs.fail(GSPN_ERR_NULL);
    bufs.buffer(w, p.C * es, 16, false, true);
    bufs.buffer(w_post, p.C * es, 16, false, true);
    bufs.buffer(scale, p.C * es, 16, false, true);
    bufs.buffer(gate, (int64_t)p.B * p.C * es, 16, false, true);
    p.w = w, p.w_post = w_post, p.scale = scale, p.gate = gate;
}

}  // namespace
}  // namespace gspn

using namespace gspn;

extern "C" int gspn_short_conv_fwd(const void *x, const void *w, const void *bias, const void *state, const int32_t *lens,
                                   void *y, void *state_out, const int64_t *strides, int B, int T, int C, int K, int act,
                                   int dtype, void *stream)
{
    ConvProblem p;
    const int st = make_conv(p, B, T, C, K, act, dtype);
    if (st != GSPN_OK)
        return st;
    const int64_t es = storage(dtype), states = (int64_t)B * (K - 1) * C * es;
    Buffers bufs;
    p.x = bufs.rows(x, at(strides, 0), B, T, C, dtype, false);
    bufs.buffer(w, (int64_t)C * K * es, 16, false);
    bufs.buffer(bias, C * es, 16, false, true);
    if (state != state_out)   // a state may be continued in place
        bufs.buffer(state, states, 16, false, true);
    bufs.buffer(lens, (int64_t)B * 4, 4, false, true);
    p.y = bufs.rows(y, at(strides, 1), B, T, C, dtype, true);
    bufs.buffer(state_out, states, 16, true, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.w = w, p.bias = bias, p.state = state, p.state_out = state_out, p.lens = lens;
    return run(p, launch_conv_fwd, bufs, nullptr, 0, stream);
}

extern "C" int gspn_short_conv_workspace_size(int B, int T, int C, int K, int dtype, int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    ConvProblem p;
    const int st = make_conv(p, B, T, C, K, GSPN_ACT_SILU, dtype);
    if (st != GSPN_OK)
        return st;
    p.dw = bytes;   // counted as if it were wanted
    return count(p, launch_conv_bwd, bytes);
}

extern "C" int gspn_short_conv_bwd(const void *x, const void *w, const void *bias, const void *dy, const void *dstate_out,
                                   const void *state, const int32_t *lens, void *dx, void *dw, void *dbias, void *dstate,
                                   const int64_t *strides, int B, int T, int C, int K, int act, int dtype, void *workspace,
                                   int64_t workspace_bytes, void *stream)
{
    ConvProblem p;
    const int st = make_conv(p, B, T, C, K, act, dtype);
    if (st != GSPN_OK)
        return st;
    const int64_t es = storage(dtype), states = (int64_t)B * (K - 1) * C * es;
    Buffers bufs;
    p.x = bufs.rows(x, at(strides, 0), B, T, C, dtype, false);
    bufs.buffer(w, (int64_t)C * K * es, 16, false);
    bufs.buffer(bias, C * es, 16, false, true);
    p.dy = bufs.rows(dy, at(strides, 1), B, T, C, dtype, false);
    bufs.buffer(dstate_out, states, 16, false, true);
    bufs.buffer(state, states, 16, false, true);
    bufs.buffer(lens, (int64_t)B * 4, 4, false, true);
    p.dx = bufs.rows(dx, at(strides, 2), B, T, C, dtype, true);
    bufs.buffer(dw, (int64_t)C * K * es, 16, true);
    if (bias)   // a bias that was given has a gradient
        bufs.buffer(dbias, C * es, 16, true);
    bufs.buffer(dstate, states, 16, true, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.w = w, p.bias = bias, p.state = state, p.dstate = dstate_out, p.lens = lens;
    p.dw = dw, p.dbias = bias ? dbias : nullptr, p.dstate_in = dstate;
    return run(p, launch_conv_bwd, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_selective_scan_workspace_size(int op, int B, int T, int C, int G, int N, int dtype, int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    if (op != GSPN_SELECTIVE_FWD && op != GSPN_SELECTIVE_FWD_TRAIN && op != GSPN_SELECTIVE_BWD_RESERVE)
        return GSPN_ERR_UNSUPPORTED;
    SelectiveProblem p;
    const int st = make_selective(p, B, T, C, G, N, 1, dtype);
    if (st != GSPN_OK)
        return st;
    Workspace rs;
    rs.counting = true;
    if (op != GSPN_SELECTIVE_FWD)
        p.rs = &rs;
    return count(p, op == GSPN_SELECTIVE_BWD_RESERVE ? launch_selective_bwd : launch_selective_fwd, bytes);
}

extern "C" int gspn_selective_scan_reserve_size(int B, int T, int C, int G, int N, int dtype, int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    SelectiveProblem p;
    const int st = make_selective(p, B, T, C, G, N, 1, dtype);
    if (st == GSPN_OK)
        *bytes = selective_reserve(p);
    return st;
}

extern "C" int gspn_selective_scan_fwd(const void *x, const void *dt, const float *A, const void *Bm, const void *Cm,
                                       const float *D, const void *z, const float *dt_bias, const float *state,
                                       const int32_t *lens, void *y, float *state_out, const int64_t *strides, int B,
                                       int T, int C, int G, int N, int softplus, int dtype, void *workspace,
                                       int64_t workspace_bytes, void *stream)
{
    return selective_fwd(x, dt, A, Bm, Cm, D, z, dt_bias, state, lens, y, state_out, strides, B, T, C, G, N, softplus, dtype,
                         nullptr, 0, false, workspace, workspace_bytes, stream);
}

extern "C" int gspn_selective_scan_fwd_train(const void *x, const void *dt, const float *A, const void *Bm, const void *Cm,
                                             const float *D, const void *z, const float *dt_bias, const float *state,
                                             const int32_t *lens, void *y, float *state_out, const int64_t *strides, int B,
                                             int T, int C, int G, int N, int softplus, int dtype, void *reserve,
                                             int64_t reserve_bytes, void *workspace, int64_t workspace_bytes, void *stream)
{
    return selective_fwd(x, dt, A, Bm, Cm, D, z, dt_bias, state, lens, y, state_out, strides, B, T, C, G, N, softplus, dtype,
                         reserve, reserve_bytes, true, workspace, workspace_bytes, stream);
}

extern "C" int gspn_selective_scan_bwd_reserve(const void *x, const void *dt, const float *A, const void *Bm, const void *Cm,
                                               const float *D, const void *z, const float *dt_bias, const void *dy,
                                               const float *dstate_out, const int32_t *lens, void *dx, void *ddt, float *dA,
                                               void *dBm, void *dCm, float *dD, void *dz, float *ddt_bias, float *dstate,
                                               const int64_t *strides, int B, int T, int C, int G, int N, int softplus,
                                               int dtype, void *reserve, int64_t reserve_bytes, void *workspace,
                                               int64_t workspace_bytes, void *stream)
{
    SelectiveProblem p;
    const int st = make_selective(p, B, T, C, G, N, softplus, dtype);
    if (st != GSPN_OK)
        return st;
    const int es = (int)storage(dtype);
    const int64_t states = (int64_t)B * C * N * 4;
    Buffers bufs;
    selective_inputs(p, bufs, x, dt, A, Bm, Cm, D, z, dt_bias, lens, strides);
    p.dy = bufs.rows(dy, at(strides, 5), B, T, C, dtype, false);
    bufs.buffer(dstate_out, states, 16, false, true);
    p.dx = bufs.rows(dx, at(strides, 6), B, T, C, dtype, true);
    p.ddt = bufs.rows(ddt, at(strides, 7), B, T, C, dtype, true);
    bufs.buffer(dA, (int64_t)C * N * 4, 16, true);
    p.dBm = bufs.heads(dBm, at(strides, 8), B, T, G, N, dtype, true, -1, es);
    p.dCm = bufs.heads(dCm, at(strides, 9), B, T, G, N, dtype, true, -1, es);
    // what was given has a gradient
    if (D)
        bufs.buffer(dD, (int64_t)C * 4, 16, true);
    if (z)
        p.dz = bufs.rows(dz, at(strides, 10), B, T, C, dtype, true);
    if (dt_bias)
        bufs.buffer(ddt_bias, (int64_t)C * 4, 16, true);
    bufs.buffer(dstate, states, 16, true, true);
    p.dstate = dstate_out, p.dstate_in = dstate;
    p.dA = dA, p.dD = D ? dD : nullptr, p.ddt_bias = dt_bias ? ddt_bias : nullptr;
    const int64_t need = selective_reserve(p);
    if (bufs.status == GSPN_OK && (reserve == nullptr || reserve_bytes < need))
        return GSPN_ERR_WORKSPACE;
    bufs.buffer(reserve, need, 16, false);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    Workspace rs;
    rs.base = static_cast<char *>(reserve);
    rs.size = (size_t)need;
    p.rs = &rs;
    return run(p, launch_selective_bwd, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_residual_norm_fwd(const void *r, const void *f, const void *w, const void *w_post, const void *scale,
                                      const void *gate, void *y, void *r_out, const int64_t *strides, int B, int T, int C,
                                      float eps, int dtype, int residual_dtype, void *stream)
{
    JoinProblem p;
    const int st = make_join(p, B, T, C, eps, dtype, residual_dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.r = bufs.rows(r, at(strides, 0), B, T, C, residual_dtype, false);
    if (f)
        p.f = bufs.rows(f, at(strides, 1), B, T, C, dtype, false);
    join_vectors(p, bufs, w, w_post, scale, gate);
    p.y = bufs.rows(y, at(strides, 2), B, T, C, dtype, true);
    if (f)   // a sum has to go somewhere
        p.ro = bufs.rows(r_out, at(strides, 3), B, T, C, residual_dtype, true, 0);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    return run(p, launch_join_fwd, bufs, nullptr, 0, stream);
}

extern "C" int gspn_residual_norm_workspace_size(int B, int T, int C, int gated, int dtype, int residual_dtype,
                                                 int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    JoinProblem p;
    const int st = make_join(p, B, T, C, 0.f, dtype, residual_dtype);
    if (st != GSPN_OK)
        return st;
    if (gated != 0 && gated != 1)
        return GSPN_ERR_DIM;
    p.dw = bytes;   // counted as if all were there
    p.gate = gated ? bytes : nullptr;
    return count(p, launch_join_bwd, bytes);
}

extern "C" int gspn_residual_norm_bwd(const void *r, const void *f, const void *w, const void *w_post, const void *scale,
                                      const void *gate, const void *dy, const void *dr_out, void *dr, void *df, void *dw,
                                      void *dw_post, void *dscale, void *dgate, const int64_t *strides, int B, int T, int C,
                                      float eps, int dtype, int residual_dtype, void *workspace, int64_t workspace_bytes,
                                      void *stream)
{
    JoinProblem p;
    const int st = make_join(p, B, T, C, eps, dtype, residual_dtype);
    if (st != GSPN_OK)
        return st;
    const int64_t es = storage(dtype);
    Buffers bufs;
    int sum = -1;   // the buffer that dr may be
    p.r = bufs.rows(r, at(strides, 0), B, T, C, residual_dtype, false);
    if (f)
        p.f = bufs.rows(f, at(strides, 1), B, T, C, dtype, false);
    join_vectors(p, bufs, w, w_post, scale, gate);
    p.dy = bufs.rows(dy, at(strides, 2), B, T, C, dtype, false);
    if (dr_out) {
        sum = bufs.n;
        p.dro = bufs.rows(dr_out, at(strides, 3), B, T, C, residual_dtype, false);
    }
    p.dr = bufs.rows(dr, at(strides, 4), B, T, C, residual_dtype, true, sum);
    if (f)
        p.df = bufs.rows(df, at(strides, 5), B, T, C, dtype, true);
    // a vector that was given has a gradient
    if (w)
        bufs.buffer(dw, C * es, 16, true);
    if (w_post)
        bufs.buffer(dw_post, C * es, 16, true);
    if (scale)
        bufs.buffer(dscale, C * es, 16, true);
    if (gate)
        bufs.buffer(dgate, (int64_t)B * C * es, 16, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.dw = w ? dw : nullptr, p.dw_post = w_post ? dw_post : nullptr;
    p.dscale = scale ? dscale : nullptr, p.dgate = gate ? dgate : nullptr;
    return run(p, launch_join_bwd, bufs, workspace, workspace_bytes, stream);
}
