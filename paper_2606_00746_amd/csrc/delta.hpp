// The gated delta rule: the problem and what its kernels share (internal).
//
//   S_t = exp(g_t) (I - b_t k_t k_t^T) S_{t-1} + b_t k_t v_t^T,   o_t = scale S_t^T q_t
//
// In chunks of 64 tokens, with G the running sum of g in the chunk, S the state
// ahead of it and M_ts = exp(G_t - G_s) k_t.k_s for s < t (0 elsewhere):
//   X = V - exp(G) K S,  U = (I + b M)^-1 b X
//   O = scale (exp(G) Q S + A U),  A_ts = exp(G_t - G_s) q_t.k_s for s <= t
//   S' = exp(G_63) S + (exp(G_63 - G) K)^T U
// The inverse of a chunk needs no state, so all chunks' are formed at once
// (delta_inverse_kernel), then one kernel takes the chunks in turn for U and
// the states (delta_state_kernel), and one forms all outputs (delta_out_kernel).
// Backwards, with dS the gradient of S':
//   dU = scale A^T dO + exp(G_63 - G) K dS,  R = (I + b M)^-T dU,  dX = b R = dV
//   dS_before = exp(G_63) dS + scale (exp(G) Q)^T dO - (exp(G) K)^T dX
// in turn from the last chunk (delta_dstate_kernel), and what is left for all
// chunks at once (delta_grad_kernel).
//
// States, inverses and everything on their way are fp32 and their products run
// on the fp32 matrix instructions (16 x 16 x 4): a state is carried through all
// chunks, and with 8 significant bits its error would be some 10^4 times as
// large.  A contraction takes index 4 u + i in step i from lane l = 16 u + n of
// either operand, in whichever order it is stored, so a result's registers
// (rows 4 u + i, column n) are the next product's B operand as they stand.
#pragma once

#include "attn.hpp"

namespace gspn {

struct DeltaProblem {
    Heads q, k, v, o;                // [B][T][Hq][Dk] x 2, [B][T][Hv][Dv] x 2
    Heads dout, dq, dk, dv;          // backward
    const void *g, *beta;            // [B][T][Hv], storage type
    void *dg, *dbeta;
    const float *state;              // [B][Hv][Dk][Dv] or null: zeros
    float *state_out;                // or null
    const float *dstate;             // gradient of state_out, or null: zeros
    float *dstate_in;                // gradient of state, or null
    const int32_t *lens;             // [B], or null: T
    int B, T, Hq, Hv, Dk, Dv;
    float scale;
    int dtype;
    Workspace *ws;
    Workspace *rs;                   // what the forward leaves for the backward; null: in ws
};

hipError_t launch_delta_fwd(const DeltaProblem &p, hipStream_t s);
hipError_t launch_delta_bwd(const DeltaProblem &p, hipStream_t s);
// bf16 storage (delta_bf16.hip), and what its training forward takes from p.rs.
hipError_t launch_delta16_fwd(const DeltaProblem &p, hipStream_t s);
hipError_t launch_delta16_bwd(const DeltaProblem &p, hipStream_t s);
hipError_t delta16_reserve(const DeltaProblem &p);

constexpr int kDeltaMaxHead = 128;
constexpr int kChunk = 64;

// Per (b, value head, chunk): the inverse [64][64], U [64][Sv], the state ahead
// of the chunk [DKP][Sv] (DKP: Dk as 64 or 128; Sv: Dv as a multiple of 16).
struct DeltaKept {
    float *inv = nullptr, *u = nullptr, *s = nullptr;
};

// The row length of U and of states: Dv as a multiple of 16.
inline int delta_sv(const DeltaProblem &p) { return (p.Dv + 15) / 16 * 16; }
inline int delta_chunks(const DeltaProblem &p) { return (p.T + kChunk - 1) / kChunk; }

inline hipError_t take_delta_kept(const DeltaProblem &p, Workspace *w, DeltaKept *k)
{
    const int64_t n = (int64_t)p.B * p.Hv * delta_chunks(p), sv = delta_sv(p), dk = p.Dk <= 64 ? 64 : 128;
    void *a = nullptr, *b = nullptr, *c = nullptr;
    hipError_t e = w->take(&a, (size_t)(n * kChunk * kChunk * 4));
    if (e == hipSuccess)
        e = w->take(&b, (size_t)(n * kChunk * sv * 4));
    if (e == hipSuccess)
        e = w->take(&c, (size_t)(n * dk * sv * 4));
    k->inv = static_cast<float *>(a);
    k->u = static_cast<float *>(b);
    k->s = static_cast<float *>(c);
    return e;
}

#ifdef __HIPCC__

namespace delta {

using namespace attn;

constexpr int kPitch = kChunk + 4;   // row of a 64 x 64 matrix in LDS

__device__ __forceinline__ f32x4_t mma4(float a, float b, f32x4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float at_f(const void *p, int64_t i, int dtype)
{
    return dtype == 0 ? load_f(static_cast<const float *>(p) + i) : load_f(static_cast<const bf16_t *>(p) + i);
}

// Four or eight consecutive values as fp32.
__device__ __forceinline__ f32x4_t load4(const float *p) { return *reinterpret_cast<const f32x4_t *>(p); }
__device__ __forceinline__ f32x4_t load4(const bf16_t *p)
{
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    return f32x4_t{bf_lo(v.x), bf_hi(v.x), bf_lo(v.y), bf_hi(v.y)};
}

// The decay of a token: exp(-100) is 0 to fp32 next to anything, and a bound
// keeps running sums finite where a token forgets everything.
constexpr float kLeastGate = -100.f;
__device__ __forceinline__ float bounded(float g) { return g < kLeastGate ? kLeastGate : g; }   // (a NaN stays one)

// A chunk's gates by lane (token): the running sum of g and beta; tokens from n on
// decay and write nothing.  The sum is G + D, two floats: behind tokens that forget
// everything G is some hundreds or thousands, whose fp32 steps (2^-12 at 4000) would
// be errors of the decays exp(G_t - G_s) between the ordinary tokens that follow.
struct Gates {
    float G, D, beta;
};
__device__ __forceinline__ Gates load_gates(const DeltaProblem &p, int b, int h, int t0, int n, int lane)
{
    Gates x{0.f, 0.f, 0.f};
    if (lane < n) {
        const int64_t at = ((int64_t)b * p.T + t0 + lane) * p.Hv + h;
        x.G = bounded(at_f(p.g, at, p.dtype));
        x.beta = at_f(p.beta, at, p.dtype);
    }
    return x;
}
__device__ __forceinline__ void sum_gates(Gates &x, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const float g = __shfl_up(x.G, d), r = __shfl_up(x.D, d);
        if (lane >= d) {   // the sum and, exactly, what it leaves
            const float s = x.G + g, part = s - x.G;
            const float rest = ((x.G - (s - part)) + (g - part)) + (x.D + r);
            x.G = s + rest;
            x.D = rest - (x.G - s);
        }
    }
}

__device__ __forceinline__ float exp_f(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// exp(G_t - G_s) from the sums' two floats.
__device__ __forceinline__ float decay(float gt, float dt, float gs, float ds)
{
    return exp_f((gt - gs) + (dt - ds));
}

__device__ __forceinline__ int delta_len(const DeltaProblem &p, int b)
{
    return p.lens ? min(max(p.lens[b], 0), p.T) : p.T;
}

// 64 rows of DP columns (rows from n, columns from D on as zero) in registers,
// then in LDS as fp32 rows of DP + 4.
template <typename T, int DP>
struct Rows {
    static constexpr int kN = kChunk * DP / 8 / kThreads;
    f32x4_t r[kN][2];
    __device__ __forceinline__ void load(const T *base, int64_t st, int n, int D)
    {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int x = threadIdx.x + i * kThreads, row = x / (DP / 8), c = x % (DP / 8) * 8;
            r[i][0] = r[i][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (row < n && c < D) {
                r[i][0] = load4(base + row * st + c);
                r[i][1] = load4(base + row * st + c + 4);
            }
        }
    }
    __device__ __forceinline__ void store(float *lds) const
    {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int x = threadIdx.x + i * kThreads, row = x / (DP / 8), c = x % (DP / 8) * 8;
            *reinterpret_cast<f32x4_t *>(lds + row * (DP + 4) + c) = r[i][0];
            *reinterpret_cast<f32x4_t *>(lds + row * (DP + 4) + c + 4) = r[i][1];
        }
    }
};

// A 64 x 64 fp32 matrix in registers, then in LDS as rows of kPitch.
struct Square {
    f32x4_t r[4];
    __device__ __forceinline__ void load(const float *m)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[i] = load4(m + 4 * (threadIdx.x + i * kThreads));
    }
    __device__ __forceinline__ void store(float *lds) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = threadIdx.x + i * kThreads;
            *reinterpret_cast<f32x4_t *>(lds + x / 16 * kPitch + x % 16 * 4) = r[i];
        }
    }
};

}  // namespace delta

#endif

}  // namespace gspn
