// Forward of the gated delta rule (gspn_delta_rule_fwd, _fwd_train); see delta.hpp.
#include <algorithm>

#include "delta.hpp"

namespace gspn {
namespace {

using namespace delta;

// (I + b M)^-1 of every chunk, a wave each.  K K^T on the matrix cores, then
// forward substitution with a lane per column: x_i = e_i - sum_{s<i} (b M)_is x_s,
// the row of b M broadcast from LDS.
template <typename T>
__global__ __launch_bounds__(kThreads) void delta_inverse_kernel(DeltaProblem p, float *inv, int nc)
{
    __shared__ __attribute__((aligned(16))) float lds[4][kChunk * kPitch];
    const int w = threadIdx.x / 64, l = threadIdx.x % 64, c = l % 32, h = l / 32;
    const int64_t id = (int64_t)blockIdx.x * 4 + w;
    if (id >= (int64_t)p.B * p.Hv * nc)
        return;
    const int ch = (int)(id % nc), hv = (int)(id / nc % p.Hv), b = (int)(id / nc / p.Hv);
    const int t0 = ch * kChunk, n = max(0, min(kChunk, delta_len(p, b) - t0));
    const T *k = static_cast<const T *>(p.k.p) + b * p.k.sb + (hv / (p.Hv / p.Hq)) * p.k.sh + (int64_t)t0 * p.k.st;
    Gates x = load_gates(p, b, hv, t0, n, l);
    sum_gates(x, l);

    f32x16_t kk[3];
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            kk[i][r] = 0.f;
    constexpr int kPer = 16 / (int)sizeof(T);
    for (int s = 0; s * 2 * kPer < p.Dk; ++s) {
        Frag<T> a = {}, d = {};
        if (c < n)
            a = row_frag(k + c * p.k.st, 2 * s + h, p.Dk);
        if (32 + c < n)
            d = row_frag(k + (32 + c) * p.k.st, 2 * s + h, p.Dk);
        kk[0] = mma(a, a, kk[0]);
        kk[1] = mma(d, a, kk[1]);
        kk[2] = mma(d, d, kk[2]);
    }
    float *m = lds[w];
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int t = (i ? 32 : 0) + 8 * (r / 4) + 4 * h + r % 4, s = (i == 2 ? 32 : 0) + c;
            const float gt = __shfl(x.G, t), bt = __shfl(x.beta, t), gs = __shfl(x.G, s);
            const float dt = __shfl(x.D, t), ds = __shfl(x.D, s);
            m[t * kPitch + s] = s < t ? bt * decay(gt, dt, gs, ds) * kk[i][r] : 0.f;
        }
    __builtin_amdgcn_wave_barrier();
    float col[kChunk];
    float *out = inv + id * kChunk * kChunk + l;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
        float a = i == l ? 1.f : 0.f;
#pragma unroll
        for (int s = 0; s < i; s += 4) {
            const f32x4_t v = *reinterpret_cast<const f32x4_t *>(m + i * kPitch + s);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (s + e < i)
                    a = fmaf(-v[e], col[s + e], a);
        }
        col[i] = a;
        out[i * kChunk] = a;
    }
}

// U and the states, the chunks of one (b, head) in turn for 16 columns of the
// state: wave w holds rows 16 (NB w + j) of it as results of 16 x 16 products.
template <typename T, int DKP>
__global__ __launch_bounds__(kThreads) void delta_state_kernel(DeltaProblem p, DeltaKept kept, int nc, int sv)
{
    constexpr int NB = DKP / 64, kKP = DKP + 4, kXP = 20;
    __shared__ __attribute__((aligned(16))) float kl[kChunk * kKP], tl[kChunk * kPitch];
    __shared__ __attribute__((aligned(16))) float part[4][kChunk * kXP], xl[kChunk * kXP], ul[kChunk * kXP];
    __shared__ float gl[kChunk], gd[kChunk], bl[kChunk];

    const int nv = sv / 16;
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int v0 = id % nv * 16;
    id /= nv;
    const int hv = id % p.Hv, b = id / p.Hv;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int len = delta_len(p, b);
    const T *k = static_cast<const T *>(p.k.p) + b * p.k.sb + (hv / (p.Hv / p.Hq)) * p.k.sh;
    const int xt = threadIdx.x / 4, xc = threadIdx.x % 4 * 4;   // this thread's token and columns of X
    const T *v = static_cast<const T *>(p.v.p) + b * p.v.sb + hv * p.v.sh + v0 + xc;
    const bool vin = v0 + xc < p.Dv;
    const int64_t head = (int64_t)b * p.Hv + hv;
    const float *inv = kept.inv + head * nc * kChunk * kChunk;
    float *ug = kept.u + head * nc * kChunk * sv + v0, *sg = kept.s + head * nc * DKP * sv + v0;

    f32x4_t S[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 16 * (NB * w + j) + 4 * u + i;
            S[j][i] = p.state && r < p.Dk && v0 + c < p.Dv ? p.state[(head * p.Dk + r) * p.Dv + v0 + c] : 0.f;
        }

    Rows<T, DKP> kr;
    Square tr;
    Gates gr{0.f, 0.f, 0.f};
    f32x4_t vr;
    const auto fetch = [&](int ch) {
        const int t0 = ch * kChunk, n = max(0, min(kChunk, len - t0));
        kr.load(k + (int64_t)t0 * p.k.st, p.k.st, n, p.Dk);
        tr.load(inv + (int64_t)ch * kChunk * kChunk);
        vr = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (vin && xt < n)
            vr = load4(v + (int64_t)(t0 + xt) * p.v.st);
        if (w == 0)
            gr = load_gates(p, b, hv, t0, n, l);
    };
    fetch(0);
    for (int ch = 0; ch < nc; ++ch) {
        kr.store(kl);
        tr.store(tl);
        if (w == 0) {
            sum_gates(gr, l);
            gl[l] = gr.G;
            gd[l] = gr.D;
            bl[l] = gr.beta;
        }
        const f32x4_t vc = vr;
        lds_barrier();
        if (ch + 1 < nc)
            fetch(ch + 1);
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sg[((int64_t)ch * DKP + 16 * (NB * w + j) + 4 * u + i) * sv + c] = S[j][i];
        // K S, this wave's rows of S
        f32x4_t acc[4];
#pragma unroll
        for (int rb = 0; rb < 4; ++rb)
            acc[rb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int rb = 0; rb < 4; ++rb) {
                const f32x4_t a = load4(kl + (16 * rb + c) * kKP + 16 * (NB * w + j) + 4 * u);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[rb] = mma4(a[i], S[j][i], acc[rb]);
            }
#pragma unroll
        for (int rb = 0; rb < 4; ++rb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                part[w][(16 * rb + 4 * u + i) * kXP + c] = acc[rb][i];
        lds_barrier();
        {
            f32x4_t x = load4(part[0] + xt * kXP + xc);
#pragma unroll
            for (int q = 1; q < 4; ++q)
                x += load4(part[q] + xt * kXP + xc);
            const float e = exp_f(gl[xt]), be = bl[xt];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = be * (vc[i] - e * x[i]);
            *reinterpret_cast<f32x4_t *>(xl + xt * kXP + xc) = x;
        }
        lds_barrier();
        // U = inverse (b X), 16 rows a wave
        const float last = gl[kChunk - 1], rest = gd[kChunk - 1];
        f32x4_t y = {0.f, 0.f, 0.f, 0.f};
        for (int kk = 0; kk <= w; ++kk) {
            const f32x4_t a = load4(tl + (16 * w + c) * kPitch + 16 * kk + 4 * u);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                y = mma4(a[i], xl[(16 * kk + 4 * u + i) * kXP + c], y);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * w + 4 * u + i;
            ug[((int64_t)ch * kChunk + t) * sv + c] = y[i];
            ul[t * kXP + c] = decay(last, rest, gl[t], gd[t]) * y[i];
        }
        const float keep = exp_f(last);
        lds_barrier();
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            S[j] *= keep;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 16 * tb + 4 * u + i;
                    S[j] = mma4(kl[t * kKP + 16 * (NB * w + j) + c], ul[t * kXP + c], S[j]);
                }
        }
        lds_barrier();
    }
    if (p.state_out && v0 + c < p.Dv)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 16 * (NB * w + j) + 4 * u + i;
                if (r < p.Dk)
                    p.state_out[(head * p.Dk + r) * p.Dv + v0 + c] = S[j][i];
            }
}

// O of every chunk, transposed (a lane holds four columns of one token).
template <typename T, int DKP>
__global__ __launch_bounds__(kThreads) void delta_out_kernel(DeltaProblem p, DeltaKept kept, int nc, int sv)
{
    constexpr int kKP = DKP + 4;
    __shared__ __attribute__((aligned(16))) float ql[kChunk * kKP], al[kChunk * kPitch];
    __shared__ float gl[kChunk];
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int ch = id % nc;
    id /= nc;
    const int hv = id % p.Hv, b = id / p.Hv;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int t0 = ch * kChunk, n = max(0, min(kChunk, delta_len(p, b) - t0)), hq = hv / (p.Hv / p.Hq);
    const T *q = static_cast<const T *>(p.q.p) + b * p.q.sb + hq * p.q.sh + (int64_t)t0 * p.q.st;
    const T *k = static_cast<const T *>(p.k.p) + b * p.k.sb + hq * p.k.sh + (int64_t)t0 * p.k.st;
    T *o = static_cast<T *>(p.o.p) + b * p.o.sb + hv * p.o.sh + (int64_t)t0 * p.o.st;
    const int64_t at = ((int64_t)b * p.Hv + hv) * nc + ch;
    const float *S = kept.s + at * DKP * sv, *U = kept.u + at * kChunk * sv;

    Rows<T, DKP> qr;
    qr.load(q, p.q.st, n, p.Dk);
    qr.store(ql);
    Gates x = load_gates(p, b, hv, t0, n, l);
    sum_gates(x, l);
    if (w == 0)
        gl[l] = x.G;
    if (w < 3) {
        constexpr int kPer = 16 / (int)sizeof(T);
        const int c2 = l % 32, h2 = l / 32, rb = w > 0, cb = w == 2;
        f32x16_t qk;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            qk[r] = 0.f;
        for (int s = 0; s * 2 * kPer < p.Dk; ++s) {
            Frag<T> a = {}, d = {};
            if (32 * rb + c2 < n)
                a = row_frag(q + (32 * rb + c2) * p.q.st, 2 * s + h2, p.Dk);
            if (32 * cb + c2 < n)
                d = row_frag(k + (32 * cb + c2) * p.k.st, 2 * s + h2, p.Dk);
            qk = mma(a, d, qk);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int t = 32 * rb + 8 * (r / 4) + 4 * h2 + r % 4, s = 32 * cb + c2;
            const float gt = __shfl(x.G, t), gs = __shfl(x.G, s), dt = __shfl(x.D, t), ds = __shfl(x.D, s);
            al[t * kPitch + s] = s <= t ? p.scale * decay(gt, dt, gs, ds) * qk[r] : 0.f;
        }
    }
    lds_barrier();
    for (int vb = w; vb < sv / 16; vb += 4) {
        f32x4_t acc[4];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
            acc[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < DKP / 16; ++kb) {
            f32x4_t a;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                a[i] = S[(16 * kb + 4 * u + i) * sv + 16 * vb + c];
#pragma unroll
            for (int tb = 0; tb < 4; ++tb) {
                const f32x4_t d = load4(ql + (16 * tb + c) * kKP + 16 * kb + 4 * u);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[tb] = mma4(a[i], d[i], acc[tb]);
            }
        }
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
            acc[tb] *= p.scale * exp_f(gl[16 * tb + c]);
#pragma unroll
        for (int sb = 0; sb < 4; ++sb) {
            f32x4_t a;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                a[i] = U[(16 * sb + 4 * u + i) * sv + 16 * vb + c];
#pragma unroll
            for (int tb = sb; tb < 4; ++tb) {
                const f32x4_t d = load4(al + (16 * tb + c) * kPitch + 16 * sb + 4 * u);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[tb] = mma4(a[i], d[i], acc[tb]);
            }
        }
        const int d = 16 * vb + 4 * u;
        if (d < p.Dv)
#pragma unroll
            for (int tb = 0; tb < 4; ++tb) {
                const int t = 16 * tb + c;
                const float f = t < n ? 1.f : 0.f;
                if (t0 + t < p.T)
                    store4(o + t * p.o.st + d, acc[tb][0] * f, acc[tb][1] * f, acc[tb][2] * f, acc[tb][3] * f);
            }
    }
}

// The recurrence itself, for few tokens: a workgroup holds kCols columns of a
// state, a thread four columns of some rows.  o_t = exp(g) S^T q + u (k.q), so
// S^T k and S^T q are summed over the threads' rows in one pass.  Bound by memory: a
// token of 64 sequences, 16 heads of 128 x 128, reads and writes 134 MB of states in 31
// us, 4.3 TB/s.
constexpr int kStepCols = 32, kStepRows = kThreads / (kStepCols / 4);   // 8 lanes a row, 32 rows at once

template <typename T, int DKP>
__global__ __launch_bounds__(kThreads) void delta_step_kernel(DeltaProblem p)
{
    constexpr int NR = DKP / kStepRows;
    __shared__ __attribute__((aligned(16))) float sums[4][2][kStepCols];
    const int nv = (p.Dv + kStepCols - 1) / kStepCols;
    int id = blockIdx.x;
    const int v0 = id % nv * kStepCols;
    id /= nv;
    const int hv = id % p.Hv, b = id / p.Hv, hq = hv / (p.Hv / p.Hq);
    const int w = threadIdx.x / 64, r0 = threadIdx.x / 8, c = threadIdx.x % 8 * 4, col = v0 + c;
    const bool in = col < p.Dv;
    const int len = delta_len(p, b);
    const int64_t head = (int64_t)b * p.Hv + hv;
    const T *q = static_cast<const T *>(p.q.p) + b * p.q.sb + hq * p.q.sh;
    const T *k = static_cast<const T *>(p.k.p) + b * p.k.sb + hq * p.k.sh;
    const T *v = static_cast<const T *>(p.v.p) + b * p.v.sb + hv * p.v.sh + col;
    T *o = static_cast<T *>(p.o.p) + b * p.o.sb + hv * p.o.sh + col;

    f32x4_t S[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int r = r0 + i * kStepRows;
        S[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (p.state && in && r < p.Dk)
            S[i] = load4(p.state + (head * p.Dk + r) * p.Dv + col);
    }
    for (int t = 0; t < p.T; ++t) {
        if (t >= len) {
            if (in && r0 == 0)
                store4(o + t * p.o.st, 0.f, 0.f, 0.f, 0.f);
            continue;
        }
        const int64_t at = ((int64_t)b * p.T + t) * p.Hv + hv;
        const float a = exp_f(bounded(at_f(p.g, at, p.dtype))), be = at_f(p.beta, at, p.dtype);
        float kr[NR], qr[NR], kq = 0.f;
        f32x4_t sk = {0.f, 0.f, 0.f, 0.f}, sq = sk;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int r = r0 + i * kStepRows;
            kr[i] = r < p.Dk ? load_f(k + t * p.k.st + r) : 0.f;
            qr[i] = r < p.Dk ? load_f(q + t * p.q.st + r) : 0.f;
            kq = fmaf(kr[i], qr[i], kq);
            sk += kr[i] * S[i];
            sq += qr[i] * S[i];
        }
        f32x4_t vt = {0.f, 0.f, 0.f, 0.f};
        if (in)
            vt = load4(v + t * p.v.st);
        // over the wave's 8 rows of lanes, then the 4 waves
#pragma unroll
        for (int d = 8; d < 64; d *= 2) {
            kq += __shfl_xor(kq, d);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sk[e] += __shfl_xor(sk[e], d);
                sq[e] += __shfl_xor(sq[e], d);
            }
        }
        __shared__ float dots[4];
        if (threadIdx.x % 64 < 8) {
            *reinterpret_cast<f32x4_t *>(&sums[w][0][c]) = sk;
            *reinterpret_cast<f32x4_t *>(&sums[w][1][c]) = sq;
            if (c == 0)
                dots[w] = kq;
        }
        lds_barrier();
        sk = sq = f32x4_t{0.f, 0.f, 0.f, 0.f};
        kq = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            sk += load4(&sums[x][0][c]);
            sq += load4(&sums[x][1][c]);
            kq += dots[x];
        }
        const f32x4_t u = be * (vt - a * sk);
#pragma unroll
        for (int i = 0; i < NR; ++i)
            S[i] = a * S[i] + kr[i] * u;
        if (in && r0 == 0) {
            const f32x4_t y = p.scale * (a * sq + kq * u);
            store4(o + t * p.o.st, y[0], y[1], y[2], y[3]);
        }
        lds_barrier();
    }
    if (p.state_out && in)
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int r = r0 + i * kStepRows;
            if (r < p.Dk)
                store4(p.state_out + (head * p.Dk + r) * p.Dv + col, S[i][0], S[i][1], S[i][2], S[i][3]);
        }
}

template <typename T, int DKP>
hipError_t run(const DeltaProblem &p, hipStream_t s)
{
    const int nc = delta_chunks(p), sv = delta_sv(p);
    const int64_t heads = (int64_t)p.B * p.Hv;
    DeltaKept kept;
    hipError_t e = take_delta_kept(p, p.rs ? p.rs : p.ws, &kept);
    if (heads * nc * kThreads > kMaxThreads || heads * (sv / 16) * kThreads > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (e != hipSuccess || p.ws->counting)
        return e;
    delta_inverse_kernel<T><<<dim3((unsigned)((heads * nc + 3) / 4)), kThreads, 0, s>>>(p, kept.inv, nc);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    delta_state_kernel<T, DKP><<<dim3((unsigned)(heads * (sv / 16))), kThreads, 0, s>>>(p, kept, nc, sv);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    delta_out_kernel<T, DKP><<<dim3((unsigned)(heads * nc)), kThreads, 0, s>>>(p, kept, nc, sv);
    return hipGetLastError();
}

template <typename T, int DKP>
hipError_t step(const DeltaProblem &p, hipStream_t s)
{
    const int64_t n = (int64_t)p.B * p.Hv * ((p.Dv + kStepCols - 1) / kStepCols);
    if (n * kThreads > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (p.ws->counting)
        return hipSuccess;
    delta_step_kernel<T, DKP><<<dim3((unsigned)n), kThreads, 0, s>>>(p);
    return hipGetLastError();
}

// Tokens up to which the recurrence itself runs: it keeps its state in
// registers and writes no intermediate.  In chunks any number up to 64 takes 30 us for
// 16 heads of 128 x 128, the recurrence 2.2 and 1.4 a token (8 tokens 18, 16 tokens 33);
// for 64 sequences 122, and 9 a token behind 28 (8 tokens 89, 16 tokens 163).
constexpr int kFewTokens = 8;

template <typename T>
hipError_t few(const DeltaProblem &p, hipStream_t s)
{
    return p.Dk <= 64 ? step<T, 64>(p, s) : step<T, 128>(p, s);
}

}  // namespace

hipError_t launch_delta_fwd(const DeltaProblem &p, hipStream_t s)
{
    if (!p.rs && p.T <= kFewTokens)
        return p.dtype == 0 ? few<float>(p, s) : few<bf16_t>(p, s);
    if (p.dtype != 0)
        return launch_delta16_fwd(p, s);
    return p.Dk <= 64 ? run<float, 64>(p, s) : run<float, 128>(p, s);
}

}  // namespace gspn
