// Gradient of the gated delta rule (gspn_delta_rule_bwd_reserve); see delta.hpp.
#include <algorithm>

#include "delta.hpp"

namespace gspn {
namespace {

using namespace delta;

// What the backward adds to what the forward left, per (b, head, chunk):
// scale A^T dO, then R [64][Sv]; the gradient of the state behind the chunk
// [DKP][Sv].
struct DeltaGrads {
    float *r = nullptr, *ds = nullptr;
};

// scale A^T dO of every chunk, transposed like the outputs.
template <typename T>
__global__ __launch_bounds__(kThreads) void delta_du_kernel(DeltaProblem p, float *du, int nc, int sv)
{
    __shared__ __attribute__((aligned(16))) float al[kChunk * kPitch];
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int ch = id % nc;
    id /= nc;
    const int hv = id % p.Hv, b = id / p.Hv;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int t0 = ch * kChunk, n = max(0, min(kChunk, delta_len(p, b) - t0)), hq = hv / (p.Hv / p.Hq);
    const T *q = static_cast<const T *>(p.q.p) + b * p.q.sb + hq * p.q.sh + (int64_t)t0 * p.q.st;
    const T *k = static_cast<const T *>(p.k.p) + b * p.k.sb + hq * p.k.sh + (int64_t)t0 * p.k.st;
    const T *d = static_cast<const T *>(p.dout.p) + b * p.dout.sb + hv * p.dout.sh + (int64_t)t0 * p.dout.st;
    float *out = du + (((int64_t)b * p.Hv + hv) * nc + ch) * kChunk * sv;
    Gates x = load_gates(p, b, hv, t0, n, l);
    sum_gates(x, l);
    if (w < 3) {
        constexpr int kPer = 16 / (int)sizeof(T);
        const int c2 = l % 32, h2 = l / 32, rb = w > 0, cb = w == 2;
        f32x16_t qk;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            qk[r] = 0.f;
        for (int s = 0; s * 2 * kPer < p.Dk; ++s) {
            Frag<T> a = {}, e = {};
            if (32 * rb + c2 < n)
                a = row_frag(q + (32 * rb + c2) * p.q.st, 2 * s + h2, p.Dk);
            if (32 * cb + c2 < n)
                e = row_frag(k + (32 * cb + c2) * p.k.st, 2 * s + h2, p.Dk);
            qk = mma(a, e, qk);
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
        for (int sb = 0; sb < 4; ++sb)
            acc[sb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        const bool in = 16 * vb + c < p.Dv;
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
            f32x4_t a;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 16 * tb + 4 * u + i;
                a[i] = in && t < n ? load_f(d + t * p.dout.st + 16 * vb + c) : 0.f;
            }
#pragma unroll
            for (int sb = 0; sb <= tb; ++sb)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[sb] = mma4(a[i], al[(16 * tb + 4 * u + i) * kPitch + 16 * sb + c], acc[sb]);
        }
#pragma unroll
        for (int sb = 0; sb < 4; ++sb)
            store4(out + (16 * sb + c) * sv + 16 * vb + 4 * u, acc[sb][0], acc[sb][1], acc[sb][2], acc[sb][3]);
    }
}

// R, dV and the states' gradients, the chunks from the last on, for 16 columns.
template <typename T, int DKP>
__global__ __launch_bounds__(kThreads) void delta_dstate_kernel(DeltaProblem p, DeltaKept kept, DeltaGrads gr,
                                                                int nc, int sv)
{
    constexpr int NB = DKP / 64, kKP = DKP + 4, kXP = 20;
    __shared__ __attribute__((aligned(16))) float kl[kChunk * kKP], ql[kChunk * kKP], tl[kChunk * kPitch];
    __shared__ __attribute__((aligned(16))) float part[4][kChunk * kXP], xl[kChunk * kXP], zl[kChunk * kXP];
    __shared__ float gl[kChunk], gd[kChunk], bl[kChunk];

    const int nv = sv / 16;
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int v0 = id % nv * 16;
    id /= nv;
    const int hv = id % p.Hv, b = id / p.Hv, hq = hv / (p.Hv / p.Hq);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int len = delta_len(p, b);
    const T *q = static_cast<const T *>(p.q.p) + b * p.q.sb + hq * p.q.sh;
    const T *k = static_cast<const T *>(p.k.p) + b * p.k.sb + hq * p.k.sh;
    const int xt = threadIdx.x / 4, xc = threadIdx.x % 4 * 4;
    const bool vin = v0 + xc < p.Dv;
    const T *d = static_cast<const T *>(p.dout.p) + b * p.dout.sb + hv * p.dout.sh + v0 + xc;
    T *dv = static_cast<T *>(p.dv.p) + b * p.dv.sb + hv * p.dv.sh + v0 + xc;
    const int64_t head = (int64_t)b * p.Hv + hv;
    const float *inv = kept.inv + head * nc * kChunk * kChunk;
    float *rg = gr.r + head * nc * kChunk * sv + v0, *sg = gr.ds + head * nc * DKP * sv + v0;

    f32x4_t S[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 16 * (NB * w + j) + 4 * u + i;
            S[j][i] = p.dstate && r < p.Dk && v0 + c < p.Dv ? p.dstate[(head * p.Dk + r) * p.Dv + v0 + c] : 0.f;
        }

    Rows<T, DKP> kr, qr;
    Square tr;
    Gates gt{0.f, 0.f, 0.f};
    f32x4_t dr, ur;
    const auto fetch = [&](int ch) {
        const int t0 = ch * kChunk, n = max(0, min(kChunk, len - t0));
        kr.load(k + (int64_t)t0 * p.k.st, p.k.st, n, p.Dk);
        qr.load(q + (int64_t)t0 * p.q.st, p.q.st, n, p.Dk);
        tr.load(inv + (int64_t)ch * kChunk * kChunk);
        dr = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (vin && xt < n)
            dr = load4(d + (int64_t)(t0 + xt) * p.dout.st);
        ur = load4(rg + ((int64_t)ch * kChunk + xt) * sv + xc);
        if (w == 0)
            gt = load_gates(p, b, hv, t0, n, l);
    };
    fetch(nc - 1);
    for (int ch = nc - 1; ch >= 0; --ch) {
        kr.store(kl);
        qr.store(ql);
        tr.store(tl);
        if (w == 0) {
            sum_gates(gt, l);
            gl[l] = gt.G;
            gd[l] = gt.D;
            bl[l] = gt.beta;
        }
        const f32x4_t dc = dr, uc = ur;
        lds_barrier();
        if (ch > 0)
            fetch(ch - 1);
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sg[((int64_t)ch * DKP + 16 * (NB * w + j) + 4 * u + i) * sv + c] = S[j][i];
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
        const float last = gl[kChunk - 1], rest = gd[kChunk - 1];
        {
            f32x4_t x = load4(part[0] + xt * kXP + xc);
#pragma unroll
            for (int y = 1; y < 4; ++y)
                x += load4(part[y] + xt * kXP + xc);
            x = uc + decay(last, rest, gl[xt], gd[xt]) * x;
            *reinterpret_cast<f32x4_t *>(xl + xt * kXP + xc) = x;
        }
        lds_barrier();
        // R = inverse^T dU, 16 rows a wave
        f32x4_t y = {0.f, 0.f, 0.f, 0.f};
        for (int kk = w; kk < 4; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 16 * kk + 4 * u + i;
                y = mma4(tl[t * kPitch + 16 * w + c], xl[t * kXP + c], y);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * w + 4 * u + i;
            rg[((int64_t)ch * kChunk + t) * sv + c] = y[i];
            zl[t * kXP + c] = bl[t] * y[i];
        }
        const float keep = exp_f(last);
        lds_barrier();
        {   // dV, and in place of dX and dO what multiplies K and Q
            const f32x4_t z = load4(zl + xt * kXP + xc);
            const int t = ch * kChunk + xt;
            if (vin && t < p.T)
                store4(dv + (int64_t)t * p.dv.st, z[0], z[1], z[2], z[3]);
            const float e = exp_f(gl[xt]);
            *reinterpret_cast<f32x4_t *>(xl + xt * kXP + xc) = (p.scale * e) * dc;
            *reinterpret_cast<f32x4_t *>(part[0] + xt * kXP + xc) = -e * z;
        }
        lds_barrier();
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            S[j] *= keep;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 16 * tb + 4 * u + i, m = 16 * (NB * w + j) + c;
                    S[j] = mma4(kl[t * kKP + m], part[0][t * kXP + c], S[j]);
                    S[j] = mma4(ql[t * kKP + m], xl[t * kXP + c], S[j]);
                }
        }
        lds_barrier();
    }
    if (p.dstate_in && v0 + c < p.Dv)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 16 * (NB * w + j) + 4 * u + i;
                if (r < p.Dk)
                    p.dstate_in[(head * p.Dk + r) * p.Dv + v0 + c] = S[j][i];
            }
}

__device__ __forceinline__ float row16_sum(float v)   // over the 16 lanes of one u
{
#pragma unroll
    for (int d = 1; d < 16; d *= 2)
        v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float col4_sum(float v)    // over the four u of one lane
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// dQ, dK, dg and dbeta of every chunk.  Products over the value columns first
// (C1 = dO U^T and C2 = R U^T as 64 x 64 matrices; S dO^T, S R^T and dS U^T by
// rows of the state), then those over the tokens.  The value heads that share a
// query and key head are taken in turn, so that their sum needs no atomics.
template <typename T, int DKP>
__global__ __launch_bounds__(kThreads, 1) void delta_grad_kernel(DeltaProblem p, DeltaKept kept, DeltaGrads gr,
                                                                 int nc, int sv)
{
    constexpr int NB = DKP / 64, kKP = DKP + 4;
    __shared__ __attribute__((aligned(16))) float ql[kChunk * kKP], kl[kChunk * kKP];
    __shared__ __attribute__((aligned(16))) float pl[kChunk * kPitch], nl[kChunk * kPitch];
    __shared__ float gl[kChunk], gd[kChunk], bl[kChunk], down[4][kChunk], rows[3][kChunk], dots[4][3][kChunk], ss[4];

    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int ch = id % nc;
    id /= nc;
    const int hq = id % p.Hq, b = id / p.Hq, rep = p.Hv / p.Hq;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int t0 = ch * kChunk, n = max(0, min(kChunk, delta_len(p, b) - t0));
    const T *q = static_cast<const T *>(p.q.p) + b * p.q.sb + hq * p.q.sh + (int64_t)t0 * p.q.st;
    const T *k = static_cast<const T *>(p.k.p) + b * p.k.sb + hq * p.k.sh + (int64_t)t0 * p.k.st;

    Rows<T, DKP> x;
    x.load(q, p.q.st, n, p.Dk);
    x.store(ql);
    x.load(k, p.k.st, n, p.Dk);
    x.store(kl);
    f32x4_t dq[NB][4], dk[NB][4];   // transposed: rows 16 (NB w + j) + 4 u + i of token 16 tb + c
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
            dq[j][tb] = dk[j][tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    for (int h = 0; h < rep; ++h) {
        const int hv = hq * rep + h;
        const int64_t at = ((int64_t)b * p.Hv + hv) * nc + ch;
        const float *U = kept.u + at * kChunk * sv, *R = gr.r + at * kChunk * sv;
        const float *S = kept.s + at * DKP * sv, *dS = gr.ds + at * DKP * sv;
        const T *d = static_cast<const T *>(p.dout.p) + b * p.dout.sb + hv * p.dout.sh + (int64_t)t0 * p.dout.st;
        const T *v = static_cast<const T *>(p.v.p) + b * p.v.sb + hv * p.v.sh + (int64_t)t0 * p.v.st;
        // four value columns of a token's dO or v (zero past the ends)
        const auto quad = [&](const T *m, int64_t st, int t, int e) {
            f32x4_t r = {0.f, 0.f, 0.f, 0.f};
            if (t < n && e < p.Dv)
                r = load4(m + t * st + e);
            return r;
        };
        lds_barrier();
        if (w == 0) {
            Gates g = load_gates(p, b, hv, t0, n, l);
            sum_gates(g, l);
            gl[l] = g.G;
            gd[l] = g.D;
            bl[l] = g.beta;
        }
        down[w][l] = 0.f;
        lds_barrier();
        const float last = gl[kChunk - 1], rest = gd[kChunk - 1];

        {   // rows 16 w .. of C1, C2, Q K^T, K K^T, up to the diagonal
            f32x4_t c1[4], c2[4], qk[4], kk[4];
#pragma unroll
            for (int sb = 0; sb < 4; ++sb)
                c1[sb] = c2[sb] = qk[sb] = kk[sb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            for (int e = 4 * u; e < sv; e += 16) {
                const f32x4_t ad = quad(d, p.dout.st, 16 * w + c, e), ar = load4(R + (16 * w + c) * sv + e);
#pragma unroll
                for (int sb = 0; sb < 4; ++sb)
                    if (sb <= w) {
                        const f32x4_t bu = load4(U + (16 * sb + c) * sv + e);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            c1[sb] = mma4(ad[i], bu[i], c1[sb]);
                            c2[sb] = mma4(ar[i], bu[i], c2[sb]);
                        }
                    }
            }
#pragma unroll
            for (int kb = 0; kb < DKP / 16; ++kb) {
                const f32x4_t aq = load4(ql + (16 * w + c) * kKP + 16 * kb + 4 * u);
                const f32x4_t ak = load4(kl + (16 * w + c) * kKP + 16 * kb + 4 * u);
#pragma unroll
                for (int sb = 0; sb < 4; ++sb)
                    if (sb <= w) {
                        const f32x4_t bk = load4(kl + (16 * sb + c) * kKP + 16 * kb + 4 * u);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            qk[sb] = mma4(aq[i], bk[i], qk[sb]);
                            kk[sb] = mma4(ak[i], bk[i], kk[sb]);
                        }
                    }
            }
            float along[4] = {0.f, 0.f, 0.f, 0.f}, db[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int sb = 0; sb < 4; ++sb)
                if (sb <= w) {
                    float col = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = 16 * w + 4 * u + i, s = 16 * sb + c;
                        const float kept_ts = s <= t ? decay(gl[t], gd[t], gl[s], gd[s]) : 0.f;
                        const float strict = s < t ? kept_ts : 0.f;
                        const float pp = p.scale * kept_ts * c1[sb][i], mc = strict * c2[sb][i], nn = -bl[t] * mc;
                        pl[t * kPitch + s] = pp;
                        nl[t * kPitch + s] = nn;
                        const float ef = pp * qk[sb][i] + nn * kk[sb][i];
                        along[i] += ef;
                        col += ef;
                        db[i] -= mc * kk[sb][i];
                    }
                    col = col4_sum(col);
                    if (u == 0)
                        down[w][16 * sb + c] = col;
                }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                along[i] = row16_sum(along[i]);
                db[i] = row16_sum(db[i]);
                if (c == 0) {
                    rows[0][16 * w + 4 * u + i] = along[i];
                    rows[1][16 * w + 4 * u + i] = db[i];
                }
            }
        }
        {   // R.v of a token, by 4 lanes
            const int t = threadIdx.x / 4;
            float s = 0.f;
            for (int e = threadIdx.x % 4 * 4; e < p.Dv; e += 16) {
                const f32x4_t a = load4(R + t * sv + e), y = quad(v, p.v.st, t, e);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s = fmaf(a[i], y[i], s);
            }
            s += __shfl_xor(s, 1);
            s += __shfl_xor(s, 2);
            if (threadIdx.x % 4 == 0)
                rows[2][t] = s;
        }
        float dot = 0.f;   // <S, dS>
        float qy[4] = {0.f, 0.f, 0.f, 0.f}, ky[4] = {0.f, 0.f, 0.f, 0.f}, kz[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int m0 = 16 * (NB * w + j);
            f32x4_t y1[4], y2[4], y3[4];
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
                y1[tb] = y2[tb] = y3[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            for (int e = 4 * u; e < sv; e += 16) {
                const f32x4_t as = load4(S + (m0 + c) * sv + e), ad = load4(dS + (m0 + c) * sv + e);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    dot = fmaf(as[i], ad[i], dot);
#pragma unroll
                for (int tb = 0; tb < 4; ++tb) {
                    const f32x4_t b1 = quad(d, p.dout.st, 16 * tb + c, e), b2 = load4(R + (16 * tb + c) * sv + e);
                    const f32x4_t b3 = load4(U + (16 * tb + c) * sv + e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        y1[tb] = mma4(as[i], b1[i], y1[tb]);
                        y2[tb] = mma4(as[i], b2[i], y2[tb]);
                        y3[tb] = mma4(ad[i], b3[i], y3[tb]);
                    }
                }
            }
#pragma unroll
            for (int tb = 0; tb < 4; ++tb) {
                const int t = 16 * tb + c;
                const float eg = exp_f(gl[t]), fq = p.scale * eg, fk = bl[t] * eg, fs = decay(last, rest, gl[t], gd[t]);
                const f32x4_t qq = load4(ql + t * kKP + m0 + 4 * u), kx = load4(kl + t * kKP + m0 + 4 * u);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    qy[tb] = fmaf(qq[i], fq * y1[tb][i], qy[tb]);
                    ky[tb] = fmaf(kx[i], eg * y2[tb][i], ky[tb]);
                    kz[tb] = fmaf(kx[i], fs * y3[tb][i], kz[tb]);
                    dq[j][tb][i] += fq * y1[tb][i];
                    dk[j][tb][i] += fs * y3[tb][i] - fk * y2[tb][i];
                }
            }
        }
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
            const float a = col4_sum(qy[tb]), e = col4_sum(ky[tb]), f = col4_sum(kz[tb]);
            if (u == 0) {
                dots[w][0][16 * tb + c] = a;
                dots[w][1][16 * tb + c] = e;
                dots[w][2][16 * tb + c] = f;
            }
        }
        dot = col4_sum(row16_sum(dot));
        if (l == 0)
            ss[w] = dot;
        lds_barrier();
        // over the tokens: dQ^T += K^T P^T, dK^T += Q^T P + K^T (N + N^T)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int m0 = 16 * (NB * w + j);
#pragma unroll
            for (int sb = 0; sb < 4; ++sb) {
                f32x4_t ak, aq;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ak[i] = kl[(16 * sb + 4 * u + i) * kKP + m0 + c];
                    aq[i] = ql[(16 * sb + 4 * u + i) * kKP + m0 + c];
                }
#pragma unroll
                for (int tb = 0; tb < 4; ++tb) {
                    if (sb <= tb) {   // rows t = 16 tb + c, columns s of block sb
                        const f32x4_t bp = load4(pl + (16 * tb + c) * kPitch + 16 * sb + 4 * u);
                        const f32x4_t bn = load4(nl + (16 * tb + c) * kPitch + 16 * sb + 4 * u);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            dq[j][tb] = mma4(ak[i], bp[i], dq[j][tb]);
                            dk[j][tb] = mma4(ak[i], bn[i], dk[j][tb]);
                        }
                    }
                    if (tb <= sb)     // rows t of block sb, column s = 16 tb + c
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int t = 16 * sb + 4 * u + i;
                            dk[j][tb] = mma4(aq[i], pl[t * kPitch + 16 * tb + c], dk[j][tb]);
                            dk[j][tb] = mma4(ak[i], nl[t * kPitch + 16 * tb + c], dk[j][tb]);
                        }
                }
            }
        }
        if (w == 0) {   // dbeta and dg, a lane a token
            const float eg = exp_f(last), dt = eg * (((ss[0] + ss[1]) + ss[2]) + ss[3]);
            const auto sum4 = [&](int i) { return ((dots[0][i][l] + dots[1][i][l]) + dots[2][i][l]) + dots[3][i][l]; };
            const float a = sum4(0), e = sum4(1), f = sum4(2);
            float dG = a + rows[0][l] - (((down[0][l] + down[1][l]) + down[2][l]) + down[3][l]) - bl[l] * e - f;
            float all = f;   // the last token's running sum scales the whole state
#pragma unroll
            for (int x2 = 1; x2 < 64; x2 *= 2)
                all += __shfl_xor(all, x2);
            if (l == kChunk - 1)
                dG += all + dt;
            // dg_t = sum of dG from t on
#pragma unroll
            for (int x2 = 1; x2 < 64; x2 *= 2) {
                const float o = __shfl_down(dG, x2);
                if (l + x2 < 64)
                    dG += o;
            }
            if (t0 + l < p.T) {
                const int64_t to = ((int64_t)b * p.T + t0 + l) * p.Hv + hv;
                const bool live = l < n;
                store_f(static_cast<T *>(p.dg) + to, live ? dG : 0.f);
                store_f(static_cast<T *>(p.dbeta) + to, live ? rows[2][l] - e + rows[1][l] : 0.f);
            }
        }
    }
    T *dqo = static_cast<T *>(p.dq.p) + b * p.dq.sb + hq * p.dq.sh + (int64_t)t0 * p.dq.st;
    T *dko = static_cast<T *>(p.dk.p) + b * p.dk.sb + hq * p.dk.sh + (int64_t)t0 * p.dk.st;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
            const int t = 16 * tb + c, m = 16 * (NB * w + j) + 4 * u;
            if (t0 + t < p.T && m < p.Dk) {
                const float f = t < n ? 1.f : 0.f;
                store4(dqo + t * p.dq.st + m, f * dq[j][tb][0], f * dq[j][tb][1], f * dq[j][tb][2], f * dq[j][tb][3]);
                store4(dko + t * p.dk.st + m, f * dk[j][tb][0], f * dk[j][tb][1], f * dk[j][tb][2], f * dk[j][tb][3]);
            }
        }
}

template <typename T, int DKP>
hipError_t run(const DeltaProblem &p, hipStream_t s)
{
    const int nc = delta_chunks(p), sv = delta_sv(p);
    const int64_t heads = (int64_t)p.B * p.Hv, n = heads * nc;
    DeltaKept kept;
    hipError_t e = take_delta_kept(p, p.rs, &kept);
    void *r = nullptr, *ds = nullptr;
    if (e == hipSuccess)
        e = p.ws->take(&r, (size_t)(n * kChunk * sv * 4));
    if (e == hipSuccess)
        e = p.ws->take(&ds, (size_t)(n * DKP * sv * 4));
    if (n * kThreads > kMaxThreads || heads * (sv / 16) * kThreads > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (e != hipSuccess || p.ws->counting)
        return e;
    DeltaGrads g;
    g.r = static_cast<float *>(r);
    g.ds = static_cast<float *>(ds);
    delta_du_kernel<T><<<dim3((unsigned)n), kThreads, 0, s>>>(p, g.r, nc, sv);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    delta_dstate_kernel<T, DKP><<<dim3((unsigned)(heads * (sv / 16))), kThreads, 0, s>>>(p, kept, g, nc, sv);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    delta_grad_kernel<T, DKP><<<dim3((unsigned)((int64_t)p.B * p.Hq * nc)), kThreads, 0, s>>>(p, kept, g, nc, sv);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_bwd(const DeltaProblem &p, hipStream_t s)
{
    if (p.dtype != 0)
        return launch_delta16_bwd(p, s);
    return p.Dk <= 64 ? run<float, 64>(p, s) : run<float, 128>(p, s);
}

}  // namespace gspn
