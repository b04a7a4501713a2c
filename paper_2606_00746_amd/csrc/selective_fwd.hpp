// The selective state space scan, forward (gspn_selective_scan_fwd, _fwd_train), of one
// storage type.
//
// A lane holds a channel with all its states: h_t = 2^(d A log2 e) h_{t-1} + d x B_t and
// y = C_t . h need nothing of another lane, and B and C of a token, the same for all
// channels of a group, are scalars.  A state and token take a product, an exponential, a
// product, two multiply-adds: bound by the vector units, not by memory (34225 tokens of 2304
// channels, 16 states, bf16: first pass 225 us, outputs 287, vector units active 88 and 92%
// of the cycles; their bytes alone would take 113).
#pragma once

#include <algorithm>

#include "selective_dev.hpp"

namespace gspn {
namespace {

using namespace sel;

constexpr int kBlk = 256;

// ---------------------------------------------------------------------------
// B and C as fp32
// ---------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(kBlk) void pack_kernel(SelectiveProblem p, int np, int parts, float *bc)
{
    const int b = (int)(blockIdx.x / (unsigned)parts), t0 = (int)(blockIdx.x % (unsigned)parts) * kPackTokens, row = p.G * 2 * np;
    const int len = length_of(p, b), n = min(kPackTokens, p.T - t0) * row;
    float *const to = bc + ((int64_t)b * p.T + t0 + 1) * row;
    for (int i = threadIdx.x; i < n; i += kBlk) {
        const int s = i % np, gs = i / np, g = gs % (2 * p.G) / 2, t = t0 + gs / (2 * p.G);
        const Heads &m = gs & 1 ? p.Cm : p.Bm;
        to[i] = s < p.N && t < len ? load_f(static_cast<const T *>(m.p) + b * m.sb + t * m.st + g * m.sh + s) : 0.f;
    }
}

template <typename T>
hipError_t launch_pack(const SelectiveProblem &p, float *bc, hipStream_t s)
{
    const int np = sel_states(p), parts = (p.T + kPackTokens - 1) / kPackTokens;
    pack_kernel<T><<<(unsigned)sel_pack_groups(p), kBlk, 0, s>>>(p, np, parts, bc);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// chunks of tokens
// ---------------------------------------------------------------------------

struct Chunks {
    int n, len;     // how many, tokens of each (a multiple of kSelKeep)
    int blocks;     // waves that a group's channels take
};

// OUT: the outputs, from `starts`, or from the sequence's state where there is one chunk.
// Otherwise what the chunk adds to its states from zeros, into `starts`, and the sum of
// its steps.  Z: with a gate.  KEEP: with the states of every kSelKeep-th token.  PAD: fewer
// states than NP, of which those past N stay 0.
//
// Rows' addresses are a scalar and the lane's channel; eight tokens are in flight ahead of
// the eight that are worked on, B and C of a token one token ahead: they are what the scalar
// registers hold, and loads from its beginning come too late (64 x 64, us: C from the token's
// beginning 281, a token ahead 255).
template <typename T, int NP, bool OUT, bool Z, bool KEEP, bool PAD>
__global__ __launch_bounds__(64) void chunk_kernel(SelectiveProblem p, Chunks ch, const float *bc, float *starts, float *steps, float *kept)
{
    constexpr int U = kSelKeep;
    const int per = p.G * ch.blocks, nch = OUT ? ch.n : ch.n - 1;
    const int gb = (int)(blockIdx.x % per), kb = (int)(blockIdx.x / per);
    const int k = kb % nch, b = kb / nch, g = gb / ch.blocks;
    const int cpg = p.C / p.G, c0 = gb % ch.blocks * 64;
    const bool on = c0 + (int)threadIdx.x < cpg;
    const uint32_t l = g * cpg + (on ? c0 + threadIdx.x : 0), off = l * (uint32_t)sizeof(T);
    const int t0 = k * ch.len, te = max(t0, min(min(t0 + ch.len, p.T), length_of(p, b)));
    const bool soft = p.softplus;
    const float bias = p.dt_bias ? p.dt_bias[l] : 0.f, skip = OUT && p.D ? p.D[l] : 0.f;
    float A2[NP], h[NP], sum = 0.f;
    const int64_t slot = (((int64_t)b * ch.n + k) * NP) * p.C;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        A2[n] = n < p.N ? rate(p.A[(int64_t)l * p.N + n]) : 0.f;
        if (!OUT)
            h[n] = 0.f;
        else if (ch.n > 1)
            h[n] = PAD && n >= p.N ? 0.f : (starts + slot + (int64_t)n * p.C)[l];
        else
            h[n] = p.state && n < p.N ? p.state[((int64_t)b * p.C + l) * p.N + n] : 0.f;
    }

    // B and C of the states of a part, the next part's asked for ahead of it: 16 states are what
    // the scalar registers hold twice.  A token's behind the last is read too (the buffer has
    // room).
    constexpr int P = NP < 16 ? NP : 16;
    cfloat *m = constant(bc) + (((int64_t)b * p.T + t0 + 1) * p.G + g) * 2 * NP;
    const int mstep = p.G * 2 * NP;
    float Bt[P], Ct[P];
#pragma unroll
    for (int n = 0; n < P; ++n)
        Bt[n] = m[n], Ct[n] = OUT ? m[NP + n] : 0.f;
    const auto token = [&](uint32_t xr, uint32_t dr, uint32_t zr, const RowAt<T> &to) {
        const float xv = widened<T>(xr), raw = widened<T>(dr) + bias, sp = softplus(raw), d = soft ? sp : raw, u = d * xv;
        float out = skip * xv;
        if (!OUT)
            sum += d;
#pragma unroll
        for (int q = 0; q < NP; q += P) {
            float nB[P], nC[P];
            cfloat *const next = q + P < NP ? m + q + P : m + mstep;
#pragma unroll
            for (int n = 0; n < P; ++n)
                nB[n] = next[n], nC[n] = OUT ? next[NP + n] : 0.f;
            step_fence();
#pragma unroll
            for (int n = 0; n < P; ++n) {
                h[q + n] = fmaf(exp2_hw(d * A2[q + n]), h[q + n], u * Bt[n]);
                if (OUT && !PAD)
                    out = fmaf(Ct[n], h[q + n], out);
            }
            if (PAD) {
                if (any_infinite(u))
#pragma unroll
                    for (int n = 0; n < P; ++n)
                        h[q + n] = q + n < p.N ? h[q + n] : 0.f;
#pragma unroll
                for (int n = 0; n < P; ++n)
                    out = fmaf(Ct[n], h[q + n], out);
            }
            if (OUT && q + P == NP) {
                if (Z)
                    out *= silu(widened<T>(zr));
                if (on)
                    to.store(off, out);
            }
            step_fence();
#pragma unroll
            for (int n = 0; n < P; ++n)
                Bt[n] = nB[n], Ct[n] = nC[n];
        }
        m += mstep;
    };

    RowAt<T> x(p.x, b, t0), dt(p.dt, b, t0), z(Z ? p.z : p.x, b, t0), y(OUT ? p.y : p.x, b, t0);
    const int64_t keep_step = (int64_t)NP * p.C;
    float *keep = kept;
    if (KEEP)
        keep += ((int64_t)b * ((p.T + U - 1) / U) + t0 / U) * keep_step;
    const auto put_states = [&]() {
        if (KEEP) {
            if (on)
#pragma unroll
                for (int n = 0; n < NP; ++n)
                    (keep + (int64_t)n * p.C)[l] = h[n];
            keep += keep_step;
        }
    };
    const int full = (te - t0) / U;
    uint32_t xr[U], dr[U], zr[U];
    const auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            xr[i] = x.load(off), dr[i] = dt.load(off), zr[i] = OUT && Z ? z.load(off) : 0;
            x.next(), dt.next();
            if (OUT && Z)
                z.next();
        }
    };
    if (full > 0)
        fetch();
    for (int blk = 0; blk < full; ++blk) {
        uint32_t xc[U], dc[U], zc[U];
#pragma unroll
        for (int i = 0; i < U; ++i)
            xc[i] = xr[i], dc[i] = dr[i], zc[i] = zr[i];
        if (blk + 1 < full)
            fetch();
        put_states();   // behind the loads, whose waits are not for these stores then
#pragma unroll
        for (int i = 0; i < U; ++i) {
            token(xc[i], dc[i], zc[i], y);
            if (OUT)
                y.next();
        }
    }
    int t = t0 + full * U;
    if (t < te)
        put_states();
    for (; t < te; ++t) {
        token(x.load(off), dt.load(off), OUT && Z ? z.load(off) : 0, y);
        x.next(), dt.next();
        if (OUT && Z)
            z.next();
        if (OUT)
            y.next();
    }
    if (!on)
        return;
    if (OUT) {
        for (; t < min(t0 + ch.len, p.T); ++t, y.next())
            y.store(off, 0.f);
        if (k == ch.n - 1 && p.state_out)
#pragma unroll
            for (int n = 0; n < NP; ++n)
                if (n < p.N)
                    p.state_out[((int64_t)b * p.C + l) * p.N + n] = h[n];
    } else {
#pragma unroll
        for (int n = 0; n < NP; ++n)
            (starts + slot + (int64_t)n * p.C)[l] = h[n];
        steps[((int64_t)b * ch.n + k) * p.C + l] = sum;
    }
}

// ---------------------------------------------------------------------------
// whole sequences in one pass: four lanes a channel
// ---------------------------------------------------------------------------

// A quad of lanes holds a channel, a quarter of its states each, and goes along the whole
// sequence: no chunk is gone through twice.  Of four tokens lane s has token s's entries of x,
// dt and z, whose step it forms for the quad (one exchange inside the multiplication that
// takes it), and is left with token s's sum over the states.  B and C of eight tokens come
// through the wave's own piece of LDS, one wide load a lane.
template <typename T, int NP, bool Z, bool KEEP, bool PAD>
__global__ __launch_bounds__(kBlk) void quad_kernel(SelectiveProblem p, int blocks, const float *bc, float *kept)
{
    constexpr int NS = NP / 4, U = kSelKeep, TB = NS <= 4 ? 4 : 16 / NS;   // TB: tokens whose B and C are read at once
    const int item = blockIdx.x * (kBlk / 64) + (int)__builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int per = p.G * blocks, gb = item % per, b = item / per, g = gb / blocks;
    if (b >= p.B)
        return;
    const int lane = threadIdx.x % 64, s = lane % 4, cpg = p.C / p.G, ci = gb % blocks * 16 + lane / 4;
    const bool on = ci < cpg, soft = p.softplus;
    const int c = g * cpg + (on ? ci : 0), n0 = s * NS, te = length_of(p, b);
    const float bias = p.dt_bias ? p.dt_bias[c] : 0.f, skip = p.D ? p.D[c] : 0.f;
    const int64_t st = ((int64_t)b * p.C + c) * p.N + n0;
    float A2[NS], h[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
        const bool in = n0 + n < p.N;
        A2[n] = in ? rate(p.A[(int64_t)c * p.N + n0 + n]) : 0.f;
        h[n] = in && p.state ? p.state[st + n] : 0.f;
    }
    const T *x = static_cast<const T *>(p.x.p) + b * p.x.sb + s * p.x.st + c;
    const T *dt = static_cast<const T *>(p.dt.p) + b * p.dt.sb + s * p.dt.st + c;
    const T *z = Z ? static_cast<const T *>(p.z.p) + b * p.z.sb + s * p.z.st + c : nullptr;
    T *y = static_cast<T *>(p.y.p) + b * p.y.sb + s * p.y.st + c;
    constexpr int MR = (U * NP / 2 + 63) / 64;   // float4s of B and C of U tokens, a lane
    __shared__ float4 mat_[kBlk / 64][U][NP / 2];
    float(*const mat)[2 * NP] = reinterpret_cast<float(*)[2 * NP]>(&mat_[threadIdx.x / 64][0][0]);
    const float *const mats = bc + (((int64_t)b * p.T + 1) * p.G + g) * 2 * NP;
    float *keep = KEEP ? kept + ((int64_t)b * ((p.T + U - 1) / U) * NP + n0) * p.C + c : nullptr;

    uint32_t xn[U / 4], dn[U / 4], zn[U / 4];
    const auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < U / 4; ++i) {
            const bool live = t + 4 * i + s < te;
            xn[i] = live ? load_raw<T, 1>(x + (int64_t)(t + 4 * i) * p.x.st).w[0] : 0;
            dn[i] = live ? load_raw<T, 1>(dt + (int64_t)(t + 4 * i) * p.dt.st).w[0] : 0;
            zn[i] = Z && live ? load_raw<T, 1>(z + (int64_t)(t + 4 * i) * p.z.st).w[0] : 0;
        }
    };
    Raw<float, 4> mn[MR];
    const auto fetch_mats = [&](int t) {   // of tokens past the last: zeros
#pragma unroll
        for (int j = 0; j < MR; ++j) {
            const int i = lane + 64 * j, at = t + i / (NP / 2);
            mn[j] = at < p.T && (NP >= 16 || i < U * NP / 2) ? load_raw<float, 4>(mats + (int64_t)at * p.G * 2 * NP + i % (NP / 2) * 4)
                                                             : zero_raw<float, 4>();
        }
    };
    fetch(0);
    fetch_mats(0);
    for (int t = 0; t < te; t += U) {
        if (KEEP) {
            if (on)
#pragma unroll
                for (int n = 0; n < NS; ++n)
                    keep[(int64_t)n * p.C] = h[n];
            keep += (int64_t)NP * p.C;
        }
        float xv[U / 4], d[U / 4], u[U / 4], gate[U / 4];
#pragma unroll
        for (int i = 0; i < U / 4; ++i) {
            const bool live = t + 4 * i + s < te;
            xv[i] = widened<T>(xn[i]);
            const float raw = widened<T>(dn[i]) + bias, sp = softplus(raw);
            d[i] = live ? (soft ? sp : raw) : 0.f;
            u[i] = d[i] * xv[i];
            gate[i] = Z ? silu(widened<T>(zn[i])) : 1.f;
        }
#pragma unroll
        for (int j = 0; j < MR; ++j)
            if (NP >= 16 || lane + 64 * j < U * NP / 2) {
                float f[4];
                widen_all(mn[j], f);
                put_lds(&mat[0][0] + 4 * (lane + 64 * j), f);
            }
        fetch(t + U);
        fetch_mats(t + U);
#pragma unroll
        for (int i = 0; i < U / 4; ++i) {
            const bool odd = PAD && any_infinite(u[i]);
            float sum[4];
#pragma unroll
            for (int k0 = 0; k0 < 4; k0 += TB) {
                float Bt[TB][NS], Ct[TB][NS];
#pragma unroll
                for (int j = 0; j < TB; ++j) {
                    get_lds(&mat[4 * i + k0 + j][n0], Bt[j]);
                    get_lds(&mat[4 * i + k0 + j][NP + n0], Ct[j]);
                }
                const auto token = [&](auto kc) {
                    constexpr int k = decltype(kc)::value, j = k % TB;
                    const float dk = dpp<k * 0x55>(d[i]), uk = dpp<k * 0x55>(u[i]);
                    sum[k] = 0.f;
#pragma unroll
                    for (int n = 0; n < NS; ++n) {
                        h[n] = fmaf(exp2_hw(dk * A2[n]), h[n], uk * Bt[j][n]);
                        if (!PAD)
                            sum[k] = fmaf(Ct[j][n], h[n], sum[k]);
                    }
                    if (PAD) {
                        if (odd)
#pragma unroll
                            for (int n = 0; n < NS; ++n)
                                h[n] = n0 + n < p.N ? h[n] : 0.f;
#pragma unroll
                        for (int n = 0; n < NS; ++n)
                            sum[k] = fmaf(Ct[j][n], h[n], sum[k]);
                    }
                };
                if (k0 == 0)
                    token(std::integral_constant<int, 0>{});
                if (k0 <= 1 && 1 < k0 + TB)
                    token(std::integral_constant<int, 1>{});
                if (k0 <= 2 && 2 < k0 + TB)
                    token(std::integral_constant<int, 2>{});
                if (k0 <= 3 && 3 < k0 + TB)
                    token(std::integral_constant<int, 3>{});
            }
            // lane s: token s over the quad
            const float a = in_lanes(sum[0], sum[1], kOddLanes) + dpp<kXor1>(in_lanes(sum[1], sum[0], kOddLanes));
            const float e = in_lanes(sum[2], sum[3], kOddLanes) + dpp<kXor1>(in_lanes(sum[3], sum[2], kOddLanes));
            float out = in_lanes(a, e, kOddPairs) + dpp<kXor2>(in_lanes(e, a, kOddPairs));
            out = fmaf(skip, xv[i], out);
            if (Z)
                out *= gate[i];
            const int at = t + 4 * i + s;
            if (on && at < p.T)
                store_f(y + (int64_t)(t + 4 * i) * p.y.st, at < te ? out : 0.f);
            step_fence();
        }
    }
    if (!on)
        return;
    for (int t = (te + U - 1) / U * U; t + s < p.T; t += 4)
        store_f(y + (int64_t)t * p.y.st, 0.f);
    if (p.state_out)
#pragma unroll
        for (int n = 0; n < NS; ++n)
            if (n0 + n < p.N)
                p.state_out[st + n] = h[n];
}

// ---------------------------------------------------------------------------
// a few tokens: four lanes a channel, B and C as they lie
// ---------------------------------------------------------------------------

constexpr int kFewTokens = 8;

template <typename T, int NP>
__global__ __launch_bounds__(kBlk) void token_kernel(SelectiveProblem p)
{
    constexpr int NS = NP / 4;   // states of a lane
    const int64_t i = ((int64_t)blockIdx.x * kBlk + threadIdx.x) / 4;
    if (i >= (int64_t)p.B * p.C)
        return;
    const int s = threadIdx.x % 4, c = (int)(i % p.C), b = (int)(i / p.C), g = c / (p.C / p.G), n0 = s * NS;
    const int te = length_of(p, b);
    const T *x = static_cast<const T *>(p.x.p) + b * p.x.sb + c;
    const T *dt = static_cast<const T *>(p.dt.p) + b * p.dt.sb + c;
    const T *z = p.z.p ? static_cast<const T *>(p.z.p) + b * p.z.sb + c : nullptr;
    const T *Bm = static_cast<const T *>(p.Bm.p) + b * p.Bm.sb + g * p.Bm.sh + n0;
    const T *Cm = static_cast<const T *>(p.Cm.p) + b * p.Cm.sb + g * p.Cm.sh + n0;
    T *y = static_cast<T *>(p.y.p) + b * p.y.sb + c;
    const float bias = p.dt_bias ? p.dt_bias[c] : 0.f, skip = p.D ? p.D[c] : 0.f;
    const float *A = p.A + (int64_t)c * p.N + n0, *from = p.state ? p.state + i * p.N + n0 : nullptr;
    float A2[NS], h[NS];
    if (NS % 4 == 0 && p.N == NP) {
        load_all<float, NS>(A, A2);
        widen_all(from ? load_raw<float, NS>(from) : zero_raw<float, NS>(), h);
    } else {
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            A2[n] = n0 + n < p.N ? A[n] : 0.f;
            h[n] = from && n0 + n < p.N ? from[n] : 0.f;
        }
    }
#pragma unroll
    for (int n = 0; n < NS; ++n)
        A2[n] = rate(A2[n]);
    for (int t = 0; t < p.T; ++t) {
        float out = 0.f, xv = 0.f;
        if (t < te) {
            xv = load_f(x + (int64_t)t * p.x.st);
            const float raw = load_f(dt + (int64_t)t * p.dt.st) + bias;
            const float d = p.softplus ? softplus(raw) : raw, u = d * xv;
#pragma unroll
            for (int n = 0; n < NS; ++n)
                if (n0 + n < p.N) {
                    h[n] = fmaf(exp2_hw(d * A2[n]), h[n], u * load_f(Bm + (int64_t)t * p.Bm.st + n));
                    out = fmaf(load_f(Cm + (int64_t)t * p.Cm.st + n), h[n], out);
                }
        }
        out += dpp<kXor1>(out);
        out += dpp<kXor2>(out);
        if (t < te) {
            out = fmaf(skip, xv, out);
            if (z)
                out *= silu(load_f(z + (int64_t)t * p.z.st));
        }
        if (s == 0)
            store_f(y + (int64_t)t * p.y.st, out);
    }
    if (p.state_out) {
        float *to = p.state_out + i * p.N + n0;
        if (NS % 4 == 0 && p.N == NP)
            store_all(to, h);
        else
#pragma unroll
            for (int n = 0; n < NS; ++n)
                if (n0 + n < p.N)
                    to[n] = h[n];
    }
}

// Waves that the chunks of a call are cut for (us, 4096, 6144, 8192 and 12288: 34225 tokens of
// 2304 channels 619, 561, 543 and 562; 8 x 4096 of 1536 383, 362, 385 and 359; 4 x 8191 of
// 768, 8 states, fp32, 152, 162, 157 and 169).
constexpr int64_t kWaves = 8192;

Chunks chunks_of(const SelectiveProblem &p)
{
    Chunks c;
    c.blocks = (p.C / p.G + 63) / 64;
    const int64_t waves = (int64_t)p.B * p.G * c.blocks, want = std::max<int64_t>(1, kWaves / waves);
    const int64_t len = std::max(least_tokens(p.T), (p.T + want - 1) / want);
    c.len = (int)((len + kSelKeep - 1) / kSelKeep * kSelKeep);
    c.n = (p.T + c.len - 1) / c.len;
    return c;
}

template <typename T, int NP, bool PAD>
hipError_t one_pass(const SelectiveProblem &p, hipStream_t s)
{
    const int blocks = (p.C / p.G + 15) / 16;
    const int64_t groups = ((int64_t)p.B * p.G * blocks + 3) / 4;
    if (groups * kBlk > kMaxThreads || sel_pack_groups(p) * kBlk > kMaxThreads)
        return hipErrorInvalidConfiguration;
    void *bc = nullptr, *kept = nullptr;
    hipError_t e = p.rs ? take_sel_kept(p, p.rs, &kept, &bc) : p.ws->take(&bc, sel_packed(p));
    if (e != hipSuccess || p.ws->counting)
        return e;
    float *const m = static_cast<float *>(bc), *const k = static_cast<float *>(kept);
    e = launch_pack<T>(p, m, s);
    if (e != hipSuccess)
        return e;
    const dim3 grid((unsigned)groups);
    if (k && p.z.p)
        quad_kernel<T, NP, true, true, PAD><<<grid, kBlk, 0, s>>>(p, blocks, m, k);
    else if (k)
        quad_kernel<T, NP, false, true, PAD><<<grid, kBlk, 0, s>>>(p, blocks, m, k);
    else if (p.z.p)
        quad_kernel<T, NP, true, false, PAD><<<grid, kBlk, 0, s>>>(p, blocks, m, nullptr);
    else
        quad_kernel<T, NP, false, false, PAD><<<grid, kBlk, 0, s>>>(p, blocks, m, nullptr);
    return hipGetLastError();
}

template <typename T, int NP, bool PAD>
hipError_t fwd(const SelectiveProblem &p, hipStream_t s)
{
    if constexpr (NP >= 4) {   // fewer states are held as four there
        if (p.T <= kFewTokens && !p.rs) {
            const int64_t n = ((int64_t)p.B * p.C * 4 + kBlk - 1) / kBlk;
            if (n * kBlk > kMaxThreads)
                return hipErrorInvalidConfiguration;
            if (p.ws->counting)
                return hipSuccess;
            token_kernel<T, NP><<<dim3((unsigned)n), kBlk, 0, s>>>(p);
            return hipGetLastError();
        }
        if (sel_one_pass(p))
            return one_pass<T, NP, PAD>(p, s);
    }
    const Chunks ch = chunks_of(p);
    const int64_t waves = (int64_t)p.B * p.G * ch.blocks * ch.n;
    if (waves * 64 > kMaxThreads || (ch.n > 1 && p.B > 65535) || sel_pack_groups(p) * kBlk > kMaxThreads)
        return hipErrorInvalidConfiguration;
    void *bc = nullptr, *starts = nullptr, *steps = nullptr, *kept = nullptr;
    hipError_t e = p.rs ? take_sel_kept(p, p.rs, &kept, &bc) : p.ws->take(&bc, sel_packed(p));
    if (e == hipSuccess && ch.n > 1)
        e = p.ws->take(&starts, (size_t)p.B * ch.n * NP * p.C * 4);
    if (e == hipSuccess && ch.n > 1)
        e = p.ws->take(&steps, (size_t)p.B * ch.n * p.C * 4);
    if (e != hipSuccess || p.ws->counting)
        return e;
    float *const m = static_cast<float *>(bc), *const st = static_cast<float *>(starts), *const sm = static_cast<float *>(steps);
    e = launch_pack<T>(p, m, s);
    if (e == hipSuccess && ch.n > 1) {
        chunk_kernel<T, NP, false, false, false, false><<<dim3((unsigned)(waves / ch.n * (ch.n - 1))), 64, 0, s>>>(p, ch, m, st, sm, nullptr);
        e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        e = join_chunks<NP, false>(p, ch.n, st, sm, p.state, s);
    }
    if (e != hipSuccess)
        return e;
    const dim3 grid((unsigned)waves);
    float *const kp = static_cast<float *>(kept);
    if constexpr (NP >= 4)
        if (kp) {
            if (p.z.p)
                chunk_kernel<T, NP, true, true, true, PAD><<<grid, 64, 0, s>>>(p, ch, m, st, sm, kp);
            else
                chunk_kernel<T, NP, true, false, true, PAD><<<grid, 64, 0, s>>>(p, ch, m, st, sm, kp);
            return hipGetLastError();
        }
    if (p.z.p)
        chunk_kernel<T, NP, true, true, false, PAD><<<grid, 64, 0, s>>>(p, ch, m, st, sm, nullptr);
    else
        chunk_kernel<T, NP, true, false, false, PAD><<<grid, 64, 0, s>>>(p, ch, m, st, sm, nullptr);
    return hipGetLastError();
}

template <typename T>
hipError_t pick(const SelectiveProblem &p, hipStream_t s)
{
    const int np = sel_states(p);
    const bool pad = p.N < np;
    switch (np) {
    case 1: return fwd<T, 1, false>(p, s);
    case 2: return fwd<T, 2, false>(p, s);
    case 4: return pad ? fwd<T, 4, true>(p, s) : fwd<T, 4, false>(p, s);
    case 8: return pad ? fwd<T, 8, true>(p, s) : fwd<T, 8, false>(p, s);
    case 16: return pad ? fwd<T, 16, true>(p, s) : fwd<T, 16, false>(p, s);
    case 32: return pad ? fwd<T, 32, true>(p, s) : fwd<T, 32, false>(p, s);
    default: return pad ? fwd<T, 64, true>(p, s) : fwd<T, 64, false>(p, s);
    }
}

}  // namespace

}  // namespace gspn
