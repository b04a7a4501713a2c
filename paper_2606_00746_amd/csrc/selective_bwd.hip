// The selective state space scan, backward (gspn_selective_scan_bwd_reserve).
//
// With d the step, u = d x, a_t = 2^(d A log2 e), dy' = dy silu(z) and g_t the gradient of h_t:
//   g_t = C_t dy' + a_{t+1} g_{t+1},  q = g_t a_t h_{t-1}
//   dB = sum over channels of g u, dC = sum over channels of h dy'
//   du = g . B,  dx = du d + D dy',  dd = q . A + du x,  dA = sum of q d,  dz = dy (C . h + D x) silu'(z)
//
// Chunks of tokens, as forward: what each chunk passes on from a gradient of zero behind it,
// a chain over the chunks from the last, and the chunks again.  There a lane holds some
// channels and a quarter of their states, so that the sums over states take two exchanges
// and the sums over channels begin inside a lane; these are formed in LDS for several tokens
// at once, over the channels of a workgroup.  The states come from the forward's reserve for
// every kSelKeep-th token, and from there again into registers.  8 x 4096 tokens of 1536
// channels, 16 states, bf16: what chunks pass on 170 us, the gradients 637; these are bound by
// the vector units, 23 instructions a state and token and 83% of the cycles.
#include <algorithm>

#include "selective_dev.hpp"

namespace gspn {
namespace {

using namespace sel;

constexpr int kBlk = 256, K = kSelKeep;

struct Chunks {
    int n, len;     // how many, tokens of each (a multiple of kSelKeep)
    int waves;      // waves that a group's channels take a lane a channel
    int blocks;     // workgroups of the gradient kernel that they take
};

// ---------------------------------------------------------------------------
// what a chunk passes on, and the chain
// ---------------------------------------------------------------------------

// A lane a channel: g from 0 behind the chunk's last token to ahead of its first.  Chunks 1 ..
// Addresses and loads ahead as in the forward.
template <typename T, int NP, bool Z>
__global__ __launch_bounds__(64) void back_kernel(SelectiveProblem p, Chunks ch, const float *bc, float *ends, float *steps)
{
    constexpr int U = K;
    const int per = p.G * ch.waves;
    const int gb = (int)(blockIdx.x % per), kb = (int)(blockIdx.x / per);
    const int k = 1 + kb % (ch.n - 1), b = kb / (ch.n - 1), g = gb / ch.waves;
    const int cpg = p.C / p.G, c0 = gb % ch.waves * 64;
    const bool on = c0 + (int)threadIdx.x < cpg;
    const uint32_t l = g * cpg + (on ? c0 + threadIdx.x : 0), off = l * (uint32_t)sizeof(T);
    const int t0 = k * ch.len, te = max(t0, min(min(t0 + ch.len, p.T), length_of(p, b)));
    const bool soft = p.softplus;
    const float bias = p.dt_bias ? p.dt_bias[l] : 0.f;
    float A2[NP], G[NP], sum = 0.f;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        A2[n] = n < p.N ? rate(p.A[(int64_t)l * p.N + n]) : 0.f;
        G[n] = 0.f;
    }
    // C from the last token on, a part of the states at a time, as B and C in the forward; a
    // token's ahead of the first is read too
    constexpr int P = NP < 16 ? NP : 16;
    const int mstep = p.G * 2 * NP;
    cfloat *m = constant(bc) + ((((int64_t)b * p.T + te) * p.G + g) * 2 + 1) * NP;
    float Ct[P];
#pragma unroll
    for (int n = 0; n < P; ++n)
        Ct[n] = m[n];
    const auto token = [&](uint32_t dr, uint32_t zr, uint32_t yr) {
        const float raw = widened<T>(dr) + bias, sp = softplus(raw), d = soft ? sp : raw;
        float up = widened<T>(yr);
        if (Z)
            up *= silu(widened<T>(zr));
        sum += d;
#pragma unroll
        for (int q = 0; q < NP; q += P) {
            float nC[P];
            cfloat *const next = q + P < NP ? m + q + P : m - mstep;
#pragma unroll
            for (int n = 0; n < P; ++n)
                nC[n] = next[n];
            step_fence();
#pragma unroll
            for (int n = 0; n < P; ++n)
                G[q + n] = exp2_hw(d * A2[q + n]) * fmaf(Ct[n], up, G[q + n]);
            step_fence();
#pragma unroll
            for (int n = 0; n < P; ++n)
                Ct[n] = nC[n];
        }
        m -= mstep;
    };
    const int last = max(te - 1, t0);
    RowAt<T> dt(p.dt, b, last), z(Z ? p.z : p.dt, b, last), dy(p.dy, b, last);
    dt.step = -dt.step, z.step = -z.step, dy.step = -dy.step;
    uint32_t dr[U], zr[U], yr[U];
    const auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            dr[i] = dt.load(off), yr[i] = dy.load(off), zr[i] = Z ? z.load(off) : 0;
            dt.next(), dy.next();
            if (Z)
                z.next();
        }
    };
    const int full = (te - t0) / U;
    if (full > 0)
        fetch();
    for (int blk = 0; blk < full; ++blk) {
        uint32_t dc[U], zc[U], yc[U];
#pragma unroll
        for (int i = 0; i < U; ++i)
            dc[i] = dr[i], zc[i] = zr[i], yc[i] = yr[i];
        if (blk + 1 < full)
            fetch();
#pragma unroll
        for (int i = 0; i < U; ++i)
            token(dc[i], zc[i], yc[i]);
    }
    for (int t = te - full * U; t > t0; --t) {
        token(dt.load(off), Z ? z.load(off) : 0, dy.load(off));
        dt.next(), dy.next();
        if (Z)
            z.next();
    }
    if (!on)
        return;
    const int64_t slot = (((int64_t)b * ch.n + k) * NP) * p.C;
#pragma unroll
    for (int n = 0; n < NP; ++n)
        (ends + slot + (int64_t)n * p.C)[l] = G[n];
    steps[((int64_t)b * ch.n + k) * p.C + l] = sum;
}

// ---------------------------------------------------------------------------
// the gradients
// ---------------------------------------------------------------------------

// Shares of a workgroup: part_bc[b][t][g][block][B, C][states], part_a[b][chunk][states][C],
// part_d[b][chunk][D, bias][C].
struct Parts {
    float *bc, *a, *d;
};

// Lane 4 q + s: channels CH q .. of its wave's 16 CH, states NS s .. of 4 NS.
// Z: with a gate.  PAD: fewer states than 4 NS; those past N stay 0.
template <typename T, int NS, int CH, bool Z, bool PAD>
__global__ __launch_bounds__(kBlk) void selective_grad_kernel(SelectiveProblem p, Chunks ch, const float *bc, const float *kept, const float *ends, Parts parts)
{
    constexpr int NP = 4 * NS, CW = 16 * CH, V = 2 * CH;   // states; channels of a wave; a lane's, of a token, at the ends
    constexpr int TR = NS <= 4 ? 8 : 32 / NS;                // tokens whose sums are formed at once
    __shared__ float4 tok_[4][3][K][CW / 4];                // d, u, dy' of a wave's tokens; then C . h, du, dd
    __shared__ float4 mat_[2][K][2][NS];                    // B and C of the tokens; zeros
    __shared__ float4 red_[4][TR][2][NS][16];               // a wave's terms of dB and dC: float4 over s

    int64_t at = blockIdx.x;
    const int per = p.G * ch.blocks;
    const int gb = (int)(at % per);
    at /= per;
    const int k = (int)(at % ch.n), b = (int)(at / ch.n), g = gb / ch.blocks, blk = gb % ch.blocks;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, s = lane % 4, q = lane / 4;
    const int cpg = p.C / p.G, w0 = (blk * 4 + wave) * CW;   // the wave's first channel in the group
    const int len = length_of(p, b), t0 = k * ch.len, t1 = min(t0 + ch.len, p.T);
    float(*const dts)[CW] = reinterpret_cast<float(*)[CW]>(&tok_[wave][0][0][0]);
    float(*const us)[CW] = reinterpret_cast<float(*)[CW]>(&tok_[wave][1][0][0]);
    float(*const ups)[CW] = reinterpret_cast<float(*)[CW]>(&tok_[wave][2][0][0]);
    float *const mat = reinterpret_cast<float *>(mat_);

    // in the scan: channels cq .., states n0 ..
    const bool qon = w0 + q * CH < cpg;
    const int cq = g * cpg + (qon ? w0 + q * CH : 0), n0 = s * NS;
    float A2[CH][NS], G[CH][NS], dA[CH][NS];
#pragma unroll
    for (int e = 0; e < CH; ++e)
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const bool in = qon && n0 + i < p.N;
            A2[e][i] = in ? rate(p.A[(int64_t)(cq + e) * p.N + n0 + i]) : 0.f;
            dA[e][i] = 0.f;
            if (ch.n > 1)
                G[e][i] = in ? ends[(((int64_t)b * ch.n + k) * NP + n0 + i) * p.C + cq + e] : 0.f;
            else
                G[e][i] = in && p.dstate ? p.dstate[((int64_t)b * p.C + cq + e) * p.N + n0 + i] : 0.f;
        }
    // lanes without a channel have B and C of 0: what they add to the sums over channels is 0 then,
    // which with its own 0s it is not where B or C is infinite
    for (int i = threadIdx.x; i < K * 2 * NP; i += kBlk)
        mat[K * 2 * NP + i] = 0.f;
    const float *const mine = mat + (qon ? 0 : K * 2 * NP) + n0;

    // ahead of the scan and behind it: token lane / 8, channels cv ..
    const int tl = lane / 8, cl = lane % 8 * V;
    const bool von = w0 + cl < cpg;
    const int cv = g * cpg + (von ? w0 + cl : 0);
    float dD[V] = {}, db[V] = {};
    const bool soft = p.softplus;
    const T *x = static_cast<const T *>(p.x.p) + b * p.x.sb + cv;
    const T *dt = static_cast<const T *>(p.dt.p) + b * p.dt.sb + cv;
    const T *z = Z ? static_cast<const T *>(p.z.p) + b * p.z.sb + cv : nullptr;
    const T *dy = static_cast<const T *>(p.dy.p) + b * p.dy.sb + cv;
    const int nkept = (p.T + K - 1) / K;

    // a block of tokens past the sequence: gradients of 0
    int tb = t0 + (t1 - 1 - t0) / K * K;
    const int64_t out_step = (int64_t)p.G * ch.blocks * 2 * NP;
    const auto sums_at = [&](int t) { return parts.bc + ((((int64_t)b * p.T + t) * p.G + g) * ch.blocks + blk) * 2 * NP; };
    for (; tb >= t0 && tb >= len; tb -= K) {
        const int t = tb + tl;
        const float none[V] = {};
        if (von && t < t1) {
            store_all(static_cast<T *>(p.dx.p) + b * p.dx.sb + t * p.dx.st + cv, none);
            store_all(static_cast<T *>(p.ddt.p) + b * p.ddt.sb + t * p.ddt.st + cv, none);
            if (Z)
                store_all(static_cast<T *>(p.dz.p) + b * p.dz.sb + t * p.dz.st + cv, none);
        }
        for (int i = threadIdx.x; i < K * 2 * NP; i += kBlk)
            if (tb + i / (2 * NP) < t1)
                sums_at(tb)[i / (2 * NP) * out_step + i % (2 * NP)] = 0.f;
    }
    // what a block reads, asked for while the one behind it is worked on
    constexpr int MR = (K * 2 * NP + kBlk - 1) / kBlk;
    Raw<T, V> xn, dn, yn, zn;
    Raw<float, CH> hn[NS];
    float mn[MR];
    const auto fetch = [&](int at) {
        const int t = at + tl;
        const bool live = von && t < len;
        xn = live ? load_raw<T, V>(x + t * p.x.st) : zero_raw<T, V>();
        dn = live ? load_raw<T, V>(dt + t * p.dt.st) : zero_raw<T, V>();
        yn = live ? load_raw<T, V>(dy + t * p.dy.st) : zero_raw<T, V>();
        zn = Z && live ? load_raw<T, V>(z + t * p.z.st) : zero_raw<T, V>();
#pragma unroll
        for (int i = 0; i < NS; ++i)
            hn[i] = load_raw<float, CH>(kept + ((int64_t)(b * (int64_t)nkept + at / K) * NP + n0 + i) * p.C + cq);
#pragma unroll
        for (int j = 0; j < MR; ++j) {
            const int i = threadIdx.x + j * kBlk, ti = at + i / (2 * NP);
            mn[j] = i < K * 2 * NP && ti < p.T ? bc[(((int64_t)b * p.T + ti + 1) * p.G + g) * 2 * NP + i % (2 * NP)] : 0.f;
        }
    };
    if (tb >= t0)
        fetch(tb);
    for (; tb >= t0; tb -= K) {
        const int t = tb + tl;
        const bool live = von && t < len;
        float *const out_bc = sums_at(tb);
        const Raw<T, V> xr = xn, dr = dn, yr = yn, zr = zn;
        float first[CH][NS];
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int e = 0; e < CH; ++e)
                first[e][i] = qon ? get(hn[i], e) : 0.f;
#pragma unroll
        for (int j = 0; j < MR; ++j)
            if ((int)threadIdx.x + j * kBlk < K * 2 * NP)
                mat[threadIdx.x + j * kBlk] = mn[j];
        float bias[V] = {}, skip[V] = {};
        if (p.dt_bias)
            load_all<float, V>(p.dt_bias + cv, bias);
        // of dd and C . h + D x: what ddt and dz are of them; 0 where there is no token
        float d[V], u[V], up[V], fd[V], fz[V];
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float raw = get(dr, e) + bias[e];
            float grad;
            const float v = softplus(raw, grad);
            d[e] = live ? (soft ? v : raw) : 0.f;
            fd[e] = live ? (soft ? grad : 1.f) : 0.f;
            u[e] = d[e] * get(xr, e);
            up[e] = get(yr, e);
            if (Z) {
                fz[e] = up[e];
                up[e] *= silu(get(zr, e), grad);
                fz[e] *= grad;
            }
            if (PAD)
                most = fmaxf(fmaxf(most, fabsf(d[e])), fmaxf(fabsf(u[e]), fabsf(up[e])));
        }
        const bool odd = PAD && any_infinite(most);
        put_lds(&dts[tl][cl], d);
        put_lds(&us[tl][cl], u);
        put_lds(&ups[tl][cl], up);
        if (p.D)
            load_all<float, V>(p.D + cv, skip);
        lds_barrier();
        if (tb > t0)
            fetch(tb - K);

        // the block's states, and their terms, TR tokens at a time; odd: where inputs are infinite
        float h[K][CH][NS];
        const auto states = [&](auto odd_block) {
#pragma unroll
            for (int j = 0; j < K; ++j) {
                float dv[CH], uv[CH], Bv[NS];
                step_fence();
                asm volatile("" ::: "memory");   // read again for each token: kept, they take the registers of more waves
                get_lds(&dts[j][q * CH], dv);
                get_lds(&us[j][q * CH], uv);
                get_lds(mine + j * 2 * NP, Bv);
#pragma unroll
                for (int e = 0; e < CH; ++e)
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        const float v = fmaf(exp2_hw(dv[e] * A2[e][i]), j ? h[j - 1][e][i] : first[e][i], uv[e] * Bv[i]);
                        h[j][e][i] = !odd_block || n0 + i < p.N ? v : 0.f;
                    }
            }
        };
        if (PAD && odd)
            states(std::true_type{});
        else
            states(std::false_type{});
        const auto terms = [&](auto odd_block, int jr) {
#pragma unroll
            for (int jj = TR - 1; jj >= 0; --jj) {
                const int j = jr + jj;
                if (tb + j >= len)   // no token: a state that is not finite would reach dA
                    continue;
                float dv[CH], uv[CH], gv[CH], Bv[NS], Cv[NS];
                step_fence();
                asm volatile("" ::: "memory");
                get_lds(&dts[j][q * CH], dv);
                get_lds(&us[j][q * CH], uv);
                get_lds(&ups[j][q * CH], gv);
                get_lds(mine + j * 2 * NP, Bv);
                get_lds(mine + j * 2 * NP + NP, Cv);
                float tB[NS] = {}, tC[NS] = {}, res[CH];
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    float yh = 0.f, du = 0.f, dd = 0.f;
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        const bool in = !odd_block || n0 + i < p.N;
                        const float gt = in ? fmaf(Cv[i], gv[e], G[e][i]) : 0.f;
                        if (Z)
                            yh = fmaf(Cv[i], h[j][e][i], yh);
                        du = fmaf(gt, Bv[i], du);
                        tB[i] = fmaf(gt, uv[e], tB[i]);
                        tC[i] = fmaf(h[j][e][i], gv[e], tC[i]);
                        G[e][i] = in ? exp2_hw(dv[e] * A2[e][i]) * gt : 0.f;
                        const float w = G[e][i] * (j ? h[j - 1][e][i] : first[e][i]);
                        dd = fmaf(w, A2[e][i], dd);
                        dA[e][i] = fmaf(w, dv[e], dA[e][i]);
                        asm volatile("" : "+v"(dA[e][i]));   // here, not behind the block with every w kept
                    }
                    // over the quad: du's sum to lane 0, dd's to lane 1, C . h's to lane 2
                    const float own = in_lanes(du, dd, kOddLanes) + dpp<kXor1>(in_lanes(dd, du, kOddLanes));
                    if (Z) {
                        yh += dpp<kXor1>(yh);
                        res[e] = in_lanes(own, yh, kOddPairs) + dpp<kXor2>(in_lanes(yh, own, kOddPairs));
                    } else {
                        res[e] = own + dpp<kXor2>(own);
                    }
                }
                // over d, u and dy' of the token, which have been read
                if (s < 2 + Z)
                    put_lds(&dts[s * K + j][q * CH], res);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    reinterpret_cast<float *>(&red_[wave][jj][0][i][0])[lane] = tB[i];
                    reinterpret_cast<float *>(&red_[wave][jj][1][i][0])[lane] = tC[i];
                }
            }
        };
#pragma unroll
        for (int jr = K - TR; jr >= 0; jr -= TR) {
            if (PAD && odd)
                terms(std::true_type{}, jr);
            else
                terms(std::false_type{}, jr);
            lds_barrier();
            // a row of 16 float4 a token, matrix and i: float4 (over s) q of all waves; RT threads a row
            constexpr int rows = TR * 2 * NS, RT = kBlk / rows >= 16 ? 16 : kBlk / rows;
            if ((int)threadIdx.x < rows * RT) {
                const int row = threadIdx.x / RT, part = threadIdx.x % RT;
                float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < 4; ++w)
#pragma unroll
                    for (int i = 0; i < 16 / RT; ++i) {
                        // rows begin at different q, so that neighbouring rows lie in different banks
                        const float4 f = (&red_[w][0][0][0][0])[row * 16 + (i * RT + part + RT * row) % 16];
                        a.x += f.x, a.y += f.y, a.z += f.z, a.w += f.w;
                    }
                a.x = lanes_sum(a.x, RT), a.y = lanes_sum(a.y, RT), a.z = lanes_sum(a.z, RT), a.w = lanes_sum(a.w, RT);
                const int i = row % NS, m = row / NS % 2, j = jr + row / NS / 2;
                if (part == 0 && tb + j < t1) {
                    float *to = out_bc + j * out_step + m * NP + i;
                    if (tb + j >= len)   // also where a state is not finite
                        a = make_float4(0.f, 0.f, 0.f, 0.f);
                    if constexpr (NS == 1) {   // neighbours: one store, with its wait states
                        const float row[4] = {a.x, a.y, a.z, a.w};
                        store_all(to, row);
                    } else {
                        to[0] = a.x, to[NS] = a.y, to[2 * NS] = a.z, to[3 * NS] = a.w;
                    }
                }
            }
            if (jr > 0)
                lds_barrier();
        }

        float du[V], dd[V], yh[V];
        get_lds(&dts[tl][cl], du);
        get_lds(&dts[K + tl][cl], dd);
        if (Z)
            get_lds(&dts[2 * K + tl][cl], yh);
        float odx[V], odt[V], odz[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float xv = get(xr, e);
            // 0 where there is no token, also where what it is taken times is not finite
            odx[e] = live ? fmaf(du[e], d[e], skip[e] * up[e]) : 0.f;
            odt[e] = fd[e] != 0.f ? fmaf(dd[e], kLn2, du[e] * xv) * fd[e] : 0.f;
            if (Z)
                odz[e] = live ? fmaf(skip[e], xv, yh[e]) * fz[e] : 0.f;
            dD[e] = fmaf(up[e], xv, dD[e]);
            db[e] += odt[e];
            asm volatile("" : "+v"(dD[e]), "+v"(db[e]));
        }
        if (von && t < t1) {
            store_all(static_cast<T *>(p.dx.p) + b * p.dx.sb + t * p.dx.st + cv, odx);
            store_all(static_cast<T *>(p.ddt.p) + b * p.ddt.sb + t * p.ddt.st + cv, odt);
            if (Z)
                store_all(static_cast<T *>(p.dz.p) + b * p.dz.sb + t * p.dz.st + cv, odz);
        }
    }

    const int64_t slot = (int64_t)b * ch.n + k;
    if (qon)
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            float f[CH];
#pragma unroll
            for (int e = 0; e < CH; ++e)
                f[e] = dA[e][i];
            store_all(parts.a + (slot * NP + n0 + i) * p.C + cq, f);
        }
    if (k == 0 && p.dstate_in && qon)
#pragma unroll
        for (int e = 0; e < CH; ++e)
#pragma unroll
            for (int i = 0; i < NS; ++i)
                if (n0 + i < p.N)
                    p.dstate_in[((int64_t)b * p.C + cq + e) * p.N + n0 + i] = G[e][i];
#pragma unroll
    for (int e = 0; e < V; ++e) {   // over the lanes of a channel's tokens
        dD[e] += __shfl_xor(dD[e], 8), db[e] += __shfl_xor(db[e], 8);
        dD[e] += __shfl_xor(dD[e], 16), db[e] += __shfl_xor(db[e], 16);
        dD[e] += __shfl_xor(dD[e], 32), db[e] += __shfl_xor(db[e], 32);
    }
    if (lane < 8 && von) {
        store_all(parts.d + slot * 2 * p.C + cv, dD);
        store_all(parts.d + (slot * 2 + 1) * p.C + cv, db);
    }
}

// ---------------------------------------------------------------------------
// sums of the workgroups' shares, in order
// ---------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(kBlk) void selective_sum_bc_kernel(SelectiveProblem p, int np, int parts, int blocks, const float *part)
{
    const int b = (int)(blockIdx.x / (unsigned)parts), t0 = (int)(blockIdx.x % (unsigned)parts) * kPackTokens, row = p.G * 2 * np;
    const int n = min(kPackTokens, p.T - t0) * row;
    const float *const from = part + ((int64_t)b * p.T + t0) * row * blocks;
    for (int i = threadIdx.x; i < n; i += kBlk) {
        const int s = i % (2 * np), gt = i / (2 * np), g = gt % p.G, t = t0 + gt / p.G;
        if (s % np >= p.N)
            continue;
        const float *in = from + (int64_t)gt * blocks * 2 * np + s;
        float a = 0.f;
#pragma unroll 4
        for (int k = 0; k < blocks; ++k)
            a += in[(int64_t)k * 2 * np];
        const Heads &m = s < np ? p.dBm : p.dCm;
        store_f(static_cast<T *>(m.p) + b * m.sb + t * m.st + g * m.sh + s % np, a);
    }
}

// Rows 0 .. states - 1 of shares: dA; the next two dD and ddt_bias.  16 channels a workgroup,
// whose rows of threads add every 64th share, eight in flight, then their sums in order.
constexpr int kSumRows = 64;
__global__ __launch_bounds__(16 * kSumRows) void selective_sum_channels_kernel(SelectiveProblem p, int np, int shares, Parts parts)
{
    __shared__ float sums[kSumRows][17];
    const int r = blockIdx.y, c = blockIdx.x * 16 + threadIdx.x % 16, i0 = threadIdx.x / 16;
    const bool a_row = r < p.N;
    const float *in = a_row ? parts.a + (int64_t)r * p.C + c : parts.d + (int64_t)(r - p.N) * p.C + c;
    const int64_t step = (int64_t)(a_row ? np : 2) * p.C;
    float s = 0.f;
    if (c < p.C)
        for (int i = i0; i < shares; i += 8 * kSumRows) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                x[k] = i + k * kSumRows < shares ? in[(i + k * kSumRows) * step] : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                s += x[k];
        }
    sums[i0][threadIdx.x % 16] = s;
    __syncthreads();
    if (i0 == 0 && c < p.C) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < kSumRows; ++i)
            a += sums[i][threadIdx.x];
        if (a_row && p.dA)
            p.dA[(int64_t)c * p.N + r] = a;
        if (r == p.N && p.dD)
            p.dD[c] = a;
        if (r == p.N + 1 && p.ddt_bias)
            p.ddt_bias[c] = a;
    }
}

// Waves of the first pass that the chunks are cut for (8 x 4096 tokens of 1536 channels, the
// whole call, us, 4096, 6144 and 8192: 867, 842 and 883).
constexpr int64_t kWaves = 6144;

template <typename T, int NP, bool PAD>
hipError_t bwd(const SelectiveProblem &p, hipStream_t s)
{
    constexpr int NS = NP / 4, CH = NS <= 4 ? 2 : 1;
    Chunks ch;
    const int cpg = p.C / p.G;
    ch.waves = (cpg + 63) / 64;
    ch.blocks = (cpg + 64 * CH - 1) / (64 * CH);
    const int64_t waves = (int64_t)p.B * p.G * ch.waves, want = std::max<int64_t>(1, kWaves / waves);
    const int64_t len = std::max(least_tokens(p.T), (p.T + want - 1) / want);
    ch.len = (int)((len + K - 1) / K * K);
    ch.n = (p.T + ch.len - 1) / ch.len;
    const int64_t groups = (int64_t)p.B * p.G * ch.blocks * ch.n, passes = (int64_t)p.B * p.G * ch.waves * (ch.n - 1);
    if (groups * kBlk > kMaxThreads || passes * 64 > kMaxThreads || (ch.n > 1 && p.B > 65535) ||
        sel_pack_groups(p) * kBlk > kMaxThreads)
        return hipErrorInvalidConfiguration;
    void *bc = nullptr, *ends = nullptr, *steps = nullptr, *kept = nullptr, *pbc = nullptr, *pa = nullptr, *pd = nullptr;
    const int64_t slots = (int64_t)p.B * ch.n, tokens = (int64_t)p.B * p.T * p.G;
    hipError_t e = take_sel_kept(p, p.rs, &kept, &bc);
    if (e == hipSuccess && ch.n > 1)
        e = p.ws->take(&ends, (size_t)slots * NP * p.C * 4);
    if (e == hipSuccess && ch.n > 1)
        e = p.ws->take(&steps, (size_t)slots * p.C * 4);
    if (e == hipSuccess)
        e = p.ws->take(&pbc, (size_t)tokens * ch.blocks * 2 * NP * 4);
    if (e == hipSuccess)
        e = p.ws->take(&pa, (size_t)slots * NP * p.C * 4);
    if (e == hipSuccess)
        e = p.ws->take(&pd, (size_t)slots * 2 * p.C * 4);
    if (e != hipSuccess || p.ws->counting)
        return e;
    const float *const m = static_cast<const float *>(bc);
    float *const en = static_cast<float *>(ends), *const sm = static_cast<float *>(steps);
    const Parts parts{static_cast<float *>(pbc), static_cast<float *>(pa), static_cast<float *>(pd)};
    if (ch.n > 1) {
        if (p.z.p)
            back_kernel<T, NP, true><<<dim3((unsigned)passes), 64, 0, s>>>(p, ch, m, en, sm);
        else
            back_kernel<T, NP, false><<<dim3((unsigned)passes), 64, 0, s>>>(p, ch, m, en, sm);
        e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        e = join_chunks<NP, true>(p, ch.n, en, sm, p.dstate, s);
    }
    if (e != hipSuccess)
        return e;
    if (p.z.p)
        selective_grad_kernel<T, NS, CH, true, PAD><<<dim3((unsigned)groups), kBlk, 0, s>>>(p, ch, m, static_cast<const float *>(kept), en, parts);
    else
        selective_grad_kernel<T, NS, CH, false, PAD><<<dim3((unsigned)groups), kBlk, 0, s>>>(p, ch, m, static_cast<const float *>(kept), en, parts);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    selective_sum_bc_kernel<T><<<dim3((unsigned)sel_pack_groups(p)), kBlk, 0, s>>>(p, NP, (p.T + kPackTokens - 1) / kPackTokens, ch.blocks, parts.bc);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    selective_sum_channels_kernel<<<dim3((unsigned)((p.C + 15) / 16), (unsigned)(p.N + 2)), 16 * kSumRows, 0, s>>>(p, NP, (int)slots, parts);
    return hipGetLastError();
}

template <typename T>
hipError_t pick(const SelectiveProblem &p, hipStream_t s)
{
    const int np = sel_states(p);
    const bool pad = p.N < np;
    switch (np) {
    case 4: return pad ? bwd<T, 4, true>(p, s) : bwd<T, 4, false>(p, s);
    case 8: return pad ? bwd<T, 8, true>(p, s) : bwd<T, 8, false>(p, s);
    case 16: return pad ? bwd<T, 16, true>(p, s) : bwd<T, 16, false>(p, s);
    case 32: return pad ? bwd<T, 32, true>(p, s) : bwd<T, 32, false>(p, s);
    default: return pad ? bwd<T, 64, true>(p, s) : bwd<T, 64, false>(p, s);
    }
}

}  // namespace

hipError_t launch_selective_bwd(const SelectiveProblem &p, hipStream_t s)
{
    return p.dtype == 0 ? pick<float>(p, s) : pick<bf16_t>(p, s);
}

}  // namespace gspn
