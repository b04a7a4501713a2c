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
// every kSelKeep-th token, and from there again into registers.
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
template <typename T, int NP>
__global__ __launch_bounds__(64) void back_kernel(SelectiveProblem p, Chunks ch, const float *bc, float *ends, float *steps)
{
    int64_t at = blockIdx.x;
    const int per = p.G * ch.waves;
    const int gb = (int)(at % per);
    at /= per;
    const int k = 1 + (int)(at % (ch.n - 1)), b = (int)(at / (ch.n - 1)), g = gb / ch.waves;
    const int cpg = p.C / p.G, ci = gb % ch.waves * 64 + threadIdx.x;
    const bool on = ci < cpg;
    const int c = g * cpg + min(ci, cpg - 1);
    const int t0 = k * ch.len, te = min(min(t0 + ch.len, p.T), length_of(p, b));

    const T *dt = static_cast<const T *>(p.dt.p) + b * p.dt.sb + c;
    const T *z = p.z.p ? static_cast<const T *>(p.z.p) + b * p.z.sb + c : nullptr;
    const T *dy = static_cast<const T *>(p.dy.p) + b * p.dy.sb + c;
    const float bias = p.dt_bias ? p.dt_bias[c] : 0.f;
    float A2[NP], G[NP], sum = 0.f;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        A2[n] = n < p.N ? p.A[(int64_t)c * p.N + n] * kLog2e : 0.f;
        G[n] = 0.f;
    }
    Raw<T, 1> dr[K], zr[K], yr[K];
    const auto fetch = [&](int t) {   // tokens t, t - 1, ..
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const bool live = t - i >= t0;
            dr[i] = live ? load_raw<T, 1>(dt + (int64_t)(t - i) * p.dt.st) : zero_raw<T, 1>();
            yr[i] = live ? load_raw<T, 1>(dy + (int64_t)(t - i) * p.dy.st) : zero_raw<T, 1>();
            zr[i] = live && z ? load_raw<T, 1>(z + (int64_t)(t - i) * p.z.st) : zero_raw<T, 1>();
        }
    };
    fetch(te - 1);
    for (int t = te - 1; t >= t0; t -= K) {
        Raw<T, 1> dc[K], zc[K], yc[K];
#pragma unroll
        for (int i = 0; i < K; ++i)
            dc[i] = dr[i], zc[i] = zr[i], yc[i] = yr[i];
        fetch(t - K);
#pragma unroll
        for (int i = 0; i < K; ++i) {
            if (t - i < t0)
                break;
            cfloat *m = constant(bc) + ((((int64_t)b * p.T + t - i) * p.G + g) * 2 + 1) * NP;
            const float raw = get(dc[i], 0) + bias, d = p.softplus ? softplus(raw) : raw;
            float up = get(yc[i], 0);
            if (z)
                up *= silu(get(zc[i], 0));
            sum += d;
#pragma unroll
            for (int n = 0; n < NP; ++n)
                G[n] = exp2_hw(d * A2[n]) * fmaf(m[n], up, G[n]);
        }
    }
    if (!on)
        return;
    const int64_t slot = (((int64_t)b * ch.n + k) * NP) * p.C + c;
#pragma unroll
    for (int n = 0; n < NP; ++n)
        ends[slot + (int64_t)n * p.C] = G[n];
    steps[((int64_t)b * ch.n + k) * p.C + c] = sum;
}

// From what each chunk passes on to the gradient that arrives behind it, in the same place.
template <int NP>
__global__ __launch_bounds__(kBlk) void back_chain_kernel(SelectiveProblem p, Chunks ch, float *ends, const float *steps)
{
    const int64_t i = (int64_t)blockIdx.x * kBlk + threadIdx.x;
    if (i >= (int64_t)p.B * NP * p.C)
        return;
    const int c = (int)(i % p.C), n = (int)(i / p.C % NP), b = (int)(i / p.C / NP);
    const float a2 = n < p.N ? p.A[(int64_t)c * p.N + n] * kLog2e : 0.f;
    float h = p.dstate && n < p.N ? p.dstate[((int64_t)b * p.C + c) * p.N + n] : 0.f;
    const int64_t step = (int64_t)NP * p.C;
    float *at = ends + (int64_t)b * ch.n * step + (int64_t)n * p.C + c;
    const float *s = steps + (int64_t)b * ch.n * p.C + c;
    constexpr int U = 8;
    for (int k = ch.n - 1; k >= 0; k -= U) {
        float add[U], sum[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const bool in = k - j > 0;
            add[j] = in ? at[(k - j) * step] : 0.f;
            sum[j] = in ? s[(int64_t)(k - j) * p.C] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (k - j >= 0) {
                at[(k - j) * step] = h;
                h = fmaf(exp2_hw(a2 * sum[j]), h, add[j]);
            }
    }
}

// ---------------------------------------------------------------------------
// the gradients
// ---------------------------------------------------------------------------

// V neighbouring floats in LDS.
template <int V>
__device__ __forceinline__ void get_lds(const float *p, float (&f)[V])
{
    if constexpr (V == 1) {
        f[0] = p[0];
    } else if constexpr (V == 2) {
        const float2 u = *reinterpret_cast<const float2 *>(p);
        f[0] = u.x, f[1] = u.y;
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 u = *reinterpret_cast<const float4 *>(p + i);
            f[i] = u.x, f[i + 1] = u.y, f[i + 2] = u.z, f[i + 3] = u.w;
        }
    }
}
template <int V>
__device__ __forceinline__ void put_lds(float *p, const float (&f)[V])
{
    if constexpr (V == 1)
        p[0] = f[0];
    else if constexpr (V == 2)
        *reinterpret_cast<float2 *>(p) = make_float2(f[0], f[1]);
    else
#pragma unroll
        for (int i = 0; i < V; i += 4)
            *reinterpret_cast<float4 *>(p + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
}

// Shares of a workgroup: part_bc[b][t][g][block][B, C][states], part_a[b][chunk][states][C],
// part_d[b][chunk][D, bias][C].
struct Parts {
    float *bc, *a, *d;
};

// Lane 4 q + s: channels CH q .. of its wave's 16 CH, states NS s .. of 4 NS.
template <typename T, int NS, int CH>
__global__ __launch_bounds__(kBlk) void grad_kernel(SelectiveProblem p, Chunks ch, const float *bc, const float *kept, const float *ends, Parts parts)
{
    constexpr int NP = 4 * NS, CW = 16 * CH, V = 2 * CH;   // states; channels of a wave; a lane's, of a token, at the ends
    constexpr int TR = NS >= 16 ? 1 : NS <= 2 ? 8 : 16 / NS;   // tokens whose sums are formed at once
    __shared__ float4 tok_[4][3][K][CW / 4];                // d, u, dy' of a wave's tokens; then C . h, du, dd
    __shared__ float4 mat_[K][2][NS];                       // B and C of the tokens
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
            A2[e][i] = in ? p.A[(int64_t)(cq + e) * p.N + n0 + i] * kLog2e : 0.f;
            dA[e][i] = 0.f;
            if (ch.n > 1)
                G[e][i] = in ? ends[(((int64_t)b * ch.n + k) * NP + n0 + i) * p.C + cq + e] : 0.f;
            else
                G[e][i] = in && p.dstate ? p.dstate[((int64_t)b * p.C + cq + e) * p.N + n0 + i] : 0.f;
        }

    // ahead of the scan and behind it: token lane / 8, channels cv ..
    const int tl = lane / 8, cl = lane % 8 * V;
    const bool von = w0 + cl < cpg;
    const int cv = g * cpg + (von ? w0 + cl : 0);
    float bias[V], skip[V], dD[V], db[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        bias[e] = p.dt_bias ? p.dt_bias[cv + e] : 0.f;
        skip[e] = p.D ? p.D[cv + e] : 0.f;
        dD[e] = db[e] = 0.f;
    }
    const T *x = static_cast<const T *>(p.x.p) + b * p.x.sb + cv;
    const T *dt = static_cast<const T *>(p.dt.p) + b * p.dt.sb + cv;
    const T *z = p.z.p ? static_cast<const T *>(p.z.p) + b * p.z.sb + cv : nullptr;
    const T *dy = static_cast<const T *>(p.dy.p) + b * p.dy.sb + cv;
    const int nkept = (p.T + K - 1) / K;

    for (int tb = t0 + (t1 - 1 - t0) / K * K; tb >= t0; tb -= K) {
        const int t = tb + tl;
        const bool live = von && t < len;
        float *const out_bc = parts.bc + ((((int64_t)b * p.T + tb) * p.G + g) * ch.blocks + blk) * 2 * NP;
        const int64_t out_step = (int64_t)p.G * ch.blocks * 2 * NP;
        if (tb >= len) {   // past the sequence: gradients of 0
            const float none[V] = {};
            if (von && t < t1) {
                store_all(static_cast<T *>(p.dx.p) + b * p.dx.sb + t * p.dx.st + cv, none);
                store_all(static_cast<T *>(p.ddt.p) + b * p.ddt.sb + t * p.ddt.st + cv, none);
                if (z)
                    store_all(static_cast<T *>(p.dz.p) + b * p.dz.sb + t * p.dz.st + cv, none);
            }
            for (int i = threadIdx.x; i < K * 2 * NP; i += kBlk)
                if (tb + i / (2 * NP) < t1)
                    out_bc[i / (2 * NP) * out_step + i % (2 * NP)] = 0.f;
            continue;
        }
        const Raw<T, V> xr = live ? load_raw<T, V>(x + t * p.x.st) : zero_raw<T, V>();
        const Raw<T, V> dr = live ? load_raw<T, V>(dt + t * p.dt.st) : zero_raw<T, V>();
        const Raw<T, V> yr = live ? load_raw<T, V>(dy + t * p.dy.st) : zero_raw<T, V>();
        const Raw<T, V> zr = live && z ? load_raw<T, V>(z + t * p.z.st) : zero_raw<T, V>();
        float first[CH][NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            float f[CH];
            load_all<float, CH>(kept + ((int64_t)(b * (int64_t)nkept + tb / K) * NP + n0 + i) * p.C + cq, f);
#pragma unroll
            for (int e = 0; e < CH; ++e)
                first[e][i] = qon ? f[e] : 0.f;
        }
        for (int i = threadIdx.x; i < K * 2 * NP; i += kBlk) {
            const int ti = tb + i / (2 * NP);
            mat[i] = ti < p.T ? bc[(((int64_t)b * p.T + ti) * p.G + g) * 2 * NP + i % (2 * NP)] : 0.f;
        }
        float d[V], u[V], up[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float raw = get(dr, e) + bias[e], v = p.softplus ? softplus(raw) : raw;
            d[e] = live ? v : 0.f;
            u[e] = d[e] * get(xr, e);
            up[e] = get(yr, e);
            if (z)
                up[e] *= silu(get(zr, e));
        }
        put_lds(&dts[tl][cl], d);
        put_lds(&us[tl][cl], u);
        put_lds(&ups[tl][cl], up);
        __syncthreads();

        float h[K][CH][NS];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            float dv[CH], uv[CH], Bv[NS];
            get_lds(&dts[j][q * CH], dv);
            get_lds(&us[j][q * CH], uv);
            get_lds(mat + j * 2 * NP + n0, Bv);
#pragma unroll
            for (int e = 0; e < CH; ++e)
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    h[j][e][i] = fmaf(exp2_hw(dv[e] * A2[e][i]), j ? h[j - 1][e][i] : first[e][i], uv[e] * Bv[i]);
        }
#pragma unroll
        for (int jr = K - TR; jr >= 0; jr -= TR) {
#pragma unroll
            for (int jj = TR - 1; jj >= 0; --jj) {
                const int j = jr + jj;
                float dv[CH], uv[CH], gv[CH], Bv[NS], Cv[NS];
                get_lds(&dts[j][q * CH], dv);
                get_lds(&us[j][q * CH], uv);
                get_lds(&ups[j][q * CH], gv);
                get_lds(mat + j * 2 * NP + n0, Bv);
                get_lds(mat + j * 2 * NP + NP + n0, Cv);
                float tB[NS] = {}, tC[NS] = {}, res[CH];
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    float yh = 0.f, du = 0.f, dd = 0.f;
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        const float gt = fmaf(Cv[i], gv[e], G[e][i]);
                        yh = fmaf(Cv[i], h[j][e][i], yh);
                        du = fmaf(gt, Bv[i], du);
                        tB[i] = fmaf(gt, uv[e], tB[i]);
                        tC[i] = fmaf(h[j][e][i], gv[e], tC[i]);
                        G[e][i] = exp2_hw(dv[e] * A2[e][i]) * gt;
                        const float w = G[e][i] * (j ? h[j - 1][e][i] : first[e][i]);
                        dd = fmaf(w, A2[e][i], dd);
                        dA[e][i] = fmaf(w, dv[e], dA[e][i]);
                    }
                    yh += dpp<kXor1>(yh), du += dpp<kXor1>(du), dd += dpp<kXor1>(dd);
                    yh += dpp<kXor2>(yh), du += dpp<kXor2>(du), dd += dpp<kXor2>(dd);
                    res[e] = s == 0 ? yh : s == 1 ? du : dd;
                }
                // over d, u and dy' of the token, which have been read
                if (s < 3)
                    put_lds(&dts[s * K + j][q * CH], res);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    reinterpret_cast<float *>(&red_[wave][jj][0][i][0])[lane] = tB[i];
                    reinterpret_cast<float *>(&red_[wave][jj][1][i][0])[lane] = tC[i];
                }
            }
            __syncthreads();
            // a row of 16 float4 a token, matrix and i: float4 (over s) q of all waves; RT threads a row
            constexpr int rows = TR * 2 * NS, RT = kBlk / rows >= 16 ? 16 : kBlk / rows;
            if ((int)threadIdx.x < rows * RT) {
                const int row = threadIdx.x / RT, part = threadIdx.x % RT;
                float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < 4; ++w)
#pragma unroll
                    for (int i = 0; i < 16 / RT; ++i) {
                        const float4 f = (&red_[w][0][0][0][0])[row * 16 + i * RT + part];
                        a.x += f.x, a.y += f.y, a.z += f.z, a.w += f.w;
                    }
                a.x = lanes_sum(a.x, RT), a.y = lanes_sum(a.y, RT), a.z = lanes_sum(a.z, RT), a.w = lanes_sum(a.w, RT);
                const int i = row % NS, m = row / NS % 2, j = jr + row / NS / 2;
                if (part == 0 && tb + j < t1) {
                    float *to = out_bc + j * out_step + m * NP + i;
                    to[0] = a.x, to[NS] = a.y, to[2 * NS] = a.z, to[3 * NS] = a.w;
                }
            }
            if (jr > 0)
                __syncthreads();
        }

        float yh[V], du[V], dd[V];
        get_lds(&dts[tl][cl], yh);
        get_lds(&dts[K + tl][cl], du);
        get_lds(&dts[2 * K + tl][cl], dd);
        float odx[V], odt[V], odz[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float xv = get(xr, e);
            odx[e] = live ? fmaf(du[e], d[e], skip[e] * up[e]) : 0.f;
            float v = fmaf(dd[e], kLn2, du[e] * xv);
            if (p.softplus)
                v *= logistic(get(dr, e) + bias[e]);
            odt[e] = live ? v : 0.f;
            odz[e] = z && live ? get(yr, e) * fmaf(skip[e], xv, yh[e]) * silu_grad(get(zr, e)) : 0.f;
            dD[e] = fmaf(up[e], xv, dD[e]);
            db[e] += odt[e];
        }
        if (von && t < t1) {
            store_all(static_cast<T *>(p.dx.p) + b * p.dx.sb + t * p.dx.st + cv, odx);
            store_all(static_cast<T *>(p.ddt.p) + b * p.ddt.sb + t * p.ddt.st + cv, odt);
            if (z)
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
__global__ __launch_bounds__(kBlk) void sum_bc_kernel(SelectiveProblem p, int np, int blocks, const float *part)
{
    const int64_t n = (int64_t)p.B * p.T * p.G * 2 * np;
    for (int64_t i = (int64_t)blockIdx.x * kBlk + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlk) {
        const int s = (int)(i % np);
        int64_t at = i / np;
        const int second = (int)(at & 1);
        at >>= 1;
        if (s >= p.N)
            continue;
        const float *in = part + at * blocks * 2 * np + second * np + s;
        float a = 0.f;
        for (int k = 0; k < blocks; ++k)
            a += in[(int64_t)k * 2 * np];
        const int g = (int)(at % p.G);
        at /= p.G;
        const int t = (int)(at % p.T), b = (int)(at / p.T);
        const Heads &m = second ? p.dCm : p.dBm;
        store_f(static_cast<T *>(m.p) + b * m.sb + t * m.st + g * m.sh + s, a);
    }
}

// Rows 0 .. states - 1 of shares: dA; the next two dD and ddt_bias.  16 channels a workgroup,
// whose rows of threads add every 64th share, eight in flight, then their sums in order.
constexpr int kSumRows = 64;
__global__ __launch_bounds__(16 * kSumRows) void sum_channels_kernel(SelectiveProblem p, int np, int shares, Parts parts)
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

constexpr int64_t kWaves = 4096;
constexpr int kLeast = 32;

template <typename T, int NP>
hipError_t bwd(const SelectiveProblem &p, hipStream_t s)
{
    constexpr int NS = NP / 4, CH = NS <= 2 ? 4 : NS <= 4 ? 2 : 1;
    Chunks ch;
    const int cpg = p.C / p.G;
    ch.waves = (cpg + 63) / 64;
    ch.blocks = (cpg + 64 * CH - 1) / (64 * CH);
    const int64_t waves = (int64_t)p.B * p.G * ch.blocks * 4, want = std::max<int64_t>(1, kWaves / waves);
    const int64_t len = std::max<int64_t>(kLeast, (p.T + want - 1) / want);
    ch.len = (int)((len + K - 1) / K * K);
    ch.n = (p.T + ch.len - 1) / ch.len;
    const int64_t groups = (int64_t)p.B * p.G * ch.blocks * ch.n, passes = (int64_t)p.B * p.G * ch.waves * (ch.n - 1);
    const int64_t joins = ((int64_t)p.B * NP * p.C + kBlk - 1) / kBlk;
    if (groups * kBlk > kMaxThreads || passes * 64 > kMaxThreads || joins * kBlk > kMaxThreads)
        return hipErrorInvalidConfiguration;
    void *bc = nullptr, *ends = nullptr, *steps = nullptr, *kept = nullptr, *pbc = nullptr, *pa = nullptr, *pd = nullptr;
    const int64_t slots = (int64_t)p.B * ch.n, tokens = (int64_t)p.B * p.T * p.G;
    hipError_t e = p.ws->take(&bc, (size_t)tokens * 2 * NP * 4);
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
    if (e == hipSuccess)
        e = take_sel_kept(p, p.rs, &kept);
    if (e != hipSuccess || p.ws->counting)
        return e;
    float *const m = static_cast<float *>(bc), *const en = static_cast<float *>(ends), *const sm = static_cast<float *>(steps);
    const Parts parts{static_cast<float *>(pbc), static_cast<float *>(pa), static_cast<float *>(pd)};
    e = launch_sel_pack(p, m, s);
    if (e == hipSuccess && ch.n > 1) {
        back_kernel<T, NP><<<dim3((unsigned)passes), 64, 0, s>>>(p, ch, m, en, sm);
        e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        back_chain_kernel<NP><<<dim3((unsigned)joins), kBlk, 0, s>>>(p, ch, en, sm);
        e = hipGetLastError();
    }
    if (e != hipSuccess)
        return e;
    grad_kernel<T, NS, CH><<<dim3((unsigned)groups), kBlk, 0, s>>>(p, ch, m, static_cast<const float *>(kept), en, parts);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const int64_t sums = (tokens * 2 * NP + kBlk - 1) / kBlk;
    sum_bc_kernel<T><<<dim3((unsigned)std::min<int64_t>(sums, 65536)), kBlk, 0, s>>>(p, NP, ch.blocks, parts.bc);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    sum_channels_kernel<<<dim3((unsigned)((p.C + 15) / 16), (unsigned)(p.N + 2)), 16 * kSumRows, 0, s>>>(p, NP, (int)slots, parts);
    return hipGetLastError();
}

template <typename T>
hipError_t pick(const SelectiveProblem &p, hipStream_t s)
{
    switch (sel_states(p)) {
    case 4: return bwd<T, 4>(p, s);
    case 8: return bwd<T, 8>(p, s);
    case 16: return bwd<T, 16>(p, s);
    case 32: return bwd<T, 32>(p, s);
    default: return bwd<T, 64>(p, s);
    }
}

}  // namespace

hipError_t launch_selective_bwd(const SelectiveProblem &p, hipStream_t s)
{
    return p.dtype == 0 ? pick<float>(p, s) : pick<bf16_t>(p, s);
}

}  // namespace gspn
