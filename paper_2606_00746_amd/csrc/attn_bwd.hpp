// Gradient of windowed attention (gspn_window_attn_bwd): the kernels of one storage
// type, which attn_bwd.hip (bf16) and attn_bwd_f32.hip take.
//
//   p_ij = exp(scale q_i k_j - lse_i)          (again from q, k and the forward's lse)
//   d_i  = sum_e do_ie o_ie
//   ds_ij = p_ij (do_i v_j - d_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i
//
// Two kernels, so that no sum crosses workgroups in an order of its own:
//  * attn_dq_kernel owns 128 queries and runs over their keys as the forward
//    does; it also forms d_i, which the other kernel reads;
//  * attn_dkv_kernel owns 128 keys (a wave 32 of them) and runs over the
//    queries that see them, of every head that shares the keys.
// The scores are formed twice, which costs 2 of the 7 products; the sums over
// queries of either kernel are in a fixed order and need no atomics.  Keys that
// all later queries see (sinks), and calls with few keys, have their
// queries split over several workgroups, whose fp32 shares are added up, in
// order, by attn_dkv_sum_kernel.
//
// 8 x 4100 tokens of 12 heads of 64, bf16, a window of 448 to either side: 211 us for dq
// (609 TFLOP/s of its three products) and 311 for dk and dv (551 of its four); heads of
// 128, 2 x 8192 tokens of 16 heads on 4, a causal window of 1023: 273 and 391.  As in the
// forward the matrix cores are busy 27 to 32% of the cycles, at 2.1 GHz of 2.4; a wave waits
// 30 to 40% of its time, for LDS and the other waves, and 20 to 30% for its turn to issue.
//
// bf16: p and ds are rounded to 8 significant bits for their products, and d_i comes
// from the rounded o_i.  The first costs an error of the size of the results' own
// rounding.  The second is small beside it where a row has many keys, so that
// |o_i| << |v_j|, but not where it has few (attn_few_keys): FINE kernels form d_i
// as sum_j p_ij (do_i v_j), in a pass of its own, and add what rounding p and ds
// leaves as a second term (relative error of dq and dk at sequences of 16 to 128
// tokens, against 1.7e-3 for rounded exact results: 2.9e-3 -> 1.7e-3).
#pragma once

#include <algorithm>

#include "attn.hpp"

namespace gspn {
namespace {

using namespace attn;

// KW: waves that share their rows, each with its part of a tile (1, or 2 with 32
// rows of it each): the odd wave's sums are added to its neighbour's at the end.
template <int N>
__device__ __forceinline__ void join_pair(float *lds, f32x16_t (&acc)[N], int w, int l)
{
    float *mine = lds + w / 2 * (64 * 16 * N);
    lds_barrier();
    if (w & 1)
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                mine[(16 * i + r) * 64 + l] = acc[i][r];
    lds_barrier();
    if (!(w & 1))
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[i][r] += mine[(16 * i + r) * 64 + l];
}

// acc += X^T p: with FINE, p to 16 significant bits.
template <int DP, bool FINE, typename T>
__device__ __forceinline__ void add_turned(const Turned<T, DP> &x, const f32x16_t &p, f32x16_t (&acc)[DP / 32])
{
    mma_turned<DP>(x, Probs<T>(p), acc);
    if constexpr (FINE) {
        f32x16_t rest;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            rest[r] = p[r] - (float)(__bf16)p[r];
        mma_turned<DP>(x, Probs<T>(rest), acc);
    }
}

template <typename T>
__device__ __forceinline__ float dot(Frag<T> a, Frag<T> b)
{
    constexpr int n = 16 / sizeof(T);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < n; ++e)
        s = fmaf((float)a.v[e], (float)b.v[e], s);
    return s;
}

template <typename T, int DP, int KW, bool FINE>
__global__ __launch_bounds__(kThreads, (DP * sizeof(T) <= 128 ? 2 : 1))
void attn_dq_kernel(AttnProblem a, float *delta)
{
    using X = Tile<T, DP>;
    constexpr int kSlices = X::kPieces / 2, kTQ = 128 / KW;
    constexpr bool kFlows = sizeof(T) == 2;   // as in the forward
    static_assert(!FINE || (kFlows && KW == 2), "");
    __shared__ __attribute__((aligned(X::kRow))) char lds[2][2][X::kBytes];
    __shared__ float sums[kThreads];

    const int G = a.Hq / a.Hkv, nqt = (a.Tq + kTQ - 1) / kTQ;
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int g = id % G;
    id /= G;
    const int qt = id % nqt;
    id /= nqt;
    const int hk = id % a.Hkv, b = id / a.Hkv, hq = hk * G + g;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64;
    const int c = l % 32, h = l / 32;
    const int len = seq_len(a, b);

    const T *kp = static_cast<const T *>(a.k.p) + b * a.k.sb + hk * a.k.sh;
    const T *vp = static_cast<const T *>(a.v.p) + b * a.v.sb + hk * a.v.sh;
    const int t0 = qt * kTQ, tw = t0 + w / KW * 32, t = tw + c, tr = min(t, a.Tq - 1);
    const int kb0 = KW == 2 ? w % 2 : 0;
    const KeyTiles wg(a, len, t0, min(kTQ, a.Tq - t0));
    const KeyRange wave(a, len, tw, 32);
    int lo, hi;
    key_bounds(a, len, t + a.offset, lo, hi);

    Frag<T> qf[kSlices], df[kSlices];
    const T *qr = static_cast<const T *>(a.q.p) + b * a.q.sb + hq * a.q.sh + tr * a.q.st;
    const T *dr = static_cast<const T *>(a.dout.p) + b * a.dout.sb + hq * a.dout.sh + tr * a.dout.st;
    const T *orow = static_cast<const T *>(a.o.p) + b * a.o.sb + hq * a.o.sh + tr * a.o.st;
    float d = 0.f;
#pragma unroll
    for (int s = 0; s < kSlices; ++s) {
        qf[s] = row_frag(qr, 2 * s + h, a.D);
        df[s] = row_frag(dr, 2 * s + h, a.D);
        if (!FINE)
            d += dot(df[s], row_frag(orow, 2 * s + h, a.D));
    }
    const int64_t stat = ((int64_t)b * a.Hq + hq) * a.Tq + tr;
    const float s2 = a.scale * kLog2e, lse2 = a.lse[stat] * kLog2e;
    // d over the lanes (FINE: and waves) that share it; for the keys' gradients: d,
    // and lse to the base of 2
    const auto whole = [&] {
        d = half_sum(d);
        if constexpr (FINE) {
            sums[threadIdx.x] = d;
            lds_barrier();
            d += sums[threadIdx.x ^ 64];
        }
        if (t < a.Tq)
            delta[(int64_t)h * a.B * a.Hq * a.Tq + stat] = h == 0 ? d : lse2;
    };
    if (!FINE)
        whole();

    f32x16_t acc[DP / 32];
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            acc[db][r] = 0.f;

    X kt, vt;
    Flow<DP> kw, vw;
    const int n = wg.n;
    const auto flow = [&](int it) {
        if constexpr (kFlows) {
            kw.load(lds[it & 1][0], kp, wg.row(it), len, w);
            vw.load(lds[it & 1][1], vp, wg.row(it), len, w);
        }
    };
    arrived(qf);
    arrived(df);
    if constexpr (kFlows) {
        kw.start(a.k.st, a.D);
        vw.start(a.v.st, a.D);
    } else {
        kt.start(a.k.st, a.D);
        vt.start(a.v.st, a.D);
        if (n > 0) {
            kt.load(kp, a.k.st, wg.row(0), len, a.D);
            vt.load(vp, a.v.st, wg.row(0), len, a.D);
            kt.store(lds[0][0]);
            vt.store(lds[0][1]);
        }
        lds_barrier();
    }
    for (int pass = FINE ? 0 : 1; pass < 2; ++pass) {
        const bool sums_up = FINE && pass == 0;
        if (kFlows && n > 0)
            flow(0);
        for (int it = 0; it < n; ++it) {
            const int k0 = wg.row(it);
            const char *kl = lds[it & 1][0], *vl = lds[it & 1][1];
            if constexpr (kFlows) {
                landed();
                if (it + 1 < n)
                    flow(it + 1);
            } else if (it + 1 < n) {
                kt.load(kp, a.k.st, wg.row(it + 1), len, a.D);
                vt.load(vp, a.v.st, wg.row(it + 1), len, a.D);
            }
            if (wave.some(k0)) {
                const bool all = wave.all(k0);
                // the 32 keys of block `blk`, a constant where it is an address
                const auto block = [&](auto blk) {
                    constexpr int kb = decltype(blk)::value;
                    f32x16_t s, dp;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[r] = dp[r] = 0.f;
                    RowFrags<T, DP> kf, vf;
                    Turned<T, DP> kx;
                    if constexpr (kFlows) {
                        flow_rows<DP, kb>(lds_offset(kl), kf.f);
#pragma unroll
                        for (int sl = 0; sl < kSlices; ++sl)
                            s = mma(kf.at(sl), qf[sl], s);
                        flow_rows<DP, kb>(lds_offset(vl), vf.f);
#pragma unroll
                        for (int sl = 0; sl < kSlices; ++sl)
                            dp = mma(vf.at(sl), df[sl], dp);
                    } else {
                        kf.load(kl, 32 * kb + c);
                        vf.load(vl, 32 * kb + c);
                        reads_first<T>();
#pragma unroll
                        for (int sl = 0; sl < kSlices; ++sl) {
                            s = mma(kf.at(sl), qf[sl], s);
                            dp = mma(vf.at(sl), df[sl], dp);
                        }
                    }
                    if constexpr (kFlows)
                        flow_turned<DP, kb>(lds_offset(kl), kx);
                    else
                        kx.load(kl, 32 * kb);
                    const float less = sums_up ? 0.f : d;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], s2, -lse2)) * (dp[r] - less);
                    if (!all) {
                        const bool sunk = k0 < a.sinks;
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int j = k0 + 32 * kb + 8 * (r / 4) + 4 * h + r % 4;
                            s[r] = sees(j, lo, hi, a.sinks, sunk) ? s[r] : 0.f;
                        }
                    }
                    if (sums_up) {
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            d += s[r];
                    } else {
                        add_turned<DP, FINE>(kx, s, acc);
                    }
                };
                if (KW == 1 || kb0 == 0)
                    block(std::integral_constant<int, 0>{});
                if (KW == 1 || kb0 == 1)
                    block(std::integral_constant<int, 1>{});
            }
            if constexpr (!kFlows) {
                if (it + 1 < n) {
                    kt.store(lds[(it + 1) & 1][0]);
                    vt.store(lds[(it + 1) & 1][1]);
                }
                lds_barrier();
            }
        }
        if (sums_up)
            whole();   // (its barrier: the tiles are free)
    }
    if (KW == 2)
        join_pair(reinterpret_cast<float *>(lds), acc, w, l);
    if (t < a.Tq && (KW == 1 || !(w & 1)))
        store_column<T, DP>(static_cast<T *>(a.dq.p) + b * a.dq.sb + hq * a.dq.sh + t * a.dq.st, acc,
                            a.scale, a.D);
}

// How the keys' tiles of one (b, head) go to workgroups: `sunk` tiles that hold
// sinks, each split over `sparts` of them, then the others over `parts`.
struct KeySplit {
    int tiles, sunk, sparts, parts;
    int64_t slots;           // fp32 shares of a tile, over the batch
    __host__ __device__ int blocks() const { return sunk * sparts + (tiles - sunk) * parts; }
    // shares ahead of this (b, head)'s tile: tiles with one part have none
    __host__ __device__ int shares() const
    {
        return (sparts > 1 ? sunk * sparts : 0) + (parts > 1 ? (tiles - sunk) * parts : 0);
    }
    __host__ __device__ int share(int tile, int part) const
    {
        if (tile < sunk)
            return tile * sparts + part;
        return (sparts > 1 ? sunk * sparts : 0) + (tile - sunk) * parts + part;
    }
};

// ONLY: of dv (1) or dk (2), 0 both.
template <typename T, int DP, int KW, bool FINE, int ONLY>
__global__ __launch_bounds__(kThreads, (DP * sizeof(T) <= 128 ? 2 : 1))
void attn_dkv_kernel(AttnProblem a, const float *delta, KeySplit ks, float *shares)
{
    using X = Tile<T, DP>;
    constexpr bool kDv = ONLY != 2, kDk = ONLY != 1;
    constexpr int kSlices = X::kPieces / 2, kKeys = 128 / KW;
    // as in the forward; larger heads leave one wave a SIMD, which reads by hand would
    // stop (heads of 128: 393 us, 481 with them)
    constexpr bool kFlows = sizeof(T) == 2 && DP <= 64;
    __shared__ __attribute__((aligned(X::kRow))) char lds[2][2][X::kBytes];
    __shared__ __attribute__((aligned(16))) float stats[2][2][kRows];

    const int G = a.Hq / a.Hkv, per = ks.blocks();
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int x = id % per;
    id /= per;
    const int hk = id % a.Hkv, b = id / a.Hkv;
    int tile, part, parts;
    if (x < ks.sunk * ks.sparts) {
        tile = x / ks.sparts, part = x % ks.sparts, parts = ks.sparts;
    } else {
        const int y = x - ks.sunk * ks.sparts;
        tile = ks.sunk + y / ks.parts, part = y % ks.parts, parts = ks.parts;
    }
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64;
    const int c = l % 32, h = l / 32;
    const int len = seq_len(a, b);
    const int k0 = tile * kKeys, kw = k0 + 32 * (w / KW), j = kw + c, qb0 = KW == 2 ? w % 2 : 0;

    // queries t that see some key of the workgroup, of the wave (some, all), of the lane
    const auto after = [&](int key) { return a.right < 0 ? 0 : max(0, key - a.right - a.offset); };
    const auto until = [&](int key) {
        const int e = a.left < 0 || key < a.sinks ? len - 1 : min(len - 1, key + a.left);
        return key >= len ? -1 : min(a.Tq - 1, e - a.offset);
    };
    const int ta = after(k0), tb = max(until(k0), until(min(len - 1, k0 + kKeys - 1)));
    const int some_a = after(kw), some_b = max(until(kw), until(min(len - 1, kw + 31)));
    const int all_a = after(kw + 31);
    const int all_b = kw + 31 >= len ? -1 : min(until(kw + 31), until(max(kw, min(a.sinks, kw + 31))));
    const int lane_a = after(j), lane_b = until(j);

    const int first = ta / kRows, nt = k0 >= len || tb < ta ? 0 : tb / kRows + 1 - first;
    const int total = nt * G;
    const int i0 = (int)((int64_t)total * part / parts), i1 = (int)((int64_t)total * (part + 1) / parts);

    Frag<T> kf[kSlices], vf[kSlices];
    const int jr = max(0, min(j, len - 1));
    const T *kr = static_cast<const T *>(a.k.p) + b * a.k.sb + hk * a.k.sh + jr * a.k.st;
    const T *vr = static_cast<const T *>(a.v.p) + b * a.v.sb + hk * a.v.sh + jr * a.v.st;
#pragma unroll
    for (int s = 0; s < kSlices; ++s) {
        kf[s] = row_frag(kr, 2 * s + h, a.D);
        if (kDk)
            vf[s] = row_frag(vr, 2 * s + h, a.D);
    }
    f32x16_t dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            dk[db][r] = dv[db][r] = 0.f;
    const float s2 = a.scale * kLog2e;

    X qt, dt;
    Flow<DP> qw, dw;
    float stat = 0.f;
    // queries from qrows on stand past the sequence's end: no tile begins there
    const int qrows = max(0, min(a.Tq, len - a.offset));
    const int64_t stats_all = (int64_t)a.B * a.Hq * a.Tq;
    // tile i of the queries into slot i & 1
    const auto fetch = [&](int i) {
        const int hq = hk * G + i / nt, t0 = (first + i % nt) * kRows;
        const T *qp = static_cast<const T *>(a.q.p) + b * a.q.sb + hq * a.q.sh;
        const T *dp = static_cast<const T *>(a.dout.p) + b * a.dout.sb + hq * a.dout.sh;
        const float *sp = delta + ((int64_t)b * a.Hq + hq) * a.Tq + t0;
        if constexpr (kFlows) {
            qw.load(lds[i & 1][0], qp, t0, qrows, w);
            dw.load(lds[i & 1][1], dp, t0, qrows, w);
            // wave 0: the rows' d, 1: their lse; the others the same again
            const rsrc_t r = make_rsrc(sp + (w & 1) * stats_all, 0xffffffffu);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                r, (__attribute__((address_space(3))) void *)(stats[i & 1][1 - (w & 1)]), 4,
                4u * (uint32_t)min(l, qrows - t0 - 1), 0, 0, 0);
        } else {
            qt.load(qp, a.q.st, t0, qrows, a.D);
            dt.load(dp, a.dout.st, t0, qrows, a.D);
            if (threadIdx.x < 2 * kRows)
                stat = t0 + (int)threadIdx.x % kRows < qrows
                           ? sp[threadIdx.x % kRows + (threadIdx.x < kRows ? stats_all : 0)] : 0.f;
        }
    };
    const auto put = [&](int i) {
        qt.store(lds[i & 1][0]);
        dt.store(lds[i & 1][1]);
        if (threadIdx.x < 2 * kRows)
            stats[i & 1][threadIdx.x / kRows][threadIdx.x % kRows] = stat;
    };
    arrived(kf);
    arrived(vf);
    if constexpr (kFlows) {
        qw.start(a.q.st, a.D);
        dw.start(a.dout.st, a.D);
        if (i0 < i1)
            fetch(i0);
    } else {
        qt.start(a.q.st, a.D);
        dt.start(a.dout.st, a.D);
        if (i0 < i1) {
            fetch(i0);
            put(i0);
        }
        lds_barrier();
    }
    for (int i = i0; i < i1; ++i) {
        const int buf = i & 1, t0 = (first + i % nt) * kRows;
        const char *ql = lds[buf][0], *dl = lds[buf][1];
        if constexpr (kFlows)
            landed();
        if (i + 1 < i1)
            fetch(i + 1);
        if (t0 <= some_b && t0 + kRows > some_a) {
            const bool all = t0 >= all_a && t0 + kRows - 1 <= all_b;
            const auto block = [&](auto blk) {
                constexpr int qb = decltype(blk)::value;
                f32x16_t s, dp;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[r] = dp[r] = 0.f;
                RowFrags<T, DP> qf, df;
                Turned<T, DP> qx, dx;
                if constexpr (kFlows) {
                    flow_rows<DP, qb>(lds_offset(ql), qf.f);
#pragma unroll
                    for (int sl = 0; sl < kSlices; ++sl)
                        s = mma(qf.at(sl), kf[sl], s);
                    flow_rows<DP, qb>(lds_offset(dl), df.f);
#pragma unroll
                    for (int sl = 0; sl < kSlices; ++sl)
                        dp = mma(df.at(sl), vf[sl], dp);
                } else {
                    qf.load(ql, 32 * qb + c);
                    if (kDk)
                        df.load(dl, 32 * qb + c);
                    reads_first<T>();
#pragma unroll
                    for (int sl = 0; sl < kSlices; ++sl) {
                        s = mma(qf.at(sl), kf[sl], s);
                        if (kDk)
                            dp = mma(df.at(sl), vf[sl], dp);
                    }
                }
                f32x4_t ls[4], de[4];
                if constexpr (kFlows) {
                    flow_stats<qb>(lds_offset(stats[buf][0]), ls);
                    flow_stats<qb>(lds_offset(stats[buf][1]), de);
                    flow_turned<DP, qb>(lds_offset(dl), dx);
                } else {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        ls[g] = *reinterpret_cast<const f32x4_t *>(&stats[buf][0][32 * qb + 8 * g + 4 * h]);
                        de[g] = *reinterpret_cast<const f32x4_t *>(&stats[buf][1][32 * qb + 8 * g + 4 * h]);
                    }
                    if (kDv)
                        dx.load(dl, 32 * qb);
                    reads_first<T>();
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], s2, -ls[r / 4][r % 4]));
                    dp[r] = s[r] * (dp[r] - de[r / 4][r % 4]);
                }
                if (!all) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int t = t0 + 32 * qb + 8 * (r / 4) + 4 * h + r % 4;
                        const bool see = (uint32_t)(t - lane_a) <= (uint32_t)(lane_b - lane_a) && lane_b >= lane_a;
                        s[r] = see ? s[r] : 0.f;
                        dp[r] = see ? dp[r] : 0.f;
                    }
                }
                if (kDv)
                    add_turned<DP, FINE>(dx, s, dv);
                if (!kDk)
                    return;
                if constexpr (kFlows)
                    flow_turned<DP, qb>(lds_offset(ql), qx);
                else
                    qx.load(ql, 32 * qb);
                add_turned<DP, FINE>(qx, dp, dk);
            };
            if (KW == 1 || qb0 == 0)
                block(std::integral_constant<int, 0>{});
            if (KW == 1 || qb0 == 1)
                block(std::integral_constant<int, 1>{});
        }
        if constexpr (!kFlows) {
            if (i + 1 < i1)
                put(i + 1);
            lds_barrier();
        }
    }

    if (KW == 2) {
        if (kDk)
            join_pair(reinterpret_cast<float *>(lds), dk, w, l);
        if (kDv)
            join_pair(reinterpret_cast<float *>(lds), dv, w, l);
        if (w & 1)
            return;
    }
    if (parts > 1) {
        float *out = shares + ((int64_t)(b * a.Hkv + hk) * ks.shares() + ks.share(tile, part)) *
                                  (2 * kKeys * DP) + (32 * (w / KW) + c) * DP;
        if (kDk)
            store_column<float, DP>(out, dk, 1.f, DP);
        if (kDv)
            store_column<float, DP>(out + kKeys * DP, dv, 1.f, DP);
    } else if (j < a.Tk) {
        if (kDk)
            store_column<T, DP>(static_cast<T *>(a.dk.p) + b * a.dk.sb + hk * a.dk.sh + j * a.dk.st, dk,
                                a.scale, a.D);
        if (kDv)
            store_column<T, DP>(static_cast<T *>(a.dv.p) + b * a.dv.sb + hk * a.dv.sh + j * a.dv.st, dv, 1.f,
                                a.D);
    }
}

// Adds up the shares of the tiles first .. first + count - 1 (of `parts` each),
// four entries of a key a thread.
template <typename T, int DP, int kKeys>
__global__ __launch_bounds__(kThreads) void attn_dkv_sum_kernel(AttnProblem a, KeySplit ks, int first,
                                                                int count, int parts,
                                                                const float *shares)
{
    constexpr int kQuads = DP / 4, kAll = 2 * kKeys * kQuads;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= (int64_t)a.B * a.Hkv * count * kAll)
        return;
    const int e = (int)(id % kAll);
    const int64_t item = id / kAll;
    const int tile = first + (int)(item % count), hk = (int)(item / count % a.Hkv);
    const int b = (int)(item / count / a.Hkv);
    const int which = e / (kKeys * kQuads), key = e / kQuads % kKeys, d = e % kQuads * 4;
    const int j = tile * kKeys + key;
    if (j >= a.Tk || d >= a.D)
        return;
    const float *in = shares + ((int64_t)(b * a.Hkv + hk) * ks.shares() + ks.share(tile, 0)) *
                                   (2 * kKeys * DP) + which * kKeys * DP + key * DP + d;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < parts; ++i)
        sum += *reinterpret_cast<const f32x4_t *>(in + (int64_t)i * (2 * kKeys * DP));
    const Heads &o = which ? a.dv : a.dk;
    const float f = which ? 1.f : a.scale;
    store4(static_cast<T *>(o.p) + b * o.sb + hk * o.sh + j * o.st + d, sum[0] * f, sum[1] * f,
           sum[2] * f, sum[3] * f);
}

// Workgroups wanted at least, and query tiles that a part has at least: shares of fewer
// cost more than they save (us of both kernels, 4 tiles and 2: 2 x 777 tokens, 6 heads of
// 72, a window of 161, bf16 24 and 41, fp32 74 and 90; 1024 tokens, causal, the same).
constexpr int kWanted = 512, kLeast = 4;
// Workgroups that keys with sinks are split over at most.
constexpr int64_t kMostShares = 4096;

KeySplit key_split(const AttnProblem &p, int kKeys)
{
    KeySplit k;
    const int G = p.Hq / p.Hkv;
    const int64_t whole = (int64_t)G * ((p.Tq + kRows - 1) / kRows);
    const int64_t window = p.left < 0 || p.right < 0
                               ? whole
                               : std::min<int64_t>(whole, (int64_t)G * (((int64_t)kKeys + p.left + p.right) / kRows + 1));
    k.tiles = (p.Tk + kKeys - 1) / kKeys;
    k.sunk = p.left < 0 ? 0 : std::min(k.tiles, (p.sinks + kKeys - 1) / kKeys);
    const int64_t groups = (int64_t)p.B * p.Hkv * k.tiles;
    k.parts = (int)std::max<int64_t>(1, std::min((kWanted + groups - 1) / groups, window / kLeast));
    // sinks: parts about as long as the window's, as long as they do not crowd the card
    const int64_t each = std::max<int64_t>(kLeast, window / k.parts);
    const int64_t sunk = (int64_t)p.B * p.Hkv * std::max(1, k.sunk);
    k.sparts = (int)std::max<int64_t>(1, std::min(whole / each, kMostShares / sunk));
    k.slots = (int64_t)p.B * p.Hkv * k.shares();
    return k;
}

// The keys' gradients, in tiles of 128 / KW keys, from delta.
template <typename T, int DP, int KW, bool FINE>
hipError_t run_dkv(const AttnProblem &p, const float *delta, hipStream_t s)
{
    constexpr int kKeys = 128 / KW;
    const KeySplit ks = key_split(p, kKeys);
    void *shares = nullptr;
    hipError_t e = hipSuccess;
    if (ks.slots > 0)
        e = p.ws->take(&shares, (size_t)ks.slots * 2 * kKeys * DP * 4);
    const int64_t nk = (int64_t)p.B * p.Hkv * ks.blocks();
    if (nk * kThreads > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (e != hipSuccess || p.ws->counting)
        return e;
    // fp32 keys, values and both sums at heads of 128 are more than a lane's 512 registers
    // hold: dv and dk one after the other form the scores twice but spill less (4096 tokens
    // of 8 heads, a causal window of 1023: 680 us together, 218 and 331 apart)
    constexpr int kFirst = sizeof(T) == 4 && DP == 128 ? 1 : 0;
    float *const out = static_cast<float *>(shares);
    attn_dkv_kernel<T, DP, KW, FINE, kFirst><<<dim3((unsigned)nk), kThreads, 0, s>>>(p, delta, ks, out);
    e = hipGetLastError();
    if constexpr (kFirst == 1) {
        if (e == hipSuccess) {
            attn_dkv_kernel<T, DP, KW, FINE, 2><<<dim3((unsigned)nk), kThreads, 0, s>>>(p, delta, ks, out);
            e = hipGetLastError();
        }
    }
    const auto sum = [&](int first, int count, int parts) {
        if (e != hipSuccess || count == 0 || parts == 1)
            return;
        const int64_t n = (int64_t)p.B * p.Hkv * count * (2 * kKeys * DP / 4);
        attn_dkv_sum_kernel<T, DP, kKeys><<<dim3((unsigned)((n + kThreads - 1) / kThreads)), kThreads, 0, s>>>(
            p, ks, first, count, parts, static_cast<const float *>(shares));
        e = hipGetLastError();
    };
    sum(0, ks.sunk, ks.sparts);
    sum(ks.sunk, ks.tiles - ks.sunk, ks.parts);
    return e;
}

template <typename T, int DP, int KW, bool FINE>
hipError_t run_dq(const AttnProblem &p, float *delta, hipStream_t s)
{
    const int64_t n = (int64_t)p.B * p.Hq * ((p.Tq + 128 / KW - 1) / (128 / KW));
    if (n * kThreads > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (p.ws->counting)
        return hipSuccess;
    attn_dq_kernel<T, DP, KW, FINE><<<dim3((unsigned)n), kThreads, 0, s>>>(p, delta);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t run(const AttnProblem &p, hipStream_t s)
{
    void *delta = nullptr;
    hipError_t e = p.ws->take(&delta, (size_t)p.B * p.Hq * p.Tq * 8);   // d and lse
    if (e != hipSuccess)
        return e;
    float *d = static_cast<float *>(delta);
    if constexpr (sizeof(T) == 2) {
        if (attn_few_keys(p)) {
            e = run_dq<T, DP, 2, true>(p, d, s);
            return e == hipSuccess ? run_dkv<T, DP, 2, true>(p, d, s) : e;
        }
    }
    e = attn_dq_pairs(p) ? run_dq<T, DP, 2, false>(p, d, s) : run_dq<T, DP, 1, false>(p, d, s);
    if (e != hipSuccess)
        return e;
    return attn_dkv_pairs(p) ? run_dkv<T, DP, 2, false>(p, d, s) : run_dkv<T, DP, 1, false>(p, d, s);
}

template <typename T>
hipError_t run(const AttnProblem &p, hipStream_t s)
{
    return p.D <= 32   ? run<T, 32>(p, s)
           : p.D <= 64 ? run<T, 64>(p, s)
           : p.D <= 96 ? run<T, 96>(p, s)
                       : run<T, 128>(p, s);
}

}  // namespace
}  // namespace gspn
