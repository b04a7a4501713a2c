// Forward of windowed attention (gspn_window_attn_fwd).
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i k_j - lse_i),
//   lse_i = log sum_j exp(scale q_i k_j)     over the keys j that query i sees
//
// One pass over the keys with a running maximum and sum.  A workgroup owns 128
// queries of one head, a wave 32 of them; tiles of 64 keys and values are staged
// in LDS for all four waves, double buffered: the next tile is on its way while one
// is multiplied, bf16 straight into LDS (0.7 of the cycles that it takes through
// registers), fp32 through registers, whose order in LDS differs.  The tiles are those
// of the sinks, then those of the window; a wave passes over tiles that none of its
// queries sees and masks only those that not all see.
// S^T = K Q^T is formed, so that a query's scores are one lane's (and its
// neighbour's, 32 lanes on) and their exponentials, as they stand in registers, are
// an operand of O^T += V^T P^T.
//
// 34229 tokens, 18 heads of 64, bf16, a window of 1110 to either side and 4 sinks, take
// 467 to 485 us = 710 to 740 TFLOP/s (a large matrix product reaches 1250 on the same
// card).  The matrix cores are busy a third of the cycles, vector instructions
// (exponentials, maxima, sums, roundings) a quarter; a wave waits another third, for LDS
// and the other waves; and the clock is 2.0 GHz of 2.4 while it lasts.  64 queries a wave
// take the LDS reads that a product needs to half, but leave one wave a SIMD: slower.
// Softmax weights of 16 bits instead of 8 (a second product with what the rounding
// leaves) would take the error of o from 2.3e-3 to 1.7e-3, that of its own rounding,
// and the time from 467 to 625 us: not done here, unlike where memory is the bound
// (attn_split.hip).
#include "attn.hpp"

namespace gspn {
namespace {

using namespace attn;

// How far (in powers of two) a row's scores may exceed the maximum that its
// sums are kept against before they are scaled to a new one: the exponentials
// stay below 2^8, their bf16 roundings are relative, and few tiles rescale.
constexpr float kSlack = 8.f;

// KW: waves that share their queries, each with its part of every tile's keys
// (1, or 2 of 32 keys each); their shares are joined at the end.
template <typename T, int DP, int KW>
__global__ __launch_bounds__(kThreads, (DP * sizeof(T) <= 128 ? 3 : DP * sizeof(T) <= 256 ? 2 : 1))
void attn_fwd_kernel(AttnProblem a)
{
    using X = Tile<T, DP>;
    constexpr int kSlices = X::kPieces / 2, kTQ = 128 / KW, NK = 2 / KW;
    // bf16 tiles flow straight into LDS, fp32 tiles come through registers
    constexpr bool kFlows = sizeof(T) == 2;
    __shared__ __attribute__((aligned(X::kRow))) char lds[2][2][X::kBytes];

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

    const T *qp = static_cast<const T *>(a.q.p) + b * a.q.sb + hq * a.q.sh;
    const T *kp = static_cast<const T *>(a.k.p) + b * a.k.sb + hk * a.k.sh;
    const T *vp = static_cast<const T *>(a.v.p) + b * a.v.sb + hk * a.v.sh;

    const int t0 = qt * kTQ, tw = t0 + w / KW * 32, kb0 = KW == 2 ? w % 2 : 0;
    const KeyTiles wg(a, len, t0, min(kTQ, a.Tq - t0));
    const KeyRange wave(a, len, tw, 32);

    Frag<T> qf[kSlices];
    int lo, hi;
    const int t = tw + c;
    const T *row = qp + (int64_t)min(t, a.Tq - 1) * a.q.st;
#pragma unroll
    for (int s = 0; s < kSlices; ++s)
        qf[s] = row_frag(row, 2 * s + h, a.D);
    key_bounds(a, len, t + a.offset, lo, hi);

    f32x16_t acc[DP / 32];
    float m = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            acc[db][r] = 0.f;
    const float s2 = a.scale * kLog2e, slack = fminf(kSlack / s2, 3e38f);   // (finite: below, m may be -infinity)

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
    if constexpr (kFlows) {
        kw.start(a.k.st, a.D);
        vw.start(a.v.st, a.D);
        if (n > 0)
            flow(0);
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

    for (int it = 0; it < n; ++it) {
        const int k0 = wg.row(it);
        const char *kl = lds[it & 1][0], *vl = lds[it & 1][1];
        if constexpr (kFlows) {
            // this tile has come, and every wave is done with the one before it
            landed();
            if (it + 1 < n)
                flow(it + 1);
        } else if (it + 1 < n) {
            kt.load(kp, a.k.st, wg.row(it + 1), len, a.D);
            vt.load(vp, a.v.st, wg.row(it + 1), len, a.D);
        }
        if (wave.some(k0)) {
            const bool all = wave.all(k0);
            f32x16_t s[NK];
            RowFrags<T, DP> kf;
            Turned<T, DP> vf;
#pragma unroll
            for (int kb = 0; kb < NK; ++kb) {
                if constexpr (kFlows) {
                    if (kb0 + kb == 0)
                        flow_rows<DP, 0>(lds_offset(kl), kf.f);
                    else
                        flow_rows<DP, 1>(lds_offset(kl), kf.f);
                } else {
                    kf.load(kl, 32 * (kb0 + kb) + c);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[kb][r] = 0.f;
#pragma unroll
                for (int sl = 0; sl < kSlices; ++sl)
                    s[kb] = mma(kf.at(sl), qf[sl], s[kb]);
            }
            const auto turn = [&](int kb) {
                if constexpr (kFlows) {
                    if (kb == 0)
                        flow_turned<DP, 0>(lds_offset(vl), vf);
                    else
                        flow_turned<DP, 1>(lds_offset(vl), vf);
                } else {
                    vf.load(vl, 32 * kb);
                }
            };
            turn(kb0);
            if (!all) {
                const bool sunk = k0 < a.sinks;
#pragma unroll
                for (int kb = 0; kb < NK; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int j = k0 + 32 * (kb0 + kb) + 8 * (r / 4) + 4 * h + r % 4;
                        s[kb][r] = sees(j, lo, hi, a.sinks, sunk) ? s[kb][r] : -__builtin_inff();
                    }
            }
            float mx = -__builtin_inff();
#pragma unroll
            for (int kb = 0; kb < NK; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    mx = fmaxf(mx, s[kb][r]);
            mx = half_max(mx);
            if (__any(mx > m + slack)) {
                const float mn = fmaxf(m, mx);
                const float f = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((m - mn) * s2);
                m = mn;
                sum *= f;
#pragma unroll
                for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        acc[db][r] *= f;
            }
            const float base = m == -__builtin_inff() ? 0.f : m * s2;
#pragma unroll
            for (int kb = 0; kb < NK; ++kb) {
                float part = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], s2, -base));
                    part += s[kb][r];
                }
                sum += part;
                mma_turned<DP>(vf, Probs<T>(s[kb]), acc);
                if (kb + 1 < NK)
                    turn(1);
            }
        }
        if constexpr (!kFlows) {
            if (it + 1 < n) {
                kt.store(lds[(it + 1) & 1][0]);
                vt.store(lds[(it + 1) & 1][1]);
            }
            lds_barrier();
        }
    }
    if (KW == 2) {   // the odd wave's share to its neighbour, scaled to a common maximum
        float *mine = reinterpret_cast<float *>(lds) + w / 2 * (64 * (DP / 2 + 2));
        if (kFlows)
            lds_barrier();
        if (w & 1) {
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    mine[(16 * db + r) * 64 + l] = acc[db][r];
            mine[DP / 2 * 64 + l] = m;
            mine[(DP / 2 + 1) * 64 + l] = sum;
        }
        lds_barrier();
        if (w & 1)
            return;
        const float mo = mine[DP / 2 * 64 + l], mn = fmaxf(m, mo);
        const float f = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((m - mn) * s2);
        const float fo = mo == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((mo - mn) * s2);
        m = mn;
        sum = f * sum + fo * mine[(DP / 2 + 1) * 64 + l];
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[db][r] = f * acc[db][r] + fo * mine[(16 * db + r) * 64 + l];
    }
    T *op = static_cast<T *>(a.o.p) + b * a.o.sb + hq * a.o.sh;
    const float z = half_sum(sum);
    if (t < a.Tq) {
        // (a sum of 0: the query sees no key; one that is NaN stays so)
        store_column<T, DP>(op + t * a.o.st, acc, z == 0.f ? 0.f : 1.f / z, a.D);
        if (a.lse && h == 0)
            a.lse[((int64_t)b * a.Hq + hq) * a.Tq + t] =
                z == 0.f ? -__builtin_inff() : fmaf(m, s2, __builtin_amdgcn_logf(z)) * kLn2;
    }
}

template <typename T, int DP, int KW>
hipError_t run(const AttnProblem &p, hipStream_t s)
{
    constexpr int kTQ = 128 / KW;
    const int64_t tiles = (p.Tq + kTQ - 1) / kTQ, blocks = tiles * p.B * p.Hq;
    if (blocks * kThreads > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (p.ws->counting)
        return hipSuccess;
    attn_fwd_kernel<T, DP, KW><<<dim3((unsigned)blocks), kThreads, 0, s>>>(p);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t pick(const AttnProblem &p, hipStream_t s)
{
    return attn_fwd_pairs(p) ? run<T, DP, 2>(p, s) : run<T, DP, 1>(p, s);
}

template <typename T>
hipError_t run(const AttnProblem &p, hipStream_t s)
{
    return p.D <= 32   ? pick<T, 32>(p, s)
           : p.D <= 64 ? pick<T, 64>(p, s)
           : p.D <= 96 ? pick<T, 96>(p, s)
                       : pick<T, 128>(p, s);
}

}  // namespace

hipError_t launch_attn_fwd(const AttnProblem &p, hipStream_t s)
{
    if (attn_split_preferred(p))
        return launch_attn_split(p, s);
    return p.dtype == 0 ? run<float>(p, s) : run<bf16_t>(p, s);
}

}  // namespace gspn
