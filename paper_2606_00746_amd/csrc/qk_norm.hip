// RMS norm of query and key heads with the position rotation in the same pass
// (gspn_qk_norm_rotate_fwd, _bwd).
//
//   n = x / sqrt(mean(x^2) + eps),  z = w n,  y = R z
//   R turns the pairs (a, b) of z's first R entries by their position's angles:
//   (a cos - b sin, a sin + b cos)
// and backwards, t = R^T dy:
//   dw = sum t n,  dx = (t w - n mean(t w n)) / sqrt(mean(x^2) + eps)
//
// Bound by memory: x (and dy) read once, y (dx) written once.  A head's row
// lies in a group of up to 16 lanes, 16 entries each as two runs of 8.  Where
// the rotation pairs entry i with R/2 + i and R/2 is a multiple of 8, a lane
// owns both runs of its pairs and nothing is exchanged; adjacent pairs lie in
// one run; other pairings go through LDS.  A group of the forward takes several
// heads of one token, whose rows are in flight together and share the token's
// angles (32 x 5476 tokens of 18 + 18 heads of 64, bf16, slices of a fused buffer: 348 to
// 365 us, 4.4 to 4.6 TB/s, where a large copy reaches 4.9); of the backward one, which
// leaves registers for more waves (8 x 4096 tokens of 12 + 12 heads of 64: 66 us, 4.6
// TB/s, and 5 for the weights' shares; two heads at once 80).
#include <algorithm>

#include "attn.hpp"
#include "qk_norm.hpp"

namespace gspn {
namespace {

using namespace cdna;

constexpr int kBlk = 256;

enum Pairing { kNone, kHalfRuns, kAdjacent, kHalfAny };

template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&f)[8]);
template <>
__device__ __forceinline__ void load8(const bf16_t *p, float (&f)[8])
{
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        f[e] = elem(u, e);
}
template <>
__device__ __forceinline__ void load8(const float *p, float (&f)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&f)[8])
{
    put16(p, u32x4{pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])});
}
__device__ __forceinline__ void store8(float *p, const float (&f)[8])
{
    put16(p, u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])});
    put16(p + 4, u32x4{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])});
}

// Sum over groups of n lanes (a power of two up to 16), in every lane of a group.
__device__ __forceinline__ float group_sum(float v, int n)
{
    const auto dpp = [](float x, auto ctrl) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    if (n > 1)
        v += dpp(v, std::integral_constant<int, 0xB1>{});    // lanes 1 0 3 2
    if (n > 2)
        v += dpp(v, std::integral_constant<int, 0x4E>{});    // lanes 2 3 0 1
    if (n > 4)
        v += dpp(v, std::integral_constant<int, 0x141>{});   // mirrored in 8
    if (n > 8)
        v += dpp(v, std::integral_constant<int, 0x140>{});   // mirrored in 16
    return v;
}

// The runs of a lane: entries at a and b, or -1.
struct Runs {
    int a, b;
};
template <int P>
__device__ __forceinline__ Runs runs_of(int lane, int D, int R)
{
    Runs r{16 * lane, 16 * lane + 8};
    if (P == kHalfRuns) {
        if (lane < R / 16)
            return Runs{8 * lane, R / 2 + 8 * lane};
        r.a = R + 16 * (lane - R / 16);
        r.b = r.a + 8;
    }
    if (r.b >= D)
        r.b = -1;
    if (r.a >= D)
        r.a = -1;
    return r;
}

// cos and sin of a lane's 16 entries (1 and 0 where an entry is not turned)
struct Angles {
    float c[2][8], s[2][8];
};
template <int P>
__device__ __forceinline__ void load_angles(Angles &g, const float *cs, const float *sn, Runs r, int R)
{
    if (P == kNone)
        return;
    if (P == kHalfRuns) {
        const bool on = r.a >= 0 && r.a < R / 2;
        load8(cs + (on ? r.a : 0), g.c[0]);
        load8(sn + (on ? r.a : 0), g.s[0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            g.c[0][e] = on ? g.c[0][e] : 1.f;
            g.s[0][e] = on ? g.s[0][e] : 0.f;
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int at = (k ? r.b : r.a) + e;
            const bool on = (k ? r.b : r.a) >= 0 && at < R;
            const int i = P == kAdjacent ? at / 2 : at < R / 2 ? at : at - R / 2;
            g.c[k][e] = on ? cs[i] : 1.f;
            g.s[k][e] = on ? sn[i] : 0.f;
        }
}

// Turns a lane's entries by sign * its angles.  `row`: LDS for the group's row.
template <int P>
__device__ __forceinline__ void turn(float (&x)[2][8], const Angles &g, float sign, Runs r, int R, float *row)
{
    if (P == kHalfRuns) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = x[0][e], b = x[1][e], c = g.c[0][e], s = sign * g.s[0][e];
            x[0][e] = a * c - b * s;
            x[1][e] = a * s + b * c;
        }
    } else if (P == kAdjacent) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float a = x[k][e], b = x[k][e + 1], c = g.c[k][e], s = sign * g.s[k][e];
                x[k][e] = a * c - b * s;
                x[k][e + 1] = a * s + b * c;
            }
    } else if (P == kHalfAny) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = k ? r.b : r.a;
            if (at >= 0)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    row[at + e] = x[k][e];
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = k ? r.b : r.a;
            if (at >= 0)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (at + e < R) {
                        const bool low = at + e < R / 2;
                        const float o = row[low ? at + e + R / 2 : at + e - R / 2];
                        const float s = sign * g.s[k][e];
                        x[k][e] = x[k][e] * g.c[k][e] + (low ? -o * s : o * s);
                    }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T>
__device__ __forceinline__ void load_row(const T *p, Runs r, float (&x)[2][8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        x[0][e] = x[1][e] = 0.f;
    if (r.a >= 0)
        load8(p + r.a, x[0]);
    if (r.b >= 0)
        load8(p + r.b, x[1]);
}
template <typename T>
__device__ __forceinline__ void store_row(T *p, Runs r, const float (&x)[2][8])
{
    if (r.a >= 0)
        store8(p + r.a, x[0]);
    if (r.b >= 0)
        store8(p + r.b, x[1]);
}
template <typename T>
__device__ __forceinline__ void load_weights(const void *w, Runs r, float (&f)[2][8])
{
    load_row(static_cast<const T *>(w), w ? r : Runs{-1, -1}, f);
    if (!w)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            f[0][e] = f[1][e] = 1.f;
}

__device__ __forceinline__ int table_row(const NormProblem &p, int b, int t)
{
    return p.positions ? min(max(p.positions[(int64_t)b * p.T + t], 0), p.rows - 1) : p.first + t;
}

template <typename T, int P, int HL>
__global__ __launch_bounds__(kBlk) void norm_fwd_kernel(NormProblem p, int lanes)
{
    __shared__ float rows[P == kHalfAny ? kBlk * 16 : 1];
    const int per = kBlk / lanes, grp = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    const int64_t tokens = (int64_t)p.B * p.T;
    const int bq = (p.Hq + HL - 1) / HL, bk = (p.Hk + HL - 1) / HL;
    int64_t item = (int64_t)blockIdx.x * per + grp;
    if (item >= tokens * (bq + bk))
        return;
    const bool second = item >= tokens * bq;
    if (second)
        item -= tokens * bq;
    const int nb = second ? bk : bq, H = second ? p.Hk : p.Hq, h0 = (int)(item % nb) * HL;
    const int64_t bt = item / nb;
    const int b = (int)(bt / p.T), t = (int)(bt % p.T);
    const Heads &xi = second ? p.k : p.q, &yo = second ? p.yk : p.yq;
    const T *x = static_cast<const T *>(xi.p) + b * xi.sb + t * xi.st + h0 * xi.sh;
    T *y = static_cast<T *>(yo.p) + b * yo.sb + t * yo.st + h0 * yo.sh;
    const Runs r = runs_of<P>(lane, p.D, p.R);

    float v[HL][2][8];
#pragma unroll
    for (int h = 0; h < HL; ++h)
        load_row(x + h * xi.sh, h0 + h < H ? r : Runs{-1, -1}, v[h]);
    float w[2][8];
    load_weights<T>(second ? p.wk : p.wq, r, w);
    Angles g;
    const int64_t at = P == kNone ? 0 : (int64_t)table_row(p, b, t) * (p.R / 2);
    load_angles<P>(g, p.cos + at, p.sin + at, r, p.R);
#pragma unroll
    for (int h = 0; h < HL; ++h) {
        if (h0 + h >= H)
            break;
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                ss = fmaf(v[h][k][e], v[h][k][e], ss);
        ss = group_sum(ss, lanes);
        const float f = rsqrtf(ss / (float)p.D + p.eps);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[h][k][e] *= f * w[k][e];
        turn<P>(v[h], g, 1.f, r, p.R, rows + grp * lanes * 16);
        store_row(y + h * yo.sh, r, v[h]);
    }
}

// Blocks 0 .. nbq - 1 take the queries, the others the keys; every block adds
// up its rows' share of dw in a fixed order and leaves it in part[block].
template <typename T, int P>
__global__ __launch_bounds__(kBlk) void norm_bwd_kernel(NormProblem p, int lanes, int nbq, float *part)
{
    __shared__ float rows[kBlk * 16];
    const int per = kBlk / lanes, grp = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    const bool second = (int)blockIdx.x >= nbq;
    const int blk = second ? blockIdx.x - nbq : blockIdx.x, nblk = second ? gridDim.x - nbq : nbq;
    const int H = second ? p.Hk : p.Hq;
    const int64_t items = (int64_t)p.B * p.T * H;
    const Heads &xi = second ? p.k : p.q, &yi = second ? p.dyk : p.dyq, &dx = second ? p.dk : p.dq;
    const Runs r = runs_of<P>(lane, p.D, p.R);
    float *row = rows + grp * lanes * 16;

    float w[2][8], dw[2][8];
    load_weights<T>(second ? p.wk : p.wq, r, w);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        dw[0][e] = dw[1][e] = 0.f;
    for (int64_t item = (int64_t)blk * per + grp; item < items; item += (int64_t)nblk * per) {
        const int h = (int)(item % H);
        const int64_t bt = item / H;
        const int b = (int)(bt / p.T), t = (int)(bt % p.T);
        const T *x = static_cast<const T *>(xi.p) + b * xi.sb + t * xi.st + h * xi.sh;
        const T *dy = static_cast<const T *>(yi.p) + b * yi.sb + t * yi.st + h * yi.sh;
        T *out = static_cast<T *>(dx.p) + b * dx.sb + t * dx.st + h * dx.sh;
        float v[2][8], d[2][8];
        load_row(x, r, v);
        load_row(dy, r, d);
        Angles g;
        const int64_t at = P == kNone ? 0 : (int64_t)table_row(p, b, t) * (p.R / 2);
        load_angles<P>(g, p.cos + at, p.sin + at, r, p.R);
        turn<P>(d, g, -1.f, r, p.R, row);
        float ss = 0.f, sd = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ss = fmaf(v[k][e], v[k][e], ss);
                sd = fmaf(v[k][e], d[k][e] * w[k][e], sd);
            }
        ss = group_sum(ss, lanes);
        sd = group_sum(sd, lanes);
        const float f = rsqrtf(ss / (float)p.D + p.eps), m = f * f * (sd / (float)p.D);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[k][e] = fmaf(d[k][e], v[k][e] * f, dw[k][e]);
                d[k][e] = f * (d[k][e] * w[k][e] - v[k][e] * m);
            }
        store_row(out, r, d);
    }
    if ((second ? p.wk : p.wq) == nullptr)
        return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((k ? r.b : r.a) >= 0)
                row[(k ? r.b : r.a) + e] = dw[k][e];
    __syncthreads();
    for (int e = threadIdx.x; e < p.D; e += kBlk) {
        float s = 0.f;
        for (int i = 0; i < per; ++i)
            s += rows[i * lanes * 16 + e];
        part[(int64_t)blockIdx.x * p.D + e] = s;
    }
}

// dw from the blocks' shares: 16 columns a workgroup, its 64 rows of threads
// adding every 64th share, eight in flight, then their sums in order.
constexpr int kSumRows = 64;
template <typename T>
__global__ __launch_bounds__(16 * kSumRows) void norm_dw_kernel(NormProblem p, const float *part, int nbq, int nbk)
{
    __shared__ float sums[kSumRows][17];
    const int cols = (p.D + 15) / 16, second = blockIdx.x / cols;
    const int e = blockIdx.x % cols * 16 + threadIdx.x % 16, i0 = threadIdx.x / 16;
    const int n = second ? nbk : nbq;
    const float *in = part + (second ? (int64_t)nbq * p.D : 0);
    void *out = second ? p.dwk : p.dwq;
    if (out == nullptr)
        return;
    float s = 0.f;
    if (e < p.D)
        for (int i = i0; i < n; i += 8 * kSumRows) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = i + j * kSumRows < n ? in[(int64_t)(i + j * kSumRows) * p.D + e] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s += x[j];
        }
    sums[i0][threadIdx.x % 16] = s;
    __syncthreads();
    if (i0 == 0 && e < p.D) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < kSumRows; ++i)
            a += sums[i][threadIdx.x];
        store_f(static_cast<T *>(out) + e, a);
    }
}

Pairing pairing(const NormProblem &p)
{
    if (p.R == 0)
        return kNone;
    if (p.adjacent)
        return kAdjacent;
    return p.R % 16 == 0 ? kHalfRuns : kHalfAny;
}

int group_lanes(const NormProblem &p)
{
    const int n = pairing(p) == kHalfRuns ? p.R / 16 + (p.D - p.R + 15) / 16 : (p.D + 15) / 16;
    int l = 1;
    while (l < n)
        l *= 2;
    return l;
}

// Heads that a group of lanes of the forward takes together: four, one where that
// leaves the card with fewer than kFewThreads threads (us, one and four: 4096 tokens of
// 2 x 12 heads of 64 7.1 and 7.6, 8192 12.7 and 11.4, 65536 90 and 86; 8 tokens 3.5 and 5.5).
constexpr int64_t kFewThreads = 256 * 1024;

template <typename T, int P, int HL>
hipError_t fwd(const NormProblem &p, hipStream_t s)
{
    const int lanes = group_lanes(p), per = kBlk / lanes;
    const int64_t items = (int64_t)p.B * p.T * ((p.Hq + HL - 1) / HL + (p.Hk + HL - 1) / HL);
    const int64_t n = (items + per - 1) / per;
    if (n * kBlk > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (p.ws->counting)
        return hipSuccess;
    norm_fwd_kernel<T, P, HL><<<dim3((unsigned)n), kBlk, 0, s>>>(p, lanes);
    return hipGetLastError();
}

// Workgroups of the backward at most, and how many there are at least before a group of
// lanes has kRowsEach rows of its own: each leaves a share of dw to be added up (us at 4096
// tokens of 2 x 12 heads of 64 15.6 without the latter, 13.8 with it; 4096 tokens of 2 x 16
// heads of 128 27.4 and 22.8).
constexpr int kBwdBlocks = 2048, kBwdFew = 512, kRowsEach = 4;

template <typename T, int P>
hipError_t bwd(const NormProblem &p, hipStream_t s)
{
    const int lanes = group_lanes(p), per = kBlk / lanes;
    const auto blocks = [&](int H) {
        const int64_t all = ((int64_t)p.B * p.T * H + per - 1) / per;
        const auto part = [&](int64_t n) { return std::max<int64_t>(1, n * H / (p.Hq + p.Hk)); };
        return (int)std::min({all, part(kBwdBlocks), std::max(part(kBwdFew), all / kRowsEach)});
    };
    const int nbq = blocks(p.Hq), nbk = blocks(p.Hk);
    void *part = nullptr;
    if (p.wq || p.wk) {
        const hipError_t e = p.ws->take(&part, (size_t)(nbq + nbk) * p.D * 4);
        if (e != hipSuccess)
            return e;
    }
    if (p.ws->counting)
        return hipSuccess;
    norm_bwd_kernel<T, P><<<dim3((unsigned)(nbq + nbk)), kBlk, 0, s>>>(p, lanes, nbq, static_cast<float *>(part));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !part)
        return e;
    norm_dw_kernel<T><<<dim3((unsigned)(2 * ((p.D + 15) / 16))), 16 * kSumRows, 0, s>>>(p, static_cast<const float *>(part), nbq, nbk);
    return hipGetLastError();
}

template <typename T, bool BWD, int P>
hipError_t pick(const NormProblem &p, hipStream_t s)
{
    if constexpr (BWD)
        return bwd<T, P>(p, s);
    else
        return norm_heads_each(p) == 1 ? fwd<T, P, 1>(p, s) : fwd<T, P, 4>(p, s);
}

template <typename T, bool BWD>
hipError_t pick(const NormProblem &p, hipStream_t s)
{
    switch (pairing(p)) {
    case kNone: return pick<T, BWD, kNone>(p, s);
    case kHalfRuns: return pick<T, BWD, kHalfRuns>(p, s);
    case kAdjacent: return pick<T, BWD, kAdjacent>(p, s);
    default: return pick<T, BWD, kHalfAny>(p, s);
    }
}

}  // namespace

int norm_heads_each(const NormProblem &p)
{
    const int64_t n = (int64_t)p.B * p.T * ((p.Hq + 3) / 4 + (p.Hk + 3) / 4) * group_lanes(p);
    return n < kFewThreads ? 1 : 4;
}

hipError_t launch_norm_rotate_fwd(const NormProblem &p, hipStream_t s)
{
    return p.dtype == 0 ? pick<float, false>(p, s) : pick<bf16_t, false>(p, s);
}

hipError_t launch_norm_rotate_bwd(const NormProblem &p, hipStream_t s)
{
    return p.dtype == 0 ? pick<float, true>(p, s) : pick<bf16_t, true>(p, s);
}

}  // namespace gspn
