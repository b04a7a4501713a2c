// What joins two sublayers (gspn_residual_norm_fwd, _bwd).
//
//   n_f = f / sqrt(mean(f^2) + eps), p = w_post n_f  (or p = f without w_post)
//   r' = r + scale gate p,  n = r' / sqrt(mean(r'^2) + eps),  y = w n
// and backwards, with g the whole gradient of r':
//   g = dr' + (t - n mean(t n)) / sqrt(mean(r'^2) + eps),  t = w dy;  dr = g
//   df = scale gate g, through the first norm where there is one
//   Q_b = sum_t g n_f (or g f):  dgate_b = scale w_post Q_b, dscale = sum_b gate_b w_post Q_b,
//   dw_post = sum_b gate_b scale Q_b;  dw = sum dy n
//
// Bound by memory: r and f read once, r' and y written once (r, f, dy and dr' read, dr and
// df written; r' is formed again from r and f, as r' itself may have been rounded to 16
// bits).  A row lies in the registers of a group of lanes, part of a wave to a whole
// workgroup, as runs of 8 entries; its sums are exchanged inside the group.  Backwards a
// group keeps its columns' shares of Q and dw over all its rows; they are added up in a
// fixed order by one or two small launches.  bf16: forward 290 us for 32 x 5476 tokens of
// 1152 channels (5.6 TB/s); with an fp32 stream, 8 x 4096 tokens of 768 channels, 61 us (5.0)
// and the gradient 100 (4.5).  Rows above 8192 channels take 1024 threads, which leaves 128
// registers to each: their gradient does not hold a row without scratch memory (107 to 124
// registers spilled; 2 x 4096 rows of 8200 and 16384, bf16: 782 and 928 us, 1.0 and 1.7 TB/s;
// of 8192 225, 3.6).
#include <algorithm>

#include "residual_norm.hpp"
#include "vec.hpp"

namespace gspn {
namespace {

using namespace vec;

// How rows lie on lanes.
struct Shape {
    int lanes, per;        // per: rows that a workgroup has at once
    int runs;              // 16-byte (bf16) runs of a row
    int step_b, step_t;    // from a group's row to its next
};

// A row of a group: its sequence and token.
struct At {
    int b, t;
    __device__ __forceinline__ At(int64_t row, int T) : b((int)(row / T)), t((int)(row % T)) {}
    __device__ __forceinline__ void next(const Shape &s, int T)
    {
        b += s.step_b, t += s.step_t;
        if (t >= T)
            t -= T, ++b;
    }
};

// Sum over the group's lanes.  WIDE: the group is the workgroup, whose waves exchange
// their sums through `cell` (two of them, taken in turn, so that one barrier a sum is
// enough: a cell is written again only behind the next sum's barrier).
template <bool WIDE>
__device__ __forceinline__ float row_sum(float v, int lanes, float (*cell)[16], int &turn)
{
    if constexpr (!WIDE) {
        return lanes_sum(v, lanes);
    } else {
        v = lanes_sum(v, 64);
        float *to = cell[turn];
        turn ^= 1;
        if (threadIdx.x % 64 == 0)
            to[threadIdx.x / 64] = v;
        __syncthreads();
        float s = 0.f;
        for (int i = 0; i < lanes / 64; ++i)
            s += to[i];
        return s;
    }
}

template <typename T, int P>
__device__ __forceinline__ void load_row(const T *p, int lane, int lanes, int runs, float (&v)[P][8])
{
#pragma unroll
    for (int k = 0; k < P; ++k) {
        const int at = lane + k * lanes;
        widen_all(p && at < runs ? load_raw<T, 8>(p + 8 * at) : zero_raw<T, 8>(), v[k]);
    }
}
template <typename T, int P>
__device__ __forceinline__ void load_raws(const T *p, int lane, int lanes, int runs, Raw<T, 8> (&v)[P])
{
#pragma unroll
    for (int k = 0; k < P; ++k) {
        const int at = lane + k * lanes;
        v[k] = p && at < runs ? load_raw<T, 8>(p + 8 * at) : zero_raw<T, 8>();
    }
}
template <typename T, int P>
__device__ __forceinline__ void store_row(T *p, int lane, int lanes, int runs, const float (&v)[P][8])
{
#pragma unroll
    for (int k = 0; k < P; ++k) {
        const int at = lane + k * lanes;
        if (at < runs)
            store_all(p + 8 * at, v[k]);
    }
}
// v times a vector's entries (null: ones)
template <typename T, int P>
__device__ __forceinline__ void times(const void *w, int64_t off, int lane, int lanes, int runs, float (&v)[P][8])
{
    if (w == nullptr)
        return;
#pragma unroll
    for (int k = 0; k < P; ++k) {
        const int at = lane + k * lanes;
        if (at < runs) {
            float f[8];
            load_all<T, 8>(static_cast<const T *>(w) + off + 8 * at, f);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[k][e] *= f[e];
        }
    }
}
template <int P>
__device__ __forceinline__ float dot(const float (&a)[P][8], const float (&b)[P][8])
{
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            s = fmaf(a[k][e], b[k][e], s);
    return s;
}
template <int P>
__device__ __forceinline__ void scaled(float (&v)[P][8], float f)
{
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[k][e] *= f;
}

// 1 / sqrt(sum / C + eps)
__device__ __forceinline__ float inverse_rms(float sum, const JoinProblem &p)
{
    return 1.f / sqrtf(sum / (float)p.C + p.eps);
}

template <typename T, typename R, int P, int BLK, bool WIDE>
__global__ __launch_bounds__(BLK) void join_fwd_kernel(JoinProblem p, Shape s)
{
    __shared__ float cell[2][16];
    int turn = 0;
    const int lane = threadIdx.x % s.lanes, grp = threadIdx.x / s.lanes;
    for (At at((int64_t)blockIdx.x * s.per + grp, p.T); at.b < p.B; at.next(s, p.T)) {
        const int b = at.b, t = at.t;
        float r[P][8], f[P][8];
        load_row<R, P>(static_cast<const R *>(p.r.p) + b * p.r.sb + t * p.r.st, lane, s.lanes, s.runs, r);
        if (p.f.p) {
            load_row<T, P>(static_cast<const T *>(p.f.p) + b * p.f.sb + t * p.f.st, lane, s.lanes, s.runs, f);
            if (p.w_post) {
                const float i = inverse_rms(row_sum<WIDE>(dot(f, f), s.lanes, cell, turn), p);
                scaled(f, i);
                times<T, P>(p.w_post, 0, lane, s.lanes, s.runs, f);
            }
            times<T, P>(p.gate, (int64_t)b * p.C, lane, s.lanes, s.runs, f);
            times<T, P>(p.scale, 0, lane, s.lanes, s.runs, f);
#pragma unroll
            for (int k = 0; k < P; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    r[k][e] += f[k][e];
            store_row<R, P>(static_cast<R *>(p.ro.p) + b * p.ro.sb + t * p.ro.st, lane, s.lanes, s.runs, r);
        }
        const float i = inverse_rms(row_sum<WIDE>(dot(r, r), s.lanes, cell, turn), p);
        scaled(r, i);
        times<T, P>(p.w, 0, lane, s.lanes, s.runs, r);
        store_row<T, P>(static_cast<T *>(p.y.p) + b * p.y.sb + t * p.y.st, lane, s.lanes, s.runs, r);
    }
}

// Workgroups blockIdx.x = 0.. of sequence blockIdx.y (one sequence of all rows without a
// gate); their shares: part[sequence][workgroup][Q, dw][C].
template <typename T, typename R, int P, int BLK, bool WIDE>
__global__ __launch_bounds__(BLK) void join_bwd_kernel(JoinProblem p, Shape s, float *part)
{
    __shared__ float cell[2][16];
    __shared__ float sums[WIDE ? 1 : 256 * 8];
    int turn = 0;
    const int lane = threadIdx.x % s.lanes, grp = threadIdx.x / s.lanes, end = p.gate ? blockIdx.y + 1 : p.B;
    float q[P][8] = {}, dw[P][8] = {}, k[P][8];
    // what takes g to the gradient of n_f (or f), the same for all of the workgroup's rows
#pragma unroll
    for (int j = 0; j < P; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            k[j][e] = 1.f;
    times<T, P>(p.gate, (int64_t)blockIdx.y * p.C, lane, s.lanes, s.runs, k);
    times<T, P>(p.scale, 0, lane, s.lanes, s.runs, k);
    times<T, P>(p.w_post, 0, lane, s.lanes, s.runs, k);
    Raw<T, 8> w[P];
    load_raws<T, P>(static_cast<const T *>(p.w), lane, s.lanes, s.runs, w);
    for (At at((int64_t)blockIdx.x * s.per + grp + (p.gate ? (int64_t)blockIdx.y * p.T : 0), p.T); at.b < end; at.next(s, p.T)) {
        const int b = at.b, t = at.t;
        // all of a row's loads ahead of its sums
        Raw<R, 8> rr[P], ro[P];
        Raw<T, 8> ry[P], rf[P];
        load_raws<R, P>(static_cast<const R *>(p.r.p) + b * p.r.sb + t * p.r.st, lane, s.lanes, s.runs, rr);
        load_raws<T, P>(static_cast<const T *>(p.dy.p) + b * p.dy.sb + t * p.dy.st, lane, s.lanes, s.runs, ry);
        load_raws<T, P>(p.f.p ? static_cast<const T *>(p.f.p) + b * p.f.sb + t * p.f.st : nullptr, lane, s.lanes, s.runs, rf);
        load_raws<R, P>(p.dro.p ? static_cast<const R *>(p.dro.p) + b * p.dro.sb + t * p.dro.st : nullptr, lane, s.lanes, s.runs, ro);
        step_fence();
        float r[P][8], g[P][8], f[P][8], i = 0.f;   // r', which is formed again; g; n_f (or f)
#pragma unroll
        for (int j = 0; j < P; ++j)
            widen_all(rr[j], r[j]), widen_all(ry[j], g[j]), widen_all(rf[j], f[j]);
        if (p.f.p) {
            if (p.w_post) {
                i = inverse_rms(row_sum<WIDE>(dot(f, f), s.lanes, cell, turn), p);
                scaled(f, i);
            }
#pragma unroll
            for (int j = 0; j < P; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    r[j][e] = fmaf(k[j][e], f[j][e], r[j][e]);
        }
        const float ir = inverse_rms(row_sum<WIDE>(dot(r, r), s.lanes, cell, turn), p);
#pragma unroll
        for (int j = 0; j < P; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                r[j][e] *= ir;
                dw[j][e] = fmaf(g[j][e], r[j][e], dw[j][e]);
                if (p.w)
                    g[j][e] *= get(w[j], e);
            }
        const float mr = row_sum<WIDE>(dot(g, r), s.lanes, cell, turn) / (float)p.C;
#pragma unroll
        for (int j = 0; j < P; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[j][e] = ir * (g[j][e] - r[j][e] * mr);
                if (p.dro.p)
                    g[j][e] += get(ro[j], e);
            }
        store_row<R, P>(static_cast<R *>(p.dr.p) + b * p.dr.sb + t * p.dr.st, lane, s.lanes, s.runs, g);
        if (!p.f.p)
            continue;
#pragma unroll
        for (int j = 0; j < P; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                q[j][e] = fmaf(g[j][e], f[j][e], q[j][e]);
                g[j][e] *= k[j][e];
            }
        if (p.w_post) {
            const float m = row_sum<WIDE>(dot(g, f), s.lanes, cell, turn) / (float)p.C;
#pragma unroll
            for (int j = 0; j < P; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    g[j][e] = i * (g[j][e] - f[j][e] * m);
        }
        store_row<T, P>(static_cast<T *>(p.df.p) + b * p.df.sb + t * p.df.st, lane, s.lanes, s.runs, g);
    }
    if (part == nullptr)
        return;
    float *out = part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * p.C;
    if constexpr (WIDE) {
        store_row<float, P>(out, lane, s.lanes, s.runs, q);
        store_row<float, P>(out + p.C, lane, s.lanes, s.runs, dw);
    } else {
#pragma unroll
        for (int k = 0; k < 2 * P; ++k) {
            const float(&v)[8] = k < P ? q[k % P] : dw[k % P];
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sums[threadIdx.x * 8 + e] = v[e];
            __syncthreads();
            for (int i = threadIdx.x; i < s.lanes * 8; i += 256) {
                const int at = i / 8 + k % P * s.lanes;
                float a = 0.f;
                for (int j = 0; j < s.per; ++j)
                    a += sums[j * s.lanes * 8 + i];
                if (at < s.runs)
                    out[(k < P ? 0 : p.C) + at * 8 + i % 8] = a;
            }
        }
    }
}

// Sums over a sequence's workgroups: 16 columns a workgroup, whose rows of threads add every
// 64th share, eight in flight, then their sums in order.  One sequence: the gradients;
// several: the sequence's dgate, and its Q and dw for join_total_kernel.
constexpr int kSumRows = 64;

template <typename T>
__device__ __forceinline__ float entry(const void *w, int64_t i)
{
    return w ? load_f(static_cast<const T *>(w) + i) : 1.f;
}

__device__ __forceinline__ float column_sum(const float *in, int64_t step, int n, bool on, float (&sums)[kSumRows][17])
{
    const int i0 = threadIdx.x / 16;
    float s = 0.f;
    if (on)
        for (int i = i0; i < n; i += 8 * kSumRows) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                x[k] = i + k * kSumRows < n ? in[(i + k * kSumRows) * step] : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                s += x[k];
        }
    sums[i0][threadIdx.x % 16] = s;
    __syncthreads();
    float a = 0.f;
    if (i0 == 0)
#pragma unroll
        for (int i = 0; i < kSumRows; ++i)
            a += sums[i][threadIdx.x];
    __syncthreads();
    return a;
}

template <typename T>
__device__ __forceinline__ void put(void *out, int64_t i, float v)
{
    if (out)
        store_f(static_cast<T *>(out) + i, v);
}

template <typename T>
__global__ __launch_bounds__(16 * kSumRows) void join_sum_kernel(JoinProblem p, const float *part, int n, float *each)
{
    __shared__ float sums[kSumRows][17];
    const int c = blockIdx.x * 16 + threadIdx.x % 16, b = blockIdx.y;
    const bool on = c < p.C;
    const float *in = part + (int64_t)b * n * 2 * p.C + c;
    const float q = column_sum(in, 2 * p.C, n, on, sums), d = column_sum(in + p.C, 2 * p.C, n, on, sums);
    if (threadIdx.x >= 16 || !on)
        return;
    const float sc = entry<T>(p.scale, c), wp = entry<T>(p.w_post, c);
    if (p.gate) {
        put<T>(p.dgate, (int64_t)b * p.C + c, sc * wp * q);
        each[((int64_t)b * 2) * p.C + c] = q;
        each[((int64_t)b * 2 + 1) * p.C + c] = d;
        return;
    }
    put<T>(p.dw, c, d);
    put<T>(p.dw_post, c, sc * q);
    put<T>(p.dscale, c, wp * q);
}

// The sums over sequences, Q's weighted by their gates.
template <typename T>
__global__ __launch_bounds__(16 * kSumRows) void join_total_kernel(JoinProblem p, const float *each)
{
    __shared__ float sums[kSumRows][17];
    const int c = blockIdx.x * 16 + threadIdx.x % 16, i0 = threadIdx.x / 16;
    const bool on = c < p.C;
    float q = 0.f;
    if (on)
        for (int b = i0; b < p.B; b += kSumRows)
            q = fmaf(each[(int64_t)b * 2 * p.C + c], entry<T>(p.gate, (int64_t)b * p.C + c), q);
    sums[i0][threadIdx.x % 16] = q;
    __syncthreads();
    float a = 0.f;
    if (i0 == 0)
#pragma unroll
        for (int i = 0; i < kSumRows; ++i)
            a += sums[i][threadIdx.x];
    __syncthreads();
    const float d = column_sum(each + p.C + c, 2 * p.C, p.B, on, sums);
    if (threadIdx.x >= 16 || !on)
        return;
    put<T>(p.dw, c, d);
    put<T>(p.dw_post, c, entry<T>(p.scale, c) * a);
    put<T>(p.dscale, c, entry<T>(p.w_post, c) * a);
}

// A row's lanes: the fewest that hold it in `most` runs each, at least 8.
Shape shape_of(const JoinProblem &p, int most)
{
    Shape s;
    s.runs = p.C / 8;
    s.lanes = 8;
    while (s.lanes < 64 && s.runs > s.lanes)
        s.lanes *= 2;
    while (s.lanes < 1024 && s.runs > s.lanes * most)
        s.lanes *= 4;
    s.per = std::max(256, s.lanes) / s.lanes;
    s.step_b = s.step_t = 0;
    return s;
}

Shape stepping(Shape s, int64_t groups, int T)
{
    s.step_b = (int)(groups * s.per / T);
    s.step_t = (int)(groups * s.per % T);
    return s;
}

// Workgroups that a launch has at most; a group goes along several rows then.
constexpr int64_t kFwdBlocks = 16384, kBwdBlocks = 1024;

template <typename T, typename R, int P, int BLK, bool WIDE>
hipError_t fwd(const JoinProblem &p, const Shape &s, hipStream_t st)
{
    if (p.ws->counting)
        return hipSuccess;
    const int64_t n = std::min(((int64_t)p.B * p.T + s.per - 1) / s.per, kFwdBlocks);
    join_fwd_kernel<T, R, P, BLK, WIDE><<<dim3((unsigned)n), BLK, 0, st>>>(p, stepping(s, n, p.T));
    return hipGetLastError();
}

template <typename T, typename R, int P, int BLK, bool WIDE>
hipError_t bwd(const JoinProblem &p, const Shape &s, hipStream_t st)
{
    const int64_t seqs = p.gate ? p.B : 1, rows = p.gate ? p.T : (int64_t)p.B * p.T;
    if (seqs > 65535)
        return hipErrorInvalidConfiguration;
    const int64_t n = std::max<int64_t>(1, std::min((rows + s.per - 1) / s.per, kBwdBlocks / seqs));
    const bool sums = p.dw || p.dw_post || p.dscale || p.dgate;
    void *part = nullptr, *each = nullptr;
    hipError_t e = sums ? p.ws->take(&part, (size_t)(seqs * n * 2 * p.C * 4)) : hipSuccess;
    if (e == hipSuccess && sums && p.gate)
        e = p.ws->take(&each, (size_t)(seqs * 2 * p.C * 4));
    if (e != hipSuccess || p.ws->counting)
        return e;
    join_bwd_kernel<T, R, P, BLK, WIDE><<<dim3((unsigned)n, (unsigned)seqs), BLK, 0, st>>>(p, stepping(s, n, p.T), static_cast<float *>(part));
    e = hipGetLastError();
    if (e != hipSuccess || !sums)
        return e;
    const unsigned cols = (unsigned)((p.C + 15) / 16);
    join_sum_kernel<T><<<dim3(cols, (unsigned)seqs), 16 * kSumRows, 0, st>>>(p, static_cast<const float *>(part), (int)n, static_cast<float *>(each));
    e = hipGetLastError();
    if (e != hipSuccess || !p.gate)
        return e;
    join_total_kernel<T><<<dim3(cols), 16 * kSumRows, 0, st>>>(p, static_cast<const float *>(each));
    return hipGetLastError();
}

template <typename T, typename R, bool BWD, int P>
hipError_t pick(const JoinProblem &p, const Shape &s, hipStream_t st)
{
    if constexpr (P * 8 * 1024 <= kJoinMaxRow)   // what rows of more than 256 lanes can take
        if (s.lanes > 256)
            return BWD ? bwd<T, R, P, 1024, true>(p, s, st) : fwd<T, R, P, 1024, true>(p, s, st);
    if (s.lanes > 64)
        return BWD ? bwd<T, R, P, 256, true>(p, s, st) : fwd<T, R, P, 256, true>(p, s, st);
    return BWD ? bwd<T, R, P, 256, false>(p, s, st) : fwd<T, R, P, 256, false>(p, s, st);
}

template <typename T, typename R, bool BWD>
hipError_t pick(const JoinProblem &p, hipStream_t st)
{
    const Shape s = shape_of(p, 3);
    switch ((s.runs + s.lanes - 1) / s.lanes) {
    case 1: return pick<T, R, BWD, 1>(p, s, st);
    case 2: return pick<T, R, BWD, 2>(p, s, st);
    default: return pick<T, R, BWD, 3>(p, s, st);
    }
}

template <bool BWD>
hipError_t pick(const JoinProblem &p, hipStream_t st)
{
    if (p.dtype == 0)
        return pick<float, float, BWD>(p, st);
    return p.rdtype == 0 ? pick<bf16_t, float, BWD>(p, st) : pick<bf16_t, bf16_t, BWD>(p, st);
}

}  // namespace

hipError_t launch_join_fwd(const JoinProblem &p, hipStream_t s) { return pick<false>(p, s); }
hipError_t launch_join_bwd(const JoinProblem &p, hipStream_t s) { return pick<true>(p, s); }

}  // namespace gspn
