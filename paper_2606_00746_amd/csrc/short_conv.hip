// The short causal convolution of channels along the tokens (gspn_short_conv_fwd, _bwd).
//
//   u_t = bias + sum_j w_j x_{t-K+1+j},  y = u sigmoid(u) (or u)
//   du = dy (s + u s (1 - s)),  dx_t = sum_j w_j du_{t+K-1-j},
//   dw_j = sum_t du_t x_{t-K+1+j},  dbias = sum_t du_t
//
// Bound by memory: x read once and y written (x and dy read, dx written).  A thread owns
// a run of neighbouring channels and a segment of tokens, which it goes along with the
// last K - 1 inputs (and gradients) in registers; the tokens ahead of a segment are read
// again, from the caches.  The weights' gradients are shares per workgroup, added up in
// a fixed order by a second launch.  bf16, 4 taps: forward 169 us for 32 x 5476 tokens of
// 1152 channels (4.8 TB/s); 8 x 4096 tokens of 1536 channels 41 us (4.9), gradient 75 (4.0).
#include <algorithm>

#include "short_conv.hpp"
#include "vec.hpp"

namespace gspn {
namespace {

using namespace vec;

constexpr int kBlk = 256;

// How a call's channels and tokens lie on threads.  Forward: run after run of V channels,
// segment after segment.  Backward, whose workgroups add up the shares of a channel: pb runs
// by sb segments a workgroup.
struct Shape {
    int runs, pb, sb, segs;   // runs of a row; of a workgroup; segments of a workgroup, of a sequence
    int len;                  // tokens of a segment
    dim3 grid;
    bool fits;
};

Shape shape_of(const ConvProblem &p, int V, int len, bool bwd)
{
    Shape s;
    s.runs = p.C / V;
    s.segs = (p.T + len - 1) / len;
    s.len = len;
    if (!bwd) {
        const int64_t n = ((int64_t)p.B * s.segs * s.runs + kBlk - 1) / kBlk;
        s.pb = s.sb = 0;
        s.fits = n * kBlk <= kMaxThreads;
        s.grid = dim3((unsigned)n);
        return s;
    }
    const int cols = (s.runs + 63) / 64;
    s.pb = (s.runs + cols - 1) / cols;
    s.sb = kBlk / s.pb;
    const int64_t rows = ((int64_t)p.B * s.segs + s.sb - 1) / s.sb;
    // rows vary along x, whose limit is the larger one
    s.fits = rows * cols * kBlk <= kMaxThreads && cols <= 65535;
    s.grid = dim3((unsigned)rows, (unsigned)cols);
    return s;
}

template <typename T, int V, int K>
__device__ __forceinline__ void load_taps(const void *w, int c, float (&f)[K][V])
{
    const T *p = static_cast<const T *>(w) + (int64_t)c * K;
    float flat[K * V];
#pragma unroll
    for (int i = 0; i < K; ++i) {
        float part[V];
        load_all<T, V>(p + i * V, part);
#pragma unroll
        for (int e = 0; e < V; ++e)
            flat[i * V + e] = part[e];
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
#pragma unroll
        for (int j = 0; j < K; ++j)
            f[j][e] = flat[e * K + j];
}

__device__ __forceinline__ int length_of(const ConvProblem &p, int b)
{
    return p.lens ? min(max(p.lens[b], 0), p.T) : p.T;
}

// The K - 1 inputs ahead of token t0: the sequence's own, or the state's.
template <typename T, int V, int K>
__device__ __forceinline__ void load_window(const ConvProblem &p, const T *x, int b, int c, int t0, int n, float (&win)[K][V])
{
#pragma unroll
    for (int i = 0; i < K - 1; ++i) {
        const int t = t0 - (K - 1) + i;
        Raw<T, V> r = zero_raw<T, V>();
        if (t >= 0) {
            if (t < n)
                r = load_raw<T, V>(x + (int64_t)t * p.x.st);
        } else if (p.state) {
            r = load_raw<T, V>(static_cast<const T *>(p.state) + ((int64_t)b * (K - 1) + (K - 1 + t)) * p.C + c);
        }
        widen_all(r, win[i]);
    }
}

// Tokens that a thread has in flight.
constexpr int kAhead = 8;

template <typename T, int V, int K>
__global__ __launch_bounds__(kBlk) void conv_fwd_kernel(ConvProblem p, Shape s)
{
    const unsigned item = blockIdx.x * (unsigned)kBlk + threadIdx.x, seg = item / (unsigned)s.runs;
    if (seg >= (uint64_t)p.B * s.segs)
        return;
    const int b = (int)(seg / (unsigned)s.segs), t0 = (int)(seg % (unsigned)s.segs) * s.len, t1 = min(t0 + s.len, p.T);
    const int n = length_of(p, b), c = (int)(item % (unsigned)s.runs) * V;
    const T *x = static_cast<const T *>(p.x.p) + b * p.x.sb + c;
    T *y = static_cast<T *>(p.y.p) + b * p.y.sb + c;

    float w[K][V], bias[V], win[K][V];
    load_taps<T, V, K>(p.w, c, w);
    widen_all(p.bias ? load_raw<T, V>(static_cast<const T *>(p.bias) + c) : zero_raw<T, V>(), bias);
    load_window<T, V, K>(p, x, b, c, t0, n, win);

    if (t0 == 0 && p.state_out) {
        // The last K - 1 inputs of state and sequence.  The one thread that reads the
        // state's channels writes them, each row behind its last reading, so that a
        // state may be continued in place.
        T *end = static_cast<T *>(p.state_out) + (int64_t)b * (K - 1) * p.C + c;
        const T *st = static_cast<const T *>(p.state) + (int64_t)b * (K - 1) * p.C + c;
        for (int i = 0; i < K - 1; ++i) {
            const int t = n + i - (K - 1);
            float f[V];
            widen_all(t >= 0 ? load_raw<T, V>(x + (int64_t)t * p.x.st) : p.state ? load_raw<T, V>(st + (int64_t)(n + i) * p.C) : zero_raw<T, V>(), f);
            store_all(end + (int64_t)i * p.C, f);
        }
    }
    for (int t = t0; t < t1; t += kAhead) {
        Raw<T, V> in[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            in[i] = t + i < min(t1, n) ? load_raw<T, V>(x + (int64_t)(t + i) * p.x.st) : zero_raw<T, V>();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (t + i >= t1)
                break;
            float u[V];
            widen_all(in[i], win[K - 1]);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                u[e] = bias[e];
#pragma unroll
                for (int j = 0; j < K; ++j)
                    u[e] = fmaf(w[j][e], win[j][e], u[e]);
                u[e] = t + i < n ? (p.silu ? silu(u[e]) : u[e]) : 0.f;
            }
            store_all(y + (int64_t)(t + i) * p.y.st, u);
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    win[j][e] = win[j + 1][e];
        }
    }
}

// Step t has du_t in hand, and with the K - 1 before it the gradient of x_{t-K+1}.  The
// workgroup's shares of dw and dbias: part[row of workgroups][K + 1][C].
template <typename T, int V, int K>
__global__ __launch_bounds__(kBlk) void conv_bwd_kernel(ConvProblem p, Shape s, float *part)
{
    __shared__ float sums[(K + 1) * V * kBlk];
    const int pc = threadIdx.x % s.pb, sl = threadIdx.x / s.pb;
    const int run = blockIdx.y * s.pb + pc;
    const int64_t seg = (int64_t)blockIdx.x * s.sb + sl;
    const bool on = sl < s.sb && run < s.runs && seg < (int64_t)p.B * s.segs;
    float dw[K][V] = {}, db[V] = {};
    if (on) {
        const int b = (int)(seg / s.segs), t0 = (int)(seg % s.segs) * s.len, t1 = min(t0 + s.len, p.T), c = run * V;
        const int n = length_of(p, b);
        const T *x = static_cast<const T *>(p.x.p) + b * p.x.sb + c;
        const T *dy = static_cast<const T *>(p.dy.p) + b * p.dy.sb + c;
        T *dx = static_cast<T *>(p.dx.p) + b * p.dx.sb + c;
        const int64_t state = (int64_t)b * (K - 1) * p.C + c;

        float w[K][V], bias[V], win[K][V], du[K][V] = {};
        load_taps<T, V, K>(p.w, c, w);
        widen_all(p.bias ? load_raw<T, V>(static_cast<const T *>(p.bias) + c) : zero_raw<T, V>(), bias);
        load_window<T, V, K>(p, x, b, c, t0, n, win);
        constexpr int kStep = kAhead / 2;
        for (int t = t0; t < t1 + K - 1; t += kStep) {
            Raw<T, V> in[kStep], up[kStep];
#pragma unroll
            for (int i = 0; i < kStep; ++i) {
                const bool live = t + i < min(t1 + K - 1, n);
                in[i] = live ? load_raw<T, V>(x + (int64_t)(t + i) * p.x.st) : zero_raw<T, V>();
                up[i] = live ? load_raw<T, V>(dy + (int64_t)(t + i) * p.dy.st) : zero_raw<T, V>();
            }
#pragma unroll
            for (int i = 0; i < kStep; ++i) {
                const int at = t + i;
                if (at >= t1 + K - 1)
                    break;
                widen_all(in[i], win[K - 1]);
                widen_all(up[i], du[K - 1]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float u = bias[e];
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        u = fmaf(w[j][e], win[j][e], u);
                    if (p.silu)
                        du[K - 1][e] *= silu_grad(u);
                    if (at >= n)   // also where u is not a number
                        du[K - 1][e] = 0.f;
                    if (at < min(t1, n)) {
                        db[e] += du[K - 1][e];
#pragma unroll
                        for (int j = 0; j < K; ++j)
                            dw[j][e] = fmaf(du[K - 1][e], win[j][e], dw[j][e]);
                    }
                }
                const int to = at - (K - 1);   // the input whose gradient is whole now
                if (to >= t0 || (t0 == 0 && p.dstate_in)) {
                    float g[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        g[e] = 0.f;
#pragma unroll
                        for (int j = 0; j < K; ++j)
                            g[e] = fmaf(w[K - 1 - j][e], du[j][e], g[e]);
                    }
                    const int row = to - n + K - 1;   // of state_out, which may have taken it
                    if (p.dstate && row >= 0 && row < K - 1) {
                        float d[V];
                        load_all<T, V>(static_cast<const T *>(p.dstate) + state + (int64_t)row * p.C, d);
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            g[e] += d[e];
                    }
                    if (to >= n)
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            g[e] = 0.f;
                    if (to >= 0)
                        store_all(dx + (int64_t)to * p.dx.st, g);
                    else
                        store_all(static_cast<T *>(p.dstate_in) + state + (int64_t)(to + K - 1) * p.C, g);
                }
#pragma unroll
                for (int j = 0; j < K - 1; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        win[j][e] = win[j + 1][e];
                        du[j][e] = du[j + 1][e];
                    }
            }
        }
    }
    if (part == nullptr)
        return;
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int j = 0; j < K; ++j)
            sums[(j * V + e) * kBlk + threadIdx.x] = dw[j][e];
        sums[(K * V + e) * kBlk + threadIdx.x] = db[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (K + 1) * V * s.pb; i += kBlk) {
        const int q = i % s.pb, je = i / s.pb, at = blockIdx.y * s.pb + q;
        if (at >= s.runs)
            continue;
        float a = 0.f;
        for (int k = 0; k < s.sb; ++k)
            a += sums[je * kBlk + k * s.pb + q];
        part[((int64_t)blockIdx.x * (K + 1) + je / V) * p.C + at * V + je % V] = a;
    }
}

// dw and dbias from the workgroups' shares: 16 channels a workgroup, whose rows of
// threads add every 64th share, eight in flight, then their sums in order.
constexpr int kSumRows = 64;
template <typename T>
__global__ __launch_bounds__(16 * kSumRows) void conv_dw_kernel(ConvProblem p, const float *part, int n)
{
    __shared__ float sums[kSumRows][17];
    const int j = blockIdx.y, c = blockIdx.x * 16 + threadIdx.x % 16, i0 = threadIdx.x / 16;
    const int64_t step = (int64_t)(p.K + 1) * p.C;
    const float *in = part + (int64_t)j * p.C + c;
    float s = 0.f;
    if (c < p.C)
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
    if (i0 == 0 && c < p.C) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < kSumRows; ++i)
            a += sums[i][threadIdx.x];
        if (j < p.K && p.dw)
            store_f(static_cast<T *>(p.dw) + (int64_t)c * p.K + j, a);
        if (j == p.K && p.dbias)
            store_f(static_cast<T *>(p.dbias) + c, a);
    }
}

// Channels of a thread: forward 8 where the taps leave registers for them (us with 8 and 4, 8 x
// 4096 tokens of 1536 channels and 32 x 5476 of 1152: bf16 40 and 40, 175 and 169; fp32 92 and
// 87, 349 and 323: the 8 are not what carries it), backward 4 (for the waves that fewer
// registers allow: bf16 97 and 75, 329 and 385; fp32 150 and 140, 549 and 652).
// Tokens of a thread's segment: many, so that few are read twice, but fewer where that
// leaves the card with few threads.
constexpr int64_t kFewThreads = 128 * 1024;
int segment(const ConvProblem &p, int V, int most)
{
    int len = most;
    while (len > 8 && (int64_t)p.B * ((p.T + len - 1) / len) * (p.C / V) < kFewThreads)
        len /= 2;
    return len;
}

template <typename T, int K>
hipError_t fwd(const ConvProblem &p, hipStream_t s)
{
    constexpr int V = K <= 4 ? 8 : 4;
    const Shape sh = shape_of(p, V, segment(p, V, 32), false);
    if (!sh.fits)
        return hipErrorInvalidConfiguration;
    if (p.ws->counting)
        return hipSuccess;
    conv_fwd_kernel<T, V, K><<<sh.grid, kBlk, 0, s>>>(p, sh);
    return hipGetLastError();
}

template <typename T, int K>
hipError_t bwd(const ConvProblem &p, hipStream_t s)
{
    constexpr int V = 4;
    const Shape sh = shape_of(p, V, segment(p, V, 64), true);
    if (!sh.fits)
        return hipErrorInvalidConfiguration;
    void *part = nullptr;
    if (p.dw || p.dbias) {
        const hipError_t e = p.ws->take(&part, (size_t)sh.grid.x * (K + 1) * p.C * 4);
        if (e != hipSuccess)
            return e;
    }
    if (p.ws->counting)
        return hipSuccess;
    conv_bwd_kernel<T, V, K><<<sh.grid, kBlk, 0, s>>>(p, sh, static_cast<float *>(part));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !part)
        return e;
    conv_dw_kernel<T><<<dim3((unsigned)((p.C + 15) / 16), K + 1), 16 * kSumRows, 0, s>>>(p, static_cast<const float *>(part), (int)sh.grid.x);
    return hipGetLastError();
}

template <typename T, bool BWD>
hipError_t pick(const ConvProblem &p, hipStream_t s)
{
    switch (p.K) {
#define GSPN_TAPS(k) case k: return BWD ? bwd<T, k>(p, s) : fwd<T, k>(p, s);
        GSPN_TAPS(2) GSPN_TAPS(3) GSPN_TAPS(4) GSPN_TAPS(5) GSPN_TAPS(6) GSPN_TAPS(7)
#undef GSPN_TAPS
    default: return BWD ? bwd<T, 8>(p, s) : fwd<T, 8>(p, s);
    }
}

}  // namespace

hipError_t launch_conv_fwd(const ConvProblem &p, hipStream_t s)
{
    return p.dtype == 0 ? pick<float, false>(p, s) : pick<bf16_t, false>(p, s);
}

hipError_t launch_conv_bwd(const ConvProblem &p, hipStream_t s)
{
    return p.dtype == 0 ? pick<float, true>(p, s) : pick<bf16_t, true>(p, s);
}

}  // namespace gspn
