// Device code that both passes of the selective scan share (internal).
#pragma once

#include <algorithm>

#include "selective.hpp"
#include "vec.hpp"

namespace gspn {
namespace sel {

using namespace vec;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 2^x, one instruction (relative error 2^-23; below 2^-126: 0)
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// A log2 e, kept finite: a step of 0 (a token past a sequence's end) leaves a state as it is
// at any rate, where 0 times an infinite one is NaN, and 2^(d A) is 0 as soon as d > 2^-120.
__device__ __forceinline__ float rate(float A)
{
    const float a = A * kLog2e;
    return a < -3.402823466e38f ? -3.402823466e38f : a;
}

// log(1 + e^x) = max(x, 0) + log(1 + e), e = exp(-|x|) <= 1: with w = 1 + e rounded, log(1 + e)
// is log w plus what the rounding lost, e - (w - 1), as small e would otherwise be.
__device__ __forceinline__ float softplus(float x)
{
    const float e = exp2_hw(-fabsf(x) * kLog2e), w = 1.f + e;
    return fmaxf(x, 0.f) + (__builtin_amdgcn_logf(w) * kLn2 + (e - (w - 1.f)));
}

// The same with its derivative, 1 / (1 + e^-x), which shares e and w.
__device__ __forceinline__ float softplus(float x, float &grad)
{
    const float e = exp2_hw(-fabsf(x) * kLog2e), w = 1.f + e, i = __builtin_amdgcn_rcpf(w);
    grad = x < 0.f ? e * i : i;
    return fmaxf(x, 0.f) + (__builtin_amdgcn_logf(w) * kLn2 + (e - (w - 1.f)));
}

__device__ __forceinline__ int length_of(const SelectiveProblem &p, int b)
{
    return p.lens ? min(max(p.lens[b], 0), p.T) : p.T;
}

// Packed B and C are not written while these kernels run, and their addresses are the same
// in all lanes: constant address space, so that they come through scalar loads.
typedef const float __attribute__((address_space(4))) cfloat;
__device__ __forceinline__ cfloat *constant(const float *p)
{
    return (cfloat *)(uintptr_t)p;
}

// A row of a [B][T][C] tensor: a scalar address and a scalar step from token to token in
// bytes (strides are up to 2^23 elements); a lane adds the offset of its channel, in bytes
// too, so that an access takes the address as it is.
template <typename T>
struct RowAt {
    const char *p;
    int step;
    __device__ __forceinline__ RowAt(const Heads &h, int b, int t)
        : p(static_cast<const char *>(h.p) + (b * h.sb + t * h.st) * (int64_t)sizeof(T)), step((int)(h.st * (int64_t)sizeof(T)))
    {
    }
    __device__ __forceinline__ void next() { p += step; }
    __device__ __forceinline__ uint32_t load(uint32_t off) const
    {
        if constexpr (sizeof(T) == 2)
            return *reinterpret_cast<const uint16_t *>(p + off);
        else
            return *reinterpret_cast<const uint32_t *>(p + off);
    }
    __device__ __forceinline__ void store(uint32_t off, float v) const { store_f(reinterpret_cast<T *>(const_cast<char *>(p) + off), v); }
};
template <typename T>
__device__ __forceinline__ float widened(uint32_t raw)
{
    return sizeof(T) == 2 ? bf_lo(raw) : __uint_as_float(raw);
}

// Whether v is infinite in any lane.  States past N, where the kernels hold more, have B and C
// of 0 and stay 0, but for products with infinite inputs: these are looked for a token (or more)
// at once, so that what puts the states right costs nothing else.  (NaN reaches all states.)
__device__ __forceinline__ bool any_infinite(float v) { return __any(fabsf(v) == __builtin_inff()); }

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

// The chain over n chunks: from what each adds to the states (or gradients, BACK: from the
// last chunk on) that it begins with, to these, in the same place; `from` is what the first
// begins with, null for zeros.  The last adds to nothing.  A workgroup takes 64 columns (a
// state of a channel), up to 16 runs of chunks side by side: each run from zeros with its
// whole decay, then, from what the runs ahead of it come to, its chunks one by one.  Where
// chunks are many and channels few that is what the chain's time goes by (34225 tokens of 16
// channels: the call 201 us with one run, 84 with 16); runs of fewer chunks than are loaded at
// once cost more than they save (43 chunks of 196608 columns: 37 us in 16 runs, 18 in three).
constexpr int kJoinRuns = 16, kJoinColumns = 64, kJoinAhead = 16;

template <int NP, bool BACK>
__global__ __launch_bounds__(kJoinRuns *kJoinColumns) void join_chunks_kernel(SelectiveProblem p, int n, float *ends, const float *steps, const float *from)
{
    constexpr int U = kJoinAhead;
    __shared__ float h_[kJoinRuns][kJoinColumns], s_[kJoinRuns][kJoinColumns];
    const int col = threadIdx.x % kJoinColumns, run = threadIdx.x / kJoinColumns, b = blockIdx.y;
    const int64_t i = (int64_t)blockIdx.x * kJoinColumns + col, step = (int64_t)NP * p.C;
    const bool on = i < step;
    const int c = (int)(i % p.C), st = on ? (int)(i / p.C) : NP;
    const int runs = blockDim.x / kJoinColumns, per = (n + runs - 1) / runs, k0 = run * per, k1 = min(k0 + per, n);
    const float a2 = st < p.N ? rate(p.A[(int64_t)c * p.N + st]) : 0.f;
    float *const at = ends + (int64_t)b * n * step + i;
    const float *const s = steps + (int64_t)b * n * p.C + c;
    const auto chunk = [&](int k) { return (int64_t)(BACK ? n - 1 - k : k); };
    float add[U], sum[U];
    const auto fetch = [&](int k) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const bool in = on && k + j < min(k1, n - 1);
            add[j] = in ? at[chunk(k + j) * step] : 0.f;
            sum[j] = in ? s[chunk(k + j) * p.C] : 0.f;
        }
    };
    float h = 0.f, total = 0.f;
    for (int k = k0; k < k1; k += U) {
        fetch(k);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            h = fmaf(exp2_hw(a2 * sum[j]), h, add[j]);
            total += sum[j];
        }
    }
    h_[run][col] = h, s_[run][col] = total;
    __syncthreads();
    h = from && st < p.N ? from[((int64_t)b * p.C + c) * p.N + st] : 0.f;
    for (int r = 0; r < run; ++r)
        h = fmaf(exp2_hw(a2 * s_[r][col]), h, h_[r][col]);
    for (int k = k0; k < k1; k += U) {
        if (per > U)   // else they are still here
            fetch(k);
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (on && k + j < k1) {
                at[chunk(k + j) * step] = h;
                h = fmaf(exp2_hw(a2 * sum[j]), h, add[j]);
            }
    }
}

template <int NP, bool BACK>
hipError_t join_chunks(const SelectiveProblem &p, int n, float *ends, const float *steps, const float *from, hipStream_t s)
{
    const int64_t groups = ((int64_t)NP * p.C + kJoinColumns - 1) / kJoinColumns;
    const int runs = std::min(kJoinRuns, (n + kJoinAhead - 1) / kJoinAhead);
    join_chunks_kernel<NP, BACK><<<dim3((unsigned)groups, (unsigned)p.B), runs * kJoinColumns, 0, s>>>(p, n, ends, steps, from);
    return hipGetLastError();
}

// Tokens of a chunk, at least: few, where waves are few, but as many chunks as these take a
// chain (a channel's 34225 tokens of one sequence: chunks of 16 are 2140).
inline int64_t least_tokens(int T)
{
    int64_t n = 16;
    while (16 * n * n < T)
        n += 8;
    return n;
}

}  // namespace sel
}  // namespace gspn
