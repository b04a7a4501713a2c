// Device code that both passes of the selective scan share (internal).
#pragma once

#include "selective.hpp"
#include "vec.hpp"

namespace gspn {
namespace sel {

using namespace vec;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 2^x, one instruction (relative error 2^-23; below 2^-126: 0)
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

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

}  // namespace sel
}  // namespace gspn
