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

// Step of a token from its entry of dt.
__device__ __forceinline__ float step_of(float raw, bool soft) { return soft ? softplus(raw) : raw; }

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

}  // namespace sel
}  // namespace gspn
