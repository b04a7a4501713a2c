// Runs of 1 to 8 neighbouring elements of a row, in the storage type: loaded as they lie
// (the widest loads that their alignment allows), widened to fp32, stored rounded to
// nearest even.  Sums over groups of lanes.
#pragma once

#include <type_traits>

#include "cdna.hpp"
#include "device.hpp"

namespace gspn {
namespace vec {

using namespace cdna;

// V elements of T as they lie in memory.
template <typename T, int V>
struct Raw {
    static constexpr int kWords = (V * (int)sizeof(T) + 3) / 4;
    uint32_t w[kWords];
};

template <typename T, int V>
__device__ __forceinline__ Raw<T, V> load_raw(const T *p)
{
    constexpr int n = V * (int)sizeof(T);
    Raw<T, V> r;
    if constexpr (n == 2) {
        r.w[0] = *reinterpret_cast<const uint16_t *>(p);
    } else if constexpr (n == 4) {
        r.w[0] = *reinterpret_cast<const uint32_t *>(p);
    } else if constexpr (n == 8) {
        const uint2 u = *reinterpret_cast<const uint2 *>(p);
        r.w[0] = u.x, r.w[1] = u.y;
    } else {
        static_assert(n % 16 == 0);
#pragma unroll
        for (int i = 0; i < n / 16; ++i) {
            const uint4 u = reinterpret_cast<const uint4 *>(p)[i];
            r.w[4 * i] = u.x, r.w[4 * i + 1] = u.y, r.w[4 * i + 2] = u.z, r.w[4 * i + 3] = u.w;
        }
    }
    return r;
}

template <typename T, int V>
__device__ __forceinline__ Raw<T, V> zero_raw()
{
    Raw<T, V> r;
#pragma unroll
    for (int i = 0; i < Raw<T, V>::kWords; ++i)
        r.w[i] = 0;
    return r;
}

// Element e, a constant once unrolled.
template <int V>
__device__ __forceinline__ float get(const Raw<bf16_t, V> &r, int e)
{
    return (e & 1) ? bf_hi(r.w[e >> 1]) : bf_lo(r.w[e >> 1]);
}
template <int V>
__device__ __forceinline__ float get(const Raw<float, V> &r, int e)
{
    return __uint_as_float(r.w[e]);
}

template <typename T, int V>
__device__ __forceinline__ void widen_all(const Raw<T, V> &r, float (&f)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e)
        f[e] = get(r, e);
}

template <typename T, int V>
__device__ __forceinline__ void load_all(const T *p, float (&f)[V])
{
    widen_all(load_raw<T, V>(p), f);
}

__device__ __forceinline__ void store_words(void *p, const uint32_t *w, std::integral_constant<int, 1>)
{
    *reinterpret_cast<uint32_t *>(p) = w[0];
}
// Data of wide stores is opaque ahead of them: of constants the compiler would otherwise
// form a second copy for the wait states behind a store, and write over the first.
__device__ __forceinline__ void store_words(void *p, const uint32_t *w, std::integral_constant<int, 2>)
{
    u32x2 v{w[0], w[1]};
    asm volatile("" : "+v"(v));
    put8(p, v);
}
template <int N>
__device__ __forceinline__ void store_words(void *p, const uint32_t *w, std::integral_constant<int, N>)
{
    static_assert(N % 4 == 0);
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        u32x4 v{w[i], w[i + 1], w[i + 2], w[i + 3]};
        asm volatile("" : "+v"(v));
        put16(reinterpret_cast<uint32_t *>(p) + i, v);
    }
}

template <int V>
__device__ __forceinline__ void store_all(float *p, const float (&f)[V])
{
    uint32_t w[V];
#pragma unroll
    for (int e = 0; e < V; ++e)
        w[e] = __float_as_uint(f[e]);
    store_words(p, w, std::integral_constant<int, V>{});
}
template <int V>
__device__ __forceinline__ void store_all(bf16_t *p, const float (&f)[V])
{
    if constexpr (V == 1) {
        store_f(p, f[0]);
    } else {
        uint32_t w[V / 2];
#pragma unroll
        for (int e = 0; e < V; e += 2)
            w[e / 2] = pack2(f[e], f[e + 1]);
        store_words(p, w, std::integral_constant<int, V / 2>{});
    }
}

// x of another lane of the same 16, all of which are there (with bound_ctrl the compiler
// makes it part of the addition that takes it).
template <int CTRL>
__device__ __forceinline__ float dpp(float x)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;

// Sum over groups of n lanes (a power of two up to 64), in every lane of a group; the
// order of the additions is the same in all of them.
__device__ __forceinline__ float lanes_sum(float v, int n)
{
    if (n > 1)
        v += dpp<kXor1>(v);
    if (n > 2)
        v += dpp<kXor2>(v);
    if (n > 4)
        v += dpp<kMirror8>(v);
    if (n > 8)
        v += dpp<kMirror16>(v);
    if (n > 16)
        v += __shfl_xor(v, 16);
    if (n > 32)
        v += __shfl_xor(v, 32);
    return v;
}

// b in the lanes of a mask, a in the others (a branch around what forms b costs more).
__device__ __forceinline__ float in_lanes(float a, float b, uint64_t mask)
{
    float r;
    asm("v_cndmask_b32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(mask));
    return r;
}
constexpr uint64_t kOddLanes = 0xAAAAAAAAAAAAAAAAull, kOddPairs = 0xCCCCCCCCCCCCCCCCull;

// x sigmoid(x) and its derivative; -inf gives 0 (not NaN) in both.
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.f + __expf(-x)); }
__device__ __forceinline__ float silu(float x)
{
    const float s = logistic(x);
    return s == 0.f ? 0.f : x * s;
}
__device__ __forceinline__ float silu_grad(float x)
{
    const float s = logistic(x), m = s * (1.f - s);
    return m == 0.f ? s : fmaf(x, m, s);
}
// Both.
__device__ __forceinline__ float silu(float x, float &grad)
{
    const float s = logistic(x), m = s * (1.f - s);
    grad = m == 0.f ? s : fmaf(x, m, s);
    return s == 0.f ? 0.f : x * s;
}

}  // namespace vec
}  // namespace gspn
