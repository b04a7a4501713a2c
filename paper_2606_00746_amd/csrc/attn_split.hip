// Windowed attention of few queries a sequence (gspn_window_attn_decode, and
// forwards of few queries): the keys split over waves and workgroups.
//
// What counts is one pass over the keys and values that the queries see.  The
// G query heads that share a key head, times the Tq queries, are the rows of
// one problem, 16 of them a workgroup, so that shared keys are read once.  A
// wave takes blocks of 32 keys in turn: K straight into registers as the A
// operand of S^T = K Q^T (16 x 16 matrix instructions, lane l: key l % 16, 16
// bytes of it), V through a piece of LDS of the wave's own, where it is turned
// around for O^T = V^T P^T.  The next block's loads are in flight meanwhile.
// Each wave keeps its running maximum, sum and output; the workgroup's four are
// joined in LDS, and those of several workgroups by attn_join_kernel, in order.
//
// Bound by memory where there is work: one token each of 64 sequences over caches of
// up to 8192, 16 heads of 128 on 4, bf16, in 166 to 173 us, 4.8 TB/s, and 5 for the join;
// for a token of one sequence with a window of 4096 a trace has 10.4 and 3.9 us.
// Made for few rows: every 16 of them read the keys again.  One sequence of 8192 keys, 16
// heads of 128 on 4, whole prompts at the end (us, here and by the forward proper): 256
// tokens 101 and 138, 512 170 and 137, 2048 564 and 174; 8 sequences: 32 tokens 98 and 136,
// 128 320 and 138, 2048 4098 and 999.
#include <algorithm>

#include "attn.hpp"

namespace gspn {
namespace {

using namespace attn;

constexpr int kCol = 16;     // query rows of a workgroup
constexpr int kBlock = 32;   // keys of a block

// v over the four lanes l % 16 + 16 u of a row.
__device__ __forceinline__ float quad_max(float v)
{
    v = half_max(v);
    const uint32_t b = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float v)
{
    v = half_sum(v);
    const uint32_t b = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ f32x4_t mma16(Frag<bf16_t> a, Frag<bf16_t> b, f32x4_t acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mma16(Frag<float> a, Frag<float> b, f32x4_t acc)
{
#pragma unroll
    for (int e = 0; e < 4; ++e)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], acc, 0, 0, 0);
    return acc;
}

// acc[db] += V^T P over the wave's block of 32 keys; p[t]: keys 16 t + 4 u + 0..3.
// bf16: P as a sum of two bf16 terms, 16 bits, so that what is left of an output's error
// is its own rounding: memory bounds this kernel, and the second product is free.
template <int DP>
__device__ __forceinline__ void mma16_turned(const char *lds, const f32x4_t (&p)[2],
                                             f32x4_t (&acc)[DP / 16], const bf16_t *)
{
    using X = Tile<bf16_t, DP>;
    const int l = threadIdx.x % 64, u = l / 16, i = l % 16, r = 4 * u + (i >> 2);
    const uint4 w = make_uint4(pack2(p[0][0], p[0][1]), pack2(p[0][2], p[0][3]),
                               pack2(p[1][0], p[1][1]), pack2(p[1][2], p[1][3]));
    const uint4 x = make_uint4(pack2(p[0][0] - bf_lo(w.x), p[0][1] - bf_hi(w.x)), pack2(p[0][2] - bf_lo(w.y), p[0][3] - bf_hi(w.y)),
                               pack2(p[1][0] - bf_lo(w.z), p[1][1] - bf_hi(w.z)), pack2(p[1][2] - bf_lo(w.w), p[1][3] - bf_hi(w.w)));
    const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, w), rest = __builtin_bit_cast(bf16x8_t, x);
#pragma unroll
    for (int db = 0; db < DP / 16; ++db) {
        const int c = 2 * db + ((i & 3) >> 1), in = 8 * (i & 1);
        struct {
            s16x4_t a, b;
        } both = {read_turned(lds + X::at(r, c) + in), read_turned(lds + X::at(16 + r, c) + in)};
        const bf16x8_t v = __builtin_bit_cast(bf16x8_t, both);
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, rest, acc[db], 0, 0, 0);
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pb, acc[db], 0, 0, 0);
    }
}
template <int DP>
__device__ __forceinline__ void mma16_turned(const char *lds, const f32x4_t (&p)[2],
                                             f32x4_t (&acc)[DP / 16], const float *)
{
    using X = Tile<float, DP>;
    const int l = threadIdx.x % 64, u = l / 16, d = l % 16;
#pragma unroll
    for (int db = 0; db < DP / 16; ++db)
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const float a = *reinterpret_cast<const float *>(
                lds + X::at(16 * (r / 4) + 4 * u + r % 4, 4 * db + d / 4) + 4 * (d % 4));
            acc[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, p[r / 4][r % 4], acc[db], 0, 0, 0);
        }
}

// One block's K and V in registers: pieces past the last key or column are zero.
template <typename T, int DP>
struct Block {
    using X = Tile<T, DP>;
    static constexpr int kSlices = X::kPieces / 4, kLoads = kBlock * X::kPieces / 64;
    Frag<T> k[2][kSlices];
    uint4 v[kLoads];
    __device__ __forceinline__ void load(const T *kp, int64_t ks, const T *vp, int64_t vs, int j0, int end,
                                         int D)
    {
        const int l = threadIdx.x % 64;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int j = j0 + 16 * t + l % 16;
#pragma unroll
            for (int s = 0; s < kSlices; ++s) {
                k[t][s].v = decltype(k[t][s].v){};
                if (j < end)
                    k[t][s] = row_frag(kp + j * ks, 4 * s + l / 16, D);
            }
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int x = l + 64 * i, r = x / X::kPieces, c = x % X::kPieces;
            v[i] = make_uint4(0, 0, 0, 0);
            if (j0 + r < end && c * X::kPer < D)
                v[i] = *reinterpret_cast<const uint4 *>(vp + (j0 + r) * vs + c * X::kPer);
        }
    }
    __device__ __forceinline__ void store_v(char *lds) const
    {
        const int l = threadIdx.x % 64;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int x = l + 64 * i;
            *reinterpret_cast<uint4 *>(lds + X::at(x / X::kPieces, x % X::kPieces)) = v[i];
        }
    }
};

// Each workgroup's share of a row: its maximum, its sum and the output over its keys.
struct Shares {
    float *out;      // [tile][split][16][DP]
    float *stat;     // [tile][split][16][2]
    int splits;
};

template <typename T, int DP>
__global__ __launch_bounds__(kThreads, 1) void attn_split_kernel(AttnProblem a, Shares sh)
{
    using X = Tile<T, DP>;
    constexpr int kSlices = X::kPieces / 4, kPitch = DP + 4;
    constexpr int kV = kBlock * X::kS * 16, kO = kCol * kPitch * 4, kWave = kV > kO ? kV : kO;
    __shared__ __attribute__((aligned(16))) char lds[4][kWave];
    __shared__ float stats[4][kCol][2];

    const int G = a.Hq / a.Hkv, rows = a.Tq * G, nt = (rows + kCol - 1) / kCol;
    int id = blockIdx.x;
    const int split = id % sh.splits;
    id /= sh.splits;
    const int tile = id, rt = id % nt;
    id /= nt;
    const int hk = id % a.Hkv, b = id / a.Hkv;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64;
    const int c = l % 16, u = l / 16;
    const int len = seq_len(a, b), off = a.tail ? len - a.Tq : a.offset;

    // the keys that the tile's rows see, in blocks: the sinks ahead of the window, then the window
    const int ta = rt * kCol / G, tb = min(rows - 1, rt * kCol + kCol - 1) / G;
    int lo_t, hi_t, lo_b, hi_b;
    key_bounds(a, len, max(0, ta + off), lo_t, hi_t);
    key_bounds(a, len, tb + off, lo_b, hi_b);
    const int top = min(len - 1, a.right < 0 ? len - 1 : tb + off + a.right);
    const bool none = tb + off < 0 || max(0, ta + off) >= len;
    const int sunk = min(min(a.sinks, lo_t), top + 1), ns = (sunk + kBlock - 1) / kBlock;
    const int n = none ? 0 : ns + (top < lo_t ? 0 : (top - lo_t) / kBlock + 1);
    const int i0 = (int)((int64_t)n * split / sh.splits), i1 = (int)((int64_t)n * (split + 1) / sh.splits);
    const auto key_of = [&](int i) { return i < ns ? i * kBlock : lo_t + (i - ns) * kBlock; };
    const auto end_of = [&](int i) { return i < ns ? sunk : top + 1; };

    const int row = rt * kCol + c, t = min(row, rows - 1) / G, hq = hk * G + min(row, rows - 1) % G;
    int lo, hi;
    key_bounds(a, len, t + off, lo, hi);
    const T *qr = static_cast<const T *>(a.q.p) + b * a.q.sb + t * a.q.st + hq * a.q.sh;
    const T *kp = static_cast<const T *>(a.k.p) + b * a.k.sb + hk * a.k.sh;
    const T *vp = static_cast<const T *>(a.v.p) + b * a.v.sb + hk * a.v.sh;
    Frag<T> qf[kSlices];
#pragma unroll
    for (int s = 0; s < kSlices; ++s)
        qf[s] = row_frag(qr, 4 * s + u, a.D);

    f32x4_t acc[DP / 16];
#pragma unroll
    for (int db = 0; db < DP / 16; ++db)
        acc[db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_inff(), sum = 0.f;
    const float s2 = a.scale * kLog2e;

    Block<T, DP> x;
    if (i0 + w < i1)
        x.load(kp, a.k.st, vp, a.v.st, key_of(i0 + w), end_of(i0 + w), a.D);
    for (int i = i0 + w; i < i1; i += 4) {
        const int k0 = key_of(i), end = end_of(i);
        f32x4_t s[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            s[kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int sl = 0; sl < kSlices; ++sl)
                s[kt] = mma16(x.k[kt][sl], qf[sl], s[kt]);
        }
        x.store_v(lds[w]);
        __builtin_amdgcn_wave_barrier();
        if (i + 4 < i1)
            x.load(kp, a.k.st, vp, a.v.st, key_of(i + 4), end_of(i + 4), a.D);
        float mx = -__builtin_inff();
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = k0 + 16 * kt + 4 * u + e;
                const bool see = j < end && j <= hi && (j >= lo || j < a.sinks);
                s[kt][e] = see ? s[kt][e] : -__builtin_inff();
                mx = fmaxf(mx, s[kt][e]);
            }
        mx = quad_max(mx);
        if (__any(mx > m)) {
            const float mn = fmaxf(m, mx);
            const float f = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((m - mn) * s2);
            m = mn;
            sum *= f;
#pragma unroll
            for (int db = 0; db < DP / 16; ++db)
                acc[db] *= f;
        }
        const float base = m == -__builtin_inff() ? 0.f : m * s2;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[kt][e] = __builtin_amdgcn_exp2f(fmaf(s[kt][e], s2, -base));
                sum += s[kt][e];
            }
        mma16_turned<DP>(lds[w], s, acc, static_cast<const T *>(nullptr));
        __builtin_amdgcn_wave_barrier();
    }
    sum = quad_sum(sum);

    // the four waves' shares, joined
    lds_barrier();
    float *mine = reinterpret_cast<float *>(lds[w]);
#pragma unroll
    for (int db = 0; db < DP / 16; ++db)
        *reinterpret_cast<f32x4_t *>(mine + c * kPitch + 16 * db + 4 * u) = acc[db];
    if (u == 0) {
        stats[w][c][0] = m * s2;
        stats[w][c][1] = sum;
    }
    lds_barrier();
    for (int x4 = threadIdx.x; x4 < kCol * (DP / 4); x4 += kThreads) {
        const int r = x4 / (DP / 4), d = x4 % (DP / 4) * 4;
        float top2 = -__builtin_inff();
#pragma unroll
        for (int v = 0; v < 4; ++v)
            top2 = fmaxf(top2, stats[v][r][0]);
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
        float z = 0.f;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const float mv = stats[v][r][0];
            const float f = mv == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(mv - top2);
            z = fmaf(f, stats[v][r][1], z);
            o += f * *reinterpret_cast<const f32x4_t *>(reinterpret_cast<const float *>(lds[v]) + r * kPitch + d);
        }
        if (sh.splits > 1) {
            const int64_t at = ((int64_t)tile * sh.splits + split) * kCol + r;
            store4(sh.out + at * DP + d, o[0], o[1], o[2], o[3]);
            if (d == 0)
                put8(sh.stat + 2 * at, u32x2{__float_as_uint(top2), __float_as_uint(z)});
        } else if (rt * kCol + r < rows) {
            const int tt = (rt * kCol + r) / G, hh = hk * G + (rt * kCol + r) % G;
            const float f = z == 0.f ? 0.f : 1.f / z;
            if (d < a.D)
                store4(static_cast<T *>(a.o.p) + b * a.o.sb + tt * a.o.st + hh * a.o.sh + d, o[0] * f,
                       o[1] * f, o[2] * f, o[3] * f);
            if (d == 0 && a.lse)
                a.lse[((int64_t)b * a.Hq + hh) * a.Tq + tt] =
                    z == 0.f ? -__builtin_inff() : (top2 + __builtin_amdgcn_logf(z)) * kLn2;
        }
    }
}

// Joins the splits' shares of a row: four entries a thread.
template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnProblem a, Shares sh)
{
    constexpr int kQuads = DP / 4;
    const int G = a.Hq / a.Hkv, rows = a.Tq * G, nt = (rows + kCol - 1) / kCol;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, all = (int64_t)a.B * a.Hkv * rows;
    const int64_t item = id / kQuads;
    const int d = (int)(id % kQuads) * 4;
    if (item >= all || d >= a.D)
        return;
    const int row = (int)(item % rows), hk = (int)(item / rows % a.Hkv), b = (int)(item / rows / a.Hkv);
    const int64_t at = (((int64_t)b * a.Hkv + hk) * nt + row / kCol) * sh.splits * kCol + row % kCol;
    // eight shares at a time, all in flight together
    constexpr int kAt = 8;
    float top2 = -__builtin_inff(), z = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < sh.splits; i0 += kAt) {
        float m[kAt], y[kAt];
        f32x4_t x[kAt];
#pragma unroll
        for (int i = 0; i < kAt; ++i) {
            const int64_t j = at + min(i0 + i, sh.splits - 1) * kCol;
            m[i] = i0 + i < sh.splits ? sh.stat[2 * j] : -__builtin_inff();
            y[i] = sh.stat[2 * j + 1];
            x[i] = *reinterpret_cast<const f32x4_t *>(sh.out + j * DP + d);
        }
        float mn = top2;
#pragma unroll
        for (int i = 0; i < kAt; ++i)
            mn = fmaxf(mn, m[i]);
        const float keep = top2 == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(top2 - mn);
        z *= keep;
        o *= keep;
#pragma unroll
        for (int i = 0; i < kAt; ++i) {
            const float f = m[i] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m[i] - mn);
            z = fmaf(f, y[i], z);
            o += f * x[i];
        }
        top2 = mn;
    }
    const int t = row / G, hq = hk * G + row % G;
    const float f = z == 0.f ? 0.f : 1.f / z;
    store4(static_cast<T *>(a.o.p) + b * a.o.sb + t * a.o.st + hq * a.o.sh + d, o[0] * f, o[1] * f,
           o[2] * f, o[3] * f);
    if (d == 0 && a.lse)
        a.lse[((int64_t)b * a.Hq + hq) * a.Tq + t] =
            z == 0.f ? -__builtin_inff() : (top2 + __builtin_amdgcn_logf(z)) * kLn2;
}

int64_t tiles_of(const AttnProblem &p)
{
    return (int64_t)p.B * p.Hkv * (((int64_t)p.Tq * (p.Hq / p.Hkv) + kCol - 1) / kCol);
}

// Keys that one tile's rows see at most.
int64_t keys_of(const AttnProblem &p)
{
    const int G = p.Hq / p.Hkv;
    const int64_t span = std::min<int64_t>(p.Tq, (kCol - 1) / G + 2);
    if (p.left < 0 || p.right < 0)
        return p.Tk;
    return std::min<int64_t>(p.Tk, (int64_t)p.left + p.right + span + p.sinks);
}

// Workgroups wanted at least (for 64 caches of up to 8192 tokens 2048 take 166 us, 1024
// 173), and blocks of keys that a wave of one has at least.
constexpr int kWanted = 2048, kLeast = 2;

template <typename T, int DP>
hipError_t run(const AttnProblem &p, hipStream_t s)
{
    const int64_t tiles = tiles_of(p), blocks = keys_of(p) / kBlock + 2;
    Shares sh{};
    sh.splits = (int)std::max<int64_t>(1, std::min((kWanted + tiles - 1) / tiles, blocks / (4 * kLeast)));
    if (sh.splits > 1) {
        void *out = nullptr, *stat = nullptr;
        hipError_t e = p.ws->take(&out, (size_t)tiles * sh.splits * kCol * DP * 4);
        if (e == hipSuccess)
            e = p.ws->take(&stat, (size_t)tiles * sh.splits * kCol * 2 * 4);
        if (e != hipSuccess)
            return e;
        sh.out = static_cast<float *>(out);
        sh.stat = static_cast<float *>(stat);
    }
    const int64_t n = tiles * sh.splits;
    if (n * kThreads > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (p.ws->counting)
        return hipSuccess;
    attn_split_kernel<T, DP><<<dim3((unsigned)n), kThreads, 0, s>>>(p, sh);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || sh.splits == 1)
        return e;
    const int64_t m = (int64_t)p.B * p.Tq * p.Hq * (DP / 4);
    attn_join_kernel<T, DP><<<dim3((unsigned)((m + kThreads - 1) / kThreads)), kThreads, 0, s>>>(p, sh);
    return hipGetLastError();
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

// Whether a forward is faster here.  The forward proper takes a query tile of 64 rows
// through its keys one tile after the other, 0.0119 us a key at heads of 64 and 0.0168
// at heads of 128, for some 512 of its workgroups at a time; this one has a launch more
// and takes about 2e-8 us a row, key and entry, whatever the rows' number.  Both, bf16
// (us; here and there): 64 queries of 8 heads of 64, 8192 keys 17 and 97, 512 keys 8.2
// and 10.2; 512 queries 49 and 97, 1024 queries 84 and 98; 16 x 32 queries, 1024 keys 19
// and 16; 16 heads of 128 on 4, 256 queries, 8192 keys 94 and 138, 512 queries 162 and 138.
// fp32 goes by the same figures, though its forward proper takes some 5 times as long a
// key: between the two lines it is up to 1.3 times slower than it could be (the same heads
// and keys, 512 queries 757 there, 622 here; 8 sequences of 64 queries 766 and 627).
bool attn_split_preferred(const AttnProblem &p)
{
    const double rows = (double)p.B * p.Hq * p.Tq, keys = (double)keys_of(p);
    const int64_t blocks = (int64_t)p.B * p.Hq * ((p.Tq + 63) / 64);
    const double forward = keys * (0.007 + 0.00008 * p.D) * (double)((blocks + 511) / 512);
    return rows * keys * p.D * 2.5e-8 + 6.0 < forward;
}

hipError_t launch_attn_split(const AttnProblem &p, hipStream_t s)
{
    return p.dtype == 0 ? run<float>(p, s) : run<bf16_t>(p, s);
}

}  // namespace gspn
