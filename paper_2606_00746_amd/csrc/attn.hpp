// Attention with a sliding window and sinks: the problem, and the tiles and
// matrix-core fragments that its kernels share (internal).
//
// Every product runs on 32 x 32 (decode: 16 x 16) matrix instructions in the
// orientation that leaves a softmax row in one lane: the scores are formed
// transposed, S^T = K Q^T, so that lane l of a wave holds query l % 32 and, in
// the registers r = 0..15 of a 32-key block, the keys 8 (r / 4) + 4 (l / 32) +
// r % 4.  The second product, O^T = V^T P^T, takes P^T as its B operand
// straight from those registers: a contraction may run over the keys in any
// order that both operands share, so V^T is read in the order that P^T has.
// bf16: V's tile lies in LDS as rows of keys, and ds_read_b64_tr_b16 turns four
// rows of 16 columns around on the way out.  fp32: one ds_read_b32 a step.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cdna.hpp"
#include "device.hpp"
#include "launch.hpp"

namespace gspn {

// A [B][T][H][D] tensor: base and strides of b, t, h in elements; D is contiguous.
struct Heads {
    void *p = nullptr;
    int64_t sb = 0, st = 0, sh = 0;
};

struct AttnProblem {
    Heads q, k, v, o, dout, dq, dk, dv;
    float *lse;              // [B][Hq][Tq]
    const int32_t *lens;     // [B], or null: Tk
    int B, Tq, Tk, Hq, Hkv, D;
    int left, right;         // < 0: no bound
    int sinks, offset;       // query t stands at position t + offset
    bool tail;               // query t stands at lens[b] - Tq + t instead
    float scale;
    int dtype;
    Workspace *ws;
};

hipError_t launch_attn_fwd(const AttnProblem &p, hipStream_t s);
hipError_t launch_attn_bwd(const AttnProblem &p, hipStream_t s);
hipError_t launch_attn_bwd_f32(const AttnProblem &p, hipStream_t s);
hipError_t launch_attn_split(const AttnProblem &p, hipStream_t s);
bool attn_split_preferred(const AttnProblem &p);

constexpr int kAttnMaxHead = 128;

// Tiles of 128 rows up to which pairs of waves share 32 rows: twice as many workgroups
// then, of half the rows.  Forward (us, with and without: 42 tiles 8.8 and 13.1, 224
// 14.3 and 17.9, 512 20.2 and 22.6, 768 30.4 and 28.3); gradients (both kernels: 42 tiles
// of heads of 72 21 and 29, 128 of 64 51 and 56, 160 49 and 50, of 128 94 and 80, 512 of
// 64 71 and 56).
constexpr int64_t kAttnFwdPairs = 512, kAttnBwdPairs = 128;
inline int64_t attn_tiles(const AttnProblem &p, int64_t H, int64_t T) { return p.B * H * ((T + 127) / 128); }
inline bool attn_fwd_pairs(const AttnProblem &p) { return attn_tiles(p, p.Hq, p.Tq) <= kAttnFwdPairs; }
inline bool attn_dq_pairs(const AttnProblem &p) { return attn_tiles(p, p.Hq, p.Tq) <= kAttnBwdPairs; }
inline bool attn_dkv_pairs(const AttnProblem &p) { return attn_tiles(p, p.Hkv, p.Tk) <= kAttnBwdPairs; }

// Gradients of bf16 rows with few keys, which take longer sums (attn_bwd.hpp): the
// sequences' buffer is short, or the window narrow.  What that costs, both kernels: 16 x 16
// heads of 64, causal, 512 tokens 170 us, 516 tokens (without) 110; heads of 128 381 and
// 203; 8 x 4096 tokens, 12 heads, a window of 33 253 us, of 34 184.
inline bool attn_few_keys(const AttnProblem &p)
{
    return p.Tk <= 512 || (p.left >= 0 && p.right >= 0 && (int64_t)p.left + p.right <= 32);
}

#ifdef __HIPCC__

namespace attn {

using namespace cdna;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kRows = 64;        // rows of a staged tile
constexpr int kThreads = 256;    // 4 waves

// v of this lane's row in both halves of the wave.
__device__ __forceinline__ float half_max(float v)
{
    const uint32_t b = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v)
{
    const uint32_t b = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 16-byte pieces of a tile of DP columns in LDS.  Rows are S pieces apart, a
// power of two, and piece c of row r lies at c ^ swizzle(r): 16 consecutive
// rows of one piece (a row-wise fragment) and 4 consecutive rows of four
// adjacent pieces (a turned-around one) then fall in different banks, both
// measured at the rate of linear addresses.
template <typename T, int DP>
struct Tile {
    static constexpr int kPer = 16 / (int)sizeof(T);     // elements of a piece
    static constexpr int kPieces = DP / kPer;
    static constexpr int kS = kPieces <= 4 ? 4 : kPieces <= 8 ? 8 : kPieces <= 16 ? 16 : 32;
    static constexpr int kRow = kS * 16;                 // bytes of a row
    static constexpr int kBytes = kRows * kRow;
    static constexpr int kLoads = kRows * kPieces / kThreads;
    static_assert(kRows * kPieces % kThreads == 0, "a tile is whole pieces per thread");

    __device__ static __forceinline__ int swizzle(int r)
    {
        if (kS == 4)
            return (r >> 2) & 3;
        if (kS == 8)
            return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
        return (r & 3) << 2 | ((r >> 2) & 3);
    }
    __device__ static __forceinline__ int at(int r, int c) { return (r * kS + (c ^ swizzle(r))) * 16; }

    uint4 reg[kLoads];
    // where the threads' pieces repeat every kStep rows, one offset and a uniform
    // step stand for all of a thread's
    static constexpr bool kEven = kThreads % kPieces == 0;
    static constexpr int kStep = kThreads / kPieces;
    uint32_t off[kEven ? 1 : kLoads];   // of this thread's pieces in a tile of the tensor

    // Before the first load: a tensor with row stride st, columns from D on read as zero.
    __device__ __forceinline__ void start(int64_t st, int D)
    {
#pragma unroll
        for (int i = 0; i < (kEven ? 1 : kLoads); ++i) {
            const int x = threadIdx.x + i * kThreads, r = x / kPieces, c = x % kPieces;
            off[i] = c * kPer < D ? (uint32_t)(r * (int)st * (int)sizeof(T) + c * 16) : 0x80000000u;
        }
    }
    // Rows row0 .. row0 + 63 into registers; rows from `rows` on read as zero, where
    // rows do not overlap (st >= D; else as parts of rows ahead of them).  The
    // buffer's range does both: a tile is below 2^31 bytes (token strides are below
    // 2^23), pieces that count as absent lie beyond.
    __device__ __forceinline__ void load(const T *base, int64_t st, int row0, int rows, int D)
    {
        const int n = min(rows - row0, kRows);
        const uint32_t bytes = n <= 0 ? 0u : (uint32_t)((n - 1) * (int)st + D) * (uint32_t)sizeof(T);
        const rsrc_t r = make_rsrc(base + (int64_t)row0 * st, bytes);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            reg[i] = kEven ? ld128(r, off[0], i * kStep * (int)st * (int)sizeof(T)) : ld128(r, off[i], 0);
    }
    // The same where a row that should read as zero counts, whatever its weight:
    // tokens that share memory (a stride below D, 0 for a view that broadcasts) leave
    // rows past the last inside the range.
    __device__ __forceinline__ void load_strict(const T *base, int64_t st, int row0, int rows, int D)
    {
        load(base, st, row0, rows, D);
        if (st < D)
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                if (row0 + (int)(threadIdx.x + i * kThreads) / kPieces >= rows)
                    reg[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void store(char *lds) const
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int x = threadIdx.x + i * kThreads, r = x / kPieces, c = x % kPieces;
            *reinterpret_cast<uint4 *>(lds + at(r, c)) = reg[i];
        }
    }
};

// The offset of an LDS address, as LDS instructions take it.
__device__ __forceinline__ uint32_t lds_offset(const void *p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)(p);
}

// bf16 tiles on their way from memory straight into LDS, through no registers, in
// Tile's order: a load writes 64 lanes' pieces one after the
// other, so a lane reads the piece that belongs at its place.  Rows past the last
// and columns past D read as the last: their products count for nothing (weights
// of 0, columns that are not stored), and what they read is finite.
template <int DP>
struct Flow {
    using X = Tile<bf16_t, DP>;
    static constexpr int kLoads = kRows * X::kS / kThreads;   // loads of a wave and tile
    static constexpr int kStep = kThreads / X::kS;            // rows between a thread's pieces
    int row, col;      // of this thread's first piece: row of the tile, byte in the row
    uint32_t off;
    int64_t st;
    __device__ __forceinline__ void start(int64_t stride, int D)
    {
        st = stride;
        row = threadIdx.x / X::kS;
        col = 16 * min((int)(threadIdx.x % X::kS) ^ X::swizzle(row), D / 8 - 1);
        off = (uint32_t)(row * (int)st * 2 + col);
    }
    // Rows row0 .. row0 + 63 (row0 < rows) to lds.
    __device__ __forceinline__ void load(char *lds, const bf16_t *base, int row0, int rows, int w) const
    {
        const rsrc_t r = make_rsrc(base + (int64_t)row0 * st, 0xffffffffu);
        const int n = rows - row0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            auto to = (__attribute__((address_space(3))) void *)(lds + i * (kThreads * 16) + w * 1024);
            if (n >= kRows)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 16, off, i * kStep * (int)st * 2, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 16, (uint32_t)(min(row + i * kStep, n - 1) * (int)st * 2 + col), 0, 0, 0);
        }
    }
};

// Waits for the wave's loads, then for the other waves'.
__device__ __forceinline__ void landed()
{
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// Reads of such tiles: the compiler would hold every LDS read until all of the
// loads into LDS have come, so these are its instructions by hand, each group with
// its wait, into registers of their own.
template <int N, int O>
__device__ __forceinline__ void lds_read4(const uint32_t (&a)[N], int at, u32x4 (&v)[N])
{
    asm volatile("ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\t"
                 "ds_read_b128 %2, %6 offset:%8\n\tds_read_b128 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(v[at]), "=&v"(v[at + 1]), "=&v"(v[at + 2]), "=&v"(v[at + 3])
                 : "v"(a[at]), "v"(a[at + 1]), "v"(a[at + 2]), "v"(a[at + 3]), "n"(O)
                 : "memory");
}
template <int N, int O>
__device__ __forceinline__ void lds_read2(const uint32_t (&a)[N], int at, u32x4 (&v)[N])
{
    asm volatile("ds_read_b128 %0, %2 offset:%4\n\tds_read_b128 %1, %3 offset:%4\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(v[at]), "=&v"(v[at + 1])
                 : "v"(a[at]), "v"(a[at + 1]), "n"(O)
                 : "memory");
}

// A row-wise fragment: 16 bytes of a row, the columns 2 s + l / 32 pieces in.
template <typename T>
struct Frag;
template <>
struct Frag<bf16_t> {
    bf16x8_t v;
};
template <>
struct Frag<float> {
    f32x4_t v;
};

template <typename T, int DP>
__device__ __forceinline__ Frag<T> tile_frag(const char *lds, int row, int piece)
{
    return *reinterpret_cast<const Frag<T> *>(lds + Tile<T, DP>::at(row, piece));
}

// The same from global memory (columns from D on as zero).
template <typename T>
__device__ __forceinline__ Frag<T> row_frag(const T *row, int piece, int D)
{
    constexpr int kPer = 16 / (int)sizeof(T);
    Frag<T> f;
    uint4 u = make_uint4(0, 0, 0, 0);
    if (piece * kPer < D)
        u = *reinterpret_cast<const uint4 *>(row + piece * kPer);
    f.v = __builtin_bit_cast(decltype(f.v), u);
    return f;
}

// The loads that filled these are waited for here, once, and not again where a
// loop that follows first uses them.
template <typename T, int N>
__device__ __forceinline__ void arrived(Frag<T> (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        asm volatile("" : "+v"(f[i].v));
}

// acc += A B^T over the columns of one pair of pieces (bf16: 16, fp32: 8).
__device__ __forceinline__ f32x16_t mma(Frag<bf16_t> a, Frag<bf16_t> b, f32x16_t acc)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mma(Frag<float> a, Frag<float> b, f32x16_t acc)
{
#pragma unroll
    for (int e = 0; e < 4; ++e)
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], acc, 0, 0, 0);
    return acc;
}

// The B operand of the second product, from the 16 registers of a 32 x 32
// block: bf16 rounds to nearest even (the products that follow take 8
// significant bits; sums of the unrounded values stay in fp32), fp32 takes
// them as they are.
template <typename T>
struct Probs;
template <>
struct Probs<bf16_t> {
    bf16x8_t v[2];
    __device__ __forceinline__ explicit Probs(const f32x16_t &p)
    {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint4 u = make_uint4(pack2(p[8 * t], p[8 * t + 1]), pack2(p[8 * t + 2], p[8 * t + 3]),
                                       pack2(p[8 * t + 4], p[8 * t + 5]), pack2(p[8 * t + 6], p[8 * t + 7]));
            v[t] = __builtin_bit_cast(bf16x8_t, u);
        }
    }
};
template <>
struct Probs<float> {
    f32x16_t v;
    __device__ __forceinline__ explicit Probs(const f32x16_t &p) : v(p) {}
};

__device__ __forceinline__ s16x4_t read_turned(const char *lds)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4_t *)(lds));
}

// The A operands of X^T P over the 32 rows row0.. of a tile X, read ahead of P.
template <typename T, int DP>
struct Turned;
template <int DP>
struct Turned<bf16_t, DP> {
    bf16x8_t v[2][DP / 32];
    __device__ __forceinline__ void load(const char *lds, int row0)
    {
        using X = Tile<bf16_t, DP>;
        const int l = threadIdx.x % 64, h = l / 32, i = l % 16, r = row0 + 4 * h + (i >> 2);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int db = 0; db < DP / 32; ++db) {
                const int c = 4 * db + 2 * (l % 32 / 16) + ((i & 3) >> 1), in = 8 * (i & 1);
                struct {
                    s16x4_t a, b;
                } both = {read_turned(lds + X::at(16 * t + r, c) + in), read_turned(lds + X::at(16 * t + 8 + r, c) + in)};
                v[t][db] = __builtin_bit_cast(bf16x8_t, both);
            }
    }
};
template <int DP>
struct Turned<float, DP> {   // read where they are used: 16 products take their time
    const char *lds;
    int row0;
    __device__ __forceinline__ void load(const char *tile, int row) { lds = tile, row0 = row; }
};

// acc[db] += X^T P (columns 32 db .. of X).
template <int DP>
__device__ __forceinline__ void mma_turned(const Turned<bf16_t, DP> &x, const Probs<bf16_t> &p, f32x16_t (&acc)[DP / 32])
{
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
            acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.v[t][db], p.v[t], acc[db], 0, 0, 0);
}
template <int DP>
__device__ __forceinline__ void mma_turned(const Turned<float, DP> &x, const Probs<float> &p, f32x16_t (&acc)[DP / 32])
{
    using X = Tile<float, DP>;
    const int l = threadIdx.x % 64, h = l / 32, d = l % 32;
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
            const float a = *reinterpret_cast<const float *>(
                x.lds + X::at(x.row0 + 8 * (r / 4) + 4 * h + r % 4, 8 * db + d / 4) + 4 * (d % 4));
            acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p.v[r], acc[db], 0, 0, 0);
        }
}

// This lane's row of a tile as row-wise fragments; bf16: all read at once.
template <typename T, int DP>
struct RowFrags;
template <int DP>
struct RowFrags<bf16_t, DP> {
    static constexpr int kSlices = Tile<bf16_t, DP>::kPieces / 2;
    Frag<bf16_t> f[kSlices];
    __device__ __forceinline__ void load(const char *lds, int row)
    {
        const int h = threadIdx.x % 64 / 32;
#pragma unroll
        for (int s = 0; s < kSlices; ++s)
            f[s] = tile_frag<bf16_t, DP>(lds, row, 2 * s + h);
    }
    __device__ __forceinline__ Frag<bf16_t> at(int s) const { return f[s]; }
};
template <int DP>
struct RowFrags<float, DP> {
    const char *lds;
    int row;
    __device__ __forceinline__ void load(const char *tile, int r) { lds = tile, row = r; }
    __device__ __forceinline__ Frag<float> at(int s) const
    {
        return tile_frag<float, DP>(lds, row, 2 * s + (int)(threadIdx.x % 64 / 32));
    }
};

// The same from tiles that flowed in: `tile` is their LDS offset.  The piece and
// the row lie in different bits of an address, so that pieces differ by exclusive
// ors and 32-row blocks by constants: tiles begin at multiples of a row's bytes
// (Tile::kRow), which the arrays they lie in are declared with.
template <int DP, int BLOCK>
__device__ __forceinline__ void flow_rows(uint32_t tile, Frag<bf16_t> (&f)[DP / 16])
{
    using X = Tile<bf16_t, DP>;
    const int c = threadIdx.x % 32, h = threadIdx.x % 64 / 32;
    const uint32_t a0 = tile + X::at(c, h);
    uint32_t a[DP / 16];
    u32x4 v[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
        a[s] = a0 ^ (32 * s);
    constexpr int kAt = BLOCK * 32 * X::kS * 16;
#pragma unroll
    for (int s = 0; s + 4 <= DP / 16; s += 4)
        lds_read4<DP / 16, kAt>(a, s, v);
    if constexpr (DP / 16 % 4 == 2)
        lds_read2<DP / 16, kAt>(a, DP / 16 - 2, v);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
        f[s].v = __builtin_bit_cast(bf16x8_t, v[s]);
}
template <int DP, int BLOCK>
__device__ __forceinline__ void flow_turned(uint32_t tile, Turned<bf16_t, DP> &x)
{
    using X = Tile<bf16_t, DP>;
    const int l = threadIdx.x % 64, h = l / 32, i = l % 16, r = 4 * h + (i >> 2);
    const uint32_t a0 = tile + X::at(r, 2 * (l % 32 / 16) + ((i & 3) >> 1)) + 8 * (i & 1);
    constexpr int kAt = BLOCK * 32 * X::kS * 16, kRow = X::kS * 16;
#pragma unroll
    for (int db = 0; db < DP / 32; ++db) {
        // rows 8 on: the other exclusive or
        const uint32_t a = a0 ^ (64 * db), b = a ^ 32;
        u32x2 v[4];
        asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %5 offset:%7\n\t"
                     "ds_read_b64_tr_b16 %2, %4 offset:%8\n\tds_read_b64_tr_b16 %3, %5 offset:%9\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
                     : "v"(a), "v"(b), "n"(kAt), "n"(kAt + 8 * kRow), "n"(kAt + 16 * kRow), "n"(kAt + 24 * kRow)
                     : "memory");
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const u32x4 w = {v[2 * t][0], v[2 * t][1], v[2 * t + 1][0], v[2 * t + 1][1]};
            x.v[t][db] = __builtin_bit_cast(bf16x8_t, w);
        }
    }
}

// The rows' statistics of a 32 x 32 block as its registers need them: rows 8 g +
// 4 (l / 32) .. of 64 values at `at`.
template <int BLOCK>
__device__ __forceinline__ void flow_stats(uint32_t at, f32x4_t (&v)[4])
{
    const uint32_t a = at + 16 * (threadIdx.x % 64 / 32);
    asm volatile("ds_read_b128 %0, %4 offset:%5\n\tds_read_b128 %1, %4 offset:%6\n\t"
                 "ds_read_b128 %2, %4 offset:%7\n\tds_read_b128 %3, %4 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
                 : "v"(a), "n"(128 * BLOCK), "n"(128 * BLOCK + 32), "n"(128 * BLOCK + 64), "n"(128 * BLOCK + 96)
                 : "memory");
}

// bf16: reads of LDS stay ahead of the products they are for, as written (the
// compiler otherwise puts each read next to its use and waits for it).
template <typename T>
__device__ __forceinline__ void reads_first()
{
    if (sizeof(T) == 2)
        step_fence();
}

// Stores a column (4 consecutive rows of a 32 x 32 result a register quad:
// entries d .. d + 3 of one token) scaled by f.
__device__ __forceinline__ void store4(bf16_t *p, float a, float b, float c, float d)
{
    put8(p, u32x2{pack2(a, b), pack2(c, d)});
}
__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d)
{
    put16(p, u32x4{__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d)});
}
template <typename T, int DP>
__device__ __forceinline__ void store_column(T *row, const f32x16_t (&acc)[DP / 32], float f, int D)
{
    const int h = threadIdx.x % 64 / 32;
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * db + 8 * g + 4 * h;
            if (d < D)
                store4(row + d, acc[db][4 * g] * f, acc[db][4 * g + 1] * f, acc[db][4 * g + 2] * f,
                       acc[db][4 * g + 3] * f);
        }
}

__device__ __forceinline__ int seq_len(const AttnProblem &p, int b)
{
    return p.lens ? min(max(p.lens[b], 0), p.Tk) : p.Tk;
}

// The keys that the query at position p sees: j <= hi, and j >= lo or j < sinks.
__device__ __forceinline__ void key_bounds(const AttnProblem &a, int len, int p, int &lo, int &hi)
{
    hi = p < 0 || p >= len ? -1 : a.right < 0 ? len - 1 : min(len - 1, p + a.right);
    lo = a.left < 0 ? 0 : max(0, p - a.left);
}

// Whether a query that sees lo .. hi, and sinks up to hi, sees key j; sunk: whether
// the tile of j holds sinks.
__device__ __forceinline__ bool sees(int j, int lo, int hi, int sinks, bool sunk)
{
    return sunk ? j <= hi && (j >= lo || j < sinks) : (uint32_t)(j - lo) <= (uint32_t)(hi - lo) && hi >= lo;
}

// The tiles of kRows keys that the queries t0 .. t0 + nt - 1 see: those that
// hold sinks ahead of the window, then the window's.
struct KeyTiles {
    int ns, first, n;
    __device__ __forceinline__ KeyTiles(const AttnProblem &a, int len, int t0, int nt)
    {
        const int p0 = t0 + a.offset, p1 = p0 + nt - 1;
        const int hi = p0 >= len ? -1 : a.right < 0 ? len - 1 : min(len - 1, p1 + a.right);
        const int lo = a.left < 0 ? 0 : max(0, p0 - a.left);
        ns = (min(a.sinks, lo) + kRows - 1) / kRows;
        first = max(ns, lo / kRows);
        n = hi < 0 ? 0 : ns + max(0, hi / kRows + 1 - first);
    }
    __device__ __forceinline__ int row(int it) const
    {
        return (it < ns ? it : first + it - ns) * kRows;
    }
};

// Whether some, or all, of the queries t0 .. t0 + nt - 1 see keys of the tile
// at k0 (all: every key of it).
struct KeyRange {
    int lo_some, hi_some, lo_all, hi_all, sinks;
    __device__ __forceinline__ KeyRange(const AttnProblem &a, int len, int t0, int nt)
    {
        const int p0 = t0 + a.offset, p1 = p0 + nt - 1;
        hi_some = p0 >= len ? -1 : a.right < 0 ? len - 1 : min(len - 1, p1 + a.right);
        hi_all = p1 >= len ? -1 : a.right < 0 ? len - 1 : min(len - 1, p0 + a.right);
        lo_some = a.left < 0 ? 0 : p0 - a.left;
        lo_all = a.left < 0 ? 0 : p1 - a.left;
        sinks = a.sinks;
    }
    __device__ __forceinline__ bool some(int k0) const
    {
        return k0 <= hi_some && (k0 + kRows > lo_some || k0 < sinks);
    }
    __device__ __forceinline__ bool all(int k0) const
    {
        return k0 + kRows - 1 <= hi_all && (k0 >= lo_all || k0 + kRows <= sinks);
    }
};

}  // namespace attn

#endif

}  // namespace gspn
