// The gated delta rule with bf16 storage (see delta.hpp for the formulas).
//
// Queries, keys, values and dO are bf16 and enter the products as they are.
// What is fp32 (states, inverses and everything on their way) enters as a sum
// of bf16 terms, each the rounding of what the ones before it leave: three hold
// 24 bits, two 16.  A product of two such sums takes the pairs of terms that
// matter (1 x 3: three, 3 x 3: six, 2 x 2: three), accumulated in fp32 by the
// matrix cores: 16 x 16 x 32 takes 16 cycles where the fp32 instructions take
// 256, so that six products are still 2.7 times as fast.  The way of the states
// has three terms and its results differ from fp32 products' in the last bits;
// what only goes into a bf16 output has two.
//
// The chunks of one head are a chain: X from S, U from X, S' from U.  A workgroup
// takes 16 columns of a state through it, each of its waves 32 rows of the state
// and a share of the tokens.  The rows of a 16 x 16 result stand for the indexes
//   32 g + 8 u + 4 blk + i    (register i of lane 16 u + c, blocks blk = 0, 1)
// so that a pair of blocks holds 8 consecutive indexes in a lane, which is the B
// operand of a product that contracts over them, and the 16-byte pieces of rows
// are its A operands.  The chain leaves its states and U behind as such operands,
// 1 KB a wave and term.
#include <algorithm>

#include "delta.hpp"

namespace gspn {
namespace {

using namespace delta;

template <int N>
struct Terms {
    bf16x8_t v[N];
};

// a, b (8 consecutive indexes) as N terms.
template <int N>
__device__ __forceinline__ Terms<N> split(f32x4_t a, f32x4_t b)
{
    Terms<N> t;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const uint4 w = make_uint4(pack2(a[0], a[1]), pack2(a[2], a[3]), pack2(b[0], b[1]), pack2(b[2], b[3]));
        t.v[n] = __builtin_bit_cast(bf16x8_t, w);
        if (n + 1 < N) {
            a -= f32x4_t{bf_lo(w.x), bf_hi(w.x), bf_lo(w.y), bf_hi(w.y)};
            b -= f32x4_t{bf_lo(w.z), bf_hi(w.z), bf_lo(w.w), bf_hi(w.w)};
        }
    }
    return t;
}

template <int NA, int NB>
__device__ __forceinline__ f32x4_t mma(const Terms<NA> &a, const Terms<NB> &b, f32x4_t c)
{
    constexpr int most = (NA > NB ? NA : NB) - 1;
#pragma unroll
    for (int s = most; s >= 0; --s)   // the small ones first
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB)
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[s - i], c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ Terms<1> one(uint4 v) { return Terms<1>{{__builtin_bit_cast(bf16x8_t, v)}}; }
__device__ __forceinline__ uint4 ld16(const void *p) { return *reinterpret_cast<const uint4 *>(p); }

// Operands left in memory: [unit][term][lane] of 16 bytes.
template <int N>
__device__ __forceinline__ Terms<N> load_terms(const uint4 *p, int64_t unit, int l)
{
    Terms<N> t;
#pragma unroll
    for (int n = 0; n < N; ++n)
        t.v[n] = __builtin_bit_cast(bf16x8_t, p[(unit * N + n) * 64 + l]);
    return t;
}
template <int N, int M>
__device__ __forceinline__ void store_terms(uint4 *p, int64_t unit, int l, const Terms<M> &t)
{
#pragma unroll
    for (int n = 0; n < N; ++n)
        put16(p + (unit * N + n) * 64 + l, __builtin_bit_cast(u32x4, t.v[n]));
}

constexpr int kGateRows = 6;   // beta, beta exp(G), exp(G_63 - G), exp(G), and G in its two floats
constexpr int kInvUnits = 6;   // 16-row blocks x 32-column groups on and below the diagonal
constexpr int kKeep = 2;       // terms of the states and U that are left behind

// Per (b, value head, chunk): gates [6][64]; the inverse and its transpose as A
// operands of three terms; U (units: slice of 16 columns x 2 groups of tokens)
// and the state ahead of the chunk (slice x groups of Dk) as operands of two.
struct Kept16 {
    float *gates = nullptr;
    uint4 *inv = nullptr, *turned = nullptr, *u = nullptr, *s = nullptr;
};

// Units of the inverse: block tb (rows 32 (tb / 2) ..) by group g of columns; its
// transpose has the groups on and above the diagonal.
__device__ __forceinline__ constexpr int inv_unit(int tb, int g) { return tb < 2 ? tb : 2 * tb - 2 + g; }
__device__ __forceinline__ constexpr int turned_unit(int tb, int g) { return tb < 2 ? 2 * tb + g : tb + 2; }

__device__ __forceinline__ int index_of(int tb, int m) { return 32 * (tb / 2) + 8 * (m / 4) + 4 * (tb & 1) + m % 4; }

// Gates, and (I + b M)^-1 by forward substitution, a wave a chunk, a lane a column.
// 8 x 4096 tokens of 12 heads of 64: 96 us, most of it the substitution's 64 dependent
// rows, broadcast from LDS.
template <int DKP>
__global__ __launch_bounds__(kThreads) void delta16_inverse_kernel(DeltaProblem p, Kept16 kept, int nc)
{
    __shared__ __attribute__((aligned(16))) float lds[4][kChunk * kPitch];
    const int w = threadIdx.x / 64, l = threadIdx.x % 64, c = l % 32, h = l / 32;
    const int64_t id = (int64_t)blockIdx.x * 4 + w;
    if (id >= (int64_t)p.B * p.Hv * nc)
        return;
    const int ch = (int)(id % nc), hv = (int)(id / nc % p.Hv), b = (int)(id / nc / p.Hv);
    const int t0 = ch * kChunk, n = max(0, min(kChunk, delta_len(p, b) - t0));
    const bf16_t *k = static_cast<const bf16_t *>(p.k.p) + b * p.k.sb + (hv / (p.Hv / p.Hq)) * p.k.sh + (int64_t)t0 * p.k.st;
    Gates x = load_gates(p, b, hv, t0, n, l);
    sum_gates(x, l);
    const float last = __shfl(x.G, kChunk - 1), rest = __shfl(x.D, kChunk - 1), eg = exp_f(x.G);
    float *gates = kept.gates + id * kGateRows * kChunk + l;
    gates[0] = x.beta;
    gates[kChunk] = x.beta * eg;
    gates[2 * kChunk] = decay(last, rest, x.G, x.D);
    gates[3 * kChunk] = eg;
    gates[4 * kChunk] = x.G;
    gates[5 * kChunk] = x.D;

    f32x16_t kk[3];
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            kk[i][r] = 0.f;
    Frag<bf16_t> ka[DKP / 16], kd[DKP / 16];
#pragma unroll
    for (int s = 0; s < DKP / 16; ++s) {
        ka[s] = kd[s] = Frag<bf16_t>{};
        if (c < n)
            ka[s] = row_frag(k + c * p.k.st, 2 * s + h, p.Dk);
        if (32 + c < n)
            kd[s] = row_frag(k + (32 + c) * p.k.st, 2 * s + h, p.Dk);
    }
#pragma unroll
    for (int s = 0; s < DKP / 16; ++s) {
        kk[0] = attn::mma(ka[s], ka[s], kk[0]);
        kk[1] = attn::mma(kd[s], ka[s], kk[1]);
        kk[2] = attn::mma(kd[s], kd[s], kk[2]);
    }
    float *m = lds[w];
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int t = (i ? 32 : 0) + 8 * (r / 4) + 4 * h + r % 4, s = (i == 2 ? 32 : 0) + c;
            const float gt = __shfl(x.G, t), bt = __shfl(x.beta, t), gs = __shfl(x.G, s);
            const float dt = __shfl(x.D, t), ds = __shfl(x.D, s);
            m[t * kPitch + s] = s < t ? bt * decay(gt, dt, gs, ds) * kk[i][r] : 0.f;
        }
    __builtin_amdgcn_wave_barrier();
    float col[kChunk];
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
        float a = i == l ? 1.f : 0.f;
#pragma unroll
        for (int s = 0; s < i; s += 4) {
            const f32x4_t v = load4(m + i * kPitch + s);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (s + e < i)
                    a = fmaf(-v[e], col[s + e], a);
        }
        col[i] = a;
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < kChunk; ++i)
        m[i * kPitch + l] = col[i];
    __builtin_amdgcn_wave_barrier();
    const int r16 = l % 16, u = l / 16;
#pragma unroll
    for (int tb = 0; tb < 4; ++tb)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int row = index_of(tb, r16), at = 32 * g + 8 * u;
            if (g <= tb / 2)
                store_terms<3>(kept.inv + id * (kInvUnits * 3 * 64), inv_unit(tb, g), l,
                               split<3>(load4(m + row * kPitch + at), load4(m + row * kPitch + at + 4)));
            if (kept.turned && g >= tb / 2) {
                f32x4_t a, d;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    a[e] = m[(at + e) * kPitch + row];
                    d[e] = m[(at + 4 + e) * kPitch + row];
                }
                store_terms<3>(kept.turned + id * (kInvUnits * 3 * 64), turned_unit(tb, g), l, split<3>(a, d));
            }
        }
}

// A chunk's 64 rows of 32 columns of K (or Q), a wave's share: as A operands of
// products over those columns, and in LDS, turned around, of products over the
// tokens.  Rows past the sequence's end read as its last: what they are multiplied
// with is 0.
struct KeyShare {
    using X = Tile<bf16_t, 32>;
    uint4 r[4];
    // base: the chunk's first row (uniform); st: row stride in elements; col: this
    // lane's first column (read only where `in`: r starts as zeros)
    __device__ __forceinline__ void load(const bf16_t *base, int64_t st, int n, int col, bool in, int l)
    {
        const int t0 = 8 * (l % 16 / 4) + l % 4;
        if (!in)
            return;
        if (n >= kChunk) {
            const uint32_t off = (uint32_t)(t0 * (int)st + col) * 2;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
                r[tb] = ld16(reinterpret_cast<const char *>(base + (32 * (tb / 2) + 4 * (tb & 1)) * st) + off);
        } else {
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
                r[tb] = ld16(base + min(32 * (tb / 2) + 4 * (tb & 1) + t0, n - 1) * st + col);
        }
    }
    __device__ __forceinline__ void store(char *lds, int l) const
    {
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
            *reinterpret_cast<uint4 *>(lds + X::at(index_of(tb, l % 16), l / 16)) = r[tb];
    }
    // block blk (of 16 of the 32 columns) of the transpose, tokens 32 g .. 32 g + 31
    __device__ static __forceinline__ Terms<1> turned(const char *lds, int blk, int g, int l)
    {
        const int i = l % 16, row = 32 * g + 8 * (l / 16) + (i >> 2);
        struct {
            s16x4_t a, b;
        } v = {read_turned(lds + X::at(row, i & 3) + 8 * blk), read_turned(lds + X::at(row + 4, i & 3) + 8 * blk)};
        return Terms<1>{{__builtin_bit_cast(bf16x8_t, v)}};
    }
};

// A chunk's results by blocks of 16 tokens, exchanged between the waves as B
// operands of three terms: [group of 32 tokens][term][lane] of 16 bytes, of which
// a block fills half.
struct Exchange {
    __attribute__((aligned(16))) char b[2 * 3 * 1024];
    __device__ __forceinline__ void put(int tb, int l, f32x4_t v)
    {
        const Terms<3> t = split<3>(v, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            const uint4 w = __builtin_bit_cast(uint4, t.v[n]);
            *reinterpret_cast<uint2 *>(b + ((tb / 2 * 3 + n) * 64 + l) * 16 + 8 * (tb & 1)) = make_uint2(w.x, w.y);
        }
    }
    __device__ __forceinline__ Terms<3> get(int g, int l) const
    {
        Terms<3> t;
#pragma unroll
        for (int n = 0; n < 3; ++n)
            t.v[n] = __builtin_bit_cast(bf16x8_t, ld16(b + ((g * 3 + n) * 64 + l) * 16));
        return t;
    }
};
// The half of an operand of two terms that a block of tokens fills, to memory.
__device__ __forceinline__ void store_half(uint4 *p, int64_t unit, int tb, int l, f32x4_t v)
{
    const Terms<kKeep> t = split<kKeep>(v, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int n = 0; n < kKeep; ++n) {
        const uint4 w = __builtin_bit_cast(uint4, t.v[n]);
        put8(reinterpret_cast<uint2 *>(p + (unit * kKeep + n) * 64 + l) + (tb & 1), u32x2{w.x, w.y});
    }
}

// This lane's column of four consecutive tokens 8 u + t .. of a chunk (t uniform);
// tokens past the sequence's end read as its last.
__device__ __forceinline__ void load_column(uint32_t (&r)[4], const bf16_t *base, int64_t st, int t, int n, int col,
                                            bool in, int u)
{
    if (!in)
        return;
    if (n >= kChunk) {
        const uint32_t off = (uint32_t)(8 * u * (int)st + col) * 2;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[i] = *reinterpret_cast<const bf16_t *>(reinterpret_cast<const char *>(base + (t + i) * st) + off);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[i] = base[(int64_t)min(8 * u + t + i, n - 1) * st + col];
    }
}

// The chain's own tokens: the blocks that wave w of NW takes through the inverse,
// paired so that the triangle's work is even.
template <int NW>
__device__ __forceinline__ int own_block(int w, int j)
{
    return j == 0 ? w : 3 - w;
}

// U and the states of 16 columns, all chunks in turn.  Wave w holds the rows
// 32 w .. 32 w + 31 of the state, forms their share of K S, and takes the
// blocks own_block of the tokens through X and U: the three exchanges are the
// chain's length, its work is shared.  64 chunks of heads of 64 (8 x 12 of them) in 195
// us, 128 chunks of heads of 128 (2 x 16) in 265: 2 to 3 us a chunk, of which loads that
// all hit would leave 2; 16 columns a workgroup give the card 384 and 256 of them.
template <int DKP>
__global__ __launch_bounds__(DKP * 2) void delta16_state_kernel(DeltaProblem p, Kept16 kept, int nc, int nv)
{
    constexpr int NW = DKP / 32, NT = 4 / NW;
    __shared__ __attribute__((aligned(16))) char kl[NW][KeyShare::X::kBytes];
    __shared__ __attribute__((aligned(16))) f32x4_t part[NW][4][64];
    __shared__ Exchange xl, ul;
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int sl = id % nv;
    id /= nv;
    const int hv = id % p.Hv, b = id / p.Hv;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int col = 16 * sl + c, len = delta_len(p, b), live = (len + kChunk - 1) / kChunk;
    const bf16_t *k = static_cast<const bf16_t *>(p.k.p) + b * p.k.sb + (hv / (p.Hv / p.Hq)) * p.k.sh;
    const bf16_t *v = static_cast<const bf16_t *>(p.v.p) + b * p.v.sb + hv * p.v.sh;
    const bool in = col < p.Dv, kin = 32 * w + 8 * u < p.Dk;
    const int64_t head = (int64_t)b * p.Hv + hv;

    f32x4_t S[2];
#pragma unroll
    for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 32 * w + 8 * u + 4 * blk + i;
            S[blk][i] = p.state && r < p.Dk && in ? p.state[(head * p.Dk + r) * p.Dv + col] : 0.f;
        }

    // what a chunk reads beside the state: loaded a chunk ahead of its use
    struct Ahead {
        KeyShare kr;
        Terms<3> inv[NT][2];
        uint32_t vr[NT][4];
        f32x4_t gb[NT], ge[NT], gl[NT];
        float gk;
    } even{}, odd{};
    int lane0 = 0;   // 0, but not to the compiler: a scalar load would be waited for with LDS
    asm("" : "+v"(lane0));
    const auto fetch = [&](int ch, Ahead &x) {
        const int n = len - ch * kChunk;
        const float *g = kept.gates + (head * nc + ch) * kGateRows * kChunk;
        const uint4 *m = kept.inv + (head * nc + ch) * (kInvUnits * 3 * 64);
        x.kr.load(k + (int64_t)ch * kChunk * p.k.st, p.k.st, n, 32 * w + 8 * u, kin, l);
        x.gk = g[4 * kChunk - 1 + lane0];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tb = own_block<NW>(w, j), t = 32 * (tb / 2) + 4 * (tb & 1);
            load_column(x.vr[j], v + (int64_t)ch * kChunk * p.v.st, p.v.st, t, n, col, in, u);
            x.gb[j] = load4(g + t + 8 * u);
            x.ge[j] = load4(g + kChunk + t + 8 * u);
            x.gl[j] = load4(g + 2 * kChunk + t + 8 * u);
            x.inv[j][0] = load_terms<3>(m, inv_unit(tb, 0), l);
            if (tb >= 2)
                x.inv[j][1] = load_terms<3>(m, inv_unit(tb, 1), l);
        }
    };
    const auto chunk = [&](int ch, Ahead &now, Ahead &next) {
        const int64_t at = head * nc + ch;
        if (ch + 1 < live)
            fetch(ch + 1, next);
        now.kr.store(kl[w], l);
        {
            const Terms<3> s = split<3>(S[0], S[1]);
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
                part[w][tb][l] = mma(one(now.kr.r[tb]), s, f32x4_t{0.f, 0.f, 0.f, 0.f});
            store_terms<kKeep>(kept.s, (at * nv + sl) * NW + w, l, s);
        }
        lds_barrier();
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tb = own_block<NW>(w, j);
            f32x4_t x = part[0][tb][l];
#pragma unroll
            for (int n = 1; n < NW; ++n)
                x += part[n][tb][l];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = now.gb[j][i] * bf_lo(now.vr[j][i]) - now.ge[j][i] * x[i];
            xl.put(tb, l, x);
        }
        lds_barrier();
        f32x4_t y[NT];
        const Terms<3> x0 = xl.get(0, l), x1 = xl.get(1, l);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tb = own_block<NW>(w, j);
            y[j] = mma(now.inv[j][0], x0, f32x4_t{0.f, 0.f, 0.f, 0.f});
            if (tb >= 2)
                y[j] = mma(now.inv[j][1], x1, y[j]);
            ul.put(tb, l, now.gl[j] * y[j]);
        }
        lds_barrier();
        const Terms<3> u0 = ul.get(0, l), u1 = ul.get(1, l);
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            S[blk] *= now.gk;
            S[blk] = mma(KeyShare::turned(kl[w], blk, 0, l), u0, S[blk]);
            S[blk] = mma(KeyShare::turned(kl[w], blk, 1, l), u1, S[blk]);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tb = own_block<NW>(w, j);
            store_half(kept.u, (at * nv + sl) * 2 + tb / 2, tb, l, y[j]);
        }
        __builtin_amdgcn_wave_barrier();
    };
    if (live > 0)
        fetch(0, even);
    for (int ch = 0; ch < live; ch += 2) {
        chunk(ch, even, odd);
        if (ch + 1 < live)
            chunk(ch + 1, odd, even);
    }
    if (p.state_out && in)
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 32 * w + 8 * u + 4 * blk + i;
                if (r < p.Dk)
                    p.state_out[(head * p.Dk + r) * p.Dv + col] = S[blk][i];
            }
}

// A row's 16-byte piece of a [T][D] matrix in chunk order (rows past n and
// columns past D as zero).
__device__ __forceinline__ uint4 piece_of(const bf16_t *m, int64_t st, int t, int n, int e, int D)
{
    uint4 v = make_uint4(0, 0, 0, 0);
    if (t < n && e < D)
        v = ld16(m + t * st + e);
    return v;
}

using Square16 = Tile<bf16_t, kChunk>;   // a 64 x 64 matrix of bf16 in LDS

// Four consecutive columns of row r, N terms, each a matrix of its own.
template <int N>
__device__ __forceinline__ void put4(char *lds, int r, int col, f32x4_t v)
{
    const Terms<N> t = split<N>(v, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const uint4 w = __builtin_bit_cast(uint4, t.v[n]);
        *reinterpret_cast<uint2 *>(lds + n * Square16::kBytes + Square16::at(r, col / 8) + 2 * (col % 8)) = make_uint2(w.x, w.y);
    }
}
template <int N>
__device__ __forceinline__ Terms<N> row_terms(const char *lds, int row, int piece)
{
    Terms<N> t;
#pragma unroll
    for (int n = 0; n < N; ++n)
        t.v[n] = __builtin_bit_cast(bf16x8_t, ld16(lds + n * Square16::kBytes + Square16::at(row, piece)));
    return t;
}

// O of a chunk, transposed: a lane holds four columns of one token.  8 x 4096 tokens
// of 12 heads of 64: 112 us, 341 MB moved; forming Q K^T and its decays for a chunk's
// four waves bounds it, not memory.
template <int DKP>
__global__ __launch_bounds__(kThreads) void delta16_out_kernel(DeltaProblem p, Kept16 kept, int nc, int nv)
{
    constexpr int NG = DKP / 32;
    __shared__ __attribute__((aligned(16))) char pl[2 * Square16::kBytes];
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int ch = id % nc;
    id /= nc;
    const int hv = id % p.Hv, b = id / p.Hv;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int t0 = ch * kChunk, n = max(0, min(kChunk, delta_len(p, b) - t0)), hq = hv / (p.Hv / p.Hq);
    const bf16_t *q = static_cast<const bf16_t *>(p.q.p) + b * p.q.sb + hq * p.q.sh + (int64_t)t0 * p.q.st;
    const bf16_t *k = static_cast<const bf16_t *>(p.k.p) + b * p.k.sb + hq * p.k.sh + (int64_t)t0 * p.k.st;
    bf16_t *o = static_cast<bf16_t *>(p.o.p) + b * p.o.sb + hv * p.o.sh + (int64_t)t0 * p.o.st;
    const int64_t at = ((int64_t)b * p.Hv + hv) * nc + ch;
    const float *gates = kept.gates + at * kGateRows * kChunk;

    if (n == 0) {   // past the sequence's end: nothing was left for it
        for (int x = threadIdx.x; x < kChunk * p.Dv / 4; x += kThreads) {
            const int t = x / (p.Dv / 4), d = x % (p.Dv / 4) * 4;
            if (t0 + t < p.T)
                store4(o + t * p.o.st + d, 0.f, 0.f, 0.f, 0.f);
        }
        return;
    }
    uint4 qr[4][NG];
#pragma unroll
    for (int tb = 0; tb < 4; ++tb)
#pragma unroll
        for (int g = 0; g < NG; ++g)
            qr[tb][g] = piece_of(q, p.q.st, 16 * tb + c, n, 32 * g + 8 * u, p.Dk);
    // the wave's first slice of the state and U is in flight while P is formed
    Terms<kKeep> sf[NG], uf[2];
    const auto fetch = [&](int sl) {
#pragma unroll
        for (int g = 0; g < NG; ++g)
            sf[g] = load_terms<kKeep>(kept.s, (at * nv + sl) * NG + g, l);
#pragma unroll
        for (int g = 0; g < 2; ++g)
            uf[g] = load_terms<kKeep>(kept.u, (at * nv + sl) * 2 + g, l);
    };
    if (w < nv)
        fetch(w);
    {   // P[t][s] for the 16 tokens t of block w
        const float gt = gates[4 * kChunk + 16 * w + c], gd = gates[5 * kChunk + 16 * w + c];
        uint4 mine[NG], kr[4][NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            mine[g] = piece_of(q, p.q.st, 16 * w + c, n, 32 * g + 8 * u, p.Dk);
#pragma unroll
            for (int sb = 0; sb < 4; ++sb)
                if (sb <= w)
                    kr[sb][g] = piece_of(k, p.k.st, 16 * sb + c, n, 32 * g + 8 * u, p.Dk);
        }
#pragma unroll
        for (int sb = 0; sb < 4; ++sb)
            if (sb <= (w | 1)) {
                f32x4_t a = {0.f, 0.f, 0.f, 0.f};
                if (sb <= w) {
#pragma unroll
                    for (int g = 0; g < NG; ++g)
                        a = mma(one(kr[sb][g]), one(mine[g]), a);
                    const f32x4_t gs = load4(gates + 4 * kChunk + 16 * sb + 4 * u);
                    const f32x4_t ds = load4(gates + 5 * kChunk + 16 * sb + 4 * u);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        a[i] = 16 * sb + 4 * u + i <= 16 * w + c ? p.scale * decay(gt, gd, gs[i], ds[i]) * a[i] : 0.f;
                }
                put4<2>(pl, 16 * w + c, 16 * sb + 4 * u, a);
            }
    }
    lds_barrier();
    for (int sl = w; sl < nv; sl += 4) {
        f32x4_t acc[4];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
            acc[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        const Terms<kKeep> u0 = uf[0], u1 = uf[1];
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
                acc[tb] = mma(sf[g], one(qr[tb][g]), acc[tb]);
        if (sl + 4 < nv)
            fetch(sl + 4);
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
            acc[tb] *= p.scale * gates[3 * kChunk + 16 * tb + c];
            acc[tb] = mma(u0, row_terms<2>(pl, 16 * tb + c, u), acc[tb]);
            if (tb >= 2)
                acc[tb] = mma(u1, row_terms<2>(pl, 16 * tb + c, 4 + u), acc[tb]);
            const int t = 16 * tb + c, d = 16 * sl + 4 * u;
            const float f = t < n ? 1.f : 0.f;
            if (d < p.Dv && t0 + t < p.T)
                store4(o + t * p.o.st + d, acc[tb][0] * f, acc[tb][1] * f, acc[tb][2] * f, acc[tb][3] * f);
        }
    }
}

// What the backward adds, per (b, value head, chunk): scale A^T dO as results
// (slice x block of 16 tokens, fp32), R and the gradient of the state behind the
// chunk as operands of two terms, laid out as U and the states.
struct Grads16 {
    float *du = nullptr;
    uint4 *r = nullptr, *ds = nullptr;
};

// scale A^T dO of a chunk (8 x 4096 tokens of 12 heads of 64: 63 us).
template <int DKP, int DVP>
__global__ __launch_bounds__(kThreads) void delta16_du_kernel(DeltaProblem p, Kept16 kept, Grads16 gr, int nc, int nv)
{
    using X = Tile<bf16_t, DVP>;
    __shared__ __attribute__((aligned(16))) char pl[3 * Square16::kBytes], dl[X::kBytes];
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int ch = id % nc;
    id /= nc;
    const int hv = id % p.Hv, b = id / p.Hv;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int t0 = ch * kChunk, n = max(0, min(kChunk, delta_len(p, b) - t0)), hq = hv / (p.Hv / p.Hq);
    const bf16_t *q = static_cast<const bf16_t *>(p.q.p) + b * p.q.sb + hq * p.q.sh + (int64_t)t0 * p.q.st;
    const bf16_t *k = static_cast<const bf16_t *>(p.k.p) + b * p.k.sb + hq * p.k.sh + (int64_t)t0 * p.k.st;
    const bf16_t *d = static_cast<const bf16_t *>(p.dout.p) + b * p.dout.sb + hv * p.dout.sh + (int64_t)t0 * p.dout.st;
    const int64_t at = ((int64_t)b * p.Hv + hv) * nc + ch;
    const float *gates = kept.gates + at * kGateRows * kChunk;

    if (n == 0)
        return;
    X x;
    x.start(p.dout.st, p.Dv);
    x.load_strict(d, p.dout.st, 0, n, p.Dv);
    {   // P[t][s] as rows of s, for the 16 columns s of block w
        const float gs = gates[4 * kChunk + 16 * w + c], ds = gates[5 * kChunk + 16 * w + c];
        f32x4_t a[4];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
            a[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        uint4 kf[DKP / 32], qf[4][DKP / 32];
#pragma unroll
        for (int g = 0; g < DKP / 32; ++g) {
            kf[g] = piece_of(k, p.k.st, 16 * w + c, n, 32 * g + 8 * u, p.Dk);
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
                if (tb >= w)
                    qf[tb][g] = piece_of(q, p.q.st, 16 * tb + c, n, 32 * g + 8 * u, p.Dk);
        }
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
            if (tb >= w)
#pragma unroll
                for (int g = 0; g < DKP / 32; ++g)
                    a[tb] = mma(one(qf[tb][g]), one(kf[g]), a[tb]);
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
            if (tb >= (w & 2)) {
                const f32x4_t gt = load4(gates + 4 * kChunk + 16 * tb + 4 * u);
                const f32x4_t dt = load4(gates + 5 * kChunk + 16 * tb + 4 * u);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    a[tb][i] = 16 * w + c <= 16 * tb + 4 * u + i ? p.scale * decay(gt[i], dt[i], gs, ds) * a[tb][i] : 0.f;
                put4<3>(pl, 16 * w + c, 16 * tb + 4 * u, a[tb]);
            }
    }
    x.store(dl);
    lds_barrier();
    const int i16 = l % 16;
    for (int sl = w; sl < nv; sl += 4) {
        Terms<1> df[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int row = 32 * g + 8 * u + (i16 >> 2), piece = 2 * sl + ((i16 & 3) >> 1), in = 8 * (i16 & 1);
            struct {
                s16x4_t a, b;
            } v = {read_turned(dl + X::at(row, piece) + in), read_turned(dl + X::at(row + 4, piece) + in)};
            df[g].v[0] = __builtin_bit_cast(bf16x8_t, v);
        }
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
            f32x4_t a = {0.f, 0.f, 0.f, 0.f};
            if (tb < 2)
                a = mma(row_terms<3>(pl, index_of(tb, c), u), df[0], a);
            a = mma(row_terms<3>(pl, index_of(tb, c), 4 + u), df[1], a);
            store4(gr.du + (((at * nv + sl) * 4 + tb) * 64 + l) * 4, a[0], a[1], a[2], a[3]);
        }
    }
}

// R, dV and the gradients of the states of 16 columns, the chunks from the last
// on; shared among the waves like delta16_state_kernel (8 x 4096 tokens of 12 heads of
// 64: 263 us, 4 us a chunk: it has dO's share of the state's gradient beside).
template <int DKP>
__global__ __launch_bounds__(DKP * 2) void delta16_dstate_kernel(DeltaProblem p, Kept16 kept, Grads16 gr, int nc, int nv)
{
    constexpr int NW = DKP / 32, NT = 4 / NW;
    __shared__ __attribute__((aligned(16))) char kl[NW][KeyShare::X::kBytes], ql[NW][KeyShare::X::kBytes];
    __shared__ __attribute__((aligned(16))) f32x4_t part[NW][4][64];
    __shared__ Exchange xl, zl, yl;
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int sl = id % nv;
    id /= nv;
    const int hv = id % p.Hv, b = id / p.Hv, hq = hv / (p.Hv / p.Hq);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int col = 16 * sl + c, len = delta_len(p, b), live = (len + kChunk - 1) / kChunk;
    const bf16_t *q = static_cast<const bf16_t *>(p.q.p) + b * p.q.sb + hq * p.q.sh;
    const bf16_t *k = static_cast<const bf16_t *>(p.k.p) + b * p.k.sb + hq * p.k.sh;
    const bf16_t *d = static_cast<const bf16_t *>(p.dout.p) + b * p.dout.sb + hv * p.dout.sh;
    bf16_t *dv = static_cast<bf16_t *>(p.dv.p) + b * p.dv.sb + hv * p.dv.sh + col;
    const bool in = col < p.Dv, kin = 32 * w + 8 * u < p.Dk;
    const int64_t head = (int64_t)b * p.Hv + hv;

    f32x4_t S[2];
#pragma unroll
    for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 32 * w + 8 * u + 4 * blk + i;
            S[blk][i] = p.dstate && r < p.Dk && in ? p.dstate[(head * p.Dk + r) * p.Dv + col] : 0.f;
        }

    struct Ahead {   // as in delta16_state_kernel
        KeyShare kr, qr;
        Terms<3> inv[NT][2];
        uint32_t dr[NT][4];
        f32x4_t gb[NT], ge[NT], gl[NT], gq[NT], du[NT];
        float gk;
    } even{}, odd{};
    int lane0 = 0;
    asm("" : "+v"(lane0));
    const auto fetch = [&](int ch, Ahead &x) {
        const int64_t at = head * nc + ch;
        const int n = len - ch * kChunk;
        const float *g = kept.gates + at * kGateRows * kChunk;
        const uint4 *m = kept.turned + at * (kInvUnits * 3 * 64);
        x.kr.load(k + (int64_t)ch * kChunk * p.k.st, p.k.st, n, 32 * w + 8 * u, kin, l);
        x.qr.load(q + (int64_t)ch * kChunk * p.q.st, p.q.st, n, 32 * w + 8 * u, kin, l);
        x.gk = g[4 * kChunk - 1 + lane0];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tb = own_block<NW>(w, j), t = 32 * (tb / 2) + 4 * (tb & 1);
            load_column(x.dr[j], d + (int64_t)ch * kChunk * p.dout.st, p.dout.st, t, n, col, in, u);
            x.gb[j] = load4(g + t + 8 * u);
            x.ge[j] = load4(g + kChunk + t + 8 * u);
            x.gl[j] = load4(g + 2 * kChunk + t + 8 * u);
            x.gq[j] = load4(g + 3 * kChunk + t + 8 * u);
            x.du[j] = load4(gr.du + (((at * nv + sl) * 4 + tb) * 64 + l) * 4);
            if (tb < 2)
                x.inv[j][0] = load_terms<3>(m, turned_unit(tb, 0), l);
            x.inv[j][1] = load_terms<3>(m, turned_unit(tb, 1), l);
        }
    };
    const auto chunk = [&](int ch, Ahead &now, Ahead &next) {
        const int64_t at = head * nc + ch;
        const int n = len - ch * kChunk;
        if (ch > 0)
            fetch(ch - 1, next);
        now.kr.store(kl[w], l);
        now.qr.store(ql[w], l);
        {
            const Terms<3> s = split<3>(S[0], S[1]);
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
                part[w][tb][l] = mma(one(now.kr.r[tb]), s, f32x4_t{0.f, 0.f, 0.f, 0.f});
            store_terms<kKeep>(gr.ds, (at * nv + sl) * NW + w, l, s);
        }
        // dO's share of the states' gradient needs nothing from the chain
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tb = own_block<NW>(w, j), t = 32 * (tb / 2) + 8 * u + 4 * (tb & 1);
            f32x4_t y;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                y[i] = t + i < n ? p.scale * now.gq[j][i] * bf_lo(now.dr[j][i]) : 0.f;
            yl.put(tb, l, y);
        }
        lds_barrier();
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tb = own_block<NW>(w, j), t = 32 * (tb / 2) + 8 * u + 4 * (tb & 1);
            f32x4_t x = part[0][tb][l];
#pragma unroll
            for (int m = 1; m < NW; ++m)
                x += part[m][tb][l];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = t + i < n ? now.du[j][i] + now.gl[j][i] * x[i] : 0.f;
            xl.put(tb, l, x);
        }
        lds_barrier();
        f32x4_t r[NT];
        const Terms<3> x0 = xl.get(0, l), x1 = xl.get(1, l);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tb = own_block<NW>(w, j);
            r[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (tb < 2)
                r[j] = mma(now.inv[j][0], x0, r[j]);
            r[j] = mma(now.inv[j][1], x1, r[j]);
            zl.put(tb, l, -(now.ge[j] * r[j]));
        }
        lds_barrier();
        const Terms<3> z0 = zl.get(0, l), z1 = zl.get(1, l), y0 = yl.get(0, l), y1 = yl.get(1, l);
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            S[blk] *= now.gk;
            S[blk] = mma(KeyShare::turned(ql[w], blk, 0, l), y0, S[blk]);
            S[blk] = mma(KeyShare::turned(ql[w], blk, 1, l), y1, S[blk]);
            S[blk] = mma(KeyShare::turned(kl[w], blk, 0, l), z0, S[blk]);
            S[blk] = mma(KeyShare::turned(kl[w], blk, 1, l), z1, S[blk]);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int tb = own_block<NW>(w, j), t = 32 * (tb / 2) + 8 * u + 4 * (tb & 1);
            store_half(gr.r, (at * nv + sl) * 2 + tb / 2, tb, l, r[j]);
            if (in)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t + i < n)
                        store_f(dv + (int64_t)(ch * kChunk + t + i) * p.dv.st, now.gb[j][i] * r[j][i]);
        }
        lds_barrier();   // yl is written ahead of the next chunk's first exchange
    };
    if (live > 0)
        fetch(live - 1, even);
    for (int ch = live - 1; ch >= 0; ch -= 2) {
        chunk(ch, even, odd);
        if (ch > 0)
            chunk(ch - 1, odd, even);
    }
    if (p.dstate_in && in)
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rr = 32 * w + 8 * u + 4 * blk + i;
                if (rr < p.Dk)
                    p.dstate_in[(head * p.Dk + rr) * p.Dv + col] = S[blk][i];
            }
    // tokens that no chunk above has
    for (int64_t t = len + threadIdx.x / 16; t < p.T; t += DKP * 2 / 16)
        if (in)
            store_f(dv + t * p.dv.st, 0.f);
}

__device__ __forceinline__ float over_c(float v)   // over the 16 lanes of one u
{
    const auto dpp = [](float x, auto ctrl) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    v += dpp(v, std::integral_constant<int, 0xB1>{});
    v += dpp(v, std::integral_constant<int, 0x4E>{});
    v += dpp(v, std::integral_constant<int, 0x141>{});
    return v + dpp(v, std::integral_constant<int, 0x140>{});
}
__device__ __forceinline__ float over_u(float v)   // over the four u of one lane
{
    v = half_sum(v);
    const uint32_t b = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Operands that were left as [unit of 16 columns][32 rows in pieces of 8] on
// their way into LDS as rows of 64 entries, one row a column: piece 4 g + u of
// row 16 sl + c.  A 16-byte piece a thread and step; columns that no slice has
// are zero.
template <int DVP>
struct Unpacked {
    uint4 r[DVP / 16];
    __device__ __forceinline__ void load(const uint4 *units, int64_t first, int stride, int g0, int nv)
    {
#pragma unroll
        for (int i = 0; i < DVP / 16; ++i) {
            const int l = threadIdx.x % 64, n = threadIdx.x / 64 % kKeep, g = threadIdx.x / 128;
            r[i] = make_uint4(0, 0, 0, 0);
            if (i < nv)
                r[i] = units[((first + (int64_t)i * stride + g0 + g) * kKeep + n) * 64 + l];
        }
    }
    __device__ __forceinline__ void store(char *lds) const
    {
        const int l = threadIdx.x % 64, n = threadIdx.x / 64 % kKeep, g = threadIdx.x / 128;
#pragma unroll
        for (int i = 0; i < DVP / 16; ++i)
            *reinterpret_cast<uint4 *>(lds + n * DVP * 128 + Square16::at(16 * i + l % 16, 4 * g + l / 16)) = r[i];
    }
};
// A or B operand from such rows: entries 16 blk + c (of 64), rows 32 g + 8 u ..
__device__ __forceinline__ Terms<kKeep> turned_terms(const char *lds, int blk, int g, int l, int rows)
{
    const int i = l % 16, row = 32 * g + 8 * (l / 16) + (i >> 2), piece = 2 * blk + ((i & 3) >> 1), in = 8 * (i & 1);
    Terms<kKeep> t;
#pragma unroll
    for (int n = 0; n < kKeep; ++n) {
        struct {
            s16x4_t a, b;
        } v = {read_turned(lds + n * rows * 128 + Square16::at(row, piece) + in),
               read_turned(lds + n * rows * 128 + Square16::at(row + 4, piece) + in)};
        t.v[n] = __builtin_bit_cast(bf16x8_t, v);
    }
    return t;
}

// dQ, dK, dg and dbeta of a chunk, with the value heads that share its queries
// and keys in turn.  Wave w holds the rows 64 j + 16 w .. of dQ^T and dK^T.  8 x 4096
// tokens of 12 heads of 64: 286 us, two workgroups a CU (with dO in registers instead of
// LDS and the loads where they are used 12% longer); waits 68% of its time, on LDS reads of
// operands in two terms and the barriers between its phases.
template <int DKP, int DVP>
__global__ __launch_bounds__(kThreads, (DKP + DVP <= 128 ? 2 : 1))
void delta16_grad_kernel(DeltaProblem p, Kept16 kept, Grads16 gr, int nc, int nv)
{
    constexpr int NB = DKP / 64, NG = DKP / 32, NE = DVP / 32;
    using X = Tile<bf16_t, DKP>;
    using E = Tile<bf16_t, DVP>;
    constexpr int kMat = DVP * 128;                        // one term of [DVP][64]
    constexpr int kPN = 2 * kKeep * Square16::kBytes;      // P and N lie over U and R
    constexpr int kUR = 2 * kKeep * kMat > kPN ? 2 * kKeep * kMat : kPN;
    __shared__ __attribute__((aligned(16))) char ur[kUR], sd[kKeep * kMat], kl[X::kBytes], ql[X::kBytes], dl[E::kBytes];
    __shared__ float sums[4][4][kChunk], ss[4];
    char *ul = ur, *rl = ur + kKeep * kMat, *pl = ur, *nl = ur + kKeep * Square16::kBytes;

    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int ch = id % nc;
    id /= nc;
    const int hq = id % p.Hq, b = id / p.Hq, rep = p.Hv / p.Hq;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, c = l % 16, u = l / 16;
    const int t0 = ch * kChunk, n = max(0, min(kChunk, delta_len(p, b) - t0));
    const bf16_t *q = static_cast<const bf16_t *>(p.q.p) + b * p.q.sb + hq * p.q.sh + (int64_t)t0 * p.q.st;
    const bf16_t *k = static_cast<const bf16_t *>(p.k.p) + b * p.k.sb + hq * p.k.sh + (int64_t)t0 * p.k.st;
    bf16_t *dqo = static_cast<bf16_t *>(p.dq.p) + b * p.dq.sb + hq * p.dq.sh + (int64_t)t0 * p.dq.st;
    bf16_t *dko = static_cast<bf16_t *>(p.dk.p) + b * p.dk.sb + hq * p.dk.sh + (int64_t)t0 * p.dk.st;
    if (n == 0) {   // past the sequence's end
        for (int x = threadIdx.x; x < kChunk * p.Dk / 4; x += kThreads) {
            const int t = x / (p.Dk / 4), m = x % (p.Dk / 4) * 4;
            if (t0 + t < p.T) {
                store4(dqo + t * p.dq.st + m, 0.f, 0.f, 0.f, 0.f);
                store4(dko + t * p.dk.st + m, 0.f, 0.f, 0.f, 0.f);
            }
        }
        for (int x = threadIdx.x; x < kChunk * rep; x += kThreads)
            if (t0 + x / rep < p.T) {
                const int64_t to = ((int64_t)b * p.T + t0 + x / rep) * p.Hv + hq * rep + x % rep;
                store_f(static_cast<bf16_t *>(p.dg) + to, 0.f);
                store_f(static_cast<bf16_t *>(p.dbeta) + to, 0.f);
            }
        return;
    }
    X qt, kt;
    qt.start(p.q.st, p.Dk);
    kt.start(p.k.st, p.Dk);
    qt.load_strict(q, p.q.st, 0, n, p.Dk);
    kt.load_strict(k, p.k.st, 0, n, p.Dk);
    f32x4_t dq[NB][4], dk[NB][4];   // rows 64 j + 16 w + 4 u + i, token 16 tb + c
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
            dq[j][tb] = dk[j][tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    for (int h = 0; h < rep; ++h) {
        const int hv = hq * rep + h;
        const int64_t at = ((int64_t)b * p.Hv + hv) * nc + ch;
        const float *gates = kept.gates + at * kGateRows * kChunk;
        const bf16_t *d = static_cast<const bf16_t *>(p.dout.p) + b * p.dout.sb + hv * p.dout.sh + (int64_t)t0 * p.dout.st;
        const bf16_t *v = static_cast<const bf16_t *>(p.v.p) + b * p.v.sb + hv * p.v.sh + (int64_t)t0 * p.v.st;
        // all that a head reads is on its way at once
        Unpacked<DVP> iu, ir, is;
        iu.load(kept.u, at * nv * 2, 2, 0, nv);
        ir.load(gr.r, at * nv * 2, 2, 0, nv);
        is.load(kept.s, at * nv * NG, NG, 0, nv);
        E dt;
        dt.start(p.dout.st, p.Dv);
        dt.load_strict(d, p.dout.st, 0, n, p.Dv);
        const int t = 16 * w + c;   // this lane's token of the 64 x 64 matrices
        uint4 vp[NE];
#pragma unroll
        for (int g = 0; g < NE; ++g)
            vp[g] = piece_of(v, p.v.st, t, n, 32 * g + 8 * u, p.Dv);
        const float bt = gates[t], gt = gates[4 * kChunk + t], gd = gates[5 * kChunk + t];
        f32x4_t gs[4], ds[4];
        float ge[4], gq[4], gl[4];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
            gs[tb] = load4(gates + 4 * kChunk + 16 * tb + 4 * u);
            ds[tb] = load4(gates + 5 * kChunk + 16 * tb + 4 * u);
            gq[tb] = gates[3 * kChunk + 16 * tb + c];
            ge[tb] = gates[kChunk + 16 * tb + c];
            gl[tb] = gates[2 * kChunk + 16 * tb + c];
        }
        step_fence();
        lds_barrier();   // the waves are done with the last head's P and N
        if (h == 0) {
            qt.store(ql);
            kt.store(kl);
        }
        iu.store(ul);
        ir.store(rl);
        is.store(sd);
        dt.store(dl);
        lds_barrier();
        is.load(gr.ds, at * nv * NG, NG, 0, nv);

        f32x4_t pm[4], nm[4];
        float along = 0.f, db = 0.f, colsum[4][4];
        {
            uint4 mine[NE];
            Terms<kKeep> rf[NE];
#pragma unroll
            for (int g = 0; g < NE; ++g) {
                mine[g] = ld16(dl + E::at(t, 4 * g + u));
                rf[g] = turned_terms(rl, w, g, l, DVP);
            }
#pragma unroll
            for (int sb = 0; sb < 4; ++sb) {
                pm[sb] = nm[sb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    colsum[sb][i] = 0.f;
                if (sb <= w) {
                    f32x4_t c1 = pm[sb], c2 = c1, qk = c1, kk = c1;
#pragma unroll
                    for (int g = 0; g < NE; ++g) {
                        const Terms<kKeep> uf = turned_terms(ul, sb, g, l, DVP);
                        c1 = mma(uf, one(mine[g]), c1);
                        c2 = mma(uf, rf[g], c2);
                    }
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const Terms<1> ks = one(ld16(kl + X::at(16 * sb + c, 4 * g + u)));
                        qk = mma(ks, one(ld16(ql + X::at(t, 4 * g + u))), qk);
                        kk = mma(ks, one(ld16(kl + X::at(t, 4 * g + u))), kk);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int s = 16 * sb + 4 * u + i;
                        const float kept_ts = s <= t ? decay(gt, gd, gs[sb][i], ds[sb][i]) : 0.f, strict = s < t ? kept_ts : 0.f;
                        pm[sb][i] = p.scale * kept_ts * c1[i];
                        nm[sb][i] = -bt * strict * c2[i];
                        const float ef = pm[sb][i] * qk[i] + nm[sb][i] * kk[i];
                        along += ef;
                        db -= strict * c2[i] * kk[i];
                        colsum[sb][i] = over_c(ef);
                    }
                }
            }
            along = over_u(along);
            db = over_u(db);
        }
        if (c == 0)
#pragma unroll
            for (int sb = 0; sb < 4; ++sb)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sums[w][3][16 * sb + 4 * u + i] = colsum[sb][i];
        // products with the states: S first, then dS in its place
        float qy[4] = {0.f, 0.f, 0.f, 0.f}, ky[4] = {0.f, 0.f, 0.f, 0.f}, kz[4] = {0.f, 0.f, 0.f, 0.f}, dot = 0.f;
        const float last = gates[4 * kChunk + kChunk - 1];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int m0 = 64 * j + 16 * w + 4 * u;
            if (j > 0) {
                lds_barrier();
                is.store(sd);
                lds_barrier();
                is.load(gr.ds, at * nv * NG, NG, 2 * j, nv);
            }
            f32x4_t y1[4], y2[4];
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
                y1[tb] = y2[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            Terms<kKeep> sf[NE];
#pragma unroll
            for (int g = 0; g < NE; ++g) {
                sf[g] = turned_terms(sd, w, g, l, DVP);
#pragma unroll
                for (int tb = 0; tb < 4; ++tb) {
                    y1[tb] = mma(sf[g], one(ld16(dl + E::at(16 * tb + c, 4 * g + u))), y1[tb]);
                    y2[tb] = mma(sf[g], turned_terms(rl, tb, g, l, DVP), y2[tb]);
                }
            }
#pragma unroll
            for (int tb = 0; tb < 4; ++tb) {
                const int row = 16 * tb + c;
                const uint2 qw = *reinterpret_cast<const uint2 *>(ql + X::at(row, m0 / 8) + 2 * (m0 % 8));
                const uint2 kw = *reinterpret_cast<const uint2 *>(kl + X::at(row, m0 / 8) + 2 * (m0 % 8));
                const f32x4_t qq = {bf_lo(qw.x), bf_hi(qw.x), bf_lo(qw.y), bf_hi(qw.y)};
                const f32x4_t kx = {bf_lo(kw.x), bf_hi(kw.x), bf_lo(kw.y), bf_hi(kw.y)};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = p.scale * gq[tb] * y1[tb][i];
                    qy[tb] = fmaf(qq[i], a, qy[tb]);
                    ky[tb] = fmaf(kx[i], gq[tb] * y2[tb][i], ky[tb]);
                    dq[j][tb][i] += a;
                    dk[j][tb][i] -= ge[tb] * y2[tb][i];
                }
            }
            lds_barrier();
            is.store(sd);
            lds_barrier();
            if (j + 1 < NB)
                is.load(kept.s, at * nv * NG, NG, 2 * j + 2, nv);
            f32x4_t y3[4];
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
                y3[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < NE; ++g) {
                const Terms<kKeep> ef = turned_terms(sd, w, g, l, DVP);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    dot = fmaf((float)sf[g].v[0][e] + (float)sf[g].v[1][e], (float)ef.v[0][e] + (float)ef.v[1][e], dot);
#pragma unroll
                for (int tb = 0; tb < 4; ++tb)
                    y3[tb] = mma(ef, turned_terms(ul, tb, g, l, DVP), y3[tb]);
            }
#pragma unroll
            for (int tb = 0; tb < 4; ++tb) {
                const uint2 kw = *reinterpret_cast<const uint2 *>(kl + X::at(16 * tb + c, m0 / 8) + 2 * (m0 % 8));
                const f32x4_t kx = {bf_lo(kw.x), bf_hi(kw.x), bf_lo(kw.y), bf_hi(kw.y)};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = gl[tb] * y3[tb][i];
                    kz[tb] = fmaf(kx[i], a, kz[tb]);
                    dk[j][tb][i] += a;
                }
            }
        }
        // R.v of token t: a quarter of the entries a wave's quarter
        float rv = 0.f;
#pragma unroll
        for (int g = 0; g < NE; ++g) {
            const Terms<kKeep> rf = turned_terms(rl, w, g, l, DVP);
            const bf16x8_t vf = one(vp[g]).v[0];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                rv = fmaf((float)rf.v[0][e] + (float)rf.v[1][e], (float)vf[e], rv);
        }
        rv = over_u(rv);
        dot = over_u(over_c(dot));
        if (l == 0)
            ss[w] = dot;
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
            const float a = over_u(qy[tb]), e = over_u(ky[tb]), f = over_u(kz[tb]);
            if (u == 0) {
                sums[w][0][16 * tb + c] = a;
                sums[w][1][16 * tb + c] = e;
                sums[w][2][16 * tb + c] = f;
            }
        }
        lds_barrier();   // U and R are done with
#pragma unroll
        for (int sb = 0; sb < 4; ++sb)
            if (sb <= (w | 1)) {
                put4<kKeep>(pl, t, 16 * sb + 4 * u, pm[sb]);
                put4<kKeep>(nl, t, 16 * sb + 4 * u, nm[sb]);
            }
        if (u == 0) {   // the row sums, by the wave that has them
            const auto sum4 = [&](int i) { return ((sums[0][i][t] + sums[1][i][t]) + sums[2][i][t]) + sums[3][i][t]; };
            const float a = sum4(0), e = sum4(1), f = sum4(2), cs = sum4(3);
            if (t0 + t < p.T)
                store_f(static_cast<bf16_t *>(p.dbeta) + ((int64_t)b * p.T + t0 + t) * p.Hv + hv, t < n ? rv - e + db : 0.f);
            sums[0][3][t] = a + along - cs - bt * e - f;   // dG, but for what the last token has beside
            sums[0][2][t] = f;
        }
        lds_barrier();
        if (w == 0) {
            float dG = sums[0][3][l], all = sums[0][2][l];
#pragma unroll
            for (int x = 1; x < 64; x *= 2)
                all += __shfl_xor(all, x);
            if (l == kChunk - 1)
                dG += all + exp_f(last) * (((ss[0] + ss[1]) + ss[2]) + ss[3]);
#pragma unroll
            for (int x = 1; x < 64; x *= 2) {
                const float o = __shfl_down(dG, x);
                if (l + x < 64)
                    dG += o;
            }
            if (t0 + l < p.T)
                store_f(static_cast<bf16_t *>(p.dg) + ((int64_t)b * p.T + t0 + l) * p.Hv + hv, l < n ? dG : 0.f);
        }
        // over the tokens: dQ^T += K^T P^T, dK^T += Q^T P + K^T (N + N^T)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int i = l % 16, row = 32 * g + 8 * u + (i >> 2), piece = 2 * (4 * j + w) + ((i & 3) >> 1), in = 8 * (i & 1);
                struct {
                    s16x4_t a, b;
                } kw = {read_turned(kl + X::at(row, piece) + in), read_turned(kl + X::at(row + 4, piece) + in)},
                  qw = {read_turned(ql + X::at(row, piece) + in), read_turned(ql + X::at(row + 4, piece) + in)};
                const Terms<1> kx{{__builtin_bit_cast(bf16x8_t, kw)}}, qx{{__builtin_bit_cast(bf16x8_t, qw)}};
#pragma unroll
                for (int tb = 0; tb < 4; ++tb) {
                    if (g <= tb / 2) {   // columns s of group g, rows t = 16 tb + c
                        dq[j][tb] = mma(kx, row_terms<kKeep>(pl, 16 * tb + c, 4 * g + u), dq[j][tb]);
                        dk[j][tb] = mma(kx, row_terms<kKeep>(nl, 16 * tb + c, 4 * g + u), dk[j][tb]);
                    }
                    if (g >= tb / 2) {   // rows t of group g, column s = 16 tb + c
                        dk[j][tb] = mma(qx, turned_terms(pl, tb, g, l, kChunk), dk[j][tb]);
                        dk[j][tb] = mma(kx, turned_terms(nl, tb, g, l, kChunk), dk[j][tb]);
                    }
                }
            }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
            const int t = 16 * tb + c, m = 64 * j + 16 * w + 4 * u;
            if (t0 + t < p.T && m < p.Dk) {
                const float f = t < n ? 1.f : 0.f;
                store4(dqo + t * p.dq.st + m, f * dq[j][tb][0], f * dq[j][tb][1], f * dq[j][tb][2], f * dq[j][tb][3]);
                store4(dko + t * p.dk.st + m, f * dk[j][tb][0], f * dk[j][tb][1], f * dk[j][tb][2], f * dk[j][tb][3]);
            }
        }
}

hipError_t take(const DeltaProblem &p, Kept16 *kept)
{
    const int64_t n = (int64_t)p.B * p.Hv * delta_chunks(p), nv = delta_sv(p) / 16, ng = p.Dk <= 64 ? 2 : 4;
    Workspace *w = p.rs ? p.rs : p.ws;
    void *a[5] = {};
    hipError_t e = w->take(&a[0], (size_t)(n * kGateRows * kChunk * 4));
    if (e == hipSuccess)
        e = w->take(&a[1], (size_t)(n * nv * 2 * kKeep * 1024));
    if (e == hipSuccess)
        e = w->take(&a[2], (size_t)(n * nv * ng * kKeep * 1024));
    if (e == hipSuccess && p.rs)
        e = w->take(&a[3], (size_t)(n * kInvUnits * 3 * 1024));
    kept->gates = static_cast<float *>(a[0]);
    kept->u = static_cast<uint4 *>(a[1]);
    kept->s = static_cast<uint4 *>(a[2]);
    kept->turned = static_cast<uint4 *>(a[3]);
    return e;
}

template <int DKP>
hipError_t fwd(const DeltaProblem &p, hipStream_t s)
{
    const int nc = delta_chunks(p), nv = delta_sv(p) / 16;
    const int64_t heads = (int64_t)p.B * p.Hv;
    Kept16 kept;
    hipError_t e = take(p, &kept);
    void *inv = nullptr;
    if (e == hipSuccess)
        e = p.ws->take(&inv, (size_t)(heads * nc * kInvUnits * 3 * 1024));
    kept.inv = static_cast<uint4 *>(inv);
    if (heads * nc * kThreads > kMaxThreads || heads * nv * DKP * 2 > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (e != hipSuccess || p.ws->counting)
        return e;
    delta16_inverse_kernel<DKP><<<dim3((unsigned)((heads * nc + 3) / 4)), kThreads, 0, s>>>(p, kept, nc);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    delta16_state_kernel<DKP><<<dim3((unsigned)(heads * nv)), DKP * 2, 0, s>>>(p, kept, nc, nv);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    delta16_out_kernel<DKP><<<dim3((unsigned)(heads * nc)), kThreads, 0, s>>>(p, kept, nc, nv);
    return hipGetLastError();
}

template <int DKP, int DVP>
hipError_t bwd(const DeltaProblem &p, hipStream_t s)
{
    const int nc = delta_chunks(p), nv = delta_sv(p) / 16;
    const int64_t heads = (int64_t)p.B * p.Hv, n = heads * nc;
    Kept16 kept;
    hipError_t e = take(p, &kept);
    void *du = nullptr, *r = nullptr, *ds = nullptr;
    if (e == hipSuccess)
        e = p.ws->take(&du, (size_t)(n * nv * 4 * 1024));
    if (e == hipSuccess)
        e = p.ws->take(&r, (size_t)(n * nv * 2 * kKeep * 1024));
    if (e == hipSuccess)
        e = p.ws->take(&ds, (size_t)(n * nv * (DKP / 32) * kKeep * 1024));
    if (n * kThreads > kMaxThreads || heads * nv * DKP * 2 > kMaxThreads)
        return hipErrorInvalidConfiguration;
    if (e != hipSuccess || p.ws->counting)
        return e;
    Grads16 g;
    g.du = static_cast<float *>(du);
    g.r = static_cast<uint4 *>(r);
    g.ds = static_cast<uint4 *>(ds);
    delta16_du_kernel<DKP, DVP><<<dim3((unsigned)n), kThreads, 0, s>>>(p, kept, g, nc, nv);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    delta16_dstate_kernel<DKP><<<dim3((unsigned)(heads * nv)), DKP * 2, 0, s>>>(p, kept, g, nc, nv);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    delta16_grad_kernel<DKP, DVP><<<dim3((unsigned)((int64_t)p.B * p.Hq * nc)), kThreads, 0, s>>>(p, kept, g, nc, nv);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta16_bwd(const DeltaProblem &p, hipStream_t s)
{
    if (p.Dk <= 64)
        return p.Dv <= 64 ? bwd<64, 64>(p, s) : bwd<64, 128>(p, s);
    return p.Dv <= 64 ? bwd<128, 64>(p, s) : bwd<128, 128>(p, s);
}

hipError_t delta16_reserve(const DeltaProblem &p)
{
    Kept16 kept;
    return take(p, &kept);
}

hipError_t launch_delta16_fwd(const DeltaProblem &p, hipStream_t s)
{
    return p.Dk <= 64 ? fwd<64>(p, s) : fwd<128>(p, s);
}

}  // namespace gspn
