// The selective state space scan (internal).
//
//   d = softplus(dt + dt_bias),  h_t = exp(d A) h_{t-1} + d x B_t,  y = (C_t . h_t + D x) silu(z)
//
// for every channel with its own N states.  The tokens are cut into chunks where the
// channels alone do not fill the card: what a chunk adds to its states from zeros, and the
// sum of its steps, whose exponentials are the chunk's whole decay; a chain over the
// chunks; and the chunks again from the states they begin with.
#pragma once

#include "attn.hpp"

namespace gspn {

struct SelectiveProblem {
    Heads x, dt, z, y;                    // [B][T][C], strides of b and t; z.p may be null
    Heads Bm, Cm;                         // [B][T][G][N]
    const float *A;                       // [C][N]
    const float *D, *dt_bias;             // [C] or null
    const float *state;                   // [B][C][N], or null: zeros
    float *state_out;                     // the same, or null: not wanted
    Heads dy, dx, ddt, dz, dBm, dCm;      // backward
    const float *dstate;                  // gradient of state_out, or null: zeros
    float *dA, *dD, *ddt_bias, *dstate_in;
    const int32_t *lens;                  // [B], or null: T
    int B, T, C, G, N;
    bool softplus;
    int dtype;
    Workspace *ws;
    Workspace *rs = nullptr;              // the training pair's reserve
};

constexpr int kSelMaxStates = 64;

// Tokens between the states that a training forward keeps for its backward.
constexpr int kSelKeep = 8;

// Whether a forward goes along whole sequences in one pass, four lanes a channel (16 of them a
// wave), instead of in chunks that it goes through twice: by what either takes.  One pass:
// 17 us and, a token, `first` ns with up to one wave a SIMD and `more` for each further one.
// Chunks: 30 us and, a token and wave's worth of channels, `chunks` ps.  Measured (us, one pass
// and chunks, 1024 tokens of 1536 channels, with the states kept): 4 states batch 1 120 and
// 34, 64 412 and 351; 8 states batch 32 360 and 259, 64 476 and 481; 16 states batch 1 138
// and 44, 8 140 and 135, 32 381 and 397, 64 753 and 706; 32 states batch 1 231 and 73, 8 295
// and 259, 32 562 and 842; 64 states batch 1 371 and 128, 8 447 and 573, 32 1160 and 1834;
// 64 tokens, 16 states, batch 1 23 and 34, 32 28 and 65.  Without: 16 states batch 8 120 and
// 127, 32 250 and 366, 64 463 and 655; 32 states batch 8 219 and 230.  It errs at 16 states
// batch 64 and 32 states batch 8 with the states kept, and at 16 batch 8 without (5 to 14%).
inline bool sel_one_pass(const SelectiveProblem &p)
{
    struct Cost {
        int first, more, chunks;
    };
    constexpr Cost cost[2][5] = {{{158, 40, 53}, {162, 42, 75}, {108, 68, 111}, {180, 102, 225}, {292, 170, 495}},
                                 {{165, 50, 57}, {165, 55, 82}, {120, 105, 115}, {186, 185, 260}, {310, 300, 585}}};
    int i = 0;
    while (4 << i < p.N)
        ++i;
    const Cost &c = cost[p.rs ? 1 : 0][i];
    const int64_t waves = (int64_t)p.B * p.G * ((p.C / p.G + 15) / 16), simds = 1024;
    const double one = 17000. + (double)p.T * (c.first + c.more * (double)((waves - 1) / simds));
    return one < 30000. + (double)p.T * (double)waves * c.chunks / 1000.;
}

// States as the kernels hold them: N rounded up to a power of two, at least the four that
// quads of lanes share out (in one pass, and in the backward); entries past N are 0.
inline int sel_states(const SelectiveProblem &p)
{
    int n = p.rs || sel_one_pass(p) ? 4 : 1;
    while (n < p.N)
        n *= 2;
    return n;
}

// B and C of every token as fp32, [B][T][G][B, C][states], entries past N and tokens past a
// sequence's end 0: the kernels read them as scalars, one token ahead, and there is room for
// a token's before the first and behind the last.
constexpr int kPackTokens = 16;   // of a workgroup
inline int64_t sel_pack_groups(const SelectiveProblem &p) { return (int64_t)p.B * ((p.T + kPackTokens - 1) / kPackTokens); }
inline size_t sel_packed(const SelectiveProblem &p) { return ((size_t)p.B * p.T + 2) * p.G * 2 * sel_states(p) * 4; }

// The reserve: the states ahead of every kSelKeep-th token, [B][ceil(T / kSelKeep)][states][C],
// and B and C as they are packed.
inline hipError_t take_sel_kept(const SelectiveProblem &p, Workspace *rs, void **kept, void **bc)
{
    const hipError_t e = rs->take(kept, (size_t)p.B * ((p.T + kSelKeep - 1) / kSelKeep) * sel_states(p) * p.C * 4);
    return e == hipSuccess ? rs->take(bc, sel_packed(p)) : e;
}

hipError_t launch_selective_fwd(const SelectiveProblem &p, hipStream_t s);
hipError_t launch_selective_fwd_f32(const SelectiveProblem &p, hipStream_t s);   // of launch_selective_fwd
hipError_t launch_selective_bwd(const SelectiveProblem &p, hipStream_t s);

}  // namespace gspn
