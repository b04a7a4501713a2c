// C ABI of the token mixers beside the scan: the norm of query and key heads
// with the position rotation, windowed attention, and the gated delta rule.
// Argument checks (host only, before any HIP call), workspaces, launches.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/gspn.h"
#include "attn.hpp"
#include "delta.hpp"
#include "launch.hpp"
#include "qk_norm.hpp"

namespace gspn {
namespace {

int64_t storage(int dtype) { return dtype == GSPN_F32 ? 4 : 2; }

// A buffer of a call as its checks see it: pieces of `inner` bytes, repeated in
// up to three dimensions, over `bytes` in all.
struct Span {
    struct Dim {
        int64_t step, n;
    };
    uintptr_t p = 0;
    int64_t bytes = 0, inner = 0;
    Dim dim[3] = {{0, 1}, {0, 1}, {0, 1}};
    bool output = false;

    // What the dimensions that step by less than s cover, where the others step by
    // multiples of s and it fits between them; else more than s.
    int64_t below(int64_t s) const
    {
        int64_t ext = inner;
        for (const Dim &d : dim) {
            if (d.n <= 1)
                continue;
            if (d.step < s)
                ext += (d.n - 1) * d.step;
            else if (d.step % s != 0)
                return s + 1;
        }
        return ext;
    }
    bool same(const Span &o) const
    {
        bool is = p == o.p && bytes == o.bytes && inner == o.inner;
        for (int i = 0; i < 3; ++i)
            is = is && dim[i].n == o.dim[i].n && (dim[i].n <= 1 || dim[i].step == o.dim[i].step);
        return is;
    }
};

// A contiguous buffer (aligned to its elements).
Span flat(const void *p, int64_t bytes, bool output = false)
{
    Span x;
    x.p = reinterpret_cast<uintptr_t>(p);
    x.bytes = x.inner = bytes;
    x.output = output;
    return x;
}

// Two buffers have no byte in common: their ranges are apart, or they are slices
// of one buffer's tokens, heads or batch entries: some step of theirs repeats both,
// and what lies within one repetition is apart.
bool apart(const Span &a, const Span &b)
{
    if (a.p + (uintptr_t)a.bytes <= b.p || b.p + (uintptr_t)b.bytes <= a.p)
        return true;
    for (const Span *x : {&a, &b})
        for (const Span::Dim &d : x->dim) {
            const int64_t s = d.step;
            if (d.n <= 1 || s <= 0)
                continue;
            const int64_t ea = a.below(s), eb = b.below(s), off = (int64_t)(b.p - a.p) % s, r = off < 0 ? off + s : off;
            if (ea <= s && eb <= s && r >= ea && r + eb <= s)
                return true;
        }
    return false;
}

// The checks of a call's buffers, one after the other.
struct Buffers {
    Span all[20];
    int n = 0;
    int status = GSPN_OK;

    void fail(int st)
    {
        if (status == GSPN_OK)
            status = st;
    }
    void add(const Span &s)
    {
        for (int i = 0; i < n; ++i)
            if ((all[i].output || s.output) && !apart(all[i], s))
                fail(GSPN_ERR_ALIAS);
        all[n++] = s;
    }
    // a contiguous buffer whose elements are `align` bytes; `same`: may equal buffer `same` exactly
    void buffer(const void *p, int64_t bytes, int align, bool output, bool optional = false)
    {
        if (p == nullptr)
            return optional ? void() : fail(GSPN_ERR_NULL);
        if (reinterpret_cast<uintptr_t>(p) % align != 0)
            return fail(GSPN_ERR_ALIGN);
        add(flat(p, bytes, output));
    }
    // a [B][T][H][D] tensor with strides s (batch, token, head), null: contiguous.
    // inplace: the index of a tensor that it may be, byte for byte
    Heads heads(const void *p, const int64_t *s, int64_t B, int64_t T, int64_t H, int64_t D, int dtype, bool output,
                int inplace = -1)
    {
        const int64_t es = storage(dtype);
        Heads h;
        h.p = const_cast<void *>(p);
        h.sh = H > 1 ? (s ? s[2] : D) : D;
        h.st = T > 1 ? (s ? s[1] : H * D) : D;
        h.sb = B > 1 ? (s ? s[0] : T * H * D) : 0;
        if (p == nullptr) {
            fail(GSPN_ERR_NULL);
            return h;
        }
        // token strides: 64 rows of any tile are within 32-bit offsets of its first
        constexpr int64_t kMost = (int64_t)1 << 44, kMostStep = (int64_t)1 << 23;
        if (h.sh < 0 || h.st < 0 || h.sb < 0 || h.sh > kMost || h.st > kMost || h.sb > kMost / std::max<int64_t>(1, B) ||
            h.st > kMostStep) {
            fail(GSPN_ERR_UNSUPPORTED);
            return h;
        }
        if (reinterpret_cast<uintptr_t>(p) % 16 != 0 || h.sh * es % 16 != 0 || h.st * es % 16 != 0 ||
            h.sb * es % 16 != 0) {
            fail(GSPN_ERR_ALIGN);
            return h;
        }
        if (output) {   // no element of an output is written twice
            Span::Dim dim[3] = {{h.sh, H}, {h.st, T}, {h.sb, B}};
            std::sort(dim, dim + 3, [](const Span::Dim &x, const Span::Dim &y) { return x.step < y.step; });
            int64_t ext = D;
            for (const Span::Dim &d : dim) {
                if (d.n > 1 && d.step < ext)
                    fail(GSPN_ERR_ALIAS);
                ext += (d.n - 1) * d.step;
            }
        }
        Span x;
        x.p = reinterpret_cast<uintptr_t>(p);
        x.inner = D * es;
        x.bytes = x.inner + ((H - 1) * h.sh + (T - 1) * h.st + (B - 1) * h.sb) * es;
        x.dim[0] = {h.sh * es, H}, x.dim[1] = {h.st * es, T}, x.dim[2] = {h.sb * es, B};
        x.output = output;
        if (inplace >= 0 && inplace < n && status == GSPN_OK && all[inplace].same(x)) {
            for (int i = 0; i < n; ++i)
                if (i != inplace && !apart(all[i], x))
                    fail(GSPN_ERR_ALIAS);
            all[inplace].output = true;
            return h;
        }
        add(x);
        return h;
    }
};

template <typename P>
struct requires_reserve : std::false_type {};
template <>
struct requires_reserve<DeltaProblem> : std::true_type {};

// Runs `launch` in counting mode for the bytes it takes, checks the caller's
// workspace against them and the other buffers, and launches.
template <typename P>
int run(P &p, hipError_t (*launch)(const P &, hipStream_t), Buffers &bufs, void *workspace, int64_t bytes, void *stream)
{
    Workspace ws;
    ws.counting = true;
    p.ws = &ws;
    hipError_t e = launch(p, nullptr);
    if (e == hipErrorInvalidConfiguration)   // more workgroups than a launch may have
        return GSPN_ERR_UNSUPPORTED;
    if (e != hipSuccess)
        return hip_status(e);
    const int64_t need = (int64_t)ws.used;
    if (need > 0) {
        if (workspace == nullptr || bytes < need)
            return GSPN_ERR_WORKSPACE;
        bufs.buffer(workspace, need, 16, true);
        if (bufs.status != GSPN_OK)
            return bufs.status;
    }
    if constexpr (requires_reserve<P>::value)
        if (p.rs)
            p.rs->used = 0;
    ws = Workspace{};
    ws.base = static_cast<char *>(workspace);
    ws.size = (size_t)std::max<int64_t>(0, bytes);
    return hip_status(launch(p, static_cast<hipStream_t>(stream)));
}

template <typename P>
int count(P &p, hipError_t (*launch)(const P &, hipStream_t), int64_t *bytes)
{
    Workspace ws;
    ws.counting = true;
    p.ws = &ws;
    const hipError_t e = launch(p, nullptr);
    if (e == hipErrorInvalidConfiguration)
        return GSPN_ERR_UNSUPPORTED;
    if (e != hipSuccess)
        return hip_status(e);
    *bytes = (int64_t)ws.used;
    return GSPN_OK;
}

// Positions stay below 2^30, so that a position and a window add up in 32 bits.
constexpr int64_t kMostTokens = (int64_t)1 << 28;
constexpr int kMostWindow = 1 << 30;

int check_sizes(int64_t B, int64_t T, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D, int most, int dtype)
{
    if (dtype != GSPN_F32 && dtype != GSPN_BF16)
        return GSPN_ERR_DTYPE;
    if (B < 1 || T < 1 || Tk < 1 || Hq < 1 || Hkv < 1 || D < 1)
        return GSPN_ERR_DIM;
    if (D % 8 != 0 || D > most || T > kMostTokens || Tk > kMostTokens || B > kMostTokens || Hq > 65536 || Hkv > 65536 ||
        B * Hq > kMostTokens || B * Hkv > kMostTokens || T > GSPN_MAX_ELEMS / (B * Hq) / D ||
        Tk > GSPN_MAX_ELEMS / (B * Hkv) / D)
        return GSPN_ERR_UNSUPPORTED;
    return GSPN_OK;
}

// Sizes, window and scale of an attention call.
int make_attn(AttnProblem &p, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left, int right, int sinks, int offset,
              float scale, int dtype)
{
    const int st = check_sizes(B, Tq, Tk, Hq, Hkv, D, kAttnMaxHead, dtype);
    if (st != GSPN_OK)
        return st;
    if (Hq % Hkv != 0 || sinks < 0 || offset < 0 || !(scale > 0.f) || !isfinite(scale))
        return GSPN_ERR_DIM;
    if (offset > kMostTokens)
        return GSPN_ERR_UNSUPPORTED;
    p = AttnProblem{};
    p.B = B, p.Tq = Tq, p.Tk = Tk, p.Hq = Hq, p.Hkv = Hkv, p.D = D;
    p.left = left < 0 ? -1 : std::min(left, kMostWindow);
    p.right = right < 0 ? -1 : std::min(right, kMostWindow);
    p.sinks = std::min(sinks, Tk);
    p.offset = offset;
    p.scale = scale;
    p.dtype = dtype;
    return GSPN_OK;
}

const int64_t *at(const int64_t *strides, int i) { return strides ? strides + 3 * i : nullptr; }

int make_norm(NormProblem &p, int B, int T, int Hq, int Hk, int D, int R, int rows, int first, int pairs, float eps,
              int dtype, bool table, bool positions)
{
    const int st = check_sizes(B, T, 1, Hq, Hk, D, kNormMaxHead, dtype);
    if (st != GSPN_OK)
        return st;
    if (R < 0 || R > D || R % 2 != 0 || !(eps >= 0.f) || !isfinite(eps) ||
        (pairs != GSPN_PAIRS_HALF && pairs != GSPN_PAIRS_ADJACENT))
        return GSPN_ERR_DIM;
    if (R > 0 && (rows < 1 || (!positions && (first < 0 || (int64_t)first + T > rows))))
        return GSPN_ERR_DIM;
    if (R > 0 && !table)
        return GSPN_ERR_NULL;
    p = NormProblem{};
    p.B = B, p.T = T, p.Hq = Hq, p.Hk = Hk, p.D = D, p.R = R;
    p.rows = rows, p.first = first;
    p.adjacent = pairs == GSPN_PAIRS_ADJACENT;
    p.eps = eps;
    p.dtype = dtype;
    return GSPN_OK;
}

int make_delta(DeltaProblem &p, int B, int T, int Hq, int Hv, int Dk, int Dv, float scale, int dtype)
{
    int st = check_sizes(B, T, 1, Hq, Hv, Dk, kDeltaMaxHead, dtype);
    if (st == GSPN_OK)
        st = check_sizes(B, T, 1, Hv, Hq, Dv, kDeltaMaxHead, dtype);
    if (st != GSPN_OK)
        return st;
    if (Hv % Hq != 0 || !isfinite(scale))
        return GSPN_ERR_DIM;
    p = DeltaProblem{};
    p.B = B, p.T = T, p.Hq = Hq, p.Hv = Hv, p.Dk = Dk, p.Dv = Dv;
    p.scale = scale;
    p.dtype = dtype;
    return GSPN_OK;
}

// Bytes of the training pair's reserve.
int64_t delta_reserve(const DeltaProblem &p)
{
    Workspace rs;
    rs.counting = true;
    DeltaKept kept;
    DeltaProblem q = p;
    q.rs = &rs;
    if (p.dtype == GSPN_F32)
        take_delta_kept(q, &rs, &kept);
    else
        delta16_reserve(q);
    return (int64_t)rs.used;
}

// The inputs that both passes of the delta rule read.
void delta_inputs(DeltaProblem &p, Buffers &bufs, const void *q, const void *k, const void *v, const void *g,
                  const void *beta, const int32_t *lens, const int64_t *strides)
{
    const int64_t gates = (int64_t)p.B * p.T * p.Hv * storage(p.dtype);
    p.q = bufs.heads(q, at(strides, 0), p.B, p.T, p.Hq, p.Dk, p.dtype, false);
    p.k = bufs.heads(k, at(strides, 1), p.B, p.T, p.Hq, p.Dk, p.dtype, false);
    p.v = bufs.heads(v, at(strides, 2), p.B, p.T, p.Hv, p.Dv, p.dtype, false);
    bufs.buffer(g, gates, (int)storage(p.dtype), false);
    bufs.buffer(beta, gates, (int)storage(p.dtype), false);
    bufs.buffer(lens, (int64_t)p.B * 4, 4, false, true);
    p.g = g, p.beta = beta, p.lens = lens;
}

int delta_fwd(const void *q, const void *k, const void *v, const void *g, const void *beta, const float *state,
              const int32_t *lens, void *o, float *state_out, const int64_t *strides, int B, int T, int Hq, int Hv, int Dk,
              int Dv, float scale, int dtype, void *reserve, int64_t reserve_bytes, bool train, void *workspace,
              int64_t workspace_bytes, void *stream)
{
    DeltaProblem p;
    const int st = make_delta(p, B, T, Hq, Hv, Dk, Dv, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    delta_inputs(p, bufs, q, k, v, g, beta, lens, strides);
    const int64_t states = (int64_t)B * Hv * Dk * Dv * 4;
    if (state != state_out)   // a state may be continued in place
        bufs.buffer(state, states, 16, false, true);
    p.o = bufs.heads(o, at(strides, 3), B, T, Hv, Dv, dtype, true);
    bufs.buffer(state_out, states, 16, true, true);
    p.state = state, p.state_out = state_out;
    Workspace rs;
    if (train) {
        const int64_t need = delta_reserve(p);
        if (bufs.status == GSPN_OK && (reserve == nullptr || reserve_bytes < need))
            return GSPN_ERR_WORKSPACE;
        bufs.buffer(reserve, need, 16, true);
        rs.base = static_cast<char *>(reserve);
        rs.size = (size_t)need;
        p.rs = &rs;
    }
    if (bufs.status != GSPN_OK)
        return bufs.status;
    return run(p, launch_delta_fwd, bufs, workspace, workspace_bytes, stream);
}

// The weights and tables that both passes of the norm read.
void norm_inputs(NormProblem &p, Buffers &bufs, const void *wq, const void *wk, const float *cos_t, const float *sin_t,
                 const int32_t *positions)
{
    const int64_t es = storage(p.dtype), table = (int64_t)p.rows * (p.R / 2) * 4;
    bufs.buffer(wq, p.D * es, 16, false, true);
    bufs.buffer(wk, p.D * es, 16, false, true);
    if (p.R > 0) {
        bufs.buffer(cos_t, table, 16, false);
        bufs.buffer(sin_t, table, 16, false);
        bufs.buffer(positions, (int64_t)p.B * p.T * 4, 4, false, true);
        p.cos = cos_t, p.sin = sin_t, p.positions = positions;
    }
    p.wq = wq, p.wk = wk;
}

}  // namespace
}  // namespace gspn

using namespace gspn;

extern "C" int gspn_qk_norm_rotate_fwd(const void *q, const void *k, const void *wq, const void *wk, const float *cos_t,
                                       const float *sin_t, const int32_t *positions, void *yq, void *yk,
                                       const int64_t *strides, int B, int T, int Hq, int Hk, int D, int R, int table_rows,
                                       int first, int pairs, float eps, int dtype, void *stream)
{
    NormProblem p;
    const int st = make_norm(p, B, T, Hq, Hk, D, R, table_rows, first, pairs, eps, dtype, cos_t && sin_t, positions);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, T, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, T, Hk, D, dtype, false);
    norm_inputs(p, bufs, wq, wk, cos_t, sin_t, positions);
    p.yq = bufs.heads(yq, at(strides, 2), B, T, Hq, D, dtype, true, 0);
    p.yk = bufs.heads(yk, at(strides, 3), B, T, Hk, D, dtype, true, 1);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    return run(p, launch_norm_rotate_fwd, bufs, nullptr, 0, stream);
}

extern "C" int gspn_qk_norm_rotate_workspace_size(int B, int T, int Hq, int Hk, int D, int R, int pairs, int dtype,
                                                  int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    NormProblem p;
    const int st = make_norm(p, B, T, Hq, Hk, D, R, T, 0, pairs, 0.f, dtype, true, false);
    if (st != GSPN_OK)
        return st;
    p.wq = p.wk = bytes;   // counted as if both were there
    return count(p, launch_norm_rotate_bwd, bytes);
}

extern "C" int gspn_qk_norm_rotate_bwd(const void *q, const void *k, const void *wq, const void *wk, const float *cos_t,
                                       const float *sin_t, const int32_t *positions, const void *dyq, const void *dyk,
                                       void *dq, void *dk, void *dwq, void *dwk, const int64_t *strides, int B, int T,
                                       int Hq, int Hk, int D, int R, int table_rows, int first, int pairs, float eps,
                                       int dtype, void *workspace, int64_t workspace_bytes, void *stream)
{
    NormProblem p;
    const int st = make_norm(p, B, T, Hq, Hk, D, R, table_rows, first, pairs, eps, dtype, cos_t && sin_t, positions);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, T, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, T, Hk, D, dtype, false);
    norm_inputs(p, bufs, wq, wk, cos_t, sin_t, positions);
    p.dyq = bufs.heads(dyq, at(strides, 2), B, T, Hq, D, dtype, false);
    p.dyk = bufs.heads(dyk, at(strides, 3), B, T, Hk, D, dtype, false);
    p.dq = bufs.heads(dq, at(strides, 4), B, T, Hq, D, dtype, true);
    p.dk = bufs.heads(dk, at(strides, 5), B, T, Hk, D, dtype, true);
    // a weight that was given has a gradient
    if (wq)
        bufs.buffer(dwq, D * storage(dtype), 16, true);
    if (wk)
        bufs.buffer(dwk, D * storage(dtype), 16, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.dwq = wq ? dwq : nullptr;
    p.dwk = wk ? dwk : nullptr;
    return run(p, launch_norm_rotate_bwd, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_window_attn_workspace_size(int op, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left, int right,
                                               int sinks, int offset, int dtype, int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    if (op != GSPN_ATTN_FWD && op != GSPN_ATTN_BWD && op != GSPN_ATTN_DECODE)
        return GSPN_ERR_UNSUPPORTED;
    AttnProblem p;
    const int st = make_attn(p, B, Tq, Tk, Hq, Hkv, D, left, op == GSPN_ATTN_DECODE ? 0 : right, sinks,
                             op == GSPN_ATTN_DECODE ? 0 : offset, 1.f, dtype);
    if (st != GSPN_OK)
        return st;
    return count(p, op == GSPN_ATTN_FWD ? launch_attn_fwd : op == GSPN_ATTN_BWD ? launch_attn_bwd : launch_attn_split, bytes);
}

extern "C" int gspn_window_attn_fwd(const void *q, const void *k, const void *v, const int32_t *lens, void *o, float *lse,
                                    const int64_t *strides, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left,
                                    int right, int sinks, int offset, float scale, int dtype, void *workspace,
                                    int64_t workspace_bytes, void *stream)
{
    AttnProblem p;
    const int st = make_attn(p, B, Tq, Tk, Hq, Hkv, D, left, right, sinks, offset, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, Tq, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, Tk, Hkv, D, dtype, false);
    p.v = bufs.heads(v, at(strides, 2), B, Tk, Hkv, D, dtype, false);
    bufs.buffer(lens, (int64_t)B * 4, 4, false, true);
    p.o = bufs.heads(o, at(strides, 3), B, Tq, Hq, D, dtype, true);
    bufs.buffer(lse, (int64_t)B * Hq * Tq * 4, 4, true, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.lens = lens;
    p.lse = lse;
    return run(p, launch_attn_fwd, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_window_attn_bwd(const void *q, const void *k, const void *v, const void *o, const float *lse,
                                    const void *dout, const int32_t *lens, void *dq, void *dk, void *dv,
                                    const int64_t *strides, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left,
                                    int right, int sinks, int offset, float scale, int dtype, void *workspace,
                                    int64_t workspace_bytes, void *stream)
{
    AttnProblem p;
    const int st = make_attn(p, B, Tq, Tk, Hq, Hkv, D, left, right, sinks, offset, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, Tq, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, Tk, Hkv, D, dtype, false);
    p.v = bufs.heads(v, at(strides, 2), B, Tk, Hkv, D, dtype, false);
    p.o = bufs.heads(o, at(strides, 3), B, Tq, Hq, D, dtype, false);
    p.dout = bufs.heads(dout, at(strides, 4), B, Tq, Hq, D, dtype, false);
    bufs.buffer(lse, (int64_t)B * Hq * Tq * 4, 4, false);
    bufs.buffer(lens, (int64_t)B * 4, 4, false, true);
    p.dq = bufs.heads(dq, at(strides, 5), B, Tq, Hq, D, dtype, true);
    p.dk = bufs.heads(dk, at(strides, 6), B, Tk, Hkv, D, dtype, true);
    p.dv = bufs.heads(dv, at(strides, 7), B, Tk, Hkv, D, dtype, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.lens = lens;
    p.lse = const_cast<float *>(lse);
    return run(p, launch_attn_bwd, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_window_attn_decode(const void *q, const void *k, const void *v, const int32_t *lens, void *o,
                                       const int64_t *strides, int B, int Tq, int Tk, int Hq, int Hkv, int D, int left,
                                       int sinks, float scale, int dtype, void *workspace, int64_t workspace_bytes,
                                       void *stream)
{
    AttnProblem p;
    const int st = make_attn(p, B, Tq, Tk, Hq, Hkv, D, left, 0, sinks, 0, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    p.q = bufs.heads(q, at(strides, 0), B, Tq, Hq, D, dtype, false);
    p.k = bufs.heads(k, at(strides, 1), B, Tk, Hkv, D, dtype, false);
    p.v = bufs.heads(v, at(strides, 2), B, Tk, Hkv, D, dtype, false);
    bufs.buffer(lens, (int64_t)B * 4, 4, false, true);
    p.o = bufs.heads(o, at(strides, 3), B, Tq, Hq, D, dtype, true);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    p.lens = lens;
    p.tail = true;
    return run(p, launch_attn_split, bufs, workspace, workspace_bytes, stream);
}

extern "C" int gspn_delta_rule_reserve_size(int B, int T, int Hq, int Hv, int Dk, int Dv, int dtype, int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    DeltaProblem p;
    const int st = make_delta(p, B, T, Hq, Hv, Dk, Dv, 1.f, dtype);
    if (st == GSPN_OK)
        *bytes = delta_reserve(p);
    return st;
}

extern "C" int gspn_delta_rule_workspace_size(int op, int B, int T, int Hq, int Hv, int Dk, int Dv, int dtype,
                                              int64_t *bytes)
{
    if (bytes == nullptr)
        return GSPN_ERR_NULL;
    *bytes = 0;
    if (op != GSPN_DELTA_FWD && op != GSPN_DELTA_FWD_TRAIN && op != GSPN_DELTA_BWD_RESERVE)
        return GSPN_ERR_UNSUPPORTED;
    DeltaProblem p;
    const int st = make_delta(p, B, T, Hq, Hv, Dk, Dv, 1.f, dtype);
    if (st != GSPN_OK)
        return st;
    Workspace rs;
    rs.counting = true;
    if (op != GSPN_DELTA_FWD)
        p.rs = &rs;
    return count(p, op == GSPN_DELTA_BWD_RESERVE ? launch_delta_bwd : launch_delta_fwd, bytes);
}

extern "C" int gspn_delta_rule_fwd(const void *q, const void *k, const void *v, const void *g, const void *beta,
                                   const float *state, const int32_t *lens, void *o, float *state_out,
                                   const int64_t *strides, int B, int T, int Hq, int Hv, int Dk, int Dv, float scale,
                                   int dtype, void *workspace, int64_t workspace_bytes, void *stream)
{
    return delta_fwd(q, k, v, g, beta, state, lens, o, state_out, strides, B, T, Hq, Hv, Dk, Dv, scale, dtype, nullptr, 0,
                     false, workspace, workspace_bytes, stream);
}

extern "C" int gspn_delta_rule_fwd_train(const void *q, const void *k, const void *v, const void *g, const void *beta,
                                         const float *state, const int32_t *lens, void *o, float *state_out,
                                         const int64_t *strides, int B, int T, int Hq, int Hv, int Dk, int Dv, float scale,
                                         int dtype, void *reserve, int64_t reserve_bytes, void *workspace,
                                         int64_t workspace_bytes, void *stream)
{
    return delta_fwd(q, k, v, g, beta, state, lens, o, state_out, strides, B, T, Hq, Hv, Dk, Dv, scale, dtype, reserve,
                     reserve_bytes, true, workspace, workspace_bytes, stream);
}

extern "C" int gspn_delta_rule_bwd_reserve(const void *q, const void *k, const void *v, const void *g, const void *beta,
                                           const void *dout, const float *dstate_out, const int32_t *lens, void *dq,
                                           void *dk, void *dv, void *dg, void *dbeta, float *dstate, const int64_t *strides,
                                           int B, int T, int Hq, int Hv, int Dk, int Dv, float scale, int dtype,
                                           void *reserve, int64_t reserve_bytes, void *workspace, int64_t workspace_bytes,
                                           void *stream)
{
    DeltaProblem p;
    const int st = make_delta(p, B, T, Hq, Hv, Dk, Dv, scale, dtype);
    if (st != GSPN_OK)
        return st;
    Buffers bufs;
    delta_inputs(p, bufs, q, k, v, g, beta, lens, strides);
    const int64_t states = (int64_t)B * Hv * Dk * Dv * 4, gates = (int64_t)B * T * Hv * storage(dtype);
    p.dout = bufs.heads(dout, at(strides, 3), B, T, Hv, Dv, dtype, false);
    bufs.buffer(dstate_out, states, 16, false, true);
    p.dq = bufs.heads(dq, at(strides, 4), B, T, Hq, Dk, dtype, true);
    p.dk = bufs.heads(dk, at(strides, 5), B, T, Hq, Dk, dtype, true);
    p.dv = bufs.heads(dv, at(strides, 6), B, T, Hv, Dv, dtype, true);
    bufs.buffer(dg, gates, (int)storage(dtype), true);
    bufs.buffer(dbeta, gates, (int)storage(dtype), true);
    bufs.buffer(dstate, states, 16, true, true);
    p.dg = dg, p.dbeta = dbeta, p.dstate = dstate_out, p.dstate_in = dstate;
    const int64_t need = delta_reserve(p);
    if (bufs.status == GSPN_OK && (reserve == nullptr || reserve_bytes < need))
        return GSPN_ERR_WORKSPACE;
    bufs.buffer(reserve, need, 16, false);
    if (bufs.status != GSPN_OK)
        return bufs.status;
    Workspace rs;
    rs.base = static_cast<char *>(reserve);
    rs.size = (size_t)need;
    p.rs = &rs;
    return run(p, launch_delta_bwd, bufs, workspace, workspace_bytes, stream);
}
