// Argument checks shared by the C entry points of the token mixers and of the state
// space sublayer (host only, internal): a call's buffers, their alignment and overlap,
// its workspace.
#pragma once

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/gspn.h"
#include "attn.hpp"
#include "launch.hpp"

namespace gspn {

inline int64_t storage(int dtype) { return dtype == GSPN_F32 ? 4 : 2; }

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
inline Span flat(const void *p, int64_t bytes, bool output = false)
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
inline bool apart(const Span &a, const Span &b)
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
    Span all[32];
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
    // inplace: the index of a tensor that it may be, byte for byte; align: of its base
    // and strides, in bytes
    Heads heads(const void *p, const int64_t *s, int64_t B, int64_t T, int64_t H, int64_t D, int dtype, bool output,
                int inplace = -1, int64_t align = 16)
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
        if (reinterpret_cast<uintptr_t>(p) % align != 0 || h.sh * es % align != 0 || h.st * es % align != 0 ||
            h.sb * es % align != 0) {
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
    // a [B][T][C] tensor with strides s (batch, token), null: contiguous
    Heads rows(const void *p, const int64_t *s, int64_t B, int64_t T, int64_t C, int dtype, bool output, int inplace = -1)
    {
        const int64_t three[3] = {s ? s[0] : T * C, s ? s[1] : C, C};
        return heads(p, three, B, T, 1, C, dtype, output, inplace);
    }
};

template <typename P>
struct requires_reserve : std::false_type {};

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

}  // namespace gspn
