// gs_xattn.h -- cross attention: what its translation units share.
//
// Query rows are packed per key head: with G = Hq / Hkv query heads on key head hk, packed row
// r = l * G + g is query l of head hk * G + g, so that a tile of rows shares its keys and values
// across the group and the gradients of a shared key head sum over its rows by themselves.
#pragma once

#include <algorithm>

#include "gs_internal.h"

namespace gs {

struct HeadView {  // element strides of b, l, h; the last axis is dense
    char* p;
    long long b, l, h;
};

// A sliding window: row l of sequence b stands at position start + l and reads the keys up to itself, the last `window` of them
// (kNoWindow: all) and the first `sinks`.
constexpr int kNoWindow = 0x7fffffff;
struct KeyWindow {
    int window, sinks, start;
    const int* starts;  // one per sequence, or NULL: start
};
// Keys and values in pages (the views' b is then the page, l the row in it); the last of a sequence's query rows is its last key.
struct KeyPages {
    int pages, page, cols, shift;  // page = 1 << shift, or shift < 0
    const int* table;              // B x cols
    long long ldt;
    const int* qlens;  // query rows of each sequence, or NULL: Lq
};

struct XattnArgs {
    int dtype, B, Lq, Lk, Hq, Hkv, G, dk, dv;
    long long rows;  // Lq * G packed rows per (b, key head)
    float scale;
    const int* lens;
    const unsigned char* mask;
    long long ldm;
    HeadView q, k, v, o, dO, dQ, dK, dV;
    float* lse;    // B x Hq x Lq (forward: optional output; backward: input)
    float* ws;     // workspace
    int splits;    // forward, dQ: parts of the key axis
    int rsplits;   // dK / dV: parts of the packed rows
    int pkeys;     // .. of the keys before this one (Lk, or a whole number of tiles): the others' rows are one part
    int vec;       // CUDA-core kernels: which arrays allow loads of four elements
    long long stats;  // backward: floats of the rows' statistics at the start of the workspace
    bool flags;       // forward on tcgen05 through a window: a byte a row in the workspace
    KeyWindow win;
    KeyPages pg;
};

// What a kernel reads the keys through.
enum KeyMode { kAllKeys = 0, kWindowKeys = 1, kPagedKeys = 2 };

// Keys [0, sink) and [lo, hi), sink <= lo: all that a row, or some row of several, sees (before lengths and masks of keys).
struct KeySpan {
    int sink, lo, hi;
    __device__ __forceinline__ int count() const { return sink + hi - lo; }
    __device__ __forceinline__ int key(int i) const { return i < sink ? i : i - sink + lo; }  // the i-th
};
// of the rows l0..l1 of sequence b with n keys (l0 <= l1)
template <int MODE>
static __device__ __forceinline__ KeySpan key_span(const XattnArgs& a, int b, long long l0, long long l1, int n) {
    KeySpan s;
    if constexpr (MODE == kAllKeys) {
        s.sink = s.lo = 0;
        s.hi = n;
    } else {
        long long p0 = l0, p1 = l1;
        if constexpr (MODE == kPagedKeys) {
            const int m = a.pg.qlens ? min(max(__ldg(a.pg.qlens + b), 0), a.Lq) : a.Lq;
            p1 = l0 < m ? (l1 < m ? l1 : m - 1) : m - 1 - (long long)n;  // (no row: a position before the first key)
            p0 += (long long)n - m;
            p1 += (long long)n - m;
        } else {
            const long long first = a.win.starts ? __ldg(a.win.starts + b) : a.win.start;
            p0 += first;
            p1 += first;
        }
        s.hi = (int)(p1 + 1 < 0 ? 0 : p1 + 1 < n ? p1 + 1 : n);
        const long long lo = a.win.window == kNoWindow ? 0 : p0 - a.win.window + 1;
        s.lo = (int)(lo < 0 ? 0 : lo < s.hi ? lo : s.hi);
        s.sink = a.win.sinks < s.lo ? a.win.sinks : s.lo;
    }
    return s;
}
static __device__ __forceinline__ uint32_t bits_below(int x) { return x >= 32 ? 0xffffffffu : x <= 0 ? 0u : (1u << x) - 1u; }
static __device__ __forceinline__ uint32_t bits_between(int c0, int c1) { return bits_below(c1) & ~bits_below(c0); }
// bit i: key j + i is one of the span's
static __device__ __forceinline__ uint32_t seen_word(const KeySpan& s, int j) {
    return bits_between(s.lo - j, s.hi - j) | bits_below(s.sink - j);
}

// How many parts a kernel cuts its long axis into, so that about `want` blocks run: `base` blocks
// exist without a split, `tiles` is the axis' length in tiles, and a part has `least` tiles or more.
inline int xattn_parts(long long base, long long tiles, int want, int least) {
    if (base <= 0 || tiles <= 1 || base >= want) return 1;
    long long s = want / base;
    const long long most = tiles / least;
    if (s > most) s = most;
    return s < 1 ? 1 : (int)s;
}

// Parts of the rows for the key tiles that sinks show to every row, where all tiles are in one part so far (`base` of them, with all
// heads and sequences): such a tile meets `rows` row tiles, others about `typical`, and is the last to end where that is more than a slot
// (there are `slots`; `more` steps besides) has in all.
inline int xattn_sink_parts(long long base, long long rows, long long typical, long long more, long long slots) {
    const long long share = std::max(typical, (base * typical + more) / std::max(slots, 1ll));
    if (4 * rows <= 5 * share) return 1;
    return (int)std::min({16ll, (rows + share - 1) / share, std::max(1ll, rows / 2)});
}

// Workspace in floats; every section starts on a 16-byte boundary.
// Forward (splits > 1): per part and row dv sums, then the row's maximum (base 2) and sum.
// Backward: the rows' statistics (a.stats), then the parts of dQ (splits > 1), of dK and of dV (rsplits > 1).
#define GS_XWS __host__ __device__ inline long long
GS_XWS xattn_round4(long long n) { return (n + 3) / 4 * 4; }
GS_XWS xattn_rows(const XattnArgs& a) { return (long long)a.B * a.Hq * a.Lq; }
GS_XWS xattn_keys(const XattnArgs& a) { return (long long)a.B * a.Hkv * a.pkeys; }  // in parts
GS_XWS xattn_ws_ml(const XattnArgs& a) { return xattn_round4(a.splits * xattn_rows(a) * a.dv); }
GS_XWS xattn_ws_forward(const XattnArgs& a) {
    return a.splits > 1 ? xattn_ws_ml(a) + a.splits * xattn_rows(a) * 2 : a.flags ? xattn_round4((xattn_rows(a) + 3) / 4) : 0;
}
GS_XWS xattn_ws_dq(const XattnArgs& a) { return a.stats; }
GS_XWS xattn_ws_dk(const XattnArgs& a) {
    return xattn_ws_dq(a) + (a.splits > 1 ? xattn_round4(a.splits * xattn_rows(a) * a.dk) : 0);
}
GS_XWS xattn_ws_dv(const XattnArgs& a) {
    return xattn_ws_dk(a) + (a.rsplits > 1 ? xattn_round4(a.rsplits * xattn_keys(a) * a.dk) : 0);
}
GS_XWS xattn_ws_backward(const XattnArgs& a) {
    return xattn_ws_dv(a) + (a.rsplits > 1 ? a.rsplits * xattn_keys(a) * a.dv : 0);
}
#undef GS_XWS

// The keys of [j0, j1) that sequence b may read under its mask, where they are kFewKeys or fewer: lane i of the warp gets the
// i-th in `mine`, the result is their number; -1 where there are more (found within the first keys, unless the mask is nearly empty).
// D of the gradient is then summed from P and dP: a bf16 O gives <dO, O> to 2^-8 of the sum of |dO O|, which with weights on
// one of a few keys passes what dP - D is rounded to (error of dQ and dK, logits of standard deviation 1.5 / 4, from a bf16 O:
// 2 keys 3.4e-3 / 6.4e-3 of their norm, 16 keys 1.3e-3 / 3.5e-3, 1,024 keys 4e-4 / 2.3e-3; dS in bf16: 1.7e-3).
constexpr int kFewKeys = 16;
static __device__ __forceinline__ int few_keys(const XattnArgs& a, int b, int j0, int j1, int& mine) {
    constexpr int kAhead = 16;  // masks of 32 keys on their way
    const int lane = threadIdx.x & 31;
    const unsigned char* mask = a.mask + (long long)b * a.ldm;
    int found = 0;
    for (; j0 < j1; j0 += 32 * kAhead) {
        unsigned char m[kAhead];
        unsigned any = 0;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int j = j0 + 32 * u + lane;
            m[u] = j < j1 ? __ldg(mask + j) : 0;
            any |= m[u];
        }
        if (!__any_sync(0xffffffffu, any)) continue;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            unsigned w = __ballot_sync(0xffffffffu, m[u] != 0);
            if (found + __popc(w) > kFewKeys) return -1;
            for (; w; w &= w - 1, ++found)
                if (lane == found) mine = j0 + 32 * u + __ffs(w) - 1;
        }
    }
    return found;
}

// The same of what one row sees through a window (span), whether a mask thins it out or not: LANES neighbouring lanes work on a
// row of their own, in step with the warp's others; the i-th key is lane i % LANES's `mine` where i < LANES.
template <int LANES>
static __device__ __forceinline__ int few_seen(const XattnArgs& a, int b, const KeySpan& span, int& mine) {
    static_assert(LANES >= kFewKeys, "a key a lane");
    const int lane = threadIdx.x & (LANES - 1), shift = (threadIdx.x & 31) & ~(LANES - 1);
    const unsigned all = LANES == 32 ? 0xffffffffu : (1u << (LANES & 31)) - 1u;
    const unsigned char* mask = a.mask ? a.mask + (long long)b * a.ldm : nullptr;
    const int count = span.count();
    int found = 0;
    bool done = count == 0 || (!mask && count > kFewKeys);
    if (done && count) found = -1;
    for (int i0 = 0; __any_sync(0xffffffffu, !done); i0 += LANES) {
        const int i = i0 + lane, j = span.key(i);
        const bool in = !done && i < count && (!mask || __ldg(mask + j) != 0);
        unsigned w = __ballot_sync(0xffffffffu, in) >> shift & all;
        if (!done) {
            if (found + __popc(w) > kFewKeys) {
                found = -1;
                done = true;
            } else {
                for (; w; w &= w - 1, ++found)
                    if (lane == found) mine = span.key(i0 + __ffs(w) - 1);
                done = i0 + LANES >= count;
            }
        }
    }
    return found;
}

// Query rows [first, end) of sequence b that see some of the keys [j0, j1).
struct RowSpan {
    long long first, end;
};
static __device__ __forceinline__ RowSpan row_span(const XattnArgs& a, int b, int j0, int j1) {
    const long long start = a.win.starts ? __ldg(a.win.starts + b) : a.win.start;
    RowSpan r;
    r.first = min(max(j0 - start, 0ll), (long long)a.Lq);
    r.end = j0 < a.win.sinks || a.win.window == kNoWindow ? a.Lq : min(max(j1 - 1 + (long long)a.win.window - start, r.first), (long long)a.Lq);
    if (j1 <= j0) r.end = r.first;
    return r;
}

// ----------------------------------------------------------------- few rows (gs_xattn_rows.cu)
void xattn_rows_plan(XattnArgs& a, int sms, KeyMode mode);
cudaError_t launch_xattn_rows(const XattnArgs& a, KeyMode mode, cudaStream_t s);

// ----------------------------------------------------------------- CUDA cores (gs_xattn_simt.cu)
// the parts (splits, rsplits) that the CUDA-core kernels take on `sms` multiprocessors
void xattn_simt_plan(XattnArgs& a, bool backward, int sms, KeyMode mode);
cudaError_t launch_xattn_simt(const XattnArgs& a, KeyMode mode, cudaStream_t s);
cudaError_t launch_xattn_simt_backward(const XattnArgs& a, KeyMode mode, cudaStream_t s);
cudaError_t launch_xattn_simt_window(const XattnArgs& a, cudaStream_t s);  // (gs_xattn_simt_window.cu, without the join)
cudaError_t launch_xattn_simt_window_backward(const XattnArgs& a, cudaStream_t s);
// O and lse from a.splits parts; dQ, dK, dV from theirs
cudaError_t launch_xattn_join(const XattnArgs& a, cudaStream_t s);
cudaError_t launch_xattn_join_dq(const XattnArgs& a, cudaStream_t s);
cudaError_t launch_xattn_join_dkv(const XattnArgs& a, cudaStream_t s);

// ----------------------------------------------------------------- tcgen05 (gs_xattn_tc.cu)
// bf16, at most 128 query heads to a key head, inputs on 16-byte boundaries with strides in multiples of 8
void xattn_tc_plan(XattnArgs& a, KeyMode mode, int sms);
cudaError_t launch_xattn_tc(const XattnArgs& a, KeyMode mode, int sms, int device, cudaStream_t s);
unsigned take_device_error_xattn();
// the gradient (gs_xattn_bwd_tc.cu)
void xattn_bwd_tc_plan(XattnArgs& a, KeyMode mode, int sms);
cudaError_t launch_xattn_bwd_tc(const XattnArgs& a, KeyMode mode, int device, cudaStream_t s);
unsigned take_device_error_xbwd();

// ----------------------------------------------------------------- odd widths for the tensor cores (gs_xattn_pack.cu)
enum { kPackQ = 1, kPackK = 2, kPackV = 4, kPackDO = 8 };
// whether inputs may be laid out again for this call; which arrays the workspace has room for (by their widths); which a
// tensor map cannot describe as they lie
bool xattn_packs(const XattnArgs& a, bool backward, bool forced);
int xattn_pack_room(const XattnArgs& a, bool backward);
int xattn_pack_need(const XattnArgs& a, bool backward);
long long xattn_ws_pack(const XattnArgs& a, int which);  // floats
// copies the arrays `which` to `room` and turns a's views to them
cudaError_t launch_xattn_pack(XattnArgs& a, int which, float* room, cudaStream_t s);

// ----------------------------------------------------------------- sampling (gs_sample.cu)
struct SampleArgs {
    const void* S;
    bool bf16;
    long long N, lds;
    int M;
    gs_sampling how;
    const float* U;
    int* index;
    float* prob;
};
cudaError_t launch_sample(const SampleArgs& a, int sms, int device, cudaStream_t s);

}  // namespace gs
