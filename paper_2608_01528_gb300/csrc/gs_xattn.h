// gs_xattn.h -- cross attention: what its translation units share.
//
// Query rows are packed per key head: with G = Hq / Hkv query heads on key head hk, packed row
// r = l * G + g is query l of head hk * G + g, so that a tile of rows shares its keys and values
// across the group and the gradients of a shared key head sum over its rows by themselves.
#pragma once

#include "gs_internal.h"

namespace gs {

struct HeadView {  // element strides of b, l, h; the last axis is dense
    char* p;
    long long b, l, h;
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
    int vec;       // CUDA-core kernels: which arrays allow loads of four elements
    long long stats;  // backward: floats of the rows' statistics at the start of the workspace
};

// How many parts a kernel cuts its long axis into, so that about `want` blocks run: `base` blocks
// exist without a split, `tiles` is the axis' length in tiles, and a part has `least` tiles or more.
inline int xattn_parts(long long base, long long tiles, int want, int least) {
    if (base <= 0 || tiles <= 1 || base >= want) return 1;
    long long s = want / base;
    const long long most = tiles / least;
    if (s > most) s = most;
    return s < 1 ? 1 : (int)s;
}

// Workspace in floats; every section starts on a 16-byte boundary.
// Forward (splits > 1): per part and row dv sums, then the row's maximum (base 2) and sum.
// Backward: the rows' statistics (a.stats), then the parts of dQ (splits > 1), of dK and of dV (rsplits > 1).
#define GS_XWS __host__ __device__ inline long long
GS_XWS xattn_round4(long long n) { return (n + 3) / 4 * 4; }
GS_XWS xattn_rows(const XattnArgs& a) { return (long long)a.B * a.Hq * a.Lq; }
GS_XWS xattn_keys(const XattnArgs& a) { return (long long)a.B * a.Hkv * a.Lk; }
GS_XWS xattn_ws_ml(const XattnArgs& a) { return xattn_round4(a.splits * xattn_rows(a) * a.dv); }
GS_XWS xattn_ws_forward(const XattnArgs& a) { return a.splits > 1 ? xattn_ws_ml(a) + a.splits * xattn_rows(a) * 2 : 0; }
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

// ----------------------------------------------------------------- few rows (gs_xattn_rows.cu)
void xattn_rows_plan(XattnArgs& a, int sms);
cudaError_t launch_xattn_rows(const XattnArgs& a, cudaStream_t s);

// ----------------------------------------------------------------- CUDA cores (gs_xattn_simt.cu)
// the parts (splits, rsplits) that the CUDA-core kernels take on `sms` multiprocessors
void xattn_simt_plan(XattnArgs& a, bool backward, int sms);
cudaError_t launch_xattn_simt(const XattnArgs& a, cudaStream_t s);
cudaError_t launch_xattn_simt_backward(const XattnArgs& a, cudaStream_t s);
// O and lse from a.splits parts; dQ, dK, dV from theirs
cudaError_t launch_xattn_join(const XattnArgs& a, cudaStream_t s);
cudaError_t launch_xattn_join_dq(const XattnArgs& a, cudaStream_t s);
cudaError_t launch_xattn_join_dkv(const XattnArgs& a, cudaStream_t s);

// ----------------------------------------------------------------- tcgen05 (gs_xattn_tc.cu)
// bf16, at most 128 query heads to a key head, inputs on 16-byte boundaries with strides in multiples of 8
void xattn_tc_plan(XattnArgs& a, int sms);
cudaError_t launch_xattn_tc(const XattnArgs& a, int sms, int device, cudaStream_t s);
unsigned take_device_error_xattn();
// the gradient (gs_xattn_bwd_tc.cu)
void xattn_bwd_tc_plan(XattnArgs& a, int sms);
cudaError_t launch_xattn_bwd_tc(const XattnArgs& a, int device, cudaStream_t s);
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
