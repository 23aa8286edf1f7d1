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
