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

// Workspace in floats.  Forward: per part and row dv sums, the row's maximum (base 2) and sum.
// Backward: D_i per row, then the parts of dQ (splits > 1) and of dK, dV (rsplits > 1).
inline long long xattn_ws_forward(const XattnArgs& a) {
    return a.splits > 1 ? (long long)a.splits * a.B * a.Hq * a.Lq * (a.dv + 2) : 0;
}
__host__ __device__ inline long long xattn_ws_delta(const XattnArgs& a) { return ((long long)a.B * a.Hq * a.Lq + 3) / 4 * 4; }
inline long long xattn_ws_backward(const XattnArgs& a) {
    long long n = xattn_ws_delta(a);
    if (a.splits > 1) n += (long long)a.splits * a.B * a.Hq * a.Lq * a.dk;
    if (a.rsplits > 1) n += (long long)a.rsplits * a.B * a.Hkv * a.Lk * (a.dk + a.dv);
    return n;
}

// ----------------------------------------------------------------- CUDA cores (gs_xattn_simt.cu)
// the parts (splits, rsplits) that the CUDA-core kernels take on `sms` multiprocessors
void xattn_simt_plan(XattnArgs& a, bool backward, int sms);
cudaError_t launch_xattn_simt(const XattnArgs& a, cudaStream_t s);
cudaError_t launch_xattn_simt_backward(const XattnArgs& a, cudaStream_t s);
// D_i = <dO_i, O_i> into ws
cudaError_t launch_xattn_delta(const XattnArgs& a, cudaStream_t s);
// O and lse from a.splits parts; dQ, dK, dV from theirs
cudaError_t launch_xattn_join(const XattnArgs& a, cudaStream_t s);
cudaError_t launch_xattn_join_dq(const XattnArgs& a, cudaStream_t s);
cudaError_t launch_xattn_join_dkv(const XattnArgs& a, cudaStream_t s);

// ----------------------------------------------------------------- tcgen05 (gs_xattn_tc.cu)
// bf16, at most 128 query heads to a key head, Q, K, V on 16-byte boundaries with strides in multiples of 8
bool xattn_tc_supported(const XattnArgs& a);
void xattn_tc_plan(XattnArgs& a, int sms);
cudaError_t launch_xattn_tc(const XattnArgs& a, int sms, int device, cudaStream_t s);
unsigned take_device_error_xattn();

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
cudaError_t launch_sample(const SampleArgs& a, int sms, cudaStream_t s);

}  // namespace gs
