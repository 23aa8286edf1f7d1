// gs_xattn_simt.cu -- attention on CUDA cores over all keys, and what joins parts of any path.

#include "gs_xattn_simt.cuh"

namespace gs {
namespace {

// O and lse of the rows from their parts: one warp per row.
template <typename T>
__global__ void __launch_bounds__(256) k_xattn_join(const XattnArgs a) {
    const long long nrows = (long long)a.B * a.Hq * a.Lq;
    const long long at = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (at >= nrows) return;
    const float* ml = a.ws + xattn_ws_ml(a);
    float m = -INFINITY;
    for (int s = lane; s < a.splits; s += 32) m = fmaxf(m, ml[((long long)s * nrows + at) * 2]);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float ms = m == -INFINITY ? 0.f : m;
    float l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) {
        const float2 p = *reinterpret_cast<const float2*>(ml + ((long long)s * nrows + at) * 2);
        if (p.y == 0.f) continue;  // nothing in this part (NaN is not 0)
        const float f = exp2f(p.x - ms);
        l = fmaf(p.y, f, l);
        const float* po = a.ws + ((long long)s * nrows + at) * a.dv;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (lane + 32 * q < a.dv) acc[q] = fmaf(po[lane + 32 * q], f, acc[q]);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const long long i = at % a.Lq, bh = at / a.Lq;
    T* out = reinterpret_cast<T*>(a.o.p) + (bh / a.Hq) * a.o.b + i * a.o.l + (bh % a.Hq) * a.o.h;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (lane + 32 * q < a.dv) out[lane + 32 * q] = from_f32<T>(acc[q] * inv);
    if (lane == 0 && a.lse) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// out (B x L x H x w, of longer sequences perhaps) = mul * the sum, in order, of `parts` arrays (B, H, L, w): one, or dK and dV at once
struct Sum {
    const float* src;
    long long n;
    HeadView out;
    int w;
    float mul;
};
template <typename T>
__global__ void __launch_bounds__(256) k_xattn_sum(const Sum first, const Sum second, int parts, int H, int L) {
    const Sum& x = blockIdx.y ? second : first;
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < x.n; e += (long long)gridDim.x * 256) {
        float v = 0.f;
        for (int s = 0; s < parts; ++s) v += x.src[(long long)s * x.n + e];
        const int c = (int)(e % x.w);
        const long long at = e / x.w, l = at % L, bh = at / L;
        (reinterpret_cast<T*>(x.out.p) + (bh / H) * x.out.b + l * x.out.l + (bh % H) * x.out.h)[c] = from_f32<T>(v * x.mul);
    }
}

unsigned sum_grid(long long n) { return (unsigned)std::min<long long>((n + 255) / 256, 152 * 16); }

}  // namespace

void xattn_simt_plan(XattnArgs& a, bool backward, int sms, KeyMode mode) {
    const int R = backward ? bwd_rows(a) : kTile;
    const long long rt = (a.rows + R - 1) / R, kt = (a.Lk + kTile - 1) / kTile;
    long long keys = kt, rows = rt;  // tiles that one of the other kind meets
    if (mode == kWindowKeys) {
        const long long w = a.win.window, k = w + a.win.sinks + R / a.G;
        keys = std::min(kt, k / kTile + 2);
        if (a.win.sinks == 0) rows = std::min(rt, (w + kTile) * a.G / R + 2);
    }
    // up to four blocks a multiprocessor, and parts of two tiles or more
    long long base = rt, kbase = kt;
    if (mode == kWindowKeys && backward) base = kbase = rt + kt;  // (one launch; 160 blocks of keys and 288 of rows leave nothing to sum)
    a.splits = xattn_parts(base * a.Hkv * a.B, keys, 4 * sms, 2);
    a.rsplits = backward ? xattn_parts(kbase * a.Hkv * a.B, rows, 4 * sms, 2) : 1;
    a.pkeys = a.Lk;
    if (backward && mode == kWindowKeys && a.win.sinks > 0 && a.rsplits == 1) {
        const long long some = std::min(rt, ((long long)a.win.window + kTile) * a.G / R + 1);
        a.rsplits = xattn_sink_parts(kt * a.Hkv * a.B, rt, some, rt * keys * a.Hkv * a.B, 2 * sms);
        if (a.rsplits > 1) a.pkeys = (int)std::min<long long>(a.Lk, (a.win.sinks + kTile - 1ll) / kTile * kTile);
    }
    if (rt == 0) a.splits = 1;   // (nothing to cut, and no sums to launch, although the other axis alone may ask for parts)
    if (kt == 0) a.rsplits = 1;
    a.stats = xattn_round4(xattn_rows(a));  // D_i
}

cudaError_t launch_xattn_simt(const XattnArgs& a, KeyMode mode, cudaStream_t s) {
    const cudaError_t e = mode == kWindowKeys ? launch_xattn_simt_window(a, s) : forward_all<false>(a, s);
    if (e != cudaSuccess || a.splits == 1) return e;
    return launch_xattn_join(a, s);
}

cudaError_t launch_xattn_simt_backward(const XattnArgs& a, KeyMode mode, cudaStream_t s) {
    return mode == kWindowKeys ? launch_xattn_simt_window_backward(a, s) : backward_all<false>(a, s);
}

cudaError_t launch_xattn_join(const XattnArgs& a, cudaStream_t s) {
    const long long rows = (long long)a.B * a.Hq * a.Lq;
    if (a.dtype == GS_F32)
        k_xattn_join<float><<<(unsigned)((rows + 7) / 8), 256, 0, s>>>(a);
    else
        k_xattn_join<__nv_bfloat16><<<(unsigned)((rows + 7) / 8), 256, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_xattn_join_dq(const XattnArgs& a, cudaStream_t s) {
    const Sum q{a.ws + xattn_ws_dq(a), (long long)a.B * a.Hq * a.Lq * a.dk, a.dQ, a.dk, a.scale};
    if (a.dtype == GS_F32)
        k_xattn_sum<float><<<sum_grid(q.n), 256, 0, s>>>(q, q, a.splits, a.Hq, a.Lq);
    else
        k_xattn_sum<__nv_bfloat16><<<sum_grid(q.n), 256, 0, s>>>(q, q, a.splits, a.Hq, a.Lq);
    return cudaGetLastError();
}

cudaError_t launch_xattn_join_dkv(const XattnArgs& a, cudaStream_t s) {
    const long long rows = xattn_keys(a);
    const Sum k{a.ws + xattn_ws_dk(a), rows * a.dk, a.dK, a.dk, a.scale}, v{a.ws + xattn_ws_dv(a), rows * a.dv, a.dV, a.dv, 1.f};
    const dim3 grid(sum_grid(std::max(k.n, v.n)), 2);
    if (a.dtype == GS_F32)
        k_xattn_sum<float><<<grid, 256, 0, s>>>(k, v, a.rsplits, a.Hkv, a.pkeys);
    else
        k_xattn_sum<__nv_bfloat16><<<grid, 256, 0, s>>>(k, v, a.rsplits, a.Hkv, a.pkeys);
    return cudaGetLastError();
}

}  // namespace gs
