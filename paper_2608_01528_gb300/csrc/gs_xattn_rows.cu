// gs_xattn_rows.cu -- cross attention of a few query rows against a memory (a decoding step, a handful of panels) on CUDA
// cores: any type, width, alignment and stride.
//
// A block takes up to R packed rows of a key head; the keys go to its eight warps in batches.  LK lanes share a key, each
// holding 16 bytes of it: a key's dot products with the R rows (in registers) are summed across the LK lanes by
// shuffles, and the same lanes then add the weighted value -- K and V are read once, 16 bytes a lane, straight from memory, four keys of
// each in flight per lane.  Every LK lanes keep a running maximum, sum and output of their own; they meet in
// registers, then shared memory, and parts of long memories in k_xattn_join.
//
// Bound by memory with one row (64 sequences of 1,500 keys, 16 heads of 64), by instructions (about 12 per key, row and
// 16 bytes) with more.

#include <algorithm>

#include "gs_xattn_tc.cuh"

namespace gs {
namespace {

using xtc::ex2;
using xtc::kLn2;
using xtc::kLog2e;
using xtc::keys_of;

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kBatch = 4;  // keys in flight per LK lanes
constexpr int kVecQ = 1, kVecK = 2, kVecV = 4;

template <typename T>
struct Vec {
    static constexpr int N = 16 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ void get(float (&f)[N]) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
    // elements [0, left) of p, zeros behind them
    __device__ __forceinline__ void load(const T* p, int left, bool vec) {
        if (vec && left >= N) {
            raw = __ldg(reinterpret_cast<const uint4*>(p));
            return;
        }
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < left) {
                if constexpr (sizeof(T) == 4)
                    w[e] = __float_as_uint(__ldg(reinterpret_cast<const float*>(p) + e));
                else
                    w[e >> 1] |= (uint32_t)__ldg(reinterpret_cast<const unsigned short*>(p) + e) << (16 * (e & 1));
            }
        raw = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

template <typename T, int LK, int R>
__global__ void __launch_bounds__(kThreads, R == 1 ? 3 : 2) k_xattn_rows(const XattnArgs a, long long chunks) {
    using V = Vec<T>;
    constexpr int N = V::N, W = LK * N, KS = 32 / LK;
    __shared__ float acc_s[kWarps][R][W];
    __shared__ float2 ml_s[kWarps][R];
    long long i = blockIdx.x;
    const long long chunk = i % chunks;
    i /= chunks;
    const int part = (int)(i % a.splits);
    i /= a.splits;
    const int hk = (int)(i % a.Hkv), b = (int)(i / a.Hkv);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, slot = lane / LK, e0 = (lane % LK) * N;
    const int n = keys_of(a, b);
    const int k0 = (int)((long long)a.Lk * part / a.splits), k1 = min(n, (int)((long long)a.Lk * (part + 1) / a.splits));
    const float cs = a.scale * kLog2e;

    float q[R][N], acc[R][N], m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const long long pr = chunk * R + r;
        const bool has = pr < a.rows;
        const long long ql = has ? pr / a.G : 0;
        const int h = hk * a.G + (has ? (int)(pr - ql * a.G) : 0);
        V x;
        x.load(reinterpret_cast<const T*>(a.q.p) + b * a.q.b + ql * a.q.l + h * a.q.h + e0, has ? a.dk - e0 : 0, a.vec & kVecQ);
        x.get(q[r]);
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) acc[r][e] = 0.f;
    }
    const T* kp = reinterpret_cast<const T*>(a.k.p) + b * a.k.b + hk * a.k.h + e0;
    const T* vp = reinterpret_cast<const T*>(a.v.p) + b * a.v.b + hk * a.v.h + e0;
    const unsigned char* mask = a.mask ? a.mask + (long long)b * a.ldm : nullptr;
    for (int j0 = k0 + warp * (KS * kBatch); j0 < k1; j0 += kWarps * KS * kBatch) {
        V kx[kBatch], vx[kBatch];
        bool ok[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int j = j0 + u * KS + slot;
            ok[u] = j < k1 && (!mask || __ldg(mask + j) != 0);
            kx[u].load(kp + (ok[u] ? (long long)j * a.k.l : 0), ok[u] ? a.dk - e0 : 0, a.vec & kVecK);
            vx[u].load(vp + (ok[u] ? (long long)j * a.v.l : 0), ok[u] ? a.dv - e0 : 0, a.vec & kVecV);
        }
        float s[R][kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            float f[N];
            kx[u].get(f);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float d = 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e) d = fmaf(q[r][e], f[e], d);
                s[r][u] = d;
            }
        }
#pragma unroll
        for (int o = LK / 2; o; o >>= 1)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int u = 0; u < kBatch; ++u) s[r][u] += __shfl_xor_sync(0xffffffffu, s[r][u], o);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float mn = m[r];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                s[r][u] = ok[u] ? s[r][u] * cs : -INFINITY;
                mn = fmaxf(mn, s[r][u]);
            }
            const float ms = mn == -INFINITY ? 0.f : mn;
            const float f = ex2(m[r] - ms);
            m[r] = mn;
            l[r] *= f;
#pragma unroll
            for (int e = 0; e < N; ++e) acc[r][e] *= f;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                s[r][u] = ex2(s[r][u] - ms);
                l[r] += s[r][u];
            }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            float f[N];
            vx[u].get(f);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < N; ++e) acc[r][e] = fmaf(s[r][u], f[e], acc[r][e]);
        }
    }
    // the keys of a warp's lanes, then the warps
#pragma unroll
    for (int o = LK; o < 32; o <<= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float mo = __shfl_xor_sync(0xffffffffu, m[r], o), lo = __shfl_xor_sync(0xffffffffu, l[r], o);
            const float mn = fmaxf(m[r], mo), ms = mn == -INFINITY ? 0.f : mn;
            const float f = ex2(m[r] - ms), g = ex2(mo - ms);
            m[r] = mn;
            l[r] = l[r] * f + lo * g;
#pragma unroll
            for (int e = 0; e < N; ++e) acc[r][e] = acc[r][e] * f + __shfl_xor_sync(0xffffffffu, acc[r][e], o) * g;
        }
    if (slot == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int e = 0; e < N; ++e) acc_s[warp][r][e0 + e] = acc[r][e];
            if (lane == 0) ml_s[warp][r] = make_float2(m[r], l[r]);
        }
    }
    __syncthreads();
    const long long all = xattn_rows(a);
    for (int x = threadIdx.x; x < R * W; x += kThreads) {
        const int r = x / W, c = x % W;
        const long long pr = chunk * R + r;
        if (pr >= a.rows || (c >= a.dv && c != 0)) continue;
        float mm = -INFINITY, ll = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, ml_s[w][r].x);
        const float ms = mm == -INFINITY ? 0.f : mm;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 p = ml_s[w][r];
            const float f = ex2(p.x - ms);
            ll = fmaf(p.y, f, ll);
            o = fmaf(acc_s[w][r][c], f, o);
        }
        const long long ql = pr / a.G;
        const int h = hk * a.G + (int)(pr - ql * a.G);
        const long long at = ((long long)b * a.Hq + h) * a.Lq + ql;
        if (a.splits > 1) {
            a.ws[((long long)part * all + at) * a.dv + c] = o;
            if (c == 0) reinterpret_cast<float2*>(a.ws + xattn_ws_ml(a))[(long long)part * all + at] = make_float2(mm, ll);
        } else {
            const float v = ll == 0.f ? 0.f : o / ll;
            T* out = reinterpret_cast<T*>(a.o.p) + b * a.o.b + ql * a.o.l + h * a.o.h + c;
            if constexpr (sizeof(T) == 4)
                *out = v;
            else
                *out = __float2bfloat16_rn(v);
            if (c == 0 && a.lse) a.lse[at] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * kLn2;
        }
    }
}

int rows_per_block(long long rows) { return rows >= 4 ? 4 : rows >= 2 ? 2 : 1; }

template <typename T, int LK>
cudaError_t launch(const XattnArgs& a, cudaStream_t s) {
    const int R = rows_per_block(a.rows);
    const long long chunks = (a.rows + R - 1) / R;
    const unsigned grid = (unsigned)(chunks * a.splits * a.Hkv * a.B);
    if (R == 4)
        k_xattn_rows<T, LK, 4><<<grid, kThreads, 0, s>>>(a, chunks);
    else if (R == 2)
        k_xattn_rows<T, LK, 2><<<grid, kThreads, 0, s>>>(a, chunks);
    else
        k_xattn_rows<T, LK, 1><<<grid, kThreads, 0, s>>>(a, chunks);
    return cudaGetLastError();
}

bool on_16(const XattnArgs& a, const HeadView& v, int L, int H) {
    const int n = a.dtype == GS_F32 ? 4 : 8;
    return (uintptr_t)v.p % 16 == 0 && (a.B <= 1 || v.b % n == 0) && (L <= 1 || v.l % n == 0) && (H <= 1 || v.h % n == 0);
}

}  // namespace

void xattn_rows_plan(XattnArgs& a, int sms) {
    const int R = rows_per_block(a.rows);
    // four blocks a multiprocessor, and parts of 256 keys or more
    a.splits = xattn_parts((a.rows + R - 1) / R * a.Hkv * a.B, a.Lk / 256, 4 * sms, 1);
    a.rsplits = 1;
}

cudaError_t launch_xattn_rows(const XattnArgs& args, cudaStream_t s) {
    XattnArgs a = args;
    a.vec = (on_16(a, a.q, a.Lq, a.Hq) ? kVecQ : 0) | (on_16(a, a.k, a.Lk, a.Hkv) ? kVecK : 0) |
            (on_16(a, a.v, a.Lk, a.Hkv) ? kVecV : 0);
    const int w = std::max(a.dk, a.dv);
    cudaError_t e;
    if (a.dtype == GS_BF16)
        e = w <= 64 ? launch<__nv_bfloat16, 8>(a, s) : launch<__nv_bfloat16, 16>(a, s);
    else
        e = w <= 32 ? launch<float, 8>(a, s) : w <= 64 ? launch<float, 16>(a, s) : launch<float, 32>(a, s);
    if (e != cudaSuccess || a.splits == 1) return e;
    return launch_xattn_join(a, s);
}

}  // namespace gs
