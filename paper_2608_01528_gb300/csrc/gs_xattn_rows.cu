// gs_xattn_rows.cu -- cross attention of a few query rows against a memory (a decoding step, a handful of panels) on CUDA
// cores: any type, width, alignment and stride.
//
// A block takes up to R packed rows of a key head; the keys go to its eight warps in batches.  LK lanes share a key, each
// holding 16 bytes of it: a key's dot products with the R rows (in registers) are summed across the LK lanes, and the same
// lanes then add the weighted value -- K and V are read once, 16 bytes a lane, straight from memory, four keys of
// each in flight per lane.  The sums of four keys and R rows go by halving: at each step a lane passes on half of its values
// and keeps the others', so that each lane ends with a logit of its own (15 shuffles for 16 of them instead of 64), takes its
// exponential, and the weights come back by shuffles.  Every LK lanes keep running maxima, sums and an output of their own;
// they meet in registers, then shared memory, and parts of long memories in k_xattn_join.
//
// One row is bound by the loads in flight (64 x 750 to 1,500 keys, 16 heads of 64, bf16: 4.7 TB/s; fp32 8 x 8,192 keys, 16
// heads of 128: 5.1 TB/s), more rows by instructions.

#include <algorithm>

#include "gs_xattn_tc.cuh"

namespace gs {
namespace {

using xtc::ex2;
using xtc::kLn2;
using xtc::kLog2e;
using xtc::keys_of;

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kBatch = 4;  // keys that LK lanes work on at a time
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
    // Two rows leave registers for the next four keys on their way as well (8 x 8,192 keys, 16 heads of 128, fp32: 209 -> 195 us);
    // one row does better with a third block a multiprocessor (242 against 297 us).
    constexpr bool kAhead = R == 2;
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

    // After the halving, lane x of a key's LK holds values x * kOwn .. + kOwn - 1 of row-major [R][kBatch] (kOwn values, or one
    // that kSame lanes share); m and l are those of that value's row.
    constexpr int kValues = R * kBatch, kOwn = kValues > LK ? kValues / LK : 1, kSame = kValues > LK ? 1 : LK / kValues;
    static_assert(kOwn <= kBatch, "a lane's values belong to one row");
    const int x = lane % LK, own = x * kOwn / kSame;
    float q[R][N], acc[R][N], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const long long pr = chunk * R + r;
        const bool has = pr < a.rows;
        const long long ql = has ? pr / a.G : 0;
        const int h = hk * a.G + (has ? (int)(pr - ql * a.G) : 0);
        V y;
        y.load(reinterpret_cast<const T*>(a.q.p) + b * a.q.b + ql * a.q.l + h * a.q.h + e0, has ? a.dk - e0 : 0, a.vec & kVecQ);
        y.get(q[r]);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[r][e] = 0.f;
    }
    const T* kp = reinterpret_cast<const T*>(a.k.p) + b * a.k.b + hk * a.k.h + e0;
    const T* vp = reinterpret_cast<const T*>(a.v.p) + b * a.v.b + hk * a.v.h + e0;
    const unsigned char* mask = a.mask ? a.mask + (long long)b * a.ldm : nullptr;
    V kx[kBatch], vx[kBatch], kn[kBatch], vn[kBatch];
    bool ok[kBatch], okn[kBatch];
    auto fetch = [&](int j0, V(&kk)[kBatch], V(&vv)[kBatch], bool(&o)[kBatch]) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int j = j0 + u * KS + slot;
            o[u] = j < k1 && (!mask || __ldg(mask + j) != 0);
            kk[u].load(kp + (o[u] ? (long long)j * a.k.l : 0), o[u] ? a.dk - e0 : 0, a.vec & kVecK);
            vv[u].load(vp + (o[u] ? (long long)j * a.v.l : 0), o[u] ? a.dv - e0 : 0, a.vec & kVecV);
        }
    };
    constexpr int kStep = kWarps * KS * kBatch;
    int j0 = k0 + warp * (KS * kBatch);
    if (kAhead && j0 < k1) fetch(j0, kn, vn, okn);
    for (; j0 < k1; j0 += kStep) {
        if constexpr (kAhead) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                kx[u] = kn[u];
                vx[u] = vn[u];
                ok[u] = okn[u];
            }
            if (j0 + kStep < k1) fetch(j0 + kStep, kn, vn, okn);
        } else {
            fetch(j0, kx, vx, ok);
        }
        float s[kValues];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            float f[N];
            kx[u].get(f);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float d = 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e) d = fmaf(q[r][e], f[e], d);
                s[r * kBatch + u] = d;
            }
        }
        // lanes with bit o keep the upper half of the values that are left, the others the lower
#pragma unroll
        for (int o = LK / 2, left = kValues; o; o >>= 1) {
            if (left > 1) {
                left /= 2;
                const bool up = (x & o) != 0;
#pragma unroll
                for (int i = 0; i < kValues / 2; ++i)
                    if (i < left) {
                        const float mine = up ? s[i + left] : s[i], other = up ? s[i] : s[i + left];
                        s[i] = mine + __shfl_xor_sync(0xffffffffu, other, o);
                    }
            } else {
                s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
            }
        }
        float mn = m;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int u = (own + i) % kBatch;
            bool in = ok[0];
#pragma unroll
            for (int k = 1; k < kBatch; ++k) in = u == k ? ok[k] : in;
            s[i] = in ? s[i] * cs : -INFINITY;
            mn = fmaxf(mn, s[i]);
        }
        // the row's maximum over the lanes that hold its other keys
#pragma unroll
        for (int o = kSame; o < kSame * kBatch / kOwn; o <<= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
        const float ms = mn == -INFINITY ? 0.f : mn;
        const float f = ex2(m - ms);
        if (__any_sync(0xffffffffu, f != 1.f)) {  // (NaN too)
            l *= f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float fr = __shfl_sync(0xffffffffu, f, r * (LK / R), LK);
#pragma unroll
                for (int e = 0; e < N; ++e) acc[r][e] *= fr;
            }
        }
        m = mn;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            s[i] = ex2(s[i] - ms);
            l += s[i];
        }
        float w[kValues];
#pragma unroll
        for (int i = 0; i < kValues; ++i) w[i] = __shfl_sync(0xffffffffu, s[i % kOwn], i / kOwn * kSame, LK);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            float f2[N];
            vx[u].get(f2);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < N; ++e) acc[r][e] = fmaf(w[r * kBatch + u], f2[e], acc[r][e]);
        }
    }
    // a row's sum over the lanes that hold its keys; then every lane has every row's maximum and sum
#pragma unroll
    for (int o = kSame; o < kSame * kBatch / kOwn; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    float mr[R], lr[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        mr[r] = __shfl_sync(0xffffffffu, m, r * (LK / R), LK);
        lr[r] = __shfl_sync(0xffffffffu, l, r * (LK / R), LK);
    }
    // the keys of a warp's lanes, then the warps
#pragma unroll
    for (int o = LK; o < 32; o <<= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float mo = __shfl_xor_sync(0xffffffffu, mr[r], o), lo = __shfl_xor_sync(0xffffffffu, lr[r], o);
            const float mn = fmaxf(mr[r], mo), ms = mn == -INFINITY ? 0.f : mn;
            const float f = ex2(mr[r] - ms), g = ex2(mo - ms);
            mr[r] = mn;
            lr[r] = lr[r] * f + lo * g;
#pragma unroll
            for (int e = 0; e < N; ++e) acc[r][e] = acc[r][e] * f + __shfl_xor_sync(0xffffffffu, acc[r][e], o) * g;
        }
    if (slot == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int e = 0; e < N; ++e) acc_s[warp][r][e0 + e] = acc[r][e];
            if (lane == 0) ml_s[warp][r] = make_float2(mr[r], lr[r]);
        }
    }
    __syncthreads();
    const long long all = xattn_rows(a);
    for (int e = threadIdx.x; e < R * W; e += kThreads) {
        const int r = e / W, c = e % W;
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
    // parts of 256 keys or more, up to four blocks a multiprocessor (three of one row or two of more are resident at a time)
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
