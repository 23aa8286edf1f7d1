// gs_xattn_simt.cuh -- attention and its gradient on fp32 CUDA cores, over all keys or through a window: every type, width
// (1 to 128), alignment and stride that the calls take.
//
// Forward, one pass over the keys with the running maximum m and sum l of each row (base-2 units,
// c = scale log2 e):  m' = max(m, max_j c s_j),  l = l 2^(m - m') + sum_j 2^(c s_j - m'),
// O = O 2^(m - m') + sum_j 2^(c s_j - m') v_j;  at the end O / l and lse = (m + log2 l) ln 2.
// A block of 256 threads holds 64 packed rows; per tile of 64 keys each thread has a 4 x 4 piece of S and
// 4 rows x dv / 16 columns of O in registers, Q, K, V and the weights (over K) in shared memory, rows
// padded by 4 floats so that 16-byte reads of 8 consecutive rows take 8 different bank groups.  Bound by
// the shared-memory reads that feed the FMAs (8 16-byte reads per 64 FMAs; fp32, 16 x 64 x 2,048, 4 heads of 64: 89 us,
// 24 TFLOP/s; 8 x 1,024 x 1,500, 16 heads of 64: 1.62 ms, 31 TFLOP/s).  With few blocks the keys are cut into parts whose (O, m, l) a second kernel joins.
//
// Backward, with the forward's lse: P = 2^(c s - lse log2 e), dS = P (dO V^T - D).  One kernel per row
// tile runs over the keys for dQ, one per key tile over the packed rows for dK and dV (S is
// computed twice; no sums meet in atomics, so results repeat bit for bit): 16 x 100 x 129 to 257, 4 / 2 heads of 40 and 30,
// fp32: 70 us in a graph, 82 us as calls (up to six launches: D, dQ and its sum, dK and dV and theirs); 8 x 1,024 x 1,500, 16 heads
// of 64: 6.3 ms, 20 TFLOP/s.

#pragma once

#include <math.h>

#include <algorithm>

#include "gs_xattn.h"

namespace gs {
namespace {

constexpr int kTile = 64;      // rows and keys of a tile
constexpr int kThreads = 256;  // 16 x 16, a 4 x 4 piece of the tile each
constexpr int kPP = kTile + 4; // pitch of a tile of weights
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// bits of XattnArgs::vec: the array's rows start on boundaries of four elements
constexpr int kVecQ = 1, kVecK = 2, kVecV = 4, kVecDO = 8, kVecO = 16;

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) {
    return v;
}
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) {
    return __bfloat162float(v);
}
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) {
    return v;
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) {
    return __float2bfloat16_rn(v);
}

__device__ __forceinline__ int keys_of(const XattnArgs& a, int b) {
    return a.lens ? min(max(a.lens[b], 0), a.Lk) : a.Lk;
}

// Address of packed row r of (b, key head hk) in a query-side array.
template <typename T>
__device__ __forceinline__ T* row_at(const XattnArgs& a, const HeadView& v, int b, int hk, long long r) {
    const int l = (int)((unsigned)r / (unsigned)a.G), g = (int)r - l * a.G;  // (rows are fewer than 2^31)
    return reinterpret_cast<T*>(v.p) + b * v.b + l * v.l + (long long)(hk * a.G + g) * v.h;
}
// Index of packed row r in the (B, Hq, Lq) arrays.
__device__ __forceinline__ long long row_index(const XattnArgs& a, int b, int hk, long long r) {
    const int l = (int)((unsigned)r / (unsigned)a.G), g = (int)r - l * a.G;  // (rows are fewer than 2^31)
    return ((long long)b * a.Hq + hk * a.G + g) * a.Lq + l;
}

// Four elements from p (zeros from the w-th on), as one load where the array allows it (vec) and all are there.
__device__ __forceinline__ float4 load4(const float* p, int left, bool vec) {
    if (vec && left >= 4) return __ldg(reinterpret_cast<const float4*>(p));
    return make_float4(left > 0 ? p[0] : 0.f, left > 1 ? p[1] : 0.f, left > 2 ? p[2] : 0.f, left > 3 ? p[3] : 0.f);
}
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p, int left, bool vec) {
    if (vec && left >= 4) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                           __uint_as_float(v.y & 0xffff0000u));
    }
    return make_float4(left > 0 ? to_f32(p[0]) : 0.f, left > 1 ? to_f32(p[1]) : 0.f, left > 2 ? to_f32(p[2]) : 0.f,
                       left > 3 ? to_f32(p[3]) : 0.f);
}
// R packed rows from r0, D floats each (zero past the width w and past the last row): four threads a row, so that a row's
// address is worked out once.
template <typename T, int D, int R = kTile>
__device__ __forceinline__ void load_rows(float* dst, const XattnArgs& a, const HeadView& v, int b, int hk,
                                          long long r0, int w, bool vec) {
    const int i = threadIdx.x >> 2, c0 = (threadIdx.x & 3) * 4;
    if (i >= R) return;
    const bool has = r0 + i < a.rows;
    const T* p = row_at<T>(a, v, b, hk, has ? r0 + i : 0);
#pragma unroll
    for (int c = 0; c < D; c += 16)
        *reinterpret_cast<float4*>(dst + i * (D + 4) + c + c0) = load4(p + c + c0, has ? w - c - c0 : 0, vec);
}
// Whether key j0 + threadIdx.x / 4 is read, also in ok[] for the others.
// (WIN: of those that `seen`, the keys of the tile's rows, has)
template <bool WIN>
__device__ __forceinline__ bool load_valid(int* ok, const XattnArgs& a, int b, int j0, int n, const KeySpan& seen) {
    const int i = threadIdx.x >> 2, j = j0 + i;
    bool in = j < n;
    if constexpr (WIN) in = in && j < seen.hi && (j >= seen.lo || j < seen.sink);
    if (in && a.mask) in = a.mask[b * a.ldm + j] != 0;
    if ((threadIdx.x & 3) == 0) ok[i] = in;
    return in;
}
// This thread's part of 64 keys and values from j0, four threads a key (zero where it is not read): all on their way before the first
// goes to shared memory.  True where an entry of V is not finite.
template <typename T, int DK, int DV>
__device__ __forceinline__ bool load_keys(float* Ks, float* Vs, const XattnArgs& a, int b, int hk, int j0, bool has) {
    const int i = threadIdx.x >> 2, c0 = (threadIdx.x & 3) * 4;
    const long long j = has ? j0 + i : 0;
    const T *k = reinterpret_cast<const T*>(a.k.p) + b * a.k.b + hk * a.k.h + j * a.k.l;
    const T *v = reinterpret_cast<const T*>(a.v.p) + b * a.v.b + hk * a.v.h + j * a.v.l;
    float4 x[DK / 16], y[DV / 16];
#pragma unroll
    for (int c = 0; c < DK / 16; ++c) x[c] = load4(k + 16 * c + c0, has ? a.dk - 16 * c - c0 : 0, a.vec & kVecK);
#pragma unroll
    for (int c = 0; c < DV / 16; ++c) y[c] = load4(v + 16 * c + c0, has ? a.dv - 16 * c - c0 : 0, a.vec & kVecV);
    float odd = 0.f;  // NaN as soon as an entry is an infinity or a NaN
#pragma unroll
    for (int c = 0; c < DK / 16; ++c) *reinterpret_cast<float4*>(Ks + i * (DK + 4) + 16 * c + c0) = x[c];
#pragma unroll
    for (int c = 0; c < DV / 16; ++c) {
        odd = fmaf(y[c].x, 0.f, fmaf(y[c].y, 0.f, fmaf(y[c].z, 0.f, fmaf(y[c].w, 0.f, odd))));
        *reinterpret_cast<float4*>(Vs + i * (DV + 4) + 16 * c + c0) = y[c];
    }
    return odd != 0.f;
}

// acc[i][j] += <A row ty + 16 i, B row tx + 16 j>
template <int D, int RI>
__device__ __forceinline__ void dots(float (&acc)[RI][4], const float* A, const float* B, int w) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 4
    for (int d = 0; d < w; d += 4) {
        float4 x[RI], y[4];
#pragma unroll
        for (int i = 0; i < RI; ++i) x[i] = *reinterpret_cast<const float4*>(A + (ty + 16 * i) * (D + 4) + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(B + (tx + 16 * j) * (D + 4) + d);
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[i][j] = fmaf(x[i].x, y[j].x, acc[i][j]);
                acc[i][j] = fmaf(x[i].y, y[j].y, acc[i][j]);
                acc[i][j] = fmaf(x[i].z, y[j].z, acc[i][j]);
                acc[i][j] = fmaf(x[i].w, y[j].w, acc[i][j]);
            }
    }
}
// Column of a row of D that a thread's q-th sum belongs to: four (D = 32: two) neighbouring ones every 64.
template <int D>
__device__ __forceinline__ int column(int q) {
    const int tx = threadIdx.x & 15;
    return D == 32 ? 2 * tx + q : 64 * (q / 4) + 4 * tx + q % 4;
}
// out[i][q] += sum_k W[ty + 16 i][k] X[k][column(q)] over a tile of K
// (OWN: a zero weight keeps out whatever X holds there, for tiles whose rows see different keys that are not all finite)
template <int D, int K = kTile, bool OWN = false, int RI>
__device__ __forceinline__ void weigh(float (&out)[RI][D / 16], const float* W, const float* X) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 2
    for (int k = 0; k < K; k += 4) {
        float4 w[RI];
#pragma unroll
        for (int i = 0; i < RI; ++i) w[i] = *reinterpret_cast<const float4*>(W + (ty + 16 * i) * (K + 4) + k);
        if constexpr (D == 32) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float2 x = *reinterpret_cast<const float2*>(X + (k + q) * (D + 4) + 2 * tx);
#pragma unroll
                for (int i = 0; i < RI; ++i) {
                    const float p = q == 0 ? w[i].x : q == 1 ? w[i].y : q == 2 ? w[i].z : w[i].w;
                    if (OWN && p == 0.f) continue;
                    out[i][0] = fmaf(p, x.x, out[i][0]);
                    out[i][1] = fmaf(p, x.y, out[i][1]);
                }
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                const float4 x = *reinterpret_cast<const float4*>(X + (k + q) * (D + 4) + 64 * c + 4 * tx);
#pragma unroll
                for (int i = 0; i < RI; ++i) {
                    const float p = q == 0 ? w[i].x : q == 1 ? w[i].y : q == 2 ? w[i].z : w[i].w;
                    if (OWN && p == 0.f) continue;
                    out[i][4 * c + 0] = fmaf(p, x.x, out[i][4 * c + 0]);
                    out[i][4 * c + 1] = fmaf(p, x.y, out[i][4 * c + 1]);
                    out[i][4 * c + 2] = fmaf(p, x.z, out[i][4 * c + 2]);
                    out[i][4 * c + 3] = fmaf(p, x.w, out[i][4 * c + 3]);
                }
            }
    }
}
// over the 16 threads that share a row of the tile
__device__ __forceinline__ float row_max(float v) {
#pragma unroll
    for (int o = 8; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

struct Block {  // which tile, part, key head and sequence a block has
    long long tile;
    int part, hk, b;
};
__device__ __forceinline__ Block block_of(long long i, long long tiles, int parts, int Hkv) {
    Block k;
    k.tile = i % tiles;
    i /= tiles;
    k.part = (int)(i % parts);
    i /= parts;
    k.hk = (int)(i % Hkv);
    k.b = (int)(i / Hkv);
    return k;
}

// Which keys a tile of packed rows [r0, r0 + R) reads: tiles [0, sinks) and [from, to) of 64, in this order.
struct KeyTiles {
    int sinks, from, count;
    KeySpan seen;  // by some row
    __device__ __forceinline__ int tile(int i) const { return i < sinks ? i : i - sinks + from; }
};
template <bool WIN, int R>
__device__ __forceinline__ KeyTiles key_tiles(const XattnArgs& a, int b, long long r0, int n) {
    KeyTiles t;
    if constexpr (!WIN) {
        t.sinks = t.from = 0;
        t.count = (a.Lk + kTile - 1) / kTile;
    } else {
        const KeySpan s = t.seen = key_span<kWindowKeys>(a, b, r0 / a.G, (min(a.rows, r0 + R) - 1) / a.G, n);
        const int to = (s.hi + kTile - 1) / kTile;
        t.from = s.lo / kTile;
        t.sinks = min((s.sink + kTile - 1) / kTile, t.from);
        t.count = t.sinks + max(0, to - t.from);
    }
    return t;
}
// The keys that the rows ty + 16 i of a tile see: those of [lo, hi), and the sinks.
struct RowKeys {
    int lo, hi;
};
template <bool WIN, int RI>
__device__ __forceinline__ void row_spans(RowKeys (&span)[RI], const XattnArgs& a, int b, long long r0, int n) {
    if constexpr (WIN) {
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            const long long l = (unsigned)min(a.rows - 1, r0 + (threadIdx.x >> 4) + 16 * i) / (unsigned)a.G;
            const KeySpan s = key_span<kWindowKeys>(a, b, l, l, n);
            span[i] = {s.lo, s.hi};
        }
    }
}
template <bool WIN>
__device__ __forceinline__ bool sees(const RowKeys& s, int j, int sinks) {
    return !WIN || (j < s.hi && (j >= s.lo || j < sinks));
}

// (WIN: the spans take the registers of a second block of a multiprocessor unless told; 16 x 200 rows, 4 / 2 heads of 40 and 30:
// 41 us with one)
template <typename T, int DK, int DV, bool WIN>
__global__ void __launch_bounds__(kThreads, WIN ? 2 : 1) k_xattn(const XattnArgs a, long long tiles) {
    extern __shared__ float4 sm4[];
    float* Qs = reinterpret_cast<float*>(sm4);
    float* Ks = Qs + kTile * (DK + 4);  // then the weights
    constexpr int kKs = (DK + 4 > kPP ? DK + 4 : kPP) * kTile;
    float* Vs = Ks + kKs;
    __shared__ int ok[kTile];
    const Block bl = block_of(blockIdx.x, tiles, a.splits, a.Hkv);
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    const long long r0 = bl.tile * kTile;
    const int n = keys_of(a, bl.b);
    const KeyTiles kt = key_tiles<WIN, kTile>(a, bl.b, r0, n);
    const int t0 = (int)((long long)kt.count * bl.part / a.splits), t1 = (int)((long long)kt.count * (bl.part + 1) / a.splits);
    const float c = a.scale * kLog2e;
    [[maybe_unused]] RowKeys span[4];
    row_spans<WIN>(span, a, bl.b, r0, n);
    load_rows<T, DK>(Qs, a, a.q, bl.b, bl.hk, r0, a.dk, a.vec & kVecQ);
    float m[4], l[4], o[4][DV / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int q = 0; q < DV / 16; ++q) o[i][q] = 0.f;
    }
    for (int i = t0; i < t1; ++i) {
        const int t = kt.tile(i);
        if (t * kTile >= n) break;
        __syncthreads();  // the last tile's weights and values have been read
        const bool has = load_valid<WIN>(ok, a, bl.b, t * kTile, n, kt.seen), odd = load_keys<T, DK, DV>(Ks, Vs, a, bl.b, bl.hk, t * kTile, has);
        bool own = false;  // through a window 0 * NaN of a value that only other rows of the tile see is kept out
        if constexpr (WIN)
            own = __syncthreads_or(odd);
        else
            __syncthreads();
        float s[4][4] = {};
        dots<DK>(s, Qs, Ks, a.dk);
        __syncthreads();  // K has been read: the weights go over it
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = ok[tx + 16 * j] && sees<WIN>(span[i], t * kTile + tx + 16 * j, a.win.sinks) ? s[i][j] * c : -INFINITY;
                mx = fmaxf(mx, s[i][j]);
            }
            const float mn = fmaxf(m[i], row_max(mx));
            const float ms = mn == -INFINITY ? 0.f : mn;
            const float f = exp2f(m[i] - ms);
            float add = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = exp2f(s[i][j] - ms);
                add += p;
                Ks[(ty + 16 * i) * kPP + tx + 16 * j] = p;
            }
            l[i] = l[i] * f + row_sum(add);
            m[i] = mn;
#pragma unroll
            for (int q = 0; q < DV / 16; ++q) o[i][q] *= f;
        }
        __syncthreads();
        if (WIN && own)
            weigh<DV, kTile, true>(o, Ks, Vs);
        else
            weigh<DV>(o, Ks, Vs);
    }
    const long long nrows = (long long)a.B * a.Hq * a.Lq;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long r = r0 + ty + 16 * i;
        if (r >= a.rows) continue;
        const long long at = row_index(a, bl.b, bl.hk, r);
        if (a.splits > 1) {
            float* po = a.ws + ((long long)bl.part * nrows + at) * a.dv;
#pragma unroll
            for (int q = 0; q < DV / 16; ++q) {
                const int col = column<DV>(q);
                if (col < a.dv) po[col] = o[i][q];
            }
            if (tx == 0) {
                float* ml = a.ws + xattn_ws_ml(a) + ((long long)bl.part * nrows + at) * 2;
                ml[0] = m[i];
                ml[1] = l[i];
            }
        } else {
            T* po = row_at<T>(a, a.o, bl.b, bl.hk, r);
            const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
            for (int q = 0; q < DV / 16; ++q) {
                const int col = column<DV>(q);
                if (col < a.dv) po[col] = from_f32<T>(o[i][q] * inv);
            }
            if (tx == 0 && a.lse) a.lse[at] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * kLn2;
        }
    }
}

// D_i = <dO_i, O_i>: one warp per row.  Under a mask that leaves few keys, from bf16: sum_j P dP (few_keys).
// (WIN: what a row sees is its own; up to few_seen keys are taken one by one.)
template <typename T, bool WIN>
__global__ void __launch_bounds__(256) k_xattn_delta(const XattnArgs a) {
    const long long nrows = (long long)a.B * a.Hq * a.Lq;
    const long long at = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (at >= nrows) return;
    const long long i = at % a.Lq, bh = at / a.Lq;
    const T* o = reinterpret_cast<const T*>(a.o.p) + (bh / a.Hq) * a.o.b + i * a.o.l + (bh % a.Hq) * a.o.h;
    const T* d = reinterpret_cast<const T*>(a.dO.p) + (bh / a.Hq) * a.dO.b + i * a.dO.l + (bh % a.Hq) * a.dO.h;
    float acc = 0.f;
    for (int q = lane; q < a.dv; q += 32) acc = fmaf(to_f32(o[q]), to_f32(d[q]), acc);
#pragma unroll
    for (int k = 16; k; k >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, k);
    if constexpr (sizeof(T) == 2) {
        const int b = (int)(bh / a.Hq), h = (int)(bh % a.Hq), hk = h / a.G, n = keys_of(a, b);
        int key = 0;
        int few = 0;
        if constexpr (WIN)
            few = few_seen<32>(a, b, key_span<kWindowKeys>(a, b, i, i, n), key);
        else
            few = a.mask && n > kTile ? few_keys(a, b, 0, n, key) : 0;  // (up to a tile's: k_xattn_dq sums D)
        if (few > 0) {
            const T* q = reinterpret_cast<const T*>(a.q.p) + b * a.q.b + i * a.q.l + h * a.q.h;
            const float cs = a.scale * kLog2e, L = a.lse[at] * kLog2e;
            acc = 0.f;
            for (int f = 0; f < few; ++f) {
                const long long j = __shfl_sync(0xffffffffu, key, f);
                const T* kr = reinterpret_cast<const T*>(a.k.p) + b * a.k.b + j * a.k.l + hk * a.k.h;
                const T* vr = reinterpret_cast<const T*>(a.v.p) + b * a.v.b + j * a.v.l + hk * a.v.h;
                float s = 0.f, dp = 0.f;
                for (int c = lane; c < a.dk; c += 32) s = fmaf(to_f32(q[c]), to_f32(kr[c]), s);
                for (int c = lane; c < a.dv; c += 32) dp = fmaf(to_f32(d[c]), to_f32(vr[c]), dp);
#pragma unroll
                for (int k = 16; k; k >>= 1) {
                    s += __shfl_xor_sync(0xffffffffu, s, k);
                    dp += __shfl_xor_sync(0xffffffffu, dp, k);
                }
                acc = fmaf(exp2f(s * cs - L), dp, acc);
            }
        }
    }
    if (lane == 0) a.ws[at] = acc;
}

// P and dS of a tile from S, dO V^T and the rows' statistics; a row without weight (lse = -inf) has P = 0
// (WIN: key j0 + tx + 16 j is seen by the row as its span says)
template <bool WIN, int RI>
__device__ __forceinline__ void tile_grad(float (&s)[RI][4], float (&dp)[RI][4], const int* ok, const float* lse2,
                                          const float* delta, float c, const RowKeys (&span)[RI], int j0, int sinks) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
    for (int i = 0; i < RI; ++i) {
        const float L = lse2[ty + 16 * i], D = delta[ty + 16 * i];
        // (a row whose span is one key at most has no dS, exactly: its weight is 1 whatever its logit)
        const bool one = WIN && span[i].hi - span[i].lo + min(sinks, span[i].lo) <= 1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool use = ok[tx + 16 * j] && L != INFINITY && sees<WIN>(span[i], j0 + tx + 16 * j, sinks);
            s[i][j] = use ? exp2f(s[i][j] * c - L) : 0.f;
            dp[i][j] = use && !one ? s[i][j] * (dp[i][j] - D) : 0.f;
        }
    }
}
// lse (base 2; +inf: the row has no weight) and D (OWN: not here) of R packed rows
template <int R, bool OWN>
__device__ __forceinline__ void load_stats(float* lse2, float* delta, const XattnArgs& a, int b, int hk, long long r0) {
    if (threadIdx.x < R) {
        const long long r = r0 + threadIdx.x;
        float L = INFINITY, D = 0.f;
        if (r < a.rows) {
            const long long at = row_index(a, b, hk, r);
            const float v = a.lse[at];
            if (v != -INFINITY) {
                // (a +inf here is a row whose forward result is NaN: P = NaN, as there)
                L = v == INFINITY ? NAN : v * kLog2e;
                if constexpr (!OWN) D = a.ws[at];
            }
        }
        lse2[threadIdx.x] = L;
        if constexpr (!OWN) delta[threadIdx.x] = D;
    }
}

// In fp32 a window's kernels take D = <dO, O> of their R rows themselves, which spares a launch: rows of dO go to dst as by load_rows,
// four threads a row, and D to delta.
template <typename T, int D, int R>
__device__ __forceinline__ void load_rows_delta(float* dst, float* delta, const XattnArgs& a, int b, int hk, long long r0) {
    const int i = threadIdx.x >> 2, c0 = (threadIdx.x & 3) * 4;
    const bool has = i < R && r0 + i < a.rows;
    const T *p = row_at<T>(a, a.dO, b, hk, has ? r0 + i : 0), *o = row_at<T>(a, a.o, b, hk, has ? r0 + i : 0);
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < D; c += 16) {
        const float4 x = load4(p + c + c0, has ? a.dv - c - c0 : 0, a.vec & kVecDO), y = load4(o + c + c0, has ? a.dv - c - c0 : 0, a.vec & kVecO);
        if (i < R) *reinterpret_cast<float4*>(dst + i * (D + 4) + c + c0) = x;
        sum = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, sum))));
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    if (i < R && (threadIdx.x & 3) == 0) delta[i] = sum;
}

// Tiles of R rows: 64, or 16 where a key head has few (a tile's products are taken whole).  fp32, 17 x 832 keys, 16 / 64: 14 rows,
// 16 key heads of 128 and 81, 499 / 948 us; 32 rows of 128 988 / 1,212; 20 rows of 64 438 / 425 (the rule loses 3 % there).
int bwd_rows(const XattnArgs& a) { return a.rows <= 32 ? 16 : kTile; }

template <int DK, int DV, int R>
constexpr size_t bwd_smem() {  // weights: R x 64, or 64 keys x R
    return sizeof(float) * ((kTile + R) * ((DK + 4) + (DV + 4)) + (R * kPP > kTile * (R + 4) ? R * kPP : kTile * (R + 4)));
}

template <typename T, int DK, int DV, int R, bool WIN>
__device__ __forceinline__ void dq_block(const XattnArgs& a, long long block, long long tiles) {
    extern __shared__ float4 sm4[];
    constexpr bool kOwn = WIN && sizeof(T) == 4;
    float* Qs = reinterpret_cast<float*>(sm4);
    float* Ks = Qs + R * (DK + 4);
    float* Vs = Ks + kTile * (DK + 4);
    float* Ds = Vs + kTile * (DV + 4);  // dO
    float* Ws = Ds + R * (DV + 4);
    __shared__ int ok[kTile];
    __shared__ float lse2[R], delta[R];
    constexpr int RI = R / 16;
    const Block bl = block_of(block, tiles, a.splits, a.Hkv);
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    const long long r0 = bl.tile * R;
    const int n = keys_of(a, bl.b);
    const KeyTiles kt = key_tiles<WIN, R>(a, bl.b, r0, n);
    const int t0 = (int)((long long)kt.count * bl.part / a.splits), t1 = (int)((long long)kt.count * (bl.part + 1) / a.splits);
    RowKeys span[RI];
    row_spans<WIN>(span, a, bl.b, r0, n);
    load_rows<T, DK, R>(Qs, a, a.q, bl.b, bl.hk, r0, a.dk, a.vec & kVecQ);
    if constexpr (kOwn)
        load_rows_delta<T, DV, R>(Ds, delta, a, bl.b, bl.hk, r0);
    else
        load_rows<T, DV, R>(Ds, a, a.dO, bl.b, bl.hk, r0, a.dv, a.vec & kVecDO);
    if (t0 < t1 && kt.tile(t0) * kTile < n) load_stats<R, kOwn>(lse2, delta, a, bl.b, bl.hk, r0);  // (the part that has the keys may write D)
    float o[RI][DK / 16] = {};
    for (int i = t0; i < t1; ++i) {
        const int t = kt.tile(i);
        if (t * kTile >= n) break;
        __syncthreads();
        load_keys<T, DK, DV>(Ks, Vs, a, bl.b, bl.hk, t * kTile, load_valid<WIN>(ok, a, bl.b, t * kTile, n, kt.seen));
        __syncthreads();
        float s[RI][4] = {}, dp[RI][4] = {};
        dots<DK>(s, Qs, Ks, a.dk);
        dots<DV>(dp, Ds, Vs, a.dv);
        if (!WIN && sizeof(T) == 2 && n <= kTile) {
            // every key of the sequence is here, whatever its padding (other parts have no tile): D = sum_j P dP, for this kernel
            // and the next (a bf16 O gives it to 2^-8 of the sum of |dO O|, which with a few keys is more than dP - D; an fp32 O gives
            // it more exactly than this sum, in which P is off by lse's rounding, |lse| 2^-24)
#pragma unroll
            for (int i = 0; i < RI; ++i) {
                const float L = lse2[ty + 16 * i];
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (ok[tx + 16 * j] && L != INFINITY) sum = fmaf(exp2f(s[i][j] * a.scale * kLog2e - L), dp[i][j], sum);
                sum = row_sum(sum);
                const long long r = r0 + ty + 16 * i;
                if (tx == 0) {
                    delta[ty + 16 * i] = sum;
                    if (r < a.rows) a.ws[row_index(a, bl.b, bl.hk, r)] = sum;
                }
            }
            __syncthreads();
        }
        tile_grad<WIN>(s, dp, ok, lse2, delta, a.scale * kLog2e, span, t * kTile, a.win.sinks);
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) Ws[(ty + 16 * i) * kPP + tx + 16 * j] = dp[i][j];
        __syncthreads();
        weigh<DK>(o, Ws, Ks);
    }
    const long long nrows = (long long)a.B * a.Hq * a.Lq;
#pragma unroll
    for (int i = 0; i < RI; ++i) {
        const long long r = r0 + ty + 16 * i;
        if (r >= a.rows) continue;
#pragma unroll
        for (int q = 0; q < DK / 16; ++q) {
            const int col = column<DK>(q);
            if (col >= a.dk) continue;
            if (a.splits > 1)
                a.ws[xattn_ws_dq(a) + ((long long)bl.part * nrows + row_index(a, bl.b, bl.hk, r)) * a.dk + col] = o[i][q];
            else
                row_at<T>(a, a.dQ, bl.b, bl.hk, r)[col] = from_f32<T>(o[i][q] * a.scale);
        }
    }
}

template <typename T, int DK, int DV, int R, bool WIN>
__device__ __forceinline__ void dkv_block(const XattnArgs& a, long long block, int ktiles) {
    extern __shared__ float4 sm4[];
    constexpr bool kOwn = WIN && sizeof(T) == 4;
    float* Qs = reinterpret_cast<float*>(sm4);
    float* Ks = Qs + R * (DK + 4);
    float* Vs = Ks + kTile * (DK + 4);
    float* Ds = Vs + kTile * (DV + 4);
    float* Ws = Ds + R * (DV + 4);  // P^T, then dS^T: [key][row]
    __shared__ int ok[kTile];
    __shared__ float lse2[R], delta[R];
    constexpr int RI = R / 16, kPR = R + 4;
    Block bl;
    int parts = a.rsplits;
    if constexpr (WIN) {  // key tiles slowest: the first ones, which sinks show to all rows, begin first
        const int per = a.Hkv * a.B;
        bl = block_of(block % per, 1, 1, a.Hkv);
        const long long at = block / per, in_parts = (a.pkeys + kTile - 1) / kTile;
        if (at < in_parts * parts) {
            bl.tile = at / parts;
            bl.part = (int)(at % parts);
        } else {
            bl.tile = at - in_parts * (parts - 1);
            parts = 1;
        }
    } else {
        bl = block_of(block, ktiles, a.rsplits, a.Hkv);
    }
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    const int j0 = (int)bl.tile * kTile;
    const int n = keys_of(a, bl.b);
    const long long rtiles = (a.rows + R - 1) / R;
    long long t0 = rtiles * bl.part / parts, t1 = rtiles * (bl.part + 1) / parts;
    if constexpr (WIN) {
        const RowSpan rs = row_span(a, bl.b, j0, min(n, j0 + kTile));
        const long long first = rs.first * a.G / R, some = max(0ll, (rs.end * a.G + R - 1) / R - first);
        t0 = first + some * bl.part / parts;
        t1 = first + some * (bl.part + 1) / parts;
    }
    if (j0 >= n) t1 = t0;  // no key of the tile is read
    load_keys<T, DK, DV>(Ks, Vs, a, bl.b, bl.hk, j0, load_valid<false>(ok, a, bl.b, j0, n, KeySpan()));
    float ok_[4][DK / 16] = {}, ov[4][DV / 16] = {};
    for (long long t = t0; t < t1; ++t) {
        __syncthreads();
        load_rows<T, DK, R>(Qs, a, a.q, bl.b, bl.hk, t * R, a.dk, a.vec & kVecQ);
        if constexpr (kOwn)
            load_rows_delta<T, DV, R>(Ds, delta, a, bl.b, bl.hk, t * R);
        else
            load_rows<T, DV, R>(Ds, a, a.dO, bl.b, bl.hk, t * R, a.dv, a.vec & kVecDO);
        load_stats<R, kOwn>(lse2, delta, a, bl.b, bl.hk, t * R);
        __syncthreads();
        float s[RI][4] = {}, dp[RI][4] = {};
        dots<DK>(s, Qs, Ks, a.dk);
        dots<DV>(dp, Ds, Vs, a.dv);
        RowKeys span[RI];
        row_spans<WIN>(span, a, bl.b, t * R, n);
        tile_grad<WIN>(s, dp, ok, lse2, delta, a.scale * kLog2e, span, j0, a.win.sinks);
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) Ws[(tx + 16 * j) * kPR + ty + 16 * i] = s[i][j];
        __syncthreads();
        weigh<DV, R>(ov, Ws, Ds);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) Ws[(tx + 16 * j) * kPR + ty + 16 * i] = dp[i][j];
        __syncthreads();
        weigh<DK, R>(ok_, Ws, Qs);
    }
    const long long nk = xattn_keys(a);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = j0 + ty + 16 * i;
        if (j >= a.Lk) continue;
        const long long at = ((long long)bl.b * a.Hkv + bl.hk) * a.pkeys + j;
#pragma unroll
        for (int q = 0; q < DK / 16; ++q) {
            const int col = column<DK>(q);
            if (col >= a.dk) continue;
            if (parts > 1)
                a.ws[xattn_ws_dk(a) + ((long long)bl.part * nk + at) * a.dk + col] = ok_[i][q];
            else
                (reinterpret_cast<T*>(a.dK.p) + bl.b * a.dK.b + j * a.dK.l + bl.hk * a.dK.h)[col] =
                    from_f32<T>(ok_[i][q] * a.scale);
        }
#pragma unroll
        for (int q = 0; q < DV / 16; ++q) {
            const int col = column<DV>(q);
            if (col >= a.dv) continue;
            if (parts > 1)
                a.ws[xattn_ws_dv(a) + ((long long)bl.part * nk + at) * a.dv + col] = ov[i][q];
            else
                (reinterpret_cast<T*>(a.dV.p) + bl.b * a.dV.b + j * a.dV.l + bl.hk * a.dV.h)[col] = from_f32<T>(ov[i][q]);
        }
    }
}

template <typename T, int DK, int DV, int R, bool WIN>
__global__ void __launch_bounds__(kThreads) k_xattn_dq(const XattnArgs a, long long tiles) {
    dq_block<T, DK, DV, R, WIN>(a, blockIdx.x, tiles);
}
template <typename T, int DK, int DV, int R, bool WIN>
__global__ void __launch_bounds__(kThreads) k_xattn_dkv(const XattnArgs a, int ktiles) {
    dkv_block<T, DK, DV, R, WIN>(a, blockIdx.x, ktiles);
}
// Through a window both in one launch, as a row or key tile alone meets few of the other kind: first `keys` blocks of keys, then
// those of rows.
template <typename T, int DK, int DV, int R>
__global__ void __launch_bounds__(kThreads, 2) k_xattn_bwd(const XattnArgs a, long long keys, int ktiles, long long tiles) {
    if (blockIdx.x < keys)
        dkv_block<T, DK, DV, R, true>(a, blockIdx.x, ktiles);
    else
        dq_block<T, DK, DV, R, true>(a, blockIdx.x - keys, tiles);
}

template <typename F>
cudaError_t allow_smem(F* f, size_t bytes) {
    return bytes <= 47 * 1024 ? cudaSuccess  // (48 KB with the static arrays)
                              : cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T, int DK, int DV, bool WIN>
cudaError_t forward(const XattnArgs& a, cudaStream_t s) {
    const long long tiles = (a.rows + kTile - 1) / kTile;
    const long long grid = tiles * a.splits * a.Hkv * a.B;
    const size_t smem = sizeof(float) * kTile * ((DK + 4) + (DK + 4 > kPP ? DK + 4 : kPP) + (DV + 4));
    const auto kernel = k_xattn<T, DK, DV, WIN>;
    cudaError_t e = allow_smem(kernel, smem);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)grid, kThreads, smem, s>>>(a, tiles);
    return cudaGetLastError();
}
template <typename T, int DK, int DV, int R, bool WIN>
cudaError_t backward_r(const XattnArgs& a, cudaStream_t s) {
    const size_t smem = bwd_smem<DK, DV, R>();
    cudaError_t e = cudaSuccess;
    if constexpr (WIN) {
        const long long tiles = (a.rows + R - 1) / R, per = (long long)a.Hkv * a.B;
        const int ktiles = (a.Lk + kTile - 1) / kTile;
        const long long in_parts = (a.pkeys + kTile - 1) / kTile;
        const long long keys = (ktiles + in_parts * (a.rsplits - 1)) * per, grid = keys + tiles * a.splits * per;
        if (grid == 0) return e;
        if (grid > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
        const auto kernel = k_xattn_bwd<T, DK, DV, R>;
        if ((e = allow_smem(kernel, smem)) != cudaSuccess) return e;
        kernel<<<(unsigned)grid, kThreads, smem, s>>>(a, keys, ktiles, tiles);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        if (a.splits > 1 && (e = launch_xattn_join_dq(a, s)) != cudaSuccess) return e;
        return a.rsplits > 1 ? launch_xattn_join_dkv(a, s) : cudaSuccess;
    } else {
        if (a.rows > 0) {
            const long long tiles = (a.rows + R - 1) / R;
            const auto kernel = k_xattn_dq<T, DK, DV, R, WIN>;
            if ((e = allow_smem(kernel, smem)) != cudaSuccess) return e;
            kernel<<<(unsigned)(tiles * a.splits * a.Hkv * a.B), kThreads, smem, s>>>(a, tiles);
            if ((e = cudaGetLastError()) != cudaSuccess) return e;
            if (a.splits > 1 && (e = launch_xattn_join_dq(a, s)) != cudaSuccess) return e;
        }
        if (a.Lk > 0) {
            const int ktiles = (a.Lk + kTile - 1) / kTile;
            const auto kernel = k_xattn_dkv<T, DK, DV, R, WIN>;
            if ((e = allow_smem(kernel, smem)) != cudaSuccess) return e;
            kernel<<<(unsigned)((long long)ktiles * a.rsplits * a.Hkv * a.B), kThreads, smem, s>>>(a, ktiles);
            if ((e = cudaGetLastError()) != cudaSuccess) return e;
            if (a.rsplits > 1) e = launch_xattn_join_dkv(a, s);
        }
        return e;
    }
}

template <typename T, int DK, int DV, bool WIN>
cudaError_t backward(const XattnArgs& a, cudaStream_t s) {
    return bwd_rows(a) == 16 ? backward_r<T, DK, DV, 16, WIN>(a, s) : backward_r<T, DK, DV, kTile, WIN>(a, s);
}

bool on_fours(const XattnArgs& a, const HeadView& v, int L, int H) {
    const int bytes = a.dtype == GS_F32 ? 16 : 8;
    return (uintptr_t)v.p % bytes == 0 && (a.B <= 1 || v.b % 4 == 0) && (L <= 1 || v.l % 4 == 0) && (H <= 1 || v.h % 4 == 0);
}

template <typename T, bool WIN>
cudaError_t forward_t(XattnArgs a, cudaStream_t s) {
    a.vec = (on_fours(a, a.q, a.Lq, a.Hq) ? kVecQ : 0) | (on_fours(a, a.k, a.Lk, a.Hkv) ? kVecK : 0) |
            (on_fours(a, a.v, a.Lk, a.Hkv) ? kVecV : 0);
    if (a.dk <= 64)
        return a.dv <= 32 ? forward<T, 64, 32, WIN>(a, s) : a.dv <= 64 ? forward<T, 64, 64, WIN>(a, s) : forward<T, 64, 128, WIN>(a, s);
    return a.dv <= 64 ? forward<T, 128, 64, WIN>(a, s) : forward<T, 128, 128, WIN>(a, s);
}
template <typename T, bool WIN>
cudaError_t backward_t(XattnArgs a, cudaStream_t s) {
    a.vec = (on_fours(a, a.q, a.Lq, a.Hq) ? kVecQ : 0) | (on_fours(a, a.k, a.Lk, a.Hkv) ? kVecK : 0) |
            (on_fours(a, a.v, a.Lk, a.Hkv) ? kVecV : 0) | (on_fours(a, a.dO, a.Lq, a.Hq) ? kVecDO : 0) |
            (on_fours(a, a.o, a.Lq, a.Hq) ? kVecO : 0);
    if (a.dk <= 32 && a.dv <= 32) return backward<T, 32, 32, WIN>(a, s);
    if (a.dk <= 64)
        return a.dv <= 32 ? backward<T, 64, 32, WIN>(a, s) : a.dv <= 64 ? backward<T, 64, 64, WIN>(a, s) : backward<T, 64, 128, WIN>(a, s);
    return a.dv <= 64 ? backward<T, 128, 64, WIN>(a, s) : backward<T, 128, 128, WIN>(a, s);
}

template <typename T, bool WIN>
cudaError_t launch_delta(const XattnArgs& a, cudaStream_t s) {
    const long long rows = (long long)a.B * a.Hq * a.Lq;
    if (rows == 0) return cudaSuccess;
    // (in fp32 what a row sees makes no difference)
    k_xattn_delta<T, WIN && sizeof(T) == 2><<<(unsigned)((rows + 7) / 8), 256, 0, s>>>(a);
    return cudaGetLastError();
}
template <bool WIN>
cudaError_t forward_all(const XattnArgs& a, cudaStream_t s) {
    return a.dtype == GS_F32 ? forward_t<float, WIN>(a, s) : forward_t<__nv_bfloat16, WIN>(a, s);
}
template <bool WIN>
cudaError_t backward_all(const XattnArgs& a, cudaStream_t s) {
    const cudaError_t e = a.dtype != GS_F32 ? launch_delta<__nv_bfloat16, WIN>(a, s) : WIN ? cudaSuccess : launch_delta<float, WIN>(a, s);
    if (e != cudaSuccess) return e;
    return a.dtype == GS_F32 ? backward_t<float, WIN>(a, s) : backward_t<__nv_bfloat16, WIN>(a, s);
}

}  // namespace
}  // namespace gs
