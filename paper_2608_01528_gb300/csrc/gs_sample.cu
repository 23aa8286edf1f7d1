// gs_sample.cu -- one random entry of each score row (temperature, top-k, top-p, min-p).
//
// Every rule keeps a prefix of the row in (score descending, index ascending) order, so what is
// kept is always "key > t, or key == t and among the first `ties` of those in index order", with
// key the score as an ordered integer.  t comes from a radix select over the keys, 8 bits a pass, by counts
// (top-k) or by weights (top-p); nothing is sorted.
//
// Weights are integers: w = round(2^44 exp((s - max) / T)).  Integer sums are the same in any
// order, and 2^19 of them fit 63 bits; next to that, fp32 sums of a large vocabulary are off by more than its
// small probabilities, and a draw whose number ends near a border would go to a neighbour.
//
// The row is read once per pass by one block.

#include <math.h>

#include <algorithm>

#include "gs_xattn.h"

namespace gs {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kOneBits = 44;  // the largest weight is 2^44

// Order-preserving key of a score; 0 for what is never drawn (-inf, NaN).  -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return x > -INFINITY ? k : 0u;
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}

__device__ __forceinline__ float load_score(const void* row, bool bf16, int i) {
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(row)[i]) : static_cast<const float*>(row)[i];
}

// 2^(j / 64), j = -32..32, times 2^44, rounded
struct PowTable {
    u64 v[65];
};

struct Weigher {
    float half_max;    // max / 2 (halves: the difference of two finite scores does not overflow)
    float chi, clo;    // 2 log2(e) / T in two floats
    uint32_t top;      // the largest score's key
    bool only_top;     // weights are 1 for the largest scores and 0 for the others
    const u64* pow;    // 2^(j / 64)

    // round(2^44 exp((x - max) / T)), relative error below 2^-38: the exponent and the difference are kept in
    // two floats each, 2^(j/64) comes from the table, exp of the remainder |t| < 0.0055 from its series.
    __device__ __forceinline__ u64 operator()(uint32_t key) const {
        if (only_top || key == 0u) return key == top && key != 0u ? 1ull << kOneBits : 0ull;
        const float a = 0.5f * value_of(key), b = half_max;
        const float d = a - b, bb = d - a;
        const float dl = (a - (d - bb)) - (b + bb);
        const float ph = d * chi;
        const float pl = fmaf(d, chi, -ph) + fmaf(d, clo, dl * chi);
        if (!(ph > -46.f)) return 0ull;
        const float n = rintf(ph), rh = ph - n, j = rintf(rh * 64.f), sh = rh - j * 0.015625f;
        constexpr float kLnHi = 0.693147182464599609375f, kLnLo = -1.904654299957767878541e-9f;
        const float th0 = sh * kLnHi;
        const float tl0 = fmaf(sh, kLnHi, -th0) + fmaf(sh, kLnLo, pl * kLnHi);
        const float th = th0 + tl0, tl = tl0 - (th - th0);
        const float e = fmaf(th * th, fmaf(th, fmaf(th, fmaf(th, 1.f / 120.f, 1.f / 24.f), 1.f / 6.f), 0.5f), tl);
        const u64 T = pow[(int)j + 32];
        constexpr float kDown = 1.f / 17592186044416.f;
        const float Tf = __ull2float_rn(T) * kDown;
        const float Tl = __ll2float_rn((long long)(T - (u64)__float2ull_rn(Tf * 17592186044416.f))) * kDown;
        const float m = Tf * th;
        const float me = fmaf(Tf, th, -m) + fmaf(Tl, th, Tf * e);
        u64 w = T + (u64)__float2ll_rn(m * 17592186044416.f) + (u64)(long long)__float2ll_rn(me * 17592186044416.f);
        const int s = -(int)n;
        return s > 0 ? (w + (1ull << (s - 1))) >> s : w;
    }
};

__device__ __forceinline__ u64 warp_sum_u64(u64 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// the sum over the block, in every thread
__device__ u64 block_sum(u64 v, u64* sh) {
    v = warp_sum_u64(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    u64 t = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) t += sh[i];
    return t;
}

// floor (up: ceiling) of f * total, 0 <= f < 1, exactly
__device__ __forceinline__ u64 share_of(float f, u64 total, bool up) {
    const u64 F = __float2ull_rz(f * 18446744073709551616.f);
    const u64 hi = __umul64hi(F, total), lo = F * total;
    return hi + (up && lo != 0 ? 1 : 0);
}

__global__ void __launch_bounds__(kThreads) k_sample(const SampleArgs a, const __grid_constant__ PowTable table) {
    __shared__ u64 hist[256];
    __shared__ u64 sh[kWarps];
    __shared__ u64 pow[65];
    __shared__ u64 found[4];
    const long long n = blockIdx.x;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int M = a.M;
    const void* row = static_cast<const char*>(a.S) + n * a.lds * (a.bf16 ? 2 : 4);
    auto key_at = [&](int i) { return key_of(load_score(row, a.bf16, i)); };
    for (int i = tid; i < 65; i += kThreads) pow[i] = table.v[i];

    // the largest key, its first index
    u64 best = 0;
    for (int i = tid; i < M; i += kThreads) {
        const u64 k = (u64)key_at(i) << 32 | (uint32_t)~i;
        best = k > best ? k : best;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const u64 k = __shfl_xor_sync(0xffffffffu, best, o);
        best = k > best ? k : best;
    }
    if (lane == 0) sh[warp] = best;
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) best = sh[i] > best ? sh[i] : best;
    const uint32_t top = (uint32_t)(best >> 32);
    const int first = (int)~(uint32_t)best;
    const float T = a.how.temperature_rows ? a.how.temperature_rows[n] : a.how.temperature;
    if (top == 0u || !(T > 0.f)) {
        if (tid == 0) {
            if (a.index) a.index[n] = top ? first : -1;
            if (a.prob) a.prob[n] = top ? 1.f : 0.f;
        }
        return;
    }
    const int top_k = a.how.top_k_rows ? a.how.top_k_rows[n] : a.how.top_k;
    const float top_p = a.how.top_p_rows ? a.how.top_p_rows[n] : a.how.top_p;
    const float min_p = a.how.min_p_rows ? a.how.min_p_rows[n] : a.how.min_p;
    float u = a.U[n];
    u = u >= 0.f ? fminf(u, 1.f - 5.9604644775390625e-8f) : 0.f;

    Weigher w;
    const double c = 2.8853900817779268 / (double)T;
    w.half_max = 0.5f * value_of(top);
    w.chi = (float)c;
    w.clo = (float)(c - (double)w.chi);
    w.top = top;
    w.only_top = value_of(top) == INFINITY || !(c < 1e38);
    w.pow = pow;

    // smallest key t such that the measure (count or weight) of the keys >= t reaches need; `above`: that of keys > t
    auto select = [&](bool by_weight, u64 need, u64& above) {
        uint32_t prefix = 0;
        above = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            for (int i = tid; i < 256; i += kThreads) hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < M; i += kThreads) {
                const uint32_t k = key_at(i);
                if (k == 0u || (shift < 24 && (k >> (shift + 8)) != (prefix >> (shift + 8)))) continue;
                atomicAdd(&hist[(k >> shift) & 255u], by_weight ? w(k) : 1ull);
            }
            __syncthreads();
            if (tid == 0) {
                int b = 255;
                u64 run = above;
                while (b > 0 && run + hist[b] < need) run += hist[b--];
                found[0] = (u64)b;
                found[1] = run;
            }
            __syncthreads();
            prefix |= (uint32_t)found[0] << shift;
            above = found[1];
        }
        return prefix;
    };

    uint32_t t = 1;         // kept: key > t, or key == t and among the first `ties` in index order
    u64 ties = ~0ull;
    bool all = true;
    if (top_k >= 1 && top_k < M) {
        u64 above;
        u64 valid = 0;
        for (int i = tid; i < M; i += kThreads) valid += key_at(i) != 0u;
        valid = block_sum(valid, sh);
        if ((u64)top_k < valid) {
            t = select(false, (u64)top_k, above);
            ties = (u64)top_k - above;
            all = false;
        }
    }
    // the kept weight; the tied ones' share by their number
    auto kept_weight = [&]() {
        u64 s = 0, eq = 0;
        for (int i = tid; i < M; i += kThreads) {
            const uint32_t k = key_at(i);
            if (k > t) s += w(k);
            eq += k == t;
        }
        s = block_sum(s, sh);
        eq = block_sum(eq, sh);
        return s + w(t) * (eq < ties ? eq : ties);
    };
    u64 total = kept_weight();
    if (top_p < 1.f) {
        const u64 share = share_of(fmaxf(top_p, 0.f), total, true);
        const u64 need = share > 0 ? share : 1;
        u64 above;
        t = select(true, need, above);
        const u64 wt = w(t);
        ties = wt ? (need - above + wt - 1) / wt : ~0ull;
        all = false;
        total = above + wt * ties;
    }
    if (min_p > 0.f) {
        uint32_t least = top;
        if (min_p < 1.f && !w.only_top) {
            const double at = (double)value_of(top) + (double)T * log((double)min_p);
            float f = (float)at;
            if ((double)f < at) f = nextafterf(f, INFINITY);
            least = min(key_of(f), top);
        }
        if (least > t) {
            t = least;
            ties = ~0ull;
            all = false;
            total = kept_weight();
        }
    }
    // with fewer ties kept than there are: the index of the last one
    const int seg = (M + kWarps - 1) / kWarps;
    const int s0 = min(M, warp * seg), s1 = min(M, s0 + seg);
    int cut = M - 1;
    if (!all && ties != ~0ull) {
        u64 cnt = 0;
        for (int i = s0 + lane; i < s1; i += 32) cnt += key_at(i) == t;
        cnt = warp_sum_u64(cnt);
        __syncthreads();
        if (lane == 0) sh[warp] = cnt;
        if (tid == 0) found[2] = (u64)(M - 1);
        __syncthreads();
        u64 before = 0;
        for (int i = 0; i < warp; ++i) before += sh[i];
        if (before < ties && before + cnt >= ties) {
            for (int i = s0; i < s1; i += 32) {
                const bool eq = i + lane < s1 && key_at(i + lane) == t;
                const unsigned b = __ballot_sync(0xffffffffu, eq);
                if (before + __popc(b) >= ties) {
                    if (eq && before + __popc(b & ((2u << lane) - 1u)) == ties) found[2] = (u64)(i + lane);
                    break;
                }
                before += __popc(b);
            }
        }
        __syncthreads();
        cut = (int)found[2];
    }
    // the first index whose running kept weight exceeds u * total
    const u64 target = share_of(u, total, false);
    auto kept = [&](int i) {
        const uint32_t k = key_at(i);
        return k > t || (k == t && i <= cut) ? w(k) : 0ull;
    };
    u64 mine = 0;
    for (int i = s0 + lane; i < s1; i += 32) mine += kept(i);
    mine = warp_sum_u64(mine);
    __syncthreads();
    if (lane == 0) sh[warp] = mine;
    __syncthreads();
    u64 before = 0;
    for (int i = 0; i < warp; ++i) before += sh[i];
    if (before <= target && before + mine > target) {
        for (int i = s0; i < s1; i += 32) {
            const u64 v = i + lane < s1 ? kept(i + lane) : 0ull;
            u64 run = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 x = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += x;
            }
            const unsigned past = __ballot_sync(0xffffffffu, before + run > target);
            if (past) {
                if (lane == __ffs(past) - 1) {
                    if (a.index) a.index[n] = i + lane;
                    if (a.prob) a.prob[n] = __ull2float_rn(v) / __ull2float_rn(total);
                }
                break;
            }
            before += __shfl_sync(0xffffffffu, run, 31);
        }
    }
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, int sms, cudaStream_t s) {
    (void)sms;
    static const PowTable table = [] {
        PowTable t;
        for (int j = 0; j <= 64; ++j) t.v[j] = (u64)llrintl(exp2l((long double)(j - 32) / 64) * 17592186044416.0L);
        return t;
    }();
    k_sample<<<(unsigned)a.N, kThreads, 0, s>>>(a, table);
    return cudaGetLastError();
}

}  // namespace gs
