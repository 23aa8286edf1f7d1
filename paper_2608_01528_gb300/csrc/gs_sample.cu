// gs_sample.cu -- one random entry of each score row (temperature, top-k, top-p, min-p).
//
// Top-k and top-p keep a prefix of the row in (score descending, index ascending) order, so what they keep is
// "key > t, or key == t and index <= cut", with key the score as an ordered integer; min-p is a bound on
// the weight.  The draw then runs over what is kept in index order.
//
// Weights are integers, w = round(2^41 exp((s - max) / T)) to a relative error below 2^-34.  Integer sums are
// the same in any order, and 2^19 of them fit 60 bits; fp32 sums over a large vocabulary are off by more than its
// small probabilities, and a draw whose number ends near a border would go to a neighbour.  (fp64 runs at 1/64
// of the fp32 rate here: the exponentials of 256 rows of 128,000 alone would take milliseconds.)
//
// Rows of up to 512 scores (k_sample_warp): a warp a row, scores and weights in registers; t is built bit by bit
// from the highest, by the count or weight of the keys at or above it.  Up to 4,096 (k_sample_row): a block sorts the row
// in shared memory; prefix sums of the sorted weights give t and cut.  Warps are bound by integer instructions (4,096 x 256 with
// top-p: 19 us, ALU pipe 70 % busy, 41 us if sorted; 7.6 us without top-k and top-p), the sort by shared memory (1,024 x 2,048
// with top-p: 112 us, L1 86 % busy; 18 us without).
//
// Longer rows (k_sample_wide): a cluster of up to 8 CTAs a row, re-reading the row from L2.  Pass 0: largest and
// smallest score.  Pass 1: a histogram over up to 2,048 equal steps of log weight -- counts for top-k; for top-p fp32
// weights cut to hb bits, so many that a 32-bit counter holds all scores of a CTA (20 at most, 14 for 128,000 of them), which
// bounds the running weight to 2^(2 - hb) of it.  Pass 2: the few entries of the steps in which t
// can lie (top-k: and all above) go to one CTA's list, which sorts them; the exact weight of what lies above is summed
// per warp's stretch of the row, and that of the whole row.  The draw then only looks through the one stretch in which it
// falls.  Where the list overflows (more than 4,096 ties, or top_k beyond that), and for tiny rows, one block takes
// the row by radix selects over its bits: 2 ms for a row of 131,072 to 200,000 scores, where top_k = 4,000 takes 0.1 ms.
// No unit is full: 256 rows of 128,000 fp32 scores, top-p, 196 us, issue slots 61 %, ALU 50 %, the longest waits for loads (one
// vector ahead) and fixed latencies; 64 rows of 131,071 bf16 scores, top-k 50 for all, 32 us, issue slots 45 %, block barriers,
// instruction fetches and loads.

#include <math.h>

#include <algorithm>
#include <atomic>

#include "gs_tc_ptx.cuh"
#include "gs_xattn.h"

namespace gs {
namespace {

typedef unsigned long long u64;

constexpr int kOneBits = 41;  // the largest weight is 2^41
constexpr u64 kOne = 1ull << kOneBits;
constexpr int kList = 4096;   // entries that a block sorts
constexpr int kWideThreads = 512, kWideWarps = kWideThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kBins = 2048;
constexpr int kBits = 10, kSteps = 1 << kBits;  // 2^(j / 1024) comes from a table

// 2^(j / 1024) * 2^41, rounded, from 2^(2^-k) for k = 1..10 (square roots of 2, of that, ..., as 2^62 times their value)
struct PowTable {
    u64 v[kSteps];
};
constexpr u64 isqrt_fixed(unsigned __int128 x) {  // floor(sqrt(x))
    unsigned __int128 lo = 0, hi = (unsigned __int128)1 << 64;
    while (hi - lo > 1) {
        const unsigned __int128 m = (lo + hi) / 2;
        if (m * m <= x) lo = m; else hi = m;
    }
    return (u64)lo;
}
constexpr PowTable make_pow() {
    PowTable t{};
    u64 root[kBits] = {};
    unsigned __int128 x = (unsigned __int128)2 << 124;  // 2 at 2^124: its root at 2^62
    for (int k = 0; k < kBits; ++k) {
        root[k] = isqrt_fixed(x);
        x = (unsigned __int128)root[k] << 62;
    }
    for (int j = 0; j < kSteps; ++j) {
        unsigned __int128 p = (unsigned __int128)1 << 62;
        for (int k = 0; k < kBits; ++k)
            if (j >> (kBits - 1 - k) & 1) p = p * root[k] >> 62;
        t.v[j] = (u64)((p + ((unsigned __int128)1 << 20)) >> 21);
    }
    return t;
}
__device__ constexpr PowTable g_pow = make_pow();

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
// a list entry, largest first: key, then the lower index
__device__ __forceinline__ u64 entry_of(uint32_t key, int i) { return (u64)key << 32 | (uint32_t)~(uint32_t)i; }
__device__ __forceinline__ uint32_t entry_key(u64 e) { return (uint32_t)(e >> 32); }
__device__ __forceinline__ int entry_index(u64 e) { return (int)~(uint32_t)e; }

// Halves of scores below 2^-125, and quotients by a T below 2^-126, lose bits.  Where the largest score and T are both below
// 2^-60, the row is drawn with all scores and T kUp times as large: the weights are the same, and scores so far below the
// largest that they overflow to -inf weigh 0 either way.  (Where only one of them is small, what is lost moves no weight.)
constexpr float kUp = 36893488147419103232.f;  // 2^65
__device__ __forceinline__ bool tiny_row(float most, float T) {
    constexpr float kSmall = 8.673617379884035e-19f;  // 2^-60
    return T < kSmall && fabsf(most) < kSmall;
}

// A row's settings and its weights.
struct Weigher {
    float half_max;  // max / 2 (halves: the difference of two finite scores does not overflow)
    float chi, clo;  // 2 log2(e) / T in two floats
    uint32_t top;    // the largest score's key
    bool only_top;   // a +inf, or a T so small: the largest scores weigh 1 and the others 0

    __device__ __forceinline__ void set(uint32_t top_, float T) {
        constexpr float kHi = 2.885390043258667f, kLo = 3.851926e-8f;  // 2 log2(e) = kHi + kLo to 2^-49
        top = top_;
        half_max = 0.5f * value_of(top);
        chi = __fdiv_rn(kHi, T);
        clo = __fdiv_rn(fmaf(-chi, T, kHi) + kLo, T);
        if (T == INFINITY) chi = clo = 0.f;
        only_top = value_of(top) == INFINITY || !(chi < 1e38f);
    }
    // log2 of the weight in two floats: the difference to the maximum and its product with the factor, each exact to
    // 2^-47.  The first float alone falls with the score (rounded differences and products are monotone).
    __device__ __forceinline__ float log2_hi(float x, float& lo) const {
        const float a = 0.5f * x, b = half_max;
        const float d = a - b, bb = d - a;
        const float dl = (a - (d - bb)) - (b + bb);
        const float ph = d * chi;
        lo = fmaf(d, chi, -ph) + fmaf(d, clo, dl * chi);
        return ph;
    }
    __device__ __forceinline__ float log2_only(float x) const {
        const float d = 0.5f * x - half_max;
        return d * chi;
    }
    // round(2^41 2^(ph + pl)): 2^(j/1024) from the table, 2^r - 1 of the rest |r| <= 2^-11 from its series in fp32; the
    // roundings of r, of the series and of its last product are 2^-36 each
    __device__ __forceinline__ u64 from_log2(float ph, float pl, const u64* pow) const {
        ph = fmaxf(ph, -43.f);
        const float magic = 12582912.f;  // 1.5 * 2^23: adding it rounds to an integer
        const float t = fmaf(ph, 1024.f, magic);
        const int k = __float_as_int(t) - 0x4B400000;
        const float r = fmaf(t - magic, -1.f / 1024.f, ph) + pl;
        constexpr float kUp = 2199023255552.f;  // 2^41
        const float q = r * fmaf(r, fmaf(r, 0.0555041087f * kUp, 0.2402265070f * kUp), 0.6931471806f * kUp);
        const u64 T = pow[k & (kSteps - 1)];
        const long long w = (long long)T + (((long long)(int)(T >> 11) * __float2int_rn(q)) >> 30);
        const int s = -(k >> kBits);
        return s > 0 ? (u64)((w + (1ll << (s - 1))) >> s) : (u64)w;
    }
    __device__ __forceinline__ u64 weight(float x, uint32_t key, const u64* pow) const {
        if (key == 0u) return 0ull;
        if (only_top) return key == top ? kOne : 0ull;
        float pl;
        const float ph = log2_hi(x, pl);
        return from_log2(ph, pl, pow);
    }
};

struct Settings {
    float T, top_p, u;
    int top_k;
    u64 least;  // min_p: the smallest weight that is kept
    __device__ __forceinline__ void load(const SampleArgs& a, long long n) {
        T = a.how.temperature_rows ? a.how.temperature_rows[n] : a.how.temperature;
        top_k = a.how.top_k_rows ? a.how.top_k_rows[n] : a.how.top_k;
        top_p = a.how.top_p_rows ? a.how.top_p_rows[n] : a.how.top_p;
        const float mp = a.how.min_p_rows ? a.how.min_p_rows[n] : a.how.min_p;
        least = mp > 0.f ? max(1ull, __float2ull_ru(fminf(mp, 1.f) * 2199023255552.f)) : 1ull;
        u = a.U[n];
        u = u >= 0.f ? fminf(u, 1.f - 5.9604644775390625e-8f) : 0.f;
    }
};

// floor (up: ceiling) of f * total, 0 <= f < 1, exactly
__device__ __forceinline__ u64 share_of(float f, u64 total, bool up) {
    const u64 F = __float2ull_rz(f * 18446744073709551616.f);
    const u64 hi = __umul64hi(F, total), lo = F * total;
    return hi + (up && lo != 0 ? 1 : 0);
}
// the weight that top_p asks for, of `total`
__device__ __forceinline__ u64 needed(float top_p, u64 total) {
    const u64 s = share_of(fmaxf(top_p, 0.f), total, true);
    return s > 0 ? s : 1ull;
}

__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ u64 warp_scan(u64 v) {  // inclusive
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    return v;
}
// The sum over the block, in every thread (sh: a word per warp).
__device__ __forceinline__ u64 block_sum(u64 v, u64* sh) {
    const int warps = (blockDim.x + 31) / 32;
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    u64 t = 0;
    for (int i = 0; i < warps; ++i) t += sh[i];
    return t;
}
// Exclusive prefix sum over the block's threads; total: the whole.
__device__ __forceinline__ u64 block_scan(u64 v, u64* sh, u64& total) {
    const int warp = threadIdx.x >> 5, warps = (blockDim.x + 31) / 32;
    const u64 inc = warp_scan(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 31) sh[warp] = inc;
    __syncthreads();
    u64 before = 0;
    total = 0;
    for (int i = 0; i < warps; ++i) {
        if (i < warp) before += sh[i];
        total += sh[i];
    }
    return before + inc - v;
}

// Sorts n2 (a power of two) entries, largest first (up: smallest first).  A warp's pairs of a step of up to 32 lie in
// its own 64 entries, so those steps need no block barrier.
__device__ void bitonic(u64* e, int n2, bool up) {
    __syncthreads();
    for (int size = 2; size <= n2; size <<= 1)
        for (int st = size >> 1; st; st >>= 1) {
            for (int p = threadIdx.x; p < n2 / 2; p += blockDim.x) {
                const int i = 2 * p - (p & (st - 1)), j = i + st;
                const bool desc = ((i & size) == 0) != up;
                const u64 x = e[i], y = e[j];
                if ((x < y) == desc) {
                    e[i] = y;
                    e[j] = x;
                }
            }
            if (st > 32 || (st == 1 && size >= 64) || n2 / 2 > (int)blockDim.x)
                __syncthreads();
            else
                __syncwarp();
        }
    __syncthreads();
}

// What is kept of sorted entries (a block): the first n_top of them for top_k, then the shortest run whose weight, added to
// `above` (of larger entries elsewhere), reaches what top_p asks for.  total: of everything top-k kept, or 0: to be
// summed here.  Returns the last kept entry.
__device__ u64 last_kept(const u64* e, int n, const Weigher& w, const u64* pow, float top_p, u64 above, u64 total, u64* sh,
                         u64* found) {
    const int per = (n + blockDim.x - 1) / blockDim.x;
    const int i0 = min(n, (int)threadIdx.x * per), i1 = min(n, i0 + per);
    u64 mine = 0, all;
    for (int i = i0; i < i1; ++i) mine += w.weight(value_of(entry_key(e[i])), entry_key(e[i]), pow);
    u64 run = above + block_scan(mine, sh, all);
    if (total == 0) total = all;
    if (threadIdx.x == 0) *found = e[n - 1];
    __syncthreads();
    if (top_p < 1.f) {
        const u64 need = needed(top_p, total);
        if (run < need && run + mine >= need)
            for (int i = i0; i < i1; ++i) {
                run += w.weight(value_of(entry_key(e[i])), entry_key(e[i]), pow);
                if (run >= need) {
                    *found = e[i];
                    break;
                }
            }
    }
    __syncthreads();
    return *found;
}

__device__ __forceinline__ void answer(const SampleArgs& a, long long n, int i, u64 w, u64 total) {
    if (a.index) a.index[n] = i;
    if (a.prob) a.prob[n] = total ? __ull2float_rn(w) / __ull2float_rn(total) : 0.f;
}

// ----------------------------------------------------------------- rows of up to 32 E scores: a warp each
// Sum over the warp of numbers below 2^47.
__device__ __forceinline__ u64 warp_total(u64 v) {
    const u64 lo = __reduce_add_sync(0xffffffffu, (unsigned)v & 0xffffffu);
    const u64 hi = __reduce_add_sync(0xffffffffu, (unsigned)(v >> 24));
    return lo + (hi << 24);
}

template <int E>
__global__ void __launch_bounds__(128) k_sample_warp(const SampleArgs a, long long n0) {
    const long long n = n0 + (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (n >= a.N) return;
    const int lane = threadIdx.x & 31, M = a.M;
    const void* row = static_cast<const char*>(a.S) + n * a.lds * (a.bf16 ? 2 : 4);
    Settings st;
    st.load(a, n);
    uint32_t key[E], top = 0, low = 0xffffffffu;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int i = lane + 32 * e;
        key[e] = i < M ? key_of(load_score(row, a.bf16, i)) : 0u;
        top = max(top, key[e]);
        low = key[e] ? min(low, key[e]) : low;
    }
    top = __reduce_max_sync(0xffffffffu, top);
    low = __reduce_min_sync(0xffffffffu, low);
    if (top == 0u || !(st.T > 0.f)) {
        unsigned first = 0x7fffffffu;
#pragma unroll
        for (int e = E - 1; e >= 0; --e) first = key[e] == top ? lane + 32 * e : first;
        first = __reduce_min_sync(0xffffffffu, first);
        if (lane == 0) answer(a, n, top ? (int)first : -1, top ? 1 : 0, top ? 1 : 0);
        return;
    }
    if (tiny_row(value_of(top), st.T)) {
        st.T *= kUp;
        low = 0xffffffffu;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            key[e] = key[e] ? key_of(value_of(key[e]) * kUp) : 0u;
            low = key[e] ? min(low, key[e]) : low;
        }
        top = key_of(value_of(top) * kUp);
        low = __reduce_min_sync(0xffffffffu, low);
    }
    Weigher w;
    w.set(top, st.T);
    u64 wt[E];
#pragma unroll
    for (int e = 0; e < E; ++e) wt[e] = w.weight(value_of(key[e]), key[e], g_pow.v);
    // t: the largest key with enough at or above it; bits above the highest in which keys differ are the same in all
    uint32_t t = 1;
    int ties = 0x7fffffff;  // kept ones of the keys equal to t, in index order
    const int bits = 32 - __clz(top ^ low);
    const uint32_t common = bits < 32 ? top >> bits << bits : 0u;
    if (st.top_k >= 1 && st.top_k < M) {
        auto count = [&](uint32_t from) {
            int c = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) c += key[e] >= from;
            return __reduce_add_sync(0xffffffffu, c);
        };
        if (count(1) > st.top_k) {
            t = common;
            for (int b = bits - 1; b >= 0; --b)
                if (count(t | 1u << b) >= st.top_k) t |= 1u << b;
            ties = st.top_k - (t == 0xffffffffu ? 0 : count(t + 1));
        }
    }
    auto rank_kept = [&](int e, int& before) {  // whether entry e is kept among the ties; e in ascending order
        const unsigned m = __ballot_sync(0xffffffffu, key[e] == t);
        const bool in = key[e] > t || (key[e] == t && before + __popc(m & ((1u << lane) - 1u)) < ties);
        before += __popc(m);
        return in;
    };
    if (ties != 0x7fffffff) {  // what top-k drops weighs nothing from here on
        int before = 0;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (!rank_kept(e, before)) {
                wt[e] = 0;
                key[e] = 0;
            }
        t = 1;
        ties = 0x7fffffff;
    }
    if (st.top_p < 1.f) {
        auto weigh = [&](uint32_t from) {
            u64 s = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) s += key[e] >= from ? wt[e] : 0ull;
            return warp_total(s);
        };
        const u64 need = needed(st.top_p, weigh(1));
        t = common;
        for (int b = bits - 1; b >= 0; --b)
            if (weigh(t | 1u << b) >= need) t |= 1u << b;
        const u64 above = t == 0xffffffffu ? 0 : weigh(t + 1), one = w.weight(value_of(t), t, g_pow.v);
        ties = (int)min((need - above + one - 1) / max(one, 1ull), 0x7ffffffeull);
    }
    u64 total = 0;
    {
        int before = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (!rank_kept(e, before) || wt[e] < st.least) wt[e] = 0;
            total += wt[e];
        }
    }
    total = warp_total(total);
    const u64 target = share_of(st.u, total, false);
    u64 before = 0;
    bool found = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (found) continue;
        const u64 all = warp_total(wt[e]);
        if (before + all > target) {
            const u64 run = before + warp_scan(wt[e]);
            const unsigned past = __ballot_sync(0xffffffffu, run > target);
            if (lane == __ffs(past) - 1) answer(a, n, lane + 32 * e, wt[e], total);
            found = true;
        }
        before += all;
    }
}

// ----------------------------------------------------------------- rows of up to kList scores: a block each
// (a function of its own: unrolled into the kernel it cost every row 2 to 5 %)
__device__ __noinline__ void scale_up(uint32_t* keys, int M) {
    for (int i = threadIdx.x; i < M; i += blockDim.x) keys[i] = keys[i] ? key_of(value_of(keys[i]) * kUp) : 0u;
    __syncthreads();
}

__global__ void k_sample_row(const SampleArgs a, long long n0, int n2) {
    extern __shared__ u64 list[];  // n2 sorted entries, then M keys
    uint32_t* keys = reinterpret_cast<uint32_t*>(list + n2);
    __shared__ u64 sh[32];
    __shared__ u64 found;
    const long long n = n0 + blockIdx.x;
    const int tid = threadIdx.x, M = a.M;
    const u64* pow = g_pow.v;
    const void* row = static_cast<const char*>(a.S) + n * a.lds * (a.bf16 ? 2 : 4);
    Settings st;
    st.load(a, n);
    u64 best = 0;
    for (int i = tid; i < M; i += blockDim.x) {
        const uint32_t k = key_of(load_score(row, a.bf16, i));
        keys[i] = k;
        best = max(best, entry_of(k, i));
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if ((tid & 31) == 0) sh[tid >> 5] = best;
    __syncthreads();
    for (int i = 0; i < (int)(blockDim.x + 31) / 32; ++i) best = max(best, sh[i]);
    uint32_t top = entry_key(best);
    if (top == 0u || !(st.T > 0.f)) {
        if (tid == 0) answer(a, n, top ? entry_index(best) : -1, top ? 1 : 0, top ? 1 : 0);
        return;
    }
    if (tiny_row(value_of(top), st.T)) {
        st.T *= kUp;
        top = key_of(value_of(top) * kUp);
        scale_up(keys, M);
    }
    Weigher w;
    w.set(top, st.T);
    u64 last = 1ull << 32;  // everything with a key
    const bool by_k = st.top_k >= 1 && st.top_k < M;
    if (by_k || st.top_p < 1.f) {
        for (int i = tid; i < n2; i += blockDim.x) list[i] = i < M ? entry_of(keys[i], i) : 0ull;
        bitonic(list, n2, false);
        last = last_kept(list, by_k ? st.top_k : M, w, pow, st.top_p, 0, 0, sh, &found);
        last = max(last, 1ull << 32);
    }
    // in index order
    const int per = (M + blockDim.x - 1) / blockDim.x;
    const int i0 = min(M, tid * per), i1 = min(M, i0 + per);
    auto kept = [&](int i) {
        const uint32_t k = keys[i];
        if (entry_of(k, i) < last) return 0ull;
        const u64 v = w.weight(value_of(k), k, pow);
        return v >= st.least ? v : 0ull;
    };
    u64 mine = 0, total;
    for (int i = i0; i < i1; ++i) mine += kept(i);
    u64 run = block_scan(mine, sh, total);
    const u64 target = share_of(st.u, total, false);
    if (run <= target && run + mine > target)
        for (int i = i0; i < i1; ++i) {
            const u64 v = kept(i);
            run += v;
            if (run > target) {
                answer(a, n, i, v, total);
                break;
            }
        }
}

// ----------------------------------------------------------------- longer rows: a cluster each
struct Wide {
    u64 pow[kSteps];
    u64 list[kList];
    u64 seg[kMaxCluster * kWideWarps];  // rank 0: kept weight of every warp's stretch
    u64 above[kMaxCluster];             // rank 0: weight above the list, of each CTA
    u64 total[kMaxCluster];             // and of all its scores
    u64 range[kMaxCluster];             // every CTA: each CTA's smallest and largest score
    float2 ends[kWideWarps];
    alignas(16) uint32_t hist[kBins];
    u64 sh[kWideWarps];
    u64 found[3];
    unsigned count;                     // rank 0: entries sent to the list
};

__device__ __forceinline__ void st_remote_u64(uint32_t addr, u64 v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ uint4 ld_remote_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ unsigned add_remote(uint32_t addr, unsigned v) {
    unsigned r;
    asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(r) : "r"(addr), "r"(v) : "memory");
    return r;
}

// The row in a warp's stretch [v0, v1) of vectors of 16 bytes, f(index, score); `off`: scores between the 16-byte
// boundary at or before the row's start and the start.  The next vector is on its way while one is worked on.
template <typename F>
__device__ __forceinline__ void for_scores(const void* row, bool bf16, int M, int off, int v0, int v1, F&& f) {
    const int lane = threadIdx.x & 31, V = bf16 ? 8 : 4;
    const char* p = static_cast<const char*>(row) - off * (16 / V);
    auto inside = [&](int v) { return v * V - off >= 0 && v * V - off + V <= M; };
    uint4 next = make_uint4(0, 0, 0, 0);
    if (v0 + lane < v1 && inside(v0 + lane)) next = __ldg(reinterpret_cast<const uint4*>(p) + v0 + lane);
    for (int v = v0 + lane; v < v1; v += 32) {
        const uint4 x = next;
        if (v + 32 < v1 && inside(v + 32)) next = __ldg(reinterpret_cast<const uint4*>(p) + v + 32);
        const int i = v * V - off;
        if (inside(v)) {
            const uint32_t q[4] = {x.x, x.y, x.z, x.w};
            if (bf16) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f(i + 2 * e, __uint_as_float(q[e] << 16));
                    f(i + 2 * e + 1, __uint_as_float(q[e] & 0xffff0000u));
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) f(i + e, __uint_as_float(q[e]));
            }
        } else {
            for (int e = 0; e < V; ++e)
                if (i + e >= 0 && i + e < M) f(i + e, load_score(row, bf16, i + e));
        }
    }
}

// One block, any row: t and cut by radix selects over the keys, 8 bits a pass, by counts or weights.
// Scores are taken `up` times as large.
__device__ void radix_row(const SampleArgs& a, long long n, const void* row, const Settings& st, const Weigher& w, float up, Wide& m) {
    u64* hist = m.list;  // 256
    const u64* pow = m.pow;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, M = a.M;
    auto key_at = [&](int i) { return key_of(load_score(row, a.bf16, i) * up); };
    auto weight = [&](uint32_t k) { return w.weight(value_of(k), k, pow); };
    auto select = [&](bool by_weight, u64 need, u64& above) {
        uint32_t prefix = 0;
        above = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            for (int i = tid; i < 256; i += kWideThreads) hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < M; i += kWideThreads) {
                const uint32_t k = key_at(i);
                if (k == 0u || (shift < 24 && (k >> (shift + 8)) != (prefix >> (shift + 8)))) continue;
                atomicAdd(&hist[(k >> shift) & 255u], by_weight ? weight(k) : 1ull);
            }
            __syncthreads();
            if (tid == 0) {
                int b = 255;
                u64 run = above;
                while (b > 0 && run + hist[b] < need) run += hist[b--];
                m.found[0] = (u64)b;
                m.found[1] = run;
            }
            __syncthreads();
            prefix |= (uint32_t)m.found[0] << shift;
            above = m.found[1];
        }
        return prefix;
    };
    uint32_t t = 1;  // kept: key > t, or key == t and among the first `ties` in index order
    u64 ties = ~0ull, above;
    if (st.top_k >= 1 && st.top_k < M) {
        u64 valid = 0;
        for (int i = tid; i < M; i += kWideThreads) valid += key_at(i) != 0u;
        if ((u64)st.top_k < block_sum(valid, m.sh)) {
            t = select(false, (u64)st.top_k, above);
            ties = (u64)st.top_k - above;
        }
    }
    if (st.top_p < 1.f) {
        u64 s = 0, eq = 0;
        for (int i = tid; i < M; i += kWideThreads) {
            const uint32_t k = key_at(i);
            if (k > t) s += weight(k);
            eq += k == t;
        }
        s = block_sum(s, m.sh);
        eq = block_sum(eq, m.sh);
        const u64 need = needed(st.top_p, s + weight(t) * (eq < ties ? eq : ties));
        t = select(true, need, above);
        const u64 wt = weight(t);
        ties = wt ? (need - above + wt - 1) / wt : ~0ull;
    }
    const int seg = (M + kWideWarps - 1) / kWideWarps;
    const int s0 = min(M, warp * seg), s1 = min(M, s0 + seg);
    int cut = M - 1;  // the last kept tie
    if (ties != ~0ull) {
        u64 cnt = 0;
        for (int i = s0 + lane; i < s1; i += 32) cnt += key_at(i) == t;
        cnt = warp_sum(cnt);
        __syncthreads();
        if (lane == 0) m.sh[warp] = cnt;
        if (tid == 0) m.found[2] = (u64)(M - 1);
        __syncthreads();
        u64 before = 0;
        for (int i = 0; i < warp; ++i) before += m.sh[i];
        if (before < ties && before + cnt >= ties)
            for (int i = s0; i < s1; i += 32) {
                const bool eq = i + lane < s1 && key_at(i + lane) == t;
                const unsigned b = __ballot_sync(0xffffffffu, eq);
                if (before + __popc(b) >= ties) {
                    if (eq && before + __popc(b & ((2u << lane) - 1u)) == ties) m.found[2] = (u64)(i + lane);
                    break;
                }
                before += __popc(b);
            }
        __syncthreads();
        cut = (int)m.found[2];
    }
    auto kept = [&](int i) {
        const uint32_t k = key_at(i);
        const u64 v = k > t || (k == t && i <= cut) ? weight(k) : 0ull;
        return v >= st.least ? v : 0ull;
    };
    u64 mine = 0, total = 0, before = 0;
    for (int i = s0 + lane; i < s1; i += 32) mine += kept(i);
    mine = warp_sum(mine);
    __syncthreads();
    if (lane == 0) m.sh[warp] = mine;
    __syncthreads();
    for (int i = 0; i < kWideWarps; ++i) {
        if (i < warp) before += m.sh[i];
        total += m.sh[i];
    }
    const u64 target = share_of(st.u, total, false);
    if (before <= target && before + mine > target)
        for (int i = s0; i < s1; i += 32) {
            const u64 v = i + lane < s1 ? kept(i + lane) : 0ull;
            const u64 run = before + warp_scan(v);
            const unsigned past = __ballot_sync(0xffffffffu, run > target);
            if (past) {
                if (lane == __ffs(past) - 1) answer(a, n, i + lane, v, total);
                break;
            }
            before = __shfl_sync(0xffffffffu, run, 31);
        }
}

__global__ void __launch_bounds__(kWideThreads, 2) k_sample_wide(const SampleArgs a, long long n0, int G) {
    extern __shared__ __align__(16) uint8_t wide_smem[];
    Wide& m = *reinterpret_cast<Wide*>(wide_smem);
    const int rank = (int)(blockIdx.x % (unsigned)G);
    const long long n = n0 + blockIdx.x / (unsigned)G;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, M = a.M;
    const int esize = a.bf16 ? 2 : 4, V = 16 / esize;
    const void* row = static_cast<const char*>(a.S) + n * a.lds * esize;
    const int off = (int)((uintptr_t)row % 16) / esize;
    const int nv = (M + off + V - 1) / V;
    const int per = ((nv + G * kWideWarps - 1) / (G * kWideWarps) + 31) / 32 * 32;  // vectors of a warp's stretch
    const int v0 = min(nv, (rank * kWideWarps + warp) * per), v1 = min(nv, v0 + per);
    auto remote = [&](const void* p, int r) { return ptx::mapa_shared(ptx::smem_u32(p), (uint32_t)r); };

    for (int i = tid; i < kSteps; i += kWideThreads) m.pow[i] = g_pow.v[i];
    for (int i = tid; i < kBins; i += kWideThreads) m.hist[i] = 0;
    if (tid == 0) m.count = 0;
    Settings st;
    st.load(a, n);

    // pass 0: the largest and the smallest score that can be drawn
    float hi = -INFINITY, lo = INFINITY;
    for_scores(row, a.bf16, M, off, v0, v1, [&](int, float x) {
        hi = fmaxf(hi, x);
        lo = fminf(lo, x > -INFINITY ? x : INFINITY);
    });
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    }
    if (lane == 0) m.ends[warp] = make_float2(hi, lo);
    __syncthreads();
    ptx::cluster_sync_all();  // every CTA of the cluster runs from here on
    if (warp == 0) {
        const float2 e = m.ends[lane % kWideWarps];
        hi = e.x;
        lo = e.y;
#pragma unroll
        for (int o = 8; o; o >>= 1) {
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        }
        if (lane < G) st_remote_u64(remote(&m.range[rank], lane), (u64)__float_as_uint(lo) << 32 | __float_as_uint(hi));
    }
    ptx::cluster_sync_all();
    hi = -INFINITY;
    lo = INFINITY;
    for (int i = 0; i < G; ++i) {
        hi = fmaxf(hi, __uint_as_float((uint32_t)m.range[i]));
        lo = fminf(lo, __uint_as_float((uint32_t)(m.range[i] >> 32)));
    }
    const uint32_t top = key_of(hi);
    if (top == 0u) {  // (no CTA touches another's memory any more)
        if (rank == 0 && tid == 0) answer(a, n, -1, 0, 0);
        return;
    }
    if (!(st.T > 0.f)) {
        unsigned first = 0x7fffffffu;
        for_scores(row, a.bf16, M, off, v0, v1, [&](int i, float x) { first = x == hi ? min(first, (unsigned)i) : first; });
        first = __reduce_min_sync(0xffffffffu, first);
        if (lane == 0) st_remote_u64(remote(&m.seg[rank * kWideWarps + warp], 0), first);
        ptx::cluster_sync_all();
        if (rank == 0 && warp == 0) {
            for (int i = lane; i < G * kWideWarps; i += 32) first = min(first, (unsigned)m.seg[i]);
            first = __reduce_min_sync(0xffffffffu, first);
            if (lane == 0) answer(a, n, (int)first, 1, 1);
        }
        return;
    }
    const float up = tiny_row(hi, st.T) ? kUp : 1.f;
    st.T *= up;
    Weigher w;
    w.set(key_of(hi * up), st.T);
    const bool by_k = st.top_k >= 1 && st.top_k < M, by_p = st.top_p < 1.f;
    if (w.only_top || up != 1.f) {  // (the passes below take scores as they are)
        if (rank == 0) radix_row(a, n, row, st, w, up, m);
        return;
    }
    u64 last = 1ull << 32;  // entries from this one on are kept
    u64 mine = 0;           // kept weight of this thread's scores
    if (!by_k && !by_p) {
        for_scores(row, a.bf16, M, off, v0, v1, [&](int, float x) {
            float pl;
            const float ph = w.log2_hi(x, pl);
            const u64 v = w.from_log2(ph, pl, m.pow);
            mine += v >= st.least ? v : 0ull;
        });
    } else {
        // steps of 2^-ks of log2 weight, from the largest score down to the smallest or to where weights vanish
        float pl;
        const float range = fminf(-w.log2_hi(lo, pl), 43.f);
        int ks = 5;
        while (ks < 20 && range * (float)(2 << ks) < (float)(kBins - 8)) ++ks;
        const float steps = (float)(1 << ks);
        // rounded to the nearest step by adding 1.5 * 2^23 (what cannot be drawn falls into the last one)
        auto step = [&](float ph) { return __float_as_int(fmaf(-fmaxf(ph, -range), steps, 12582912.f)) - 0x4B400000; };
        // bits of a histogram weight: a counter may have to hold all scores of this CTA
        const int hb = min(20, __clz(per * kWideWarps * V - 1) - 1);
        for_scores(row, a.bf16, M, off, v0, v1, [&](int, float x) {
            const float ph = fmaxf(w.log2_only(x), -range);
            const int b = step(ph);
            // the weight in units of 2^-hb of the step's octave b >> ks: between 2^(hb - 1.03) and 2^(hb + 0.03)
            const uint32_t v = by_k ? 1u : (uint32_t)__int_as_float(__float_as_int(ex2(ph)) + (((b >> ks) + hb) << 23));
            atomicAdd(&m.hist[b], x > -INFINITY ? v : 0u);
        });
        __syncthreads();
        ptx::cluster_sync_all();
        // the steps [b0, b1] in which the last kept entry lies
        u64 part[kBins / kWideThreads], sum = 0, all;
        constexpr int kPer = kBins / kWideThreads;
        static_assert(kPer == 4, "16 bytes of each histogram a thread");
        u64 wide[kPer] = {0, 0, 0, 0};
        for (int r = 0; r < G; ++r) {
            const uint4 v = ld_remote_v4(remote(&m.hist[tid * kPer], r));
            wide[0] += v.x;
            wide[1] += v.y;
            wide[2] += v.z;
            wide[3] += v.w;
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int up = kOneBits - hb - ((tid * kPer + e) >> ks);
            part[e] = by_k ? wide[e] : up >= 0 ? wide[e] << up : wide[e] >> -up;
            sum += part[e];
        }
        if (tid == 0) m.found[0] = m.found[1] = kBins - 1;
        u64 run = block_scan(sum, m.sh, all);
        // Counts are exact.  Weights are cut down (by less than 2^(1.03 - hb), and by a unit where a step is shifted down) and off
        // by the 2^-18 of an fp32 exponent up to 43 and its exponential.
        auto least = [&](u64 r) { return by_k ? r : r - (r >> 16); };
        auto most = [&](u64 r) { return by_k || r == 0 ? r : r + (r >> (hb - 2)) + (r >> 15) + kBins; };
        const u64 need0 = by_k ? (u64)st.top_k : needed(st.top_p, least(all));
        const u64 need1 = by_k ? (u64)st.top_k : needed(st.top_p, most(all));
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const u64 next = run + part[e];
            if (most(run) < need0 && most(next) >= need0) m.found[0] = tid * kPer + e;
            if (least(run) < need1 && least(next) >= need1) m.found[1] = tid * kPer + e;
            run = next;
        }
        __syncthreads();
        const int b0 = (int)m.found[0], b1 = (int)m.found[1];
        // pass 2: the list, the exact weight of what lies above it and of the whole row
        const uint32_t list0 = remote(m.list, 0), count0 = remote(&m.count, 0);
        u64 above = 0, total = 0;
        auto send = [&](int i, float x) {
            if (!(x > -INFINITY)) return;
            const unsigned at = add_remote(count0, 1u);
            if (at < (unsigned)kList) st_remote_u64(list0 + at * 8u, entry_of(key_of(x), i));
        };
        if (by_k) {
            for_scores(row, a.bf16, M, off, v0, v1, [&](int i, float x) {
                if (step(w.log2_only(x)) <= b1) send(i, x);
            });
        } else {
            for_scores(row, a.bf16, M, off, v0, v1, [&](int i, float x) {
                float pl;
                const float ph = w.log2_hi(x, pl);
                const u64 v = w.from_log2(ph, pl, m.pow);
                const int b = step(ph);
                total += v;
                above += b < b0 ? v : 0ull;
                mine += b < b0 && v >= st.least ? v : 0ull;
                if (b >= b0 && b <= b1) send(i, x);
            });
        }
        if (!by_k) {
            above = block_sum(above, m.sh);
            total = block_sum(total, m.sh);
            if (tid == 0) {
                st_remote_u64(remote(&m.above[rank], 0), above);
                st_remote_u64(remote(&m.total[rank], 0), total);
            }
        }
        mine = warp_sum(mine);
        if (lane == 0) st_remote_u64(remote(&m.seg[rank * kWideWarps + warp], 0), mine);
        ptx::cluster_sync_all();
        if (rank != 0) return;
        if (m.count > (unsigned)kList) {
            radix_row(a, n, row, st, w, 1.f, m);
            return;
        }
        const int nl = (int)m.count;
        int n2 = 64;
        while (n2 < nl) n2 <<= 1;
        for (int i = nl + tid; i < n2; i += kWideThreads) m.list[i] = 0;
        bitonic(m.list, n2, false);
        if (by_k) {
            const int nk = min(nl, st.top_k);
            last = last_kept(m.list, nk, w, m.pow, st.top_p, 0, 0, m.sh, &m.found[0]);
            // the kept entries in index order, weight below the index (19 + 42 bits)
            for (int i = tid; i < n2; i += kWideThreads) {
                const u64 e = m.list[i];
                u64 v = i < nk && e >= last ? w.weight(value_of(entry_key(e)), entry_key(e), m.pow) : 0ull;
                v = v >= st.least ? v : 0ull;
                m.list[i] = (u64)entry_index(e) << 42 | v;
                if (v == 0ull) m.list[i] = ~0ull << 42;  // behind the others, of no weight
            }
            bitonic(m.list, n2, true);
            const int pt = (n2 + kWideThreads - 1) / kWideThreads;
            const int i0 = min(n2, tid * pt), i1 = min(n2, i0 + pt);
            constexpr u64 kMask = (1ull << 42) - 1;
            u64 s = 0, whole;
            for (int i = i0; i < i1; ++i) s += m.list[i] & kMask;
            u64 at = block_scan(s, m.sh, whole);
            const u64 target = share_of(st.u, whole, false);
            if (at <= target && at + s > target)
                for (int i = i0; i < i1; ++i) {
                    at += m.list[i] & kMask;
                    if (at > target) {
                        answer(a, n, (int)(m.list[i] >> 42), m.list[i] & kMask, whole);
                        break;
                    }
                }
            return;
        }
        u64 over = 0;
        total = 0;
        for (int i = 0; i < G; ++i) {
            over += m.above[i];
            total += m.total[i];
        }
        last = last_kept(m.list, nl, w, m.pow, st.top_p, over, total, m.sh, &m.found[0]);
        // the list's kept entries join their stretches
        for (int i = tid; i < nl; i += kWideThreads) {
            const u64 e = m.list[i];
            if (e < last) continue;
            const u64 v = w.weight(value_of(entry_key(e)), entry_key(e), m.pow);
            if (v >= st.least) atomicAdd(&m.seg[((entry_index(e) + off) / V) / per], v);
        }
        __syncthreads();
    }
    if (!by_k && !by_p) {
        mine = warp_sum(mine);
        if (lane == 0) st_remote_u64(remote(&m.seg[rank * kWideWarps + warp], 0), mine);
        ptx::cluster_sync_all();
        if (rank != 0) return;
    }
    // rank 0: the stretch in which u * total falls, then the score in it
    const int segs = G * kWideWarps;
    const u64 sw = tid < segs ? m.seg[tid] : 0ull;
    u64 total;
    const u64 before = block_scan(sw, m.sh, total);
    const u64 target = share_of(st.u, total, false);
    if (before <= target && before + sw > target) {
        m.found[0] = (u64)tid;
        m.found[1] = before;
    }
    __syncthreads();
    const int sg = (int)m.found[0];
    const int e0 = max(0, sg * per * V - off), e1 = min(M, (sg + 1) * per * V - off);
    const int pt = (e1 - e0 + kWideThreads - 1) / kWideThreads;
    const int i0 = min(e1, e0 + tid * pt), i1 = min(e1, i0 + pt);
    auto kept = [&](int i) {
        const float x = load_score(row, a.bf16, i);
        const uint32_t k = key_of(x);
        if (entry_of(k, i) < last) return 0ull;
        const u64 v = w.weight(x, k, m.pow);
        return v >= st.least ? v : 0ull;
    };
    u64 s = 0, whole;
    for (int i = i0; i < i1; ++i) s += kept(i);
    u64 at = m.found[1] + block_scan(s, m.sh, whole);
    if (at <= target && at + s > target)
        for (int i = i0; i < i1; ++i) {
            const u64 v = kept(i);
            at += v;
            if (at > target) {
                answer(a, n, i, v, total);
                break;
            }
        }
}

std::atomic<bool> g_attr[64];

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, int sms, int device, cudaStream_t s) {
    if (device < 0 || device >= 64) return cudaErrorInvalidDevice;
    constexpr long long kRows = 1 << 27;  // rows of a launch
    if (!g_attr[device]) {
        cudaError_t e = cudaFuncSetAttribute(k_sample_row, cudaFuncAttributeMaxDynamicSharedMemorySize, kList * 12);
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(k_sample_wide, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Wide));
        if (e != cudaSuccess) return e;
        g_attr[device] = true;
    }
    if (a.M <= 512) {
        for (long long n = 0; n < a.N; n += kRows) {
            const unsigned grid = (unsigned)((std::min(kRows, a.N - n) + 3) / 4);
            if (a.M <= 64)
                k_sample_warp<2><<<grid, 128, 0, s>>>(a, n);
            else if (a.M <= 128)
                k_sample_warp<4><<<grid, 128, 0, s>>>(a, n);
            else if (a.M <= 256)
                k_sample_warp<8><<<grid, 128, 0, s>>>(a, n);
            else
                k_sample_warp<16><<<grid, 128, 0, s>>>(a, n);
            cudaError_t e = cudaGetLastError();
            if (e != cudaSuccess) return e;
        }
        return cudaSuccess;
    }
    if (a.M <= kList) {
        int n2 = 64;
        while (n2 < a.M) n2 <<= 1;
        const int threads = std::min(kWideThreads, n2 / 2);
        const size_t smem = (size_t)n2 * 8 + ((size_t)a.M * 4 + 7) / 8 * 8;
        for (long long n = 0; n < a.N; n += kRows) {
            k_sample_row<<<(unsigned)std::min(kRows, a.N - n), threads, smem, s>>>(a, n, n2);
            cudaError_t e = cudaGetLastError();
            if (e != cudaSuccess) return e;
        }
        return cudaSuccess;
    }
    // CTAs a row: as many as all rows' CTAs run at once (two a multiprocessor), with 8,192 scores each or more; up to 2^18
    // (the histogram's counters).  A cluster's waits for one another cost more than they give where rows alone fill the GPU:
    // rows of 131,072, top-p: 64 in 1 / 2 / 4 / 8 CTAs 122 / 73 / 66 / 82 us, 256 in 1 / 2 / 4 207 / 213 / 221 us.
    int G = 1;
    while (G < kMaxCluster && (a.M / G > 1 << 18 || (a.N * G * 2 <= 2ll * sms && a.M / G >= 16384))) G <<= 1;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)G;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.blockDim = dim3(kWideThreads);
    cfg.dynamicSmemBytes = sizeof(Wide);
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    for (long long n = 0; n < a.N; n += kRows) {
        cfg.gridDim = dim3((unsigned)(std::min(kRows, a.N - n) * G));
        cudaError_t e = cudaLaunchKernelEx(&cfg, k_sample_wide, a, n, G);
        if (e != cudaSuccess) return e;
    }
    return cudaGetLastError();
}

}  // namespace gs
