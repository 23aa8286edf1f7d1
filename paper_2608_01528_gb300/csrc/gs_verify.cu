// gs_verify.cu -- drafted tokens checked against the target's probabilities.
//
// Draft x_i is kept while U_i D_i(x_i) < P_i(x_i).  The token behind the kept ones is drawn from max(P_i - D_i, 0) of the first
// draft that is not kept, or from the target's row behind the last one.  Only that one row of P (and of D) is read: by a cluster of
// up to 8 CTAs, a contiguous piece a warp.  The pieces' sums meet in shared memory across the cluster, and the warp whose piece holds the
// drawn point looks through it again (by then in L1 or L2).
//
// Weights are integers in units of 2^-44, rint(p 2^44) - rint(d 2^44), so that every sum is exact in any order.  Each is off by a unit at
// most, M of them shift the drawn point by up to M 2^-44 of their sum: what is lost where little is left of P - D.  A conversion in two steps of
// fp32, p 2^21 = hi + lo 2^-23 with hi and lo read off the mantissas of sums with 1.5 2^23, costs four FMAs or adds; conversions to 64-bit
// integers run at an eighth of that rate.

#include <algorithm>

#include "gs_paged.h"
#include "gs_tc_ptx.cuh"

namespace gs {
namespace {

using u64 = unsigned long long;

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kMaxCtas = 8, kResident = 8;  // CTAs of a row; of a multiprocessor
constexpr int kAhead = 2;                   // 16-byte loads of a lane, of P and of D each, that go together
constexpr float kHigh = 2097152.f, kLow = 8388608.f, kMagic = 12582912.f;  // 2^21, 2^23, 1.5 * 2^23
constexpr int kMagicBits = 0x4B400000;

// hi 2^23 + lo units, the sums of p's parts (kMagicBits over in each term), less those of d
__device__ __forceinline__ void split(float p, int& hi, int& lo) {  // p in [0, 1]
    const float a = fmaf(p, kHigh, kMagic), t = a - kMagic;
    hi = __float_as_int(a);
    lo = __float_as_int(fmaf(fmaf(p, kHigh, -t), kLow, kMagic));  // (the inner one is exact)
}

// What the rows weigh: P alone, P without one entry, or P less D.
enum Rest { kTarget, kWithout, kLess };
struct Row {
    const void *p, *d;
    int rest, x;
};
template <typename T>
__device__ __forceinline__ float read(const void* row, int j) {
    if constexpr (sizeof(T) == 4)
        return __ldg(static_cast<const float*>(row) + j);
    else
        return __uint_as_float((uint32_t)__ldg(static_cast<const unsigned short*>(row) + j) << 16);
}
// NaN counts as 0, what is above 1 as 1; below d nothing is left, d's parts less d's parts
__device__ __forceinline__ void add(float p, float d, int& hi, int& lo) {
    p = __saturatef(p);
    int ph, pl, dh, dl;
    split(p, ph, pl);
    split(fminf(__saturatef(d), p), dh, dl);
    hi += ph - dh;
    lo += pl - dl;
}
__device__ __forceinline__ void add(float p, int& hi, int& lo) {
    int ph, pl;
    split(__saturatef(p), ph, pl);
    hi += ph - kMagicBits;
    lo += pl - kMagicBits;
}
__device__ __forceinline__ long long units(int hi, int lo) { return (long long)hi * 8388608ll + lo; }
template <typename T>
__device__ __forceinline__ u64 weight(const Row& r, int j) {
    const float p = read<T>(r.p, j), d = r.rest == kLess ? read<T>(r.d, j) : r.rest == kWithout && j == r.x ? 1.f : 0.f;
    int hi = 0, lo = 0;
    add(p, d, hi, lo);
    return (u64)units(hi, lo);
}

// What 16 bytes of P (and D) weigh, added to hi and lo.
template <typename T, bool LESS>
__device__ __forceinline__ void add16(const uint4& a, const uint4& b, int& hi, int& lo) {
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
    auto one = [&](uint32_t u, uint32_t v) {
        if constexpr (LESS)
            add(__uint_as_float(u), __uint_as_float(v), hi, lo);
        else
            add(__uint_as_float(u), hi, lo);
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) {
            one(x[e], y[e]);
        } else {
            one(x[e] << 16, y[e] << 16);
            one(x[e] & 0xffff0000u, y[e] & 0xffff0000u);
        }
    }
}
// Steps of 16 bytes at p (and d), `step` entries apart: kAhead on their way while as many are added.
template <typename T, bool LESS>
__device__ __forceinline__ long long sum_steps(const T* p, const T* d, int steps, int step) {
    long long sum = 0;
    uint4 a[2][kAhead], b[2][kAhead];
    auto load = [&](uint4(&x)[kAhead], uint4(&y)[kAhead], int w) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const bool in = w + u < steps;
            x[u] = in ? __ldg(reinterpret_cast<const uint4*>(p + (long long)(w + u) * step)) : make_uint4(0, 0, 0, 0);
            y[u] = LESS && in ? __ldg(reinterpret_cast<const uint4*>(d + (long long)(w + u) * step)) : make_uint4(0, 0, 0, 0);
        }
    };
    load(a[0], b[0], 0);
    for (int w = 0; w < steps; w += 2 * kAhead) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            load(a[k ^ 1], b[k ^ 1], w + (k + 1) * kAhead);
            int hi = 0, lo = 0;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) add16<T, LESS>(a[k][u], b[k][u], hi, lo);
            sum += units(hi, lo);
        }
    }
    return sum;
}
// Sum of the weights [j0, j1): entries j0 + first, .. + 16 bytes, then `step` entries on, as long as they lie inside; then those that
// are left, one to each of `lanes` lanes.
template <typename T>
__device__ __forceinline__ u64 sum_of(const Row& r, int j0, int j1, int first, int step, int lanes, bool vec) {
    constexpr int N = 16 / sizeof(T);
    long long sum = 0;
    int j = j0;
    if (vec) {
        const int steps = (j1 - j0) / step;
        const T *p = static_cast<const T*>(r.p) + j0 + first, *d = static_cast<const T*>(r.d) + j0 + first;
        sum = r.rest == kLess ? sum_steps<T, true>(p, d, steps, step) : sum_steps<T, false>(p, p, steps, step);
        j += steps * step;
        const int x = r.x - j0;  // the entry that is left out is taken off again by the lane that added it
        if (r.rest == kWithout && x >= 0 && x < j - j0 && x % step >= first && x % step < first + N) {
            int hi = 0, lo = 0;
            add(read<T>(r.p, r.x), hi, lo);
            sum -= units(hi, lo);
        }
    }
    for (j += first / N; j < j1; j += lanes) sum += (long long)weight<T>(r, j);
    return (u64)sum;
}
// of a warp: every lane gets it
template <typename T>
__device__ __forceinline__ u64 sum_piece(const Row& r, int j0, int j1, bool vec) {
    constexpr int N = 16 / sizeof(T);
    u64 v = sum_of<T>(r, j0, j1, (threadIdx.x & 31) * N, 32 * N, 32, vec);
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The first index of [j0, j1) whose running weight is above t (there is one); a warp.  Runs of 1,024 entries (fp32: 512) are summed as
// before up to the one that crosses t; then each lane sums a 32nd of that, and the lane's part that crosses t is cut into 32 again.
// (Lanes with a 32nd of all 8,192 from the start had 32 loads one behind the other: the whole call 33 us.)
template <typename T>
__device__ int locate(const Row& r, int j0, int j1, u64 t, bool vec) {
    constexpr int N = 16 / sizeof(T);
    const int lane = threadIdx.x & 31;
    if (vec) {
        constexpr int kRun = 4 * 32 * N;
        for (; j0 + kRun < j1; j0 += kRun) {
            const u64 v = sum_piece<T>(r, j0, j0 + kRun, true);
            if (v > t) {
                j1 = j0 + kRun;
                break;
            }
            t -= v;
        }
    }
    for (;;) {
        const int n = j1 - j0;
        int per = (n + 31) / 32;
        const bool wide = vec && per >= N;  // (j0 is a multiple of N then)
        if (wide) per = (per + N - 1) / N * N;
        const int a = min(j1, j0 + lane * per), b = min(j1, a + per);
        const u64 v = sum_of<T>(r, a, b, 0, N, 1, wide);
        u64 run = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 x = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += x;
        }
        const unsigned above = __ballot_sync(0xffffffffu, run > t);
        if (!above) return -1;
        const int who = __ffs(above) - 1;
        t -= __shfl_sync(0xffffffffu, run - v, who);
        j0 = __shfl_sync(0xffffffffu, a, who);
        j1 = __shfl_sync(0xffffffffu, b, who);
        if (j1 - j0 <= 1) return j0;
    }
}

__device__ __forceinline__ float unit_of(float u) {  // negative and NaN: 0; from 1 on: the last number before it
    return u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
}
__device__ __forceinline__ void put_remote(uint64_t* at, unsigned rank, u64 v) {
    uint32_t addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(ptx::smem_u32(at)), "r"(rank));
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kResident) k_verify(const VerifyArgs a, int ctas) {
    __shared__ uint64_t totals[2][kMaxCtas];
    __shared__ u64 sums[kWarps];
    __shared__ int s_kept;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.x / ctas, rank = blockIdx.x % ctas;
    const int n = a.dlens ? min(max(__ldg(a.dlens + b), 0), a.K) : a.K;
    const int* drafts = a.drafts + (long long)b * a.K;
    const float* U = a.U + (long long)b * (a.K + 1);
    const T* P = static_cast<const T*>(a.P) + b * a.pb;
    const T* D = a.D ? static_cast<const T*>(a.D) + b * a.db : nullptr;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    if (warp == 0) {
        int kept = 0;
        for (int i0 = 0; i0 < a.K; i0 += 32) {  // (up to K, so that the draft does not wait for the request's length)
            const int i = i0 + lane;
            bool ok = false;
            if (i < a.K) {
                const int x = __ldg(drafts + i);
                if (i < n && x >= 0 && x < a.M) {
                    const double d = D ? (double)read<T>(D + i * a.dr, x) : 1.0;
                    ok = (double)unit_of(__ldg(U + i)) * d < (double)read<T>(P + i * a.pr, x);
                }
            }
            const unsigned good = __ballot_sync(0xffffffffu, ok);
            kept = i0 + (good == 0xffffffffu ? 32 : __ffs(~good) - 1);
            if (good != 0xffffffffu) break;
        }
        if (lane == 0) s_kept = min(kept, n);
    }
    __syncthreads();
    const int kept = s_kept;
    Row row;
    row.p = P + kept * a.pr;
    row.d = D ? D + kept * a.dr : nullptr;
    row.rest = kept == n ? kTarget : D ? kLess : kWithout;
    row.x = kept < n ? __ldg(drafts + kept) : -1;
    constexpr int kStep = 32 * 16 / sizeof(T);  // entries of a warp's load
    const int steps = (a.M + kStep - 1) / kStep, me = rank * kWarps + warp, all = ctas * kWarps;
    const int j0 = min(a.M, (int)((long long)steps * me / all) * kStep), j1 = min(a.M, (int)((long long)steps * (me + 1) / all) * kStep);
    u64 mine = 0, before = 0, total = 0;
    bool vec = false;
    for (int turn = 0; turn < 2; ++turn) {  // (again with P alone where nothing is left of it)
        vec = ((uintptr_t)row.p | (row.rest == kLess ? (uintptr_t)row.d : 0)) % 16 == 0;
        mine = sum_piece<T>(row, j0, j1, vec);
        if (lane == 0) sums[warp] = mine;
        __syncthreads();
        if (turn == 0) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // every CTA of the cluster runs
        if (warp == 0) {
            u64 v = lane < kWarps ? sums[lane] : 0;
#pragma unroll
            for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane < ctas) put_remote(&totals[turn][rank], lane, v);
        }
        ptx::cluster_sync_all();
        __syncthreads();
        before = total = 0;
        for (int c = 0; c < ctas; ++c) {
            if (c < rank) before += totals[turn][c];
            total += totals[turn][c];
        }
        for (int w = 0; w < warp; ++w) before += sums[w];
        if (total != 0 || row.rest == kTarget) break;
        row.rest = kTarget;
        __syncthreads();
    }
    // run > U total, with U 2^64 an integer (from 2^-40 on) and run one: run > floor
    const float u = unit_of(__ldg(U + a.K));
    const u64 t = __umul64hi((u64)__float2ull_rz(u * 18446744073709551616.f), total);
    int drawn = -1;
    if (total == 0) {
        if (me != 0) return;
    } else {
        if (t < before || t >= before + mine) return;  // another warp's
        drawn = locate<T>(row, j0, j1, t - before, vec);
    }
    if (lane == 0 && a.accepted) a.accepted[b] = kept;
    if (a.tokens)
        for (int i = lane; i <= a.K; i += 32)
            a.tokens[(long long)b * (a.K + 1) + i] = i < kept ? __ldg(drafts + i) : i == kept ? drawn : -1;
}

}  // namespace

cudaError_t launch_verify(const VerifyArgs& a, int sms, cudaStream_t s) {
    // a warp's piece of four loads or more, and no more CTAs than run at once where there are more rows than that
    const long long steps = ((long long)a.M * (a.bf16 ? 2 : 4) + 511) / 512;
    int ctas = 1;
    while (ctas < kMaxCtas && steps >= 4ll * kWarps * ctas && 2ll * a.B * ctas <= (long long)kResident * sms) ctas *= 2;
    if ((long long)a.B * ctas > 0x7fffffffLL) ctas = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(a.B * (long long)ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return a.bf16 ? cudaLaunchKernelEx(&cfg, k_verify<__nv_bfloat16>, a, ctas) : cudaLaunchKernelEx(&cfg, k_verify<float>, a, ctas);
}

}  // namespace gs
