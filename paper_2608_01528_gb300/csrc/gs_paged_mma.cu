// gs_paged_mma.cu -- attention of a few rows over a paged cache on the tensor cores (bf16).
//
// The query rows of a key head (packed, 8 to 32) meet its keys in steps of 16, a warp by itself: S^T = K Q^T and O^T += V^T P^T, so
// that rows come in eights (a decoding step of four query heads to a key head fills half of one tile, not an eighth), P goes from
// one product to the other in registers, and no warp waits for another.  K and V are read once, 16 bytes a lane and copy, three steps
// in a ring; the table entry of a step is read four steps before it and its rows' addresses are known two before, so a page may end anywhere.
// A row's reference maximum moves only where it grew by more than 2^8, which spares the reduction over keys in most steps.  The weights go
// to V in two bf16 terms (error of O against 64 bits 2.1e-3 -> 1.7e-3 of its norm, the output's own rounding; 64 single rows 101 -> 96 to 103 us,
// six rows over long histories 272 -> 270 to 305).
//
// Bound by memory: 16 keys of 128 + 128 columns are 8 KB and 0.18 us of an SM's share of HBM, in which 32 rows take 96 products of
// 16 x 8 x 16 (64 x 1 to 4,096 keys, 32 / 8 heads of 128: 5.2 to 5.6 TB/s of calls, 5.9 of the kernel; 8 x 32,769 to 65,537 keys: 5.3 to 5.9 and 5.7).  A tcgen05 tile has 128 rows, of which a decoding step fills 1 to 32, and would add a pass through TMEM to each step.
//
// Work.  A unit is a request, a chunk of rows and up to four neighbouring key heads, one to each warp of a CTA, which so read 1 KB of a
// position together (fewer heads: the warps that are over take runs of their own).  Every worker takes an equal run of the steps of all
// units, wherever requests begin and end in it: lengths need not be even.  A piece that is not a whole unit goes to the workspace as
// (O, m, l), and k_paged_join adds a unit's pieces in order.  Where no unit has more than kWholeKeys keys, or units are many, a CTA
// takes one key head's unit, its warps every fourth step, and they join in shared memory.

#include <algorithm>
#include <atomic>

#include "gs_paged.h"
#include "gs_xattn_tc.cuh"

namespace gs {
namespace {

using xtc::ex2;
using xtc::kLn2;
using xtc::kLog2e;
using xtc::keys_of;

constexpr int kWarps = 4, kThreads = kWarps * 32, kStep = 16, kStages = 3;
// A CTA takes whole units where none has more keys than this: 4 x 512 keys, 32 / 8 heads of 128, whole 21.6, in pieces 22.7 us (in a graph), 16 x 512
// 22.7 / 26.8, 4 x 90 to 300, 8 heads of 64, 14.5 / 21.6, but 256 x 512 128 / 119; 4 x 1,024 30.8 / 24.7.
constexpr int kWholeKeys = 512;
// .. or where there are so many units a CTA: what the table has room for does not tell how long requests are, and short ones lose more in
// pieces than long ones gain: 20,000 of 1 to 60 keys, 4 heads to one of 64, 177 / 286 us, 1,024 of 1 to 2,048, 32 / 8 heads of 128, 786 / 697.
constexpr long long kWholeUnits = 16;
// Steps of a worker, at least: one request of 1,500 keys with 1, 2, 4, 8, 16: 44, 32, 28, 30, 38 us; four of them 34, 35, 30, 32, 38.
constexpr int kLeastSteps = 4;
constexpr float kGrow = 8.f;    // the maximum moves when it grew by more than 2^kGrow

struct Params {
    XattnArgs a;
    int chunks;     // of rows of a key head
    int whole;      // a CTA per unit of one key head
    int heads;      // key heads of a unit: 1, 2 or 4 warps side by side
    int groups;     // units of a chunk: Hkv / heads
    int ctas;
    long long* starts;  // B + 1: steps before each request (joined pieces only)
    float* part;        // 2 pieces a warp: R x DV sums
    float2* ml;         // and R maxima (base 2) and sums
};

template <int DK, int DV>
struct Shared {
    __nv_bfloat16 ring[kWarps][kStages][kStep * (DK + DV)];  // K, then V; at the end of a whole unit: R x DV sums a warp
    long long where[kWarps][2][32];  // offsets of a step's 16 rows of K and 16 of V in elements, or -1
    float2 ml[kWarps][32];
    long long scan[kWarps];
    long long found[kWarps][2];
};

template <int DK, int DV, int NR>
constexpr int resident() {  // CTAs that run at once on a multiprocessor
    return DK + DV <= 128 ? (NR <= 2 ? 4 : 3) : DK + DV <= 192 ? (NR <= 2 ? 3 : 2) : 2;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldmatrix(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {  // an 8 x 8 tile, two entries of a row a lane
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// byte offset of 16-byte chunk c of row r in a tile of W columns: eight rows' same chunk lies in different banks
template <int W>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
    return (uint32_t)(r * W * 2 + ((c ^ (r & 7)) << 4));
}
__device__ __forceinline__ bool odd_low(uint32_t x) { return (x & 0x7f80u) == 0x7f80u; }            // an infinity or NaN of a pair
__device__ __forceinline__ bool odd_high(uint32_t x) { return (x & 0x7f800000u) == 0x7f800000u; }

// Two weights in two bf16 terms: their upper halves, and what these leave, which is above 0 where the weight is (the smallest bf16
// number, 2^-133, at least), so that an infinite value times either term stays the same infinity.  (With terms to the nearest the second
// was 0 or negative: infinities that a row sees came out as NaN.)
__device__ __forceinline__ void two_terms(float x, float y, uint32_t& high, uint32_t& low) {
    const uint32_t u = __float_as_uint(x) & 0xffff0000u, v = __float_as_uint(y) & 0xffff0000u;
    high = u >> 16 | v;
    low = __vmaxu2(ptx::pack_bf16(x - __uint_as_float(u), y - __uint_as_float(v)), __vminu2(high, 0x00010001u));
}

__device__ __forceinline__ KeySpan unit_span(const XattnArgs& a, int b, int n) {
    return key_span<kPagedKeys>(a, b, 0, a.Lq - 1, n);
}
__device__ __forceinline__ int steps_of(const KeySpan& s) { return max(1, s.count() / kStep + (s.count() % kStep != 0)); }

// Sum over the block's 128 threads; every thread gets it.
__device__ __forceinline__ long long block_sum(long long v, long long* sh) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    return sh[0] + sh[1] + sh[2] + sh[3];
}

// How many workers share `total` steps; worker w has the steps total * w / n to total * (w + 1) / n.
__device__ __forceinline__ long long workers_of(const Params& p, long long total) {
    const long long most = (long long)p.ctas * (kWarps / p.heads);
    return max(1ll, min(most, total / kLeastSteps));
}

struct Cursor {  // a step
    int b, grp, chunk, k, n, nst;
    KeySpan span;
    __device__ __forceinline__ void request(const XattnArgs& a) {
        n = keys_of(a, b);
        span = unit_span(a, b, n);
        nst = steps_of(span);
    }
    __device__ __forceinline__ bool next(const Params& p, int by, bool more) {  // true: the unit ended
        k += by;
        if (k < nst) return false;
        k = 0;
        if (++chunk == p.chunks) {
            chunk = 0;
            if (++grp == p.groups) {
                grp = 0;
                if (more) {
                    ++b;
                    request(p.a);
                }
            }
        }
        return true;
    }
};

template <int DK, int DV, int NR>
__global__ void __launch_bounds__(kThreads, resident<DK, DV, NR>()) k_paged_mma(const Params p) {
    using Sh = Shared<DK, DV>;
    constexpr int R = NR * 8, KS = DK / 16, MT = DV / 16;  // S: steps of 16 columns; O: tiles of 16 columns
    constexpr int KC = DK / 8, VC = DV / 8;                // 16-byte chunks of a row
    static_assert(kStages * kStep * (DK + DV) * 2 >= R * DV * 4);
    extern __shared__ __align__(128) uint8_t raw[];
    Sh& sh = *reinterpret_cast<Sh*>(raw);
    const XattnArgs& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const float cs = a.scale * kLog2e;
    const int head_of = p.whole ? 0 : warp % p.heads, by = p.whole ? kWarps : 1;

    // ------------------------------------------------------------- this warp's steps, and where they begin
    long long left;
    Cursor at;
    if (p.whole) {
        const long long per_b = (long long)a.Hkv * p.chunks;
        at.b = (int)(blockIdx.x / per_b);
        const int u = (int)(blockIdx.x - at.b * per_b);
        at.grp = u / p.chunks;
        at.chunk = u - at.grp * p.chunks;
        at.k = warp;
        at.request(a);
        left = at.nst > warp ? (at.nst - warp + kWarps - 1) / kWarps : 0;
    } else {
        const long long per_b = (long long)p.groups * p.chunks;
        const int side = kWarps / p.heads;  // workers of a CTA
        long long mine = 0;
        for (int b = tid; b < a.B; b += kThreads) mine += steps_of(unit_span(a, b, keys_of(a, b)));
        const long long total = block_sum(mine, sh.scan) * per_b, all = workers_of(p, total);
        const long long w0 = (long long)blockIdx.x * side;
        if (blockIdx.x != 0 && w0 >= all) return;  // (the first CTA writes `starts`)
        const long long cta0 = total * w0 / all, cta1 = total * min(all, w0 + side) / all;
        long long before = 0;  // steps of the requests before the 128 in turn
        if (tid < 2 * kWarps) sh.found[tid >> 1][tid & 1] = 0;
        for (int b0 = 0; b0 < a.B; b0 += kThreads) {
            const int b = b0 + tid;
            const long long n = b < a.B ? steps_of(unit_span(a, b, keys_of(a, b))) * per_b : 0;
            long long run = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += x;
            }
            __syncthreads();
            if (lane == 31) sh.scan[warp] = run;
            __syncthreads();
            for (int w = 0; w < warp; ++w) run += sh.scan[w];
            run += before;
            before += sh.scan[0] + sh.scan[1] + sh.scan[2] + sh.scan[3];
            if (b < a.B && run > cta0 && run - n < cta1)
                for (int w = 0; w < side && w0 + w < all; ++w) {
                    const long long s0 = total * (w0 + w) / all;
                    if (s0 < run && s0 >= run - n) {
                        sh.found[w][0] = b;
                        sh.found[w][1] = s0 - (run - n);
                    }
                }
            if (blockIdx.x == 0 && b < a.B) {
                p.starts[b] = run - n;
                if (b == a.B - 1) p.starts[a.B] = run;
            }
            if (blockIdx.x != 0 && cta1 <= before) break;
        }
        __syncthreads();
        const int w = warp / p.heads;
        if (w0 + w >= all) return;
        left = total * (w0 + w + 1) / all - total * (w0 + w) / all;
        at.b = (int)sh.found[w][0];
        at.request(a);
        const int u = (int)(sh.found[w][1] / at.nst);
        at.k = (int)(sh.found[w][1] - (long long)u * at.nst);
        at.grp = u / p.chunks;
        at.chunk = u - at.grp * p.chunks;
    }

    // ------------------------------------------------------------- fetching: a key a lane, K of 16 keys and V of the same
    Cursor ahead = at;
    long long to_read = left;  // steps whose table entry has not been read
    int entry = -1, in_page = 0, hk_read = 0;
    auto read_entry = [&]() {
        entry = -1;
        if (to_read == 0) return;
        --to_read;
        const int i = ahead.k * kStep + (lane & 15);
        hk_read = ahead.grp * p.heads + head_of;
        if ((unsigned)i < (unsigned)ahead.span.count()) {  // (the last step may pass 2^31)
            const int j = ahead.span.key(i), col = a.pg.shift >= 0 ? j >> a.pg.shift : j / a.pg.page;
            entry = __ldg(a.pg.table + (long long)ahead.b * a.pg.ldt + col);
            in_page = j - col * a.pg.page;
        }
        ahead.next(p, by, to_read > 0);
    };
    auto resolve = [&](int buf) {  // the addresses of the step whose entry was read last; the keys that are there
        const bool ok = entry >= 0 && entry < a.pg.pages;
        const HeadView& v = lane < 16 ? a.k : a.v;
        sh.where[warp][buf][lane] = ok ? (long long)entry * v.b + (long long)in_page * v.l + (long long)hk_read * v.h : -1ll;
        return __ballot_sync(0xffffffffu, ok) & 0xffffu;
    };
    const __nv_bfloat16* kp = reinterpret_cast<const __nv_bfloat16*>(a.k.p);
    const __nv_bfloat16* vp = reinterpret_cast<const __nv_bfloat16*>(a.v.p);
    const uint32_t ring = ptx::smem_u32(sh.ring[warp][0]);
    constexpr uint32_t kStageBytes = kStep * (DK + DV) * 2, kKeyBytes = kStep * DK * 2;
    auto issue = [&](uint32_t to, int buf, bool on) {
        if (on) {
            const long long* wh = sh.where[warp][buf];
            {
                const int c = lane % KC;
#pragma unroll
                for (int r0 = 0; r0 < kStep; r0 += 32 / KC) {
                    const int r = r0 + lane / KC;
                    const long long x = wh[r];
                    const bool there = x >= 0 && c * 8 < a.dk;
                    copy16(to + chunk_at<DK>(r, c), kp + (there ? x + c * 8 : 0), there);
                }
            }
            {
                const int c = lane % VC;
#pragma unroll
                for (int r0 = 0; r0 < kStep; r0 += 32 / VC) {
                    const int r = r0 + lane / VC;
                    const long long x = wh[16 + r];
                    const bool there = x >= 0 && c * 8 < a.dv;
                    copy16(to + kKeyBytes + chunk_at<DV>(r, c), vp + (there ? x + c * 8 : 0), there);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

    unsigned ok0, ok1, ok2;  // the keys of the next three steps that are there
    read_entry();
    ok0 = resolve(0);
    __syncwarp();
    issue(ring, 0, left > 0);
    read_entry();
    ok1 = resolve(1);
    __syncwarp();
    issue(ring + kStageBytes, 1, left > 1);
    read_entry();
    ok2 = resolve(0);
    read_entry();

    uint32_t q[NR][KS][2];
    float o[MT][NR][4], top[NR][2], sum[NR][2];
    int pos[NR][2];            // the rows' positions, -1: a row that sees nothing
    int all_lo = 0, all_hi = 0;  // every row that sees anything sees [all_lo, all_hi)
    bool fresh = true;   // the step begins a piece
    bool from0 = false;  // the piece began with its unit
    int piece = 0, slot_r = 0, slot_w = 2;
    Cursor unit = at;    // of the piece
    for (long long s = 0; s < left; ++s) {
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();  // step s is in shared memory, the last one has been read, the rows of step s + 2 are known
        issue(ring + slot_w * kStageBytes, (int)(s & 1), s + 2 < left);
        const unsigned ok3 = resolve((int)(s + 1) & 1);
        read_entry();
        if (fresh) {
            fresh = false;
            unit = at;
            from0 = at.k == 0 || p.whole;
            const int hk = at.grp * p.heads + head_of;
            const int m = a.pg.qlens ? min(max(__ldg(a.pg.qlens + at.b), 0), a.Lq) : a.Lq;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const long long pr = (long long)at.chunk * R + n * 8 + g;
                const bool has = pr < a.rows;
                const long long l = has ? pr / a.G : 0;
                const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(a.q.p) + at.b * a.q.b + l * a.q.l +
                                           (long long)(hk * a.G + (has ? (int)(pr - l * a.G) : 0)) * a.q.h;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int c = k * 16 + e * 8 + 2 * t;
                        q[n][k][e] = has && c < a.dk ? __ldg(reinterpret_cast<const uint32_t*>(src + c)) : 0u;
                    }
                const int mine = has && l < m && at.n - m + l >= 0 ? (int)(at.n - m + l) : -1;
                pos[n][0] = __shfl_sync(0xffffffffu, mine, 8 * t);
                pos[n][1] = __shfl_sync(0xffffffffu, mine, 8 * t + 4);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[n][e] = -INFINITY;
                    sum[n][e] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][n][e] = 0.f;
            }
            int first = 0x7fffffff, last = -1;
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (pos[n][e] >= 0) {
                        first = min(first, pos[n][e]);
                        last = max(last, pos[n][e]);
                    }
            first = __reduce_min_sync(0xffffffffu, first);
            last = __reduce_max_sync(0xffffffffu, last);
            all_hi = last < 0 ? 0 : first + 1;
            all_lo = a.win.window == kNoWindow ? 0 : max(0, last - a.win.window + 1);
        }
        // ------------------------------------------------------------- S^T of 16 keys and the rows
        const uint32_t ks = ring + slot_r * kStageBytes, vs = ks + kKeyBytes;
        float c[NR][4];
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) c[n][e] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            uint32_t x[4];
            ldmatrix(x, ks + chunk_at<DK>(lane & 15, 2 * k + (lane >> 4)));
#pragma unroll
            for (int n = 0; n < NR; ++n) mma(c[n], x, q[n][k][0], q[n][k][1]);
        }
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) c[n][e] *= cs;
        const int i0 = at.k * kStep, j0 = at.span.key(i0), j1 = at.span.key(i0 + kStep - 1);
        const bool plain = ok0 == 0xffffu && j1 < all_hi && (j0 >= all_lo || j1 < a.win.sinks);
        int wild = 0;
        if (!plain) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = i0 + 8 * h + g, j = at.span.key(i);
                const bool there = (ok0 >> (8 * h + g)) & 1u;
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = pos[n][e];
                        if (!there || j > r || (a.win.window != kNoWindow && j <= r - a.win.window && j >= a.win.sinks))
                            c[n][2 * h + e] = -INFINITY;
                    }
            }
            if (a.Lq > 1) {  // a value that is not finite in a row of V that some rows see and others do not: 0 * NaN would reach the others
                for (int e = lane; e < kStep * VC; e += 32) {
                    uint32_t w[4];
                    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(vs + 16 * e) : "memory");
#pragma unroll
                    for (int k = 0; k < 4; ++k) wild |= odd_low(w[k]) || odd_high(w[k]);
                }
                wild = __any_sync(0xffffffffu, wild);
            }
        }
        bool grew = false;
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) grew |= fmaxf(c[n][e], c[n][2 + e]) > top[n][e] + kGrow;
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = fmaxf(c[n][e], c[n][2 + e]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
                    if (x > top[n][e] + kGrow) {  // by the row's own keys: its rounding does not depend on other rows
                        const float f = ex2(top[n][e] - x);
                        top[n][e] = x;
                        sum[n][e] *= f;
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            o[i][n][e] *= f;
                            o[i][n][2 + e] *= f;
                        }
                    }
                }
        }
        // ------------------------------------------------------------- P^T, and V^T P^T
        uint32_t pb[NR][2], pl[NR][2];  // the weights in two bf16 terms (16 bits together): the tensor pipe has room, and O keeps fp32's accuracy
#pragma unroll
        for (int n = 0; n < NR; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float ms = top[n][e] == -INFINITY ? 0.f : top[n][e];
                c[n][e] = ex2(c[n][e] - ms);
                c[n][2 + e] = ex2(c[n][2 + e] - ms);
                sum[n][e] += c[n][e] + c[n][2 + e];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float x = c[n][2 * h], y = c[n][2 * h + 1];
                uint32_t high, low;
                two_terms(x, y, high, low);
                pb[n][h] = transposed(high);
                pl[n][h] = transposed(low);
            }
        }
        if (wild) {  // what is not finite goes to the rows that see it by itself, and out of the tile
            auto value = [&](int j, int col) { return vs + chunk_at<DV>(j, col >> 3) + 2 * (col & 7); };
            for (int j = 0; j < kStep; ++j) {
                float w[NR][2];
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        w[n][e] = __bfloat162float(__float2bfloat16_rn(
                            __shfl_sync(0xffffffffu, j < 8 ? c[n][e] : c[n][2 + e], ((j & 7) << 2) | t)));
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        unsigned short x;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(value(j, 16 * i + 8 * h + g)) : "memory");
                        if (!odd_low(x)) continue;
#pragma unroll
                        for (int n = 0; n < NR; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (w[n][e] != 0.f) o[i][n][2 * h + e] += w[n][e] * __uint_as_float((uint32_t)x << 16);
                    }
            }
            __syncwarp();
            for (int e = lane; e < kStep * DV / 2; e += 32) {
                uint32_t x;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(vs + 4 * e) : "memory");
                if (!odd_low(x) && !odd_high(x)) continue;
                if (odd_low(x)) x &= 0xffff0000u;
                if (odd_high(x)) x &= 0xffffu;
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(vs + 4 * e), "r"(x) : "memory");
            }
            __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            uint32_t x[4];
            ldmatrix_t(x, vs + chunk_at<DV>((lane & 7) + ((lane >> 4) << 3), 2 * i + ((lane >> 3) & 1)));
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                mma(o[i][n], x, pb[n][0], pb[n][1]);
                mma(o[i][n], x, pl[n][0], pl[n][1]);
            }
        }
        ok0 = ok1;
        ok1 = ok2;
        ok2 = ok3;
        slot_r = slot_r + 1 == kStages ? 0 : slot_r + 1;
        slot_w = slot_w + 1 == kStages ? 0 : slot_w + 1;
        const bool end = at.next(p, by, s + 1 < left) && !p.whole;
        if (p.whole || (!end && s + 1 < left)) continue;
        // ------------------------------------------------------------- the end of a piece
        fresh = true;
        const bool full = from0 && end;
        const int hk = unit.grp * p.heads + head_of;
        const long long slot = ((long long)blockIdx.x * kWarps + warp) * 2 + (piece > 0);
        ++piece;
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float l = sum[n][e];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
                const int r = n * 8 + 2 * t + e;
                const long long pr = (long long)unit.chunk * R + r;
                if (pr >= a.rows) continue;
                const bool none = pos[n][e] < 0;  // (steps that all rows see are not masked for those that see nothing)
                if (none) l = 0.f;
                if (full) {
                    const long long ql = pr / a.G;
                    const int head = hk * a.G + (int)(pr - ql * a.G);
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.o.p) + unit.b * a.o.b + ql * a.o.l + head * a.o.h;
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int col = 16 * i + 8 * h + g;
                            if (col < a.dv) out[col] = __float2bfloat16_rn(l == 0.f ? 0.f : o[i][n][2 * h + e] * inv);
                        }
                    if (a.lse && g == 0)
                        a.lse[((long long)unit.b * a.Hq + head) * a.Lq + ql] = l == 0.f ? -INFINITY : (top[n][e] + log2f(l)) * kLn2;
                } else {
                    float* out = p.part + (slot * R + r) * DV;
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) out[16 * i + 8 * h + g] = o[i][n][2 * h + e];
                    if (g == 0) p.ml[slot * R + r] = make_float2(none ? -INFINITY : top[n][e], l);
                }
            }
    }
    if (!p.whole) return;
    // ------------------------------------------------------------- a whole unit: the four warps' sums
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    float* mine = reinterpret_cast<float*>(sh.ring[warp][0]);
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = n * 8 + 2 * t + e;
            float l = left > 0 ? sum[n][e] : 0.f;
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
            const bool none = left == 0 || pos[n][e] < 0;
            if (g == 0) sh.ml[warp][r] = none ? make_float2(-INFINITY, 0.f) : make_float2(top[n][e], l);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) mine[r * DV + 16 * i + 8 * h + g] = none ? 0.f : o[i][n][2 * h + e];
        }
    __syncthreads();
    const int hk = unit.grp;
    for (int x = tid; x < R * DV; x += kThreads) {
        const int r = x / DV, col = x - r * DV;
        const long long pr = (long long)unit.chunk * R + r;
        if (pr >= a.rows || col >= a.dv) continue;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) m = fmaxf(m, sh.ml[w][r].x);
        const float ms = m == -INFINITY ? 0.f : m;
        float l = 0.f, v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 ml = sh.ml[w][r];
            if (ml.y == 0.f) continue;  // nothing in this warp's steps (NaN is not 0)
            const float f = ex2(ml.x - ms);
            l = fmaf(ml.y, f, l);
            v = fmaf(reinterpret_cast<const float*>(sh.ring[w][0])[x], f, v);
        }
        const long long ql = pr / a.G;
        const int head = hk * a.G + (int)(pr - ql * a.G);
        reinterpret_cast<__nv_bfloat16*>(a.o.p)[unit.b * a.o.b + ql * a.o.l + head * a.o.h + col] =
            __float2bfloat16_rn(l == 0.f ? 0.f : v * (1.f / l));
        if (col == 0 && a.lse) a.lse[((long long)unit.b * a.Hq + head) * a.Lq + ql] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    }
}

// O and lse of the units that several workers had pieces of: a warp a row.
template <int DV>
__global__ void __launch_bounds__(256) k_paged_join(const Params p, int R) {
    const XattnArgs& a = p.a;
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), one = row / R;  // of a key head
    const int r = (int)(row - one * R);
    const long long per = (long long)a.Hkv * p.chunks, b = one / per;
    if (b >= a.B) return;
    const int hk = (int)((one - b * per) / p.chunks), chunk = (int)(one - b * per) - hk * p.chunks;
    const long long pr = (long long)chunk * R + r;
    if (pr >= a.rows) return;
    const long long total = p.starts[a.B], all = workers_of(p, total);
    const long long s0 = p.starts[b], nst = (p.starts[b + 1] - s0) / ((long long)p.groups * p.chunks);
    const long long u0 = s0 + ((long long)(hk / p.heads) * p.chunks + chunk) * nst, u1 = u0 + nst;
    // the last worker w that begins at or before step x: total w / all < x + 1
    const long long w0 = ((u0 + 1) * all - 1) / total, w1 = (u1 * all - 1) / total;
    if (w0 == w1) return;  // written already
    // (only the first of them can have begun before the unit: it is a later piece of that worker's then)
    const long long slot0 = (w0 * p.heads + hk % p.heads) * 2;
    const bool later = total * w0 / all < u0;
    const int n = (int)(w1 - w0 + 1);
    auto slot_of = [&](int i) { return slot0 + (long long)i * p.heads * 2 + (i == 0 && later); };
    float m = -INFINITY;
    for (int i = lane; i < n; i += 32) m = fmaxf(m, p.ml[slot_of(i) * R + r].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    const float ms = m == -INFINITY ? 0.f : m;
    float l = 0.f, acc[DV / 32];
#pragma unroll
    for (int q = 0; q < DV / 32; ++q) acc[q] = 0.f;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const float2 mine = i0 + lane < n ? p.ml[slot_of(i0 + lane) * R + r] : make_float2(0.f, 0.f);
        const bool some = mine.y != 0.f;  // (else nothing in this piece; NaN is not 0)
        const float f = some ? ex2(mine.x - ms) : 0.f;
        if (some) l = fmaf(mine.y, f, l);
        const unsigned which = __ballot_sync(0xffffffffu, some);
        const int count = min(32, n - i0);
        constexpr int kAhead = 4;  // pieces in flight
        for (int c = 0; c < count; c += kAhead) {
            float v[kAhead][DV / 32], w[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                w[u] = __shfl_sync(0xffffffffu, f, (c + u) & 31);
                const bool in = c + u < count && (which >> ((c + u) & 31) & 1u);
                const float* from = p.part + (slot_of(i0 + (in ? c + u : 0)) * R + r) * DV;
#pragma unroll
                for (int q = 0; q < DV / 32; ++q) v[u][q] = in ? from[lane + 32 * q] : 0.f;
                if (!in) w[u] = 0.f;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int q = 0; q < DV / 32; ++q) acc[q] = fmaf(v[u][q], w[u], acc[q]);
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const long long ql = pr / a.G;
    const int head = hk * a.G + (int)(pr - ql * a.G);
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.o.p) + b * a.o.b + ql * a.o.l + head * a.o.h;
#pragma unroll
    for (int q = 0; q < DV / 32; ++q)
        if (lane + 32 * q < a.dv) out[lane + 32 * q] = __float2bfloat16_rn(l == 0.f ? 0.f : acc[q] * inv);
    if (lane == 0 && a.lse) a.lse[(b * a.Hq + head) * a.Lq + ql] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

struct Plan {
    int nr, chunks, whole, heads, ctas;
    long long starts, part, ml;  // bytes
};
template <int NR>
int resident_nr(bool k2, bool v2) {
    return k2 ? (v2 ? resident<128, 128, NR>() : resident<128, 64, NR>()) : (v2 ? resident<64, 128, NR>() : resident<64, 64, NR>());
}
Plan plan_of(const XattnArgs& a, int sms) {
    Plan p{};
    p.nr = (int)std::min(4ll, (a.rows + 7) / 8);
    const bool k2 = a.dk > 64, v2 = a.dv > 64;
    const int R = 8 * p.nr, dv = v2 ? 128 : 64;
    p.chunks = (int)((a.rows + R - 1) / R);
    p.heads = a.Hkv % 4 == 0 ? 4 : a.Hkv % 2 == 0 ? 2 : 1;
    const long long units = (long long)a.B * a.Hkv * p.chunks;
    const long long keys = std::min<long long>(a.Lk, (long long)a.win.window + a.win.sinks + a.Lq);
    p.ctas = sms * (p.nr == 1 ? resident_nr<1>(k2, v2) : p.nr == 2 ? resident_nr<2>(k2, v2)
                                                     : p.nr == 3 ? resident_nr<3>(k2, v2) : resident_nr<4>(k2, v2));
    p.whole = (keys <= kWholeKeys || units >= kWholeUnits * p.ctas) && units <= 0x7fffffffLL;
    if (p.whole) {
        p.ctas = (int)units;
        p.heads = 1;
    } else {
        p.starts = (a.B + 2ll) / 2 * 16;
        p.part = 2ll * kWarps * p.ctas * R * dv * 4;
        p.ml = 2ll * kWarps * p.ctas * R * 8;
    }
    return p;
}

std::atomic<bool> g_attr[64][16];

template <int DK, int DV, int NR>
cudaError_t launch(const Params& p, int device, cudaStream_t s) {
    std::atomic<bool>& set = g_attr[device][(DK > 64) * 8 + (DV > 64) * 4 + NR - 1];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(k_paged_mma<DK, DV, NR>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)sizeof(Shared<DK, DV>));
        if (e != cudaSuccess) return e;
        set = true;
    }
    k_paged_mma<DK, DV, NR><<<(unsigned)p.ctas, kThreads, sizeof(Shared<DK, DV>), s>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || p.whole) return e;
    const long long rows = (long long)p.a.B * p.a.Hkv * p.chunks * NR * 8;
    k_paged_join<DV><<<(unsigned)((rows + 7) / 8), 256, 0, s>>>(p, NR * 8);
    return cudaGetLastError();
}
template <int NR>
cudaError_t launch_rows(const Params& p, int device, cudaStream_t s) {
    const bool k2 = p.a.dk > 64, v2 = p.a.dv > 64;
    return k2 ? (v2 ? launch<128, 128, NR>(p, device, s) : launch<128, 64, NR>(p, device, s))
              : (v2 ? launch<64, 128, NR>(p, device, s) : launch<64, 64, NR>(p, device, s));
}

}  // namespace

bool paged_mma_supported(const XattnArgs& a) {
    auto on_16 = [](const HeadView& v, int nb, int nl, int nh) {
        auto ok = [](long long s, int n) { return n <= 1 || s % 8 == 0; };
        return (uintptr_t)v.p % 16 == 0 && ok(v.b, nb) && ok(v.l, nl) && ok(v.h, nh);
    };
    return a.dtype == GS_BF16 && a.dk % 8 == 0 && a.dv % 8 == 0 && on_16(a.q, a.B, a.Lq, a.Hq) &&
           on_16(a.k, a.pg.pages, a.pg.page, a.Hkv) && on_16(a.v, a.pg.pages, a.pg.page, a.Hkv);
}

long long paged_mma_bytes(const XattnArgs& a, int sms) {
    const Plan p = plan_of(a, sms);
    return p.starts + p.part + p.ml;
}

cudaError_t launch_paged_mma(const XattnArgs& a, int sms, int device, cudaStream_t s) {
    if (device < 0 || device >= 64) return cudaErrorInvalidDevice;
    const Plan pl = plan_of(a, sms);
    Params p{};
    p.a = a;
    p.chunks = pl.chunks;
    p.whole = pl.whole;
    p.heads = pl.heads;
    p.groups = a.Hkv / pl.heads;
    p.ctas = pl.ctas;
    char* ws = (char*)a.ws;
    p.starts = (long long*)ws;
    p.part = (float*)(ws + pl.starts);
    p.ml = (float2*)(ws + pl.starts + pl.part);
    switch (pl.nr) {
        case 1: return launch_rows<1>(p, device, s);
        case 2: return launch_rows<2>(p, device, s);
        case 3: return launch_rows<3>(p, device, s);
        default: return launch_rows<4>(p, device, s);
    }
}

}  // namespace gs
