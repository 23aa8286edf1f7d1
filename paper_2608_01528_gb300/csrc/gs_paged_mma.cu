// gs_paged_mma.cu -- attention of a few rows over a paged cache on the tensor cores (bf16).
//
// The query rows of a key head (packed, up to 16 or 32) meet its keys in steps of 64.  S = Q K^T: warp w of four takes keys
// 16 w .. + 15; the rows' maxima meet in shared memory; P = 2^(c s - m) goes there as bf16 and each warp adds P V for a quarter
// of V's columns, so that no sums of warps have to be joined.  K and V are read once, 16 bytes a lane and copy, three steps in a ring; the
// addresses of a step's 64 rows are worked out two steps before it (block table -> page -> row), so a page may end anywhere.
//
// Bound by memory: 64 keys of 128 + 128 columns are 32 KB and 0.7 us of an SM's share of HBM, in which 16 rows take 256 products of
// 16 x 8 x 16 and one chain of three barriers; a tcgen05 tile has 128 rows, of which a decoding step fills 1 to 32, and would add a pass
// through TMEM to that chain.
//
// Work.  Every (request, key head, chunk of rows) has ceil(keys / 64) steps, of which each resident CTA takes an equal run, wherever
// requests begin and end in it: lengths need not be even.  A piece that is not a whole unit goes to the workspace as (O, m, l), and
// k_paged_join adds a unit's pieces in order.  Where no unit has more than kWholeSteps steps, or units are many, a CTA takes one unit
// each and there is nothing to join.

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

constexpr int kThreads = 128, kStep = 64, kStages = 3;
constexpr int kWholeSteps = 8;

struct Params {
    XattnArgs a;
    int chunks;     // of rows of a key head
    int whole;      // a CTA per unit
    int ctas;
    long long* starts;  // B + 1: steps before each request (joined pieces only)
    float* part;        // 2 pieces a CTA: R x DV sums
    float2* ml;         // and R maxima (base 2) and sums
};

struct Desc {  // a step
    int b, hk, chunk, v0;      // v0: its first key, counted among those that the unit's rows see
    int sink, lo, n;           // those keys (KeySpan), and the request's keys
    int first, last, full;     // of this CTA's piece of a unit; the piece is the whole unit
    uint32_t ok[2], all[2];    // keys whose page is there; those that every row sees as well
};
struct Where {
    long long k, v;  // offset of a key's row in elements, or -1
};

template <int DK, int DV, int MT>
struct Shared {
    __nv_bfloat16 k[kStages][kStep * DK];
    __nv_bfloat16 v[kStages][kStep * DV];
    __nv_bfloat16 p[MT * 16 * kStep];
    Where where[2][kStep];
    Desc desc[4];
    float top[4][MT * 16], sum[4][MT * 16];
    long long scan[4];
    long long found[2];
};

template <int DK, int DV, int MT>
constexpr int resident() {  // CTAs that run at once on a multiprocessor
    return std::min<int>(DK + DV <= 128 ? 4 : DK + DV <= 192 ? 3 : 2, (int)((228 * 1024) / (sizeof(Shared<DK, DV, MT>) + 1024)));
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

template <int DK, int DV, int MT>
__global__ void __launch_bounds__(kThreads, resident<DK, DV, MT>()) k_paged_mma(const Params p) {
    using Sh = Shared<DK, DV, MT>;
    constexpr int R = MT * 16, KS = DK / 16, NT = DV / 32;  // S: steps of 16 columns; O: tiles of 8 columns a warp
    extern __shared__ __align__(128) uint8_t raw[];
    Sh& sh = *reinterpret_cast<Sh*>(raw);
    const XattnArgs& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const long long per_b = (long long)a.Hkv * p.chunks;
    const float cs = a.scale * kLog2e;

    // ------------------------------------------------------------- this CTA's steps, and where they begin
    long long left;  // steps of this CTA
    int cb, cu, ck;  // request, unit of it, step of the unit
    if (p.whole) {
        cb = (int)(blockIdx.x / per_b);
        cu = (int)(blockIdx.x - cb * per_b);
        ck = 0;
        left = steps_of(unit_span(a, cb, keys_of(a, cb)));
    } else {
        long long mine = 0;
        for (int b = tid; b < a.B; b += kThreads) mine += steps_of(unit_span(a, b, keys_of(a, b)));
        const long long total = block_sum(mine, sh.scan) * per_b;
        const long long s0 = total * blockIdx.x / p.ctas, s1 = total * (blockIdx.x + 1) / p.ctas;
        long long before = 0;  // steps of the requests before the 128 in turn
        if (tid < 2) sh.found[tid] = 0;
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
            if (b < a.B && s0 < run && s0 >= run - n) {
                sh.found[0] = b;
                sh.found[1] = s0 - (run - n);
            }
            if (blockIdx.x == 0 && b < a.B) {
                p.starts[b] = run - n;
                if (b == a.B - 1) p.starts[a.B] = run;
            }
            if (blockIdx.x != 0 && s0 < before) break;
        }
        __syncthreads();
        cb = (int)sh.found[0];
        const int nst = steps_of(unit_span(a, cb, keys_of(a, cb)));
        cu = (int)(sh.found[1] / nst);
        ck = (int)(sh.found[1] - (long long)cu * nst);
        left = s1 - s0;
    }
    const long long total_steps = left;
    if (left == 0) return;

    // ------------------------------------------------------------- making steps (warps 0 and 1: a key a lane)
    int n_b = keys_of(a, cb);
    KeySpan span = unit_span(a, cb, n_b);
    int nst = steps_of(span);
    bool fresh = true;  // the next step begins a piece
    bool from0 = false; // the piece began with its unit
    auto make = [&](long long s) {
        if (s >= total_steps) return;
        const int chunk = cu % p.chunks, hk = cu / p.chunks;
        if (fresh) from0 = ck == 0;
        const bool end = ck + 1 == nst, last = end || s + 1 == total_steps;
        const int i = ck * kStep + tid, j = i < span.count() ? span.key(i) : 0;
        const int col = a.pg.shift >= 0 ? j >> a.pg.shift : j / a.pg.page;
        const int entry = i < span.count() ? __ldg(a.pg.table + (long long)cb * a.pg.ldt + col) : -1;
        const bool ok = entry >= 0 && entry < a.pg.pages;
        const int row = j - col * a.pg.page;
        Where w{-1, -1};
        if (ok) {
            w.k = (long long)entry * a.k.b + (long long)row * a.k.l + (long long)hk * a.k.h;
            w.v = (long long)entry * a.v.b + (long long)row * a.v.l + (long long)hk * a.v.h;
        }
        sh.where[s & 1][tid] = w;
        // the rows of the chunk that see anything see this key (the first and the last of them do)
        const int m = a.pg.qlens ? min(max(__ldg(a.pg.qlens + cb), 0), a.Lq) : a.Lq;
        const long long l0 = (long long)chunk * R / a.G, l1 = min((long long)chunk * R + R - 1, a.rows - 1) / a.G;
        const long long first = max(l0 + n_b - m, 0ll), final_ = min(l1, (long long)m - 1) + n_b - m;
        const bool all = ok && j <= first && (j < a.win.sinks || a.win.window == kNoWindow || j > final_ - a.win.window);
        Desc& d = sh.desc[s & 3];
        const unsigned okw = __ballot_sync(0xffffffffu, ok), allw = __ballot_sync(0xffffffffu, all);
        if (lane == 0) {
            d.ok[warp] = okw;
            d.all[warp] = allw;
        }
        if (tid == 0) {
            d.b = cb;
            d.hk = hk;
            d.chunk = chunk;
            d.v0 = ck * kStep;
            d.sink = span.sink;
            d.lo = span.lo;
            d.n = n_b;
            d.first = fresh;
            d.last = last;
            d.full = from0 && end;
        }
        fresh = last;
        if (end) {
            ck = 0;
            if (++cu == per_b && s + 1 < total_steps) {
                cu = 0;
                ++cb;
                n_b = keys_of(a, cb);
                span = unit_span(a, cb, n_b);
                nst = steps_of(span);
            }
        } else {
            ++ck;
        }
    };
    const __nv_bfloat16* kp = reinterpret_cast<const __nv_bfloat16*>(a.k.p);
    const __nv_bfloat16* vp = reinterpret_cast<const __nv_bfloat16*>(a.v.p);
    auto issue = [&](long long s) {
        if (s < total_steps) {
            const Where* wh = sh.where[s & 1];
            const uint32_t ks = ptx::smem_u32(sh.k[s % kStages]), vs = ptx::smem_u32(sh.v[s % kStages]);
            constexpr int KC = DK / 8, VC = DV / 8;  // 16-byte chunks of a row
            {
                const int c = tid % KC;
#pragma unroll
                for (int r = tid / KC; r < kStep; r += kThreads / KC) {
                    const long long at = wh[r].k;
                    const bool there = at >= 0 && c * 8 < a.dk;
                    copy16(ks + chunk_at<DK>(r, c), kp + (there ? at + c * 8 : 0), there);
                }
            }
            {
                const int c = tid % VC;
#pragma unroll
                for (int r = tid / VC; r < kStep; r += kThreads / VC) {
                    const long long at = wh[r].v;
                    const bool there = at >= 0 && c * 8 < a.dv;
                    copy16(vs + chunk_at<DV>(r, c), vp + (there ? at + c * 8 : 0), there);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

    if (warp < 2) make(0);
    __syncthreads();
    issue(0);
    if (warp < 2) make(1);
    __syncthreads();
    issue(1);
    if (warp < 2) make(2);

    uint32_t q[MT][KS][4];
    float o[MT][NT][4], top[MT][2], sum[MT][2];
    KeySpan rows[MT][2];
    int piece = 0;
    for (long long s = 0; s < total_steps; ++s) {
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncthreads();  // step s is in shared memory, the last one has been read, step s + 2's rows are known
        issue(s + 2);
        if (warp < 2) make(s + 3);
        const Desc& d = sh.desc[s & 3];
        if (d.first) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const long long pr = (long long)d.chunk * R + m * 16 + h * 8 + g;
                    const bool has = pr < a.rows;
                    const long long l = has ? pr / a.G : 0;
                    const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(a.q.p) + d.b * a.q.b + l * a.q.l +
                                               (long long)(d.hk * a.G + (has ? (int)(pr - l * a.G) : 0)) * a.q.h;
#pragma unroll
                    for (int k = 0; k < KS; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int c = k * 16 + e * 8 + 2 * t;
                            q[m][k][2 * e + h] = has && c < a.dk ? __ldg(reinterpret_cast<const uint32_t*>(src + c)) : 0u;
                        }
                    rows[m][h] = key_span<kPagedKeys>(a, d.b, l, l, d.n);
                    if (!has) rows[m][h].hi = 0;
                    top[m][h] = -INFINITY;
                    sum[m][h] = 0.f;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[m][n][e] = 0.f;
            }
        }
        // ------------------------------------------------------------- S of this warp's 16 keys
        const uint32_t ks = ptx::smem_u32(sh.k[s % kStages]), vs = ptx::smem_u32(sh.v[s % kStages]), ps = ptx::smem_u32(sh.p);
        float c[MT][2][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) c[m][n][e] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            uint32_t b[4];
            ldmatrix(b, ks + chunk_at<DK>(warp * 16 + (lane >> 4) * 8 + (lane & 7), 2 * k + ((lane >> 3) & 1)));
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                mma(c[m][0], q[m][k], b[0], b[1]);
                mma(c[m][1], q[m][k], b[2], b[3]);
            }
        }
        const bool plain = (d.all[0] & d.all[1]) == 0xffffffffu;
        if (!plain) {
            const uint32_t ok = d.ok[warp >> 1] >> (16 * (warp & 1));
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = n * 8 + 2 * t + e, i = d.v0 + warp * 16 + at, j = i < d.sink ? i : i - d.sink + d.lo;
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const KeySpan& r = rows[m][h];
                            if (!((ok >> at) & 1u) || j >= r.hi || (j < r.lo && j >= r.sink)) c[m][n][2 * h + e] = -INFINITY;
                        }
                }
        }
        // ------------------------------------------------------------- the rows' maxima over the four warps
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x = -INFINITY;
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        c[m][n][2 * h + e] *= cs;
                        x = fmaxf(x, c[m][n][2 * h + e]);
                    }
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                if (t == 0) sh.top[warp][m * 16 + h * 8 + g] = x;
            }
        // A value that is not finite in a row of V that some rows see and others do not: 0 * NaN would reach the others.
        int wild = 0;
        if (plain || a.Lq == 1) {
            __syncthreads();
        } else {
            for (int e = tid; e < kStep * DV / 8; e += kThreads) {
                const uint4 x = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(sh.v[s % kStages]) + e * 16);
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    wild |= (w[k] & 0x7f80u) == 0x7f80u || (w[k] & 0x7f800000u) == 0x7f800000u;
            }
            wild = __syncthreads_or(wild);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float f[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = m * 16 + h * 8 + g;
                const float now = fmaxf(fmaxf(fmaxf(sh.top[0][r], sh.top[1][r]), fmaxf(sh.top[2][r], sh.top[3][r])), top[m][h]);
                const float ms = now == -INFINITY ? 0.f : now;
                f[h] = ex2(top[m][h] - ms);
                top[m][h] = now;
                float add = 0.f;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float x = ex2(c[m][n][2 * h] - ms), y = ex2(c[m][n][2 * h + 1] - ms);
                    add += x + y;
                    *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(sh.p) + chunk_at<kStep>(r, 2 * warp + n) + 4 * t) =
                        ptx::pack_bf16(x, y);
                }
                sum[m][h] = sum[m][h] * f[h] + add;
            }
            if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    o[m][n][0] *= f[0];
                    o[m][n][1] *= f[0];
                    o[m][n][2] *= f[1];
                    o[m][n][3] *= f[1];
                }
            }
        }
        __syncthreads();  // P is there
        // ------------------------------------------------------------- P V for this warp's columns
        if (wild) {  // what is not finite goes to the rows that see it by itself, and out of this warp's columns
            const auto at = [&](int j, int n) {
                return reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(sh.v[s % kStages]) + chunk_at<DV>(j, warp * NT + n) + 4 * t);
            };
            for (int j = 0; j < kStep; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint32_t x = *at(j, n);
                    const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
                    if (!lo && !hi) continue;
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float w = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(
                                reinterpret_cast<const uint8_t*>(sh.p) + chunk_at<kStep>(m * 16 + h * 8 + g, j >> 3) + 2 * (j & 7)));
                            if (w == 0.f) continue;
                            if (lo) o[m][n][2 * h] += w * __uint_as_float(x << 16);
                            if (hi) o[m][n][2 * h + 1] += w * __uint_as_float(x & 0xffff0000u);
                        }
                }
            __syncwarp();
            for (int j = g; j < kStep; j += 8)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint32_t x = *at(j, n);
                    if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
                    if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
                    *at(j, n) = x;
                }
            __syncwarp();
        }
#pragma unroll
        for (int k = 0; k < kStep / 16; ++k) {
            uint32_t pa[MT][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
                ldmatrix(pa[m], ps + chunk_at<kStep>(m * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), 2 * k + (lane >> 4)));
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                uint32_t b[4];
                ldmatrix_t(b, vs + chunk_at<DV>(k * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), warp * NT + n + (lane >> 4)));
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    mma(o[m][n], pa[m], b[0], b[1]);
                    mma(o[m][n + 1], pa[m], b[2], b[3]);
                }
            }
        }
        if (!d.last) continue;
        // ------------------------------------------------------------- the end of a piece
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                sum[m][h] += __shfl_xor_sync(0xffffffffu, sum[m][h], 1);
                sum[m][h] += __shfl_xor_sync(0xffffffffu, sum[m][h], 2);
                if (t == 0) sh.sum[warp][m * 16 + h * 8 + g] = sum[m][h];
            }
        __syncthreads();
        const long long slot = (long long)blockIdx.x * 2 + (piece > 0);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = m * 16 + h * 8 + g;
                const long long pr = (long long)d.chunk * R + r;
                if (pr >= a.rows) continue;
                const bool none = rows[m][h].hi <= 0;  // (steps that all rows see are not masked for those that see nothing)
                const float l = none ? 0.f : (sh.sum[0][r] + sh.sum[1][r]) + (sh.sum[2][r] + sh.sum[3][r]);
                const long long ql = pr / a.G;
                const int head = d.hk * a.G + (int)(pr - ql * a.G);
                if (d.full) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.o.p) + d.b * a.o.b + ql * a.o.l + head * a.o.h;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const int col = (warp * NT + n) * 8 + 2 * t;
                        const float x = l == 0.f ? 0.f : o[m][n][2 * h] * inv, y = l == 0.f ? 0.f : o[m][n][2 * h + 1] * inv;
                        if (col < a.dv) out[col] = __float2bfloat16_rn(x);
                        if (col + 1 < a.dv) out[col + 1] = __float2bfloat16_rn(y);
                    }
                    if (a.lse && warp == 0 && t == 0)
                        a.lse[((long long)d.b * a.Hq + head) * a.Lq + ql] = l == 0.f ? -INFINITY : (top[m][h] + log2f(l)) * kLn2;
                } else {
                    float* out = p.part + (slot * R + r) * DV;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        *reinterpret_cast<float2*>(out + (warp * NT + n) * 8 + 2 * t) = make_float2(o[m][n][2 * h], o[m][n][2 * h + 1]);
                    if (warp == 0 && t == 0) p.ml[slot * R + r] = make_float2(none ? -INFINITY : top[m][h], l);
                }
            }
        ++piece;
    }
}

// O and lse of the units that several CTAs had pieces of: a warp a row.
template <int DV, int MT>
__global__ void __launch_bounds__(256) k_paged_join(const Params p) {
    constexpr int R = MT * 16;
    const XattnArgs& a = p.a;
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), unit = row / R;
    const int r = (int)(row - unit * R);
    const long long per_b = (long long)a.Hkv * p.chunks, b = unit / per_b;
    if (b >= a.B) return;
    const int u = (int)(unit - b * per_b), chunk = u % p.chunks, hk = u / p.chunks;
    const long long pr = (long long)chunk * R + r;
    if (pr >= a.rows) return;
    const long long total = p.starts[a.B], s0 = p.starts[b], nst = (p.starts[b + 1] - s0) / per_b;
    const long long u0 = s0 + u * nst, u1 = u0 + nst;
    // the last CTA c that begins at or before step x: total c / ctas < x + 1
    const long long c0 = ((u0 + 1) * p.ctas - 1) / total, c1 = (u1 * p.ctas - 1) / total;
    if (c0 == c1) return;  // written already
    float m = -INFINITY;
    for (long long c = c0; c <= c1; ++c) {
        if (total * c / p.ctas == total * (c + 1) / p.ctas) continue;  // a CTA without steps
        const long long slot = c * 2 + (total * c / p.ctas < u0);
        m = fmaxf(m, p.ml[slot * R + r].x);
    }
    const float ms = m == -INFINITY ? 0.f : m;
    float l = 0.f, acc[DV / 32];
#pragma unroll
    for (int q = 0; q < DV / 32; ++q) acc[q] = 0.f;
    for (long long c = c0; c <= c1; ++c) {
        if (total * c / p.ctas == total * (c + 1) / p.ctas) continue;
        const long long slot = c * 2 + (total * c / p.ctas < u0);
        const float2 x = p.ml[slot * R + r];
        if (x.y == 0.f) continue;  // nothing in this piece (NaN is not 0)
        const float f = ex2(x.x - ms);
        l = fmaf(x.y, f, l);
        const float* from = p.part + (slot * R + r) * DV;
#pragma unroll
        for (int q = 0; q < DV / 32; ++q) acc[q] = fmaf(from[lane + 32 * q], f, acc[q]);
    }
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
    int mt, chunks, whole, ctas;
    long long starts, part, ml;  // bytes
};
int resident_of(bool k2, bool v2, int mt) {
    if (mt == 1) return k2 ? (v2 ? resident<128, 128, 1>() : resident<128, 64, 1>()) : (v2 ? resident<64, 128, 1>() : resident<64, 64, 1>());
    return k2 ? (v2 ? resident<128, 128, 2>() : resident<128, 64, 2>()) : (v2 ? resident<64, 128, 2>() : resident<64, 64, 2>());
}
Plan plan_of(const XattnArgs& a, int sms) {
    Plan p{};
    p.mt = a.rows > 16 ? 2 : 1;
    const int R = 16 * p.mt, dv = a.dv > 64 ? 128 : 64;
    p.chunks = (int)((a.rows + R - 1) / R);
    const long long units = (long long)a.B * a.Hkv * p.chunks;
    const long long keys = std::min<long long>(a.Lk, (long long)a.win.window + a.win.sinks + a.Lq);
    p.ctas = sms * resident_of(a.dk > 64, a.dv > 64, p.mt);
    p.whole = (keys <= kWholeSteps * kStep || units >= 16ll * p.ctas) && units <= 0x7fffffffLL;
    if (p.whole) {
        p.ctas = (int)units;
    } else {
        p.starts = (a.B + 2ll) / 2 * 16;
        p.part = 2ll * p.ctas * R * dv * 4;
        p.ml = 2ll * p.ctas * R * 8;
    }
    return p;
}

std::atomic<bool> g_attr[64][8];

template <int DK, int DV, int MT>
cudaError_t launch(const Params& p, int device, cudaStream_t s) {
    std::atomic<bool>& set = g_attr[device][(DK > 64) * 4 + (DV > 64) * 2 + MT - 1];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(k_paged_mma<DK, DV, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)sizeof(Shared<DK, DV, MT>));
        if (e != cudaSuccess) return e;
        set = true;
    }
    k_paged_mma<DK, DV, MT><<<(unsigned)p.ctas, kThreads, sizeof(Shared<DK, DV, MT>), s>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || p.whole) return e;
    const long long rows = (long long)p.a.B * p.a.Hkv * p.chunks * MT * 16;
    k_paged_join<DV, MT><<<(unsigned)((rows + 7) / 8), 256, 0, s>>>(p);
    return cudaGetLastError();
}
template <int MT>
cudaError_t launch_mt(const Params& p, int device, cudaStream_t s) {
    const bool k2 = p.a.dk > 64, v2 = p.a.dv > 64;
    return k2 ? (v2 ? launch<128, 128, MT>(p, device, s) : launch<128, 64, MT>(p, device, s))
              : (v2 ? launch<64, 128, MT>(p, device, s) : launch<64, 64, MT>(p, device, s));
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
    p.ctas = pl.ctas;
    char* ws = (char*)a.ws;
    p.starts = (long long*)ws;
    p.part = (float*)(ws + pl.starts);
    p.ml = (float2*)(ws + pl.starts + pl.part);
    return pl.mt == 1 ? launch_mt<1>(p, device, s) : launch_mt<2>(p, device, s);
}

}  // namespace gs
