// gs_xattn_bwd_tc.cu -- the gradient of cross attention on tcgen05 (bf16 inputs).
//
// Two kernels, each with its own sums in TMEM, so that nothing meets in atomics and results repeat bit for bit:
//   k_xattn_dkv_tc: a CTA keeps a tile of 128 keys (K, V) and walks the packed rows of the key head in tiles of 128:
//     S^T = K Q^T, P^T = 2^(c s - lse log2 e), dV += P^T dO, dP^T = V dO^T, dS^T = P^T (dP^T - D), dK += dS^T Q.
//   k_xattn_dq_tc: a CTA keeps a tile of 128 packed rows (Q, dO) and walks the keys:
//     S = Q K^T, dP = dO V^T, dS = P (dP - D), dQ += dS K.
// S and dP are computed in both (7 products of the tile instead of 5); the alternative, dQ summed from the first
// kernel, needs fp32 atomics on 4 bytes per product of 128 x 128 x dk, and their order changes results.
//
// P and dS go from TMEM to registers and back as bf16, where they are the A operand (lanes are keys in the first kernel,
// rows in the second, so neither needs a transpose); the B operands Q, dO, K are read as they lie (MN-major).  The tile
// that stays lies in TMEM as well (bf16 pairs, 32 columns a chunk of 64), which leaves shared memory to the ring of streamed
// tiles: with two stages the kernels waited for loads of about 1 us each.
//
// The streamed tile is taken in halves of 64: TMEM then holds everything (width 128: 64 + 64 columns of
// operands, 256 of sums, 64 of S, 64 of dP), and two groups of eight softmax warps work in turn, group h on half h.
// Where TMEM has room (in k_xattn_dq_tc; in the first at widths up to 64) each half has an S and a dP of its own.  Warp
// w of a group reads lanes 32 (w % 4)..+31 and columns 32 (w / 4)..+31 of its half.  The rows'
// statistics (-lse log2 e, -D) are laid out per row tile by k_xattn_stats, so that a tile's come with one copy.
//
// P and dS go to bf16 for their products (half a step, 2^-8 relative): the other operands, dO, Q and K, are bf16, and the tensor
// core takes both in one type.  Error of dQ, dK and dV against 64 bits: 2.4e-3 of their norm, 1.7e-3 with fp32 P and dS (through windows of 64
// keys to all of 2,048 2.3e-3 to 2.4e-3, 1.7e-3 the outputs' own rounding).
//
// Measured at 2 sequences of 4,096 x 4,096, 32 / 8 heads of 128: dK and dV 0.71 ms, dQ 0.55 ms, statistics 0.03.  dK and dV keep the
// tensor pipe busy in 77 % of the multiprocessors' active clocks, which are 84 % of the kernel's (512 CTAs on 152 of them), dQ in
// 65 %, where the softmax warps wait for TMEM and for one another; L2, 64 KB a tile and CTA, is 18 and 26 % busy.  At width 64 (8 x
// 1,024 x 750..1,500, 16 heads: 108 and 87 us) a tile takes 1,580 and 1,470 clocks, its four and three products 1,024 and 768, and a CTA's
// start and end took 9,000 of 22,000 clocks before its own tiles came while it is set up and results went out 64 bytes of a row
// at a time (221 -> 207 us for the whole gradient).  (CTAs that go on with another item spill in the loop over tiles, which has no
// register left: 230 us for the whole gradient instead of 207.)
//
// Keys that are not read: P = dS = 0, and in the second kernel their rows of K are zeroed in shared memory before
// the MMA reads them (0 * NaN).  Rows past the end have lse = +inf: P = 0.

#include <stddef.h>

#include <algorithm>
#include <atomic>

#include "gs_xattn_tc.cuh"

namespace gs {
namespace {

using namespace xtc;

__device__ unsigned g_err_xbwd = 0;

constexpr int kSoftWarps = 16, kGroupWarps = 8;
constexpr int kMmaWarp = 16, kTmaWarp = 17, kMaskWarp = 18;
constexpr int kThreads = 19 * 32;
constexpr int kCols = 32;          // of a softmax warp
constexpr int kHalf = kTile / 2;
constexpr uint32_t kHalfBytes = kHalf * kChunk * 2;  // 64 rows of a chunk
constexpr int kStats = 2 * kTile;  // floats of a row tile: -lse log2 e (-inf: no weight), then -D

struct Ctl {
    uint64_t own_full;                               // the tiles that stay are in TMEM
    uint64_t a_full[4], a_empty[4], a_ready[4];      // Q (dkv) or K (dq) stages
    uint64_t b_full[4], b_empty[4];                  // dO (dkv) or V (dq) stages
    uint64_t st_full[4], st_empty[4];                // dkv: row statistics
    uint64_t s_full[2], p_full[2], dp_full[2], ds_full[2];  // MMA <-> softmax group
    uint64_t s_free[2];                              // dq: S has been read
    uint64_t done;
    alignas(16) float stats[4][kStats];              // dkv; read 16 bytes at a time
    float dpart[4][kTile];                           // dq: parts of D
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(offsetof(Ctl, stats) % 16 == 0, "bulk copies, float4 reads");

struct Params {
    XattnArgs a;
    int qmul, omul, kmul, khmul, vmul, vhmul;  // HeadMap multipliers: q, dO (batch), k and v (batch, head)
    int nl;
    long long rtiles;
    int ktiles;
    int vec_q, vec_k, vec_v;  // outputs on 16-byte boundaries
};

template <int DKC, int DVC>
struct Cfg {
    static constexpr int kStageBytes = (DKC + DVC) * kChunkBytes;
    static constexpr int kRoom = (227 * 1024 - 1024 - (int)sizeof(Ctl)) / kStageBytes;
    static constexpr int kStages = kRoom < 4 ? kRoom : 4;
    static constexpr size_t kSmem = 1024 + (size_t)kStageBytes * kStages + sizeof(Ctl);
    static constexpr int kBuffers = 96 * (DKC + DVC) + 256 <= 512 ? 2 : 1;  // dkv: S and dP of each half, or one for both
    static_assert(kStages >= 2, "ring too short");
    static_assert(96 * (DKC + DVC) + 128 * kBuffers <= 512 && 96 * DKC + 32 * DVC + 256 <= 512, "TMEM");
};

// The part with number `part` of four of the row at `row` (w elements, zeros where !has): bf16 pairs, CHUNKS * 8 words.
template <int CHUNKS>
__device__ __forceinline__ void load_row(uint32_t (&x)[CHUNKS][8], const __nv_bfloat16* row, int w, bool has, int part) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) load_words(x[c], row, c * kChunk + part * 16, w, has);
}
// into columns [taddr, + CHUNKS * 32) of this thread's lane, which four warps share
template <int CHUNKS>
__device__ __forceinline__ void keep_row(uint32_t taddr, const uint32_t (&x)[CHUNKS][8], int part) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) tmem_st8(taddr + (uint32_t)((c * kChunk + part * 16) / 2), x[c]);
}

// -lse log2 e of a row: -inf where the row has no weight (P = 0); a NaN or +inf lse gives NaN, as the forward result is
__device__ __forceinline__ float neg_lse2(float lse) {
    return lse == -INFINITY ? -INFINITY : lse == INFINITY ? NAN : -lse * kLog2e;
}

// 32 fp32 columns of this thread's lane to global
__device__ __forceinline__ void store32(float* dst, const float* v, int left, bool vec) {
    if (vec) {
#pragma unroll
        for (int e = 0; e < 32; e += 4)
            if (e < left) *reinterpret_cast<float4*>(dst + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    } else {
#pragma unroll
        for (int e = 0; e < 32; ++e)
            if (e < left) dst[e] = v[e];
    }
}
// Columns [c0, c1) of an accumulator of `cols` (a whole warp), times mul, zeros where !keep, to out (bf16) or part (fp32)
__device__ __forceinline__ void drain_acc(uint32_t taddr, int c0, int c1, int cols, bool any, bool keep, bool mine, float mul,
                                          __nv_bfloat16* out, bool vec, float* part) {
    for (int q = c0; q < min(c1, cols); q += 32) {
        __syncwarp();
        float v[32];
        if (any) tmem_ld32(taddr + (uint32_t)q, v);
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = any && keep ? v[e] * mul : 0.f;
        if (part) {
            if (mine) store32(part + q, v, cols - q, cols % 4 == 0);
        } else {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
            if (vec)
                store_rows(out + q, w, cols - q, mine);
            else
                store_rows_any(out + q, w, cols - q, mine);
        }
    }
}

// sum of the products of two rows' 8 bf16 elements
__device__ __forceinline__ float dot_eight(const uint4& x, const uint4& y, float acc) {
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        acc = fmaf(__uint_as_float(xs[e] << 16), __uint_as_float(ys[e] << 16), acc);
        acc = fmaf(__uint_as_float(xs[e] & 0xffff0000u), __uint_as_float(ys[e] & 0xffff0000u), acc);
    }
    return acc;
}

// Through a window: a row whose span is one key at most has no dS, exactly (its weight is 1 whatever its logit), where P (dP - D) would
// leave a rounding, as it does where a key mask leaves one key of more.  kOneKey in D's place says so; a D that is infinite goes there as NaN.
constexpr float kOneKey = INFINITY;
__device__ __forceinline__ float not_one_key(float nd) { return nd == kOneKey ? NAN : nd; }

// The key tiles that some row of a row tile sees through a window: first sinks, then the window.  Where the window's are two or fewer,
// the dQ kernel sums D = sum_j P dP itself, in a pass of its own ahead (few): with some ten keys a D from a bf16 O adds half as much
// error to dQ as the rounding of dS does.
struct RowTile {
    KeySpan span;
    int sinks, skip, count;
    bool few;
};
__device__ __forceinline__ RowTile row_tile(const XattnArgs& a, int b, int rt, int nl, int n) {
    RowTile t;
    t.span = key_span<kWindowKeys>(a, b, rt * nl, min(rt * nl + nl, a.Lq) - 1, n);
    const int from = t.span.lo / kTile, window = max(0, (t.span.hi + kTile - 1) / kTile - from);
    t.sinks = min((t.span.sink + kTile - 1) / kTile, from);
    t.skip = from - t.sinks;
    t.count = t.sinks + window;
    t.few = window <= 2 && t.sinks <= 1;
    return t;
}

// D = sum_j P dP of the rows that see kFewKeys keys or fewer, instead of <dO, O> with a rounded O (few_keys): 16 threads a row, two rows
// a warp in step.
__device__ __forceinline__ void sum_few_seen(const XattnArgs& a, int b, int hk, long long rt, int nl, int grp, int ln, int n, float* dst) {
    const __nv_bfloat16* keys = reinterpret_cast<const __nv_bfloat16*>(a.k.p) + b * a.k.b + hk * a.k.h;
    const __nv_bfloat16* values = reinterpret_cast<const __nv_bfloat16*>(a.v.p) + b * a.v.b + hk * a.v.h;
    const float cs = a.scale * kLog2e;
    const int c0 = ln * 8;
#pragma unroll 1
    for (int r = grp; r < kTile; r += 16) {
        if (r >= grp + 64) break;  // (a block's 64 slots)
        const int l = r / a.G, h = hk * a.G + r - l * a.G;
        const long long ql = rt * nl + l;
        const bool row = l < nl && ql < a.Lq;
        KeySpan sp{0, 0, 0};
        if (row) sp = key_span<kWindowKeys>(a, b, ql, ql, n);
        int key = 0;
        const int few = few_seen<16>(a, b, sp, key), most = max(few, __shfl_xor_sync(0xffffffffu, few, 16));
        if (most <= 0) continue;  // both rows of the warp
        const bool on = few > 0;
        const uint4 q = load_eight(reinterpret_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.b + (on ? ql : 0) * a.q.l + (on ? h : 0) * a.q.h,
                                   c0, a.dk, on);
        const uint4 d = load_eight(reinterpret_cast<const __nv_bfloat16*>(a.dO.p) + b * a.dO.b + (on ? ql : 0) * a.dO.l + (on ? h : 0) * a.dO.h,
                                   c0, a.dv, on);
        const float nl2 = on ? neg_lse2(a.lse[((long long)b * a.Hq + h) * a.Lq + ql]) : -INFINITY;
        float sum = 0.f;
        for (int f = 0; f < most; ++f) {
            const long long j = __shfl_sync(0xffffffffu, key, f, 16);
            const bool in = f < few;
            float s = dot_eight(q, load_eight(keys + (in ? j : 0) * a.k.l, c0, a.dk, in), 0.f);
            float dp = dot_eight(d, load_eight(values + (in ? j : 0) * a.v.l, c0, a.dv, in), 0.f);
#pragma unroll
            for (int o = 8; o; o >>= 1) {
                s += __shfl_xor_sync(0xffffffffu, s, o);
                dp += __shfl_xor_sync(0xffffffffu, dp, o);
            }
            if (in) sum = fmaf(ex2(fmaf(s, cs, nl2)), dp, sum);
        }
        if (on && ln == 0) dst[kTile + r] = nl2 == -INFINITY ? 0.f : not_one_key(-sum);
    }
}

// Statistics of every row tile of a key head: slots without a row get (-inf, 0).  16 threads a row, 8 columns each, four rows
// in flight a thread, 64 slots a block.  Bound by instructions, mostly addresses (issue 69 %; 8 x 1,024 rows of 16 heads of 64,
// 34 MB: 15 us; two rows in flight and lse read last 17).  Where a mask leaves few keys, D is summed from them instead (9 of
// 1,500 keys, 4 x 64 rows of 16 heads of 64: the whole gradient 59 -> 73 us).
// Through a window (WIN), rows that see few keys are looked at one by one: the first rows of a sequence, or all of a short window.
constexpr int kStatRows = 4, kStatBlocks = kTile / (16 * kStatRows);
template <bool WIN>
__global__ void __launch_bounds__(256) k_xattn_stats(const XattnArgs a, int nl, long long rtiles, int vec) {
    unsigned i = blockIdx.x / kStatBlocks;  // (in 32 bits, as all of these kernels' places: a grid has no more blocks)
    float* dst = a.ws + (long long)i * kStats;
    const long long rt = i % (unsigned)rtiles;
    i /= (unsigned)rtiles;
    const int b = (int)(i / (unsigned)a.Hkv), hk = (int)i - b * a.Hkv;
    const int grp = (blockIdx.x % kStatBlocks) * (16 * kStatRows) + (threadIdx.x >> 4), ln = threadIdx.x & 15, c0 = ln * 8;
    float L[kStatRows], acc[kStatRows];
    uint4 x[kStatRows], y[kStatRows];
#pragma unroll
    for (int k = 0; k < kStatRows; ++k) {
        const int r = grp + 16 * k, l = r / a.G, h = hk * a.G + r - l * a.G;
        const long long ql = rt * nl + l;
        const bool row = l < nl && ql < a.Lq;
        L[k] = -INFINITY;
        acc[k] = 0.f;
        x[k] = y[k] = make_uint4(0, 0, 0, 0);
        if (row && ln == 0) L[k] = a.lse[((long long)b * a.Hq + h) * a.Lq + ql];
        if (!row || c0 >= a.dv) continue;
        const __nv_bfloat16* o = reinterpret_cast<const __nv_bfloat16*>(a.o.p) + b * a.o.b + ql * a.o.l + h * a.o.h + c0;
        const __nv_bfloat16* d = reinterpret_cast<const __nv_bfloat16*>(a.dO.p) + b * a.dO.b + ql * a.dO.l + h * a.dO.h + c0;
        if (vec) {
            x[k] = __ldg(reinterpret_cast<const uint4*>(o));
            y[k] = __ldg(reinterpret_cast<const uint4*>(d));
        } else {
            for (int e = 0; e < 8 && c0 + e < a.dv; ++e) acc[k] = fmaf(__bfloat162float(o[e]), __bfloat162float(d[e]), acc[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < kStatRows; ++k) {
        if (vec) acc[k] = dot_eight(x[k], y[k], acc[k]);
#pragma unroll
        for (int o = 8; o; o >>= 1) acc[k] += __shfl_xor_sync(0xffffffffu, acc[k], o);
        if (ln == 0) {
            const int r = grp + 16 * k;
            const float nl2 = neg_lse2(L[k]);
            dst[r] = nl2;
            const float nd = nl2 == -INFINITY ? 0.f : -acc[k];
            dst[kTile + r] = WIN ? not_one_key(nd) : nd;
        }
    }
    const int n = keys_of(a, b);
    if constexpr (WIN) {
        // whether to look at all, by one warp (by all eight: 20 of 47 us for 2 x 4,096 rows of 32 heads of 128)
        __shared__ int look;  // 1: for rows of few keys, 2: for rows of one key
        if (threadIdx.x < 32) {  // (along a tile the number of keys grows, then falls: the first and the last row see the fewest)
            const int first = (int)rt * nl, last = min(first + nl, a.Lq) - 1;
            const int least = min(key_span<kWindowKeys>(a, b, first, first, n).count(), key_span<kWindowKeys>(a, b, last, last, n).count());
            const bool few = !row_tile(a, b, (int)rt, nl, n).few && (a.mask || least <= kFewKeys);  // (else the dQ kernel sums D)
            if (threadIdx.x == 0) look = (few ? 1 : 0) | (least <= 1 ? 2 : 0);
        }
        __syncthreads();
        if (look & 1) sum_few_seen(a, b, hk, rt, nl, grp, ln, n, dst);
        if ((look & 2) && ln == 0)
            for (int r = grp; r < grp + 16 * kStatRows; r += 16) {
                const int l = r / a.G, ql = (int)rt * nl + l;
                if (l < nl && ql < a.Lq && key_span<kWindowKeys>(a, b, ql, ql, n).count() <= 1) dst[kTile + r] = kOneKey;
            }
        return;
    }
    if (!a.mask || n <= kTile) return;  // (up to a tile's keys: k_xattn_dq_tc sums D)
    // each warp looks through an eighth of the mask (65,536 keys, nine of them read: the whole call 305 us where each took all of it)
    __shared__ int counts[8], found[8][kFewKeys];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = (n + 7) / 8, from = min(n, warp * piece);
    int key = 0, few = few_keys(a, b, from, min(n, from + piece), key);
    if (lane < few) found[warp][lane] = key;
    if (lane == 0) counts[warp] = few;
    __syncthreads();
    few = 0;
    for (int w = 0; w < 8; ++w) {
        const int m = counts[w];
        if (m < 0 || few + m > kFewKeys) return;  // too many: D stays <dO, O>
        if (lane >= few && lane < few + m) key = found[w][lane - few];
        few += m;
    }
    const __nv_bfloat16* keys = reinterpret_cast<const __nv_bfloat16*>(a.k.p) + b * a.k.b + hk * a.k.h;
    const __nv_bfloat16* values = reinterpret_cast<const __nv_bfloat16*>(a.v.p) + b * a.v.b + hk * a.v.h;
    const float cs = a.scale * kLog2e;
#pragma unroll 1
    for (int r = grp; r < grp + 16 * kStatRows; r += 16) {  // D = sum_j P dP instead
        const int l = r / a.G, h = hk * a.G + r - l * a.G;
        const bool row = l < nl && rt * nl + l < a.Lq;
        const long long ql = row ? rt * nl + l : 0;
        const uint4 q = load_eight(reinterpret_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.b + ql * a.q.l + (row ? h : 0) * a.q.h, c0, a.dk, row);
        const uint4 d = load_eight(reinterpret_cast<const __nv_bfloat16*>(a.dO.p) + b * a.dO.b + ql * a.dO.l + (row ? h : 0) * a.dO.h, c0, a.dv, row);
        const float nl2 = row ? neg_lse2(a.lse[((long long)b * a.Hq + h) * a.Lq + ql]) : -INFINITY;
        float sum = 0.f;
        for (int f = 0; f < few; ++f) {
            const long long j = __shfl_sync(0xffffffffu, key, f);
            float s = dot_eight(q, load_eight(keys + j * a.k.l, c0, a.dk, true), 0.f);
            float dp = dot_eight(d, load_eight(values + j * a.v.l, c0, a.dv, true), 0.f);
#pragma unroll
            for (int o = 8; o; o >>= 1) {
                s += __shfl_xor_sync(0xffffffffu, s, o);
                dp += __shfl_xor_sync(0xffffffffu, dp, o);
            }
            sum = fmaf(ex2(fmaf(s, cs, nl2)), dp, sum);
        }
        if (ln == 0) dst[kTile + r] = nl2 == -INFINITY ? 0.f : -sum;
    }
}

template <int DKC, int DVC, bool WIN>
__global__ void __launch_bounds__(kThreads, 1)
    k_xattn_dkv_tc(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mo, const Params p) {
    using C = Cfg<DKC, DVC>;
    constexpr int ST = C::kStages, NB = C::kBuffers;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    uint8_t* base = smem_raw + (((raw + 1023u) & ~1023u) - raw);
    uint8_t* Qr = base;                                   // ring of Q tiles
    uint8_t* Or = Qr + (size_t)ST * DKC * kChunkBytes;    // ring of dO tiles
    Ctl& c = *reinterpret_cast<Ctl*>(Or + (size_t)ST * DVC * kChunkBytes);
    volatile int* abort_flag = &c.abort_flag;
    unsigned* err = &g_err_xbwd;
    const XattnArgs& a = p.a;
    const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31;

    unsigned i = blockIdx.x;
    const unsigned rtiles = (unsigned)p.rtiles;
    int kt, part, hk, b, parts = a.rsplits;
    if constexpr (WIN) {  // key tiles slowest: the first ones, which the most rows see, begin first
        hk = (int)(i % (unsigned)a.Hkv);
        i /= (unsigned)a.Hkv;
        b = (int)(i % (unsigned)a.B);
        i /= (unsigned)a.B;
        part = 0;
        kt = (int)i;
        if (parts > 1) {
            const int in_parts = (a.pkeys + kTile - 1) / kTile;
            if ((int)i < in_parts * parts) {
                kt = (int)i / parts;
                part = (int)i - kt * parts;
            } else {
                kt = (int)i - in_parts * (parts - 1);
                parts = 1;
            }
        }
    } else {
        kt = (int)(i % (unsigned)p.ktiles);
        i /= (unsigned)p.ktiles;
        part = (int)(i % (unsigned)parts);
        i /= (unsigned)parts;
        hk = (int)(i % (unsigned)a.Hkv);
        b = (int)(i / (unsigned)a.Hkv);
    }
    const int tile_rows = p.nl * a.G;
    const int n = keys_of(a, b), j0 = kt * kTile;
    int t0 = 0, t1 = (int)rtiles;
    if constexpr (WIN) {  // the row tiles that see some key of the tile
        const RowSpan rows = row_span(a, b, j0, min(n, j0 + kTile));
        t0 = (int)rows.first / p.nl;
        t1 = max(t0, (int)((unsigned)rows.end + p.nl - 1) / p.nl);
    }
    if (parts > 1) {
        const long long first = t0, some = t1 - t0;
        t0 = (int)(first + some * part / parts);
        t1 = (int)(first + some * (part + 1) / parts);
    }
    const int nt = uniform(j0 < n ? t1 - t0 : 0);  // row tiles

    // the softmax warps' parts of K and V, on their way while the CTA is set up
    uint32_t kx[DKC][8], vx[DVC][8];
    if (warp < kSoftWarps && nt > 0) {
        const int j = j0 + (warp & 3) * 32 + lane;
        const long long jj = j < a.Lk ? j : 0;
        load_row(kx, reinterpret_cast<const __nv_bfloat16*>(a.k.p) + b * a.k.b + jj * a.k.l + hk * a.k.h, a.dk, j < a.Lk, warp >> 2);
        load_row(vx, reinterpret_cast<const __nv_bfloat16*>(a.v.p) + b * a.v.b + jj * a.v.l + hk * a.v.h, a.dv, j < a.Lk, warp >> 2);
    }
    if (threadIdx.x == 0) {
        mbar_init(&c.own_full, kSoftWarps);
        for (int s = 0; s < ST; ++s) {
            mbar_init(&c.a_full[s], 1);
            mbar_init(&c.a_empty[s], 1);
            mbar_init(&c.b_full[s], 1);
            mbar_init(&c.b_empty[s], 1);
            mbar_init(&c.st_full[s], 1);
            mbar_init(&c.st_empty[s], kSoftWarps);
        }
        for (int h = 0; h < 2; ++h) {
            mbar_init(&c.s_full[h], 1);
            mbar_init(&c.dp_full[h], 1);
            mbar_init(&c.p_full[h], kGroupWarps);
            mbar_init(&c.ds_full[h], kGroupWarps);
        }
        mbar_init(&c.done, 1);
        c.abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&c.tmem_base, 512);
        tmem_relinquish();
    }
    // rows of a tile that its box does not write (128 % G != 0) are summed over all the same: zeros
    if (tile_rows < kTile) {
        const int words = (kTile - tile_rows) * 8;  // 16-byte words per chunk
        for (int e = threadIdx.x; e < ST * (DKC + DVC) * words; e += kThreads)
            *reinterpret_cast<uint4*>(Qr + (size_t)(e / words) * kChunkBytes + tile_rows * 128 + (e % words) * 16) =
                make_uint4(0, 0, 0, 0);
        fence_proxy_async();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(c.tmem_base);
    const uint32_t t_k = tmem, t_v = t_k + 32 * DKC, t_dk = t_v + 32 * DVC, t_dv = t_dk + 64 * DKC;
    const uint32_t t_s = t_dv + 64 * DVC, t_dp = t_s + 64 * NB;  // half h: + 64 h where each has its own

    if (warp == kTmaWarp) {
        if (lane == 0 && nt > 0) {
            RingPos rp;
            int sa = 0, sb = 0, ss = 0;
            for (int t = 0; t < nt; ++t, rp.next(ST)) {
                const int s = rp.idx, l0 = (t0 + t) * p.nl;
                if (!mbar_wait_1t(&c.a_empty[s], rp.phase ^ 1u, abort_flag, err)) break;
                mbar_arrive_expect_tx(&c.a_full[s], (uint32_t)(DKC * kChunk * 2 * tile_rows));
                for (int k = 0; k < DKC; ++k)
                    tma_load_4d(Qr + (size_t)(s * DKC + k) * kChunkBytes, &mq, &c.a_full[s], k * kChunk, hk * a.G, l0,
                                b * p.qmul);
                ++sa;
                if (!mbar_wait_1t(&c.st_empty[s], rp.phase ^ 1u, abort_flag, err)) break;
                mbar_arrive_expect_tx(&c.st_full[s], (uint32_t)sizeof(c.stats[0]));
                bulk_load(c.stats[s], a.ws + (((long long)b * a.Hkv + hk) * p.rtiles + t0 + t) * kStats, sizeof(c.stats[0]),
                          &c.st_full[s]);
                ++ss;
                if (!mbar_wait_1t(&c.b_empty[s], rp.phase ^ 1u, abort_flag, err)) break;
                mbar_arrive_expect_tx(&c.b_full[s], (uint32_t)(DVC * kChunk * 2 * tile_rows));
                for (int k = 0; k < DVC; ++k)
                    tma_load_4d(Or + (size_t)(s * DVC + k) * kChunkBytes, &mo, &c.b_full[s], k * kChunk, hk * a.G, l0,
                                b * p.omul);
                ++sb;
            }
            for (int j = std::max(0, sa - ST); j < sa; ++j) mbar_drain(&c.a_full[j % ST], (uint32_t)(j / ST) & 1u, err);
            for (int j = std::max(0, ss - ST); j < ss; ++j) mbar_drain(&c.st_full[j % ST], (uint32_t)(j / ST) & 1u, err);
            for (int j = std::max(0, sb - ST); j < sb; ++j) mbar_drain(&c.b_full[j % ST], (uint32_t)(j / ST) & 1u, err);
        }
    } else if (warp == kMmaWarp) {
        if (nt > 0) {
            const uint32_t el = elect_one();
            const uint32_t id_s = idesc_bf16_f32(kHalf), id_v = idesc_bf16_bmn(DVC * kChunk), id_k = idesc_bf16_bmn(DKC * kChunk);
            const uint32_t qa = smem_u32(Qr), oa = smem_u32(Or);
            // step u: half u % 2 of row tile u / 2; S and dP run NB steps ahead of the sums
            RingPos cur, nxt;  // stages of the sums' tile and of S and dP's
            const int steps = 2 * nt;
            auto scores = [&](int u) {
                const int h = u & 1;
                if (h == 0 && !mbar_wait_warp_inline(&c.a_full[nxt.idx], nxt.phase, abort_flag, err)) return false;
                tc_fence_after();
                mma_rows_ts<DKC>(t_s + (NB == 2 ? 64u * h : 0u), t_k, qa + (uint32_t)(nxt.idx * DKC * kChunkBytes) + h * kHalfBytes,
                                 id_s, el);
                commit_to(&c.s_full[h], el);
                return true;
            };
            auto dprod = [&](int u) {
                const int h = u & 1;
                if (h == 0 && !mbar_wait_warp_inline(&c.b_full[nxt.idx], nxt.phase, abort_flag, err)) return false;
                tc_fence_after();
                mma_rows_ts<DVC>(t_dp + (NB == 2 ? 64u * h : 0u), t_v, oa + (uint32_t)(nxt.idx * DVC * kChunkBytes) + h * kHalfBytes,
                                 id_s, el);
                commit_to(&c.dp_full[h], el);
                if (h == 1) nxt.next(ST);
                return true;
            };
            bool ok = mbar_wait_warp_inline(&c.own_full, 0, abort_flag, err);
            for (int u = 0; u < NB && ok; ++u) ok = scores(u) && dprod(u);
            for (int u = 0; u < steps && ok; ++u) {
                const int h = u & 1;
                const uint32_t ph = (uint32_t)(u >> 1) & 1u, buf = NB == 2 ? 64u * h : 0u;
                if (!(ok = mbar_wait_warp_inline(&c.p_full[h], ph, abort_flag, err))) break;
                tc_fence_after();
                mma_tile_ts<32, 4>(t_dv, t_s + buf, oa + (uint32_t)(cur.idx * DVC * kChunkBytes) + h * kHalfBytes, id_v, u != 0, el);
                if (u + NB < steps && !(ok = scores(u + NB))) break;
                if (!(ok = mbar_wait_warp_inline(&c.ds_full[h], ph, abort_flag, err))) break;
                tc_fence_after();
                mma_tile_ts<32, 4>(t_dk, t_dp + buf, qa + (uint32_t)(cur.idx * DKC * kChunkBytes) + h * kHalfBytes, id_k, u != 0, el);
                if (u + NB < steps && !(ok = dprod(u + NB))) break;
                if (h == 1) {
                    commit_to(&c.b_empty[cur.idx], el);
                    commit_to(&c.a_empty[cur.idx], el);
                    cur.next(ST);
                }
            }
            commit_to(&c.done, el);
            mbar_drain(&c.done, 0, err);
        }
    } else if (warp < kSoftWarps) {
        // ------------------------------------------------------------- softmax warps: a lane is a key
        const int h = warp >> 3, cw = (warp >> 2) & 1, quad = warp & 3;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t col = lane_base + (NB == 2 ? 64u * h : 0u) + (uint32_t)(kCols * cw);
        const uint32_t ts = t_s + col, td = t_dp + col;
        const int j = j0 + quad * 32 + lane;
        const bool valid = j < n && (!a.mask || __ldg(a.mask + (long long)b * a.ldm + j) != 0);
        const bool whole_keys = __all_sync(0xffffffffu, valid);
        const float cs = a.scale * kLog2e;
        // through a window: the rows of the first tile, from its start, that see key j are first_row..end_row - 1 (before G)
        [[maybe_unused]] int first_row = 0, end_row = 0;
        if constexpr (WIN) {
            const RowSpan rows = row_span(a, b, j, j + 1);
            first_row = (int)rows.first - t0 * p.nl;
            end_row = (int)rows.end - t0 * p.nl;
        }
        if (nt > 0) {
            keep_row(t_k + lane_base, kx, warp >> 2);
            keep_row(t_v + lane_base, vx, warp >> 2);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.own_full);
        }
        RingPos rp;
        bool ok = true;
        for (int t = 0; t < nt; ++t, rp.next(ST)) {
            const uint32_t ph = (uint32_t)t & 1u;
            uint32_t see = valid ? 0xffffffffu : 0u;  // this warp's rows that see this lane's key
            bool whole = whole_keys;
            if constexpr (WIN) {
                const int l = t * p.nl, x = min(max(first_row - l, 0), p.nl) * a.G, y = min(max(end_row - l, 0), p.nl) * a.G;
                see &= bits_between(x - (kHalf * h + kCols * cw), y - (kHalf * h + kCols * cw));
                whole = __all_sync(0xffffffffu, see == 0xffffffffu);
            }
            if (!mbar_wait_warp_inline(&c.st_full[rp.idx], rp.phase, abort_flag, err) ||
                !mbar_wait_warp_inline(&c.s_full[h], ph, abort_flag, err)) {
                ok = false;
                break;
            }
            tc_fence_after();
            uint32_t sr[kCols], pk[kCols / 2];
            float* s = reinterpret_cast<float*>(sr);
            tmem_ld32_issue(ts, sr);
            tmem_wait_ld32(sr);
            const float4* nl = reinterpret_cast<const float4*>(&c.stats[rp.idx][kHalf * h + kCols * cw]);
            const float4* nd = reinterpret_cast<const float4*>(&c.stats[rp.idx][kTile + kHalf * h + kCols * cw]);
#pragma unroll
            for (int q = 0; q < kCols / 4; ++q) {
                const float4 L = nl[q];
                float* x = s + 4 * q;
                x[0] = ex2(fmaf(x[0], cs, L.x));
                x[1] = ex2(fmaf(x[1], cs, L.y));
                x[2] = ex2(fmaf(x[2], cs, L.z));
                x[3] = ex2(fmaf(x[3], cs, L.w));
            }
            if (!whole) {
#pragma unroll
                for (int q = 0; q < kCols; ++q) s[q] = (WIN ? (see >> q) & 1u : valid) ? s[q] : 0.f;
            }
#pragma unroll
            for (int q = 0; q < kCols / 2; ++q) pk[q] = pack_bf16(s[2 * q], s[2 * q + 1]);
            tmem_st16(ts, pk);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.p_full[h]);
            if (!mbar_wait_warp_inline(&c.dp_full[h], ph, abort_flag, err)) {
                ok = false;
                break;
            }
            tc_fence_after();
            uint32_t dr[kCols];
            float* d = reinterpret_cast<float*>(dr);
            tmem_ld32_issue(td, dr);
            tmem_wait_ld32(dr);
            bool all = whole;
            if constexpr (WIN) {
                see &= ~__ballot_sync(0xffffffffu, c.stats[rp.idx][kTile + kHalf * h + kCols * cw + lane] == kOneKey);
                all = __all_sync(0xffffffffu, see == 0xffffffffu);
            }
#pragma unroll
            for (int q = 0; q < kCols / 4; ++q) {
                const float4 D = nd[q];
                float* x = d + 4 * q;
                add2(x[0], x[1], D.x, D.y);
                add2(x[2], x[3], D.z, D.w);
                mul2(x[0], x[1], s[4 * q], s[4 * q + 1]);
                mul2(x[2], x[3], s[4 * q + 2], s[4 * q + 3]);
            }
            if (!all) {
#pragma unroll
                for (int q = 0; q < kCols; ++q) d[q] = (WIN ? (see >> q) & 1u : valid) ? d[q] : 0.f;
            }
#pragma unroll
            for (int q = 0; q < kCols / 2; ++q) pk[q] = pack_bf16(d[2 * q], d[2 * q + 1]);
            tmem_st16(td, pk);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&c.ds_full[h]);
                mbar_arrive(&c.st_empty[rp.idx]);
            }
        }
        if (ok && nt > 0) ok = mbar_wait_warp_inline(&c.done, 0, abort_flag, err);
        tc_fence_after();
        if (ok) {  // group 0 writes dV, group 1 dK, 64 columns a warp
            const bool mine = j < a.Lk;
            const long long jj = mine ? j : 0;
            const long long at = (long long)part * xattn_keys(a) + ((long long)b * a.Hkv + hk) * a.pkeys + jj;
            const bool sums = parts > 1;
            const int c0 = cw * 64;
            if (h == 0)
                drain_acc(t_dv + lane_base, c0, c0 + 64, a.dv, nt > 0, valid, mine, 1.f,
                          reinterpret_cast<__nv_bfloat16*>(a.dV.p) + b * a.dV.b + jj * a.dV.l + hk * a.dV.h, p.vec_v != 0,
                          sums ? a.ws + xattn_ws_dv(a) + at * a.dv : nullptr);
            else
                drain_acc(t_dk + lane_base, c0, c0 + 64, a.dk, nt > 0, valid, mine, sums ? 1.f : a.scale,
                          reinterpret_cast<__nv_bfloat16*>(a.dK.p) + b * a.dK.b + jj * a.dK.l + hk * a.dK.h, p.vec_k != 0,
                          sums ? a.ws + xattn_ws_dk(a) + at * a.dk : nullptr);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int DKC, int DVC, bool WIN>
__global__ void __launch_bounds__(kThreads, 1)
    k_xattn_dq_tc(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const Params p) {
    using C = Cfg<DKC, DVC>;
    constexpr int ST = C::kStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    uint8_t* base = smem_raw + (((raw + 1023u) & ~1023u) - raw);
    uint8_t* Kr = base;                                 // ring of K tiles
    uint8_t* Vr = Kr + (size_t)ST * DKC * kChunkBytes;  // ring of V tiles
    Ctl& c = *reinterpret_cast<Ctl*>(Vr + (size_t)ST * DVC * kChunkBytes);
    volatile int* abort_flag = &c.abort_flag;
    unsigned* err = &g_err_xbwd;
    const XattnArgs& a = p.a;
    const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31;

    unsigned i = blockIdx.x;
    int rt;
    int part, hk, b;
    if constexpr (WIN) {  // row tiles slowest, from the last one on: without a window it sees the most keys
        hk = (int)(i % (unsigned)a.Hkv);
        i /= (unsigned)a.Hkv;
        b = (int)(i % (unsigned)a.B);
        i /= (unsigned)a.B;
        part = (int)(i % (unsigned)a.splits);
        rt = (int)((unsigned)p.rtiles - 1 - i / (unsigned)a.splits);
    } else {
        rt = (int)(i % (unsigned)p.rtiles);
        i /= (unsigned)p.rtiles;
        part = (int)(i % (unsigned)a.splits);
        i /= (unsigned)a.splits;
        hk = (int)(i % (unsigned)a.Hkv);
        b = (int)(i / (unsigned)a.Hkv);
    }
    const int tile_rows = p.nl * a.G;
    const int n = keys_of(a, b);
    // the key tiles, or, through a window, those that some row of the tile sees, the first `ahead` of them D's (t0 is theirs then too)
    int t0, t1, sinks = 0, skip = 0, ahead = 0;
    bool few = false;
    KeySpan span{0, 0, 0};
    if constexpr (WIN) {
        const RowTile tile = row_tile(a, b, rt, p.nl, n);
        span = tile.span;
        sinks = tile.sinks;
        skip = tile.skip;
        few = tile.few;
        t0 = 0;
        t1 = tile.count;
        if (few) {  // all in one part
            if (part != 0) t1 = 0;
            if (t1 > 1) ahead = t1;
        } else if (a.splits > 1) {
            t0 = (int)((long long)tile.count * part / a.splits);
            t1 = (int)((long long)tile.count * (part + 1) / a.splits);
        }
    } else {
        t0 = (int)((long long)p.ktiles * part / a.splits);
        t1 = min((int)((long long)p.ktiles * (part + 1) / a.splits), (n + kTile - 1) / kTile);
    }
    if constexpr (WIN) ahead = uniform(ahead);
    const int nt = uniform(max(0, t1 - t0)) + ahead;  // key tiles to go through
    auto first_key = [&](int t) {
        if (WIN && t >= ahead) t -= ahead;
        return (WIN && t0 + t >= sinks ? t0 + t + skip : t0 + t) * kTile;
    };
    const bool fix = WIN || a.lens != nullptr || a.mask != nullptr;

    // the softmax warps' parts of Q and dO, on their way while the CTA is set up
    uint32_t qx[DKC][8], ox[DVC][8];
    if (warp < kSoftWarps && nt > 0) {
        const int r = (warp & 3) * 32 + lane, l = r / a.G;
        const bool mine = r < tile_rows && rt * tile_rows + r < a.rows;
        const long long ql = mine ? rt * p.nl + l : 0;
        const int hq = hk * a.G + (mine ? r - l * a.G : 0);
        load_row(qx, reinterpret_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.b + ql * a.q.l + hq * a.q.h, a.dk, mine, warp >> 2);
        load_row(ox, reinterpret_cast<const __nv_bfloat16*>(a.dO.p) + b * a.dO.b + ql * a.dO.l + hq * a.dO.h, a.dv, mine, warp >> 2);
    }
    if (threadIdx.x == 0) {
        mbar_init(&c.own_full, kSoftWarps);
        for (int s = 0; s < ST; ++s) {
            mbar_init(&c.a_full[s], 1);
            mbar_init(&c.a_empty[s], 1);
            mbar_init(&c.a_ready[s], 1);
            mbar_init(&c.b_full[s], 1);
            mbar_init(&c.b_empty[s], 1);
        }
        for (int h = 0; h < 2; ++h) {
            mbar_init(&c.s_full[h], 1);
            mbar_init(&c.dp_full[h], 1);
            mbar_init(&c.ds_full[h], kGroupWarps);
            mbar_init(&c.s_free[h], kGroupWarps);
        }
        mbar_init(&c.done, 1);
        c.abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&c.tmem_base, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(c.tmem_base);
    const uint32_t t_q = tmem, t_do = t_q + 32 * DKC, t_dq = t_do + 32 * DVC;
    const uint32_t t_s = t_dq + 64 * DKC, t_dp = t_s + 128;  // half h: + 64 h

    if (warp == kTmaWarp) {
        if (lane == 0 && nt > 0) {
            RingPos rp;
            int sa = 0, sb = 0;
            for (int t = 0; t < nt; ++t, rp.next(ST)) {
                const int s = rp.idx;
                if (!mbar_wait_1t(&c.a_empty[s], rp.phase ^ 1u, abort_flag, err)) break;
                mbar_arrive_expect_tx(&c.a_full[s], (uint32_t)(DKC * kChunkBytes));
                for (int k = 0; k < DKC; ++k)
                    tma_load_4d(Kr + (size_t)(s * DKC + k) * kChunkBytes, &mk, &c.a_full[s], k * kChunk, hk * p.khmul,
                                first_key(t), b * p.kmul);
                ++sa;
                if (!mbar_wait_1t(&c.b_empty[s], rp.phase ^ 1u, abort_flag, err)) break;
                mbar_arrive_expect_tx(&c.b_full[s], (uint32_t)(DVC * kChunkBytes));
                for (int k = 0; k < DVC; ++k)
                    tma_load_4d(Vr + (size_t)(s * DVC + k) * kChunkBytes, &mv, &c.b_full[s], k * kChunk, hk * p.vhmul,
                                first_key(t), b * p.vmul);
                ++sb;
            }
            for (int j = std::max(0, sa - ST); j < sa; ++j) mbar_drain(&c.a_full[j % ST], (uint32_t)(j / ST) & 1u, err);
            for (int j = std::max(0, sb - ST); j < sb; ++j) mbar_drain(&c.b_full[j % ST], (uint32_t)(j / ST) & 1u, err);
        }
    } else if (warp == kMaskWarp) {
        // ------------------------------------------------------------- rows of K that are not read
        RingPos rp;
        for (int t = 0; t < nt && fix; ++t, rp.next(ST)) {
            uint32_t w[4];
            valid_words(w, a, b, first_key(t), n);
            if constexpr (WIN) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] &= seen_word(span, first_key(t) + 32 * e);
            }
            if (!mbar_wait_warp(&c.a_full[rp.idx], rp.phase, abort_flag, err)) break;
            if ((w[0] & w[1] & w[2] & w[3]) != 0xffffffffu) {
                zero_rows(Kr + (size_t)rp.idx * DKC * kChunkBytes, DKC, w);
                fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.a_ready[rp.idx]);
        }
    } else if (warp == kMmaWarp) {
        if (nt > 0) {
            const uint32_t el = elect_one();
            const uint32_t id_s = idesc_bf16_f32(kHalf), id_q = idesc_bf16_bmn(DKC * kChunk);
            const uint32_t ka = smem_u32(Kr), va = smem_u32(Vr);
            // step u: half u % 2 of key tile u / 2; S and dP run two steps ahead of dQ
            RingPos cur, ns, nd;  // stages of dQ's tile, of S's and of dP's
            const int steps = 2 * nt;
            auto scores = [&](int u) {
                const int h = u & 1;
                if (h == 0 && !mbar_wait_warp_inline(fix ? &c.a_ready[ns.idx] : &c.a_full[ns.idx], ns.phase, abort_flag, err)) return false;
                tc_fence_after();
                mma_rows_ts<DKC>(t_s + 64u * h, t_q, ka + (uint32_t)(ns.idx * DKC * kChunkBytes) + h * kHalfBytes, id_s, el);
                commit_to(&c.s_full[h], el);
                if (h == 1) ns.next(ST);
                return true;
            };
            auto dprod = [&](int u) {
                const int h = u & 1;
                if (h == 0 && !mbar_wait_warp_inline(&c.b_full[nd.idx], nd.phase, abort_flag, err)) return false;
                tc_fence_after();
                mma_rows_ts<DVC>(t_dp + 64u * h, t_do, va + (uint32_t)(nd.idx * DVC * kChunkBytes) + h * kHalfBytes, id_s, el);
                commit_to(&c.dp_full[h], el);
                if (h == 1) {
                    commit_to(&c.b_empty[nd.idx], el);
                    nd.next(ST);
                }
                return true;
            };
            bool ok = mbar_wait_warp_inline(&c.own_full, 0, abort_flag, err);
            for (int u = 0; u < 2 && ok; ++u) ok = scores(u) && dprod(u);
            for (int u = 0; u < steps && ok; ++u) {
                const int h = u & 1;
                const uint32_t ph = (uint32_t)(u >> 1) & 1u;
                if (u + 2 < steps && !(ok = mbar_wait_warp_inline(&c.s_free[h], ph, abort_flag, err) && scores(u + 2))) break;
                if (!(ok = mbar_wait_warp_inline(&c.ds_full[h], ph, abort_flag, err))) break;
                tc_fence_after();
                if (!WIN || u >= 2 * ahead)
                    mma_tile_ts<32, 4>(t_dq, t_dp + 64u * h, ka + (uint32_t)(cur.idx * DKC * kChunkBytes) + h * kHalfBytes, id_q,
                                       u != (WIN ? 2 * ahead : 0), el);
                if (h == 1) {
                    commit_to(&c.a_empty[cur.idx], el);
                    cur.next(ST);
                }
                if (u + 2 < steps && !(ok = dprod(u + 2))) break;
            }
            commit_to(&c.done, el);
            mbar_drain(&c.done, 0, err);
        }
    } else {
        // ------------------------------------------------------------- softmax warps: a lane is a row
        const int h = warp >> 3, cw = (warp >> 2) & 1, quad = warp & 3;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t col = lane_base + 64u * h + (uint32_t)(kCols * cw);
        const uint32_t ts = t_s + col, td = t_dp + col;
        const int r = quad * 32 + lane;
        const long long pr = (long long)rt * tile_rows + r;
        const bool mine = r < tile_rows && pr < a.rows;
        const int l = r / a.G;
        const long long ql = mine ? rt * p.nl + l : 0;
        const int hq = hk * a.G + (mine ? r - l * a.G : 0);
        const float cs = a.scale * kLog2e;
        float* stats = a.ws + (((long long)b * a.Hkv + hk) * p.rtiles + rt) * kStats;
        const float nl = stats[r];
        float nd = nt > 0 ? stats[kTile + r] : 0.f;  // (the part that has all keys may write it)
        const bool none = nl == -INFINITY;  // no row, or one without weight
        [[maybe_unused]] KeySpan mine_sees{0, 0, 0};
        if constexpr (WIN) {
            if (mine) mine_sees = key_span<kWindowKeys>(a, b, ql, ql, n);
        }
        // D is summed here: by the sequence, not by its padding (other parts have no tile then)
        const bool exact = WIN ? few && nt > 0 : n <= kTile && nt == 1;
        [[maybe_unused]] float dsum = 0.f;
        const bool one = WIN && mine && mine_sees.count() <= 1;
        [[maybe_unused]] const int last_sum = max(ahead - 1, 0);  // the last tile of D's pass
        if (nt > 0) {
            keep_row(t_q + lane_base, qx, warp >> 2);
            keep_row(t_do + lane_base, ox, warp >> 2);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.own_full);
        }
        bool ok = true;
        for (int t = 0; t < nt; ++t) {
            const uint32_t ph = (uint32_t)t & 1u;
            const int j0 = first_key(t);
            const bool whole = j0 + kTile <= n && !a.mask;
            uint32_t w = 0xffffffffu;
            if (!whole) {
                const int j = j0 + kHalf * h + kCols * cw + lane;
                w = __ballot_sync(0xffffffffu, j < n && (!a.mask || __ldg(a.mask + (long long)b * a.ldm + j) != 0));
            }
            if constexpr (WIN) w &= seen_word(mine_sees, j0 + kHalf * h + kCols * cw);
            if (!mbar_wait_warp_inline(&c.s_full[h], ph, abort_flag, err)) {
                if (exact && (!WIN || t <= last_sum)) bar_sync_and(1, kSoftWarps * 32, false);
                ok = false;
                break;
            }
            tc_fence_after();
            uint32_t sr[kCols], pk[kCols / 2];
            float* s = reinterpret_cast<float*>(sr);
            tmem_ld32_issue(ts, sr);
            tmem_wait_ld32(sr);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.s_free[h]);
#pragma unroll
            for (int q = 0; q < kCols; q += 2) {
                fma2(s[q], s[q + 1], cs, nl);
                s[q] = ex2(s[q]);
                s[q + 1] = ex2(s[q + 1]);
            }
            if (!mbar_wait_warp_inline(&c.dp_full[h], ph, abort_flag, err)) {
                if (exact && (!WIN || t <= last_sum)) bar_sync_and(1, kSoftWarps * 32, false);
                ok = false;
                break;
            }
            tc_fence_after();
            uint32_t dr[kCols];
            float* d = reinterpret_cast<float*>(dr);
            tmem_ld32_issue(td, dr);
            tmem_wait_ld32(dr);
            if (exact && (!WIN || t <= last_sum)) {
                // every key of the sequence is here: D = sum_j P dP in fp32, for this kernel and the next.  From a bf16 O
                // it is off by up to 2^-8 of the sum of |dO O|, which with a few keys exceeds the rounding of dS (2 keys: dK off by
                // 5e-3, so 2e-3).
                float sum = WIN ? dsum : 0.f;
#pragma unroll
                for (int q = 0; q < kCols; ++q) sum += (w >> q) & 1u ? s[q] * d[q] : 0.f;
                if constexpr (WIN) {
                    dsum = sum;
                    if (t < last_sum) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&c.ds_full[h]);
                        continue;
                    }
                }
                c.dpart[2 * h + cw][r] = sum;
                if (!bar_sync_and(1, kSoftWarps * 32, true)) {  // a warp gave up
                    ok = false;
                    break;
                }
                nd = none ? 0.f : -((c.dpart[0][r] + c.dpart[1][r]) + (c.dpart[2][r] + c.dpart[3][r]));
                if (WIN) nd = one ? kOneKey : not_one_key(nd);
                if (warp < 4) stats[kTile + r] = nd;
                if (WIN && ahead > 0) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&c.ds_full[h]);
                    continue;
                }
            }
#pragma unroll
            for (int q = 0; q < kCols; q += 2) {
                add2(d[q], d[q + 1], nd, nd);
                mul2(d[q], d[q + 1], s[q], s[q + 1]);
            }
            if (WIN ? __any_sync(0xffffffffu, w != 0xffffffffu) : w != 0xffffffffu) {
#pragma unroll
                for (int q = 0; q < kCols; ++q) d[q] = (w >> q) & 1u ? d[q] : 0.f;
            }
#pragma unroll
            for (int q = 0; q < kCols / 2; ++q) pk[q] = none || one ? 0u : pack_bf16(d[2 * q], d[2 * q + 1]);
            tmem_st16(td, pk);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.ds_full[h]);
        }
        if (ok && nt > 0) ok = mbar_wait_warp_inline(&c.done, 0, abort_flag, err);
        tc_fence_after();
        if (ok) {  // 32 columns of dQ a warp
            const long long at = ((long long)b * a.Hq + hq) * a.Lq + ql;
            drain_acc(t_dq + lane_base, kCols * (warp >> 2), kCols * (warp >> 2) + kCols, a.dk, nt > 0, !none, mine,
                      a.splits > 1 ? 1.f : a.scale,
                      reinterpret_cast<__nv_bfloat16*>(a.dQ.p) + b * a.dQ.b + ql * a.dQ.l + hq * a.dQ.h, p.vec_q != 0,
                      a.splits > 1 ? a.ws + xattn_ws_dq(a) + ((long long)part * xattn_rows(a) + at) * a.dk : nullptr);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

std::atomic<bool> g_attr[64][8];
std::atomic<bool> g_launched;  // the error word is read (a blocking copy of some 10 us) only once a kernel may have set it

template <int DKC, int DVC, bool WIN>
cudaError_t launch(const HeadMap& q, const HeadMap& o, const HeadMap& k, const HeadMap& v, const Params& p, int device,
                   cudaStream_t s) {
    using C = Cfg<DKC, DVC>;
    const XattnArgs& a = p.a;
    std::atomic<bool>& set = g_attr[device][(DKC - 1) * 4 + (DVC - 1) * 2 + WIN];
    cudaError_t e = cudaSuccess;
    if (!set) {
        e = cudaFuncSetAttribute(k_xattn_dkv_tc<DKC, DVC, WIN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem);
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(k_xattn_dq_tc<DKC, DVC, WIN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem);
        if (e != cudaSuccess) return e;
        set = true;
    }
    // first dQ: for short sequences it leaves a more exact D to the other
    k_xattn_dq_tc<DKC, DVC, WIN><<<(unsigned)(p.rtiles * a.splits * a.Hkv * a.B), kThreads, C::kSmem, s>>>(k.map, v.map, p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    if (a.splits > 1 && (e = launch_xattn_join_dq(a, s)) != cudaSuccess) return e;
    k_xattn_dkv_tc<DKC, DVC, WIN><<<(unsigned)((p.ktiles + (a.pkeys + kTile - 1ll) / kTile * (a.rsplits - 1)) * a.Hkv * a.B), kThreads, C::kSmem, s>>>(
        q.map, o.map, p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    return a.rsplits > 1 ? launch_xattn_join_dkv(a, s) : cudaSuccess;
}

template <bool WIN>
cudaError_t launch_widths(const HeadMap& q, const HeadMap& o, const HeadMap& k, const HeadMap& v, const Params& p, int vec, int device,
                          cudaStream_t s) {
    const XattnArgs& a = p.a;
    k_xattn_stats<WIN><<<(unsigned)(kStatBlocks * p.rtiles * a.Hkv * a.B), 256, 0, s>>>(a, p.nl, p.rtiles, vec);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const bool k2 = a.dk > kChunk, v2 = a.dv > kChunk;
    return k2 ? (v2 ? launch<2, 2, WIN>(q, o, k, v, p, device, s) : launch<2, 1, WIN>(q, o, k, v, p, device, s))
              : (v2 ? launch<1, 2, WIN>(q, o, k, v, p, device, s) : launch<1, 1, WIN>(q, o, k, v, p, device, s));
}

bool on_vectors(const HeadView& v, int B, int L, int H, int w) {
    return w % 8 == 0 && (uintptr_t)v.p % 16 == 0 && (B <= 1 || v.b % 8 == 0) && (L <= 1 || v.l % 8 == 0) &&
           (H <= 1 || v.h % 8 == 0);
}

}  // namespace

unsigned take_device_error_xbwd() {
    unsigned v = 0, z = 0;
    if (!g_launched) return 0;
    cudaMemcpyFromSymbol(&v, g_err_xbwd, sizeof(v));
    if (v) cudaMemcpyToSymbol(g_err_xbwd, &z, sizeof(z));
    return v;
}

void xattn_bwd_tc_plan(XattnArgs& a, KeyMode mode, int sms) {
    const long long nl = kTile / a.G;
    const long long kt = (a.Lk + kTile - 1) / kTile, rt = (a.Lq + nl - 1) / nl;
    long long keys = kt, rows = rt;  // tiles that one of the other kind meets
    if (mode == kWindowKeys) {
        keys = std::min(kt, ((long long)a.win.window + std::min(a.win.sinks, a.Lk) + nl) / kTile + 1);
        if (a.win.sinks == 0) rows = std::min(rt, ((long long)a.win.window + kTile) / nl + 1);
    }
    // the keys (rows) are cut into parts of two tiles or more where one CTA per row (key) tile leaves multiprocessors idle
    a.splits = xattn_parts(rt * a.Hkv * a.B, keys, sms, 2);
    a.rsplits = xattn_parts(kt * a.Hkv * a.B, rows, sms, 2);
    a.pkeys = a.Lk;
    if (mode == kWindowKeys && a.win.sinks > 0 && a.rsplits == 1) {
        a.rsplits = xattn_sink_parts(kt * a.Hkv * a.B, rt, std::min(rt, ((long long)a.win.window + kTile) / nl + 1), 0, sms);
        if (a.rsplits > 1) a.pkeys = (int)std::min<long long>(a.Lk, (a.win.sinks + kTile - 1ll) / kTile * kTile);
    }
    a.stats = rt * a.Hkv * a.B * kStats;
}

cudaError_t launch_xattn_bwd_tc(const XattnArgs& a, KeyMode mode, int device, cudaStream_t s) {
    if (device < 0 || device >= 64) return cudaErrorInvalidDevice;
    g_launched = true;
    Params p{};
    p.a = a;
    p.nl = kTile / a.G;
    p.rtiles = (a.Lq + p.nl - 1) / p.nl;
    p.ktiles = (a.Lk + kTile - 1) / kTile;
    p.vec_q = on_vectors(a.dQ, a.B, a.Lq, a.Hq, a.dk);
    p.vec_k = on_vectors(a.dK, a.B, a.Lk, a.Hkv, a.dk);
    p.vec_v = on_vectors(a.dV, a.B, a.Lk, a.Hkv, a.dv);
    HeadMap q, o, k, v;
    if (!make_head_map(&q, a.q, a.B, a.Lq, a.Hq, a.dk, a.G, p.nl) || !make_head_map(&o, a.dO, a.B, a.Lq, a.Hq, a.dv, a.G, p.nl) ||
        !make_head_map(&k, a.k, a.B, a.Lk, a.Hkv, a.dk, 1, kTile) || !make_head_map(&v, a.v, a.B, a.Lk, a.Hkv, a.dv, 1, kTile))
        return cudaErrorInvalidValue;
    p.qmul = q.bmul;
    p.omul = o.bmul;
    p.kmul = k.bmul;
    p.khmul = k.hmul;
    p.vmul = v.bmul;
    p.vhmul = v.hmul;
    const int vec = on_vectors(a.o, a.B, a.Lq, a.Hq, a.dv) && on_vectors(a.dO, a.B, a.Lq, a.Hq, a.dv);
    return mode == kWindowKeys ? launch_widths<true>(q, o, k, v, p, vec, device, s) : launch_widths<false>(q, o, k, v, p, vec, device, s);
}

}  // namespace gs
