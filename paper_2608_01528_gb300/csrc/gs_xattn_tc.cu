// gs_xattn_tc.cu -- cross attention on tcgen05 (bf16 inputs).
//
// A CTA holds up to 128 packed query rows per tile (all query heads of a key head, so a key tile is read once
// for the group) and walks the keys in tiles of 128.  Per tile: S = Q K^T (tcgen05, fp32 in TMEM), one thread per row takes
// the row's maximum and 2^(c s - m) (c = scale log2 e), writes the weights back over S as bf16 -- the A operand of
// O += P V, which also accumulates in TMEM; V is read as it lies (MN-major).  The running maximum moves only
// when a row's maximum grew by more than 2^8: then O is rescaled in TMEM; otherwise weights are up to 256, which
// bf16 and the fp32 sums hold as well.
//
// Two softmax groups of four warps keep the tensor core busy in turn.  With many rows (PAIR) they hold two row tiles
// that share each key tile.  With few rows they take every other key tile of one row tile, the keys may further be cut
// into parts over CTAs, and group 0 joins the two groups' (O, m, l) at the end; parts meet in k_xattn_join.
//
// Masks: a key that is not read has its weight set to 0, and its row of V is zeroed in shared memory by a warp of
// its own before the MMA reads it, as 0 * NaN would be NaN.
//
// Work items (row unit, part, key head, sequence) are walked by one persistent CTA per multiprocessor: the next item's loads and
// first scores run while the softmax groups finish the last one (64 sequences of 1,500 keys, one row each: 113 us with a
// CTA per item).
//
// Weights go to bf16 for the product with V (half a step, 2^-8 relative): both operands of the tensor core have one type, and V
// is bf16; two bf16 terms a weight would double that product.  Their sum l takes them unrounded in fp32.  Error of O against 64
// bits: 2.3e-3 of its norm, where fp32 weights and the output's own rounding give 1.7e-3.
//
// Measured: 4 x 4,096 x 4,096, 32 / 8 heads of 128: 0.69 ms of kernel, 1.59 PFLOP/s (0.74 to 0.75 ms in a stream of calls on
// changing inputs), tensor pipe 70 %: the products and the softmax chain of a group between them; 8 x 1,024 x 750..1,500, 16
// heads of 64: 70 us, of which a third is the uneven share of 512 items over 152 CTAs and the rest the softmax warps (a step of
// 128 keys takes a group 2,500 clocks, XU 39 % and tensor pipe 39 % busy); single rows over 8 x 65,537 keys, 32 / 8 heads of
// 128: 0.30 ms, 7.1 TB/s.  A softmax thread holds 128 scores: all 168 registers that 11 warps leave it, and 128 to 172 bytes
// are spilled.
//
// Warp roles (352 threads): 0-3 and 4-7 softmax groups (warp w reads TMEM lanes 32 (w % 4)..+31), 8 TMEM allocator and
// MMA issuer, 9 TMA, 10 masks.  Every wait is bounded.

#include <float.h>

#include <algorithm>
#include <atomic>

#include "gs_xattn_tc.cuh"

namespace gs {
namespace {

using namespace xtc;

__device__ unsigned g_err_xattn = 0;

constexpr int kMmaWarp = 8, kTmaWarp = 9, kMaskWarp = 10;
constexpr int kThreads = 11 * 32;
constexpr int kMaxStages = 12;
constexpr float kGrow = 8.f;  // the maximum moves when it grew by more than 2^kGrow

struct Ctl {
    uint64_t q_full[2], q_empty[2];
    uint64_t full[kMaxStages], empty[kMaxStages], ready[kMaxStages];
    uint64_t s_full[2], p_full[2], o_done[2];
    uint64_t posted, joined;  // group 1's statistics are in ml; group 0 has read its O
    uint64_t mma_done;
    float2 ml[kTile];
    uint32_t tmem_base;
    int abort_flag;
};

struct Params {
    XattnArgs a;
    int qmul, kmul, khmul, vmul, vhmul;  // HeadMap multipliers of q (batch), k and v (batch, head)
    int nl;                              // query positions of a row tile: 128 / G
    long long units;                     // row units (pairs or single tiles) per (b, key head)
    long long items;
    int ktiles;
    int o_vec;
};

template <int DKC, int DVC, bool PAIR>
struct Cfg {
    static constexpr int kQTiles = PAIR ? 2 : 1;
    static constexpr int kQSlots = PAIR && DKC == 2 ? 1 : 2;  // (a second pair of 128-wide tiles does not fit)
    static constexpr int kStageBytes = (DKC > DVC ? DKC : DVC) * kChunkBytes;
    static constexpr int kQBytes = kQTiles * DKC * kChunkBytes;
    static constexpr int kRoom = (227 * 1024 - 1024 - (int)sizeof(Ctl) - kQSlots * kQBytes) / kStageBytes;
    static constexpr int kStages = kRoom < kMaxStages ? kRoom : kMaxStages;
    static constexpr size_t kSmem = 1024 + (size_t)kQSlots * kQBytes + (size_t)kStages * kStageBytes + sizeof(Ctl);
    static constexpr int kLead = PAIR ? 1 : 2;  // key tiles requested before the first values
    static_assert(kStages >= 4, "ring too short");
};

// A work item.
struct Item {
    long long row0;  // first packed row
    int part, hk, b, nq, n, t0, nt;
    long long unit;
};
template <bool PAIR>
__device__ __forceinline__ Item item_of(const Params& p, long long i) {
    const XattnArgs& a = p.a;
    Item m;
    m.unit = i % p.units;
    i /= p.units;
    m.part = (int)(i % a.splits);
    i /= a.splits;
    m.hk = (int)(i % a.Hkv);
    m.b = (int)(i / a.Hkv);
    const int tile_rows = p.nl * a.G;
    m.row0 = m.unit * (PAIR ? 2 : 1) * tile_rows;
    m.nq = PAIR && m.row0 + tile_rows < a.rows ? 2 : 1;
    m.n = keys_of(a, m.b);
    m.t0 = (int)((long long)p.ktiles * m.part / a.splits);
    const int t1 = min((int)((long long)p.ktiles * (m.part + 1) / a.splits), (m.n + kTile - 1) / kTile);
    m.nt = max(0, t1 - m.t0);  // key tiles
    return m;
}

template <int DKC, int DVC, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1)
    k_xattn_tc(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
               const __grid_constant__ CUtensorMap mv, const __grid_constant__ Params p) {
    using C = Cfg<DKC, DVC, PAIR>;
    constexpr int DV = DVC * kChunk;
    constexpr int ST = C::kStages, QS = C::kQSlots;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    uint8_t* base = smem_raw + (((raw + 1023u) & ~1023u) - raw);
    uint8_t* Qs = base;
    uint8_t* ring = Qs + QS * C::kQBytes;
    Ctl& c = *reinterpret_cast<Ctl*>(ring + (size_t)ST * C::kStageBytes);
    volatile int* abort_flag = &c.abort_flag;
    unsigned* err = &g_err_xattn;
    const XattnArgs& a = p.a;
    const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    const int tile_rows = p.nl * a.G;
    const bool fix = a.lens != nullptr || a.mask != nullptr;

    if (threadIdx.x == 0) {
        for (int s = 0; s < QS; ++s) {
            mbar_init(&c.q_full[s], 1);
            mbar_init(&c.q_empty[s], 1);
        }
        for (int s = 0; s < ST; ++s) {
            mbar_init(&c.full[s], 1);
            mbar_init(&c.empty[s], 1);
            mbar_init(&c.ready[s], 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&c.s_full[t], 1);
            mbar_init(&c.p_full[t], 4);
            mbar_init(&c.o_done[t], 1);
        }
        mbar_init(&c.posted, 4);
        mbar_init(&c.joined, 4);
        mbar_init(&c.mma_done, 1);
        c.abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&c.tmem_base, 512);
        tmem_relinquish();
    }
    if (warp == kTmaWarp && lane == 0) {
        prefetch_map(&mq);
        prefetch_map(&mk);
        prefetch_map(&mv);
    }
    // Rows of a tile that its box does not write (128 % G != 0) have no result, but a warp moves the maxima of its 32 rows together:
    // with what an earlier kernel left there, the other rows' roundings would change from call to call.
    if (tile_rows < kTile) {
        const int words = (kTile - tile_rows) * 8;  // 16-byte words per chunk
        for (int e = threadIdx.x; e < QS * C::kQTiles * DKC * words; e += kThreads)
            *reinterpret_cast<uint4*>(Qs + (size_t)(e / words) * kChunkBytes + tile_rows * 128 + (e % words) * 16) =
                make_uint4(0, 0, 0, 0);
        fence_proxy_async();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(c.tmem_base);

    if (warp == kTmaWarp) {
        // ------------------------------------------------------------- Q, then K and V tiles
        if (lane == 0) {
            RingPos rp, rq;
            int sent = 0, qsent = 0;
            bool ok = true;
            for (long long it = blockIdx.x; it < p.items && ok; it += gridDim.x) {
                const Item m = item_of<PAIR>(p, it);
                if (m.nt == 0) continue;
                if (!(ok = mbar_wait_1t(&c.q_empty[rq.idx], rq.phase ^ 1u, abort_flag, err))) break;
                mbar_arrive_expect_tx(&c.q_full[rq.idx], (uint32_t)(m.nq * DKC * kChunk * 2 * tile_rows));
                for (int t = 0; t < m.nq; ++t)
                    for (int k = 0; k < DKC; ++k)
                        tma_load_4d(Qs + (size_t)rq.idx * C::kQBytes + (size_t)(t * DKC + k) * kChunkBytes, &mq, &c.q_full[rq.idx],
                                    k * kChunk, m.hk * a.G, (int)(m.unit * C::kQTiles + t) * p.nl, m.b * p.qmul);
                rq.next(QS);
                ++qsent;
                auto load = [&](bool key, int j) {
                    if (!mbar_wait_1t(&c.empty[rp.idx], rp.phase ^ 1u, abort_flag, err)) return false;
                    const int chunks = key ? DKC : DVC;
                    mbar_arrive_expect_tx(&c.full[rp.idx], (uint32_t)(chunks * kChunkBytes));
                    for (int k = 0; k < chunks; ++k)
                        tma_load_4d(ring + (size_t)rp.idx * C::kStageBytes + (size_t)k * kChunkBytes, key ? &mk : &mv,
                                    &c.full[rp.idx], k * kChunk, m.hk * (key ? p.khmul : p.vhmul), (m.t0 + j) * kTile,
                                    m.b * (key ? p.kmul : p.vmul));
                    rp.next(ST);
                    ++sent;
                    return true;
                };
                for (int j = 0; j < C::kLead && j < m.nt && ok; ++j) ok = load(true, j);
                for (int j = 0; j < m.nt && ok; ++j) {
                    ok = load(false, j);
                    if (ok && j + C::kLead < m.nt) ok = load(true, j + C::kLead);
                }
            }
            for (int j = std::max(0, qsent - QS); j < qsent; ++j) mbar_drain(&c.q_full[j % QS], (uint32_t)(j / QS) & 1u, err);
            for (int j = std::max(0, sent - ST); j < sent; ++j) mbar_drain(&c.full[j % ST], (uint32_t)(j / ST) & 1u, err);
        }
    } else if (warp == kMaskWarp) {
        // ------------------------------------------------------------- rows of V that are not read
        RingPos rp;
        bool ok = fix;
        for (long long it = blockIdx.x; it < p.items && ok; it += gridDim.x) {
            const Item m = item_of<PAIR>(p, it);
            auto pass = [&](bool key, int j) {
                uint32_t w[4];
                if (!key) valid_words(w, a, m.b, (m.t0 + j) * kTile, m.n);
                if (!mbar_wait_warp(&c.full[rp.idx], rp.phase, abort_flag, err)) return false;
                if (!key && (w[0] & w[1] & w[2] & w[3]) != 0xffffffffu) {
                    zero_rows(ring + (size_t)rp.idx * C::kStageBytes, DVC, w);
                    fence_proxy_async();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&c.ready[rp.idx]);
                rp.next(ST);
                return true;
            };
            for (int j = 0; j < C::kLead && j < m.nt && ok; ++j) ok = pass(true, j);
            for (int j = 0; j < m.nt && ok; ++j) {
                ok = pass(false, j);
                if (ok && j + C::kLead < m.nt) ok = pass(true, j + C::kLead);
            }
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------- MMA issue
        {
            const uint32_t el = elect_one();
            const uint32_t id_s = idesc_bf16_f32(kTile), id_o = idesc_bf16_bmn(DV);
            const uint32_t ringa = smem_u32(ring);
            RingPos rp, rq;
            uint32_t done0 = 0, done1 = 0;  // weights consumed of each group
            bool ok = true;
            for (long long it = blockIdx.x; it < p.items && ok; it += gridDim.x) {
                Item m = item_of<PAIR>(p, it);
                m.nt = uniform(m.nt);
                m.nq = uniform(m.nq);
                if (m.nt == 0) continue;
                const uint32_t qa = smem_u32(Qs) + (uint32_t)(rq.idx * C::kQBytes);
                auto arrived = [&]() {
                    const bool in = mbar_wait_warp_inline(fix ? &c.ready[rp.idx] : &c.full[rp.idx], rp.phase, abort_flag, err);
                    tc_fence_after();
                    return in;
                };
                auto stage = [&]() { return ringa + (uint32_t)(rp.idx * C::kStageBytes); };
                auto scores = [&](int t) {
                    mma_tile_ss<DKC>(tmem + (t ? 128u : 0u), qa + (uint32_t)((PAIR ? t : 0) * DKC * kChunkBytes), stage(), id_s, el);
                    commit_to(&c.s_full[t], el);
                };
                auto values = [&](int t, bool first, uint32_t v) {  // the weights of group t's next key tile
                    if (!mbar_wait_warp_inline(&c.p_full[t], (t ? done1 : done0) & 1u, abort_flag, err)) return false;
                    (t ? done1 : done0) += 1;
                    tc_fence_after();
                    mma_tile_ts<16>(tmem + 256u + (t ? (uint32_t)DV : 0u), tmem + (t ? 128u : 0u), v, id_o, !first, el);
                    commit_to(&c.o_done[t], el);
                    return true;
                };
                if (!(ok = mbar_wait_warp_inline(&c.q_full[rq.idx], rq.phase, abort_flag, err))) break;
                if (PAIR) {
                    if (!(ok = arrived())) break;
                    for (int t = 0; t < m.nq; ++t) scores(t);
                    commit_to(&c.empty[rp.idx], el);
                    if (m.nt == 1) commit_to(&c.q_empty[rq.idx], el);
                    rp.next(ST);
                    for (int j = 0; j < m.nt && ok; ++j) {
                        if (!(ok = arrived())) break;
                        const uint32_t v = stage();
                        const int vs = rp.idx;
                        rp.next(ST);
                        for (int t = 0; t < m.nq && ok; ++t) {
                            ok = values(t, j == 0, v);
                            if (ok && j + 1 < m.nt && (t != 0 || (ok = arrived()))) scores(t);
                        }
                        if (!ok) break;
                        commit_to(&c.empty[vs], el);
                        if (j + 1 < m.nt) {
                            commit_to(&c.empty[rp.idx], el);
                            if (j + 2 == m.nt) commit_to(&c.q_empty[rq.idx], el);
                            rp.next(ST);
                        }
                    }
                } else {
                    for (int j = 0; j < 2 && j < m.nt && ok; ++j) {
                        if (!(ok = arrived())) break;
                        scores(j);
                        commit_to(&c.empty[rp.idx], el);
                        if (j + 1 == m.nt) commit_to(&c.q_empty[rq.idx], el);
                        rp.next(ST);
                    }
                    for (int j = 0; j < m.nt && ok; ++j) {
                        if (!(ok = arrived()) || !(ok = values(j & 1, j < 2, stage()))) break;
                        commit_to(&c.empty[rp.idx], el);
                        rp.next(ST);
                        if (j + 2 < m.nt) {
                            if (!(ok = arrived())) break;
                            scores(j & 1);
                            commit_to(&c.empty[rp.idx], el);
                            if (j + 3 == m.nt) commit_to(&c.q_empty[rq.idx], el);
                            rp.next(ST);
                        }
                    }
                }
                rq.next(QS);
            }
            commit_to(&c.mma_done, el);
            mbar_drain(&c.mma_done, 0, err);
        }
    } else {
        // ------------------------------------------------------------- softmax groups
        const int t = warp >> 2, quad = warp & 3;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t ts = tmem + lane_base + (t ? 128u : 0u), to0 = tmem + lane_base + 256u, to = to0 + (t ? (uint32_t)DV : 0u);
        const int r = quad * 32 + lane;  // row of the tile
        const float cs = a.scale * kLog2e;
        // The lowest maximum, instead of -inf: its product with cs is finite, so that what lies below (a dot product of -inf, a key
        // that is not read, a dot product that only the scale takes to -inf) weighs 0 without a test a tile.
        const float lowest = fmaxf(-3.3e38f / cs, -FLT_MAX);
        uint32_t taken = 0, joins = 0;  // key tiles and joined items of this group so far
        bool ok = true;
        for (long long it = blockIdx.x; it < p.items && ok; it += gridDim.x) {
            const Item im = item_of<PAIR>(p, it);
            if (PAIR && t >= im.nq) continue;
            const long long left = a.rows - (im.row0 + (long long)(PAIR ? t : 0) * tile_rows);
            const int nrows = (int)(left < tile_rows ? left : tile_rows);
            const bool busy = quad * 32 < nrows;  // a warp without a row only keeps the barriers' count
            const int steps = PAIR ? im.nt : (im.nt - t + 1) / 2;  // key tiles of this group
            float m = lowest, l = 0.f;  // m in units of the logits s
            for (int k = 0; k < steps; ++k, ++taken) {
                const int j0 = (im.t0 + (PAIR ? k : 2 * k + t)) * kTile;
                uint32_t w[4];
                bool whole = j0 + kTile <= im.n && !a.mask;
                if (busy && !whole) {
                    valid_words(w, a, im.b, j0, im.n);
                    whole = (w[0] & w[1] & w[2] & w[3]) == 0xffffffffu;
                }
                if (!mbar_wait_warp_inline(&c.s_full[t], taken & 1u, abort_flag, err)) {
                    ok = false;
                    break;
                }
                if (busy) {
                    tc_fence_after();
                    uint32_t sr[kTile];
#pragma unroll
                    for (int q = 0; q < 4; ++q) tmem_ld32_issue(ts + 32u * q, sr + 32 * q);
#pragma unroll
                    for (int q = 0; q < 4; ++q) tmem_wait_ld32(sr + 32 * q);
                    float* s = reinterpret_cast<float*>(sr);
                    if (!whole) {
#pragma unroll
                        for (int q = 0; q < kTile; ++q)
                            if (!((w[q >> 5] >> (q & 31)) & 1u)) s[q] = -INFINITY;
                    }
                    float mx[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) mx[q] = m;
#pragma unroll
                    for (int q = 0; q < kTile; q += 8)
#pragma unroll
                        for (int e = 0; e < 4; ++e) mx[e] = max3(mx[e], s[q + 2 * e], s[q + 2 * e + 1]);
                    const float mn = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    if (k == 0) {
                        m = mn;
                    } else if (__any_sync(0xffffffffu, (mn - m) * cs > kGrow)) {
                        const float f = ex2((m - mn) * cs);
                        m = mn;
                        l *= f;
                        if (!mbar_wait_warp_inline(&c.o_done[t], (taken - 1) & 1u, abort_flag, err)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
#pragma unroll
                        for (int q = 0; q < DV / 16; ++q) {
                            uint32_t orr[16];
                            tmem_ld16(to + 16u * q, reinterpret_cast<float*>(orr));
#pragma unroll
                            for (int e = 0; e < 16; ++e) orr[e] = __float_as_uint(__uint_as_float(orr[e]) * f);
                            tmem_st16(to + 16u * q, orr);
                        }
                    }
                    const float ms = -m * cs;
                    float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t pk[32];
#pragma unroll
                        for (int q = 0; q < 64; q += 4) {
                            float* x = s + 64 * h + q;
                            fma2(x[0], x[1], cs, ms);
                            fma2(x[2], x[3], cs, ms);
                            x[0] = ex2(x[0]);
                            x[1] = ex2(x[1]);
                            x[2] = ex2(x[2]);
                            x[3] = ex2(x[3]);
                            add2(l0, l1, x[0], x[1]);
                            add2(l2, l3, x[2], x[3]);
                            pk[q / 2] = pack_bf16(x[0], x[1]);
                            pk[q / 2 + 1] = pack_bf16(x[2], x[3]);
                        }
                        tmem_st32(ts + 32u * h, pk);
                    }
                    l += (l0 + l1) + (l2 + l3);
                    tmem_wait_st();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&c.p_full[t]);
            }
            if (!ok) break;
            if (steps > 0 && !(ok = mbar_wait_warp_inline(&c.o_done[t], (taken - 1) & 1u, abort_flag, err))) break;
            tc_fence_after();
            float m2 = m * cs;          // base-2 units from here on
            if (m2 == INFINITY) l = NAN;  // a logit past fp32, where the dot product may have been finite
            float fo = 1.f, f1 = 0.f;  // what group 0's and group 1's O are multiplied by
            const bool two = !PAIR && im.nt > 1;
            if (two) {
                const uint32_t ph = joins++ & 1u;
                if (t == 1) {
                    c.ml[r] = make_float2(m2, l);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&c.posted);
                    if (!(ok = mbar_wait_warp_inline(&c.joined, ph, abort_flag, err))) break;  // O is free again
                } else {
                    if (!(ok = mbar_wait_warp_inline(&c.posted, ph, abort_flag, err))) break;
                    tc_fence_after();
                    const float2 o = c.ml[r];
                    const float mm = fmaxf(m2, o.x);
                    f1 = ex2(o.x - mm);
                    fo = ex2(m2 - mm);
                    l = l * fo + o.y * f1;
                    m2 = mm;
                }
            }
            if (busy && (PAIR || t == 0)) {  // a whole warp, or none
                const bool mine = r < nrows;
                const long long pr = im.row0 + (long long)(PAIR ? t : 0) * tile_rows + (mine ? r : 0);
                const long long ql = pr / a.G;
                const int h = im.hk * a.G + (int)(pr - ql * a.G);
                const long long at = ((long long)im.b * a.Hq + h) * a.Lq + ql;
                const long long all = xattn_rows(a);
                const float inv = l == 0.f ? 0.f : 1.f / l;
                __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.o.p) + im.b * a.o.b + ql * a.o.l + h * a.o.h;
                float* po = a.ws + ((long long)im.part * all + at) * a.dv;
#pragma unroll
                for (int q = 0; q < DV / 32; ++q) {
                    if (32 * q >= a.dv) break;
                    __syncwarp();
                    float v[32];
                    if (im.nt > 0) {
                        tmem_ld32(to0 + (PAIR && t ? (uint32_t)DV : 0u) + 32u * q, v);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0.f;
                    }
                    if (two) {
                        float u[32];
                        tmem_ld32(to0 + (uint32_t)DV + 32u * q, u);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = v[e] * fo + u[e] * f1;
                    }
                    const int w = a.dv - 32 * q;  // columns left
                    if (a.splits == 1) {
                        uint32_t u[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) u[e] = pack_bf16(v[2 * e] * inv, v[2 * e + 1] * inv);
                        if (p.o_vec)
                            store_rows(out + 32 * q, u, w, mine);
                        else
                            store_rows_any(out + 32 * q, u, w, mine);
                        continue;
                    }
                    if (!mine) continue;
                    if (a.dv % 4 == 0) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            if (e < w)
                                *reinterpret_cast<float4*>(po + 32 * q + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (e < w) po[32 * q + e] = v[e];
                    }
                }
                if (mine) {
                    if (a.splits > 1) {
                        float2* ml = reinterpret_cast<float2*>(a.ws + xattn_ws_ml(a)) + (long long)im.part * all + at;
                        *ml = make_float2(m2, l);
                    } else if (a.lse) {
                        a.lse[at] = l == 0.f ? -INFINITY : (m2 + log2f(l)) * kLn2;
                    }
                }
            }
            if (two && t == 0) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&c.joined);
            }
            tc_fence_before();  // this item's reads of O come before the next one's weights
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

template <int DKC, int DVC, bool PAIR>
cudaError_t launch(const HeadMap& q, const HeadMap& k, const HeadMap& v, const Params& p, int sms, int device, cudaStream_t s) {
    using C = Cfg<DKC, DVC, PAIR>;
    std::atomic<bool>& set = g_attr[device][(DKC - 1) * 4 + (DVC - 1) * 2 + PAIR];
    if (!set) {
        cudaError_t e = cudaFuncSetAttribute(k_xattn_tc<DKC, DVC, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)C::kSmem);
        if (e != cudaSuccess) return e;
        set = true;
    }
    const long long grid = std::min<long long>(p.items, sms);
    k_xattn_tc<DKC, DVC, PAIR><<<(unsigned)grid, kThreads, C::kSmem, s>>>(q.map, k.map, v.map, p);
    return cudaGetLastError();
}

// Row tiles come in pairs when pairs alone fill the multiprocessors; else one row tile a CTA, the keys
// split over its two softmax groups and, where CTAs are still few, over CTAs in parts of four key tiles or more.
bool take_pairs(const XattnArgs& a, int sms) {
    const long long tile_rows = (long long)(kTile / a.G) * a.G;
    const long long pairs = (a.rows + 2 * tile_rows - 1) / (2 * tile_rows);
    return a.rows > tile_rows && pairs * a.Hkv * a.B >= sms;
}

}  // namespace

unsigned take_device_error_xattn() {
    unsigned v = 0, z = 0;
    if (!g_launched) return 0;
    cudaMemcpyFromSymbol(&v, g_err_xattn, sizeof(v));
    if (v) cudaMemcpyToSymbol(g_err_xattn, &z, sizeof(z));
    return v;
}

void xattn_tc_plan(XattnArgs& a, int sms) {
    const long long tile_rows = (long long)(kTile / a.G) * a.G;
    const long long kt = (a.Lk + kTile - 1) / kTile;
    a.splits = take_pairs(a, sms) ? 1 : xattn_parts((a.rows + tile_rows - 1) / tile_rows * a.Hkv * a.B, kt, sms, 4);
    a.rsplits = 1;
}

cudaError_t launch_xattn_tc(const XattnArgs& a, int sms, int device, cudaStream_t s) {
    if (device < 0 || device >= 64) return cudaErrorInvalidDevice;
    g_launched = true;
    const bool pair = take_pairs(a, sms);
    Params p{};
    p.a = a;
    p.nl = kTile / a.G;
    const long long tile_rows = (long long)p.nl * a.G;
    p.units = (a.rows + tile_rows * (pair ? 2 : 1) - 1) / (tile_rows * (pair ? 2 : 1));
    p.items = p.units * a.splits * a.Hkv * a.B;
    p.ktiles = (a.Lk + kTile - 1) / kTile;
    p.o_vec = a.dv % 8 == 0 && (uintptr_t)a.o.p % 16 == 0 && (a.B <= 1 || a.o.b % 8 == 0) && (a.Lq <= 1 || a.o.l % 8 == 0) &&
              (a.Hq <= 1 || a.o.h % 8 == 0);
    HeadMap q, k, v;
    const int Lk = std::max(a.Lk, 1);
    if (!make_head_map(&q, a.q, a.B, a.Lq, a.Hq, a.dk, a.G, p.nl) || !make_head_map(&k, a.k, a.B, Lk, a.Hkv, a.dk, 1, kTile) ||
        !make_head_map(&v, a.v, a.B, Lk, a.Hkv, a.dv, 1, kTile))
        return cudaErrorInvalidValue;
    p.qmul = q.bmul;
    p.kmul = k.bmul;
    p.khmul = k.hmul;
    p.vmul = v.bmul;
    p.vhmul = v.hmul;
    const bool k2 = a.dk > kChunk, v2 = a.dv > kChunk;
    cudaError_t e;
    if (pair)
        e = k2 ? (v2 ? launch<2, 2, true>(q, k, v, p, sms, device, s) : launch<2, 1, true>(q, k, v, p, sms, device, s))
               : (v2 ? launch<1, 2, true>(q, k, v, p, sms, device, s) : launch<1, 1, true>(q, k, v, p, sms, device, s));
    else
        e = k2 ? (v2 ? launch<2, 2, false>(q, k, v, p, sms, device, s) : launch<2, 1, false>(q, k, v, p, sms, device, s))
               : (v2 ? launch<1, 2, false>(q, k, v, p, sms, device, s) : launch<1, 1, false>(q, k, v, p, sms, device, s));
    if (e != cudaSuccess || a.splits == 1) return e;
    return launch_xattn_join(a, s);
}

}  // namespace gs
