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
// bits: 2.3e-3 of its norm, where fp32 weights and the output's own rounding give 1.7e-3 (through windows of 64 keys to all of 2,048: 2.2e-3 to 1.9e-3, 1.6e-3).
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
    uint64_t full[kMaxStages], vfull[kMaxStages], empty[kMaxStages], ready[kMaxStages];  // keys there, values, free, values mended
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
    int part, hk, b, nq, n, t0, nt;
    int l0;           // first query position
    int sinks, skip;  // through a window: tiles of first keys that stay visible, tiles between them and the window
    KeySpan span;     // what some row of the item sees
};
// the item's j-th tile of keys
template <bool WIN>
__device__ __forceinline__ int tile_of(const Item& m, int j) {
    const int t = m.t0 + j;
    return WIN && t >= m.sinks ? t + m.skip : t;
}
template <bool PAIR, bool WIN>
// (In 32 bits: items are few enough, and the divisions of 64 bits were half of an item of one key tile's 11 us.)
__device__ __forceinline__ Item item_of(const Params& p, unsigned i) {
    const XattnArgs& a = p.a;
    Item m;
    const unsigned units = (unsigned)p.units;
    m.l0 = (int)(i % units) * (PAIR ? 2 : 1) * p.nl;
    i /= units;
    m.part = 0;
    if (a.splits > 1) {
        m.part = (int)(i % (unsigned)a.splits);
        i /= (unsigned)a.splits;
    }
    m.b = (int)(i / (unsigned)a.Hkv);
    m.hk = (int)i - m.b * a.Hkv;
    m.nq = PAIR && m.l0 + p.nl < a.Lq ? 2 : 1;
    m.n = keys_of(a, m.b);
    if constexpr (WIN) {
        m.span = key_span<kWindowKeys>(a, m.b, m.l0, min(a.Lq, m.l0 + m.nq * p.nl) - 1, m.n);
        const int from = m.span.lo / kTile;
        m.sinks = min((m.span.sink + kTile - 1) / kTile, from);
        m.skip = from - m.sinks;
        const int count = m.sinks + max(0, (m.span.hi + kTile - 1) / kTile - from);
        m.t0 = 0;
        m.nt = count;
        if (a.splits > 1) {
            m.t0 = (int)((long long)count * m.part / a.splits);
            m.nt = (int)((long long)count * (m.part + 1) / a.splits) - m.t0;
        }
        return m;
    }
    if (a.splits == 1) {
        m.t0 = 0;
        m.nt = (m.n + kTile - 1) / kTile;
        return m;
    }
    m.t0 = (int)((long long)p.ktiles * m.part / a.splits);
    const int t1 = min((int)((long long)p.ktiles * (m.part + 1) / a.splits), (m.n + kTile - 1) / kTile);
    m.nt = max(0, t1 - m.t0);  // key tiles
    return m;
}

template <int DKC, int DVC, bool PAIR, bool WIN>
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
    // (What lies outside the window is not zeroed: where it is not finite, the rows that met it are taken again, k_window_mend.)
    const bool fix = a.lens != nullptr || a.mask != nullptr;

    if (threadIdx.x == 0) {
        for (int s = 0; s < QS; ++s) {
            mbar_init(&c.q_full[s], 1);
            mbar_init(&c.q_empty[s], 1);
        }
        for (int s = 0; s < ST; ++s) {
            mbar_init(&c.full[s], 1);
            mbar_init(&c.vfull[s], 1);
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
            int qsent = 0;
            uint32_t kph = 0, vph = 0, used = 0, last = 0;  // a bit a stage: phases, whether it was filled, and with values
            bool ok = true;
            for (unsigned it = blockIdx.x; it < (unsigned)p.items && ok; it += gridDim.x) {
                const Item m = item_of<PAIR, WIN>(p, it);
                if (m.nt == 0) continue;
                if (!(ok = mbar_wait_1t(&c.q_empty[rq.idx], rq.phase ^ 1u, abort_flag, err))) break;
                mbar_arrive_expect_tx(&c.q_full[rq.idx], (uint32_t)(m.nq * DKC * kChunk * 2 * tile_rows));
                for (int t = 0; t < m.nq; ++t)
                    for (int k = 0; k < DKC; ++k)
                        tma_load_4d(Qs + (size_t)rq.idx * C::kQBytes + (size_t)(t * DKC + k) * kChunkBytes, &mq, &c.q_full[rq.idx],
                                    k * kChunk, m.hk * a.G, m.l0 + t * p.nl, m.b * p.qmul);
                rq.next(QS);
                ++qsent;
                auto load = [&](bool key, int j) {
                    if (!mbar_wait_1t(&c.empty[rp.idx], rp.phase ^ 1u, abort_flag, err)) return false;
                    const int chunks = key ? DKC : DVC;
                    const uint32_t bit = 1u << rp.idx;
                    uint64_t* there = key ? &c.full[rp.idx] : &c.vfull[rp.idx];
                    mbar_arrive_expect_tx(there, (uint32_t)(chunks * kChunkBytes));
                    for (int k = 0; k < chunks; ++k)
                        tma_load_4d(ring + (size_t)rp.idx * C::kStageBytes + (size_t)k * kChunkBytes, key ? &mk : &mv,
                                    there, k * kChunk, m.hk * (key ? p.khmul : p.vhmul), tile_of<WIN>(m, j) * kTile,
                                    m.b * (key ? p.kmul : p.vmul));
                    (key ? kph : vph) ^= bit;
                    used |= bit;
                    last = key ? last & ~bit : last | bit;
                    rp.next(ST);
                    return true;
                };
                for (int j = 0; j < C::kLead && j < m.nt && ok; ++j) ok = load(true, j);
                for (int j = 0; j < m.nt && ok; ++j) {
                    ok = load(false, j);
                    if (ok && j + C::kLead < m.nt) ok = load(true, j + C::kLead);
                }
            }
            for (int j = std::max(0, qsent - QS); j < qsent; ++j) mbar_drain(&c.q_full[j % QS], (uint32_t)(j / QS) & 1u, err);
            for (int s = 0; s < ST; ++s)
                if (used >> s & 1u) mbar_drain(last >> s & 1u ? &c.vfull[s] : &c.full[s], ((last >> s & 1u ? vph : kph) >> s & 1u) ^ 1u, err);
        }
    } else if (warp == kMaskWarp) {
        // ------------------------------------------------------------- rows of V that are not read
        RingPos rp;
        uint32_t vph = 0;
        bool ok = fix;
        for (unsigned it = blockIdx.x; it < (unsigned)p.items && ok; it += gridDim.x) {
            const Item m = item_of<PAIR, WIN>(p, it);
            auto pass = [&](bool key, int j) {
                if (!key) {
                    uint32_t w[4];
                    valid_words(w, a, m.b, tile_of<WIN>(m, j) * kTile, m.n);
                    if (!mbar_wait_warp(&c.vfull[rp.idx], vph >> rp.idx & 1u, abort_flag, err)) return false;
                    vph ^= 1u << rp.idx;
                    if ((w[0] & w[1] & w[2] & w[3]) != 0xffffffffu) {
                        zero_rows(ring + (size_t)rp.idx * C::kStageBytes, DVC, w);
                        fence_proxy_async();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&c.ready[rp.idx]);
                }
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
            uint32_t kph = 0, vph = 0;      // phases of the stages' keys and values, a bit each
            bool ok = true;
            for (unsigned it = blockIdx.x; it < (unsigned)p.items && ok; it += gridDim.x) {
                Item m = item_of<PAIR, WIN>(p, it);
                m.nt = uniform(m.nt);
                m.nq = uniform(m.nq);
                if (m.nt == 0) continue;
                const uint32_t qa = smem_u32(Qs) + (uint32_t)(rq.idx * C::kQBytes);
                auto arrived = [&](bool key) {  // each kind has barriers of its own, so that the mask warp need not follow the keys
                    uint32_t& ph = key ? kph : vph;
                    const bool in = mbar_wait_warp_inline(key ? &c.full[rp.idx] : fix ? &c.ready[rp.idx] : &c.vfull[rp.idx],
                                                          ph >> rp.idx & 1u, abort_flag, err);
                    ph ^= 1u << rp.idx;
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
                    if (!(ok = arrived(true))) break;
                    for (int t = 0; t < m.nq; ++t) scores(t);
                    commit_to(&c.empty[rp.idx], el);
                    if (m.nt == 1) commit_to(&c.q_empty[rq.idx], el);
                    rp.next(ST);
                    for (int j = 0; j < m.nt && ok; ++j) {
                        if (!(ok = arrived(false))) break;
                        const uint32_t v = stage();
                        const int vs = rp.idx;
                        rp.next(ST);
                        for (int t = 0; t < m.nq && ok; ++t) {
                            ok = values(t, j == 0, v);
                            if (ok && j + 1 < m.nt && (t != 0 || (ok = arrived(true)))) scores(t);
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
                        if (!(ok = arrived(true))) break;
                        scores(j);
                        commit_to(&c.empty[rp.idx], el);
                        if (j + 1 == m.nt) commit_to(&c.q_empty[rq.idx], el);
                        rp.next(ST);
                    }
                    for (int j = 0; j < m.nt && ok; ++j) {
                        if (!(ok = arrived(false)) || !(ok = values(j & 1, j < 2, stage()))) break;
                        commit_to(&c.empty[rp.idx], el);
                        rp.next(ST);
                        if (j + 2 < m.nt) {
                            if (!(ok = arrived(true))) break;
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
        for (unsigned it = blockIdx.x; it < (unsigned)p.items && ok; it += gridDim.x) {
            const Item im = item_of<PAIR, WIN>(p, it);
            if (PAIR && t >= im.nq) continue;
            const int l0 = im.l0 + (PAIR ? t : 0) * p.nl, nrows = min(p.nl, a.Lq - l0) * a.G;
            const bool busy = quad * 32 < nrows;  // a warp without a row only keeps the barriers' count
            [[maybe_unused]] KeySpan sp;
            if constexpr (WIN) {
                sp.sink = sp.lo = 0;
                sp.hi = 0x7fffffff;  // (a lane without a row keeps no tile from the unmasked path)
                const int l = l0 + r / a.G;
                if (r < nrows) sp = key_span<kWindowKeys>(a, im.b, l, l, im.n);
            }
            const int steps = PAIR ? im.nt : (im.nt - t + 1) / 2;  // key tiles of this group
            float m = lowest, l = 0.f;  // m in units of the logits s
            for (int k = 0; k < steps; ++k, ++taken) {
                const int j0 = tile_of<WIN>(im, PAIR ? k : 2 * k + t) * kTile;
                uint32_t w[4];
                bool whole = j0 + kTile <= im.n && !a.mask;
                if constexpr (WIN) {
                    if (busy) {
                        whole = !a.mask && __all_sync(0xffffffffu, sp.lo <= j0 && sp.hi >= j0 + kTile);
                        if (!whole) {
                            if (a.mask) {
                                valid_words(w, a, im.b, j0, im.n);
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) w[i] = 0xffffffffu;  // (a row's span ends with the sequence)
                            }
#pragma unroll
                            for (int i = 0; i < 4; ++i) w[i] &= seen_word(sp, j0 + 32 * i);
                            whole = __all_sync(0xffffffffu, (w[0] & w[1] & w[2] & w[3]) == 0xffffffffu);
                        }
                    }
                } else if (busy && !whole) {
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
                        // through a window each row goes by its own keys: what only its neighbours see does not change its rounding
                        const float to_m = WIN && !((mn - m) * cs > kGrow) ? m : mn;
                        const float f = ex2((m - to_m) * cs);
                        m = to_m;
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
                const int rr = mine ? r : 0, rl = rr / a.G, h = im.hk * a.G + rr - rl * a.G;
                const long long ql = l0 + rl;
                const long long at = ((long long)im.b * a.Hq + h) * a.Lq + ql;
                const long long all = xattn_rows(a);
                const float inv = l == 0.f ? 0.f : 1.f / l;
                __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.o.p) + im.b * a.o.b + ql * a.o.l + h * a.o.h;
                float* po = a.ws + ((long long)im.part * all + at) * a.dv;
                [[maybe_unused]] float wild = 0.f;  // NaN once a sum is not finite
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
                        if constexpr (WIN) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) wild = fmaf(v[e], 0.f, wild);
                        }
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
                    } else {
                        if (a.lse) a.lse[at] = l == 0.f ? -INFINITY : (m2 + log2f(l)) * kLn2;
                        if constexpr (WIN) reinterpret_cast<unsigned char*>(a.ws)[at] = wild != 0.f;  // (for k_window_mend)
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

// Rows whose sum of values is not finite: a tile's rows see different keys, and 0 times what is not finite in a row of V that one of them
// sees is NaN in the others'.  Such a row is taken again, over what it sees: a warp each.  First its item's tiles are searched for a
// value that it does not see and that is not finite (some hundred keys); where there is none, its sum is what it should be.
// (Inputs lie on 16-byte boundaries here, as for the tensor maps.)
__device__ __forceinline__ bool odd8(const uint4& x) {  // an infinity or NaN among eight
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    return odd;
}
// some value of the keys [j0, j1) is not finite (a warp)
__device__ bool odd_values(const __nv_bfloat16* vp, const XattnArgs& a, int j0, int j1) {
    const int lane = threadIdx.x & 31;
    bool odd = false;
    for (long long e = lane; e < (j1 - j0) * 16ll; e += 32) {
        const int c = (int)(e & 15) * 8;
        const __nv_bfloat16* p = vp + (j0 + (e >> 4)) * a.v.l + c;
        if (c + 8 <= a.dv)
            odd |= odd8(__ldg(reinterpret_cast<const uint4*>(p)));
        else
            for (int x = 0; c + x < a.dv; ++x) odd |= !(fabsf(__bfloat162float(p[x])) <= FLT_MAX);
    }
    return __any_sync(0xffffffffu, odd);
}
__device__ void mend_row(const XattnArgs& a, long long at, int lane, int item_rows) {
    const long long l = at % a.Lq, bh = at / a.Lq;
    const int b = (int)(bh / a.Hq), h = (int)(bh % a.Hq), hk = h / a.G, n = keys_of(a, b);
    const KeySpan sp = key_span<kWindowKeys>(a, b, l, l, n);
    const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.b + l * a.q.l + h * a.q.h;
    const __nv_bfloat16* kp = reinterpret_cast<const __nv_bfloat16*>(a.k.p) + b * a.k.b + hk * a.k.h;
    const __nv_bfloat16* vp = reinterpret_cast<const __nv_bfloat16*>(a.v.p) + b * a.v.b + hk * a.v.h;
    {
        const long long l0 = l / item_rows * item_rows, l1 = min(l0 + item_rows, (long long)a.Lq) - 1;
        const KeySpan all = key_span<kWindowKeys>(a, b, l0, l1, n);
        const int from = all.lo / kTile, sinks = min((all.sink + kTile - 1) / kTile, from);
        const int end = (int)min((long long)n, (all.hi + kTile - 1ll) / kTile * kTile);
        if (!odd_values(vp, a, sp.sink, min(sinks * kTile, n)) && !odd_values(vp, a, from * kTile, min(sp.lo, n)) &&
            !odd_values(vp, a, max(sp.hi, from * kTile), end))
            return;
    }
    float m = -INFINITY, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < sp.count(); i0 += 32) {
        const int i = i0 + lane;
        const long long j = i < sp.count() ? sp.key(i) : -1;
        const bool in = j >= 0 && (!a.mask || a.mask[b * a.ldm + j] != 0);
        float s = 0.f;
        for (int c = 0; c < a.dk && in; c += 8) {
            if (c + 8 <= a.dk) {
                const uint4 x = __ldg(reinterpret_cast<const uint4*>(q + c)), y = __ldg(reinterpret_cast<const uint4*>(kp + j * a.k.l + c));
                const uint32_t u[4] = {x.x, x.y, x.z, x.w}, w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s = fmaf(__uint_as_float(u[e] << 16), __uint_as_float(w[e] << 16), s);
                    s = fmaf(__uint_as_float(u[e] & 0xffff0000u), __uint_as_float(w[e] & 0xffff0000u), s);
                }
            } else {
                for (int e = c; e < a.dk; ++e) s = fmaf(__bfloat162float(q[e]), __bfloat162float(kp[j * a.k.l + e]), s);
            }
        }
        s = in ? s * a.scale * kLog2e : -INFINITY;
        float mn = fmaxf(m, s);
#pragma unroll
        for (int x = 16; x; x >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, x));
        const float ms = mn == -INFINITY ? 0.f : mn, f = ex2(m - ms), p = ex2(s - ms);
        m = mn;
        sum *= f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= f;
        for (int x = 0; x < 32; ++x) {
            const float w = __shfl_sync(0xffffffffu, p, x);
            const long long jj = __shfl_sync(0xffffffffu, j, x);
            if (w == 0.f) continue;
            sum += w;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (lane + 32 * e < a.dv) o[e] = fmaf(w, __bfloat162float(vp[jj * a.v.l + lane + 32 * e]), o[e]);
        }
    }
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.o.p) + b * a.o.b + l * a.o.l + h * a.o.h;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (lane + 32 * e < a.dv) out[lane + 32 * e] = __float2bfloat16_rn(sum == 0.f ? 0.f : o[e] / sum);
}
// Flagged rows (a byte each), or, where parts were joined, the rows of O themselves.  One value flags its neighbours' rows together, so a
// block's 256 rows are 32 runs of eight, one of each to a warp, from all over the array (in order, 32 a warp one behind the other, one
// infinite value among 4 x 4,096 positions of 32 / 8 heads took the call from 0.29 to 11.8 ms; so to 0.7).  Without a flag: 2 us there.
__global__ void __launch_bounds__(256) k_window_mend(const XattnArgs a, int item_rows) {
    __shared__ unsigned found[8];
    const long long rows = xattn_rows(a);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto row_of = [&](int run, int k) { return ((long long)run * gridDim.x + blockIdx.x) * 8 + k; };
    const long long at = row_of(threadIdx.x >> 3, threadIdx.x & 7);
    bool wild = false;
    if (at < rows) {
        if (a.splits == 1) {
            wild = reinterpret_cast<const unsigned char*>(a.ws)[at] != 0;
        } else {
            const long long l = at % a.Lq, bh = at / a.Lq;
            const __nv_bfloat16* o = reinterpret_cast<const __nv_bfloat16*>(a.o.p) + (bh / a.Hq) * a.o.b + l * a.o.l + (bh % a.Hq) * a.o.h;
            for (int c = 0; c < a.dv; ++c) wild |= !(fabsf(__bfloat162float(o[c])) <= FLT_MAX);
        }
    }
    const unsigned bits = __ballot_sync(0xffffffffu, wild);
    if (lane == 0) found[warp] = bits;
    if (!__syncthreads_or(wild)) return;
    unsigned todo = __ballot_sync(0xffffffffu, found[lane >> 2] >> (8 * (lane & 3) + warp) & 1u);
    for (; todo; todo &= todo - 1) mend_row(a, row_of(__ffs(todo) - 1, warp), lane, item_rows);
}

std::atomic<bool> g_attr[64][16];
std::atomic<bool> g_launched;  // the error word is read (a blocking copy of some 10 us) only once a kernel may have set it

template <int DKC, int DVC, bool PAIR, bool WIN>
cudaError_t launch(const HeadMap& q, const HeadMap& k, const HeadMap& v, const Params& p, int sms, int device, cudaStream_t s) {
    using C = Cfg<DKC, DVC, PAIR>;
    std::atomic<bool>& set = g_attr[device][(DKC - 1) * 8 + (DVC - 1) * 4 + PAIR * 2 + WIN];
    if (!set) {
        cudaError_t e = cudaFuncSetAttribute(k_xattn_tc<DKC, DVC, PAIR, WIN>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)C::kSmem);
        if (e != cudaSuccess) return e;
        set = true;
    }
    const long long grid = std::min<long long>(p.items, sms);
    k_xattn_tc<DKC, DVC, PAIR, WIN><<<(unsigned)grid, kThreads, C::kSmem, s>>>(q.map, k.map, v.map, p);
    return cudaGetLastError();
}
template <bool WIN>
cudaError_t launch_widths(bool pair, const HeadMap& q, const HeadMap& k, const HeadMap& v, const Params& p, int sms, int device,
                          cudaStream_t s) {
    const bool k2 = p.a.dk > kChunk, v2 = p.a.dv > kChunk;
    if (pair)
        return k2 ? (v2 ? launch<2, 2, true, WIN>(q, k, v, p, sms, device, s) : launch<2, 1, true, WIN>(q, k, v, p, sms, device, s))
                  : (v2 ? launch<1, 2, true, WIN>(q, k, v, p, sms, device, s) : launch<1, 1, true, WIN>(q, k, v, p, sms, device, s));
    return k2 ? (v2 ? launch<2, 2, false, WIN>(q, k, v, p, sms, device, s) : launch<2, 1, false, WIN>(q, k, v, p, sms, device, s))
              : (v2 ? launch<1, 2, false, WIN>(q, k, v, p, sms, device, s) : launch<1, 1, false, WIN>(q, k, v, p, sms, device, s));
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

void xattn_tc_plan(XattnArgs& a, KeyMode mode, int sms) {
    const long long tile_rows = (long long)(kTile / a.G) * a.G;
    long long kt = (a.Lk + kTile - 1) / kTile;
    if (mode == kWindowKeys)  // that a row tile meets
        kt = std::min(kt, ((long long)a.win.window + std::min(a.win.sinks, a.Lk) + kTile / a.G) / kTile + 1);
    a.flags = mode == kWindowKeys;
    a.splits = take_pairs(a, sms) ? 1 : xattn_parts((a.rows + tile_rows - 1) / tile_rows * a.Hkv * a.B, kt, sms, 4);
    a.rsplits = 1;
}

cudaError_t launch_xattn_tc(const XattnArgs& a, KeyMode mode, int sms, int device, cudaStream_t s) {
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
    cudaError_t e = mode == kWindowKeys ? launch_widths<true>(pair, q, k, v, p, sms, device, s)
                                        : launch_widths<false>(pair, q, k, v, p, sms, device, s);
    if (e == cudaSuccess && a.splits > 1) e = launch_xattn_join(a, s);
    if (e != cudaSuccess || mode != kWindowKeys) return e;
    k_window_mend<<<(unsigned)((xattn_rows(a) + 255) / 256), 256, 0, s>>>(a, p.nl * (pair ? 2 : 1));
    return cudaGetLastError();
}

}  // namespace gs
