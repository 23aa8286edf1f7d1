// gs_xattn_tc.cuh -- what the tensor-core cross-attention kernels share: 4-D TMA tiles of
// (B, L, H, width) arrays, MN-major operands, packed arithmetic, valid-key words.
#pragma once

#include "gs_tc_ptx.cuh"
#include "gs_xattn.h"

namespace gs {
namespace xtc {

using namespace ptx;

constexpr int kTile = 128;                  // packed rows / keys of a tile: the MMA's M, and TMEM's lanes
constexpr int kChunk = 64;                  // width of a 128-byte-swizzled chunk (bf16)
constexpr int kChunkBytes = kTile * kChunk * 2;  // 16 KB
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

static __device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z,
                                                   int w) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(
            smem_u32(dst)),
        "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}
static __device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Descriptor of an MN-major B operand: rows of the tile are the K dimension (128 bytes apart), its 64-column
// chunks the N dimension.  128-byte swizzle; 8-row groups 1,024 bytes apart (stride offset), chunks 16 KB
// apart (leading offset).
static __device__ __forceinline__ uint64_t sdesc_mn(uint32_t saddr) {
    uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(kChunkBytes >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
__host__ __device__ constexpr uint32_t idesc_bf16_bmn(int n) { return idesc_bf16_f32(n) | (1u << 16); }

// The MMA warps run converged: all lanes take the waits and the loops, one elected lane issues.  Descriptors and addresses are
// then the same in all lanes and stay in uniform registers, where the tensor core takes them from; issued from a branch
// of one lane, a product took 46 cycles at least (and 80 beside busy softmax warps), so 32 (128 x 64 x 16).
static __device__ __forceinline__ uint32_t elect_one() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e;
}
// a value that all lanes share, known to be so
template <typename T>
static __device__ __forceinline__ T uniform(T v) {
    return __shfl_sync(0xffffffffu, v, 0);
}
static __device__ __forceinline__ void issue_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t el) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(el)
        : "memory");
}
static __device__ __forceinline__ void issue_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t el) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(el)
        : "memory");
}
static __device__ __forceinline__ void commit_to(uint64_t* bar, uint32_t el) {
    asm volatile(
        "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %1, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)),
        "r"(el)
        : "memory");
}
// D[tmem] = A[smem] B[smem]^T over CHUNKS chunks of 64 columns, both K-major.
template <int CHUNKS>
static __device__ __forceinline__ void mma_tile_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t el) {
    const uint64_t ad = sdesc_sw128(a), bd = sdesc_sw128(b);
#pragma unroll
    for (int k = 0; k < CHUNKS * 4; ++k) {
        const uint64_t off = (uint64_t)((k >> 2) * (kChunkBytes >> 4) + (k & 3) * 2);
        issue_ss(d, ad + off, bd + off, idesc, k != 0 ? 1u : 0u, el);
    }
}
// D[tmem] (+)= A[tmem: bf16 pairs] B over 16 * STEPS rows of B (MN-major): 32 rows of A's K axis (two steps of 8 columns)
// every GAP columns
template <int GAP, int STEPS = kTile / 16>
static __device__ __forceinline__ void mma_tile_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate,
                                                   uint32_t el) {
    const uint64_t bd = sdesc_mn(b);
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
        issue_ts(d, a + (uint32_t)((k >> 1) * GAP + (k & 1) * 8), bd + (uint64_t)(k * 128), idesc,
                 accumulate || k != 0 ? 1u : 0u, el);
}
// D[tmem] = A[tmem: bf16 pairs, CHUNKS * 32 columns] B[smem]^T, B K-major in chunks of 64 columns
template <int CHUNKS>
static __device__ __forceinline__ void mma_rows_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t el) {
    const uint64_t bd = sdesc_sw128(b);
#pragma unroll
    for (int k = 0; k < CHUNKS * 4; ++k)
        issue_ts(d, a + (uint32_t)(8 * k), bd + (uint64_t)((k >> 2) * (kChunkBytes >> 4) + (k & 3) * 2), idesc,
                 k != 0 ? 1u : 0u, el);
}
// 8 bf16 elements [e0, e0 + 8) of a row of w on a 16-byte boundary (zeros past w, and where !has)
static __device__ __forceinline__ uint4 load_eight(const __nv_bfloat16* row, int e0, int w, bool has) {
    if (has && e0 + 8 <= w) return __ldg(reinterpret_cast<const uint4*>(row + e0));
    uint32_t u[4] = {0, 0, 0, 0};
    if (has && e0 < w) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e0 + e < w) u[e >> 1] |= (uint32_t)__ldg(reinterpret_cast<const unsigned short*>(row) + e0 + e) << (16 * (e & 1));
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
// 16 elements [c, c + 16) as 8 words
static __device__ __forceinline__ void load_words(uint32_t (&x)[8], const __nv_bfloat16* row, int c, int w, bool has) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint4 v = load_eight(row, c + 8 * h, w, has);
        x[4 * h] = v.x;
        x[4 * h + 1] = v.y;
        x[4 * h + 2] = v.z;
        x[4 * h + 3] = v.w;
    }
}
static __device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(v[0]), "r"(v[1]),
                 "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

// Untiled copy of `bytes` (a multiple of 16, both addresses on 16-byte boundaries) to shared memory.
static __device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

static __device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
static __device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// (a0, a1) * (b, b) + (c, c)
static __device__ __forceinline__ void fma2(float& a0, float& a1, float b, float c) {
    asm("{\n\t.reg .b64 x, y, z;\n\t"
        "mov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a0), "+f"(a1)
        : "f"(b), "f"(c));
}
// (a0, a1) + (b0, b1)
static __device__ __forceinline__ void add2(float& a0, float& a1, float b0, float b1) {
    asm("{\n\t.reg .b64 x, y;\n\t"
        "mov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\t"
        "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a0), "+f"(a1)
        : "f"(b0), "f"(b1));
}
// (a0, a1) * (b0, b1)
static __device__ __forceinline__ void mul2(float& a0, float& a1, float b0, float b1) {
    asm("{\n\t.reg .b64 x, y;\n\t"
        "mov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\t"
        "mul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a0), "+f"(a1)
        : "f"(b0), "f"(b1));
}

// 32 bf16 columns (16 words) of each lane's row to global memory, a warp at once; `left` columns are there (a multiple of 8), rows
// start on 16-byte boundaries, lanes without `mine` have none.  Lane after lane would store 16 bytes to 32 rows, 32 wavefronts an
// instruction (3,100 clocks for 128 keys' dK and dV of 64); four lanes exchange their pieces, so that they store 64 bytes of a row.
static __device__ __forceinline__ void store_rows(__nv_bfloat16* row, const uint32_t (&p)[16], int left, bool mine) {
    const int lane = threadIdx.x & 31;
    const bool odd = lane & 1, high = lane & 2;
    uint32_t x[2][4], y[2][4], z[4][4];  // piece lane % 2 (x) and 2 + lane % 2 (y) of the even and the odd row; lane % 4 of four rows
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t a = __shfl_xor_sync(0xffffffffu, odd ? p[e] : p[4 + e], 1);
        const uint32_t b = __shfl_xor_sync(0xffffffffu, odd ? p[8 + e] : p[12 + e], 1);
        x[0][e] = odd ? a : p[e];
        x[1][e] = odd ? p[4 + e] : a;
        y[0][e] = odd ? b : p[8 + e];
        y[1][e] = odd ? p[12 + e] : b;
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t a = __shfl_xor_sync(0xffffffffu, high ? x[r][e] : y[r][e], 2);
            z[r][e] = high ? a : x[r][e];
            z[2 + r][e] = high ? y[r][e] : a;
        }
    const unsigned rows = __ballot_sync(0xffffffffu, mine);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int from = (lane & ~3) + r;
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), from));
        if ((rows >> from & 1u) && (lane & 3) * 8 < left)
            *reinterpret_cast<uint4*>(dst + (lane & 3) * 8) = make_uint4(z[r][0], z[r][1], z[r][2], z[r][3]);
    }
}

// The same for rows on any boundary and any number of columns: the 16 lanes of a half warp exchange their words until each has
// one word of 16 rows, so that they store 64 bytes of a row together (32 columns element by element: 1,024 wavefronts, so 64).
static __device__ __forceinline__ void store_rows_any(__nv_bfloat16* row, uint32_t (&p)[16], int left, bool mine) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int bit = 1; bit < 16; bit <<= 1)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i & bit) continue;
            const bool up = lane & bit;
            const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? p[i] : p[i | bit], bit);
            if (up)
                p[i] = got;
            else
                p[i | bit] = got;
        }
    const unsigned rows = __ballot_sync(0xffffffffu, mine);
    const int c = 2 * (lane & 15);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int from = (lane & 16) + r;
        unsigned short* dst = reinterpret_cast<unsigned short*>(
            __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), from));
        if (!(rows >> from & 1u)) continue;
        if (c + 1 < left && (reinterpret_cast<uintptr_t>(dst) & 3) == 0) {
            *reinterpret_cast<uint32_t*>(dst + c) = p[r];
        } else {
            if (c < left) dst[c] = (unsigned short)p[r];
            if (c + 1 < left) dst[c + 1] = (unsigned short)(p[r] >> 16);
        }
    }
}

static __device__ __forceinline__ int keys_of(const XattnArgs& a, int b) {
    return a.lens ? min(max(__ldg(a.lens + b), 0), a.Lk) : a.Lk;
}
// bit l of word i: key j0 + 32 i + l may be read (taken by a whole warp)
template <int W>
static __device__ __forceinline__ void valid_words(uint32_t (&w)[W], const XattnArgs& a, int b, int j0, int n) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const int j = j0 + 32 * i + lane;
        const bool ok = j < n && (!a.mask || __ldg(a.mask + (long long)b * a.ldm + j) != 0);
        w[i] = __ballot_sync(0xffffffffu, ok);
    }
}
// zeroes the rows of a tile of `chunks` chunks whose bit is clear (a whole warp, four rows at a time; generic-proxy writes)
static __device__ __forceinline__ void zero_rows(uint8_t* tile, int chunks, const uint32_t (&w)[4]) {
    const int lane = threadIdx.x & 31;
    for (int c = 0; c < chunks; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (w[i] == 0xffffffffu) continue;
            const uint32_t bits = w[i] >> (lane >> 3);
#pragma unroll
            for (int r = 0; r < 32; r += 4)
                if (!(bits >> r & 1u))
                    *reinterpret_cast<uint4*>(tile + (size_t)c * kChunkBytes + (32 * i + r + (lane >> 3)) * 128 + (lane & 7) * 16) =
                        make_uint4(0, 0, 0, 0);
        }
}

// A tensor map over a (B, L, H, width) bf16 array, axes (width, H, L, B), box {64, bh, bl, 1}.  A batch (or head) stride of 0
// becomes an axis of one, indexed by 0 * coordinate.
struct HeadMap {
    CUtensorMap map;
    int bmul, hmul;
};
// whether every row of the array starts on a 16-byte boundary and the strides fit a tensor map
inline bool map_supported(const HeadView& v, int B, int L, int H) {
    auto ok = [](long long s, int n) { return n <= 1 || (s % 8 == 0 && s < (1LL << 38)); };
    return (uintptr_t)v.p % 16 == 0 && ok(v.b, B) && ok(v.l, L) && ok(v.h, H) && (L <= 1 || v.l > 0);
}
inline bool make_head_map(HeadMap* m, const HeadView& v, int B, int L, int H, int w, int bh, int bl) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    m->bmul = B > 1 && v.b == 0 ? 0 : 1;
    m->hmul = H > 1 && v.h == 0 ? 0 : 1;
    cuuint64_t dims[4] = {(cuuint64_t)w, (cuuint64_t)(m->hmul ? H : 1), (cuuint64_t)L, (cuuint64_t)(m->bmul ? B : 1)};
    // the strides of axes of one element are never used: any legal value
    cuuint64_t strides[3] = {(cuuint64_t)(dims[1] > 1 ? v.h * 2 : 256), (cuuint64_t)(L > 1 ? v.l * 2 : 256),
                             (cuuint64_t)(dims[3] > 1 ? v.b * 2 : 256)};
    cuuint32_t box[4] = {(cuuint32_t)kChunk, (cuuint32_t)bh, (cuuint32_t)bl, 1};
    cuuint32_t es[4] = {1, 1, 1, 1};
    return fn(&m->map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, v.p, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace xtc
}  // namespace gs
