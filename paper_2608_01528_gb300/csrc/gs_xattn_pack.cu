// gs_xattn_pack.cu -- bf16 inputs whose width is not a multiple of 8, laid out again for the tensor-core kernels of cross
// attention: rows of round8(width) elements, zeros behind the width, so that every row starts on a 16-byte boundary.
//
// A copy costs one more read and a write of the inputs; the products that it makes room for run many times as fast as on CUDA
// cores: 35 x 1,472 x 384, 28 / 4 heads of 32 and 87: 0.46 ms against 4.53; gradient of 26 x 704 x 1,536, 2 / 1 heads of
// 68 and 64: 0.10 against 1.89; 32 x 20 x 4,000, 8 heads of 100: 0.27 against 0.97, 4 rows 0.27 against 0.36.  Below that the CUDA cores
// read the memory once, in less than the copies take.  One launch for all arrays; a thread writes 16 bytes.

#include <algorithm>

#include "gs_xattn_tc.cuh"

namespace gs {
namespace {

struct Copy {
    HeadView src;
    __nv_bfloat16* dst;
    int L, H, w;
    long long pieces;  // of 16 bytes
};
struct Copies {
    Copy c[4];
};

__global__ void __launch_bounds__(256) k_xattn_pack(const Copies all) {
    const Copy& c = all.c[blockIdx.y];
    const int per = (c.w + 7) / 8;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < c.pieces; i += (long long)gridDim.x * 256) {
        const long long row = i / per, bl = row / c.H, b = bl / c.L;
        const int e0 = (int)(i - row * per) * 8;
        const unsigned short* src = reinterpret_cast<const unsigned short*>(c.src.p) + b * c.src.b + (bl - b * c.L) * c.src.l +
                                    (row - bl * c.H) * c.src.h + e0;
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e0 + e < c.w) w[e >> 1] |= (uint32_t)__ldg(src + e) << (16 * (e & 1));
        *reinterpret_cast<uint4*>(c.dst + i * 8) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// the arrays in order: Q, K, V, dO
struct Array {
    HeadView* v;
    int L, H, w;
};
Array array_of(XattnArgs& a, int i) {
    return i == 0   ? Array{&a.q, a.Lq, a.Hq, a.dk}
           : i == 1 ? Array{&a.k, a.Lk, a.Hkv, a.dk}
           : i == 2 ? Array{&a.v, a.Lk, a.Hkv, a.dv}
                    : Array{&a.dO, a.Lq, a.Hq, a.dv};
}
int round8(int w) { return (w + 7) / 8 * 8; }

}  // namespace

bool xattn_packs(const XattnArgs& a, bool backward, bool forced) {
    return a.dtype == GS_BF16 && a.G <= xtc::kTile && a.Lk > 0 && a.Lq > 0 && (backward || forced || a.rows >= 4);
}

int xattn_pack_room(const XattnArgs& a, bool backward) {
    return (a.dk % 8 ? kPackQ | kPackK : 0) | (a.dv % 8 ? kPackV | (backward ? kPackDO : 0) : 0);
}

int xattn_pack_need(const XattnArgs& a, bool backward) {
    const bool q = xtc::map_supported(a.q, a.B, a.Lq, a.Hq) && (a.Hq <= 1 || a.q.h > 0);
    const bool d = !backward || (xtc::map_supported(a.dO, a.B, a.Lq, a.Hq) && (a.Hq <= 1 || a.dO.h > 0));
    return (q ? 0 : kPackQ) | (xtc::map_supported(a.k, a.B, a.Lk, a.Hkv) ? 0 : kPackK) |
           (xtc::map_supported(a.v, a.B, a.Lk, a.Hkv) ? 0 : kPackV) | (d ? 0 : kPackDO);
}

long long xattn_ws_pack(const XattnArgs& a, int which) {
    long long n = 0;
    for (int i = 0; i < 4; ++i) {
        const Array x = array_of(const_cast<XattnArgs&>(a), i);
        if (which >> i & 1) n += (long long)a.B * x.L * x.H * round8(x.w) / 2;  // (a multiple of 4 floats)
    }
    return n;
}

cudaError_t launch_xattn_pack(XattnArgs& a, int which, float* room, cudaStream_t s) {
    Copies all{};
    int n = 0;
    long long most = 0;
    for (int i = 0; i < 4; ++i) {
        if (!(which >> i & 1)) continue;
        const Array x = array_of(a, i);
        const int w = round8(x.w);
        Copy& c = all.c[n++];
        c.src = *x.v;
        c.dst = reinterpret_cast<__nv_bfloat16*>(room);
        c.L = x.L;
        c.H = x.H;
        c.w = x.w;
        c.pieces = (long long)a.B * x.L * x.H * (w / 8);
        most = std::max(most, c.pieces);
        room += c.pieces * 4;
        *x.v = {reinterpret_cast<char*>(c.dst), (long long)x.L * x.H * w, (long long)x.H * w, w};
    }
    k_xattn_pack<<<dim3((unsigned)std::min<long long>((most + 255) / 256, 152 * 8), (unsigned)n), 256, 0, s>>>(all);
    return cudaGetLastError();
}

}  // namespace gs
