// gs_paged.cu -- a paged cache's book-keeping: which slots new tokens get, and their keys and values stored there.

#include <algorithm>

#include "gs_paged.h"

namespace gs {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// ----------------------------------------------------------------- slots
// have = ceil(len / page) pages are a request's already, want = ceil(end / page) it needs; the want - have new ones come from the
// free list, in the order of the requests: request b's behind those of 0..b-1.  Every block sums the needs of the requests before
// its own (8 bytes each, from L2), so that one launch without a workspace does, and scans its own 256 at a time.
struct Request {
    int len, end, have, want;
};
__device__ __forceinline__ Request request_of(const SlotArgs& a, int b) {
    const int cap = a.cols * a.page;
    Request r;
    r.len = min(max(__ldg(a.lens + b), 0), cap);
    r.end = (int)min((long long)r.len + min(max(__ldg(a.added + b), 0), a.L), (long long)cap);
    r.have = r.len / a.page + (r.len % a.page != 0);
    r.want = r.end / a.page + (r.end % a.page != 0);
    return r;
}

__global__ void __launch_bounds__(kThreads) k_page_slots(const SlotArgs a, int per) {
    __shared__ long long s_sum[kWarps], s_first[kThreads];
    __shared__ int s_len[kThreads], s_end[kThreads], s_have[kThreads], s_want[kThreads];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int b0 = (int)min((long long)blockIdx.x * per, (long long)a.B), b1 = (int)min((long long)b0 + per, (long long)a.B);
    const long long from = a.from ? max(__ldg(a.from), 0) : 0;
    long long base = 0;  // pages that the requests before take
    for (int b = tid; b < b0; b += kThreads) {
        const Request r = request_of(a, b);
        base += r.want - r.have;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) base += __shfl_xor_sync(0xffffffffu, base, o);
    if (lane == 0) s_sum[warp] = base;
    __syncthreads();
    base = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) base += s_sum[w];

    for (int c0 = b0; c0 < b1; c0 += kThreads) {
        const int count = min(kThreads, b1 - c0);
        Request r{0, 0, 0, 0};
        if (tid < count) r = request_of(a, c0 + tid);
        const int need = r.want - r.have;
        long long run = need;  // inclusive
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += v;
        }
        __syncthreads();  // the sums, and the last requests' values, have been read
        if (lane == 31) s_sum[warp] = run;
        __syncthreads();
        long long total = 0, before = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += s_sum[w];
            total += s_sum[w];
        }
        const long long first = from + base + before + run - need;  // in the free list
        const int got = (int)min(max((long long)a.n_free - first, 0ll), (long long)need);
        const int end = min(r.end, (r.have + got) * a.page);  // up to the first token without a page
        s_first[tid] = first;
        s_len[tid] = r.len;
        s_end[tid] = end;
        s_have[tid] = r.have;
        s_want[tid] = r.want;
        if (blockIdx.y == 0 && tid < count && a.new_lens) a.new_lens[c0 + tid] = end;
        __syncthreads();
        if (blockIdx.y == 0)
            for (int i = warp; i < count; i += kWarps)
                for (int c = s_have[i] + lane; c < s_want[i]; c += 32) {
                    const long long at = s_first[i] + c - s_have[i];
                    a.table[(long long)(c0 + i) * a.ldt + c] = at < a.n_free ? __ldg(a.free_list + at) : -1;
                }
        const long long cells = (long long)count * a.L;
        for (long long e = (long long)blockIdx.y * kThreads + tid; e < cells; e += (long long)gridDim.y * kThreads) {
            const int i = (int)(e / a.L);
            const long long at = s_len[i] + (e - (long long)i * a.L);
            int slot = -1;
            if (at < s_end[i]) {  // (what the table's new cells get is read from the free list, not from them)
                const int pos = (int)at;
                const int c = pos / a.page;
                const int page = c < s_have[i] ? a.table[(long long)(c0 + i) * a.ldt + c]
                                               : __ldg(a.free_list + s_first[i] + c - s_have[i]);
                if (page >= 0 && page < a.pages) slot = page * a.page + (pos - c * a.page);
            }
            a.slots[(long long)c0 * a.L + e] = slot;
        }
        base += total;
    }
    if (a.taken && b1 == a.B && blockIdx.x == gridDim.x - 1 && blockIdx.y == 0 && tid == 0) *a.taken = (int)base;
}

// ----------------------------------------------------------------- stores
// A warp moves one token's keys or values, four 16-byte loads of a lane on their way before the first store.  Bound by memory.
// (A row has fewer than 2^31 - 1024 elements, which leaves room for the last steps' numbers, and up to 2^33 bytes.)
template <typename T>
__device__ __forceinline__ void move_row(char* dst, const char* src, int H, int per, long long dh, long long sh) {
    const int lane = threadIdx.x & 31;
    constexpr int kAhead = 4;
    const int all = H * per;
    for (int t0 = lane; t0 < all; t0 += 32 * kAhead) {
        T v[kAhead];
        long long to[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int t = t0 + 32 * u;
            if (t >= all) break;
            const int h = H == 1 ? 0 : t / per, e = t - h * per;
            v[u] = *reinterpret_cast<const T*>(src + h * sh + (long long)e * sizeof(T));
            to[u] = h * dh + (long long)e * sizeof(T);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (t0 + 32 * u >= all) break;
            *reinterpret_cast<T*>(dst + to[u]) = v[u];
        }
    }
}

__global__ void __launch_bounds__(kThreads) k_page_store(const StoreArgs a) {
    const long long n = 2ll * a.B * a.L;
    for (long long i = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); i < n; i += (long long)gridDim.x * kWarps) {
        const int x = (int)(i & 1);
        const long long token = i >> 1, b = token / a.L, l = token - b * a.L;
        const int slot = __ldg(a.slots + b * a.lds + l);
        const int page = slot / a.page, row = slot - page * a.page;
        if (slot < 0 || page >= a.pages) continue;
        const HeadView &s = a.src[x], &d = a.dst[x];
        const char* from = s.p + (b * s.b + l * s.l) * a.bytes;
        char* to = d.p + (page * d.b + row * d.l) * a.bytes;
        if (a.vec[x])
            move_row<uint4>(to, from, a.H, (int)((long long)a.w[x] * a.bytes / 16), d.h * a.bytes, s.h * a.bytes);
        else if (a.bytes == 4)
            move_row<uint32_t>(to, from, a.H, a.w[x], d.h * 4, s.h * 4);
        else
            move_row<unsigned short>(to, from, a.H, a.w[x], d.h * 2, s.h * 2);
    }
}

}  // namespace

cudaError_t launch_page_slots(const SlotArgs& a, int sms, cudaStream_t s) {
    // about 256 tokens a block, at least one request, and no more than 1,024 blocks that sum what comes before them
    const long long per = std::max({1ll, (long long)kThreads / std::max(a.L, 1), (a.B + 1023ll) / 1024});
    const long long x = std::max(1ll, (a.B + per - 1) / per);
    const long long cells = std::min<long long>(per, kThreads) * a.L;
    const long long y = std::min<long long>(std::max(1ll, (cells + 4 * kThreads - 1) / (4 * kThreads)),
                                            std::max(1ll, 8ll * sms / x));
    k_page_slots<<<dim3((unsigned)x, (unsigned)y), kThreads, 0, s>>>(a, (int)per);
    return cudaGetLastError();
}

cudaError_t launch_page_store(const StoreArgs& args, int sms, cudaStream_t s) {
    StoreArgs a = args;
    const int H = a.H;
    bool flat = true;
    for (int x = 0; x < 2; ++x) {
        auto on_16 = [&](const HeadView& v, int nb, int nl) {
            auto ok = [&](long long stride, int n) { return n <= 1 || stride * a.bytes % 16 == 0; };
            return (uintptr_t)v.p % 16 == 0 && ok(v.b, nb) && ok(v.l, nl) && ok(v.h, H);
        };
        a.vec[x] = (long long)a.w[x] * a.bytes % 16 == 0 && on_16(a.src[x], a.B, a.L) && on_16(a.dst[x], a.pages, a.page);
        flat = flat && (H == 1 || (a.src[x].h == a.w[x] && a.dst[x].h == a.w[x]));
    }
    if (flat) {  // heads lie next to one another: one row of H * w
        a.H = 1;
        a.w[0] *= H;
        a.w[1] *= H;
    }
    const long long warps = 2ll * a.B * a.L;
    const unsigned grid = (unsigned)std::min<long long>((warps + kWarps - 1) / kWarps, 64ll * sms);
    k_page_store<<<grid, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace gs
