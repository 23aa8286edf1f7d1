// gs_paged.h -- the paged cache's book-keeping and the verification of drafted tokens.
#pragma once

#include "gs_internal.h"
#include "gs_xattn.h"

namespace gs {

// ----------------------------------------------------------------- slots and stores (gs_paged.cu)
struct SlotArgs {
    const int *lens, *added;
    int B, L, page, pages;
    const int* free_list;
    int n_free;
    const int* from;
    int* table;
    long long ldt;
    int cols;
    int *slots, *new_lens, *taken;
};
cudaError_t launch_page_slots(const SlotArgs& a, int sms, cudaStream_t s);

struct StoreArgs {
    int bytes;  // of an element
    int B, L, H, w[2];
    HeadView src[2], dst[2];  // K and V: rows (b, l, h), and (page, row, h) of the cache
    const int* slots;
    long long lds;
    int pages, page;
    int vec[2];  // the array moves 16 bytes at a time
};
cudaError_t launch_page_store(const StoreArgs& a, int sms, cudaStream_t s);

// ----------------------------------------------------------------- attention on the tensor cores (gs_paged_mma.cu)
// bf16, widths in multiples of 8, arrays on 16-byte boundaries; else launch_xattn_rows through kPagedKeys
bool paged_mma_supported(const XattnArgs& a);
long long paged_mma_bytes(const XattnArgs& a, int sms);  // workspace
cudaError_t launch_paged_mma(const XattnArgs& a, int sms, int device, cudaStream_t s);

// ----------------------------------------------------------------- verification (gs_verify.cu)
struct VerifyArgs {
    const void *P, *D;
    bool bf16;
    int B, K, M;
    long long pb, pr, db, dr;
    const int *drafts, *dlens;
    const float* U;
    int *accepted, *tokens;
};
cudaError_t launch_verify(const VerifyArgs& a, int sms, cudaStream_t s);

}  // namespace gs
