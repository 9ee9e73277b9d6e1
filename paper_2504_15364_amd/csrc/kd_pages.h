// Device helpers of the kernels that read the own rows of sequences in pages: how many rows there are, and where they lie.
#pragma once
#include "kd_branch.h"

namespace kd {

// Entry i of a table, of the lengths or of the token counts, which no kernel that reads them writes.  Where i is the same for all lanes of a wave
// this is a scalar load, which is not counted among the vector loads and copies.
__device__ __forceinline__ int table_entry(const int32_t *table, int64_t i)
{
    return ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)table)[i];
}
// New tokens of a sequence that holds `len` rows and is asked to take `asked`; 0 where it has nothing to do
__device__ __forceinline__ int new_rows(int len, int asked, int Bt) { return len < 0 ? 0 : max(0, min(asked, Bt)); }
__device__ __forceinline__ int asked_rows(const Pages &pages, int Bt, int s) { return pages.n_new ? table_entry(pages.n_new, s) : Bt; }
// Rows that the sequence holds with the new ones, of those that its table can name
__device__ __forceinline__ int rows_with(const Pages &pages, int len, int fresh)
{
    const int64_t n = (int64_t)len + fresh, most = (int64_t)pages.width << pages.page_shift;
    return (int)(n < most ? n : most);
}
}  // namespace kd
