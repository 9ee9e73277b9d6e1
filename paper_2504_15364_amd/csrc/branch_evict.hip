// branch_evict: sequences with more own rows than their budget keep those of the largest weights.
//
// A row's rank is (latest positions first, weight, lower position, lower row); of n rows those of the n - budget lowest ranks are evicted.  One
// workgroup a (sequence, KV head) finds the border rank by a radix select over the 64 bits of (weight, position), eight at a time, and
// pairs the evicted rows below the budget with the kept ones behind it, both in ascending order; a second launch moves the rows.
// What bounds it: the chain of the select's passes where few rows are evicted, the moves where many are.
#include <algorithm>

#include "kd_device.h"
#include "kd_pages.h"
#include "kd_select.h"

namespace kd {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 1024;
constexpr int CACHED = 16384;   // rows whose weights are kept in LDS, in the form in which they are compared

// A row of a head in the pages of a sequence
struct Head {
    const int32_t *table;
    int shift, hkv, h;
    __device__ __forceinline__ int64_t at(int r) const
    {
        return (((int64_t)table_entry(table, r >> shift) * hkv + h) << shift) + (r & ((1 << shift) - 1));
    }
};

// Floats in the order of their values as unsigned numbers; NaN as -inf, both zeros as one
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x != x ? -INFINITY : x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(NT) void evict_select_kernel(BranchEvictParams p)
{
    __shared__ uint32_t key_s[CACHED], hist[256], wave_tot[NT / 64], found[3];
    const int tid = threadIdx.x;
    const int s = p.by_hkv.divide(blockIdx.x), h = (int)blockIdx.x - s * p.hkv;
    int32_t *moves = p.moves + (int64_t)blockIdx.x * (1 + 2 * (int64_t)p.most_moves);
    const int len = table_entry(p.pages.lens, s), fresh = new_rows(len, asked_rows(p.pages, p.Bt, s), p.Bt);
    if (tid == 0) moves[0] = 0;
    if (len < 0) return;
    const int64_t all = (int64_t)len + fresh;
    const int n = rows_with(p.pages, len, fresh), pos0 = p.pos0 ? table_entry(p.pos0, s) : 0;
    const Head head{p.pages.table + (int64_t)s * p.pages.width, p.pages.page_shift, p.hkv, h};
    auto exists = [&](int r) { return (uint32_t)table_entry(head.table, r >> head.shift) < (uint32_t)p.pages.n_pages; };
    for (int r = len + tid; r < n; r += NT)
        if (exists(r)) p.positions[head.at(r)] = (int32_t)((uint32_t)pos0 + (uint32_t)r);
    if (all <= p.budget) return;   // uniform, as all that follows
    bool absent = all > n;
    for (int e = tid; e <= (n - 1) >> head.shift; e += NT) absent |= (uint32_t)table_entry(head.table, e) >= (uint32_t)p.pages.n_pages;
    if (__syncthreads_or(absent)) {
        if (tid == 0 && p.status) atomicOr(p.status, LEFT_OUT_ROW);
        return;
    }
    const int64_t late = (int64_t)pos0 + n - p.window;   // positions from here on are kept ahead of all others
    auto position = [&](int r) { return r >= len ? (int32_t)((uint32_t)pos0 + (uint32_t)r) : p.positions[head.at(r)]; };
    auto fetch_key = [&](int r) { return p.window > 0 && position(r) >= late ? 0xFFFFFFFFu : ordered(p.w[head.at(r)]); };
    for (int r = tid; r < min(n, CACHED); r += NT) key_s[r] = fetch_key(r);
    auto key = [&](int r) { return r < CACHED ? key_s[r] : fetch_key(r); };
    auto low = [&](int r) { return ~((uint32_t)position(r) ^ 0x80000000u); };   // (of equal weights, the lower position ranks higher)
    // the border: the (n - budget)-th lowest rank
    uint64_t border = 0;
    int need = n - p.budget, digits = 0;   // of the rows that agree with the border in `digits` digits of eight bits, the `need` lowest go
    for (; digits < 8; ++digits) {
        const int down = 56 - 8 * digits;
        for (int i = tid; i < 256; i += NT) hist[i] = 0;
        __syncthreads();
        for (int r = tid; r < n; r += NT) {
            const uint64_t rank = (uint64_t)key(r) << 32 | (digits >= 4 ? low(r) : 0u);
            if (digits == 0 || rank >> (down + 8) == border >> (down + 8)) atomicAdd(&hist[rank >> down & 255], 1u);
        }
        __syncthreads();
        uint32_t total;
        const uint32_t mine = tid < 256 ? hist[tid] : 0u, before = block_exclusive_scan_t<NT, uint32_t>(mine, wave_tot, &total);
        if (tid < 256 && before < (uint32_t)need && (uint32_t)need <= before + mine) {
            found[0] = tid;
            found[1] = need - before;
            found[2] = mine;
        }
        __syncthreads();
        border |= (uint64_t)found[0] << down;
        need = (int)found[1];
        const bool whole = found[1] == found[2];   // all of them go
        __syncthreads();
        if (whole) {
            ++digits;
            break;
        }
    }
    const int down = 64 - 8 * digits;
    // Rows that agree with the border in all digits looked at go from the `need`-th last one on: more than `need` of them only where all 64 bits agree
    int from = 0;
    if (digits == 8) {
        __shared__ int row;
        if (tid == 0) row = 0;
        int left = need;
        for (int base = (n - 1) / NT * NT; base >= 0; base -= NT) {   // the last rows first
            const int r = base + NT - 1 - tid;
            uint32_t total;
            const uint32_t same = r < n && ((uint64_t)key(r) << 32 | low(r)) == border;
            __syncthreads();
            const uint32_t before = block_exclusive_scan_t<NT, uint32_t>(same, wave_tot, &total);
            if (same && (int)before == left - 1) row = r;
            left -= (int)total;
            if (left <= 0) break;
        }
        __syncthreads();
        from = row;
    }
    auto evicted = [&](int r) {
        const uint64_t rank = (uint64_t)key(r) << 32 | (digits > 4 ? low(r) : 0u);
        const uint64_t a = digits == 0 ? 0 : rank >> down, b = digits == 0 ? 0 : border >> down;
        return a < b || (a == b && r >= from);
    };
    // evicted rows below the budget and kept ones behind it, in ascending order
    int to = 0, fro = 0;
    for (int base = 0; base < n; base += NT) {
        const int r = base + tid;
        const bool out = r < n && evicted(r);
        const bool hole = out && r < p.budget, mover = r < n && !out && r >= p.budget;
        uint32_t total;
        __syncthreads();
        const uint32_t before = block_exclusive_scan_t<NT, uint32_t>((uint32_t)hole << 16 | (uint32_t)mover, wave_tot, &total);
        if (hole) moves[1 + 2 * (int64_t)(to + (int)(before >> 16)) + 1] = r;
        if (mover) moves[1 + 2 * (int64_t)(fro + (int)(before & 0xFFFFu))] = r;
        to += (int)(total >> 16);
        fro += (int)(total & 0xFFFFu);
    }
    if (tid == 0) moves[0] = fro;
}

// 16 bytes a thread
__global__ __launch_bounds__(256) void evict_move_kernel(BranchEvictParams p)
{
    const int s = p.by_hkv.divide(blockIdx.x), h = (int)blockIdx.x - s * p.hkv;
    const int32_t *moves = p.moves + (int64_t)blockIdx.x * (1 + 2 * (int64_t)p.most_moves);
    const int count = moves[0], units = p.D / 8;
    const Head head{p.pages.table + (int64_t)s * p.pages.width, p.pages.page_shift, p.hkv, h};
    for (int64_t i = (int64_t)blockIdx.y * 256 + threadIdx.x; i < (int64_t)count * units; i += (int64_t)gridDim.y * 256) {
        const int k = (int)(i / units), u = (int)(i - (int64_t)k * units);
        const int64_t a = head.at(moves[1 + 2 * (int64_t)k]), b = head.at(moves[2 + 2 * (int64_t)k]);
        reinterpret_cast<u32x4 *>(p.pages.k)[b * units + u] = reinterpret_cast<const u32x4 *>(p.pages.k)[a * units + u];
        reinterpret_cast<u32x4 *>(p.pages.v)[b * units + u] = reinterpret_cast<const u32x4 *>(p.pages.v)[a * units + u];
        if (u == 0) {
            p.w[b] = p.w[a];
            p.positions[b] = p.positions[a];
        }
    }
}

}  // namespace

size_t branch_evict_workspace(int n_seqs, int hkv, int64_t table_rows, int budget, int *most_moves)
{
    // as many rows move as there are behind the budget, and no more than there are places
    *most_moves = (int)std::max<int64_t>(std::min<int64_t>(budget, table_rows - budget), 0);
    return ((size_t)n_seqs * hkv * (1 + 2 * (size_t)*most_moves) * 4 + 255) & ~(size_t)255;
}

hipError_t launch_branch_evict(BranchEvictParams p, hipStream_t s)
{
    p.by_hkv.set((uint32_t)p.hkv);
    const unsigned heads = (unsigned)(p.n_seqs * p.hkv);
    hipLaunchKernelGGL(evict_select_kernel, dim3(heads), dim3(NT), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.most_moves == 0) return e;
    const unsigned parts = (unsigned)std::max<int64_t>(1, std::min<int64_t>(2048 / heads, ((int64_t)p.most_moves * (p.D / 8) + 255) / 256));
    hipLaunchKernelGGL(evict_move_kernel, dim3(heads, parts), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace kd
