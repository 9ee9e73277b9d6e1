// branch_evict: sequences with more own rows than their budget keep those of the largest weights.
//
// A row's rank is (latest positions first, weight, lower position, lower row); of n rows those of the n - budget lowest ranks are evicted.  One
// workgroup a (sequence, KV head) finds them and pairs the evicted rows below the budget with the kept ones behind it, both in ascending order.
// What bounds it: a chain of look-ups (length, page, weight) and barriers where few rows are evicted, the moves where many are.
//   up to 16384 rows in the table   weights and positions in registers.  One row too many, a generated token's case: the lowest rank by one reduction.  Else
//                          histograms of 2048 bins over the range of what is left narrow the border down to candidates that are ranked in pairs
//   more                   a radix select that reads weights and positions again in every pass
// Few moves are made by the workgroup itself (a second launch took 4 us for one row of each of 512 heads), many by a second launch over the whole chip.
#include <algorithm>

#include "kd_device.h"
#include "kd_pages.h"
#include "kd_select.h"

namespace kd {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int LNT = 1024;        // threads of the long form
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

using Move = BranchMove;

// Floats in the order of their values as unsigned numbers; NaN as -inf, both zeros as one
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x != x ? -INFINITY : x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Rows of one head from one place to another, 16 bytes a thread and turn: thread `tid` of `threads`
__device__ __forceinline__ void move_rows(const BranchEvictParams &p, const Move *moves, int count, int64_t tid, int64_t threads)
{
    const int units = p.D / 8, shift = units == 16 ? 5 : 4;   // of a row of K, then of V
    for (int64_t i = tid; i < (int64_t)count << shift; i += threads) {
        const Move m = moves[i >> shift];
        const int u = (int)i & (2 * units - 1);
        u32x4 *rows = reinterpret_cast<u32x4 *>(u < units ? p.pages.k : p.pages.v);
        const int at = u & (units - 1);
        if (u == 0) {
            const float w = p.w[m.from];
            const int32_t position = p.positions[m.from];
            p.w[m.to] = w;
            p.positions[m.to] = position;
        }
        rows[m.to * units + at] = rows[m.from * units + at];
    }
}

constexpr int OWN_MOVES = 128;   // moves that the workgroup of a head makes itself
constexpr int BINS = 2048, CANDIDATES = 512;

template <int NT, int RPT>
__global__ __launch_bounds__(NT) void evict_select_kernel(BranchEvictParams p)
{
    constexpr int WAVES = NT / 64, WORDS = WAVES * RPT;   // words of 64 rows
    __shared__ uint32_t hist[BINS], wave_tot[WAVES], bits[WORDS * 2], words[WORDS + 1], cand_key[CANDIDATES], cand_low[CANDIDATES], found[4], counted;
    __shared__ int cand_row[CANDIDATES];
    __shared__ uint32_t low_s[3][WAVES];
    __shared__ Move list[OWN_MOVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int s = p.by_hkv.divide(blockIdx.x), h = (int)blockIdx.x - s * p.hkv;
    const int len = table_entry(p.pages.lens, s), fresh = new_rows(len, asked_rows(p.pages, p.Bt, s), p.Bt), pos0 = p.pos0 ? table_entry(p.pos0, s) : 0;
    const int n = len < 0 ? 0 : rows_with(p.pages, len, fresh);
    const int64_t all = (int64_t)len + fresh;
    const bool evicts = len >= 0 && all > p.budget;   // uniform
    if (tid == 0) p.counts[blockIdx.x] = 0;
    // what the thread's rows tid + NT i hold.  (A sequence that does not evict: the new rows' positions alone.)
    const Head head{p.pages.table + (int64_t)s * p.pages.width, p.pages.page_shift, p.hkv, h};
    int page[RPT];
    bool absent = all > n;
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        page[i] = -1;
        if (NT * i < n && (evicts || NT * (i + 1) > len)) {   // uniform
            const int e = table_entry(head.table, min(tid + NT * i, n - 1) >> head.shift);
            page[i] = (uint32_t)e < (uint32_t)p.pages.n_pages ? e : -1;
            absent = absent || page[i] < 0;
        }
    }
    auto place = [&](int i) { return (((int64_t)max(page[i], 0) * head.hkv + h) << head.shift) + ((tid + NT * i) & ((1 << head.shift) - 1)); };
    uint32_t key[RPT], low[RPT];   // a row goes ahead of another if its key is lower, or its `low` at equal keys, or its row higher at equal both
    const int64_t late = (int64_t)pos0 + n - p.window;   // positions from here on are kept ahead of all others
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int r = tid + NT * i;
        key[i] = low[i] = 0xFFFFFFFFu;
        if (NT * i < n && (evicts || NT * (i + 1) > len)) {   // uniform
            int32_t position = (int32_t)((uint32_t)pos0 + (uint32_t)r);
            if (evicts) {
                const int32_t before = p.positions[place(i)];
                const float w = p.w[place(i)];
                position = r < len ? before : position;
                if (r < n) {
                    key[i] = p.window > 0 && position >= late ? 0xFFFFFFFFu : ordered(w);
                    low[i] = ~((uint32_t)position ^ 0x80000000u);
                }
            }
            if (r >= len && r < n && page[i] >= 0) p.positions[place(i)] = position;
        }
    }
    if (!evicts) return;
    if (__syncthreads_or(absent)) {
        if (tid == 0 && p.status) atomicOr(p.status, LEFT_OUT_ROW);
        return;
    }
    int need = n - p.budget;
    if (need == 1) {
        // the row that goes ahead of all others
        uint32_t k = 0xFFFFFFFFu, l = 0xFFFFFFFFu;
        int row = -1;
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = tid + NT * i;
            if (r < n && (row < 0 || key[i] < k || (key[i] == k && low[i] <= l))) {   // (of equal ones the higher row, which comes later)
                k = key[i];
                l = low[i];
                row = r;
            }
        }
        auto first = [&](uint32_t &k0, uint32_t &l0, int &r0, uint32_t k1, uint32_t l1, int r1) {
            const bool take = r1 >= 0 && (r0 < 0 || k1 < k0 || (k1 == k0 && (l1 < l0 || (l1 == l0 && r1 > r0))));
            k0 = take ? k1 : k0;
            l0 = take ? l1 : l0;
            r0 = take ? r1 : r0;
        };
#pragma unroll
        for (int m = 1; m < 64; m *= 2) first(k, l, row, __shfl_xor(k, m), __shfl_xor(l, m), __shfl_xor(row, m));
        if (lane == 0) {
            low_s[0][wave] = k;
            low_s[1][wave] = l;
            low_s[2][wave] = (uint32_t)row;
        }
        __syncthreads();
        k = low_s[0][lane % WAVES];
        l = low_s[1][lane % WAVES];
        row = (int)low_s[2][lane % WAVES];
#pragma unroll
        for (int m = 1; m < WAVES; m *= 2) first(k, l, row, __shfl_xor(k, m), __shfl_xor(l, m), __shfl_xor(row, m));
        row = __builtin_amdgcn_readfirstlane(row);
        if (row >= p.budget) return;   // the last row: it lies behind the budget
        if (tid < p.D / 4) {
            list[0] = Move{head.at(p.budget), head.at(row)};   // (every thread its own copy of the same)
            move_rows(p, list, 1, tid, p.D / 4);
        }
        return;
    }
    // the range of the keys
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
#pragma unroll
    for (int i = 0; i < RPT; ++i)
        if (tid + NT * i < n) {
            lo = min(lo, key[i]);
            hi = max(hi, key[i]);
        }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        lo = min(lo, (uint32_t)__shfl_xor(lo, m));
        hi = max(hi, (uint32_t)__shfl_xor(hi, m));
    }
    if (lane == 0) {
        low_s[0][wave] = lo;
        low_s[1][wave] = hi;
    }
    for (int i = tid; i < BINS; i += NT) hist[i] = 0;
    for (int i = tid; i < WORDS * 2; i += NT) bits[i] = 0;
    if (tid == 0) counted = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        lo = min(lo, low_s[0][w]);
        hi = max(hi, low_s[1][w]);
    }
    // Narrow down: of the rows whose value (the key; later, among those of key `equal`, low) lies in [lo, hi] the `need` first ones go; those below lo go, those
    // above hi stay
    bool by_low = false;
    uint32_t equal = 0, count = 0;
    for (;;) {
        const uint32_t span = hi - lo;
        const int down = span < BINS ? 0 : 32 - 11 - __builtin_clz(span);
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const uint32_t v = by_low ? low[i] : key[i];
            if (tid + NT * i < n && v >= lo && v <= hi && (!by_low || key[i] == equal)) atomicAdd(&hist[(v - lo) >> down], 1u);
        }
        __syncthreads();
        constexpr int PER = BINS / NT;
        uint32_t mine[PER], sum = 0, total;
#pragma unroll
        for (int b = 0; b < PER; ++b) {
            mine[b] = hist[tid * PER + b];
            sum += mine[b];
        }
        uint32_t before = block_exclusive_scan_t<NT, uint32_t>(sum, wave_tot, &total);
#pragma unroll
        for (int b = 0; b < PER; ++b) {
            if (before < (uint32_t)need && (uint32_t)need <= before + mine[b]) {   // one thread's
                found[0] = tid * PER + b;
                found[1] = need - before;
                found[2] = mine[b];
            }
            before += mine[b];
            hist[tid * PER + b] = 0;   // for the next turn
        }
        __syncthreads();
        const uint32_t from = lo + (found[0] << down);
        hi = hi - from >= 1u << down ? from + ((1u << down) - 1) : hi;
        lo = from;
        need = (int)found[1];
        count = found[2];
        if (count == (uint32_t)need || count <= CANDIDATES) break;
        if (lo == hi) {
            if (by_low) break;   // alike in all but their rows
            by_low = true;
            equal = lo;
            lo = 0;
            hi = 0xFFFFFFFFu;
        }
        __syncthreads();
    }
    auto value = [&](int i) { return by_low ? low[i] : key[i]; };
    auto below = [&](int i) { return by_low ? key[i] < equal || (key[i] == equal && low[i] < lo) : key[i] < lo; };
    auto inside = [&](int i) { return value(i) >= lo && value(i) <= hi && (!by_low || key[i] == equal); };
    const bool whole = count == (uint32_t)need, ranked = !whole && count <= CANDIDATES;   // uniform
    // numbers in `words` become those of all words before, the last one their sum
    auto add_up = [&]() {
        __syncthreads();
        if (wave == 0) {
            constexpr int EACH = (WORDS + 63) / 64;
            uint32_t x[EACH], sum = 0;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                x[k] = lane * EACH + k < WORDS ? words[lane * EACH + k] : 0u;
                sum += x[k];
            }
            uint32_t before = wave_inclusive_scan(sum) - sum;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                if (lane * EACH + k < WORDS) words[lane * EACH + k] = before;
                before += x[k];
            }
            if (lane == 63) words[WORDS] = before;
        }
        __syncthreads();
    };
    if (ranked) {
        // the candidates, and which of them go
#pragma unroll
        for (int i = 0; i < RPT; ++i)
            if (tid + NT * i < n && inside(i)) {
                const uint32_t c = atomicAdd(&counted, 1u);   // (their order is of no consequence)
                cand_key[c] = key[i];
                cand_low[c] = low[i];
                cand_row[c] = tid + NT * i;
            }
        __syncthreads();
        for (int c = tid; c < (int)count; c += NT) {
            const uint32_t k = cand_key[c], l = cand_low[c];
            const int r = cand_row[c];
            int rank = 0;
            for (int o = 0; o < (int)count; ++o) {
                const uint32_t ko = cand_key[o], lw = cand_low[o];
                rank += ko < k || (ko == k && (lw < l || (lw == l && cand_row[o] > r)));
            }
            if (rank < need) atomicOr(&bits[r >> 5], 1u << (r & 31));
        }
        __syncthreads();
    } else if (!whole) {
        // alike in all but their rows: the last `need` of them
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const uint64_t same = __builtin_amdgcn_ballot_w64(tid + NT * i < n && inside(i));
            if (lane == 0) words[i * WAVES + wave] = (uint32_t)__popcll(same);
        }
        add_up();
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const uint64_t same = __builtin_amdgcn_ballot_w64(tid + NT * i < n && inside(i));
            const int ahead = (int)words[i * WAVES + wave] + __popcll(same & ((1ull << lane) - 1)), r = tid + NT * i;
            if ((same >> lane & 1) && ahead >= (int)count - need) atomicOr(&bits[r >> 5], 1u << (r & 31));
        }
        __syncthreads();
    }
    // evicted rows below the budget and kept ones behind it: a word of 64 rows each wave and turn, their numbers added up in the order of the rows
    uint64_t holes[RPT], movers[RPT];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int r = tid + NT * i;
        const bool out = r < n && (below(i) || (inside(i) && (whole || (bits[r >> 5] >> (r & 31) & 1))));
        holes[i] = __builtin_amdgcn_ballot_w64(out && r < p.budget);
        movers[i] = __builtin_amdgcn_ballot_w64(r < n && !out && r >= p.budget);
        if (lane == 0) words[i * WAVES + wave] = (uint32_t)__popcll(holes[i]) << 16 | (uint32_t)__popcll(movers[i]);
    }
    add_up();
    const int count_moves = (int)(words[WORDS] & 0xFFFFu);
    const bool own = count_moves <= OWN_MOVES;   // uniform
    Move *to = own ? list : p.moves + (int64_t)blockIdx.x * p.most_moves;
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const uint32_t before = words[i * WAVES + wave];
        const uint64_t ahead = (1ull << lane) - 1;
        if (holes[i] >> lane & 1) to[(before >> 16) + __popcll(holes[i] & ahead)].to = place(i);
        if (movers[i] >> lane & 1) to[(before & 0xFFFFu) + __popcll(movers[i] & ahead)].from = place(i);
    }
    if (!own) {
        if (tid == 0) p.counts[blockIdx.x] = count_moves;
        return;
    }
    __syncthreads();
    move_rows(p, list, count_moves, tid, NT);
}

__global__ __launch_bounds__(LNT) void evict_select_long_kernel(BranchEvictParams p)
{
    __shared__ uint32_t key_s[CACHED], hist[256], wave_tot[LNT / 64], found[3];
    const int tid = threadIdx.x;
    const int s = p.by_hkv.divide(blockIdx.x), h = (int)blockIdx.x - s * p.hkv;
    Move *moves = p.moves + (int64_t)blockIdx.x * p.most_moves;
    const int len = table_entry(p.pages.lens, s), fresh = new_rows(len, asked_rows(p.pages, p.Bt, s), p.Bt);
    if (tid == 0) p.counts[blockIdx.x] = 0;
    if (len < 0) return;
    const int64_t all = (int64_t)len + fresh;
    const int n = rows_with(p.pages, len, fresh), pos0 = p.pos0 ? table_entry(p.pos0, s) : 0;
    const Head head{p.pages.table + (int64_t)s * p.pages.width, p.pages.page_shift, p.hkv, h};
    auto exists = [&](int r) { return (uint32_t)table_entry(head.table, r >> head.shift) < (uint32_t)p.pages.n_pages; };
    for (int r = len + tid; r < n; r += LNT)
        if (exists(r)) p.positions[head.at(r)] = (int32_t)((uint32_t)pos0 + (uint32_t)r);
    if (all <= p.budget) return;   // uniform, as all that follows
    bool absent = all > n;
    for (int e = tid; e <= (n - 1) >> head.shift; e += LNT) absent |= (uint32_t)table_entry(head.table, e) >= (uint32_t)p.pages.n_pages;
    if (__syncthreads_or(absent)) {
        if (tid == 0 && p.status) atomicOr(p.status, LEFT_OUT_ROW);
        return;
    }
    const int64_t late = (int64_t)pos0 + n - p.window;   // positions from here on are kept ahead of all others
    auto position = [&](int r) { return r >= len ? (int32_t)((uint32_t)pos0 + (uint32_t)r) : p.positions[head.at(r)]; };
    auto fetch_key = [&](int r) { return p.window > 0 && position(r) >= late ? 0xFFFFFFFFu : ordered(p.w[head.at(r)]); };
    for (int r = tid; r < min(n, CACHED); r += LNT) key_s[r] = fetch_key(r);
    auto key = [&](int r) { return r < CACHED ? key_s[r] : fetch_key(r); };
    auto low = [&](int r) { return ~((uint32_t)position(r) ^ 0x80000000u); };   // (of equal weights, the lower position ranks higher)
    // the border: the (n - budget)-th lowest rank
    uint64_t border = 0;
    int need = n - p.budget, digits = 0;   // of the rows that agree with the border in `digits` digits of eight bits, the `need` lowest go
    for (; digits < 8; ++digits) {
        const int down = 56 - 8 * digits;
        for (int i = tid; i < 256; i += LNT) hist[i] = 0;
        __syncthreads();
        for (int r = tid; r < n; r += LNT) {
            const uint64_t rank = (uint64_t)key(r) << 32 | (digits >= 4 ? low(r) : 0u);
            if (digits == 0 || rank >> (down + 8) == border >> (down + 8)) atomicAdd(&hist[rank >> down & 255], 1u);
        }
        __syncthreads();
        uint32_t total;
        const uint32_t mine = tid < 256 ? hist[tid] : 0u, before = block_exclusive_scan_t<LNT, uint32_t>(mine, wave_tot, &total);
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
        for (int base = (n - 1) / LNT * LNT; base >= 0; base -= LNT) {   // the last rows first
            const int r = base + LNT - 1 - tid;
            uint32_t total;
            const uint32_t same = r < n && ((uint64_t)key(r) << 32 | low(r)) == border;
            __syncthreads();
            const uint32_t before = block_exclusive_scan_t<LNT, uint32_t>(same, wave_tot, &total);
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
    for (int base = 0; base < n; base += LNT) {
        const int r = base + tid;
        const bool out = r < n && evicted(r);
        const bool hole = out && r < p.budget, mover = r < n && !out && r >= p.budget;
        uint32_t total;
        __syncthreads();
        const uint32_t before = block_exclusive_scan_t<LNT, uint32_t>((uint32_t)hole << 16 | (uint32_t)mover, wave_tot, &total);
        if (hole) moves[to + (int)(before >> 16)].to = head.at(r);
        if (mover) moves[fro + (int)(before & 0xFFFFu)].from = head.at(r);
        to += (int)(total >> 16);
        fro += (int)(total & 0xFFFFu);
    }
    if (tid == 0) p.counts[blockIdx.x] = fro;
}

__global__ __launch_bounds__(256) void evict_move_kernel(BranchEvictParams p)
{
    const int count = p.counts[blockIdx.x];
    move_rows(p, p.moves + (int64_t)blockIdx.x * p.most_moves, count, (int64_t)blockIdx.y * 256 + threadIdx.x, (int64_t)gridDim.y * 256);
}

}  // namespace

size_t branch_evict_workspace(int n_seqs, int hkv, int64_t table_rows, int budget, int *most_moves, size_t *off_moves)
{
    // as many rows move as there are behind the budget, and no more than there are places
    *most_moves = (int)std::max<int64_t>(std::min<int64_t>(budget, table_rows - budget), 0);
    *off_moves = ((size_t)n_seqs * hkv * 4 + 255) & ~(size_t)255;
    return (*off_moves + (size_t)n_seqs * hkv * *most_moves * sizeof(Move) + 255) & ~(size_t)255;
}

hipError_t launch_branch_evict(BranchEvictParams p, hipStream_t s)
{
    p.by_hkv.set((uint32_t)p.hkv);
    const unsigned heads = (unsigned)(p.n_seqs * p.hkv);
    const int64_t rows = (int64_t)p.pages.width << p.pages.page_shift;
    const bool registers = rows <= 16384;
    if (rows <= 1024) hipLaunchKernelGGL((evict_select_kernel<256, 4>), dim3(heads), dim3(256), 0, s, p);
    else if (rows <= 4096) hipLaunchKernelGGL((evict_select_kernel<512, 8>), dim3(heads), dim3(512), 0, s, p);
    else if (registers) hipLaunchKernelGGL((evict_select_kernel<1024, 16>), dim3(heads), dim3(1024), 0, s, p);
    else hipLaunchKernelGGL(evict_select_long_kernel, dim3(heads), dim3(LNT), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.most_moves == 0 || (registers && p.most_moves <= OWN_MOVES)) return e;
    const unsigned parts = (unsigned)std::max<int64_t>(1, std::min<int64_t>(2048 / heads, ((int64_t)p.most_moves * (p.D / 4) + 255) / 256));
    hipLaunchKernelGGL(evict_move_kernel, dim3(heads, parts), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace kd
