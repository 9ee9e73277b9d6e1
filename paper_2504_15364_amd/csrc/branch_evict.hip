// branch_evict: sequences with more own rows than their budget keep those of the largest weights.
//
// A row's rank is (latest positions first, weight, lower position, lower row); of n rows those of the n - budget lowest ranks are evicted.  One
// workgroup a (sequence, KV head) finds them and pairs the evicted rows below the budget with the kept ones behind it, both in ascending order.
// What bounds it: a chain of look-ups (length, page, weight) and barriers where few rows are evicted, the moves where many are.
//   up to 16384 rows in the table   weights and positions in LDS.  One row too many, a generated token's case: the lowest rank by one reduction.  Else
//                          histograms of 2048 bins over the range of what is left narrow the border down to candidates that are ranked in pairs.  Loops
//                          over LDS and not rows in registers: with 16 of them a thread, every pass unrolled, the code of each was run once and
//                          waited for from memory (16 heads of 16384 rows 51 us)
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
template <class Moves>
__device__ __forceinline__ void move_rows(const BranchEvictParams &p, Moves move, int count, int64_t tid, int64_t threads)
{
    const int units = p.D / 8, shift = units == 16 ? 5 : 4;   // of a row of K, then of V
    for (int64_t i = tid; i < (int64_t)count << shift; i += threads) {
        const Move m = move(i >> shift);
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
constexpr int BINS = 2048, CANDIDATES = 128;

template <int NT, int ROWS>
__global__ __launch_bounds__(NT) void evict_select_kernel(BranchEvictParams p)
{
    constexpr int WAVES = NT / 64, WORDS = ROWS / 64;   // words of 64 rows
    // of every row: it goes ahead of another if its key is lower, or its `low` at equal keys, or its row higher at equal both
    __shared__ uint32_t key_s[ROWS], low_s[ROWS];
    __shared__ uint32_t hist[BINS], wave_tot[WAVES], words[WORDS + 1], cand_key[CANDIDATES], cand_low[CANDIDATES], found[4], counted, best[3][WAVES], range_s[3][2][WAVES];
    __shared__ uint64_t out_s[WORDS];   // a bit for every row that goes
    __shared__ int cand_row[CANDIDATES];
    __shared__ Move list[OWN_MOVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int s = p.by_hkv.divide(blockIdx.x), h = (int)blockIdx.x - s * p.hkv;
    const int len = table_entry(p.pages.lens, s), fresh = new_rows(len, asked_rows(p.pages, p.Bt, s), p.Bt), pos0 = p.pos0 ? table_entry(p.pos0, s) : 0;
    const int n = len < 0 ? 0 : rows_with(p.pages, len, fresh);
    const int64_t all = (int64_t)len + fresh;
    const Head head{p.pages.table + (int64_t)s * p.pages.width, p.pages.page_shift, p.hkv, h};
    if (tid == 0) p.counts[blockIdx.x] = 0;
    if (len < 0 || all <= p.budget) {   // uniform: nothing to evict, the new rows' positions alone
        for (int r = len + tid; len >= 0 && r < n; r += NT)
            if ((uint32_t)table_entry(head.table, r >> head.shift) < (uint32_t)p.pages.n_pages) p.positions[head.at(r)] = (int32_t)((uint32_t)pos0 + (uint32_t)r);
        return;
    }
    int need = n - p.budget;
    const int64_t late = (int64_t)pos0 + n - p.window;   // positions from here on are kept ahead of all others
    bool absent = all > n;
    uint32_t lo = 0xFFFFFFFFu, hi = 0, low_lo = 0xFFFFFFFFu, low_hi = 0;   // the range of the keys, and of `low`
    uint32_t k_first = 0xFFFFFFFFu, l_first = 0xFFFFFFFFu;   // the thread's row that goes ahead of its others
    int r_first = -1;
    constexpr int AT_ONCE = 4;           // rows of a thread that are asked for together
    for (int base = 0; base < n; base += NT * AT_ONCE) {
        int page[AT_ONCE];
        int64_t at[AT_ONCE];
        float w[AT_ONCE];
        int32_t before[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) page[i] = table_entry(head.table, min(base + NT * i + tid, n - 1) >> head.shift);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int r = min(base + NT * i + tid, n - 1);
            const bool there = (uint32_t)page[i] < (uint32_t)p.pages.n_pages;
            absent = absent || !there;
            at[i] = (((int64_t)(there ? page[i] : 0) * head.hkv + h) << head.shift) + (r & ((1 << head.shift) - 1));
            w[i] = p.w[at[i]];
            before[i] = p.positions[at[i]];
            if (!there) at[i] = -1;
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int r = base + NT * i + tid;
            if (r >= n) continue;
            const int32_t position = r < len ? before[i] : (int32_t)((uint32_t)pos0 + (uint32_t)r);
            if (r >= len && at[i] >= 0) p.positions[at[i]] = position;
            const uint32_t key = p.window > 0 && position >= late ? 0xFFFFFFFFu : ordered(w[i]), low = ~((uint32_t)position ^ 0x80000000u);
            key_s[r] = key;
            low_s[r] = low;
            lo = min(lo, key);
            hi = max(hi, key);
            low_lo = min(low_lo, low);
            low_hi = max(low_hi, low);
            if (r_first < 0 || key < k_first || (key == k_first && low <= l_first)) {   // (of equal ones the higher row, which comes later)
                k_first = key;
                l_first = low;
                r_first = r;
            }
        }
    }
    if (__syncthreads_or(absent)) {
        if (tid == 0 && p.status) atomicOr(p.status, LEFT_OUT_ROW);
        return;
    }
    if (need == 1) {
        auto first = [&](uint32_t k1, uint32_t l1, int r1) {
            const bool take = r1 >= 0 && (r_first < 0 || k1 < k_first || (k1 == k_first && (l1 < l_first || (l1 == l_first && r1 > r_first))));
            k_first = take ? k1 : k_first;
            l_first = take ? l1 : l_first;
            r_first = take ? r1 : r_first;
        };
#pragma unroll
        for (int m = 1; m < 64; m *= 2) first(__shfl_xor(k_first, m), __shfl_xor(l_first, m), __shfl_xor(r_first, m));
        if (lane == 0) {
            best[0][wave] = k_first;
            best[1][wave] = l_first;
            best[2][wave] = (uint32_t)r_first;
        }
        __syncthreads();
        if (wave > 0) return;
        k_first = best[0][lane % WAVES];
        l_first = best[1][lane % WAVES];
        r_first = (int)best[2][lane % WAVES];
#pragma unroll
        for (int m = 1; m < WAVES; m *= 2) first(__shfl_xor(k_first, m), __shfl_xor(l_first, m), __shfl_xor(r_first, m));
        const int row = __builtin_amdgcn_readfirstlane(r_first);
        if (row >= p.budget) return;   // the last row: it lies behind the budget
        if (tid < p.D / 4) {
            const Move m{head.at(p.budget), head.at(row)};
            move_rows(p, [&](int64_t) { return m; }, 1, tid, p.D / 4);
        }
        return;
    }
    // the lowest and the highest over the workgroup
    auto range_of = [&](uint32_t &a, uint32_t &b, uint32_t (&of_waves)[2][WAVES]) {
        a = ~wave_max(~a);
        b = wave_max(b);
        if (lane == 0) {
            of_waves[0][wave] = a;
            of_waves[1][wave] = b;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            a = min(a, of_waves[0][w]);
            b = max(b, of_waves[1][w]);
        }
    };
    for (int i = tid; i < BINS; i += NT) hist[i] = 0;
    for (int i = tid; i < WORDS; i += NT) words[i] = 0;
    if (tid == 0) counted = 0;
    range_of(lo, hi, range_s[0]);
    range_of(low_lo, low_hi, range_s[1]);
    // Narrow down: of the rows whose value (the key; later, among those of key `equal`, low) lies in [lo, hi] the `need` first ones go; those below lo go, those
    // above hi stay
    bool by_low = false;
    uint32_t equal = 0, count = 0;
    auto inside = [&](int r) {
        const uint32_t v = by_low ? low_s[r] : key_s[r];
        return v >= lo && v <= hi && (!by_low || key_s[r] == equal);
    };
    for (;;) {
        const uint32_t span = hi - lo;
        const int down = span < BINS ? 0 : 32 - 11 - __builtin_clz(span);
#pragma unroll 4
        for (int r = tid; r < n; r += NT)
            if (inside(r)) atomicAdd(&hist[((by_low ? low_s[r] : key_s[r]) - lo) >> down], 1u);
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
        // many rows in one bin, often because they are alike: the range of what they hold
        uint32_t a = 0xFFFFFFFFu, b = 0;
        for (int r = tid; r < n; r += NT)
            if (inside(r)) {
                a = min(a, by_low ? low_s[r] : key_s[r]);
                b = max(b, by_low ? low_s[r] : key_s[r]);
            }
        range_of(a, b, range_s[2]);
        lo = a;
        hi = b;
        if (lo == hi) {
            if (by_low) break;   // alike in all but their rows
            by_low = true;
            equal = lo;
            lo = low_lo;
            hi = low_hi;
        }
        __syncthreads();
    }
    const bool whole = count == (uint32_t)need;   // uniform
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
    const bool ranked = !whole && count <= CANDIDATES;
    auto goes_first = [&](int r) { return by_low ? key_s[r] < equal || (key_s[r] == equal && low_s[r] < lo) : key_s[r] < lo; };
    for (int base = 0; base < n; base += NT) {
        const int r = base + tid;
        const bool in = r < n && inside(r);
        const uint64_t out = __builtin_amdgcn_ballot_w64(r < n && (goes_first(r) || (whole && in)));
        if (lane == 0) out_s[(base >> 6) + wave] = out;
        if (ranked && in) {   // a candidate (their order is of no consequence)
            const uint32_t c = atomicAdd(&counted, 1u);
            cand_key[c] = key_s[r];
            cand_low[c] = low_s[r];
            cand_row[c] = r;
        }
        if (!whole && !ranked) {
            const uint64_t same = __builtin_amdgcn_ballot_w64(in);
            if (lane == 0) words[(base >> 6) + wave] = (uint32_t)__popcll(same);
        }
    }
    auto goes = [&](int r) { atomicOr(reinterpret_cast<uint32_t *>(out_s) + (r >> 5), 1u << (r & 31)); };
    if (ranked) {
        __syncthreads();
        for (int c = wave; c < (int)count; c += WAVES) {   // a wave a candidate, against 64 others at a time
            const uint32_t k = cand_key[c], l = cand_low[c];
            const int r = cand_row[c];
            int rank = 0;
            for (int o0 = 0; o0 < (int)count; o0 += 64) {
                const int o = min(o0 + lane, CANDIDATES - 1);
                const uint32_t ko = cand_key[o], lw = cand_low[o];
                const int ro = cand_row[o];
                rank += __popcll(__builtin_amdgcn_ballot_w64(o0 + lane < (int)count && (ko < k || (ko == k && (lw < l || (lw == l && ro > r))))));
            }
            if (lane == 0 && rank < need) goes(r);
        }
    } else if (!whole) {
        // alike in all but their rows: the last `need` of them
        add_up();
        for (int base = 0; base < n; base += NT) {
            const int r = base + tid;
            const uint64_t same = __builtin_amdgcn_ballot_w64(r < n && inside(r));
            const int ahead = (int)words[(base >> 6) + wave] + __popcll(same & ((1ull << lane) - 1));
            if ((same >> lane & 1) && ahead >= (int)count - need) goes(r);
        }
    }
    __syncthreads();
    // evicted rows below the budget and kept ones behind it, counted in the order of the rows, a word of 64 a thread
    auto first_bits = [](int bits) { return bits <= 0 ? 0ull : bits >= 64 ? ~0ull : (1ull << bits) - 1; };
    auto holes_of = [&](int word) { return out_s[word] & first_bits(p.budget - 64 * word); };
    auto movers_of = [&](int word) { return ~out_s[word] & first_bits(n - 64 * word) & ~first_bits(p.budget - 64 * word); };
    for (int i = tid; i < WORDS; i += NT) words[i] = 64 * i < n ? (uint32_t)__popcll(holes_of(i)) << 16 | (uint32_t)__popcll(movers_of(i)) : 0u;
    add_up();
    const int count_moves = (int)(words[WORDS] & 0xFFFFu);
    const bool own = count_moves <= OWN_MOVES;   // uniform
    Move *to = own ? list : p.moves + (int64_t)blockIdx.x * p.most_moves;
    for (int base = 0; base < n; base += NT * AT_ONCE) {
        int page[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) page[i] = table_entry(head.table, min(base + NT * i + tid, n - 1) >> head.shift);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int r = base + NT * i + tid, word = ((base + NT * i) >> 6) + wave;
            if (64 * word >= n) break;   // uniform in the wave
            const uint64_t holes = holes_of(word), movers = movers_of(word), ahead = (1ull << lane) - 1;
            const uint32_t before = words[word];
            const int64_t at = (((int64_t)page[i] * head.hkv + h) << head.shift) + (r & ((1 << head.shift) - 1));
            if (holes >> lane & 1) to[(before >> 16) + __popcll(holes & ahead)].to = at;
            if (movers >> lane & 1) to[(before & 0xFFFFu) + __popcll(movers & ahead)].from = at;
        }
    }
    if (!own) {
        if (tid == 0) p.counts[blockIdx.x] = count_moves;
        return;
    }
    __syncthreads();
    move_rows(p, [&](int64_t i) { return list[i]; }, count_moves, tid, NT);
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
    const Move *moves = p.moves + (int64_t)blockIdx.x * p.most_moves;
    move_rows(p, [&](int64_t i) { return moves[i]; }, count, (int64_t)blockIdx.y * 256 + threadIdx.x, (int64_t)gridDim.y * 256);
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
    const bool in_lds = rows <= 16384;
    if (rows <= 1024) hipLaunchKernelGGL((evict_select_kernel<256, 1024>), dim3(heads), dim3(256), 0, s, p);
    else if (rows <= 4096) hipLaunchKernelGGL((evict_select_kernel<512, 4096>), dim3(heads), dim3(512), 0, s, p);
    else if (in_lds) hipLaunchKernelGGL((evict_select_kernel<1024, 16384>), dim3(heads), dim3(1024), 0, s, p);
    else hipLaunchKernelGGL(evict_select_long_kernel, dim3(heads), dim3(LNT), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.most_moves == 0 || (in_lds && p.most_moves <= OWN_MOVES)) return e;
    const unsigned parts = (unsigned)std::max<int64_t>(1, std::min<int64_t>(2048 / heads, ((int64_t)p.most_moves * (p.D / 4) + 255) / 256));
    hipLaunchKernelGGL(evict_move_kernel, dim3(heads, parts), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace kd
