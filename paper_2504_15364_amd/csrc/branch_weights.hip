// branch_weights: the attention weight that new tokens give to the own rows of their sequence.
//
//   w(r) <- decay w(r) [r held before the step] + sum over query rows of 2^(a - lse2),  a = scale log2(e) q.k_r,  lse2 = log2(e) lse(q)
//
// With the logarithms of the weight sums known there is one product and one exponential a pair and no second pass.  Two forms:
//   few   at most 32 query rows per (sequence, KV head), a generated token above all: the keys stream from memory once, tiles of 32 of them through
//         the registers of every wave; bound by that stream (2 D bytes a row and head)
//   many  keys stay in registers, 64 a wave and 512 a workgroup, and the query rows pass through LDS in tiles of 64; bound by the matrix pipe
//         (2 D operations a pair) and the exponentials (a quarter of the vector rate) side by side.  The pairs of (block of 512 keys, tile of 64 query rows) that
//         see one another form a list, heads outermost, of which every workgroup takes an equal part; sums of blocks that are cut are
//         joined by a second launch, in order.
// No atomics: every sum has one order.
#include <algorithm>

#include "kd_device.h"
#include "kd_pages.h"
#include "kd_select.h"

namespace kd {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float LOG2E = 1.4426950408889634f;

__device__ const u32x4 zeros[64] = {};   // what rows of pages that do not exist are read from

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// What takes part of a sequence: rows (n in all, `len` of them old) and the query rows of tokens j0 .. (rows of them)
struct Seq {
    int len, n, j0, rows;
};
__device__ __forceinline__ Seq sequence(const WeightsParams &p, int s)
{
    const int len = table_entry(p.pages.lens, s), fresh = new_rows(len, asked_rows(p.pages, p.Bt, s), p.Bt);
    if (fresh == 0) return Seq{0, 0, 0, 0};
    const int n = rows_with(p.pages, len, fresh), j0 = max(fresh - p.observe, 0);
    return Seq{min(len, n), n, j0, (fresh - j0) * p.G};
}
// The logarithm of a query's weight sum in log2 units, +inf where it gives no weight
__device__ __forceinline__ float in_log2(float lse) { return lse == -INFINITY ? INFINITY : lse * LOG2E; }

// ------------------------------------------------------------------ few query rows
constexpr int FW = 4;     // waves of a workgroup
constexpr int FK = 32;    // keys of a tile

template <int CTRL>
__device__ __forceinline__ float fetch(float x)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xF, 0xF, false));
}
// Eight numbers of each lane, summed over the 16 lanes of a row: lane u of the row gets the sum of number u / 2 (lane bits 3, 2 and 1 halve the numbers that
// a lane keeps; it hands the others to a partner on the other side of that bit)
__device__ __forceinline__ float row_sums8(const float (&v)[8], int u)
{
    float a[4], b[2];
    const bool b3 = u & 8, b2 = u & 4, b1 = u & 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = (b3 ? v[4 + i] : v[i]) + fetch<0x128>(b3 ? v[i] : v[4 + i]);   // row_ror:8
#pragma unroll
    for (int i = 0; i < 2; ++i) b[i] = (b2 ? a[2 + i] : a[i]) + fetch<0x141>(b2 ? a[i] : a[2 + i]);   // row_half_mirror
    const float c = (b1 ? b[1] : b[0]) + fetch<0x4E>(b1 ? b[0] : b[1]);                              // quad_perm [2,3,0,1]
    return c + fetch<0xB1>(c);                                                                       // quad_perm [1,0,3,2]
}

template <int D, int CB>
__global__ __launch_bounds__(64 * FW) void weights_few_kernel(WeightsParams p)
{
    constexpr int NC = D / 32;
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)blockIdx.x * FW + (int)(threadIdx.x >> 6)), waves = (int)gridDim.x * FW;
    const int shift = p.pages.page_shift;
    // the tiles of all (sequence, head) form one list, of which every wave takes a contiguous piece
    auto tiles_of = [&](int s) { return (sequence(p, s).n + FK - 1) / FK; };
    int total = 0;
    for (int base = 0; base < p.n_seqs; base += 64) {
        const int mine = base + lane < p.n_seqs ? tiles_of(base + lane) : 0;
        total += __builtin_amdgcn_readlane((int)wave_inclusive_scan((uint32_t)mine), 63);
    }
    total *= p.hkv;
    const int begin = (int)((int64_t)wave * total / waves), end = (int)((int64_t)(wave + 1) * total / waves);
    if (begin >= end) return;
    int s = 0, first = 0;
    for (int base = 0; base < p.n_seqs; base += 64) {
        const int mine = (base + lane < p.n_seqs ? tiles_of(base + lane) : 0) * p.hkv;
        const int upto = (int)wave_inclusive_scan((uint32_t)mine), all = __builtin_amdgcn_readlane(upto, 63);
        if (first + all > begin) {
            const int k = __builtin_ctzll(__builtin_amdgcn_ballot_w64(first + upto > begin));
            s = base + k;
            first += __builtin_amdgcn_readlane(upto, k) - __builtin_amdgcn_readlane(mine, k);
            break;
        }
        first += all;
    }
    Seq q = sequence(p, s);
    int nt = (q.n + FK - 1) / FK, h = (begin - first) / nt, t = begin - first - h * nt;
    bf16x8 qr[CB][NC];
    float lse2[CB];
    int vis[CB];
    u32x4 kr[2][NC];
    int page[4];
    auto open = [&]() {   // the queries of (s, h)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const int m = min(16 * cb + c16, q.rows - 1), jr = p.by_G.divide(m), hd = h * p.G + m - jr * p.G, j = q.j0 + jr;
            const uint16_t *at = p.q.p + (int64_t)s * p.q.seq + (int64_t)hd * p.q.head + (int64_t)j * p.q.token + 8 * g;
#pragma unroll
            for (int c = 0; c < NC; ++c) qr[cb][c] = as_bf16x8(*reinterpret_cast<const u32x4 *>(at + 32 * c));
            const float x = p.lse[((int64_t)s * p.hkv * p.G + hd) * p.Bt + j];
            lse2[cb] = 16 * cb + c16 < q.rows ? in_log2(x) : INFINITY;
            vis[cb] = q.len + j;   // the last row that the query sees
        }
    };
    // A tile's rows lie in groups of eight on one page each; rows behind the last one stand for it
    auto load = [&]() {
        const int32_t *table = p.pages.table + (int64_t)s * p.pages.width;
        const uint16_t *k8[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = min(t * FK + 8 * i, (q.n - 1) & ~7);
            page[i] = __builtin_amdgcn_readfirstlane(table_entry(table, row >> shift));
            const bool there = (uint32_t)page[i] < (uint32_t)p.pages.n_pages;
            if (!there) page[i] = -1;
            k8[i] = p.pages.k + ((((int64_t)(there ? page[i] : 0) * p.hkv + h) << shift) + (row & ((1 << shift) - 1))) * D;
        }
#pragma unroll
        for (int kg = 0; kg < 2; ++kg) {
            const uint16_t *kb = (c16 < 8 ? k8[2 * kg] : k8[2 * kg + 1]) + (min(t * FK + 16 * kg + c16, q.n - 1) & 7) * D + 8 * g;
#pragma unroll
            for (int c = 0; c < NC; ++c) kr[kg][c] = *reinterpret_cast<const u32x4 *>(kb + 32 * c);
        }
    };
    open();
    load();
    for (int at = begin; at < end; ++at) {
        // where the lane's sum goes: key 16 (u / 8) + 4 g + u / 2 % 4 of the tile
        const int u = c16, in_tile = 16 * (u >> 3) + 4 * g + (u >> 1 & 3), r = t * FK + in_tile, group = in_tile >> 3;
        const int pg = group == 0 ? page[0] : group == 1 ? page[1] : group == 2 ? page[2] : page[3];
        const bool mine = !(u & 1) && r < q.n && pg >= 0;
        float *wp = p.w + (((int64_t)max(pg, 0) * p.hkv + h) << shift) + (r & ((1 << shift) - 1));
        float old = 0.f;
        if (mine && r < q.len && p.decay != 0.f) old = p.decay * *wp;
        f32x4 sc[CB][2];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) sc[cb][0] = sc[cb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int kg = 0; kg < 2; ++kg)
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) sc[cb][kg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kr[kg][c]), qr[cb][c], sc[cb][kg], 0, 0, 0);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[cb][i >> 2][i & 3], p.scale_log2e, -lse2[cb]));
                v[i] += t * FK + 16 * (i >> 2) + 4 * g + (i & 3) <= vis[cb] ? e : 0.f;
            }
        }
        // the next tile's keys, as soon as this one's have been used
        if (at + 1 < end) {
            if (++t == nt) {
                t = 0;
                if (++h == p.hkv) {
                    h = 0;
                    do q = sequence(p, ++s);
                    while (q.n == 0);
                    nt = (q.n + FK - 1) / FK;
                }
                open();
            }
            load();
        }
        const float sum = row_sums8(v, u);
        if (mine) *wp = old + sum;
    }
}

// ------------------------------------------------------------------ many query rows
constexpr int NW = 8;              // waves of a workgroup, 64 keys each
constexpr int KB = 64 * NW;        // keys of a block
constexpr int QT = 64;             // query rows of a tile
constexpr int STAGES = 5;          // tiles of query rows in LDS.  (At the start the second half of the keys occupies the first four.)
constexpr int SUM_PITCH = 33;

// The blocks of a sequence: block k of KB keys is seen by the tiles from seen_from(k) on
struct Blocks {
    Seq q;
    int tiles, full, count, cost;   // tiles of query rows; blocks that all tiles see; blocks in all; pairs of both that see one another
};
__device__ __forceinline__ int seen_from(const WeightsParams &p, const Seq &q, int k) { return max(k * KB - q.len - q.j0, 0) * p.G / QT; }
__device__ __forceinline__ Blocks blocks_of(const WeightsParams &p, int s)
{
    Blocks b{sequence(p, s), 0, 0, 0, 0};
    if (b.q.n == 0) return b;
    b.tiles = (b.q.rows + QT - 1) / QT;
    b.count = (b.q.n + KB - 1) / KB;
    b.full = min((b.q.len + b.q.j0) / KB + 1, b.count);
    b.cost = b.full * b.tiles;
    for (int k = b.full; k < b.count; ++k) b.cost += b.tiles - seen_from(p, b.q, k);
    return b;
}
// Block and offset in it of pair `at` of a sequence
__device__ __forceinline__ int block_at(const WeightsParams &p, const Blocks &b, int at, int *offset)
{
    if (at < b.full * b.tiles) {
        const int k = at / b.tiles;
        *offset = at - k * b.tiles;
        return k;
    }
    at -= b.full * b.tiles;
    for (int k = b.full;; ++k) {
        const int cost = b.tiles - seen_from(p, b.q, k);
        if (at < cost) {
            *offset = at;
            return k;
        }
        at -= cost;
    }
}

struct Plan {
    int per_head, parts;
};
__device__ __forceinline__ int64_t part_begin(const WeightsParams &p, const Plan &plan, int w) { return (int64_t)w * plan.per_head * p.hkv / plan.parts; }
__device__ __forceinline__ int part_of(const WeightsParams &p, const Plan &plan, int64_t x) { return (int)(((x + 1) * plan.parts - 1) / ((int64_t)plan.per_head * p.hkv)); }
constexpr int MIN_TILES = 4;   // tiles a part at least, where there are more parts than blocks
__device__ __forceinline__ int parts_of(int64_t segments, int64_t total, int wgs)
{
    int64_t parts = segments <= wgs ? segments * (wgs / segments) : wgs;
    if (parts > segments) parts = total / MIN_TILES < parts ? (total / MIN_TILES > segments ? total / MIN_TILES : segments) : parts;
    return (int)parts;
}

template <int D>
struct Lds {
    static constexpr int ROWB = 2 * D, HALF = 32 * NW * ROWB, STAGE = QT * ROWB;
    static constexpr int RING = HALF, LSE = RING + STAGES * STAGE, BYTES = LSE + STAGES * QT * 4;
    static_assert(HALF <= (STAGES - 1) * STAGE && NW * 64 * SUM_PITCH * 4 <= LSE, "");
};

template <int N>
__device__ __forceinline__ void wait_copies()
{
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}
// Asynchronous copy of 4 bytes a lane: lane i to bytes [4 i, 4 i + 4) above lds_base
__device__ __forceinline__ void lds_copy4(uint32_t lds_base, const void *gaddr)
{
    const uint32_t base = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_base);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(base), "v"(gaddr) : "memory");
}

// Block k of sequence s and KV head h against the tiles [q0, q1) of its query rows.  part null: all tiles that see it, the weights are written
template <int D>
__device__ void weigh(const WeightsParams &p, unsigned char *smem, const Seq &sq, const int s, const int h, const int k, const int q0, const int q1, float *part)
{
    using L = Lds<D>;
    constexpr int UPR = D / 8, NC = D / 16, ROWB = 2 * D, RPL = 64 / UPR;
    constexpr int CPW = QT / RPL / NW, CPT = CPW + 1;   // copies of a wave for a tile: query rows, and the logarithms
    static_assert(CPW >= 1, "");
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hh = lane >> 5;
    const int shift = p.pages.page_shift, last = sq.n - 1, key0 = k * KB + 64 * wave;
    const int32_t *table = p.pages.table + (int64_t)s * p.pages.width;
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    const int ntl = q1 - q0;
    auto stage = [&](int i) { return (i + STAGES - 1) % STAGES; };   // of the i-th tile
    // tile q0 + i of query rows; rows behind the last one stand for it
    auto issue = [&](int i) {
        const uint32_t to = lds0 + L::RING + stage(i) * L::STAGE;
#pragma unroll
        for (int c = 0; c < CPW; ++c) {
            const int row = (wave + NW * c) * RPL + lane / UPR, m = min((q0 + i) * QT + row, sq.rows - 1), jr = p.by_G.divide(m);
            const uint16_t *at = p.q.p + (int64_t)s * p.q.seq + (int64_t)(h * p.G + m - jr * p.G) * p.q.head + (int64_t)(sq.j0 + jr) * p.q.token;
            lds_copy16(to + 1024u * (wave + NW * c), reinterpret_cast<const char *>(at) + ((lane % UPR) ^ (row & (UPR - 1))) * 16);
        }
        if (lane < QT / NW) {
            const int row = wave * (QT / NW) + lane, m = min((q0 + i) * QT + row, sq.rows - 1), jr = p.by_G.divide(m);
            lds_copy4(lds0 + L::LSE + stage(i) * QT * 4 + wave * (QT / NW) * 4, p.lse + ((int64_t)(s * p.hkv + h) * p.G + m - jr * p.G) * p.Bt + sq.j0 + jr);
        }
    };
    __syncthreads();   // nobody reads what the block before has left in LDS
    // the keys: rows of the wave, half in the place of four stages
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
        for (int i = 0; i < 32 / RPL; ++i) {
            const int in = RPL * i, row0 = min(key0 + 32 * kg + in, last & ~7), row = min(key0 + 32 * kg + in + lane / UPR, last);
            const int page = table_entry(table, min(key0 + 32 * kg + in, last) >> shift);
            const int64_t off = ((((int64_t)page * p.hkv + h) << shift) + (row & ((1 << shift) - 1))) * D;
            const char *at = (uint32_t)page < (uint32_t)p.pages.n_pages ? reinterpret_cast<const char *>(p.pages.k + off) : reinterpret_cast<const char *>(zeros);
            (void)row0;
            lds_copy16(lds0 + (kg ? L::RING : 0) + wave * 32 * ROWB + 1024u * i, at + ((lane % UPR) ^ ((in + lane / UPR) & (UPR - 1))) * 16);
        }
    issue(0);
    wait_copies<CPT>();
    bf16x8 kreg[2][NC];
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
        for (int c = 0; c < NC; ++c)
            kreg[kg][c] = as_bf16x8(*reinterpret_cast<const u32x4 *>(smem + (kg ? L::RING : 0) + (wave * 32 + l32) * ROWB + (((2 * c + hh) ^ (l32 & (UPR - 1))) * 16)));
    float acc[2][16];
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[kg][e] = 0.f;
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
        for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(kreg[kg][c]));   // (read by here)
    __syncthreads();
    if (ntl > 1) issue(1);
    if (ntl > 2) issue(2);
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < ntl; ++i) {
        if (i + 2 < ntl) wait_copies<2 * CPT>();
        else if (i + 1 < ntl) wait_copies<CPT>();
        else wait_copies<0>();
        __syncthreads();   // tile i is there, and every wave is through with tile i - 1
        if (i + 3 < ntl) issue(i + 3);
        const unsigned char *tq = smem + L::RING + stage(i) * L::STAGE;
        const float *tl = reinterpret_cast<const float *>(smem + L::LSE) + stage(i) * QT;
#pragma unroll
        for (int half = 0; half < QT / 32; ++half) {
            const int m = (q0 + i) * QT + 32 * half + l32;
            const float lse2 = m < sq.rows ? in_log2(tl[32 * half + l32]) : INFINITY;
            f32x16 sc[2];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const bf16x8 qf = as_bf16x8(*reinterpret_cast<const u32x4 *>(tq + (32 * half + l32) * ROWB + (((2 * c + hh) ^ (l32 & (UPR - 1))) * 16)));
#pragma unroll
                for (int kg = 0; kg < 2; ++kg) sc[kg] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kreg[kg][c], qf, c == 0 ? zero : sc[kg], 0, 0, 0);
            }
            // rows that not every query of the tile sees (uniform)
            const int seen = sq.len + sq.j0 + p.by_G.divide(min((q0 + i) * QT + 32 * half, sq.rows - 1));
            if (key0 + 63 > seen) {
                const int lim = sq.len + sq.j0 + p.by_G.divide(min(m, sq.rows - 1)) - key0 - 4 * hh;
#pragma unroll
                for (int kg = 0; kg < 2; ++kg)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[kg][e] = 32 * kg + 8 * (e >> 2) + (e & 3) <= lim ? sc[kg][e] : -INFINITY;
            }
#pragma unroll
            for (int kg = 0; kg < 2; ++kg)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[kg][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kg][e], p.scale_log2e, -lse2));
        }
    }
    // the sums over the lanes of a row of keys, turned in LDS: lane i gets key i
    __syncthreads();
    float *turn = reinterpret_cast<float *>(smem) + wave * 64 * SUM_PITCH;
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
        for (int e = 0; e < 16; ++e) turn[(32 * kg + 8 * (e >> 2) + 4 * hh + (e & 3)) * SUM_PITCH + l32] = acc[kg][e];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        const float *t = turn + lane * SUM_PITCH + i;
        sum += (t[0] + t[1]) + (t[2] + t[3]);
    }
    if (part) {
        part[64 * wave + lane] = sum;
        return;
    }
    const int r = key0 + lane;
    if (r > last) return;
    const int page = table_entry(table, r >> shift);
    if ((uint32_t)page >= (uint32_t)p.pages.n_pages) return;
    float *w = p.w + (((int64_t)page * p.hkv + h) << shift) + (r & ((1 << shift) - 1));
    *w = (r < sq.len && p.decay != 0.f ? p.decay * *w : 0.f) + sum;
}

struct Place {
    int h, s, k, t, left, second;   // tile t (of those that see it) of block k of sequence s; `left` pairs; second: the part has been at another block before
};

template <int D>
__global__ __launch_bounds__(64 * NW) void weights_many_kernel(WeightsParams)
{
    const WeightsParams &p = argument_at<WeightsParams>(0);   // (read where it is needed)
    __shared__ __attribute__((aligned(1024))) unsigned char smem[Lds<D>::BYTES];
    __shared__ uint32_t wave_tot[2][NW];
    __shared__ Place place;
    const int tid = threadIdx.x, wgs = (int)gridDim.x;
    const int wg = wgs % 8 == 0 ? (int)blockIdx.x % 8 * (wgs / 8) + (int)blockIdx.x / 8 : (int)blockIdx.x;   // neighbouring parts on one XCD
    const int each = (p.n_seqs + 64 * NW - 1) / (64 * NW), first = tid * each;
    int mine = 0, used = 0;
    for (int i = 0; i < each; ++i)
        if (first + i < p.n_seqs) {
            const Blocks b = blocks_of(p, first + i);
            mine += b.cost;
            used += b.count;
        }
    uint32_t total, segments;
    const int before = (int)block_exclusive_scan_t<64 * NW, uint32_t>((uint32_t)mine, wave_tot[0], &total);
    (void)block_exclusive_scan_t<64 * NW, uint32_t>((uint32_t)used, wave_tot[1], &segments);
    if (blockIdx.x == 0) {   // for the join
        int at = before;
        for (int i = 0; i < each; ++i)
            if (first + i < p.n_seqs) {
                p.plan[WEIGHTS_PLAN_WORDS + first + i] = at;
                at += blocks_of(p, first + i).cost;
            }
    }
    Plan plan{(int)total, 1};
    if (total) plan.parts = parts_of((int64_t)segments * p.hkv, (int64_t)total * p.hkv, wgs);
    if (blockIdx.x == 0 && tid == 0) {
        p.plan[0] = plan.per_head;
        p.plan[1] = plan.parts;
    }
    if (wg >= plan.parts || total == 0) return;
    {
        const int64_t begin = part_begin(p, plan, wg);
        const int h = (int)(begin / plan.per_head), from = (int)(begin - (int64_t)h * plan.per_head);
        if (from >= before && from < before + mine) {   // one thread's
            int at = before, s = first, t;
            Blocks b = blocks_of(p, s);
            while (from >= at + b.cost) {
                at += b.cost;
                b = blocks_of(p, ++s);
            }
            const int k = block_at(p, b, from - at, &t);
            place = Place{h, s, k, t, (int)(part_begin(p, plan, wg + 1) - begin), 0};
        }
    }
    __syncthreads();
    for (;;) {   // (where the part goes on is kept in LDS, not in scalar registers)
        const int h = __builtin_amdgcn_readfirstlane(place.h), s = __builtin_amdgcn_readfirstlane(place.s), k = __builtin_amdgcn_readfirstlane(place.k);
        const int t = __builtin_amdgcn_readfirstlane(place.t), left = __builtin_amdgcn_readfirstlane(place.left), second = __builtin_amdgcn_readfirstlane(place.second);
        if (left == 0) return;   // uniform
        const Seq sq = sequence(p, s);
        const int from = sq.n ? seen_from(p, sq, k) : 0, cost = sq.n ? (sq.rows + QT - 1) / QT - from : 0, take = min(cost - t, left);
        __syncthreads();
        if (tid == 0) {
            Place next{h, s, k + 1, 0, left - take, second | (take > 0)};
            if ((int64_t)(k + 1) * KB >= sq.n) next = s + 1 == p.n_seqs ? Place{h + 1, 0, 0, 0, next.left, next.second} : Place{h, s + 1, 0, 0, next.left, next.second};
            place = next;
        }
        if (take > 0) weigh<D>(p, smem, sq, s, h, k, from + t, from + t + take, take == cost ? nullptr : p.part + (int64_t)(2 * wg + second) * KB);
        __syncthreads();
    }
}

// The sums of the blocks that were cut: workgroup i those of the block whose first border inside it is that of the parts i and i + 1
__global__ __launch_bounds__(KB) void weights_join_kernel(WeightsParams p)
{
    __shared__ int where[3];
    const Plan plan{p.plan[0], p.plan[1]};
    const int w = (int)blockIdx.x + 1;
    if (w >= plan.parts) return;
    const int64_t x = part_begin(p, plan, w);
    const int h = (int)(x / plan.per_head), from = (int)(x - (int64_t)h * plan.per_head);
    for (int s = threadIdx.x; s < p.n_seqs; s += KB) {
        const int at = p.plan[WEIGHTS_PLAN_WORDS + s];
        if (from < at) continue;
        const Blocks b = blocks_of(p, s);
        if (from < at + b.cost) {   // one thread's
            where[0] = s;
            where[1] = block_at(p, b, from - at, &where[2]);
        }
    }
    __syncthreads();
    const int s = __builtin_amdgcn_readfirstlane(where[0]), k = __builtin_amdgcn_readfirstlane(where[1]), off = __builtin_amdgcn_readfirstlane(where[2]);
    const int64_t x0 = x - off, before = part_begin(p, plan, w - 1);
    if (off == 0 || before > x0) return;   // no block is cut here, or an earlier border inside it is the first
    const Seq sq = sequence(p, s);
    const int cost = (sq.rows + QT - 1) / QT - seen_from(p, sq, k), end = part_of(p, plan, x0 + cost - 1), r = k * KB + (int)threadIdx.x;
    if (r >= sq.n) return;
    float sum = p.part[(int64_t)(2 * (w - 1) + (before != x0)) * KB + threadIdx.x];
    for (int i = w; i <= end; ++i) sum += p.part[(int64_t)2 * i * KB + threadIdx.x];
    const int page = table_entry(p.pages.table + (int64_t)s * p.pages.width, r >> p.pages.page_shift);
    if ((uint32_t)page >= (uint32_t)p.pages.n_pages) return;
    float *wp = p.w + (((int64_t)page * p.hkv + h) << p.pages.page_shift) + (r & ((1 << p.pages.page_shift) - 1));
    *wp = (r < sq.len && p.decay != 0.f ? p.decay * *wp : 0.f) + sum;
}

bool few(int G, int observe) { return (int64_t)G * observe <= 32; }

template <int D>
hipError_t launch(const WeightsParams &p, hipStream_t s)
{
    if (few(p.G, p.observe)) {
        const unsigned wgs = (unsigned)p.cus * 4;
        if (p.G * p.observe <= 16) hipLaunchKernelGGL((weights_few_kernel<D, 1>), dim3(wgs), dim3(64 * FW), 0, s, p);
        else hipLaunchKernelGGL((weights_few_kernel<D, 2>), dim3(wgs), dim3(64 * FW), 0, s, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((weights_many_kernel<D>), dim3(p.cus), dim3(64 * NW), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(weights_join_kernel, dim3(p.cus - 1), dim3(KB), 0, s, p);
    return hipGetLastError();
}

}  // namespace

size_t weights_workspace(int n_seqs, int G, int Bt, int observe, int cus, size_t *off_plan)
{
    const int tokens = observe > 0 && observe < Bt ? observe : Bt;
    *off_plan = few(G, tokens) ? 0 : (size_t)2 * cus * KB * 4;
    return (*off_plan + (size_t)(WEIGHTS_PLAN_WORDS + n_seqs) * 4 + 255) & ~(size_t)255;
}

hipError_t launch_branch_weights(WeightsParams p, hipStream_t s)
{
    p.by_G.set((uint32_t)p.G);
    p.by_hkv.set((uint32_t)p.hkv);
    return p.D == 128 ? launch<128>(p, s) : p.D == 64 ? launch<64>(p, s) : hipErrorInvalidValue;
}

}  // namespace kd
