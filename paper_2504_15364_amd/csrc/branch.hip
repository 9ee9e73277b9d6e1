// branch_attention: the new tokens of sequences that continue the same prompts attend to the rows of their prompt's cache and to
// the rows in pages of their own.
//
//   o = sum_i 2^(a_i - m) v_i / sum_i 2^(a_i - m),  a_i = scale log2(e) q.k_i,  i over the N rows of the prompt and the
//   sequence's own rows up to the token itself; each wave keeps the running m, sum and output of its keys, and a second
//   launch joins the pieces of a row: with (m_w, l_w, o_w) of piece w, o = sum_w l_w 2^(m_w - m) o_w / sum_w l_w 2^(m_w - m).
//
// The queries of all sequences of a prompt that read the same KV head are rows of ONE product with the prompt's rows (fan x G x Bt
// rows), so these are read once, not once a sequence.  What bounds it: the stream of K and V, the prompt's rows once and every
// sequence's own rows once (4 D bytes a row and KV head); with hundreds of sequences the matrix cores on the shared part.
//
// Both parts are cut into tiles of 32 keys, and the chip's workgroups, one per compute unit, are dealt to the two parts by what their
// tiles take (make_plan, on every wave alike):
//   shared part  every (prompt, head, block of rows) segment is cut into as many pieces as workgroups are left to it; a workgroup takes
//                every splits-th tile (or group of tiles) of a segment, joins its waves' results in LDS and stores one partial
//   own part     the tiles of all (sequence, head, block of rows) segments form one list, of which every wave takes a
//                contiguous piece and stores a partial where the piece leaves a segment: no wave waits for another one, and
//                ragged lengths cost nothing, because the list is cut by tiles and not by sequences
// All of this follows from the lengths on the device: the launch itself does not depend on them and may be replayed from a graph.
// Where the prompts' rows and those that the tables can name are few, one launch does it, a workgroup a segment (one_launch).
// Measured (8192 shared rows, 8 KV heads of 128, both launches, back to back): one sequence 14.4 us (35 MB), 16 with up to 777 own rows 20.6
// (60 MB), 64 with up to 4096 own rows 112 (571 MB: 5.1 TB/s; its first launch alone 5.4), 256 of three query heads to a KV head with up to 33 own
// rows 57 (26 GFLOP).
#include <algorithm>

#include "kd_branch.h"
#include "kd_device.h"
#include "kd_select.h"

namespace kd {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int NW = 8;                 // waves of a workgroup
constexpr int TK = 32;                // keys of a tile
// The reference of a row's weights is put 2^LIFT above the largest logit seen and moves when one exceeds it by 2^SLACK: moving it costs a pass
// over the outputs, and with 2^16 between the two it hardly ever does.  A weight is 2^SLACK at most, so sums over the 2^24 rows that
// a prompt and a table of 2^23 each can hold stay below 2^127 with values of 2^100.
constexpr float LIFT = 13.f, SLACK = 3.f;

// max and sum over the four 16-lane rows of a wave, position by position (every lane gets it)
__device__ __forceinline__ float max_over_rows(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_rows(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// What a piece of a row leaves for the join: its reference and weight sum.  A reference of -inf stands for a piece without a key, which the join
// skips; one whose logits are all NaN has none either, and its NaN must not be lost.
__device__ __forceinline__ float2 piece_ml(float m, float L) { return make_float2(L == L ? m : 0.f, L); }
// Natural logarithm of a row's weight sum, -inf where it has seen no key
__device__ __forceinline__ float log_sum(float m, float L) { return L == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(L)) * 0.6931471805599453f; }
// New tokens of a sequence that holds `len` rows, and rows that are keys of theirs (its own and the new ones); 0 where it has nothing to do
__device__ __forceinline__ int new_of(const BranchParams &p, int len, int asked) { return len < 0 ? 0 : max(0, min(asked, p.Bt)); }
__device__ __forceinline__ int own_rows(const BranchParams &p, int len, int asked)
{
    const int fresh = new_of(p, len, asked);
    if (fresh == 0) return 0;
    const int64_t n = (int64_t)len + fresh, most = (int64_t)p.pages.width << p.pages.page_shift;
    return (int)(n < most ? n : most);
}
__device__ __forceinline__ int asked_of(const BranchParams &p, int s) { return p.pages.n_new ? p.pages.n_new[s] : p.Bt; }
__device__ __forceinline__ int own_rows(const BranchParams &p, int s) { return own_rows(p, p.pages.lens[s], asked_of(p, s)); }

// How the work is cut (uniform; the merge reads it from BranchParams::plan)
struct Plan {
    int shared_wgs;                // workgroups of the shared part; task t of its list is done by workgroup t % shared_wgs
    int splits;                    // pieces of each of its segments (prompt, head, block of rows): piece k of segment g is task k segs + g
    int own_tiles, own_chunk;      // tiles of the own part; how many of them a wave takes
};

// One wave's state of a block of 16 x CB query rows: column c16 of block cb is query row 16 cb + c16
template <int D, int CB>
struct State {
    f32x4 o[CB][D / 16];   // element i of block db: column 16 db + 4 g + i of the output
    float l[CB], m[CB];    // weight sum of the lane's own keys; reference (log2 units), the same in the four lanes of a row
    bf16x8 q[CB][D / 32];

    __device__ __forceinline__ void reset()
    {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
            for (int db = 0; db < D / 16; ++db) o[cb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            l[cb] = 0.f;
            m[cb] = -INFINITY;
        }
    }
};

// 16-byte units of a V row in LDS are permuted so that what a transposing read gathers lies in different banks, those of a K row so
// that the 16 rows of an operand read do
template <int D>
__device__ __forceinline__ int v_swizzle(int row)
{
    constexpr int UPR = D / 8, VSW = UPR / 4;
    return UPR == 16 ? (VSW * (row & 3)) ^ (2 * ((row >> 2) & 1)) : VSW * (row & 3);
}
template <int D>
__device__ __forceinline__ int k_swizzle(int row)
{
    return D == 128 ? row & 15 : (row >> 1) & 7;
}

// A tile of 32 keys in three steps.
// Logits S^T = K Q^T: element i of s[cb][kg] is key 16 kg + 4 g + i of query row 16 cb + c16; key(kg, c) gives chunk c (32 columns) of the
// lane's row of key group kg as an operand.
template <int D, int CB, class Key>
__device__ __forceinline__ void tile_logits(const State<D, CB> &st, f32x4 (&s)[CB][2], Key key)
{
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) s[cb][0] = s[cb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int kg = 0; kg < 2; ++kg) {
            const bf16x8 k = key(kg, c);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) s[cb][kg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, st.q[cb][c], s[cb][kg], 0, 0, 0);
        }
}

__device__ __forceinline__ float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }   // (fmaxf would quiet both first)

// Weights 2^(s - m) of one block of rows.  They go into the second product as two bf16 numbers, the upper half of the float and the
// rest (16 bits in all): rounded to one, their error alone would be as large as the output's own rounding.
template <int D, int CB>
__device__ __forceinline__ void tile_weights(State<D, CB> &st, const f32x4 (&s)[2], int cb, float scale_log2e, bf16x8 &ph, bf16x8 &pl)
{
    const float top = max2(max2(max2(s[0][0], s[0][1]), max2(s[0][2], s[0][3])), max2(max2(s[1][0], s[1][1]), max2(s[1][2], s[1][3])));
    if (__builtin_amdgcn_ballot_w64(top * scale_log2e > st.m[cb] + SLACK) != 0) {   // rare: the reference moves
        const float mx = max_over_rows(top) * scale_log2e;
        const bool need = mx > st.m[cb] + SLACK;
        const float alpha = need ? __builtin_amdgcn_exp2f(st.m[cb] - (mx + LIFT)) : 1.f;
        st.m[cb] = need ? mx + LIFT : st.m[cb];
        st.l[cb] *= alpha;
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.o[cb][db][i] *= alpha;
    }
    const float nm = st.m[cb] == -INFINITY ? 0.f : -st.m[cb];
    uint32_t w[8];
    u32x4 hi;
    float l[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(__builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][i % 4], scale_log2e, nm)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        l[i] = __uint_as_float(w[2 * i]) + __uint_as_float(w[2 * i + 1]);
        hi[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302);   // upper halves of both
        pl[2 * i] = (__bf16)(__uint_as_float(w[2 * i]) - __uint_as_float(w[2 * i] & 0xFFFF0000u));
        pl[2 * i + 1] = (__bf16)(__uint_as_float(w[2 * i + 1]) - __uint_as_float(w[2 * i + 1] & 0xFFFF0000u));
    }
    ph = __builtin_bit_cast(bf16x8, hi);
    st.l[cb] += (l[0] + l[1]) + (l[2] + l[3]);
}

// Outputs O^T += V^T P^T: the keys are enumerated in accumulator order (k-slot 8 g + i is key 4 g + i for i < 4 and 16 + 4 g + i - 4
// otherwise), and two transposing reads fetch exactly those.
template <int D>
__device__ __forceinline__ bf16x8 value_operand(const unsigned char *vt, int lane, int db)
{
    const int c16 = lane & 15, g = lane >> 4;
    const int rd_row = 4 * g + (c16 >> 2), rd_unit = ((c16 & 3) >> 1) ^ v_swizzle<D>(rd_row);   // (rows + 16 have the same swizzle)
    const unsigned char *ap = vt + rd_row * (2 * D) + (c16 & 1) * 8 + (((2 * db) ^ rd_unit) * 16);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)(ap));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)(ap + 16 * (2 * D)));
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <int D, int CB>
__device__ __forceinline__ void tile_outputs(State<D, CB> &st, int db, bf16x8 va, const bf16x8 (&ph)[CB], const bf16x8 (&pl)[CB])
{
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) st.o[cb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, ph[cb], st.o[cb][db], 0, 0, 0);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) st.o[cb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pl[cb], st.o[cb][db], 0, 0, 0);
}

// The three in turn; `between` runs once the keys have been used, `mask(s)` sets logits that are not seen to -inf.
template <int D, int CB, class Key, class Between, class Mask>
__device__ __forceinline__ void tile_step(State<D, CB> &st, const unsigned char *vt, float scale_log2e, int lane, Key key, Between between, Mask mask)
{
    f32x4 s[CB][2];
    tile_logits<D, CB>(st, s, key);
    between();
    mask(s);
    bf16x8 ph[CB], pl[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) tile_weights<D, CB>(st, s[cb], cb, scale_log2e, ph[cb], pl[cb]);
#pragma unroll
    for (int db = 0; db < D / 16; ++db) tile_outputs<D, CB>(st, db, value_operand<D>(vt, lane, db), ph, pl);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Logits of keys from `seen` on (counted from the tile's first) to -inf
template <int CB>
__device__ __forceinline__ void hide_from(f32x4 (&s)[CB][2], int seen, int g)
{
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int kg = 0; kg < 2; ++kg)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[cb][kg][i] = 16 * kg + 4 * g + i < seen ? s[cb][kg][i] : -INFINITY;
}

// A V tile from registers to the wave's own piece of LDS
template <int D>
__device__ __forceinline__ void store_v(unsigned char *vt, const u32x4 (&vr)[TK * D / 512], int lane)
{
    constexpr int UPR = D / 8, ROWB = D * 2, RPL = 64 / UPR, NV = TK / RPL;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int row = lane / UPR + RPL * i;
        *reinterpret_cast<u32x4 *>(vt + row * ROWB + (((lane % UPR) ^ v_swizzle<D>(row)) * 16)) = vr[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Address of query row m (order g, j) of sequence s and KV head h
__device__ __forceinline__ const uint16_t *query_row(const BranchParams &p, int s, int h, int m)
{
    const int g = p.by_Bt.divide(m), j = m - g * p.Bt;
    return p.q.p + (int64_t)s * p.q.seq + (int64_t)(h * p.G + g) * p.q.head + (int64_t)j * p.q.token;
}

// A task of the shared part: piece k of segment (prompt c, head h, block mb of rows).  Blocks of the same rows of the cache lie n_prefixes
// hkv tasks apart: with eight KV heads on the same XCD, whose L2 then serves all but one of them.
struct Segment {
    int ch, mb, c, h, k;
};
__device__ __forceinline__ Segment segment_of(const BranchParams &p, int task)
{
    Segment s;
    s.k = p.by_segs.divide(task);
    const int g = task - s.k * p.shared_segs;
    s.mb = p.by_heads.divide(g);
    s.ch = g - s.mb * p.n_prefixes * p.hkv;
    s.c = p.by_hkv.divide(s.ch);
    s.h = s.ch - s.c * p.hkv;
    return s;
}

// Floats from one row of a wave's outputs in LDS to the next: four more than the row, so that the 16 rows that a store touches lie in
// different banks (without them such a store took sixteen turns, and the join of the eight waves 5.6 us)
template <int D>
constexpr int OUT_PITCH = D + 4;

// The eight waves' results of 16 rows, in LDS, become one: store(row, column, four columns of its output, reference maximum, weight sum)
template <int D, class Store>
__device__ __forceinline__ void join_waves(const float *outs, const float2 (&ml_s)[NW][16], int rows, int tid, Store store)
{
    for (int it = tid; it < rows * (D / 4); it += 64 * NW) {
        const int m = it / (D / 4), d0 = it % (D / 4) * 4;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) mx = fmaxf(mx, ml_s[w][m].x);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        float L = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float2 ml = ml_s[w][m];
            const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - mx);
            const f32x4 o = *reinterpret_cast<const f32x4 *>(outs + ((size_t)w * 16 + m) * OUT_PITCH<D> + d0);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += f * o[i];
            L += f * ml.y;
        }
        const float inv = L > 0.f ? 1.f / L : 0.f;   // (no key seen: zero)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] *= inv;
        store(m, d0, acc, mx, L);
    }
}

// The shared part in blocks of 16 query rows: a workgroup its piece of a segment, every wave tiles of its own
template <int D>
__device__ void shared_few(const BranchParams &p, const Plan &plan, unsigned char *smem)
{
    constexpr int NC = D / 32, NDB = D / 16, UPR = D / 8, ROWB = D * 2, RPL = 64 / UPR, NV = TK / RPL, R = 16;
    __shared__ float2 ml_s[NW][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const int Mt = p.G * p.Bt, M = p.fan * Mt, nt = (p.prefix_len + TK - 1) / TK;
    unsigned char *vt = smem + (size_t)wave * TK * ROWB;
    float *outs = reinterpret_cast<float *>(smem);   // the waves' outputs of one block of 16 rows, where their V tiles were
    for (int task = blockIdx.x; task < p.shared_segs * plan.splits; task += plan.shared_wgs) {
        const Segment sg = segment_of(p, task);
        const int ch = sg.ch, mb = sg.mb, c = sg.c, h = sg.h, stride = plan.splits * NW;
        const uint16_t *kh = p.k_prefix + (size_t)ch * p.prefix_cap * D, *vh = p.v_prefix + (size_t)ch * p.prefix_cap * D;
        State<D, 1> st;
        st.reset();
        u32x4 kr[2][NC], vr[NV];
        // rows past the last repeat it: finite data whose weights are masked to zero.  (Offsets of 32 bits from the head's first row.)
        auto load_k = [&](int t) {
#pragma unroll
            for (int kg = 0; kg < 2; ++kg) {
                const uint32_t off = (uint32_t)min(t * TK + 16 * kg + c16, p.prefix_len - 1) * ROWB + 16 * g;
#pragma unroll
                for (int cc = 0; cc < NC; ++cc) kr[kg][cc] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(kh) + off + cc * 64);
            }
        };
        auto load_v = [&](int t) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t off = (uint32_t)min(t * TK + i * RPL + lane / UPR, p.prefix_len - 1) * ROWB + lane % UPR * 16;
                vr[i] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(vh) + off);
            }
        };
        int t = sg.k * NW + wave;
        load_k(t);   // (a tile behind the last repeats rows that exist)
        load_v(t);
        const int m = min(mb * R + c16, M - 1);
        const int f = p.by_Mt.divide(m);
        const uint16_t *qr = query_row(p, c * p.fan + f, h, m - f * Mt) + 8 * g;
#pragma unroll
        for (int cc = 0; cc < NC; ++cc) st.q[0][cc] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qr + cc * 32));
        for (; t < nt; t += stride) {
            store_v<D>(vt, vr, lane);
            tile_step<D, 1>(
                st, vt, p.scale_log2e, lane, [&](int kg, int cc) { return __builtin_bit_cast(bf16x8, kr[kg][cc]); },
                [&]() {
                    if (t + stride < nt) {
                        load_k(t + stride);
                        load_v(t + stride);
                    }
                },
                [&](f32x4 (&s)[1][2]) {
                    if ((t + 1) * TK > p.prefix_len) hide_from<1>(s, p.prefix_len - t * TK, g);   // uniform
                });
        }
        // the eight results become one
        const size_t slot = task;
        const float l = sum_over_rows(st.l[0]);
        __syncthreads();
        float *ow = outs + (size_t)wave * 16 * OUT_PITCH<D>;
#pragma unroll
        for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4 *>(ow + c16 * OUT_PITCH<D> + 16 * db + 4 * g) = st.o[0][db];
        if (g == 0) ml_s[wave][c16] = make_float2(st.m[0], l);
        __syncthreads();
        join_waves<D>(outs, ml_s, min(16, M - mb * R), tid, [&](int row, int d0, f32x4 acc, float mx, float L) {
            *reinterpret_cast<f32x4 *>(p.part_o + (slot * R + row) * D + d0) = acc;
            if (d0 == 0) p.part_ml[slot * R + row] = piece_ml(mx, L);
        });
        __syncthreads();   // the outputs are read before the next segment's V tiles overwrite them
    }
}

template <int N>
__device__ __forceinline__ void wait_copies()   // at most N of this wave's copies still in flight
{
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

// LDS of the shared part with many query rows: a ring of stages, each a tile of K and V for every group of waves
template <int D, int RW>
constexpr int stage_bytes() { return NW / RW * 2 * TK * D * 2; }
constexpr int stages_of(int RW) { return RW; }

// The shared part with 32 RW query rows (RW 2, 4 or 8) a workgroup: RW waves of 32 rows each work on the same tile, NW / RW groups of
// them on different tiles.  The tiles come into LDS once for all waves, by asynchronous copies (no registers) that run ahead of
// their use through a ring.  Where every wave read its own keys, 256 sequences of three query heads to a KV
// head read the shared rows 24 times, and of that traffic, 5.7 TB/s past the L2s, came all the time: 120 us.
// RW 4 and 8: the two waves of a SIMD take turns.  One is on the matrix pipe (outputs of the tile before, logits of this one) while the
// other forms its weights on the vector ALU, and barriers keep them half a step apart: in step with one another both want the same
// pipe at the same time, and a tile took 1.6 us where the longer of the two pipes needs 0.7.
template <int D, int RW>
__device__ void shared_many(const BranchParams &p, const Plan &plan, unsigned char *smem)
{
    constexpr int NC = D / 32, NDB = D / 16, UPR = D / 8, ROWB = D * 2, R = 32 * RW, KW = NW / RW, CB = 2;
    constexpr int TILEB = TK * ROWB, STAGEB = stage_bytes<D, RW>(), NS = stages_of(RW);
    constexpr int RPC = 1024 / ROWB, CPT = TILEB / 1024;   // rows of a copy (64 lanes x 16 bytes), copies of a tile
    constexpr int CPW = KW * 2 * CPT / NW;                 // copies of a stage a wave issues
    static_assert(KW * 2 * CPT % NW == 0 && CPW >= 1, "the copies of a stage are dealt evenly");
    __shared__ float2 ml_s[NW][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4, rw = wave % RW, kw = wave / RW;
    const int Mt = p.G * p.Bt, M = p.fan * Mt, nt = (p.prefix_len + TK - 1) / TK, units = (nt + KW - 1) / KW;
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    for (int task = blockIdx.x; task < p.shared_segs * plan.splits; task += plan.shared_wgs) {
        const Segment sg = segment_of(p, task);
        const int ch = sg.ch, mb = sg.mb, c = sg.c, h = sg.h;
        const uint16_t *kh = p.k_prefix + (size_t)ch * p.prefix_cap * D, *vh = p.v_prefix + (size_t)ch * p.prefix_cap * D;
        const int m0 = mb * R + 32 * rw;   // the wave's first query row
        const bool active = m0 < M;        // uniform in the wave: else it only copies
        // stage `it` of the piece (one behind its end repeats rows that exist: what a wave waits for stays the same number of copies)
        auto issue = [&](int it) {
#pragma unroll
            for (int i = 0; i < CPW; ++i) {
                const int id = wave + NW * i, grp = id / (2 * CPT), part = id % (2 * CPT), isv = part >= CPT, r0 = part % CPT * RPC;
                const int row = r0 + lane / UPR, unit = lane % UPR;
                const int key = min(((sg.k + it * plan.splits) * KW + grp) * TK + row, p.prefix_len - 1);
                const uint32_t off = (uint32_t)key * ROWB + (uint32_t)(unit ^ (isv ? v_swizzle<D>(row) : k_swizzle<D>(row))) * 16;
                lds_copy16(lds0 + (uint32_t)((it % NS) * STAGEB + grp * 2 * TILEB + isv * TILEB + r0 * ROWB), isv ? vh : kh, off);
            }
        };
        // The query rows are requested ahead of the first copies, and waited for ahead of the loop: where the compiler finds them used it
        // would wait in every step, and with them for all copies, which it does not count.
        State<D, CB> st;
        st.reset();
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const int m = min(m0 + 16 * cb + c16, M - 1);
            const int f = p.by_Mt.divide(m);
            const uint16_t *qr = query_row(p, c * p.fan + f, h, m - f * Mt) + 8 * g;
#pragma unroll
            for (int cc = 0; cc < NC; ++cc) st.q[cb][cc] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qr + cc * 32));
        }
        issue(0);
        const int steps = (units - sg.k + plan.splits - 1) / plan.splits;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int cc = 0; cc < NC; ++cc) asm volatile("" : "+v"(st.q[cb][cc]));
        auto key_operand = [&](const unsigned char *kt, int kg, int cc) {
            const int row = 16 * kg + c16;
            return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(kt + row * ROWB + (((4 * cc + g) ^ k_swizzle<D>(row)) * 16)));
        };
        auto tile_of = [&](int it) { return (sg.k + it * plan.splits) * KW + kw; };
        auto lds_of = [&](int it) { return smem + (it % NS) * STAGEB + kw * 2 * TILEB; };
        if constexpr (RW == 2) {
#pragma unroll
            for (int it = 1; it < NS - 1; ++it) issue(it);
            for (int it = 0; it < steps; ++it) {
                wait_copies<CPW *(NS - 2)>();   // this wave's part of stage `it` has landed
                __syncthreads();                // ... and every wave's, and nobody reads the stage before it any more
                issue(it + NS - 1);
                const int t = tile_of(it);
                if (!active || t >= nt) continue;   // uniform in the wave
                const unsigned char *kt = lds_of(it);
                tile_step<D, CB>(
                    st, kt + TILEB, p.scale_log2e, lane, [&](int kg, int cc) { return key_operand(kt, kg, cc); }, [&]() {},
                    [&](f32x4 (&s)[CB][2]) {
                        if ((t + 1) * TK > p.prefix_len) hide_from<CB>(s, p.prefix_len - t * TK, g);   // uniform
                    });
            }
        } else {
            // Half steps, a barrier behind each: in 2 it the first four waves multiply for step `it` and the others weigh step it - 1, in
            // 2 it + 1 the other way round.  Multiplying for step `it` reads K of stage `it` and V of stage it - 1, so stage it - 2 is free
            // once the others are through with step it - 1: behind half step 2 it - 1.
            static_assert(NS >= 4, "two stages in use, one landing");
            const bool late = wave >= 4;
            f32x4 s[CB][2];
            bf16x8 ph[CB], pl[CB];
            // (the order is pinned: operands are requested a group of products ahead of the one that uses them)
            bf16x8 va[NDB], ka[2][2];
            auto request_keys = [&](const unsigned char *kt, int cc) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int kg = 0; kg < 2; ++kg) ka[i][kg] = key_operand(kt, kg, cc + i);
            };
            auto multiply = [&](int it) {
                issue(it + NS - 2);
                if (!active) return;
                const unsigned char *kt = lds_of(it), *vt = lds_of(it - 1 + NS) + TILEB;
                if (it > 0) {
#pragma unroll
                    for (int db = 0; db < NDB; ++db) va[db] = value_operand<D>(vt, lane, db);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int db = 0; db < NDB / 2; ++db) tile_outputs<D, CB>(st, db, va[db], ph, pl);
                    request_keys(kt, 0);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int db = NDB / 2; db < NDB; ++db) tile_outputs<D, CB>(st, db, va[db], ph, pl);
                } else {
                    request_keys(kt, 0);
                }
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) s[cb][0] = s[cb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int cc = 0; cc < NC; cc += 2) {
                    bf16x8 now[2][2];
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int kg = 0; kg < 2; ++kg) now[i][kg] = ka[i][kg];
                    if (cc + 2 < NC) request_keys(kt, cc + 2);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int kg = 0; kg < 2; ++kg)
#pragma unroll
                            for (int cb = 0; cb < CB; ++cb)
                                s[cb][kg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(now[i][kg], st.q[cb][cc + i], s[cb][kg], 0, 0, 0);
                }
            };
            auto weigh = [&](int it) {
                if (active) {
                    const int t = tile_of(it);
                    if ((t + 1) * TK > p.prefix_len) hide_from<CB>(s, p.prefix_len - t * TK, g);   // uniform; a tile behind the last: all of it
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) tile_weights<D, CB>(st, s[cb], cb, p.scale_log2e, ph[cb], pl[cb]);
                }
            };
#pragma unroll
            for (int it = 1; it < NS - 2; ++it) issue(it);
            wait_copies<CPW *(NS - 3)>();   // this wave's part of stage 0 has landed
            __syncthreads();
            if (late) __syncthreads();
            for (int it = 0; it < steps; ++it) {
                multiply(it);
                if (late) wait_copies<CPW *(NS - 3)>();   // ... of stage it + 1
                __syncthreads();
                weigh(it);
                if (!late) wait_copies<CPW *(NS - 3)>();
                __syncthreads();
            }
            if (!late) __syncthreads();
            if (active) {
                const unsigned char *vt = lds_of(steps - 1) + TILEB;
#pragma unroll
                for (int db = 0; db < NDB; ++db) tile_outputs<D, CB>(st, db, value_operand<D>(vt, lane, db), ph, pl);
            }
        }
        wait_copies<0>();   // (of stages behind the end)
        const size_t slot = task;
        if constexpr (KW == 1) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const float L = sum_over_rows(st.l[cb]), inv = L > 0.f ? 1.f / L : 0.f;
                if (m0 + 16 * cb + c16 < M) {
                    const size_t r = slot * R + 32 * rw + 16 * cb + c16;
#pragma unroll
                    for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4 *>(p.part_o + r * D + 16 * db + 4 * g) = st.o[cb][db] * inv;
                    if (g == 0) p.part_ml[r] = piece_ml(st.m[cb], L);
                }
            }
            __syncthreads();   // every wave's copies have landed and its reads are done: the ring is free
        } else {
            // the results of the groups become one, a block of 16 rows of every row wave at a time
            float *outs = reinterpret_cast<float *>(smem);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const float l = sum_over_rows(st.l[cb]);
                __syncthreads();
                float *ow = outs + (size_t)wave * 16 * OUT_PITCH<D>;
#pragma unroll
                for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4 *>(ow + c16 * OUT_PITCH<D> + 16 * db + 4 * g) = st.o[cb][db];
                if (g == 0) ml_s[wave][c16] = make_float2(st.m[cb], l);
                __syncthreads();
                for (int it = tid; it < RW * 16 * (D / 4); it += 64 * NW) {
                    const int w0 = it / (16 * (D / 4)), m = it / (D / 4) % 16, d0 = it % (D / 4) * 4;
                    if (mb * R + 32 * w0 + 16 * cb + m >= M) continue;
                    float mx = -INFINITY;
#pragma unroll
                    for (int k = 0; k < KW; ++k) mx = fmaxf(mx, ml_s[w0 + k * RW][m].x);
                    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
                    float L = 0.f;
#pragma unroll
                    for (int k = 0; k < KW; ++k) {
                        const float2 ml = ml_s[w0 + k * RW][m];
                        const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - mx);
                        acc += f * *reinterpret_cast<const f32x4 *>(outs + ((size_t)(w0 + k * RW) * 16 + m) * OUT_PITCH<D> + d0);
                        L += f * ml.y;
                    }
                    const size_t r = slot * R + 32 * w0 + 16 * cb + m;
                    *reinterpret_cast<f32x4 *>(p.part_o + r * D + d0) = acc * (L > 0.f ? 1.f / L : 0.f);
                    if (d0 == 0) p.part_ml[r] = piece_ml(mx, L);
                }
            }
            __syncthreads();   // the outputs are read before the next segment's tiles overwrite them
        }
    }
}

// The own part: one wave, its piece of the list.  len0, rows0: length and own rows of sequence `lane`.
// Three tiles are under way at a time, across the ends of segments: of one the page numbers are looked up, of one the rows (and, where it
// opens a segment, the queries: the products have just used the last ones) are on their way, one is worked on.  Where every segment began
// with its own chain of look-ups, 256 sequences that had just begun took 4 us a tile.
template <int D, int CB>
__device__ void own_part(const BranchParams &p, const Plan &plan, int own_wave, int len0, int rows0, float *part_o, float2 *part_ml, unsigned char *vt)
{
    constexpr int NC = D / 32, NDB = D / 16, UPR = D / 8, RPL = 64 / UPR, NV = TK / RPL, R = 16 * CB;
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int Mt = p.G * p.Bt, blocks = (Mt + R - 1) / R, per_seq = p.hkv * blocks, shift = p.pages.page_shift;
    const int begin = own_wave * plan.own_chunk, end = min(begin + plan.own_chunk, plan.own_tiles);
    if (begin >= end) return;
    // where a tile lies: sequence s (n own rows, `len` of them old), segment `local` of it, tile t of that
    struct Place {
        int s, local, t, n, nt, len;
    };
    auto enter = [&](Place &w, int s) {
        w.s = s;
        w.n = s < 64 ? __builtin_amdgcn_readlane(rows0, s & 63) : __builtin_amdgcn_readfirstlane(own_rows(p, s));
        w.len = min(s < 64 ? __builtin_amdgcn_readlane(len0, s & 63) : __builtin_amdgcn_readfirstlane(p.pages.lens[s]), w.n);   // (more than its table has: all)
        w.nt = (w.n + TK - 1) / TK;
    };
    auto advance = [&](Place &w) {   // (there is a next tile)
        if (++w.t < w.nt) return;
        w.t = 0;
        if (++w.local < per_seq) return;
        w.local = 0;
        do enter(w, w.s + 1);
        while (w.n == 0);
    };
    Place cur;
    {
        int first = 0, s = 0;
        for (int base = 0; base < p.n_seqs; base += 64) {
            const int mine = (base == 0 ? rows0 + TK - 1 : base + lane < p.n_seqs ? own_rows(p, base + lane) + TK - 1 : 0) / TK * per_seq;
            const int upto = (int)wave_inclusive_scan((uint32_t)mine), all = __builtin_amdgcn_readlane(upto, 63);
            if (first + all > begin) {
                const int k = __builtin_ctzll(__builtin_amdgcn_ballot_w64(first + upto > begin));
                s = base + k;
                first += __builtin_amdgcn_readlane(upto, k) - __builtin_amdgcn_readlane(mine, k);
                break;
            }
            first += all;
        }
        enter(cur, s);
        cur.local = (begin - first) / cur.nt;
        cur.t = begin - first - cur.local * cur.nt;
    }
    State<D, CB> st;
    st.reset();
    u32x4 kr[2][NC], vr[NV];
    uint32_t absent = 0;   // bit i: rows 8 i .. of the tile in registers lie on a page that does not exist
    int pages[4];
    // A tile's rows lie in groups of eight on one page each (pages have a multiple of eight rows).  Rows past the last repeat it.
    auto look_up = [&](const Place &w) {
        const int32_t *table = p.pages.table + (size_t)w.s * p.pages.width;
#pragma unroll
        for (int i = 0; i < 4; ++i) pages[i] = table[min(w.t * TK + 8 * i, w.n - 1) >> shift];
    };
    auto load = [&](const Place &w) {
        const int h = p.by_own_blocks.divide(w.local), last = w.n - 1;
        const uint16_t *kg8[4], *vg8[4];   // first row of each group, head h
        absent = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = min(w.t * TK + 8 * i, last & ~7);
            int page = __builtin_amdgcn_readfirstlane(pages[i]);
            if ((uint32_t)page >= (uint32_t)p.pages.n_pages) {
                absent |= 1u << i;
                page = 0;
            }
            const size_t off = ((((size_t)page * p.hkv + h) << shift) + (size_t)(row & ((1 << shift) - 1))) * D;
            kg8[i] = p.pages.k + off;
            vg8[i] = p.pages.v + off;
        }
#pragma unroll
        for (int kg = 0; kg < 2; ++kg) {
            const int row = w.t * TK + 16 * kg + c16, in8 = min(row, last) & 7;
            const uint16_t *kb = (c16 < 8 ? kg8[2 * kg] : kg8[2 * kg + 1]) + in8 * D + 8 * g;
#pragma unroll
            for (int cc = 0; cc < NC; ++cc) kr[kg][cc] = *reinterpret_cast<const u32x4 *>(kb + cc * 32);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int row = w.t * TK + i * RPL + lane / UPR, in8 = min(row, last) & 7;
            vr[i] = *reinterpret_cast<const u32x4 *>(vg8[i * RPL / 8] + in8 * D + (lane % UPR) * 8);
        }
        if (absent) {   // (values of such rows may be anything: their weight is zero, and so are they)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (absent >> (i * RPL / 8) & 1) vr[i] = u32x4{0u, 0u, 0u, 0u};
        }
    };
    auto row_of = [&](const Place &w, int cb) { return min((w.local - p.by_own_blocks.divide(w.local) * blocks) * R + 16 * cb + c16, Mt - 1); };
    auto load_queries = [&](const Place &w) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const uint16_t *qr = query_row(p, w.s, p.by_own_blocks.divide(w.local), row_of(w, cb)) + 8 * g;
#pragma unroll
            for (int cc = 0; cc < NC; ++cc) st.q[cb][cc] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qr + cc * 32));
        }
    };
    Place nxt = cur, far = cur;
    look_up(cur);
    load_queries(cur);
    load(cur);
    if (begin + 1 < end) {
        advance(nxt);
        look_up(nxt);
    }
    for (int at = begin; at < end; ++at) {
        const uint32_t hidden = absent;
        const bool ends = at + 1 == end || nxt.t == 0;   // the wave's last tile of the segment
        // Of the two waves of a SIMD the older one goes first whenever both could: with equal shares of a long list it was done after
        // 89 us, the younger one after 108.  The younger one goes first every other tile.
        if (threadIdx.x >= 64 * NW / 2) {
            if ((at - begin) & 1) __builtin_amdgcn_s_setprio(0);
            else __builtin_amdgcn_s_setprio(1);
        }
        store_v<D>(vt, vr, lane);
        tile_step<D, CB>(
            st, vt, p.scale_log2e, lane, [&](int kg, int cc) { return __builtin_bit_cast(bf16x8, kr[kg][cc]); },
            [&]() {
                if (at + 1 < end) {
                    load(nxt);
                    if (nxt.t == 0) load_queries(nxt);
                    far = nxt;
                    if (at + 2 < end) {
                        advance(far);
                        look_up(far);
                    }
                }
            },
            [&](f32x4 (&sc)[CB][2]) {
                if ((cur.t + 1) * TK > cur.len || hidden) {   // uniform: rows that not every query sees
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        const int m = row_of(cur, cb), vis = min(cur.len + m - p.by_Bt.divide(m) * p.Bt + 1, cur.n);
                        const int lim = vis - cur.t * TK - 4 * g;
#pragma unroll
                        for (int kg = 0; kg < 2; ++kg) {
                            const bool gone = hidden >> (2 * kg + (g >> 1)) & 1;
#pragma unroll
                            for (int i = 0; i < 4; ++i) sc[cb][kg][i] = 16 * kg + i < lim && !gone ? sc[cb][kg][i] : -INFINITY;
                        }
                    }
                }
            });
        if (ends) {
            const size_t slot = (size_t)own_wave + (size_t)cur.s * per_seq + cur.local;
            const int first_row = (cur.local - p.by_own_blocks.divide(cur.local) * blocks) * R;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const float L = sum_over_rows(st.l[cb]), inv = L > 0.f ? 1.f / L : 0.f;
                if (first_row + 16 * cb + c16 < Mt) {
                    float *ow = part_o + (slot * R + 16 * cb + c16) * D;
#pragma unroll
                    for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4 *>(ow + 16 * db + 4 * g) = st.o[cb][db] * inv;
                    if (g == 0) part_ml[slot * R + 16 * cb + c16] = piece_ml(st.m[cb], L);
                }
            }
            st.reset();
        }
        cur = nxt;
        nxt = far;
    }
}

// Slots of the shared part at most: one per task
__host__ __device__ inline size_t shared_slots(int n_prefixes, int fan, int hkv, int Mt, int R, int wgs)
{
    const size_t segs = (size_t)n_prefixes * hkv * ((fan * Mt + R - 1) / R);
    return 2 * segs > (size_t)wgs ? 2 * segs : wgs;
}

// RS, RO: query rows of a block of the shared and of the own part
template <int D, int RS>
constexpr int lds_bytes()
{
    constexpr int waves = NW * 16 * OUT_PITCH<D> * 4;   // the outputs of the waves' 16 rows; a piece of V for every wave is a little less
    static_assert(waves >= NW * TK * D * 2, "");
    if constexpr (RS > 32) {
        constexpr int ring = stages_of(RS / 32) * stage_bytes<D, RS / 32>();
        return ring > waves ? ring : waves;
    }
    return waves;
}

// Prices in us, measured by stamps of the clock inside the kernel where neither part waits for the other's traffic: a step of the shared part
// (every group of waves a tile) and what a task takes besides; a tile of a wave of the own part and what a wave takes besides; and what a
// tile of own rows takes at the rate that memory gives all workgroups together, which no share of them changes.  own_end: what the end of a
// segment adds to its tile (without it the own rows of 192 sequences that had just begun got half the workgroups they needed: 87 us, now 63).
// partial: a row of a partial of the shared part written, and read again by the join (the slope of the time of calls over the bytes of their
// partials, at blocks of 64, 128 and 256 rows).
template <int D, int RS, int RO>
struct Prices {
    static constexpr bool wide = D == 128;
    static constexpr float step = RS == 256 ? (wide ? 1.3f : 1.0f) : RS == 128 ? (wide ? 1.45f : 1.1f) : RS == 64 ? (wide ? 2.35f : 1.1f) : (wide ? 2.5f : 1.5f);
    // (blocks of 16 rows read every tile for themselves)
    static __host__ __device__ float step_of(int blocks) { return RS == 16 ? step * (0.85f + 0.15f * (float)blocks) : step; }
    static constexpr float task = RS == 256 ? (wide ? 9.f : 7.f) : RS == 128 ? (wide ? 9.5f : 6.5f) : RS == 64 ? (wide ? 8.8f : 5.5f) : (wide ? 4.5f : 4.f);
    static constexpr float own_tile = RO == 16 ? (wide ? 2.7f : 1.8f) : (wide ? 3.8f : 2.2f), own_end = 0.7f, own_wave = 4.f;
    static constexpr float own_traffic = TK * D * 4 / 5.5e6f, partial = D * 4 / 2e6f;
};

// How the work is cut: the same on every wave.  rows0: own rows of sequence `lane`.
// No piece leaves its segment: the start and the end of a segment cost a workgroup several tiles' time.  Every lane prices one way to
// deal the workgroups -- `splits` pieces of each segment, or with more segments than workgroups a share of the workgroups for
// whole or halved segments -- and the cheapest is taken.
template <int D, int RS, int RO>
__device__ __forceinline__ Plan make_plan(const BranchParams &p, int units, int wgs, int rows0, int lane)
{
    using P = Prices<D, RS, RO>;
    // (An exact quotient that the reciprocal makes a bit too large counts one too many, which the host's prices below do not.  With exact counts
    // 59 sizes took 1.003 of the time on average, from 0.995 to 1.026: the choice hardly ever changes.)
    auto up = [](float x, float y) { return __builtin_ceilf(x * __builtin_amdgcn_rcpf(y)); };
    Plan plan;
    int own = (rows0 + TK - 1) / TK;
    int used = __popcll(__builtin_amdgcn_ballot_w64(own > 0));   // sequences with own rows
    for (int base = 64; base < p.n_seqs; base += 64) {
        const int more = base + lane < p.n_seqs ? (own_rows(p, base + lane) + TK - 1) / TK : 0;
        own += more;
        used += __popcll(__builtin_amdgcn_ballot_w64(more > 0));
    }
    const int per_seq = p.hkv * ((p.G * p.Bt + RO - 1) / RO);
    plan.own_tiles = __builtin_amdgcn_readlane((int)wave_inclusive_scan((uint32_t)own), 63) * per_seq;
    const float own_work = (float)plan.own_tiles * P::own_tile + (float)(used * per_seq) * P::own_end;
    const int segs = p.shared_segs, most = plan.own_tiles > 0 ? wgs - 1 : wgs;
    const float step = P::step_of((p.fan * p.G * p.Bt + RS - 1) / RS);
    int w = 0, splits = 1;
    float price = INFINITY;
    if (segs > 0 && segs <= most) {
        const int top = min(p.by_segs.divide(most), units);
        splits = min((lane + 1) * ((top + 63) / 64), top);
        w = segs * splits;
        price = up((float)units, (float)splits) * step + P::task;
    } else if (segs > 0) {
        w = max(most * (lane + 1) / 64, 1);
        const float whole = up((float)segs, (float)w) * ((float)units * step + P::task);
        const float half = up(2.f * (float)segs, (float)w) * ((float)((units + 1) / 2) * step + P::task);
        splits = units > 1 && half < whole ? 2 : 1;
        price = fminf(whole, half);
    }
    const int others = (wgs - w) * NW;
    if (plan.own_tiles > 0) {
        const float own_price = fmaxf(up(own_work, (float)others), (float)plan.own_tiles * P::own_traffic) + P::own_wave;
        price = segs > 0 ? fmaxf(price, own_price) : own_price;
    }
    const uint32_t cheap = ~__float_as_uint(price);   // (prices are not negative: the cheapest has the largest complement)
    uint32_t best = cheap;
    best = max(best, dpp_fetch<0x111, 0xF>(best));
    best = max(best, dpp_fetch<0x112, 0xF>(best));
    best = max(best, dpp_fetch<0x114, 0xF>(best));
    best = max(best, dpp_fetch<0x118, 0xF>(best));
    best = max(best, dpp_fetch<0x142, 0xA>(best));
    best = max(best, dpp_fetch<0x143, 0xC>(best));
    best = (uint32_t)__builtin_amdgcn_readlane((int)best, 63);
    const int from = __builtin_ctzll(__builtin_amdgcn_ballot_w64(cheap == best));   // (of equal ones that with the fewest pieces)
    plan.splits = __builtin_amdgcn_readlane(splits, from);
    plan.shared_wgs = segs > 0 ? __builtin_amdgcn_readlane(w, from) : 0;
    const int waves = max((wgs - plan.shared_wgs) * NW, 1);
    plan.own_chunk = max((int)((float)plan.own_tiles * __builtin_amdgcn_rcpf((float)waves)), 1);
    while ((int64_t)plan.own_chunk * waves < plan.own_tiles) ++plan.own_chunk;
    return plan;
}

template <int D, int RS, int RO>
__global__ __launch_bounds__(64 * NW) void branch_main_kernel(BranchParams p)
{
    warm_arguments<sizeof(BranchParams)>();
    __shared__ __attribute__((aligned(1024))) unsigned char smem[lds_bytes<D, RS>()];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int Mt = p.G * p.Bt, wgs = (int)gridDim.x;
    const int len0 = p.pages.lens[min(lane, p.n_seqs - 1)], asked0 = asked_of(p, min(lane, p.n_seqs - 1));
    constexpr int KW = RS > 32 ? NW / (RS / 32) : NW;   // tiles that a workgroup of the shared part works on at a time
    const int units = ((p.prefix_len + TK - 1) / TK + KW - 1) / KW;
    const int rows0 = lane < p.n_seqs ? own_rows(p, len0, asked0) : 0;
    const Plan plan = make_plan<D, RS, RO>(p, units, wgs, rows0, lane);
    if (blockIdx.x == 0 && wave == 0) {   // ... for the join
        if (lane == 0) {
            p.plan[0] = plan.splits;
            p.plan[1] = plan.own_chunk;
        }
        int first = 0;
        for (int base = 0; base < p.n_seqs; base += 64) {
            const int mine = (base == 0 ? rows0 + TK - 1 : base + lane < p.n_seqs ? own_rows(p, base + lane) + TK - 1 : 0) / TK;
            const int upto = (int)wave_inclusive_scan((uint32_t)mine);
            if (base + lane < p.n_seqs) p.plan[BRANCH_PLAN_WORDS + base + lane] = first + upto - mine;
            first += __builtin_amdgcn_readlane(upto, 63);
        }
    }
    if ((int)blockIdx.x < plan.shared_wgs) {
        if constexpr (RS > 32) shared_many<D, RS / 32>(p, plan, smem);
        else shared_few<D>(p, plan, smem);
    } else {
        const size_t rows = shared_slots(p.n_prefixes, p.fan, p.hkv, Mt, RS, wgs) * RS;
        own_part<D, RO / 16>(p, plan, ((int)blockIdx.x - plan.shared_wgs) * NW + wave, len0, rows0, p.part_o + rows * D, p.part_ml + rows,
                             smem + (size_t)wave * TK * D * 2);
    }
}

// The join of a row's pieces: `groups` groups of D / 4 threads take a row's pieces in turn, four at a time, and join what they have
// in LDS.  (Groups: where there are few rows and many pieces, the pieces requested one behind another were all the time this took: one
// sequence, 8192 shared rows, 17.7 us with one group a row.)  LSE: the logarithms of the weight sums too (a test of the pointer in the kernel alone took
// 0.3 us of the calls without)
template <int D, int RS, int RO, bool LSE>
__global__ __launch_bounds__(256) void branch_merge_kernel(BranchParams p, int wgs, int groups)
{
    constexpr int TPR = D / 4, BATCH = 4;
    __shared__ f32x4 acc_s[256];
    __shared__ float2 ml_s[256 / TPR];
    const int Mt = p.G * p.Bt;
    const int unit = (int)threadIdx.x / TPR, group = unit % groups;
    const int64_t row = (int64_t)blockIdx.x * (256 / TPR / groups) + unit / groups;
    const int d0 = (int)threadIdx.x % TPR * 4;
    const bool exists = row < (int64_t)p.n_seqs * p.hkv * Mt;
    const int sh = exists ? p.by_Mt.divide((int)row) : 0, m = exists ? (int)row - sh * Mt : 0, s = p.by_hkv.divide(sh), h = sh - s * p.hkv;
    // (all that says where the pieces are is requested at once)
    const int len = p.pages.lens[s], asked = asked_of(p, s), splits = p.plan[0], chunk = p.plan[1], tiles_before = p.plan[BRANCH_PLAN_WORDS + s];
    const bool wanted = exists && m - p.by_Bt.divide(m) * p.Bt < new_of(p, len, asked);   // else left as it was
    // the pieces: na slots of the shared part, nb slots from b0 on of the own part
    int a0 = 0, na = 0, segs = 0, b0 = 0, nb = 0, am = 0, bm = 0;
    if (wanted) {
        if (p.prefix_len > 0) {
            const int c = p.by_fan.divide(s), mm = (s - c * p.fan) * Mt + m;
            am = mm % RS;
            a0 = mm / RS * p.n_prefixes * p.hkv + c * p.hkv + h;   // piece i in slot a0 + i segs
            segs = p.shared_segs;
            na = splits;
        }
        const int n = own_rows(p, len, asked);
        if (n > 0) {
            const int blocks = (Mt + RO - 1) / RO, nt = (n + TK - 1) / TK;
            const int local = h * blocks + m / RO, first = tiles_before * p.hkv * blocks + local * nt;
            const int seg = s * p.hkv * blocks + local;
            bm = m % RO;
            b0 = first / chunk;
            nb = (first + nt - 1) / chunk + 1 - b0;
            b0 += seg;
        }
    }
    const size_t rows = shared_slots(p.n_prefixes, p.fan, p.hkv, Mt, RS, wgs) * RS;
    float mx = -INFINITY, L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = group; i0 < na + nb; i0 += groups * BATCH) {
        float2 ml[BATCH];
        f32x4 o[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int i = min(i0 + k * groups, na + nb - 1);
            const size_t at = i < na ? ((size_t)a0 + (size_t)i * segs) * RS + am : rows + (size_t)(b0 + i - na) * RO + bm;
            ml[k] = p.part_ml[at];
            o[k] = *reinterpret_cast<const f32x4 *>(p.part_o + at * D + d0);
            if (i0 + k * groups >= na + nb) ml[k] = make_float2(-INFINITY, 0.f);
        }
        float top = mx;
#pragma unroll
        for (int k = 0; k < BATCH; ++k) top = fmaxf(top, ml[k].x);
        if (top == -INFINITY) continue;
        const float old = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - top);
        L *= old;
        acc *= old;
        mx = top;
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const float f = ml[k].x == -INFINITY ? 0.f : ml[k].y * __builtin_amdgcn_exp2f(ml[k].x - mx);
            acc += f * o[k];
            L += f;
        }
    }
    if (groups > 1) {   // uniform
        acc_s[threadIdx.x] = acc;
        if (d0 == 0) ml_s[unit] = make_float2(mx, L);
        __syncthreads();
        if (group != 0) return;
        float top = -INFINITY;
        for (int k = 0; k < groups; ++k) top = fmaxf(top, ml_s[unit + k].x);
        if (LSE) mx = top;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
        L = 0.f;
        for (int k = 0; k < groups; ++k) {
            const float2 ml = ml_s[unit + k];
            const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
            acc += f * acc_s[threadIdx.x + k * TPR];
            L += f * ml.y;
        }
    }
    if (!wanted) return;
    const float inv = L > 0.f ? 1.f / L : 0.f;   // a row that sees no key is zero
    bf16x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (__bf16)(acc[i] * inv);
    *reinterpret_cast<bf16x4 *>(p.out + (((size_t)s * p.hkv + h) * Mt + m) * D + d0) = o;
    if (LSE && d0 == 0) p.lse[((size_t)s * p.hkv + h) * Mt + m] = log_sum(mx, L);
}

// Few rows: one launch, a workgroup for every (sequence, head, block of rows), whose waves take tiles of the prompt's and of the own rows in
// turn and join their results in LDS; no partials, no plan and no second launch.
template <int D, int RO, bool LSE>
__global__ __launch_bounds__(64 * NW) void branch_short_kernel(BranchParams p)
{
    constexpr int CB = RO / 16, NC = D / 32, NDB = D / 16, UPR = D / 8, ROWB = D * 2, RPL = 64 / UPR, NV = TK / RPL;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[lds_bytes<D, 16>()];
    __shared__ float2 ml_s[NW][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const int Mt = p.G * p.Bt, blocks = (Mt + RO - 1) / RO;
    const int sh = p.by_own_blocks.divide(blockIdx.x), m0 = ((int)blockIdx.x - sh * blocks) * RO, s = p.by_hkv.divide(sh), h = sh - s * p.hkv;
    const int asked = asked_of(p, s), held = p.pages.lens[s];
    const int np = (p.prefix_len + TK - 1) / TK, shift = p.pages.page_shift;
    const size_t ch = (size_t)p.by_fan.divide(s) * p.hkv + h;
    const char *kh = reinterpret_cast<const char *>(p.k_prefix + ch * p.prefix_cap * D), *vh = reinterpret_cast<const char *>(p.v_prefix + ch * p.prefix_cap * D);
    const int32_t *table = p.pages.table + (size_t)s * p.pages.width;
    unsigned char *vt = smem + (size_t)wave * TK * ROWB;
    State<D, CB> st;
    st.reset();
    u32x4 kr[2][NC], vr[NV];
    uint32_t absent = 0;   // bit i: rows 8 i .. of the tile in registers lie on a page that does not exist
    auto load_shared = [&](int t) {   // (rows past the last repeat it: their weights are masked to zero)
#pragma unroll
        for (int kg = 0; kg < 2; ++kg) {
            const uint32_t off = (uint32_t)min(t * TK + 16 * kg + c16, p.prefix_len - 1) * ROWB + 16 * g;
#pragma unroll
            for (int cc = 0; cc < NC; ++cc) kr[kg][cc] = *reinterpret_cast<const u32x4 *>(kh + off + cc * 64);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            vr[i] = *reinterpret_cast<const u32x4 *>(vh + (uint32_t)min(t * TK + i * RPL + lane / UPR, p.prefix_len - 1) * ROWB + lane % UPR * 16);
        absent = 0;
    };
    const int n = own_rows(p, held, asked), len = min(held, n), total = np + (n + TK - 1) / TK;
    auto load_own = [&](int t) {
        const uint16_t *kg8[4], *vg8[4];   // first row of each group of eight, which lies on one page
        absent = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = min(t * TK + 8 * i, (n - 1) & ~7);
            int page = table[row >> shift];
            if ((uint32_t)page >= (uint32_t)p.pages.n_pages) {
                absent |= 1u << i;
                page = 0;
            }
            const size_t off = ((((size_t)page * p.hkv + h) << shift) + (size_t)(row & ((1 << shift) - 1))) * D;
            kg8[i] = p.pages.k + off;
            vg8[i] = p.pages.v + off;
        }
#pragma unroll
        for (int kg = 0; kg < 2; ++kg) {
            const uint16_t *kb = (c16 < 8 ? kg8[2 * kg] : kg8[2 * kg + 1]) + (min(t * TK + 16 * kg + c16, n - 1) & 7) * D + 8 * g;
#pragma unroll
            for (int cc = 0; cc < NC; ++cc) kr[kg][cc] = *reinterpret_cast<const u32x4 *>(kb + cc * 32);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            vr[i] = *reinterpret_cast<const u32x4 *>(vg8[i * RPL / 8] + (min(t * TK + i * RPL + lane / UPR, n - 1) & 7) * D + lane % UPR * 8);
            if (absent >> (i * RPL / 8) & 1) vr[i] = u32x4{0u, 0u, 0u, 0u};   // (what is there may be anything)
        }
    };
    auto load = [&](int t) {
        if (t < np) load_shared(t);
        else if (t < total) load_own(t - np);
    };
    load(wave);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const uint16_t *qr = query_row(p, s, h, min(m0 + 16 * cb + c16, Mt - 1)) + 8 * g;
#pragma unroll
        for (int cc = 0; cc < NC; ++cc) st.q[cb][cc] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qr + cc * 32));
    }
    const int fresh = new_of(p, held, asked);
    if (fresh == 0) return;   // uniform: its rows are left as they were
    for (int t = wave; t < total; t += NW) {
        const uint32_t hidden = absent;
        store_v<D>(vt, vr, lane);
        tile_step<D, CB>(
            st, vt, p.scale_log2e, lane, [&](int kg, int cc) { return __builtin_bit_cast(bf16x8, kr[kg][cc]); }, [&]() { load(t + NW); },
            [&](f32x4 (&sc)[CB][2]) {
                if (t < np) {   // uniform
                    if ((t + 1) * TK > p.prefix_len) hide_from<CB>(sc, p.prefix_len - t * TK, g);
                } else if ((t - np + 1) * TK > len || hidden) {
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        const int m = min(m0 + 16 * cb + c16, Mt - 1), lim = min(len + m - p.by_Bt.divide(m) * p.Bt + 1, n) - (t - np) * TK - 4 * g;
#pragma unroll
                        for (int kg = 0; kg < 2; ++kg) {
                            const bool gone = hidden >> (2 * kg + (g >> 1)) & 1;
#pragma unroll
                            for (int i = 0; i < 4; ++i) sc[cb][kg][i] = 16 * kg + i < lim && !gone ? sc[cb][kg][i] : -INFINITY;
                        }
                    }
                }
            });
    }
    float *outs = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const float l = sum_over_rows(st.l[cb]);
        __syncthreads();   // nobody reads V tiles, or the block of rows before, any more
        float *ow = outs + (size_t)wave * 16 * OUT_PITCH<D>;
#pragma unroll
        for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4 *>(ow + c16 * OUT_PITCH<D> + 16 * db + 4 * g) = st.o[cb][db];
        if (g == 0) ml_s[wave][c16] = make_float2(st.m[cb], l);
        __syncthreads();
        join_waves<D>(outs, ml_s, min(16, Mt - m0 - 16 * cb), tid, [&](int row, int d0, f32x4 acc, float mx, float L) {
            const int m = m0 + 16 * cb + row;
            if (m - p.by_Bt.divide(m) * p.Bt >= fresh) return;
            bf16x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = (__bf16)acc[i];
            *reinterpret_cast<bf16x4 *>(p.out + ((size_t)sh * Mt + m) * D + d0) = o;
            if (LSE && d0 == 0) p.lse[(size_t)sh * Mt + m] = log_sum(mx, L);
        });
    }
}

// Query rows of a block of the own part: 16, or 32 where a sequence has more
int own_block(int64_t rows) { return rows > 16 ? 32 : 16; }

// What the shared part takes with blocks of RS rows, as make_plan prices it, a sixteenth of the workgroups left to the own part, and its partials
template <int D, int RS>
float shared_price(int64_t rows, int heads, int prefix_len, int cus)
{
    using P = Prices<D, RS, 16>;
    auto up = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
    constexpr int KW = RS == 16 ? NW : NW / (RS / 32);
    const float step = P::step_of((int)up(rows, RS));
    const int64_t segs = heads * up(rows, RS), units = up(up(prefix_len, TK), KW), wgs = std::max(cus - cus / 16, 1);
    if (segs <= wgs) {
        const int64_t splits = std::min(wgs / segs, units);
        return (float)up(units, splits) * step + P::task + (float)(splits * heads * rows) * P::partial;
    }
    return (float)up(segs, wgs) * ((float)units * step + P::task) + (float)(heads * rows) * P::partial;
}

// Query rows of a block of the shared part, and what it takes (rows, prefix_len >= 1): 16, whose waves work each for itself, or two, four or
// eight waves of 32 rows, which share tiles; of those that rows half fill at least (and of 16 up to four blocks), the cheapest.  Small blocks
// have fewer pieces of each segment, and so fewer partials, large ones read a tile for more rows.  Measured with blocks of 64, 128 and 256
// (D 128, 8 KV heads): 256 rows over 1024 shared ones 19.2, 21.7 and 23.1 us, over 8192 31.1, 29.1 and 33.7; 1024 rows over 8192 110, 71 and
// 66; with 16 and 64: 48 rows over 2000 12.2 and 14.7, over 12288 21.6 and 20.1.  Over 210 sizes the choice of 64, 128 or 256 is 0.9 % off
// the best on average; that by rows alone was 8.7 % off.
struct SharedBlock {
    int rows;
    float price;
};
template <int D>
SharedBlock shared_block(int64_t rows, int heads, int prefix_len, int cus)
{
    SharedBlock best{16, rows <= 64 ? shared_price<D, 16>(rows, heads, prefix_len, cus) : INFINITY};
    auto consider = [&](SharedBlock other) { best = other.price < best.price ? other : best; };
    if (rows > 16) consider({64, shared_price<D, 64>(rows, heads, prefix_len, cus)});
    if (rows > 64) consider({128, shared_price<D, 128>(rows, heads, prefix_len, cus)});
    if (rows > 128) consider({256, shared_price<D, 256>(rows, heads, prefix_len, cus)});
    return best;
}

// Whether one launch with a workgroup a segment (branch_short_kernel) takes the call: its time, with as many own rows as the tables can name
// (the lengths themselves are on the device: tables laid out for long answers take two launches from the first token on), against the two
// launches' with the prompts' part alone, whose pieces are dealt to all workgroups.
// Lines through the times of 345 sizes, of which the choice is as fast as the better on average (two launches always: 36 % slower).  Measured, one
// launch against two (D 128, 8 KV heads of 4 query heads): one sequence, 40 shared and 10 own rows 4.5 us against 9.1, 200 and 100 6.8
// and 9.8, 1000 and 300 15.6 and 10.4; 32 sequences, 200 and 100 7.2 and 14.8, 1000 and 100 13.7 and 16.7, 2000 and 100 22.5 and 18.6;
// 128 sequences, 40 and 10 13.9 and 17.5, 500 and 10 30.9 and 20.5.
template <int D, int RO>
bool one_launch(const BranchParams &p, const SharedBlock &block)
{
    constexpr bool wide = D == 128;
    constexpr float start = RO == 16 ? (wide ? 2.f : 1.3f) : (wide ? 4.4f : 3.2f), tile = RO == 16 ? (wide ? 2.2f : 1.15f) : (wide ? 2.4f : 1.13f);
    const int64_t segs = (int64_t)p.n_seqs * p.hkv * ((p.G * p.Bt + RO - 1) / RO);
    const int64_t own = ((int64_t)p.pages.width << p.pages.page_shift) / TK + 1, tiles = (p.prefix_len + TK - 1) / TK + own;
    const float one = 1.7f + std::max((float)segs / (float)p.cus, 1.f) * (start + tile / NW * (float)tiles);
    using P = Prices<D, 16, RO>;
    const float both = p.shared_segs > 0 ? block.price + (block.rows == 16 ? 3.5f : 2.f) : P::own_wave + P::own_tile + 2.f;   // start and join
    return one <= both && segs < (1 << 22);   // (a launch counts its threads in 32 bits)
}

}  // namespace

size_t branch_workspace(int n_seqs, int n_prefixes, int hkv, int G, int Bt, int D, int cus, size_t *off_ml, size_t *off_plan)
{
    const int64_t Mt = (int64_t)G * Bt, fan = n_prefixes > 0 ? n_seqs / n_prefixes : 0;
    const size_t RO = own_block(Mt);
    size_t shared = 0;   // (the length of the prompts' rows is not known here: the most that any block takes)
    for (const int RS : {16, 64, 128, 256})
        if (RS == 16 ? fan * Mt <= 64 : fan * Mt > (RS == 64 ? 16 : RS / 2))
            shared = std::max(shared, shared_slots(n_prefixes, (int)fan, hkv, (int)Mt, RS, cus) * RS);
    const size_t own = ((size_t)n_seqs * hkv * ((Mt + RO - 1) / RO) + (size_t)cus * NW) * RO;
    size_t off = (shared + own) * D * 4;
    off = (off + 255) & ~(size_t)255;
    *off_ml = off;
    off += ((shared + own) * 8 + 255) & ~(size_t)255;
    *off_plan = off;
    off += ((size_t)(BRANCH_PLAN_WORDS + n_seqs) * 4 + 255) & ~(size_t)255;
    return off;
}

namespace {

template <int D, int RS, int RO>
hipError_t launch_both(const BranchParams &p, hipStream_t s)
{
    const int64_t rows = (int64_t)p.n_seqs * p.hkv * p.G * p.Bt;
    const int units = 256 / (D / 4);
    int groups = 1;   // as many as the chip's threads hold at once, and no more than a workgroup
    while (groups < units && rows * (D / 4) * groups * 2 <= (int64_t)p.cus * 2048) groups *= 2;
    const int per = units / groups, wgs = p.cus;
    hipLaunchKernelGGL((branch_main_kernel<D, RS, RO>), dim3(wgs), dim3(64 * NW), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((rows + per - 1) / per));
    if (p.lse) hipLaunchKernelGGL((branch_merge_kernel<D, RS, RO, true>), grid, dim3(256), 0, s, p, wgs, groups);
    else hipLaunchKernelGGL((branch_merge_kernel<D, RS, RO, false>), grid, dim3(256), 0, s, p, wgs, groups);
    return hipGetLastError();
}

template <int D, int RO>
hipError_t launch(BranchParams p, hipStream_t s)
{
    const int64_t rows = (int64_t)p.fan * p.G * p.Bt;
    const int blocks = (p.G * p.Bt + RO - 1) / RO, heads = p.n_prefixes * p.hkv;
    const SharedBlock block = shared_block<D>(std::max<int64_t>(rows, 1), std::max(heads, 1), std::max(p.prefix_len, 1), p.cus);
    p.shared_segs = p.prefix_len > 0 ? (int32_t)(heads * ((rows + block.rows - 1) / block.rows)) : 0;
    p.by_segs.set(std::max(p.shared_segs, 1));
    p.by_heads.set(std::max(heads, 1));
    p.by_hkv.set(p.hkv);
    p.by_Mt.set((uint32_t)(p.G * p.Bt));
    p.by_Bt.set(p.Bt);
    p.by_fan.set(std::max(p.fan, 1));
    p.by_own_blocks.set((uint32_t)blocks);
    if (one_launch<D, RO>(p, block)) {
        const dim3 grid((unsigned)(p.n_seqs * p.hkv * blocks));
        if (p.lse) hipLaunchKernelGGL((branch_short_kernel<D, RO, true>), grid, dim3(64 * NW), 0, s, p);
        else hipLaunchKernelGGL((branch_short_kernel<D, RO, false>), grid, dim3(64 * NW), 0, s, p);
        return hipGetLastError();
    }
    switch (block.rows) {
    case 16: return launch_both<D, 16, RO>(p, s);
    case 64: return launch_both<D, 64, RO>(p, s);
    case 128: return launch_both<D, 128, RO>(p, s);
    default: return launch_both<D, 256, RO>(p, s);
    }
}

}  // namespace

hipError_t launch_branch_attention(const BranchParams &p, hipStream_t s)
{
    const bool few = own_block((int64_t)p.G * p.Bt) == 16;
    if (p.D == 128) return few ? launch<128, 16>(p, s) : launch<128, 32>(p, s);
    if (p.D == 64) return few ? launch<64, 16>(p, s) : launch<64, 32>(p, s);
    return hipErrorInvalidValue;
}

}  // namespace kd
