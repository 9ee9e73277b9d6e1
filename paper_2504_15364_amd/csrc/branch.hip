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
// Both parts are cut into tiles of 32 keys and 16 x CB query rows, and the chip's waves are dealt to the two parts by their tiles:
//   shared part  the tiles of all (prompt, head, block of rows) segments form one list, of which a workgroup takes a contiguous
//                piece, its eight waves in turn a tile each; where the piece leaves a segment the waves' results are joined in LDS
//                and stored as one partial
//   own part     the tiles of all (sequence, head, block of rows) segments form another list, of which every wave takes a
//                contiguous piece and stores a partial where the piece leaves a segment: no wave waits for another one, and
//                ragged lengths cost nothing, because the list is cut by tiles and not by sequences
// The lists follow from the lengths on the device: the launch itself does not depend on them and may be replayed from a graph.
#include "kd_branch.h"
#include "kd_device.h"

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
constexpr float RESCALE_SLACK = 64.f; // the reference maximum may lag by 2^64: weights, sums and outputs stay far inside float's range

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
__device__ __forceinline__ int wave_sum(int x)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    return x;
}

// Rows that are keys of a sequence's new tokens (its own rows and the new ones), 0 where it has nothing to do
__device__ __forceinline__ int new_of(const BranchParams &p, int s)
{
    if (p.pages.lens[s] < 0) return 0;
    return p.pages.n_new ? max(0, min(p.pages.n_new[s], p.Bt)) : p.Bt;
}
__device__ __forceinline__ int own_rows(const BranchParams &p, int s)
{
    const int fresh = new_of(p, s);
    if (fresh == 0) return 0;
    const int64_t n = (int64_t)p.pages.lens[s] + fresh, most = (int64_t)p.pages.width << p.pages.page_shift;
    return (int)(n < most ? n : most);
}

// How the work is cut (uniform; the merge reads it from BranchParams::plan)
struct Plan {
    int shared_wgs, shared_chunk;   // workgroups of the shared part, tiles each takes
    int own_chunk;                  // tiles a wave of the own part takes
    int shared_tiles, own_tiles;
};

// One wave's state of a block of 16 x CB query rows: column c16 of block cb is query row 16 cb + c16
template <int D, int CB>
struct State {
    f32x4 o[CB][D / 16];   // element i of block db: column 16 db + 4 g + i of the output
    float l[CB], m[CB];    // weight sum of the lane's own keys; reference maximum (log2 units), the same in the four lanes of a row
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

// 16-byte units of a V row in LDS are permuted so that what a transposing read gathers lies in different banks
template <int D>
__device__ __forceinline__ int v_swizzle(int row)
{
    constexpr int UPR = D / 8, VSW = UPR / 4;
    return UPR == 16 ? (VSW * (row & 3)) ^ (2 * ((row >> 2) & 1)) : VSW * (row & 3);
}

// One tile: kr, vr hold its rows (V's are moved to the wave's piece of LDS first; `refill` then requests the next tile's).
// Logits S^T = K Q^T: element i of s[cb][kg] is key 16 kg + 4 g + i of query row 16 cb + c16; `mask(s)` sets those that are not
// seen to -inf.  Outputs O^T += V^T P^T: the keys are enumerated in accumulator order, and two transposing reads fetch exactly those.
// The weights go into the second product as two bf16 numbers, rounded value and rest (16 bits in all): rounded to one, their error
// alone would be as large as the output's own rounding, and these products do not bound the kernel.
template <int D, int CB, class Refill, class Mask>
__device__ __forceinline__ void tile_step(State<D, CB> &st, u32x4 (&kr)[2][D / 32], u32x4 (&vr)[TK * D / 512], unsigned char *vt, float scale_log2e,
                                          int lane, Refill refill, Mask mask)
{
    constexpr int NC = D / 32, NDB = D / 16, UPR = D / 8, ROWB = D * 2, RPL = 64 / UPR, NV = TK / RPL;
    const int c16 = lane & 15, g = lane >> 4;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int row = lane / UPR + RPL * i;
        *reinterpret_cast<u32x4 *>(vt + row * ROWB + (((lane % UPR) ^ v_swizzle<D>(row)) * 16)) = vr[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    f32x4 s[CB][2];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) s[cb][0] = s[cb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int kg = 0; kg < 2; ++kg)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                s[cb][kg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[kg][c]), st.q[cb][c], s[cb][kg], 0, 0, 0);
    refill();
    mask(s);
    bf16x8 ph[CB], pl[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        float mx = fmaxf(fmaxf(fmaxf(s[cb][0][0], s[cb][0][1]), fmaxf(s[cb][0][2], s[cb][0][3])),
                         fmaxf(fmaxf(s[cb][1][0], s[cb][1][1]), fmaxf(s[cb][1][2], s[cb][1][3])));
        mx = max_over_rows(mx) * scale_log2e;
        const bool need = mx > st.m[cb] + RESCALE_SLACK;
        if (__builtin_amdgcn_ballot_w64(need) != 0) {
            const float alpha = need ? __builtin_amdgcn_exp2f(st.m[cb] - mx) : 1.f;
            st.m[cb] = need ? mx : st.m[cb];
            st.l[cb] *= alpha;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.o[cb][db][i] *= alpha;
        }
        const float nm = st.m[cb] == -INFINITY ? 0.f : -st.m[cb];
#pragma unroll
        for (int kg = 0; kg < 2; ++kg)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[cb][kg][i], scale_log2e, nm));
                st.l[cb] += w;
                const __bf16 hi = (__bf16)w;
                ph[cb][4 * kg + i] = hi;
                pl[cb][4 * kg + i] = (__bf16)(w - (float)hi);
            }
    }
    const int rd_row = 4 * g + (c16 >> 2), rd_unit = ((c16 & 3) >> 1) ^ v_swizzle<D>(rd_row);   // (rows + 16 have the same swizzle)
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
        const unsigned char *ap = vt + rd_row * ROWB + (c16 & 1) * 8 + (((2 * db) ^ rd_unit) * 16);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)(ap));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)(ap + 16 * ROWB));
        const bf16x8 va = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            st.o[cb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, ph[cb], st.o[cb][db], 0, 0, 0);
            st.o[cb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pl[cb], st.o[cb][db], 0, 0, 0);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Address of query row m (order g, j) of sequence s and KV head h
__device__ __forceinline__ const uint16_t *query_row(const BranchParams &p, int s, int h, int m)
{
    return p.q.p + (int64_t)s * p.q.seq + (int64_t)(h * p.G + m / p.Bt) * p.q.head + (int64_t)(m % p.Bt) * p.q.token;
}

// The shared part: one workgroup, its piece of the list
template <int D, int CB>
__device__ void shared_part(const BranchParams &p, const Plan &plan, unsigned char *smem)
{
    constexpr int NC = D / 32, NDB = D / 16, UPR = D / 8, ROWB = D * 2, RPL = 64 / UPR, NV = TK / RPL, R = 16 * CB;
    __shared__ float2 ml_s[NW][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const int Mt = p.G * p.Bt, M = p.fan * Mt, blocks = (M + R - 1) / R, nt = (p.prefix_len + TK - 1) / TK;
    int at = (int)blockIdx.x * plan.shared_chunk;
    const int end = min(at + plan.shared_chunk, plan.shared_tiles);
    unsigned char *vt = smem + (size_t)wave * TK * ROWB;
    float *outs = reinterpret_cast<float *>(smem);   // the waves' outputs of one block of 16 rows, where their V tiles were
    while (at < end) {
        const int seg = at / nt, t0 = at - seg * nt, t1 = min(nt, t0 + end - at);
        at += t1 - t0;
        const int ch = seg / blocks, mb = seg - ch * blocks, c = ch / p.hkv, h = ch - c * p.hkv;
        const uint16_t *kh = p.k_prefix + (size_t)ch * p.prefix_cap * D, *vh = p.v_prefix + (size_t)ch * p.prefix_cap * D;
        State<D, CB> st;
        st.reset();
        u32x4 kr[2][NC], vr[NV];
        // rows past the last repeat it: finite data whose weights are masked to zero
        auto load_k = [&](int t) {
#pragma unroll
            for (int kg = 0; kg < 2; ++kg) {
                const uint16_t *kb = kh + (size_t)min(t * TK + 16 * kg + c16, p.prefix_len - 1) * D + 8 * g;
#pragma unroll
                for (int cc = 0; cc < NC; ++cc) kr[kg][cc] = *reinterpret_cast<const u32x4 *>(kb + cc * 32);
            }
        };
        auto load_v = [&](int t) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                vr[i] = *reinterpret_cast<const u32x4 *>(vh + (size_t)min(t * TK + i * RPL + lane / UPR, p.prefix_len - 1) * D + (lane % UPR) * 8);
        };
        int t = t0 + wave;
        if (t < t1) {
            load_k(t);
            load_v(t);
        }
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const int m = min(mb * R + 16 * cb + c16, M - 1);
            const uint16_t *qr = query_row(p, c * p.fan + m / Mt, h, m % Mt) + 8 * g;
#pragma unroll
            for (int cc = 0; cc < NC; ++cc) st.q[cb][cc] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qr + cc * 32));
        }
        for (; t < t1; t += NW) {
            tile_step<D, CB>(
                st, kr, vr, vt, p.scale_log2e, lane,
                [&]() {
                    if (t + NW < t1) {
                        load_k(t + NW);
                        load_v(t + NW);
                    }
                },
                [&](f32x4 (&s)[CB][2]) {
                    if ((t + 1) * TK > p.prefix_len) {   // uniform
                        const int lim = p.prefix_len - t * TK - 4 * g;
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                            for (int kg = 0; kg < 2; ++kg)
#pragma unroll
                                for (int i = 0; i < 4; ++i) s[cb][kg][i] = 16 * kg + i < lim ? s[cb][kg][i] : -INFINITY;
                    }
                });
        }
        // the eight results become one, a block of 16 rows at a time
        const size_t slot = (size_t)blockIdx.x + seg;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const float l = sum_over_rows(st.l[cb]);
            __syncthreads();
            float *ow = outs + (size_t)wave * 16 * D;
#pragma unroll
            for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4 *>(ow + c16 * D + 16 * db + 4 * g) = st.o[cb][db];
            if (g == 0) ml_s[wave][c16] = make_float2(st.m[cb], l);
            __syncthreads();
            const int rows = min(16, M - mb * R - 16 * cb);
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
                    const f32x4 o = *reinterpret_cast<const f32x4 *>(outs + ((size_t)w * 16 + m) * D + d0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i] += f * o[i];
                    L += f * ml.y;
                }
                const float inv = L > 0.f ? 1.f / L : 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] *= inv;
                *reinterpret_cast<f32x4 *>(p.part_o + (slot * R + 16 * cb + m) * D + d0) = acc;
                if (d0 == 0) p.part_ml[slot * R + 16 * cb + m] = make_float2(mx, L);
            }
        }
        __syncthreads();   // the outputs are read before the next segment's V tiles overwrite them
    }
}

// The own part: one wave, its piece of the list.  `slots`: slots and rows of the shared part, behind which the own part's lie.
template <int D, int CB>
__device__ void own_part(const BranchParams &p, const Plan &plan, int own_wave, float *part_o, float2 *part_ml, unsigned char *vt)
{
    constexpr int NC = D / 32, NDB = D / 16, UPR = D / 8, RPL = 64 / UPR, NV = TK / RPL, R = 16 * CB;
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int Mt = p.G * p.Bt, blocks = (Mt + R - 1) / R, shift = p.pages.page_shift;
    int at = own_wave * plan.own_chunk;
    const int end = min(at + plan.own_chunk, plan.own_tiles);
    if (at >= end) return;
    // the sequence whose tiles hold tile `at`: `first` its first tile in the list
    int s = 0, first = 0, seg_of_s = 0;
    for (int base = 0; base < p.n_seqs; base += 64) {
        const int mine = base + lane < p.n_seqs ? (own_rows(p, base + lane) + TK - 1) / TK * p.hkv * blocks : 0;
        int upto = mine;   // inclusive sum over the lanes
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (first + all > at) {
            const uint64_t past = __builtin_amdgcn_ballot_w64(first + upto > at);
            const int k = __builtin_ctzll(past);
            s = base + k;
            first += __builtin_amdgcn_readlane(upto, k) - __builtin_amdgcn_readlane(mine, k);
            break;
        }
        first += all;
    }
    seg_of_s = s * p.hkv * blocks;
    while (at < end) {
        const int n = own_rows(p, s), nt = (n + TK - 1) / TK;   // uniform
        if (at >= first + nt * p.hkv * blocks) {
            first += nt * p.hkv * blocks;
            ++s;
            seg_of_s += p.hkv * blocks;
            continue;
        }
        const int local = (at - first) / nt, t0 = at - first - local * nt, t1 = min(nt, t0 + end - at);
        at += t1 - t0;
        const int h = local / blocks, mb = local - h * blocks;
        const int len = p.pages.lens[s];
        const int32_t *table = p.pages.table + (size_t)s * p.pages.width;
        State<D, CB> st;
        st.reset();
        int vis[CB];   // rows [0, vis) are seen by the lane's query
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const int m = min(mb * R + 16 * cb + c16, Mt - 1);
            vis[cb] = min(len + m % p.Bt + 1, n);
            const uint16_t *qr = query_row(p, s, h, m) + 8 * g;
#pragma unroll
            for (int cc = 0; cc < NC; ++cc) st.q[cb][cc] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qr + cc * 32));
        }
        u32x4 kr[2][NC], vr[NV];
        uint32_t absent = 0;   // bit i: rows 8 i .. of the tile in registers lie on a page that does not exist
        // A tile's rows lie in groups of eight on one page each (pages have a multiple of eight rows).  The numbers of its pages are
        // requested a tile ahead of its rows.  Rows past the last repeat it.
        int pages[4];
        auto look_up = [&](int t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) pages[i] = table[min(t * TK + 8 * i, n - 1) >> shift];
        };
        auto load = [&](int t) {
            const uint16_t *kg8[4], *vg8[4];   // first row of each group, head h
            absent = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = min(t * TK + 8 * i, (n - 1) & ~7);
                int page = __builtin_amdgcn_readfirstlane(pages[i]);
                if ((uint32_t)page >= (uint32_t)p.pages.n_pages) {
                    absent |= 1u << i;
                    page = 0;
                }
                const size_t off = ((((size_t)page * p.hkv + h) << shift) + (size_t)(row & ((1 << shift) - 1))) * D;
                kg8[i] = p.pages.k + off;
                vg8[i] = p.pages.v + off;
            }
            const int last = n - 1;
#pragma unroll
            for (int kg = 0; kg < 2; ++kg) {
                const int row = t * TK + 16 * kg + c16, in8 = min(row, last) & 7;
                const uint16_t *kb = (c16 < 8 ? kg8[2 * kg] : kg8[2 * kg + 1]) + in8 * D + 8 * g;
#pragma unroll
                for (int cc = 0; cc < NC; ++cc) kr[kg][cc] = *reinterpret_cast<const u32x4 *>(kb + cc * 32);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int row = t * TK + i * RPL + lane / UPR, in8 = min(row, last) & 7;
                vr[i] = *reinterpret_cast<const u32x4 *>(vg8[i * RPL / 8] + in8 * D + (lane % UPR) * 8);
            }
            if (absent) {   // (values of such rows may be anything: their weight is zero, and so are they)
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (absent >> (i * RPL / 8) & 1) vr[i] = u32x4{0u, 0u, 0u, 0u};
            }
        };
        look_up(t0);
        load(t0);
        look_up(t0 + 1);
        for (int t = t0; t < t1; ++t) {
            const uint32_t hidden = absent;
            tile_step<D, CB>(
                st, kr, vr, vt, p.scale_log2e, lane,
                [&]() {
                    if (t + 1 < t1) {
                        load(t + 1);
                        look_up(t + 2);
                    }
                },
                [&](f32x4 (&sc)[CB][2]) {
                    if ((t + 1) * TK > min(len, n) || hidden) {   // uniform: rows that not every query sees
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb) {
                            const int lim = vis[cb] - t * TK - 4 * g;
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
        const size_t slot = (size_t)own_wave + seg_of_s + local;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const float L = sum_over_rows(st.l[cb]), inv = L > 0.f ? 1.f / L : 0.f;
            if (mb * R + 16 * cb + c16 < Mt) {
                float *ow = part_o + (slot * R + 16 * cb + c16) * D;
#pragma unroll
                for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4 *>(ow + 16 * db + 4 * g) = st.o[cb][db] * inv;
                if (g == 0) part_ml[slot * R + 16 * cb + c16] = make_float2(st.m[cb], L);
            }
        }
    }
}

// Slots of the shared part at most: one per workgroup and segment end
__host__ __device__ inline size_t shared_slots(int n_prefixes, int fan, int hkv, int Mt, int R, int wgs)
{
    return (size_t)n_prefixes * hkv * ((fan * Mt + R - 1) / R) + wgs;
}

template <int D, int CBS, int CBO>
__global__ __launch_bounds__(64 * NW) void branch_main_kernel(BranchParams p)
{
    __shared__ __attribute__((aligned(16))) unsigned char smem[NW * TK * D * 2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int Mt = p.G * p.Bt, M = p.fan * Mt;
    const int wgs = (int)gridDim.x;
    // ---- the lists and how they are dealt: the same on every wave
    Plan plan;
    int own = 0;
    for (int base = 0; base < p.n_seqs; base += 64) own += base + lane < p.n_seqs ? (own_rows(p, base + lane) + TK - 1) / TK : 0;
    plan.own_tiles = __builtin_amdgcn_readfirstlane(wave_sum(own)) * p.hkv * ((Mt + 16 * CBO - 1) / (16 * CBO));
    plan.shared_tiles = (p.prefix_len + TK - 1) / TK * p.n_prefixes * p.hkv * ((M + 16 * CBS - 1) / (16 * CBS));
    {
        const float s = (float)plan.shared_tiles, o = (float)plan.own_tiles;
        int w = s > 0.f ? (int)(wgs * (s / (s + o)) + 0.5f) : 0;
        if (plan.shared_tiles > 0) w = max(w, 1);
        if (plan.own_tiles > 0) w = min(w, wgs - 1);
        plan.shared_chunk = w > 0 ? (plan.shared_tiles + w - 1) / w : 1;
        plan.shared_wgs = (plan.shared_tiles + plan.shared_chunk - 1) / plan.shared_chunk;
        const int waves = max((wgs - plan.shared_wgs) * NW, 1);
        plan.own_chunk = max((plan.own_tiles + waves - 1) / waves, 1);
    }
    if (blockIdx.x == 0) {   // ... for the merge
        if (tid == 0) {
            p.plan[0] = plan.shared_chunk;
            p.plan[1] = plan.own_chunk;
            p.plan[2] = plan.own_tiles;
        }
        if (wave == 0) {
            int first = 0;
            for (int base = 0; base < p.n_seqs; base += 64) {
                const int mine = base + lane < p.n_seqs ? (own_rows(p, base + lane) + TK - 1) / TK : 0;
                int upto = mine;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int o = __shfl_up(upto, d);
                    if (lane >= d) upto += o;
                }
                if (base + lane < p.n_seqs) p.plan[BRANCH_PLAN_WORDS + base + lane] = first + upto - mine;
                first += __builtin_amdgcn_readlane(upto, 63);
            }
        }
    }
    if ((int)blockIdx.x < plan.shared_wgs) {
        shared_part<D, CBS>(p, plan, smem);
    } else {
        const size_t rows = shared_slots(p.n_prefixes, p.fan, p.hkv, Mt, 16 * CBS, wgs) * (16 * CBS);
        own_part<D, CBO>(p, plan, ((int)blockIdx.x - plan.shared_wgs) * NW + wave, p.part_o + rows * D, p.part_ml + rows,
                         smem + (size_t)wave * TK * D * 2);
    }
}

// The join of a row's pieces: `groups` groups of D / 4 threads take a row's pieces in turn, four at a time, and join what they have
// in LDS.  (Groups: where there are few rows and many pieces, the pieces requested one behind another were all the time this took: one
// sequence, 8192 shared rows, 17.7 us with one group a row.)
template <int D, int CBS, int CBO>
__global__ __launch_bounds__(256) void branch_merge_kernel(BranchParams p, int wgs, int groups)
{
    constexpr int TPR = D / 4, RS = 16 * CBS, RO = 16 * CBO, BATCH = 4;
    __shared__ f32x4 acc_s[256];
    __shared__ float2 ml_s[256 / TPR];
    const int Mt = p.G * p.Bt;
    const int unit = (int)threadIdx.x / TPR, group = unit % groups;
    const int64_t row = (int64_t)blockIdx.x * (256 / TPR / groups) + unit / groups;
    const int d0 = (int)threadIdx.x % TPR * 4;
    const bool exists = row < (int64_t)p.n_seqs * p.hkv * Mt;
    const int sh = exists ? (int)(row / Mt) : 0, m = exists ? (int)(row - (int64_t)sh * Mt) : 0, s = sh / p.hkv, h = sh - s * p.hkv;
    const bool wanted = exists && m % p.Bt < new_of(p, s);   // else left as it was
    // the pieces: slots a0 .. of the shared part, b0 .. of the own part
    int a0 = 0, na = 0, b0 = 0, nb = 0, am = 0, bm = 0;
    if (wanted) {
        if (p.prefix_len > 0) {
            const int c = s / p.fan, mm = (s - c * p.fan) * Mt + m, blocks = (p.fan * Mt + RS - 1) / RS, nt = (p.prefix_len + TK - 1) / TK;
            const int seg = (c * p.hkv + h) * blocks + mm / RS, chunk = p.plan[0];
            am = mm % RS;
            a0 = seg * nt / chunk;
            na = ((seg + 1) * nt - 1) / chunk + 1 - a0;
            a0 += seg;
        }
        const int n = own_rows(p, s);
        if (n > 0) {
            const int blocks = (Mt + RO - 1) / RO, nt = (n + TK - 1) / TK, chunk = p.plan[1];
            const int local = h * blocks + m / RO, first = p.plan[BRANCH_PLAN_WORDS + s] * p.hkv * blocks + local * nt;
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
            const size_t at = i < na ? (size_t)(a0 + i) * RS + am : rows + (size_t)(b0 + i - na) * RO + bm;
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
}

// Blocks of 16 query rows a wave takes: two where there are more than 16 rows
int col_blocks(int rows) { return rows > 16 ? 2 : 1; }

}  // namespace

size_t branch_workspace(int n_seqs, int n_prefixes, int hkv, int G, int Bt, int D, int cus, size_t *off_ml, size_t *off_plan)
{
    const size_t Mt = (size_t)G * Bt, fan = n_prefixes > 0 ? (size_t)n_seqs / n_prefixes : 0;
    const size_t RS = 16 * (size_t)col_blocks((int)(fan * Mt < 64 ? fan * Mt : 64)), RO = 16 * (size_t)col_blocks((int)(Mt < 64 ? Mt : 64));
    const size_t shared = shared_slots(n_prefixes, (int)fan, hkv, (int)Mt, (int)RS, cus) * RS;
    const size_t own = ((size_t)n_seqs * hkv * ((Mt + RO - 1) / RO) + (size_t)cus * NW) * RO;
    size_t off = (shared + own) * D * 4;
    off = (off + 255) & ~(size_t)255;
    *off_ml = off;
    off += ((shared + own) * 8 + 255) & ~(size_t)255;
    *off_plan = off;
    off += ((size_t)(BRANCH_PLAN_WORDS + n_seqs) * 4 + 255) & ~(size_t)255;
    return off;
}

hipError_t launch_branch_attention(const BranchParams &p, hipStream_t s)
{
    const int Mt = p.G * p.Bt, cbs = p.prefix_len > 0 ? col_blocks(p.fan * Mt) : 1, cbo = col_blocks(Mt);
    const int wgs = p.cus;
    const int64_t rows = (int64_t)p.n_seqs * p.hkv * Mt;
    const int units = 256 / (p.D / 4);
    int groups = 1;   // as many as the chip's threads hold at once, and no more than a workgroup
    while (groups < units && rows * (p.D / 4) * groups * 2 <= (int64_t)p.cus * 2048) groups *= 2;
    const int per = units / groups;
    const dim3 merge_grid((unsigned)((rows + per - 1) / per));
#define KD_GO(D, S, O)                                                                                        \
    {                                                                                                         \
        hipLaunchKernelGGL((branch_main_kernel<D, S, O>), dim3(wgs), dim3(64 * NW), 0, s, p);                 \
        const hipError_t e = hipGetLastError();                                                               \
        if (e != hipSuccess) return e;                                                                        \
        hipLaunchKernelGGL((branch_merge_kernel<D, S, O>), merge_grid, dim3(256), 0, s, p, wgs, groups);              \
        return hipGetLastError();                                                                             \
    }
#define KD_GO_D(D)                                    \
    if (cbs == 1 && cbo == 1) KD_GO(D, 1, 1)          \
    if (cbs == 2 && cbo == 1) KD_GO(D, 2, 1)          \
    if (cbs == 1 && cbo == 2) KD_GO(D, 1, 2)          \
    KD_GO(D, 2, 2)
    if (p.D == 128) { KD_GO_D(128) }
    if (p.D == 64) { KD_GO_D(64) }
#undef KD_GO_D
#undef KD_GO
    return hipErrorInvalidValue;
}

}  // namespace kd
