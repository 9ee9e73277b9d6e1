// Norms of queries and keys for each head and the rotary position embedding, in one pass; the same on rows that go into pages.
//
//   u_i = x_i w_i / sqrt(mean_j x_j^2 + eps)                                     (per token and head; w: learned weights)
//   y_i = u_i cos - u_(i+h) sin,   y_(i+h) = u_(i+h) cos + u_i sin,   h = D / 2   (angle of position and pair i)
//
// all in float, every product and sum rounded on its own, the result rounded once to bf16.  (Two passes would round u as well.)
//
// What bounds it: 2 D bytes read and 2 D written a row; the tables (4 D bytes a token) and weights are shared by rows and come out
// of the caches.  A lane takes the same 16-byte unit of both halves of a row: the pairs of the rotation are its own, and the norm
// is one sum over the 8 (D = 64: 4) lanes of a row.  A workgroup's lanes stand for TG tokens x 32 / TG heads (D = 64: 64 / TG): with
// many tokens the rows of a head written together are one contiguous piece, with one token all heads are taken at once.
#include "kd_branch.h"

namespace kd {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x)
{
    return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xF, 0xF, false));
}

// sum over the LANES (4 or 8) consecutive lanes of a row
template <int LANES>
__device__ __forceinline__ float row_sum(float x)
{
    x = dpp_add<0xB1>(x);                     // quad_perm [1,0,3,2]
    x = dpp_add<0x4E>(x);                     // quad_perm [2,3,0,1]
    if (LANES == 8) x = dpp_add<0x141>(x);    // row_half_mirror
    return x;
}

__device__ __forceinline__ float unpack(u32x4 w, int e)
{
    return __uint_as_float(e & 1 ? (w[e / 2] & 0xFFFF0000u) : (w[e / 2] << 16));
}

__device__ __forceinline__ u32x4 pack(const float (&y)[8])
{
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        o[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y[2 * i]) | ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y[2 * i + 1]) << 16);
    return o;
}

// One row: `unit` is the lane's 16-byte unit of either half; cs, sn: the table row of the token's position; w: the head's weights (null: no norm)
template <int D>
__device__ __forceinline__ void form_row(const uint16_t *src, uint16_t *dst, const uint16_t *w, const f32x4 (&c)[2], const f32x4 (&s)[2],
                                         bool rotate, float eps, int unit)
{
    const u32x4 a = *reinterpret_cast<const u32x4 *>(src + unit * 8);
    const u32x4 b = *reinterpret_cast<const u32x4 *>(src + D / 2 + unit * 8);
    float x1[8], x2[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x1[i] = unpack(a, i);
        x2[i] = unpack(b, i);
    }
    if (w) {   // uniform over the launch
        const u32x4 wa = *reinterpret_cast<const u32x4 *>(w + unit * 8), wb = *reinterpret_cast<const u32x4 *>(w + D / 2 + unit * 8);
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sq += x1[i] * x1[i] + x2[i] * x2[i];
        sq = row_sum<D / 16>(sq);
        const float r = 1.f / sqrtf(sq * (1.f / D) + eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x1[i] = x1[i] * r * unpack(wa, i);
            x2[i] = x2[i] * r * unpack(wb, i);
        }
    }
    float y1[8], y2[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float cc = c[i / 4][i % 4], ss = s[i / 4][i % 4];
        y1[i] = rotate ? x1[i] * cc - x2[i] * ss : x1[i];
        y2[i] = rotate ? x2[i] * cc + x1[i] * ss : x2[i];
    }
    *reinterpret_cast<u32x4 *>(dst + unit * 8) = pack(y1);
    *reinterpret_cast<u32x4 *>(dst + D / 2 + unit * 8) = pack(y2);
}

template <int D>
__device__ __forceinline__ void load_angles(const RowForm &f, int64_t position, int unit, f32x4 (&c)[2], f32x4 (&s)[2])
{
    const float *cs = f.cos_t + position * (D / 2) + unit * 8, *sn = f.sin_t + position * (D / 2) + unit * 8;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        c[i] = *reinterpret_cast<const f32x4 *>(cs + 4 * i);
        s[i] = *reinterpret_cast<const f32x4 *>(sn + 4 * i);
    }
}

// The token and the heads of a group of D / 16 lanes: token blockIdx.x * tg + (group % tg), heads first, first + step, ... of `chunk` rounds
struct Place {
    int unit, first, step, token;
};
template <int D>
__device__ __forceinline__ Place place_of(int tg_shift, int chunk)
{
    constexpr int UPH = D / 16, GROUPS = 256 / UPH;
    const int group = (int)threadIdx.x / UPH, tg = 1 << tg_shift;
    Place at;
    at.unit = (int)threadIdx.x % UPH;
    at.step = GROUPS >> tg_shift;
    at.first = (int)blockIdx.y * chunk * at.step + (group >> tg_shift);
    at.token = (int)blockIdx.x * tg + (group & (tg - 1));
    return at;
}

// APPEND: keys and values go to the rows behind those that the token's sequence holds, in its pages, queries to q_out.  A token that
// has no place -- its sequence not in use, behind the sequence's new tokens, its position not in the tables, its row or page not in
// the table or the pool -- is left out: nothing of it is written, and of the last two the caller's status word tells.
template <int D, bool APPEND>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormRopeParams p, int tg_shift, int chunk)
{
    const Place at = place_of<D>(tg_shift, chunk);
    if (at.token >= p.n_seqs * p.Bt) return;
    const int seq = at.token / p.Bt, j = at.token % p.Bt;
    auto left_out = [&](int bit) {   // (one lane a token)
        if (p.status && at.unit == 0 && at.first == 0) atomicOr(p.status, bit);
    };
    int64_t position;
    size_t page_at = 0;   // APPEND: element offset of head 0's row in the pools
    if constexpr (APPEND) {
        const int len = p.pages.lens[seq];
        if (len < 0 || (p.pages.n_new && j >= p.pages.n_new[seq])) return;
        const int64_t row = (int64_t)len + j;
        const int64_t at_page = row >> p.pages.page_shift;
        if (at_page >= p.pages.width) return left_out(LEFT_OUT_ROW);
        const int page = p.pages.table[(size_t)seq * p.pages.width + at_page];
        if ((uint32_t)page >= (uint32_t)p.pages.n_pages) return left_out(LEFT_OUT_ROW);
        page_at = ((((size_t)page * p.hkv) << p.pages.page_shift) + (size_t)(row & ((1 << p.pages.page_shift) - 1))) * D;
        position = (p.positions ? (int64_t)p.positions[seq] : 0) + row;
    } else {
        position = p.positions ? (int64_t)p.positions[at.token] : p.pos0 + j;
    }
    const bool rotate = p.form.cos_t != nullptr;
    f32x4 c[2], s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) c[i] = s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (rotate) {
        if (position < 0 || position >= p.form.table_rows) return left_out(LEFT_OUT_POSITION);
        load_angles<D>(p.form, position, at.unit, c, s);
    }
    const int heads = p.hq + p.hkv + (APPEND ? p.hkv : 0);
    for (int i = 0, h = at.first; i < chunk && h < heads; ++i, h += at.step) {
        if (h < p.hq) {
            const uint16_t *src = p.q.p + seq * p.q.seq + h * p.q.head + j * p.q.token;
            uint16_t *dst = p.q_out + (((size_t)seq * p.hq + h) * p.Bt + j) * D;
            form_row<D>(src, dst, p.form.q_w ? p.form.q_w + (size_t)h * p.form.q_w_head : nullptr, c, s, rotate, p.form.eps, at.unit);
        } else if (h < p.hq + p.hkv) {
            const int hk = h - p.hq;
            const uint16_t *src = p.k.p + seq * p.k.seq + hk * p.k.head + j * p.k.token;
            uint16_t *dst = APPEND ? p.pages.k + page_at + (((size_t)hk << p.pages.page_shift) * D)
                                   : p.k_out + (((size_t)seq * p.hkv + hk) * p.Bt + j) * D;
            form_row<D>(src, dst, p.form.k_w ? p.form.k_w + (size_t)hk * p.form.k_w_head : nullptr, c, s, rotate, p.form.eps, at.unit);
        } else if constexpr (APPEND) {
            const int hv = h - p.hq - p.hkv;
            const uint16_t *src = p.v.p + seq * p.v.seq + hv * p.v.head + j * p.v.token;
            uint16_t *dst = p.pages.v + page_at + (((size_t)hv << p.pages.page_shift) * D);
            const u32x4 a = *reinterpret_cast<const u32x4 *>(src + at.unit * 8), b = *reinterpret_cast<const u32x4 *>(src + D / 2 + at.unit * 8);
            *reinterpret_cast<u32x4 *>(dst + at.unit * 8) = a;
            *reinterpret_cast<u32x4 *>(dst + D / 2 + at.unit * 8) = b;
        }
    }
}

template <int D>
__global__ __launch_bounds__(256) void norm_rope_layers_kernel(NormRopeLayers p, int tg_shift, int chunk)
{
    const NormRopeLayer &l = p.layer[blockIdx.z];
    const Place at = place_of<D>(tg_shift, chunk);
    if (at.token >= p.batch * p.Bt) return;
    const int seq = at.token / p.Bt, j = at.token % p.Bt;
    const bool rotate = l.form.cos_t != nullptr;
    f32x4 c[2], s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) c[i] = s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (rotate) load_angles<D>(l.form, p.pos0 + j, at.unit, c, s);
    for (int i = 0, h = at.first; i < chunk && h < p.hq + p.hkv; ++i, h += at.step) {
        const bool isk = h >= p.hq;
        const int hh = isk ? h - p.hq : h;
        const size_t row = (((size_t)seq * (isk ? p.hkv : p.hq) + hh) * p.Bt + j) * D;
        const uint16_t *w = isk ? l.form.k_w : l.form.q_w;
        form_row<D>((isk ? l.k : l.q) + row, (isk ? l.k_out : l.q_out) + row,
                    w ? w + (size_t)hh * (isk ? l.form.k_w_head : l.form.q_w_head) : nullptr, c, s, rotate, l.form.eps, at.unit);
    }
}

// Tokens a workgroup stands for (a power of two), rounds of heads a lane takes, and the grid.  Rounds share the token's angles, and their
// rows of a projection's output lie together: with one round a workgroup the 32768 tokens of a prompt (40 heads, 128 wide) take 180 us, with
// eight 149, with sixteen 168.  But no more rounds than leave `wgs` workgroups: 2048 fill the chip; where sequences take
// fewer tokens than Bt, many workgroups have nothing to do, and four times as many are wanted (24 pieces of up to 300 tokens 25.8 -> 20.7 us;
// eight of 1000 given tokens would go from 47 to 53).
struct Shape {
    int tg_shift, chunk;
    dim3 grid;
};
Shape shape_of(int64_t tokens, int heads, int D, int layers, int64_t wgs = 2048)
{
    const int groups = 256 / (D / 16);
    Shape f;
    f.tg_shift = 0;
    while ((1 << f.tg_shift) < groups && (1 << f.tg_shift) < tokens) ++f.tg_shift;
    const int step = groups >> f.tg_shift, rounds = (heads + step - 1) / step;
    const int64_t wide = (tokens + (1 << f.tg_shift) - 1) >> f.tg_shift;
    f.chunk = 1;
    while (f.chunk < 8 && f.chunk < rounds && wide * ((rounds + f.chunk - 1) / f.chunk) * layers > wgs) f.chunk *= 2;
    f.grid = dim3((unsigned)wide, (unsigned)((rounds + f.chunk - 1) / f.chunk), (unsigned)layers);
    return f;
}

}  // namespace

hipError_t launch_norm_rope(const NormRopeParams &p, hipStream_t s)
{
    const Shape f = shape_of((int64_t)p.n_seqs * p.Bt, p.hq + p.hkv, p.D, 1);
    if (p.D == 128) hipLaunchKernelGGL((norm_rope_kernel<128, false>), f.grid, dim3(256), 0, s, p, f.tg_shift, f.chunk);
    else if (p.D == 64) hipLaunchKernelGGL((norm_rope_kernel<64, false>), f.grid, dim3(256), 0, s, p, f.tg_shift, f.chunk);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

hipError_t launch_branch_append(const NormRopeParams &p, hipStream_t s)
{
    const Shape f = shape_of((int64_t)p.n_seqs * p.Bt, p.hq + 2 * p.hkv, p.D, 1, p.pages.n_new ? 8192 : 2048);
    if (p.D == 128) hipLaunchKernelGGL((norm_rope_kernel<128, true>), f.grid, dim3(256), 0, s, p, f.tg_shift, f.chunk);
    else if (p.D == 64) hipLaunchKernelGGL((norm_rope_kernel<64, true>), f.grid, dim3(256), 0, s, p, f.tg_shift, f.chunk);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

hipError_t launch_norm_rope_layers(const NormRopeLayers &p, hipStream_t s)
{
    if (p.layers < 1 || p.layers > NORM_ROPE_LAYERS) return hipErrorInvalidValue;
    const Shape f = shape_of((int64_t)p.batch * p.Bt, p.hq + p.hkv, p.D, p.layers);
    if (p.D == 128) hipLaunchKernelGGL((norm_rope_layers_kernel<128>), f.grid, dim3(256), 0, s, p, f.tg_shift, f.chunk);
    else if (p.D == 64) hipLaunchKernelGGL((norm_rope_layers_kernel<64>), f.grid, dim3(256), 0, s, p, f.tg_shift, f.chunk);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace kd
