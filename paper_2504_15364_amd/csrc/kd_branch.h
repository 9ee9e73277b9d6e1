// Launcher interface of the operators around the block step: norms and rotation of queries and keys, rows appended to the pages
// of the sequences that continue a prompt, and the attention that reads those pages and the prompt's cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kd {

// ------------------------------------------------------------------ norms and rotation
// bf16 rows of head_dim values: row (sequence, head, token) begins at p + sequence * seq + head * head + token * token (elements)
struct Rows {
    const uint16_t *p;
    int64_t seq, head, token;
};
// What is done to queries and keys: root mean square norm with learned weights (q_w null: none), then the rotation (cos_t null: none)
struct RowForm {
    const uint16_t *q_w, *k_w;   // [D], or [heads][D] with the stride of a head
    int32_t q_w_head, k_w_head;
    const float *cos_t, *sin_t;  // [table_rows][D / 2]
    int64_t table_rows;
    float eps;
};
// The pages of the sequences' own rows
struct Pages {
    uint16_t *k, *v;             // [n_pages][hkv][page_rows][D]
    const int32_t *table;        // [n_seqs][width]
    const int32_t *lens;         // [n_seqs] rows held; negative: the sequence is not in use
    const int32_t *n_new;        // nullable [n_seqs]
    int32_t page_shift, n_pages, width;
};
struct NormRopeParams {
    Rows q, k, v;                // (v: append only)
    uint16_t *q_out, *k_out;     // [n_seqs][heads][Bt][D]
    RowForm form;
    const int32_t *positions;    // norm_rope: nullable [n_seqs][Bt]; append: [n_seqs], the position of a sequence's first own row
    int64_t pos0;
    Pages pages;                 // append only
    int32_t *status;             // nullable: bits of tokens that were left out
    int32_t n_seqs, hq, hkv, Bt, D;
};
constexpr int LEFT_OUT_POSITION = 1, LEFT_OUT_ROW = 2;
hipError_t launch_norm_rope(const NormRopeParams &p, hipStream_t s);
hipError_t launch_branch_append(const NormRopeParams &p, hipStream_t s);

// The blocks of up to NORM_ROPE_LAYERS layers of one shape, contiguous tensors, in one launch
constexpr int NORM_ROPE_LAYERS = 32;
struct NormRopeLayer {
    const uint16_t *q, *k;
    uint16_t *q_out, *k_out;
    RowForm form;
};
struct NormRopeLayers {
    NormRopeLayer layer[NORM_ROPE_LAYERS];
    int32_t layers, batch, hq, hkv, Bt, D;
    int64_t pos0;
};
hipError_t launch_norm_rope_layers(const NormRopeLayers &p, hipStream_t s);

// ------------------------------------------------------------------ attention of sequences that share a prompt's cache
// Quotients of numbers below 2^31 by a number that the host knows (three instructions; the compiler's division, some forty that wait for one
// another, eleven of them ahead of a launch's first loads, took 1.5 us).  Division by an invariant number as by Granlund and Montgomery: with s
// the bits of d - 1 and mul = 2^32 (2^s - d) / d + 1 rounded down, n / d = (n mul / 2^32 + n) / 2^s, whose sum stays below 2^32.
struct Divisor {
    uint32_t mul, shift;
    void set(uint32_t d)
    {
        shift = 0;
        while ((1ull << shift) < d) ++shift;
        mul = (uint32_t)((((1ull << shift) - d) << 32) / d + 1);
    }
    __host__ __device__ __forceinline__ int divide(int n) const
    {
        return (int)(((uint32_t)(((uint64_t)(uint32_t)n * mul) >> 32) + (uint32_t)n) >> shift);
    }
};
struct BranchParams {
    Rows q;
    uint16_t *out;                        // [n_seqs][hq][Bt][D]
    const uint16_t *k_prefix, *v_prefix;  // [n_prefixes][hkv][prefix_cap][D]
    Pages pages;
    float *part_o;                        // partial outputs, each normalised by its weight sum: slot by slot
    float2 *part_ml;                      // (reference maximum in log2 units, weight sum) of every row of a slot
    int32_t *plan;                        // [BRANCH_PLAN_WORDS + n_seqs]: how the launch cut the work, for the merge
    int32_t n_seqs, n_prefixes, fan, hkv, G, Bt, D;
    int32_t prefix_len;
    int64_t prefix_cap;
    int32_t cus;
    float scale_log2e;
    int32_t shared_segs;                  // (prompt, head, block of rows) segments of the shared part; 0: there is none
    Divisor by_segs, by_heads, by_hkv, by_Mt, by_Bt, by_fan, by_own_blocks;   // heads: n_prefixes hkv; Mt: G Bt
};
constexpr int BRANCH_PLAN_WORDS = 8;
size_t branch_workspace(int n_seqs, int n_prefixes, int hkv, int G, int Bt, int D, int cus, size_t *off_ml, size_t *off_plan);
hipError_t launch_branch_attention(const BranchParams &p, hipStream_t s);   // (it fills in segments and divisors)

}  // namespace kd
