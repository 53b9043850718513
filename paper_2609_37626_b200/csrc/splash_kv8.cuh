// Shared by the kernels of the cache that keeps keys and values per head in e4m3 with a scale per (page, head).
#pragma once

#include <cuda_fp16.h>

#include "splash_common.cuh"

namespace splash {
namespace kv8 {

constexpr int kMinExp = -100;     // scales that an append writes are at least 2^-100 (and their reciprocals are finite)

// four e4m3 codes -> fp16 values (every e4m3 value is an fp16 value), the codes' order kept
__device__ __forceinline__ void to_f16x4(uint32_t codes, uint32_t &lo, uint32_t &hi) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(codes));
}
// two fp32 values -> two e4m3 codes, nearest even, above 448 -> 448, NaN -> NaN
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

constexpr float kLift = 7.f, kSlack = 8.f;          // softmax weights are kept below 2^(kLift + kSlack) = 2^15
constexpr float kUnset = -1e38f;                    // reference of a row that has seen no token: any logit is far above it

// ---- attention -----------------------------------------------------------------------------------------------------------

struct AttnParams {
    const void *q;
    void *out;
    float *lse;
    const int32_t *table, *seq_lens, *q_start, *kv_begin, *kv_end;
    const float *k_scales, *v_scales;
    int64_t q_row, q_head, out_row, out_head, lse_row, table_stride, k_scale_stride, v_scale_stride;
    int64_t max_tokens;               // 64 * table width: a context is cut there
    int32_t B, T, group, kv_heads, num_pages, max_rows;
    int32_t q_bf16, out_f32;
    int32_t whole;                    // 1: no piece of work is cut, and no combine kernel follows
    int32_t workers;
    int32_t clear_status;             // 1: no kernel of the call in front has cleared the error words (the decode kernel does)
    int32_t min_pairs, max_pairs;     // requests with this many (row, head of the group) pairs are this kernel's
    float scale_log2;                 // softmax scale times log2 e
    // workspace
    int32_t *status;                  // 16 ints
    int4 *cut;                        // [workers][2]: {pieces, first query row, pairs, first pair of the tile}, {key head, 0, 0, 0} of the cut item
                                      // whose first piece the worker has; pieces = 0: none
    float *part_lse;                  // [2 workers][rows], base 2
    float *part_out;                  // [2 workers][rows][D]
};

// Query rows, token range and pages of request i.
struct Request {
    int row0, rows, rows_all;         // first row; rows computed; rows that the request has (they place the rows)
    int len, lo, hi, pairs;           // context; token range of the last row; (row, head) pairs
    __device__ __forceinline__ int pages() const { return hi > lo ? (hi + kPage - 1) / kPage - lo / kPage : 0; }
};

__device__ __forceinline__ Request request(const AttnParams &p, int i) {
    Request r;
    if (p.q_start != nullptr) {
        const int a = load_l2(p.q_start + i), b = load_l2(p.q_start + i + 1);
        r.row0 = a;
        r.rows_all = b > a ? b - a : 0;
        r.rows = a >= 0 && a < p.T ? min(min(r.rows_all, p.max_rows), p.T - a) : 0;
    } else {
        r.row0 = i; r.rows_all = 1; r.rows = 1;
    }
    r.len = max(load_l2(p.seq_lens + i), 0);
    r.lo = p.kv_begin ? max(load_l2(p.kv_begin + i), 0) : 0;
    int hi = r.len;
    if (p.kv_end) hi = min(hi, load_l2(p.kv_end + i));
    r.hi = (int)min((int64_t)hi, p.max_tokens);
    r.pairs = r.rows * p.group;       // (at most 2^31 rows of 1,024 heads are refused on the host)
    return r;
}

}  // namespace kv8
}  // namespace splash
