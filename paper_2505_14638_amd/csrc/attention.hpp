// Attention with a paged key/value cache: what its front end hands to the kernel launchers, all of it validated.
#pragma once
#include "w4a8_internal.hpp"

namespace w4a8 {

// A cache of keys or values: page p is E [kv_heads, page_size, head_dim], row-major, at p * page_stride elements.
struct CacheShape {
    int64_t n_pages, page_stride;
    int page_size, page_shift;                                   // page_size = 2^page_shift
    int kv_heads, head_dim;
    int e4m3;                                                    // elements: 0 = bf16, 1 = E4M3 bytes that stand for byte * scale
};

struct RopeCacheArgs {
    const uint16_t* qkv;
    int64_t T, ldqkv;
    int q_heads;
    const float* cos_sin;
    int64_t table_rows;
    const int32_t *positions, *slots;
    int pairs;                                                   // 0: channels (i, i + D/2) turn together, 1: (2i, 2i + 1)
    uint16_t *q_out, *k_out;                                     // k_out may be null
    int64_t ldq, ldk;
    uint8_t *k_cache, *v_cache;
    const float* kv_scales;
    CacheShape c;
};

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t ldq, ldk, ldv;
    const int32_t* starts;
    int64_t T;
    int n_seqs, q_heads, kv_heads, head_dim, causal;
    float scale_log2;                                            // softmax scale * log2(e)
    void* y;
    const float* y_scale;                                        // not null: y is E4M3 bytes
    int64_t ldy;
};

struct DecodeArgs {
    const uint16_t* q;
    int64_t ldq;
    int n_seqs, q_heads;
    const uint8_t *k_cache, *v_cache;
    const float* kv_scales;
    CacheShape c;
    const int32_t* tables;
    int64_t ld_tables, table_width;
    const int32_t* lengths;
    const int32_t* prefix_pages;
    int64_t prefix_len;
    float scale_log2;
    void* y;
    const float* y_scale;
    int64_t ldy;
    float* partial;                                              // float32 [parts, rows, head_dim], then (max, sum) pairs [parts, rows]
};

// How a decode call is cut up; a function of sizes alone, so that the workspace can be sized before the call.
struct DecodePlan {
    int own_splits, prefix_splits;                               // ranges of keys per sequence, of the prefix (0: no prefix)
    int own_waves;                                               // wavefronts of a workgroup on the own tokens: 4, or 8 where it finishes its rows
    int prefix_rows;                                             // rows of a workgroup on the prefix: 16 (as on the own tokens) or 128
    int parts;                                                   // partial results per row; 0: rows are finished at once
};
DecodePlan decode_plan(int64_t n_seqs, int q_heads, int kv_heads, int head_dim, int64_t own_capacity, int64_t prefix_len);
size_t decode_partial_bytes(const DecodePlan& p, int64_t n_seqs, int q_heads, int head_dim);

int launch_rope_cache_write(const RopeCacheArgs& a, hipStream_t st);
int launch_attention_prompt(const PromptArgs& a, hipStream_t st);
int launch_attention_decode(const DecodeArgs& a, const DecodePlan& p, hipStream_t st);
int launch_cache_copy_pages(uint8_t* cache, int64_t n_planes, int64_t plane_stride, int64_t n_pages, int64_t page_stride,
                            int64_t page_bytes, const int32_t* src, const int32_t* dst, int64_t n_copies, hipStream_t st);

}  // namespace w4a8
