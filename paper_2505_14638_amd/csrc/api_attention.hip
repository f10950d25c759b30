// C-ABI front end of attention and its cache: argument validation on the host, then dispatch to the kernel launchers.  As in api.hip
// validation never touches the device.
#include "attention.hpp"

#include <math.h>

#include <algorithm>

using namespace w4a8;

namespace w4a8 {

// A workgroup on the sequences' own tokens reads one range of keys for up to 16 rows.  Few sequences need enough ranges to give every
// compute unit two workgroups (FILL), of SHORT keys at least; more of them cost more by their starts and partial results than they even out.  Figures
// in us, 32 query and 8 key heads, bf16:  3 sequences of 500 .. 16000 (E4M3) 21.0, with FILL 256 23.7; 16 of 4000 52.0, with 1024 53.3; one of
// 1000 7.5, with SHORT 256 9.0; 64 of 200 .. 8192, 64 heads, E4M3, 131 with one range, 152 with up to eight.
// Up to ONE_GO tokens one workgroup of eight wavefronts takes them all, however few there are of those: that saves the second launch, 3 us of the
// host's time beside the device's: 20 sequences of 500 10.6, in two launches 14.7; one of 200 6.0 and 7.4, of 500 8.6 and 7.5; one of 1000
// would take 13.4 and 7.4.
// On the prefix up to 16 rows go the same way (one sequence of 500 behind 4000: 10.2, as tiles 11.3).  More rows walk tiles of 64 keys that 128
// rows share (16 sequences: 15.8, by sixteens 23.7); there a range costs its tiles, and every part of a row 4 (D + 2) bytes written and read
// again, together about 3 TB/s; the figures of that sum are measured ones (32 sequences of 1 .. 512 behind 4096: 20.5, 64 of 100 .. 1000 behind 2000: 40.8; with
// 1.6 us a tile and 4.5 TB/s 22.3 and 45.9, with 2 TB/s 20.6 and 41.3).
DecodePlan decode_plan(int64_t n_seqs, int q_heads, int kv_heads, int head_dim, int64_t own_capacity, int64_t prefix_len) {
    constexpr int64_t FILL = 512, SHORT = 128, MOST = 64, CUS = 256, ONE_GO = 512;
    const int64_t group = q_heads / kv_heads, rows = n_seqs * group, own_units = n_seqs * kv_heads * ((group + 15) / 16);
    auto splits = [&](int64_t units, int64_t keys) {
        const int64_t s = std::min((FILL + units - 1) / units, (keys + SHORT - 1) / SHORT);
        return (int)std::max<int64_t>(1, std::min(s, MOST));
    };
    DecodePlan p{};
    p.own_waves = 4;
    p.own_splits = splits(own_units, own_capacity);
    p.prefix_rows = rows <= 16 ? 16 : 128;
    if (prefix_len == 0) {
        if (own_capacity <= ONE_GO && own_units <= CUS) p.own_splits = 1, p.own_waves = 8;
    } else if (p.prefix_rows == 16) {
        p.prefix_splits = splits(kv_heads, prefix_len);
    } else {
        const int64_t units = kv_heads * ((rows + p.prefix_rows - 1) / p.prefix_rows), tiles = (prefix_len + 63) / 64;
        const double part_us = (double)n_seqs * q_heads * 8 * (head_dim + 2) / 3.0e6;
        double best = 0;
        for (int64_t s = 1; s <= MOST && s <= tiles; ++s) {
            const double us = (double)((units * s + CUS - 1) / CUS) * (1.4 * (double)((tiles + s - 1) / s) + 4) + (double)s * part_us;
            if (s == 1 || us < best) best = us, p.prefix_splits = (int)s;
        }
    }
    p.parts = p.own_splits == 1 && p.prefix_splits == 0 ? 0 : p.own_splits + p.prefix_splits;
    return p;
}

size_t decode_partial_bytes(const DecodePlan& p, int64_t n_seqs, int q_heads, int head_dim) {
    return (size_t)p.parts * (size_t)(n_seqs * q_heads) * (size_t)(head_dim + 2) * sizeof(float);
}

}  // namespace w4a8

namespace {

constexpr int64_t TOKENS_MAX = (int64_t)1 << 24, LD_MAX = (int64_t)1 << 20, PAGES_MAX = (int64_t)1 << 30, SEQS_MAX = (int64_t)1 << 20;
constexpr int64_t WORKGROUPS_MAX = ((int64_t)1 << 24) - 1;       // of 256 threads: a launch stays below 2^32 threads
constexpr int64_t DECODE_ROWS_MAX = (int64_t)1 << 18;            // up to 64 ranges of each, and as many workgroups again to join them

inline bool aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

int check_heads(int q_heads, int kv_heads, int head_dim) {
    if (head_dim != 64 && head_dim != 128) return W4A8_ERR_SHAPE;
    if (kv_heads < 1 || q_heads < kv_heads || q_heads > 4096 || q_heads % kv_heads != 0) return W4A8_ERR_SHAPE;
    return W4A8_OK;
}

int check_cache(int dtype, int64_t n_pages, int64_t page_stride, int page_size, int kv_heads, int head_dim, CacheShape& c) {
    if (dtype != W4A8_CACHE_BF16 && dtype != W4A8_CACHE_E4M3) return W4A8_ERR_DTYPE;
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1))) return W4A8_ERR_SHAPE;
    if (n_pages < 1 || n_pages > PAGES_MAX / page_size || page_stride < (int64_t)kv_heads * page_size * head_dim) return W4A8_ERR_SHAPE;
    if (page_stride % (dtype == W4A8_CACHE_E4M3 ? 16 : 8) != 0) return W4A8_ERR_ALIGN;
    c.n_pages = n_pages;
    c.page_stride = page_stride;
    c.page_size = page_size;
    c.page_shift = __builtin_ctz((unsigned)page_size);
    c.kv_heads = kv_heads;
    c.head_dim = head_dim;
    c.e4m3 = dtype == W4A8_CACHE_E4M3;
    return W4A8_OK;
}

int check_scale(float softmax_scale) { return softmax_scale > 0.0f && softmax_scale <= 1e30f ? W4A8_OK : W4A8_ERR_SHAPE; }

// rows of bf16 (bytes == 2) or E4M3 (1) whose 16-byte pieces are read or written
int check_rows(const void* p, int64_t ld, int64_t width, int bytes) {
    if (ld < width || ld >= LD_MAX) return W4A8_ERR_SHAPE;
    if (!aligned(p, 16) || (ld * bytes) % 16 != 0) return W4A8_ERR_ALIGN;
    return W4A8_OK;
}

constexpr float LOG2_E = 1.44269504088896340736f;

}  // namespace

extern "C" {

int w4a8_rope_cache_write(const void* qkv_dev, int64_t T, int64_t ldqkv, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                          const float* cos_sin_dev, int64_t table_rows, w4a8_rope rope, const int32_t* positions_dev,
                          const int32_t* slots_dev, void* q_out_dev, int64_t ldq, void* k_out_dev, int64_t ldk, void* k_cache_dev,
                          void* v_cache_dev, w4a8_cache_dtype cache_dtype, const float* kv_scales_dev, int64_t n_pages,
                          int64_t page_stride, int32_t page_size, void* stream) {
    if (rope != W4A8_ROPE_HALVES && rope != W4A8_ROPE_PAIRS) return W4A8_ERR_DTYPE;
    if (int e = check_heads(q_heads, kv_heads, head_dim)) return e;
    RopeCacheArgs a{};
    if (int e = check_cache(cache_dtype, n_pages, page_stride, page_size, kv_heads, head_dim, a.c)) return e;
    const int64_t heads = q_heads + 2 * (int64_t)kv_heads;
    if (T < 0 || T > TOKENS_MAX || T * heads * (head_dim / 16) > WORKGROUPS_MAX * 256 || table_rows < 1 || table_rows > PAGES_MAX) return W4A8_ERR_SHAPE;
    if (T == 0) return W4A8_OK;
    if (!qkv_dev || !cos_sin_dev || !positions_dev || !slots_dev || !q_out_dev || !k_cache_dev || !v_cache_dev) return W4A8_ERR_NULL;
    if (a.c.e4m3 && !kv_scales_dev) return W4A8_ERR_NULL;
    if (int e = check_rows(qkv_dev, ldqkv, heads * head_dim, 2)) return e;
    if (int e = check_rows(q_out_dev, ldq, (int64_t)q_heads * head_dim, 2)) return e;
    if (k_out_dev)
        if (int e = check_rows(k_out_dev, ldk, (int64_t)kv_heads * head_dim, 2)) return e;
    if (!aligned(cos_sin_dev, 16) || !aligned(positions_dev, 4) || !aligned(slots_dev, 4) || !aligned(k_cache_dev, 16) ||
        !aligned(v_cache_dev, 16) || !aligned(kv_scales_dev, 4))
        return W4A8_ERR_ALIGN;
    a.qkv = static_cast<const uint16_t*>(qkv_dev);
    a.T = T;
    a.ldqkv = ldqkv;
    a.q_heads = q_heads;
    a.cos_sin = cos_sin_dev;
    a.table_rows = table_rows;
    a.positions = positions_dev;
    a.slots = slots_dev;
    a.pairs = rope == W4A8_ROPE_PAIRS;
    a.q_out = static_cast<uint16_t*>(q_out_dev);
    a.k_out = static_cast<uint16_t*>(k_out_dev);
    a.ldq = ldq;
    a.ldk = ldk;
    a.k_cache = static_cast<uint8_t*>(k_cache_dev);
    a.v_cache = static_cast<uint8_t*>(v_cache_dev);
    a.kv_scales = kv_scales_dev;
    return launch_rope_cache_write(a, static_cast<hipStream_t>(stream));
}

int w4a8_attention_prompt(const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk, const void* v_dev, int64_t ldv,
                          const int32_t* starts_dev, int64_t n_seqs, int64_t T, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                          int32_t causal, float softmax_scale, void* y_dev, int64_t ldy, const float* y_scale_dev, void* stream) {
    if (int e = check_heads(q_heads, kv_heads, head_dim)) return e;
    if (causal != 0 && causal != 1) return W4A8_ERR_DTYPE;
    if (int e = check_scale(softmax_scale)) return e;
    if (n_seqs < 0 || n_seqs > SEQS_MAX || T < 0 || T > TOKENS_MAX || (T / 32 + n_seqs) * q_heads > WORKGROUPS_MAX) return W4A8_ERR_SHAPE;
    if (n_seqs == 0 || T == 0) return W4A8_OK;
    if (!q_dev || !k_dev || !v_dev || !starts_dev || !y_dev) return W4A8_ERR_NULL;
    if (int e = check_rows(q_dev, ldq, (int64_t)q_heads * head_dim, 2)) return e;
    if (int e = check_rows(k_dev, ldk, (int64_t)kv_heads * head_dim, 2)) return e;
    if (int e = check_rows(v_dev, ldv, (int64_t)kv_heads * head_dim, 2)) return e;
    if (int e = check_rows(y_dev, ldy, (int64_t)q_heads * head_dim, y_scale_dev ? 1 : 2)) return e;
    if (!aligned(starts_dev, 4) || !aligned(y_scale_dev, 4)) return W4A8_ERR_ALIGN;
    PromptArgs a{};
    a.q = static_cast<const uint16_t*>(q_dev);
    a.k = static_cast<const uint16_t*>(k_dev);
    a.v = static_cast<const uint16_t*>(v_dev);
    a.ldq = ldq;
    a.ldk = ldk;
    a.ldv = ldv;
    a.starts = starts_dev;
    a.T = T;
    a.n_seqs = (int)n_seqs;
    a.q_heads = q_heads;
    a.kv_heads = kv_heads;
    a.head_dim = head_dim;
    a.causal = causal;
    a.scale_log2 = softmax_scale * LOG2_E;
    a.y = y_dev;
    a.y_scale = y_scale_dev;
    a.ldy = ldy;
    return launch_attention_prompt(a, static_cast<hipStream_t>(stream));
}

// Sizes of a decode call alone; W4A8_OK or what is wrong with them.
static int check_decode(int64_t n_seqs, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t page_size, int64_t table_width,
                        int64_t prefix_length) {
    if (int e = check_heads(q_heads, kv_heads, head_dim)) return e;
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1))) return W4A8_ERR_SHAPE;
    if (n_seqs < 0 || n_seqs > SEQS_MAX || n_seqs * q_heads > DECODE_ROWS_MAX || table_width < 0 || table_width > PAGES_MAX / page_size ||
        prefix_length < 0 || prefix_length > PAGES_MAX)
        return W4A8_ERR_SHAPE;
    return W4A8_OK;
}

size_t w4a8_attention_decode_workspace_bytes(int64_t n_seqs, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t page_size,
                                             int64_t table_width, int64_t prefix_length) {
    if (check_decode(n_seqs, q_heads, kv_heads, head_dim, page_size, table_width, prefix_length) != W4A8_OK || n_seqs == 0) return 0;
    return decode_partial_bytes(decode_plan(n_seqs, q_heads, kv_heads, head_dim, table_width * page_size, prefix_length), n_seqs, q_heads, head_dim);
}

int w4a8_attention_decode(const void* q_dev, int64_t ldq, int64_t n_seqs, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                          const void* k_cache_dev, const void* v_cache_dev, w4a8_cache_dtype cache_dtype, const float* kv_scales_dev,
                          int64_t n_pages, int64_t page_stride, int32_t page_size, const int32_t* tables_dev, int64_t table_width,
                          int64_t ld_tables, const int32_t* lengths_dev, const int32_t* prefix_pages_dev, int64_t prefix_length,
                          float softmax_scale, void* y_dev, int64_t ldy, const float* y_scale_dev, void* workspace_dev,
                          size_t workspace_bytes, void* stream) {
    if (int e = check_decode(n_seqs, q_heads, kv_heads, head_dim, page_size, table_width, prefix_length)) return e;
    DecodeArgs a{};
    if (int e = check_cache(cache_dtype, n_pages, page_stride, page_size, kv_heads, head_dim, a.c)) return e;
    if (int e = check_scale(softmax_scale)) return e;
    if (ld_tables < table_width) return W4A8_ERR_SHAPE;
    if (n_seqs == 0) return W4A8_OK;
    if (!q_dev || !k_cache_dev || !v_cache_dev || !lengths_dev || !y_dev || (table_width > 0 && !tables_dev) ||
        (prefix_length > 0 && !prefix_pages_dev) || (a.c.e4m3 && !kv_scales_dev))
        return W4A8_ERR_NULL;
    if (int e = check_rows(q_dev, ldq, (int64_t)q_heads * head_dim, 2)) return e;
    if (int e = check_rows(y_dev, ldy, (int64_t)q_heads * head_dim, y_scale_dev ? 1 : 2)) return e;
    if (!aligned(k_cache_dev, 16) || !aligned(v_cache_dev, 16) || !aligned(kv_scales_dev, 4) || !aligned(tables_dev, 4) || !aligned(lengths_dev, 4) ||
        !aligned(prefix_pages_dev, 4) || !aligned(y_scale_dev, 4))
        return W4A8_ERR_ALIGN;
    const DecodePlan p = decode_plan(n_seqs, q_heads, kv_heads, head_dim, table_width * page_size, prefix_length);
    const size_t need = decode_partial_bytes(p, n_seqs, q_heads, head_dim);
    if (need > 0) {
        if (!workspace_dev) return W4A8_ERR_NULL;
        if (!aligned(workspace_dev, 16)) return W4A8_ERR_ALIGN;
        if (workspace_bytes < need) return W4A8_ERR_WORKSPACE;
    }
    a.q = static_cast<const uint16_t*>(q_dev);
    a.ldq = ldq;
    a.n_seqs = (int)n_seqs;
    a.q_heads = q_heads;
    a.k_cache = static_cast<const uint8_t*>(k_cache_dev);
    a.v_cache = static_cast<const uint8_t*>(v_cache_dev);
    a.kv_scales = kv_scales_dev;
    a.tables = tables_dev;
    a.ld_tables = ld_tables;
    a.table_width = table_width;
    a.lengths = lengths_dev;
    a.prefix_pages = prefix_pages_dev;
    a.prefix_len = prefix_length;
    a.scale_log2 = softmax_scale * LOG2_E;
    a.y = y_dev;
    a.y_scale = y_scale_dev;
    a.ldy = ldy;
    a.partial = static_cast<float*>(workspace_dev);
    return launch_attention_decode(a, p, static_cast<hipStream_t>(stream));
}

int w4a8_cache_copy_pages(void* cache_dev, int64_t n_planes, int64_t plane_stride, int64_t n_pages, int64_t page_stride, int64_t page_bytes,
                          const int32_t* src_pages_dev, const int32_t* dst_pages_dev, int64_t n_copies, void* stream) {
    constexpr int64_t FAR = (int64_t)1 << 46;                    // bytes: products below stay within 64 bits
    if (n_planes < 0 || n_planes > 65535 || n_pages < 1 || n_pages > PAGES_MAX || page_bytes < 16 || page_bytes > PAGES_MAX ||
        page_stride < page_bytes || page_stride > FAR || n_copies < 0 || n_copies > n_pages || plane_stride > FAR || plane_stride < 0)
        return W4A8_ERR_SHAPE;
    if ((page_bytes + 32767) / 32768 * n_copies > WORKGROUPS_MAX) return W4A8_ERR_SHAPE;
    if (page_bytes % 16 != 0 || page_stride % 16 != 0 || plane_stride % 16 != 0) return W4A8_ERR_ALIGN;
    if (n_copies == 0 || n_planes == 0) return W4A8_OK;
    if (!cache_dev || !src_pages_dev || !dst_pages_dev) return W4A8_ERR_NULL;
    if (!aligned(cache_dev, 16) || !aligned(src_pages_dev, 4) || !aligned(dst_pages_dev, 4)) return W4A8_ERR_ALIGN;
    return launch_cache_copy_pages(static_cast<uint8_t*>(cache_dev), n_planes, plane_stride, n_pages, page_stride, page_bytes, src_pages_dev,
                                   dst_pages_dev, n_copies, static_cast<hipStream_t>(stream));
}

}  // extern "C"
