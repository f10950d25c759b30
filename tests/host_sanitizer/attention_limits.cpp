// The limits of the attention entry points, with stubs in the place of the kernel launchers: a launch has fewer than 2^32 threads, and the
// sizes just below a limit are accepted.
#include <stdint.h>
#include <stdio.h>

#include "../../paper_2505_14638_amd/csrc/attention.hpp"

static long launches = 0;
static int failures = 0;
static void expect(bool ok, const char* what) {
    if (!ok) {
        printf("FAILED: %s\n", what);
        ++failures;
    }
}
static void workgroups(int64_t n, const char* what) {            // of 256 threads
    ++launches;
    expect(n >= 1 && n * 256 < (int64_t)1 << 32, what);
}

namespace w4a8 {
int launch_rope_cache_write(const RopeCacheArgs& a, hipStream_t) {
    workgroups((a.T * (a.q_heads + 2 * a.c.kv_heads) * (a.c.head_dim / 16) + 255) / 256, "rope grid");
    return W4A8_OK;
}
int launch_attention_prompt(const PromptArgs& a, hipStream_t) {
    for (int64_t rows : {64, 128}) workgroups((a.n_seqs == 1 ? (a.T + rows - 1) / rows : a.T / rows + a.n_seqs) * a.q_heads, "prompt grid");
    return W4A8_OK;
}
int launch_attention_decode(const DecodeArgs& a, const DecodePlan& p, hipStream_t) {
    const int64_t group = a.q_heads / a.c.kv_heads, rows = a.n_seqs * group;
    const int64_t own = a.n_seqs * (int64_t)a.c.kv_heads * ((group + 15) / 16) * p.own_splits;
    const int64_t shared = a.c.kv_heads * ((rows + p.prefix_rows - 1) / p.prefix_rows) * (int64_t)p.prefix_splits;
    workgroups((own + (shared + 7) / 8 * 8) * (p.own_waves / 4), "decode grid");
    workgroups((int64_t)a.n_seqs * a.q_heads, "join grid");
    return W4A8_OK;
}
int launch_cache_copy_pages(uint8_t*, int64_t, int64_t, int64_t, int64_t, int64_t page_bytes, const int32_t*, const int32_t*, int64_t n_copies, hipStream_t) {
    workgroups((page_bytes + 32767) / 32768 * n_copies, "copy grid");
    return W4A8_OK;
}
}  // namespace w4a8

int main() {
    alignas(16) static char p[64];
    float* f = reinterpret_cast<float*>(p);
    int32_t* i = reinterpret_cast<int32_t*>(p);
    auto copy = [&](int64_t n, int64_t bytes) { return w4a8_cache_copy_pages(p, 1, 0, n, bytes, bytes, i, i, n, nullptr); };
    expect(copy(1 << 24, 16) == W4A8_ERR_SHAPE && copy((1 << 24) - 1, 16) == W4A8_OK, "pages of one workgroup");
    expect(copy(1 << 23, 65536) == W4A8_ERR_SHAPE && copy((1 << 23) - 1, 65536) == W4A8_OK, "pages of two");
    auto prompt = [&](int64_t n, int64_t t, int h) {
        return w4a8_attention_prompt(p, h * 64, p, 64, p, 64, i, n, t, h, 1, 64, 1, 0.1f, p, h * 64, nullptr, nullptr);
    };
    expect(prompt(1 << 20, 1, 16) == W4A8_ERR_SHAPE && prompt((1 << 20) - 1, 1, 16) == W4A8_OK, "sequences");
    expect(prompt(1 << 12, 1 << 24, 32) == W4A8_ERR_SHAPE && prompt(1 << 12, (1 << 24) - (1 << 18), 31) == W4A8_OK, "tokens and sequences");
    auto rope = [&](int64_t t, int h) {
        return w4a8_rope_cache_write(p, t, 1 << 19, h, 1, 64, f, 9, W4A8_ROPE_HALVES, i, i, p, 1 << 18, nullptr, 0, p, p, W4A8_CACHE_BF16, f, 9, 1024, 16, nullptr);
    };
    expect(rope(1 << 24, 62) == W4A8_ERR_SHAPE && rope((1 << 24) - 1, 62) == W4A8_OK, "tokens times heads");   // 64 heads of 4 threads: 256 a token
    auto decode = [&](int64_t n, int h, int hk, int64_t width, int64_t prefix) {
        const size_t need = w4a8_attention_decode_workspace_bytes(n, h, hk, 64, 16, width, prefix);
        return w4a8_attention_decode(p, h * 64, n, h, hk, 64, p, p, W4A8_CACHE_BF16, f, 9, hk * 1024, 16, i, width, width, i, i, prefix, 0.1f, p, h * 64, nullptr, p, need, nullptr);
    };
    for (int h : {1, 16, 4096})
        for (int hk : {1, h})
            for (int64_t width : {0, 1, 1 << 20})
                for (int64_t prefix : {0, 1, 1 << 30}) {
                    expect(decode((1 << 18) / h, h, hk, width, prefix) == W4A8_OK, "rows of decoding");
                    expect(decode((1 << 18) / h + 1, h, hk, width, prefix) == W4A8_ERR_SHAPE, "more rows of decoding");
                }
    if (failures == 0) printf("all checks passed (%ld launches)\n", launches);
    return failures != 0;
}
