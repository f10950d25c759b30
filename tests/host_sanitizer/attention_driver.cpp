// Drives the attention entry points' validation and planning on the host, with stubs in the place of the kernel launchers: extreme
// sizes must neither overflow nor reach a launch that the kernels' grids cannot hold.
#include <limits.h>
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

namespace w4a8 {
int launch_rope_cache_write(const RopeCacheArgs& a, hipStream_t) {
    ++launches;
    expect(a.T * (a.q_heads + 2 * a.c.kv_heads) * (a.c.head_dim / 16) <= (int64_t)1 << 32, "rope grid");
    return W4A8_OK;
}
int launch_attention_prompt(const PromptArgs& a, hipStream_t) {
    ++launches;
    expect((a.T / 32 + a.n_seqs) * a.q_heads <= 1 << 24, "prompt grid");
    return W4A8_OK;
}
int launch_attention_decode(const DecodeArgs& a, const DecodePlan& p, hipStream_t) {
    ++launches;
    const int64_t group = a.q_heads / a.c.kv_heads;
    const int64_t own = a.n_seqs * (int64_t)a.c.kv_heads * ((group + 15) / 16) * p.own_splits;
    const int64_t shared = a.c.kv_heads * ((a.n_seqs * group + 15) / 16) * (int64_t)p.prefix_splits;
    expect(own >= 0 && shared >= 0 && own + shared < 1 << 24, "decode grid");
    expect(p.own_splits >= 1 && p.own_splits <= 64 && p.prefix_splits >= 0 && p.prefix_splits <= 64, "splits");
    expect((a.prefix_len > 0) == (p.prefix_splits > 0) && (p.parts == 0 || p.parts == p.own_splits + p.prefix_splits), "parts");
    return W4A8_OK;
}
int launch_cache_copy_pages(uint8_t*, int64_t n_planes, int64_t, int64_t, int64_t, int64_t page_bytes, const int32_t*, const int32_t*, int64_t n_copies,
                            hipStream_t) {
    ++launches;
    expect(n_planes <= 65535 && (page_bytes + 32767) / 32768 * n_copies <= 1 << 24, "copy grid");
    return W4A8_OK;
}
}  // namespace w4a8

int main() {
    alignas(16) static char p[64];
    float* f = reinterpret_cast<float*>(p);
    int32_t* i = reinterpret_cast<int32_t*>(p);
    const int64_t sizes[] = {INT64_MIN, -1, 0, 1, 2, 7, 64, 4096, 65535, 1 << 16, 1 << 20, 1 << 24, (int64_t)1 << 30, ((int64_t)1 << 31) + 1, (int64_t)1 << 46, INT64_MAX};
    const int32_t small[] = {INT_MIN, -1, 0, 1, 2, 3, 8, 15, 16, 64, 128, 1024, 4096, INT_MAX};
    for (int64_t n : sizes)
        for (int64_t t : sizes)
            for (int32_t h : small)
                for (int32_t hk : small) {
                    const int64_t ld = 1 << 19;
                    w4a8_attention_prompt(p, ld, p, ld, p, ld, i, n, t, h, hk, 128, 1, 0.1f, p, ld, nullptr, nullptr);
                    w4a8_rope_cache_write(p, ld, t, h, hk, 64, f, n, W4A8_ROPE_PAIRS, i, i, p, ld, p, ld, p, p, W4A8_CACHE_E4M3, f, 1024, ld, 16, nullptr);
                    for (int32_t page : {16, 1024, 17}) {
                        const size_t need = w4a8_attention_decode_workspace_bytes(n, h, hk, 64, page, t, 1000);
                        w4a8_attention_decode(p, ld, n, h, hk, 64, p, p, W4A8_CACHE_BF16, f, 1000, (int64_t)1 << 26, page, i, t, t, i, i, 1000, 0.1f, p, ld, f, p,
                                              need, nullptr);
                        w4a8_attention_decode(p, ld, 3, h, hk, 128, p, p, W4A8_CACHE_BF16, f, n, t, page, i, 2, 2, i, i, n, 0.1f, p, ld, f, p, SIZE_MAX, nullptr);
                    }
                }
    for (int64_t a : sizes)
        for (int64_t b : sizes)
            for (int64_t c : sizes)
                for (int64_t d : sizes) w4a8_cache_copy_pages(p, 3, a, b, c, d, i, i, b / 2, nullptr), w4a8_cache_copy_pages(p, a, 64, b, c, 16, i, i, d, nullptr);
    for (int v : {INT_MIN, -1, 2, 77, INT_MAX}) {
        expect(w4a8_rope_cache_write(p, 1024, 1, 4, 2, 128, f, 9, (w4a8_rope)v, i, i, p, 512, p, 256, p, p, W4A8_CACHE_BF16, f, 9, 4096, 16, nullptr) == W4A8_ERR_DTYPE, "rope value");
        expect(w4a8_rope_cache_write(p, 1024, 1, 4, 2, 128, f, 9, W4A8_ROPE_HALVES, i, i, p, 512, p, 256, p, p, (w4a8_cache_dtype)v, f, 9, 4096, 16, nullptr) == W4A8_ERR_DTYPE, "cache type");
    }
    expect(launches > 1000, "valid calls reach a launch");
    if (failures == 0) printf("all checks passed (%ld launches)\n", launches);
    return failures != 0;
}
