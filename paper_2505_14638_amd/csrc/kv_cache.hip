// The paged key/value cache: rotary embedding with the write of a token's keys and values, and copies of pages.
#include "attention.hpp"
#include "attention_device.hpp"

namespace w4a8 {
namespace {

// Rotary embedding takes channels in pairs, (i, i + D/2) or (2i, 2i + 1): sixteen channels of a head are two chunks of eight, which turn with each
// other in the first form and lie side by side in the second.
__device__ __forceinline__ void unpack(u32x4 w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
    return u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}

// (a, b) -> (a cos - b sin, b cos + a sin) in float32, eight times.
template <bool PAIRS>
__device__ __forceinline__ void rotate(float (&a)[8], float (&b)[8], const float (&cs)[8], const float (&sn)[8]) {
    if (PAIRS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a0 = a[2 * i], a1 = a[2 * i + 1], b0 = b[2 * i], b1 = b[2 * i + 1];
            a[2 * i] = a0 * cs[i] - a1 * sn[i];
            a[2 * i + 1] = a1 * cs[i] + a0 * sn[i];
            b[2 * i] = b0 * cs[4 + i] - b1 * sn[4 + i];
            b[2 * i + 1] = b1 * cs[4 + i] + b0 * sn[4 + i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = a[i], y = b[i];
            a[i] = x * cs[i] - y * sn[i];
            b[i] = y * cs[i] + x * sn[i];
        }
    }
}

// A thread turns sixteen channels of a head of a token: they lie in two chunks of 16 bytes, and the eight angles are 64 bytes of the table.
// Memory bounds it: a token's rows are read once and written once, each instruction a run of 16 bytes a lane.  8192 tokens of 64 + 2 x 8 heads of 128
// channels, E4M3 cache and keys kept, 340 MB: 62 us, 5.5 TB/s; 32 heads into a bf16 cache, 206 MB: 32.3 us, 6.4 TB/s (part of it stays in
// the last cache); one token of 32 sequences: 2.7 us, a launch.  Four heads a thread under one load of the angles: 4.1 instead of 3.3 us at
// 256 tokens, 32.5 instead of 32.3 at 8192.
template <bool PAIRS, bool E4M3>
__global__ void __launch_bounds__(256) rope_cache_write_kernel(RopeCacheArgs a, int64_t units) {
    const int D = a.c.head_dim, UPH = D >> 4;                    // threads per head
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= units) return;
    const int rotated = a.q_heads + a.c.kv_heads, heads = rotated + a.c.kv_heads;
    const int piece = (int)(u % UPH);
    const int64_t rest = u / UPH;
    const int h = (int)(rest % heads);
    const int64_t t = rest / heads;
    const int64_t slot = a.slots[t], position = a.positions[t];
    if (slot < 0 || slot >= (a.c.n_pages << a.c.page_shift)) return;   // a padding token
    const int d_lo = PAIRS ? 16 * piece : 8 * piece, d_hi = PAIRS ? d_lo + 8 : d_lo + D / 2;
    const uint16_t* p = a.qkv + t * a.ldqkv + (int64_t)h * D;
    u32x4 x_lo = *reinterpret_cast<const u32x4*>(p + d_lo), x_hi = *reinterpret_cast<const u32x4*>(p + d_hi);
    float lo[8], hi[8];
    unpack(x_lo, lo);
    unpack(x_hi, hi);
    if (h < rotated) {
        float cs[8], sn[8];
        if (position >= 0 && position < a.table_rows) {
            const float* row = a.cos_sin + position * D + 8 * piece;
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const float4 c = *reinterpret_cast<const float4*>(row + i), s = *reinterpret_cast<const float4*>(row + D / 2 + i);
                cs[i] = c.x, cs[i + 1] = c.y, cs[i + 2] = c.z, cs[i + 3] = c.w;
                sn[i] = s.x, sn[i + 1] = s.y, sn[i + 2] = s.z, sn[i + 3] = s.w;
            }
        } else {                                                 // no such angle: nothing that could pass for a rotation
#pragma unroll
            for (int i = 0; i < 8; ++i) cs[i] = sn[i] = __builtin_nanf("");
        }
        rotate<PAIRS>(lo, hi, cs, sn);
        x_lo = pack(lo);
        x_hi = pack(hi);
        uint16_t* out = h < a.q_heads ? a.q_out + t * a.ldq + (int64_t)h * D
                        : a.k_out     ? a.k_out + t * a.ldk + (int64_t)(h - a.q_heads) * D
                                      : nullptr;
        if (out) {
            stream_out(out + d_lo, x_lo);
            stream_out(out + d_hi, x_hi);
        }
        if (h < a.q_heads) return;
    }
    const bool key = h < rotated;
    const int hk = key ? h - a.q_heads : h - rotated;
    const int64_t page = slot >> a.c.page_shift, off = slot & (a.c.page_size - 1);
    const int64_t at = page * a.c.page_stride + ((int64_t)hk * a.c.page_size + off) * D;
    uint8_t* cache = key ? a.k_cache : a.v_cache;
    if (E4M3) {
        const StaticQuantizer q(a.kv_scales[key ? 0 : 1]);
        stream_out(cache + at + d_lo, u32x2{q.four(lo[0], lo[1], lo[2], lo[3]), q.four(lo[4], lo[5], lo[6], lo[7])});
        stream_out(cache + at + d_hi, u32x2{q.four(hi[0], hi[1], hi[2], hi[3]), q.four(hi[4], hi[5], hi[6], hi[7])});
    } else {
        uint16_t* row = reinterpret_cast<uint16_t*>(cache) + at;
        stream_out(row + d_lo, x_lo);
        stream_out(row + d_hi, x_hi);
    }
}

// One workgroup copies up to 32 KiB of one page of one plane, eight 16-byte pieces per thread under way at once.  Memory bounds it: 400 pages of 64
// planes, 32 KB each, 1.68 GB read and written: 318 us, 5.3 TB/s, where a large copy by the runtime reaches 4.8; 16 pages: 11.6 us.
constexpr int COPY_PIECES = 8, COPY_BYTES = 256 * 16 * COPY_PIECES;
__global__ void __launch_bounds__(256) cache_copy_pages_kernel(uint8_t* cache, int64_t plane_stride, int64_t n_pages, int64_t page_stride,
                                                               int64_t page_bytes, const int32_t* src, const int32_t* dst, int64_t n_copies,
                                                               int blocks_per_page) {
    const int64_t i = blockIdx.x / blocks_per_page;
    const int64_t from = src[i], to = dst[i];
    if (from < 0 || from >= n_pages || to < 0 || to >= n_pages || from == to) return;
    const int64_t begin = (int64_t)(blockIdx.x % blocks_per_page) * COPY_BYTES + threadIdx.x * 16;
    uint8_t* plane = cache + (int64_t)blockIdx.y * plane_stride;
    const uint8_t* s = plane + from * page_stride + begin;
    uint8_t* d = plane + to * page_stride + begin;
    if (begin + (COPY_PIECES - 1) * 4096 < page_bytes) {
        u32x4 v[COPY_PIECES];
#pragma unroll
        for (int j = 0; j < COPY_PIECES; ++j) v[j] = *reinterpret_cast<const u32x4*>(s + j * 4096);
#pragma unroll
        for (int j = 0; j < COPY_PIECES; ++j) stream_out(d + j * 4096, v[j]);
    } else {
        for (int j = 0; begin + j * 4096 < page_bytes; ++j) stream_out(d + j * 4096, *reinterpret_cast<const u32x4*>(s + j * 4096));
    }
}

}  // namespace

int launch_rope_cache_write(const RopeCacheArgs& a, hipStream_t st) {
    const int64_t units = a.T * (a.q_heads + 2 * a.c.kv_heads) * (a.c.head_dim / 16);
    const dim3 grid((unsigned)((units + 255) / 256)), block(256);
    if (a.pairs) {
        if (a.c.e4m3) hipLaunchKernelGGL((rope_cache_write_kernel<true, true>), grid, block, 0, st, a, units);
        else hipLaunchKernelGGL((rope_cache_write_kernel<true, false>), grid, block, 0, st, a, units);
    } else {
        if (a.c.e4m3) hipLaunchKernelGGL((rope_cache_write_kernel<false, true>), grid, block, 0, st, a, units);
        else hipLaunchKernelGGL((rope_cache_write_kernel<false, false>), grid, block, 0, st, a, units);
    }
    return launch_status();
}

int launch_cache_copy_pages(uint8_t* cache, int64_t n_planes, int64_t plane_stride, int64_t n_pages, int64_t page_stride,
                            int64_t page_bytes, const int32_t* src, const int32_t* dst, int64_t n_copies, hipStream_t st) {
    const int64_t per_page = (page_bytes + COPY_BYTES - 1) / COPY_BYTES;
    hipLaunchKernelGGL(cache_copy_pages_kernel, dim3((unsigned)(n_copies * per_page), (unsigned)n_planes), dim3(256), 0, st, cache,
                       plane_stride, n_pages, page_stride, page_bytes, src, dst, n_copies, (int)per_page);
    return launch_status();
}

}  // namespace w4a8
