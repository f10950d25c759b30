// The paged key/value cache: rotary embedding with the write of a token's keys and values, and copies of pages.
#include "attention.hpp"
#include "attention_device.hpp"

namespace w4a8 {
namespace {

// Sixteen channels of one head of one token: two chunks of eight, which turn together in the halves form (i with i + D/2) and lie
// side by side in the pairs form (2i with 2i + 1).
struct Channels {
    u32x4 lo, hi;
};
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

// A thread turns sixteen channels of HEADS heads of a token, `step` heads apart, under one set of eight angles.
template <int HEADS, bool PAIRS, bool E4M3>
__global__ void __launch_bounds__(256) rope_cache_write_kernel(RopeCacheArgs a, int step, int64_t units) {
    const int D = a.c.head_dim, UPH = D >> 4;                    // threads per head
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= units) return;
    const int piece = (int)(u % UPH);
    const int64_t rest = u / UPH;
    const int first = (int)(rest % step);
    const int64_t t = rest / step;
    const int64_t slot = a.slots[t], position = a.positions[t];
    if (slot < 0 || slot >= (a.c.n_pages << a.c.page_shift)) return;   // a padding token
    const int rotated = a.q_heads + a.c.kv_heads, heads = rotated + a.c.kv_heads;
    const int d_lo = PAIRS ? 16 * piece : 8 * piece, d_hi = PAIRS ? d_lo + 8 : d_lo + D / 2;
    float cs[8], sn[8];
    if (position >= 0 && position < a.table_rows) {
        const float* row = a.cos_sin + position * D + 8 * piece;
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const float4 c = *reinterpret_cast<const float4*>(row + i), s = *reinterpret_cast<const float4*>(row + D / 2 + i);
            cs[i] = c.x, cs[i + 1] = c.y, cs[i + 2] = c.z, cs[i + 3] = c.w;
            sn[i] = s.x, sn[i + 1] = s.y, sn[i + 2] = s.z, sn[i + 3] = s.w;
        }
    } else {                                                     // no such angle: nothing that could pass for a rotation
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = sn[i] = __builtin_nanf("");
    }
    Channels x[HEADS];
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
        const int h = first + j * step;
        if (h < heads) {
            const uint16_t* p = a.qkv + t * a.ldqkv + (int64_t)h * D;
            x[j].lo = *reinterpret_cast<const u32x4*>(p + d_lo);
            x[j].hi = *reinterpret_cast<const u32x4*>(p + d_hi);
        }
    }
    const int64_t page = slot >> a.c.page_shift, off = slot & (a.c.page_size - 1);
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
        const int h = first + j * step;
        if (h >= heads) break;
        float lo[8], hi[8];
        unpack(x[j].lo, lo);
        unpack(x[j].hi, hi);
        if (h < rotated) {
            rotate<PAIRS>(lo, hi, cs, sn);
            uint16_t* out = h < a.q_heads ? a.q_out + t * a.ldq + (int64_t)h * D
                            : a.k_out     ? a.k_out + t * a.ldk + (int64_t)(h - a.q_heads) * D
                                          : nullptr;
            if (out) {
                stream_out(out + d_lo, pack(lo));
                stream_out(out + d_hi, pack(hi));
            }
        }
        if (h >= a.q_heads) {
            const bool key = h < rotated;
            const int hk = key ? h - a.q_heads : h - rotated;
            const int64_t at = page * a.c.page_stride + ((int64_t)hk * a.c.page_size + off) * D;
            uint8_t* cache = key ? a.k_cache : a.v_cache;
            if (E4M3) {
                const StaticQuantizer q(a.kv_scales[key ? 0 : 1]);
                stream_out(cache + at + d_lo, u32x2{q.four(lo[0], lo[1], lo[2], lo[3]), q.four(lo[4], lo[5], lo[6], lo[7])});
                stream_out(cache + at + d_hi, u32x2{q.four(hi[0], hi[1], hi[2], hi[3]), q.four(hi[4], hi[5], hi[6], hi[7])});
            } else {
                uint16_t* row = reinterpret_cast<uint16_t*>(cache) + at;
                stream_out(row + d_lo, key ? pack(lo) : x[j].lo);
                stream_out(row + d_hi, key ? pack(hi) : x[j].hi);
            }
        }
    }
}

// One workgroup copies up to 32 KiB of one page of one plane, eight 16-byte pieces per thread under way at once.
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

template <int HEADS>
void launch_rope(const RopeCacheArgs& a, hipStream_t st) {
    const int heads = a.q_heads + 2 * a.c.kv_heads, step = (heads + HEADS - 1) / HEADS;
    const int64_t units = a.T * step * (a.c.head_dim / 16);
    const dim3 grid((unsigned)((units + 255) / 256)), block(256);
    if (a.pairs) {
        if (a.c.e4m3) hipLaunchKernelGGL((rope_cache_write_kernel<HEADS, true, true>), grid, block, 0, st, a, step, units);
        else hipLaunchKernelGGL((rope_cache_write_kernel<HEADS, true, false>), grid, block, 0, st, a, step, units);
    } else {
        if (a.c.e4m3) hipLaunchKernelGGL((rope_cache_write_kernel<HEADS, false, true>), grid, block, 0, st, a, step, units);
        else hipLaunchKernelGGL((rope_cache_write_kernel<HEADS, false, false>), grid, block, 0, st, a, step, units);
    }
}

}  // namespace

int launch_rope_cache_write(const RopeCacheArgs& a, hipStream_t st) {
    if (a.T * (a.q_heads + 2 * a.c.kv_heads) >= 65536) launch_rope<4>(a, st);
    else launch_rope<1>(a, st);
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
