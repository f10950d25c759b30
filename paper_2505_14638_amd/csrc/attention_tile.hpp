// What the attention kernels that walk keys by tiles share: one wavefront's 32 rows against tiles of 64 keys in LDS.
//   S^T = K Q^T and O^T = V^T P^T: a lane holds one row's scores, finds their maximum in registers (and one exchange with the lane 32
//   away), and the 16 keys whose scores it has are, in the same order, those of the second product's operand: P never leaves the
//   registers.  V^T is read from LDS by transposing reads.
#pragma once
#include "attention_device.hpp"

namespace w4a8 {

// LDS keeps rows of D bf16 in 16-byte pieces, piece p of row r at p ^ swizzle(r): eight rows next to each other have any one piece in
// eight different bank groups (the rows a read of K touches), and four rows' 64-byte quarters lie in four (a transposing read of V).
template <int D> __device__ __forceinline__ constexpr int swizzle(int r) {
    return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <typename T> __device__ __forceinline__ T lds_read(uint32_t at) {
    return *reinterpret_cast<__attribute__((address_space(3))) const T*>((uintptr_t)at);
}

template <typename T> __device__ __forceinline__ void lds_write(uint32_t at, T x) {
    *reinterpret_cast<__attribute__((address_space(3))) T*>((uintptr_t)at) = x;
}

constexpr int TILE_KEYS = 64;

// LDS: two buffers of a tile of keys and the tile of values behind it, of which the wavefront takes KEYS keys from key `first` on.
template <int D, int KEYS = TILE_KEYS> struct RowBlock {
    static constexpr int ROW = 2 * D, PIECES = D / 8, TILE = TILE_KEYS * ROW, RPC = 1024 / ROW;   // RPC: rows per 64 x 16 bytes
    static constexpr int KS = D / 16, DT = D / 32, KT = KEYS / 32;
    v8bf q[KS];                                                  // Q^T, the second operand of S^T = K Q^T
    v16f o[DT];                                                  // O^T: channel 32 d + (r & 3) + 8 (r >> 2) + 4 half of row lane % 32
    float m, l;                                                  // the maximum that the sums go by (scaled, base 2), this lane's part of the sum
    // LDS addresses: K operand of step i: piece 2i + half of row lane % 32 (+ 32).  V^T operand (16 keys, channels 32 d ..): keys 4 half
    // + {0..3} and 8 more, 16 channels per 16 lanes
    uint32_t k_addr[KS], v_addr[DT][2];

    __device__ __forceinline__ RowBlock(uint32_t lds, int lane, int first = 0) {
        const int col = lane & 31, half = lane >> 5, j = lane & 15, g1 = (lane >> 4) & 1;
#pragma unroll
        for (int i = 0; i < KS; ++i) k_addr[i] = lds + (first + col) * ROW + (uint32_t)(((half ^ swizzle<D>(col)) ^ (2 * i)) << 4);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 4 * half + (j >> 2), piece = 2 * g1 + ((j & 3) >> 1);
                v_addr[d][e] = lds + TILE + (first + r + 8 * e) * ROW + (j & 1) * 8 + (uint32_t)((piece ^ swizzle<D>(r) ^ (4 * d) ^ (2 * e)) << 4);
            }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
        m = NEG_INF;
        l = 0.0f;
    }
    // Q comes through LDS, since whole rows are what memory gives fast: 32 rows at byte `at` of LDS, swizzled like keys.
    __device__ __forceinline__ void read_q(uint32_t at) {
#pragma unroll
        for (int i = 0; i < KS; ++i) q[i] = lds_read<v8bf>(k_addr[i] + at);
    }
    // s[k][r]: key first + 32 k + (r & 3) + 8 (r >> 2) + 4 half of the tile
    template <int BUFFER> __device__ __forceinline__ void scores(v16f (&s)[KT]) const {
#pragma unroll
        for (int k = 0; k < KT; ++k) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[k][r] = 0.0f;
#pragma unroll
            for (int i = 0; i < KS; ++i) s[k] = mfma_32x32x16_bf16(lds_read<v8bf>(k_addr[i] + 2 * BUFFER * TILE + k * 32 * ROW), q[i], s[k]);
        }
    }
    // The weights 2^(score * scale - m) as bf16 pairs, m and the sums brought up first where that is due.
    __device__ __forceinline__ void weights(const v16f (&s)[KT], float scale, uint32_t (&p)[KT][8]) {
        float mx = s[0][0];
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[k][r]);
        mx = max_over_32(mx) * scale;
        if (__builtin_amdgcn_ballot_w64(mx > m + RISE)) {
            const float m_new = fmaxf(m, mx), alpha = m_new == NEG_INF ? 1.0f : exp2_fast(m - m_new);
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
            m = m_new;
        }
        const float m_use = m == NEG_INF ? 0.0f : m;             // of a row that has seen nothing yet
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                p[k][r / 2] = pack_bf16(exp2_fast(fmaf(s[k][r], scale, -m_use)), exp2_fast(fmaf(s[k][r + 1], scale, -m_use)));
                l = add_pair(p[k][r / 2], l);
            }
    }
    // Weights of 16 keys, the second operand of O^T = V^T P^T, and the values that go with them.
    static __device__ __forceinline__ v8bf p_operand(const uint32_t (&p)[KT][8], int t16) {
        const uint32_t* x = p[t16 / 2] + 4 * (t16 & 1);
        return __builtin_bit_cast(v8bf, u32x4{x[0], x[1], x[2], x[3]});
    }
    template <int BUFFER> __device__ __forceinline__ u32x4 v_operand(int t16, int d) const {
        union {
            v4s part[2];
            u32x4 whole;
        } x;
#pragma unroll
        for (int e = 0; e < 2; ++e)
            x.part[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) v4s*)(uintptr_t)(v_addr[d][e] + 2 * BUFFER * TILE + t16 * 16 * ROW));
        return x.whole;
    }
    template <int BUFFER> __device__ __forceinline__ void add_values(const uint32_t (&p)[KT][8]) {
#pragma unroll
        for (int t16 = 0; t16 < KEYS / 16; ++t16)
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] = mfma_32x32x16_bf16(__builtin_bit_cast(v8bf, v_operand<BUFFER>(t16, d)), p_operand(p, t16), o[d]);
    }
};

}  // namespace w4a8
