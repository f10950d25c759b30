// Attention of one token per sequence over the paged cache, with a prefix that the whole batch shares.
//   o_b = sum_j softmax_j(q_b . k_j * scale) v_j,   j over the prefix's tokens and then sequence b's own
// Every byte of keys and values is read once from memory per 16 rows that see it: a row is one query head of one sequence; the rows of
// a sequence that share a key head (and, in the prefix, those of all sequences) are the columns of one matrix product.  The keys are
// cut into ranges, one per workgroup, whose partial results (maximum, sum and unnormalized output per row, in float32) a second launch joins.
// A wavefront takes 32 keys at a time, two such steps under way: S^T = K Q^T from keys as they lie in a page, then O^T = V^T P^T, whose
// first operand needs eight keys of a channel in one lane -- a lane loads eight keys by eight channels and turns them in registers.  Memory
// bounds it: 16 KB of bf16 keys and values per 16 matrix instructions.
#include "attention.hpp"
#include "attention_device.hpp"

namespace w4a8 {
namespace {

constexpr int STEP = 32, WAVES_D = 4;

// N bytes of a lane's part of a row.
template <int N> struct Piece;
template <> struct Piece<16> { u32x4 w; };
template <> struct Piece<8> { uint32_t w __attribute__((ext_vector_type(2))); };
template <> struct Piece<4> { uint32_t w __attribute__((ext_vector_type(1))); };

template <int D, bool E4M3> struct Step {
    static constexpr int SIZE = E4M3 ? 1 : 2, ROW = D * SIZE;
    static constexpr int KL = ROW / 64;                          // 16-byte loads of a key row per lane (four lanes share a row)
    static constexpr int VB = ROW / 16;                          // bytes of a value row per lane (sixteen lanes share one)
    u32x4 k[2][KL];                                              // keys (16 kt + lane % 16), 16 bytes at 64 i + 16 (lane / 16)
    Piece<VB> v[8];                                              // keys 4 (lane / 16) + {0..3} and 16 more, channels VB / SIZE * (lane % 16) ..
};

// The channel that element i (0..7) of the operand of step s holds in a lane of group kg, the same for keys and queries.
template <int D, bool E4M3> __device__ __forceinline__ constexpr int channel(int s, int kg) {
    return E4M3 ? 64 * (s / 2) + 16 * kg + 8 * (s & 1) : 32 * s + 8 * kg;
}

template <int D, bool E4M3, typename OutT>
__global__ void __launch_bounds__(64 * WAVES_D, 2) attention_decode_kernel(DecodeArgs a, DecodePlan plan, int own_units, int row_tiles,
                                                                           int prefix_row_tiles) {
    using S = Step<D, E4M3>;
    constexpr int KS = D / 32, VD = D / 16;                      // operands of a key row; channels of a lane's values
    __shared__ __attribute__((aligned(16))) float lds_o[WAVES_D][16][D];
    __shared__ float lds_m[WAVES_D][16], lds_l[WAVES_D][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, kg = lane >> 4;
    const int group = a.q_heads / a.c.kv_heads;

    // this workgroup's rows, key head and range of keys
    const bool prefix = (int)blockIdx.x >= own_units;
    int unit = prefix ? blockIdx.x - own_units : blockIdx.x;
    int kv_head, part, first_row, rows;
    int64_t n_keys;
    const int32_t* pages;
    if (prefix) {
        const int rt = unit % prefix_row_tiles;
        unit /= prefix_row_tiles;
        const int split = unit % plan.prefix_splits;
        kv_head = unit / plan.prefix_splits;
        part = plan.own_splits + split;
        unit = split;
        first_row = rt * 16;
        rows = a.n_seqs * group;
        n_keys = a.prefix_len;
        pages = a.prefix_pages;
    } else {
        part = unit % plan.own_splits;
        unit /= plan.own_splits;
        const int rt = unit % row_tiles;
        unit /= row_tiles;
        kv_head = unit % a.c.kv_heads;
        const int b = unit / a.c.kv_heads;
        unit = part;
        first_row = b * group + rt * 16;
        rows = (b + 1) * group;
        const int64_t cap = a.table_width << a.c.page_shift, n = a.lengths[b];
        n_keys = n < 0 ? 0 : n < cap ? n : cap;
        pages = a.tables + b * a.ld_tables;
    }
    // row i of the tile: row first_row + i of (sequence, query head of this key head)
    const int row = first_row + c;
    const bool there = row < rows;
    const int seq = there ? row / group : 0, head = kv_head * group + (there ? row % group : 0);
    const int splits = prefix ? plan.prefix_splits : plan.own_splits;
    const int64_t per_split = ((n_keys + splits - 1) / splits + STEP - 1) / STEP * STEP;
    const int64_t k_begin = per_split * unit, k_end = n_keys < k_begin + per_split ? n_keys : k_begin + per_split;

    v8bf qf[KS];
    {
        const uint16_t* q = a.q + (int64_t)seq * a.ldq + (int64_t)head * D;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const v8bf*>(q + channel<D, E4M3>(s, kg));
    }
    const float score_scale = a.scale_log2 * (E4M3 ? a.kv_scales[0] : 1.0f);

    v4f o[VD];                                                   // o[j][r]: channel VD (4 kg + r) + j of row c
#pragma unroll
    for (int j = 0; j < VD; ++j) o[j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float m = NEG_INF, l = 0.0f;

    // sixteen keys never straddle a page; a page that is no page holds no tokens
    auto page_at = [&](int64_t key, bool& ok) {
        const int64_t p = key < k_end ? pages[key >> a.c.page_shift] : -1;
        ok = p >= 0 && p < a.c.n_pages;
        return ok ? p : 0;
    };
    auto load = [&](S& x, int64_t key, bool (&ok)[2]) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int64_t base = key + 16 * kt;
            const int64_t page = page_at(base, ok[kt]);
            const int64_t at = page * a.c.page_stride + ((int64_t)kv_head * a.c.page_size + (base & (a.c.page_size - 1))) * D;
            const uint8_t* kp = a.k_cache + at * S::SIZE;
            const uint8_t* vp = a.v_cache + at * S::SIZE;
#pragma unroll
            for (int i = 0; i < S::KL; ++i) x.k[kt][i] = *reinterpret_cast<const u32x4*>(kp + c * S::ROW + 64 * i + 16 * kg);
#pragma unroll
            for (int r = 0; r < 4; ++r) x.v[4 * kt + r] = *reinterpret_cast<const Piece<S::VB>*>(vp + (4 * kg + r) * S::ROW + S::VB * c);
        }
    };
    auto compute = [&](const S& x, int64_t key, const bool (&ok)[2]) {
        v4f s[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            s[kt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                v8bf kf;
                if (E4M3) {
                    const uint32_t w0 = x.k[kt][i / 2][2 * (i & 1)], w1 = x.k[kt][i / 2][2 * (i & 1) + 1];
                    kf = __builtin_bit_cast(v8bf, u32x4{e4m3_to_bf16<false>(w0), e4m3_to_bf16<true>(w0), e4m3_to_bf16<false>(w1), e4m3_to_bf16<true>(w1)});
                } else {
                    kf = __builtin_bit_cast(v8bf, x.k[kt][i]);
                }
                s[kt] = mfma_16x16x32_bf16(kf, qf[i], s[kt]);
            }
        }
        const bool whole = key + STEP <= k_end && ok[0] && ok[1];
        bool seen[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int kt = i / 4, r = i % 4;
            seen[i] = whole || (ok[kt] && key + 16 * kt + 4 * kg + r < k_end);
            if (!seen[i]) s[kt][r] = NEG_INF;
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        mx = max_over_32(max_over_16(mx)) * score_scale;
        const float m_new = fmaxf(m, mx);
        const float m_use = m_new == NEG_INF ? 0.0f : m_new;
        if (__builtin_amdgcn_ballot_w64(m_new > m)) {
            const float alpha = exp2_fast(m - m_use);
            l *= alpha;
#pragma unroll
            for (int j = 0; j < VD; ++j) o[j] *= alpha;
            m = m_new;
        }
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = exp2_fast(fmaf(s[i / 4][i % 4], score_scale, -m_use));
            l += p[i];
        }
        const v8bf pf = __builtin_bit_cast(v8bf, u32x4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])});
        // values as bf16 pairs of channels; what no row sees may hold anything and counts as zero
        uint32_t v[8][VD / 2];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < VD / 2; ++j) {
                uint32_t w;
                if (E4M3) w = j & 1 ? e4m3_to_bf16<true>(x.v[i].w[j / 2]) : e4m3_to_bf16<false>(x.v[i].w[j / 2]);
                else w = x.v[i].w[j];
                v[i][j] = seen[i] ? w : 0u;
            }
#pragma unroll
        for (int j = 0; j < VD; ++j) {
            const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], sel);
            o[j] = mfma_16x16x32_bf16(__builtin_bit_cast(v8bf, w), pf, o[j]);
        }
    };
    constexpr int STRIDE = STEP * WAVES_D;
    int64_t key = k_begin + STEP * wave;
    S x0, x1;
    bool ok0[2], ok1[2];
    if (key < k_end) load(x0, key, ok0);
    while (key < k_end) {
        if (key + STRIDE < k_end) load(x1, key + STRIDE, ok1);
        compute(x0, key, ok0);
        key += STRIDE;
        if (key >= k_end) break;
        if (key + STRIDE < k_end) load(x0, key + STRIDE, ok0);
        compute(x1, key, ok1);
        key += STRIDE;
    }

    // the four wavefronts' results joined
    l = sum_over_32(sum_over_16(l));
#pragma unroll
    for (int j = 0; j < VD; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) lds_o[wave][c][VD * (4 * kg + r) + j] = o[j][r];
    if (kg == 0) {
        lds_m[wave][c] = m;
        lds_l[wave][c] = l;
    }
    __syncthreads();
    const int out_row = threadIdx.x / 16, ch = threadIdx.x % 16 * VD;   // VD channels of a row per thread
    if (first_row + out_row >= rows) return;
    float top = NEG_INF, sum = 0.0f, acc[VD];
#pragma unroll
    for (int w = 0; w < WAVES_D; ++w) top = fmaxf(top, lds_m[w][out_row]);
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES_D; ++w) {
        const float mw = lds_m[w][out_row];
        const float f = mw == NEG_INF ? 0.0f : exp2_fast(mw - top);
        sum = fmaf(lds_l[w][out_row], f, sum);
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[j] = fmaf(lds_o[w][out_row][ch + j], f, acc[j]);
    }
    if (E4M3) {
        const float vs = a.kv_scales[1];
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[j] *= vs;
    }
    const int r = first_row + out_row;
    const int64_t at = (int64_t)(r / group) * a.q_heads + kv_head * group + r % group;   // (sequence, query head)
    if (plan.parts == 0) {
        const float inv = inverse_sum(sum);
        const StaticQuantizer quant(a.y_scale ? *a.y_scale : 1.0f);
        OutT* y = static_cast<OutT*>(a.y) + (int64_t)(r / group) * a.ldy + (int64_t)(kv_head * group + r % group) * D + ch;
#pragma unroll
        for (int j = 0; j < VD; j += 4) store_4(y + j, acc[j] * inv, acc[j + 1] * inv, acc[j + 2] * inv, acc[j + 3] * inv, quant);
    } else {
        const int64_t total = (int64_t)a.n_seqs * a.q_heads;
        float* out = a.partial + (part * total + at) * D + ch;
#pragma unroll
        for (int j = 0; j < VD; j += 4) *reinterpret_cast<float4*>(out + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
        if (ch == 0) reinterpret_cast<float2*>(a.partial + plan.parts * total * D)[part * total + at] = make_float2(top, sum);
    }
}

// Joins the parts of every row: 16 lanes per row.
template <int D, typename OutT>
__global__ void __launch_bounds__(256) attention_join_kernel(DecodeArgs a, int parts) {
    constexpr int VD = D / 16;
    const int64_t total = (int64_t)a.n_seqs * a.q_heads, row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    if (row >= total) return;
    const int ch = threadIdx.x % 16 * VD;
    const float2* ml = reinterpret_cast<const float2*>(a.partial + parts * total * D) + row;
    float top = NEG_INF, sum = 0.0f, acc[VD];
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = 0.0f;
    for (int p = 0; p < parts; ++p) top = fmaxf(top, ml[p * total].x);
    for (int p = 0; p < parts; ++p) {
        const float2 t = ml[p * total];
        if (t.x == NEG_INF) continue;
        const float f = exp2_fast(t.x - top);
        sum = fmaf(t.y, f, sum);
        const float* part = a.partial + (p * total + row) * D + ch;
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[j] = fmaf(part[j], f, acc[j]);
    }
    const float inv = inverse_sum(sum);
    const StaticQuantizer quant(a.y_scale ? *a.y_scale : 1.0f);
    OutT* y = static_cast<OutT*>(a.y) + row / a.q_heads * a.ldy + row % a.q_heads * D + ch;
#pragma unroll
    for (int j = 0; j < VD; j += 4) store_4(y + j, acc[j] * inv, acc[j + 1] * inv, acc[j + 2] * inv, acc[j + 3] * inv, quant);
}

template <int D, bool E4M3, typename OutT>
void launch_typed(const DecodeArgs& a, const DecodePlan& p, hipStream_t st) {
    const int group = a.q_heads / a.c.kv_heads, row_tiles = (group + 15) / 16;
    const int prefix_row_tiles = (int)(((int64_t)a.n_seqs * group + 15) / 16);
    const int own = a.n_seqs * a.c.kv_heads * row_tiles * p.own_splits, shared = a.c.kv_heads * prefix_row_tiles * p.prefix_splits;
    hipLaunchKernelGGL((attention_decode_kernel<D, E4M3, OutT>), dim3((unsigned)(own + shared)), dim3(64 * WAVES_D), 0, st, a, p, own,
                       row_tiles, prefix_row_tiles);
    if (p.parts > 0) {
        const int64_t rows = (int64_t)a.n_seqs * a.q_heads;
        hipLaunchKernelGGL((attention_join_kernel<D, OutT>), dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, st, a, p.parts);
    }
}

template <int D, bool E4M3>
void launch_out(const DecodeArgs& a, const DecodePlan& p, hipStream_t st) {
    if (a.y_scale) launch_typed<D, E4M3, uint8_t>(a, p, st);
    else launch_typed<D, E4M3, uint16_t>(a, p, st);
}

}  // namespace

int launch_attention_decode(const DecodeArgs& a, const DecodePlan& p, hipStream_t st) {
    if (a.c.head_dim == 128) {
        if (a.c.e4m3) launch_out<128, true>(a, p, st);
        else launch_out<128, false>(a, p, st);
    } else {
        if (a.c.e4m3) launch_out<64, true>(a, p, st);
        else launch_out<64, false>(a, p, st);
    }
    return launch_status();
}

}  // namespace w4a8
