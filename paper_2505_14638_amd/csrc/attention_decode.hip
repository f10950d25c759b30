// Attention of one token per sequence over the paged cache, with a prefix that the whole batch shares.
//   o_b = sum_j softmax_j(q_b . k_j * scale) v_j,   j over the prefix's tokens and then sequence b's own
// Every byte of keys and values is read once from memory per 16 rows that see it: a row is one query head of one sequence; the rows of
// a sequence that share a key head (and, in the prefix, those of all sequences) are the columns of one matrix product.  The keys are
// cut into ranges, one per workgroup, whose partial results (maximum, sum and unnormalized output per row, in float32) a second launch joins.
// A wavefront takes 32 keys at a time, two such steps under way: S^T = K Q^T from keys as they lie in a page, then O^T = V^T P^T, whose
// first operand needs eight keys of a channel in one lane -- a lane loads eight keys by eight channels and turns them in registers.  Memory
// bounds it: 16 KB of bf16 keys and values per 16 matrix instructions.  16 sequences of 4000 tokens, 32 query and 8 key heads of 128 channels:
// 52 us, 5.0 TB/s; 64 sequences of 200 .. 8192, 64 heads, E4M3 (552 MB): 122 .. 132 us, 4.2 .. 4.5 TB/s, a copy's rate is 4.8; one
// sequence of 1000 tokens 7.4 us, two launches.
#include "attention.hpp"
#include "attention_tile.hpp"

namespace w4a8 {
namespace {

constexpr int STEP = 32, WAVES_D = 4;                           // keys of a step; wavefronts of most workgroups

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

// One workgroup of W wavefronts: up to 16 rows of a key head against a range of one sequence's tokens, or of the prefix's (unit counted
// from own_units).  OutT: bf16 or E4M3 rows, finished; void: a partial result.
template <int D, int W> constexpr int stream_lds() { return W * 16 * (D + 4 + 2) * 4; }
template <int D, bool E4M3, int W, typename OutT>
__device__ __forceinline__ void stream_keys(const DecodeArgs& a, const DecodePlan& plan, int unit, int own_units, uint8_t* lds) {
    using S = Step<D, E4M3>;
    constexpr int KS = D / 32, VD = D / 16;                      // operands of a key row; channels of a lane's values
    constexpr int PITCH = D + 4;                                 // floats: rows of the exchange start in different banks
    float* lds_o = reinterpret_cast<float*>(lds);                // [W][16][PITCH], then maxima and sums [W][16]
    float *lds_m = lds_o + W * 16 * PITCH, *lds_l = lds_m + W * 16;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int c = lane & 15, kg = lane >> 4;
    const int group = a.q_heads / a.c.kv_heads;

    // this workgroup's rows, key head and range of keys
    const bool prefix = unit >= own_units;
    int kv_head, part, first_row, rows;
    int64_t n_keys, listed;                                      // tokens; tokens that the table has room for
    const int32_t* pages;
    if (prefix) {
        const int row_tiles = (a.n_seqs * group + 15) / 16;
        unit -= own_units;
        const int rt = unit % row_tiles;
        unit /= row_tiles;
        const int split = unit % plan.prefix_splits;
        kv_head = unit / plan.prefix_splits;
        part = plan.own_splits + split;
        unit = split;
        first_row = rt * 16;
        rows = a.n_seqs * group;
        n_keys = listed = a.prefix_len;
        pages = a.prefix_pages;
    } else {
        const int row_tiles = (group + 15) / 16;
        part = unit % plan.own_splits;
        unit /= plan.own_splits;
        const int rt = unit % row_tiles;
        unit /= row_tiles;
        kv_head = unit % a.c.kv_heads;
        const int b = unit / a.c.kv_heads;
        unit = part;
        first_row = b * group + rt * 16;
        rows = (b + 1) * group;
        listed = a.table_width << a.c.page_shift;
        const int64_t n = a.lengths[b];
        n_keys = n < 0 ? 0 : n < listed ? n : listed;
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

    // Sixteen keys never straddle a page; a page that is no page holds no tokens.  The page numbers of this wavefront's next 32 steps
    // are in its lanes (step n's in 2 n and 2 n + 1), so that a step does not wait for them.
    constexpr int STRIDE = STEP * W;
    int listing = -1;
    auto list_pages = [&](int64_t key) {                         // of the steps from `key` on
        const int64_t mine = key + (int64_t)(lane >> 1) * STRIDE + 16 * (lane & 1);
        const int p = mine < listed ? pages[mine >> a.c.page_shift] : -1;   // not mine < k_end: that waits for the length
        listing = p < a.c.n_pages ? p : -1;
    };
    auto load = [&](S& x, int64_t key, int n, bool (&ok)[2]) {   // step n of this wavefront, at `key`
        if (n > 0 && (n & 31) == 0) list_pages(key);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int page = __builtin_amdgcn_readlane(listing, 2 * (n & 31) + kt);
            ok[kt] = page >= 0;
            const int64_t base = key + 16 * kt;
            const int64_t at = (ok[kt] ? page : 0) * a.c.page_stride + ((int64_t)kv_head * a.c.page_size + (base & (a.c.page_size - 1))) * D;
            const uint8_t* kp = a.k_cache + at * S::SIZE;
            const uint8_t* vp = a.v_cache + at * S::SIZE;
#pragma unroll
            for (int i = 0; i < S::KL; ++i) x.k[kt][i] = *reinterpret_cast<const u32x4*>(kp + c * S::ROW + 64 * i + 16 * kg);
#pragma unroll
            for (int r = 0; r < 4; ++r) x.v[4 * kt + r] = *reinterpret_cast<const Piece<S::VB>*>(vp + (4 * kg + r) * S::ROW + S::VB * c);
        }
    };
    auto compute = [&](S& x, int64_t key, const bool (&ok)[2]) {
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
        // what no row sees may hold anything and counts as zero (a loop of at most one pass: as a branch it would cost every step)
        int hides = uniform(!(key + STEP <= k_end && ok[0] && ok[1]));
        while (hides) {
            int64_t left = k_end - key - 4 * kg;
            asm volatile("" : "+v"(left));
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!ok[i / 4] || 16 * (i / 4) + i % 4 >= left) {
                    s[i / 4][i % 4] = NEG_INF;
                    x.v[i] = Piece<S::VB>{};
                }
            asm volatile("s_mov_b32 %0, 0" : "=s"(hides));
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        mx = max_over_32(max_over_16(mx)) * score_scale;
        if (__builtin_amdgcn_ballot_w64(mx > m + RISE)) {
            const float m_new = fmaxf(m, mx), alpha = m_new == NEG_INF ? 1.0f : exp2_fast(m - m_new);
            l *= alpha;
#pragma unroll
            for (int j = 0; j < VD; ++j) o[j] *= alpha;
            m = m_new;
        }
        const float m_use = m == NEG_INF ? 0.0f : m;
        u32x4 p;                                                 // rounded to bf16, as the product takes them, and so in the sum: they come to one
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v4f& x = s[i / 2];
            const int r = 2 * (i & 1);
            p[i] = pack_bf16(exp2_fast(fmaf(x[r], score_scale, -m_use)), exp2_fast(fmaf(x[r + 1], score_scale, -m_use)));
            l = add_pair(p[i], l);
        }
        const v8bf pf = __builtin_bit_cast(v8bf, p);
        // values as bf16 pairs of channels
        uint32_t v[8][VD / 2];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < VD / 2; ++j) {
                if (E4M3) v[i][j] = j & 1 ? e4m3_to_bf16<true>(x.v[i].w[j / 2]) : e4m3_to_bf16<false>(x.v[i].w[j / 2]);
                else v[i][j] = x.v[i].w[j];
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
    S x0, x1;
    bool ok0[2], ok1[2];
    int64_t key = k_begin + STEP * wave;
    list_pages(key);
    if (key < k_end) load(x0, key, 0, ok0);
    for (int n = 0; key < k_end; n += 2) {
        if (key + STRIDE < k_end) load(x1, key + STRIDE, n + 1, ok1);
        compute(x0, key, ok0);
        key += STRIDE;
        if (key >= k_end) break;
        if (key + STRIDE < k_end) load(x0, key + STRIDE, n + 2, ok0);
        compute(x1, key, ok1);
        key += STRIDE;
    }

    if (__builtin_amdgcn_ballot_w64(m == NEG_INF)) {             // no tokens, or no score above -infinity?
        bool saw = false;
        for (key = k_begin + STEP * wave; key < k_end && !saw; key += STRIDE)
            for (int64_t at = key; at < key + STEP && at < k_end; at += 16) saw |= (uint32_t)pages[at >> a.c.page_shift] < a.c.n_pages;
        if (saw) m = fmaxf(m, LOWEST);
    }

    // the wavefronts' results joined
    l = sum_over_32(sum_over_16(l));
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VD; j += 4)
            *reinterpret_cast<float4*>(lds_o + (wave * 16 + c) * PITCH + VD * (4 * kg + r) + j) = make_float4(o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]);
    if (kg == 0) {
        lds_m[wave * 16 + c] = m;
        lds_l[wave * 16 + c] = l;
    }
    __syncthreads();
    const int out_row = threadIdx.x / 16, ch = threadIdx.x % 16 * VD;   // VD channels of a row per thread
    if (out_row >= 16 || first_row + out_row >= rows) return;
    float top = NEG_INF, sum = 0.0f, acc[VD];
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, lds_m[w * 16 + out_row]);
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const float mw = lds_m[w * 16 + out_row];
        const float f = mw == NEG_INF ? 0.0f : exp2_fast(mw - top);
        sum = fmaf(lds_l[w * 16 + out_row], f, sum);
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[j] = fmaf(lds_o[(w * 16 + out_row) * PITCH + ch + j], f, acc[j]);
    }
    if (E4M3) {
        const float vs = a.kv_scales[1];
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[j] *= vs;
    }
    const int r = first_row + out_row;
    const int64_t at = (int64_t)(r / group) * a.q_heads + kv_head * group + r % group;   // (sequence, query head)
    if constexpr (!std::is_void_v<OutT>) {
        const float inv = inverse_sum(top, sum);
        const Bf16Quantizer quant(a.y_scale ? *a.y_scale : 1.0f);
        OutT* y = static_cast<OutT*>(a.y) + (int64_t)(r / group) * a.ldy + (int64_t)(kv_head * group + r % group) * D + ch;
#pragma unroll
        for (int j = 0; j < VD; j += 4) store_4(y + j, acc[j] * inv, acc[j + 1] * inv, acc[j + 2] * inv, acc[j + 3] * inv, quant);
    } else {
        const int64_t total = (int64_t)a.n_seqs * a.q_heads;
        float* out = a.partial + (part * total + at) * D + ch;
        if (k_begin < k_end)                                     // (what nothing is in is not read either)
#pragma unroll
        for (int j = 0; j < VD; j += 4) *reinterpret_cast<float4*>(out + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
        if (ch == 0) reinterpret_cast<float2*>(a.partial + plan.parts * total * D)[part * total + at] = make_float2(top, sum);
    }
}

template <int D, bool E4M3, int W, typename OutT>
__global__ void __launch_bounds__(64 * W, 2) attention_stream_kernel(DecodeArgs a, DecodePlan plan, int own_units) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[stream_lds<D, W>()];
    stream_keys<D, E4M3, W, OutT>(a, plan, blockIdx.x, own_units, lds);
}

// A lane's 16 bytes of `base` + its own offset to LDS byte address lds_addr + 16 * lane, as lds_dma_16, offsets beyond 32 bits.
__device__ __forceinline__ void lds_dma_16_far(const uint8_t* from, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(lds_addr) : "memory", "m0");
}

// The prefix for many rows: all sequences' rows of a key head, 32 per wavefront, walk a range of the prefix's tokens in tiles of 64 keys,
// which the wavefronts share in LDS.  Pages are read 16 tokens at a time (sixteen never straddle a page), one tile ahead; E4M3 becomes
// bf16 on its way to LDS.  Ends in a partial result per row.
// One wavefront on each vector unit takes 1.37 us for a tile of 64 keys by 128 rows, 32 matrix instructions (0.55 us) and then the weights; a
// prefix of 8192 tokens under 256 sequences of 64 heads, alone: 105 us, 650 TFLOP/s.  Scores formed one tile ahead, beside the weights, gain
// 10 % of that alone (E4M3: lose 15 %, its conversions and the second set of scores do not fit the registers), and with other sequences'
// own tokens on the same units lose 10 .. 25 %: the other workgroups fill these gaps already.
template <int D, bool E4M3>
__device__ __forceinline__ void walk_prefix(const DecodeArgs& a, const DecodePlan& plan, int block, int row_tiles, int units, uint8_t* lds) {
    using Block = RowBlock<D>;
    constexpr int WAVES = WAVES_D, BM = 32 * WAVES, ROW = Block::ROW, PIECES = Block::PIECES, TILE = Block::TILE, RPC = Block::RPC, KT = Block::KT;
    constexpr int GROUPS = 4 / WAVES;                            // of 16 keys, that a wavefront brings of every tile
    constexpr int SIZE = E4M3 ? 1 : 2, LOADS = 16 * D * SIZE / 1024;   // 64 x 16 bytes per group
    static_assert(BM * ROW <= 2 * TILE, "Q fits two tiles");
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;

    // row tiles of one range of keys run on one XCD, whose L2 then serves the range to all but the first
    const int per_xcd = (units + 7) / 8;
    int unit = block % 8 * per_xcd + block / 8;
    if (block / 8 >= per_xcd || unit >= units) return;
    const int row_tile = unit % row_tiles;
    unit /= row_tiles;
    const int split = unit % plan.prefix_splits, kv_head = unit / plan.prefix_splits;
    const int group = a.q_heads / a.c.kv_heads, n_rows = a.n_seqs * group;
    const int first = row_tile * BM + 32 * wave;                 // this wavefront's rows: (sequence, query head of the key head)
    const int tiles = (int)((a.prefix_len + TILE_KEYS - 1) / TILE_KEYS), per = (tiles + plan.prefix_splits - 1) / plan.prefix_splits;
    const int t_begin = min(split * per, tiles), t_end = min(t_begin + per, tiles);

    const float score_scale = a.scale_log2 * (E4M3 ? a.kv_scales[0] : 1.0f);

    // pages of the tile's four groups of 16 keys, in lanes 0..3; -1: no tokens there
    auto pages_of = [&](int t) {
        const int64_t key = (int64_t)t * TILE_KEYS + 16 * (lane & 3);
        const int p = t < t_end && key < a.prefix_len ? a.prefix_pages[key >> a.c.page_shift] : -1;
        return p < a.c.n_pages ? p : -1;
    };
    u32x4 held[E4M3 ? 2 * GROUPS * LOADS : 1];                   // E4M3 on its way to LDS
    // Brings this wavefront's groups of tile t to the buffer (E4M3: to registers).  What no row sees must still be numbers among the values: rows
    // behind the prefix's end repeat its last key, and its last value only as E4M3, which has no infinities; bf16 values there are zeros, as
    // all of a group without tokens.
    auto fetch = [&](int t, int pages, int buffer) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int grp = wave * GROUPS + g;
            const int64_t key = (int64_t)t * TILE_KEYS + 16 * grp;
            const int page = __builtin_amdgcn_readlane(pages, grp);
            const uint32_t to = lds_base + 2 * buffer * TILE + 16 * grp * ROW;
            if (page < 0) {
                if (E4M3) {
#pragma unroll
                    for (int i = 0; i < 2 * LOADS; ++i) held[2 * LOADS * g + i] = u32x4{0, 0, 0, 0};
                } else {
#pragma unroll
                    for (int i = 0; i < 2 * LOADS; ++i)
                        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>((uintptr_t)(to + i / LOADS * TILE + i % LOADS * 1024 + lane * 16)) =
                            u32x4{0, 0, 0, 0};
                }
                continue;
            }
            const int64_t at = (page * a.c.page_stride + ((int64_t)kv_head * a.c.page_size + (key & (a.c.page_size - 1))) * D) * SIZE;
            const int last = (int)(a.prefix_len - 1 - key);      // of the group's rows, if below 15
            auto copy = [&](int i, bool ends) {                  // ends: the prefix, in this group
                const int r = i * RPC + lane / PIECES;
                const uint32_t off = (uint32_t)((ends ? min(r, last) : r) * ROW + ((lane % PIECES) ^ swizzle<D>(r)) * 16);
                lds_dma_16(a.k_cache + at, off, to + i * 1024);
                if (!ends) lds_dma_16(a.v_cache + at, off, to + TILE + i * 1024);
                else lds_write(to + TILE + i * 1024 + lane * 16, r > last ? u32x4{0, 0, 0, 0} : *reinterpret_cast<const u32x4*>(a.v_cache + at + off));
            };
            if (E4M3) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const int byte = (i * 64 + lane) * 16, r = min(byte / D, last);
                    held[2 * LOADS * g + i] = *reinterpret_cast<const u32x4*>(a.k_cache + at + r * D + byte % D);
                    held[2 * LOADS * g + LOADS + i] = *reinterpret_cast<const u32x4*>(a.v_cache + at + r * D + byte % D);
                }
            } else if (last >= 15) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) copy(i, false);
            } else {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) copy(i, true);
            }
        }
    };
    auto put = [&](int buffer) {                                 // held E4M3 to LDS as bf16
#pragma unroll
        for (int i = 0; i < 2 * GROUPS * LOADS; ++i) {
            const int g = i / (2 * LOADS), is_v = i / LOADS & 1, byte = (i % LOADS * 64 + lane) * 16, r = byte / D, piece = byte % D / 8;
            const uint32_t to = lds_base + (2 * buffer + is_v) * TILE + (16 * (wave * GROUPS + g) + r) * ROW;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w0 = held[i][2 * h], w1 = held[i][2 * h + 1];
                *reinterpret_cast<__attribute__((address_space(3))) u32x4*>((uintptr_t)(to + (((piece + h) ^ swizzle<D>(r)) << 4))) =
                    u32x4{e4m3_to_bf16<false>(w0), e4m3_to_bf16<true>(w0), e4m3_to_bf16<false>(w1), e4m3_to_bf16<true>(w1)};
            }
        }
    };
    // Fetched a tile before their use, their pages a tile before that.
    int pages = pages_of(t_begin);
    uint32_t bad = 0;                                            // four bits a tile, the latest lowest: its groups that hold no tokens
    auto fetch_next = [&](int t, int buffer) {
        bad = bad << 4 | ((uint32_t)__builtin_amdgcn_ballot_w64(pages < 0) & 15);
        const int now = pages;
        pages = pages_of(t + 1);
        if (t < t_end) fetch(t, now, buffer);
    };
    // the rows of Q, a wavefront's own, on their way together with the first tile
    Block rows(lds_base, lane);
    rows.clear();
#pragma unroll
    for (int q = 0; q < 32 / RPC; ++q) {
        const int r = q * RPC + lane / PIECES, at = min(first + r, n_rows - 1);
        lds_dma_16_far(reinterpret_cast<const uint8_t*>(a.q + (int64_t)(at / group) * a.ldq + (int64_t)(kv_head * group + at % group) * D) +
                           ((lane % PIECES) ^ swizzle<D>(r)) * 16,
                       lds_base + 2 * TILE + (32 * wave + q * RPC) * ROW);
    }
    fetch_next(t_begin, 0);
    if (E4M3 && t_begin < t_end) put(0);
    lds_dma_wait_all();
    rows.read_q(2 * TILE + wave * 32 * ROW);
    const bool works = first < n_rows;                           // (wave-uniform) this wavefront has rows
    auto step = [&](int t, auto buffer_c) {
        constexpr int buffer = decltype(buffer_c)::value;
        if (!E4M3) lds_dma_wait_all();
        __syncthreads();
        fetch_next(t + 1, buffer ^ 1);
        if (works) {
            v16f s[KT];
            rows.template scores<buffer>(s);
            const int64_t left = a.prefix_len - (int64_t)t * TILE_KEYS;
            const uint32_t none = bad >> 4 & 15;                     // of this tile's groups
            int hides = uniform(left < TILE_KEYS || none);
            while (hides) {                                      // a loop of at most one pass, as in the kernel of prompts
                int edge = (int)min(left, (int64_t)TILE_KEYS) - 4 * half;
                asm volatile("" : "+v"(edge));
#pragma unroll
                for (int k = 0; k < KT; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * k + (r & 3) + 8 * (r >> 2) >= edge || (none >> (2 * k + r / 8) & 1)) s[k][r] = NEG_INF;
                asm volatile("s_mov_b32 %0, 0" : "=s"(hides));
            }
            uint32_t p[KT][8];
            rows.weights(s, score_scale, p);
            rows.template add_values<buffer>(p);
        }
        if (E4M3 && t + 1 < t_end) put(buffer ^ 1);
    };
    for (int t = t_begin; t < t_end; t += 2) {
        step(t, std::integral_constant<int, 0>{});
        if (t + 1 < t_end) step(t + 1, std::integral_constant<int, 1>{});
    }
    const float sum = sum_over_32(rows.l), v_scale = E4M3 ? a.kv_scales[1] : 1.0f;
    if (__builtin_amdgcn_ballot_w64(rows.m == NEG_INF)) {        // no tokens, or no score above -infinity?
        bool saw = false;
        for (int t = t_begin; t < t_end && !saw; ++t) saw = __builtin_amdgcn_ballot_w64(pages_of(t) >= 0);
        if (saw) rows.m = fmaxf(rows.m, LOWEST);
    }
    const int r = first + col;
    if (r >= n_rows) return;
    const int64_t total = (int64_t)a.n_seqs * a.q_heads, part = plan.own_splits + split;
    const int64_t at = (int64_t)(r / group) * a.q_heads + kv_head * group + r % group;
    float* out = a.partial + (part * total + at) * D + 4 * half;
#pragma unroll
    for (int d = 0; d < Block::DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<float4*>(out + 32 * d + 2 * i) =
                make_float4(rows.o[d][i] * v_scale, rows.o[d][i + 1] * v_scale, rows.o[d][i + 2] * v_scale, rows.o[d][i + 3] * v_scale);
    if (half == 0) reinterpret_cast<float2*>(a.partial + plan.parts * total * D)[part * total + at] = make_float2(rows.m, sum);
}

// The prefix for many rows and the sequences' own tokens in one launch: the workgroups on the prefix come first, mostly one for every
// compute unit or fewer, and those on the own tokens, which memory bounds, run beside them.  256 sequences, 64 heads, 8191 E4M3 tokens in
// common and 30 .. 1000 of their own: 124 us, where the two take 105 and 62 apart; with twice the workgroups on the prefix, which then leave
// no room beside them, 156.
template <int D, bool E4M3>
__global__ void __launch_bounds__(64 * WAVES_D, 2) attention_shared_kernel(DecodeArgs a, DecodePlan plan, int own_units, int row_tiles, int units,
                                                                           int prefix_blocks) {
    constexpr int BYTES = 4 * RowBlock<D>::TILE;
    static_assert(stream_lds<D, WAVES_D>() <= BYTES, "either body's LDS");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[BYTES];
    if ((int)blockIdx.x < prefix_blocks) walk_prefix<D, E4M3>(a, plan, blockIdx.x, row_tiles, units, lds);
    else stream_keys<D, E4M3, WAVES_D, void>(a, plan, blockIdx.x - prefix_blocks, own_units, lds);
}

// Joins the parts of a row, a wavefront per row, or four of them where a row has more parts than one reads at once and the rows are no more than
// the compute units: every lane weighs a part (or two), then sixteen lanes read a part's channels.  Latency bounds it: one sequence of 16000 tokens
// in 64 parts, stream and join, 17.0 us, 20.4 with one wavefront a row; 32 sequences behind 4096 tokens (1024 rows, 17 parts) the other way
// round, 21.4 and 16.7.
constexpr int PARTS_AT_ONCE = 16, FEW_ROWS = 256;
template <int D, int WAVES, typename OutT>
__global__ void __launch_bounds__(256) attention_join_kernel(DecodeArgs a, int parts) {
    constexpr int VD = D / 16;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), first = wave % WAVES * PARTS_AT_ONCE;
    const int64_t total = (int64_t)a.n_seqs * a.q_heads, row = (int64_t)blockIdx.x * (4 / WAVES) + wave / WAVES;
    if (row >= total) return;
    const int ch = lane % 16 * VD;
    const float* from = a.partial + row * D + ch;
    float4 x[4][VD / 4];
    auto load = [&](int base) {                                  // parts base + {0 .. 15}; one that nothing is in may hold anything
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = base + 4 * i + lane / 16;
            if (p < parts)
#pragma unroll
                for (int j = 0; j < VD / 4; ++j) x[i][j] = *reinterpret_cast<const float4*>(from + p * total * D + 4 * j);
        }
    };
    load(first);                                                 // before their weights are known: one wait instead of two
    const float2* ml = reinterpret_cast<const float2*>(a.partial + parts * total * D) + row;
    float2 t[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) t[i] = lane + 64 * i < parts ? ml[(lane + 64 * i) * total] : make_float2(NEG_INF, 0.0f);
    float top = fmaxf(t[0].x, t[1].x);
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    top = max_over_32(max_over_16(top));
    float f[2], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f[i] = t[i].x == NEG_INF ? 0.0f : exp2_fast(t[i].x - top);
        sum = fmaf(t[i].y, f[i], sum);
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) sum += __shfl_xor(sum, d);
    sum = sum_over_32(sum_over_16(sum));
    float acc[VD];
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = 0.0f;
    for (int base = first; base < parts; base += WAVES * PARTS_AT_ONCE) {
        if (base != first) load(base);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (base + 4 * i >= parts) break;
            const float w = __shfl(base < 64 ? f[0] : f[1], (base + 4 * i + lane / 16) & 63);
            if (w == 0.0f) continue;                             // no part, or one that is empty
#pragma unroll
            for (int j = 0; j < VD / 4; ++j) {
                acc[4 * j] = fmaf(x[i][j].x, w, acc[4 * j]);
                acc[4 * j + 1] = fmaf(x[i][j].y, w, acc[4 * j + 1]);
                acc[4 * j + 2] = fmaf(x[i][j].z, w, acc[4 * j + 2]);
                acc[4 * j + 3] = fmaf(x[i][j].w, w, acc[4 * j + 3]);
            }
        }
    }
    const float inv = inverse_sum(top, sum);
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = sum_over_32(sum_over_16(acc[j])) * inv;
    if constexpr (WAVES > 1) {
        __shared__ float4 others[WAVES - 1][VD / 4][16];
        if (wave > 0 && lane < 16)
#pragma unroll
            for (int j = 0; j < VD; j += 4) others[wave - 1][j / 4][lane] = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
        __syncthreads();
        if (wave > 0 || lane >= 16) return;
#pragma unroll
        for (int w = 0; w < WAVES - 1; ++w)
#pragma unroll
            for (int j = 0; j < VD; j += 4) {
                const float4 y = others[w][j / 4][lane];
                acc[j] += y.x;
                acc[j + 1] += y.y;
                acc[j + 2] += y.z;
                acc[j + 3] += y.w;
            }
    }
    if (lane >= 16) return;
    const Bf16Quantizer quant(a.y_scale ? *a.y_scale : 1.0f);
    OutT* y = static_cast<OutT*>(a.y) + row / a.q_heads * a.ldy + row % a.q_heads * D + ch;
#pragma unroll
    for (int j = 0; j < VD; j += 4) store_4(y + j, acc[j], acc[j + 1], acc[j + 2], acc[j + 3], quant);
}

template <int D, int WAVES> void launch_join(const DecodeArgs& a, int parts, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)a.n_seqs * a.q_heads * WAVES + 3) / 4)), block(256);
    if (a.y_scale) hipLaunchKernelGGL((attention_join_kernel<D, WAVES, uint8_t>), grid, block, 0, st, a, parts);
    else hipLaunchKernelGGL((attention_join_kernel<D, WAVES, uint16_t>), grid, block, 0, st, a, parts);
}

template <int D, bool E4M3, int W, typename OutT>
void launch_stream(const DecodeArgs& a, const DecodePlan& p, int own, int shared, hipStream_t st) {
    hipLaunchKernelGGL((attention_stream_kernel<D, E4M3, W, OutT>), dim3((unsigned)(own + shared)), dim3(64 * W), 0, st, a, p, own);
}

template <int D, bool E4M3>
void launch_typed(const DecodeArgs& a, const DecodePlan& p, hipStream_t st) {
    const int group = a.q_heads / a.c.kv_heads;
    const int row_tiles = (int)(((int64_t)a.n_seqs * group + p.prefix_rows - 1) / p.prefix_rows);
    const int own = a.n_seqs * a.c.kv_heads * ((group + 15) / 16) * p.own_splits, shared = a.c.kv_heads * row_tiles * p.prefix_splits;
    if (p.parts == 0) {
        if (p.own_waves == 8) {
            if (a.y_scale) launch_stream<D, E4M3, 8, uint8_t>(a, p, own, 0, st);
            else launch_stream<D, E4M3, 8, uint16_t>(a, p, own, 0, st);
        } else {
            if (a.y_scale) launch_stream<D, E4M3, WAVES_D, uint8_t>(a, p, own, 0, st);
            else launch_stream<D, E4M3, WAVES_D, uint16_t>(a, p, own, 0, st);
        }
        return;
    }
    if (p.prefix_rows == 16 || shared == 0) {
        launch_stream<D, E4M3, WAVES_D, void>(a, p, own, shared, st);
    } else {
        const int blocks = (shared + 7) / 8 * 8;
        hipLaunchKernelGGL((attention_shared_kernel<D, E4M3>), dim3((unsigned)(blocks + own)), dim3(64 * WAVES_D), 0, st, a, p, own, row_tiles, shared, blocks);
    }
    if (p.parts > PARTS_AT_ONCE && (int64_t)a.n_seqs * a.q_heads <= FEW_ROWS) launch_join<D, 4>(a, p.parts, st);
    else launch_join<D, 1>(a, p.parts, st);
}

}  // namespace

int launch_attention_decode(const DecodeArgs& a, const DecodePlan& p, hipStream_t st) {
    if (a.c.head_dim == 128) {
        if (a.c.e4m3) launch_typed<128, true>(a, p, st);
        else launch_typed<128, false>(a, p, st);
    } else {
        if (a.c.e4m3) launch_typed<64, true>(a, p, st);
        else launch_typed<64, false>(a, p, st);
    }
    return launch_status();
}

}  // namespace w4a8
