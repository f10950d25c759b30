// Attention inside whole prompts: packed sequences, grouped heads, causal or both ways.
//   o_i = sum_j softmax_j(q_i . k_j * scale) v_j,   j in i's sequence, j <= i if causal
// One pass over the keys with a running maximum and sum per row: a workgroup owns 32 rows per wavefront of one query head and walks the
// sequence's keys 64 at a time (attention_tile.hpp).  Keys and values come to LDS by copies that pass no registers, one tile ahead.  Two
// workgroups share a compute unit (64 KB of LDS and 256 registers a lane each), so that one forms weights while the other multiplies.
// One prompt of 8192 tokens, 32 query and 8 key heads of 128 channels, causal: 500 us, 1100 TFLOP/s of the products that the mask leaves; a
// bf16 product of 8192 x 8192 x 8192 reaches 1190 here, so the matrix cores bound it.  Thirteen prompts of 1 .. 1531 tokens: 129 us, 700
// TFLOP/s; there a workgroup's start (2.4 us to its tile, 1.5 to its rows) and end (2 .. 4) stand against 20 us of products, half hidden behind
// the other workgroup's.  Both ways, three sequences of 700 .. 1500, 16 heads of 64 channels: 34.3 us, 590 TFLOP/s: fewer workgroups (496)
// than there are places, the longest sequence's set the time, and half as many products for each exponential.
#include "attention.hpp"
#include "attention_tile.hpp"

namespace w4a8 {
namespace {

constexpr int XCDS_A = 8;
// Sum or maximum over the wavefront.
template <bool MAX> __device__ __forceinline__ int wave_reduce(int x) {
    auto join = [](int a, int b) { return MAX ? max(a, b) : a + b; };
    x = join(x, __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, true));    // lanes 1, 0, 3, 2
    x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, true));    // lanes 2, 3, 0, 1
    x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, true));   // mirrored in eight
    x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x140, 0xF, 0xF, true));   // mirrored in sixteen
    auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = join((int)p[0], (int)p[1]);
    p = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return uniform(join((int)p[0], (int)p[1]));
}
__device__ __forceinline__ int wave_sum(int x) { return wave_reduce<false>(x); }

// Unit t (0 .. tiles - 1) of the packed batch: a sequence and a tile of its rows; false behind the last.  Causal tiles cost what their place
// in the sequence says, so up to 64 sequences (a lane each) give their tiles in falling order of it, all the sequences' together: the
// long ones start first.  More sequences come one after the other, each from its end, and every workgroup looks through them 64 at a time: 64
// prompts of 20 .. 60 tokens, 32 heads, 27.3 us, 65 of them 29.7, 300 150, 1000 of 1 .. 60 724.
template <int BM>
__device__ __forceinline__ bool find_tile(const int32_t* starts, int n_seqs, int64_t T, int t, int& seq_start, int& len, int& tile) {
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < n_seqs; base += 64) {
        const int s = base + lane;
        int b = 0, n = 0;
        if (s < n_seqs) {
            const int64_t lo = starts[s] < 0 ? 0 : starts[s], hi = starts[s + 1] < T ? starts[s + 1] : T;
            b = (int)lo;
            n = hi > lo ? (int)(hi - lo) : 0;
        }
        const int mine = (n + BM - 1) / BM;
        int first;                                               // the lane of the sequence
        if (n_seqs == 1) {
            first = 0;
            tile = __builtin_amdgcn_readlane(mine, 0) - 1 - t;
            if (tile < 0) return false;
        } else if (n_seqs <= 64) {
            if (t >= wave_sum(mine)) return false;
            // the place: the lowest that at most t tiles lie behind
            int low = 0, high = wave_reduce<true>(mine) - 1;
            while (low < high) {
                const int middle = (low + high) >> 1;
                if (wave_sum(max(0, mine - 1 - middle)) <= t) high = middle;
                else low = middle + 1;
            }
            const int rank = t - wave_sum(max(0, mine - 1 - low));   // among the sequences that reach there
            const uint64_t reach = __builtin_amdgcn_ballot_w64(mine > low);
            const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(reach >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)reach, 0));
            first = __builtin_ctzll(__builtin_amdgcn_ballot_w64(mine > low && before == rank));
            tile = low;
        } else {
            int upto = mine;                                     // tiles of this sequence and of those before it
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int other = __shfl_up(upto, d);
                if (lane >= d) upto += other;
            }
            const uint64_t here = __builtin_amdgcn_ballot_w64(t < upto);
            if (!here) {
                t -= __builtin_amdgcn_readlane(upto, 63);
                continue;
            }
            first = __builtin_ctzll(here);
            tile = __builtin_amdgcn_readlane(upto, first) - 1 - t;
        }
        seq_start = __builtin_amdgcn_readlane(b, first);
        len = __builtin_amdgcn_readlane(n, first);
        return true;
    }
    return false;
}

// What becomes of two bf16 values in a walk: themselves; zero instead of what is no number; or one for +infinity (-infinity, either) and NaN and
// zero for all else.
enum Walk { PLAIN = 0, NUMBERS = 1, PLUS = 2, MINUS = 3, ANY = 4 };
struct SeenBy {
    uint32_t first, second, kept, marked;                        // wave-uniform
    __device__ __forceinline__ explicit SeenBy(int walk) {
        asm volatile("" : "+s"(walk));                           // (none of it is kept in registers through walks that do without)
        first = walk == MINUS ? 0xFF80u : 0x7F80u;
        second = walk == PLUS ? 0x7F80u : 0xFF80u;
        kept = walk == NUMBERS ? 0xFFFFu : 0;
        marked = walk == NUMBERS ? 0 : 0x3F80u;
    }
    __device__ __forceinline__ uint32_t one(uint32_t x) const {
        const bool hit = (x & 0x7FFFu) > 0x7F80u | x == first | x == second;
        return hit ? marked : x & kept;
    }
    __device__ __forceinline__ uint32_t two(uint32_t w) const { return one(w & 0xFFFFu) | one(w >> 16) << 16; }
};

// SHARE wavefronts share 32 rows and take a part of every tile's keys each.  A tile of 64 keys takes four wavefronts of 32 rows of 128 channels 32
// matrix instructions each and about 130 vector instructions, 1.85 us for the two workgroups of a compute unit together.  Copies are asked
// for a whole tile ahead and waited for at its start; masks are touched only in tiles that hide something.  The compiler is told how many wavefronts a
// vector unit gets at most: with 64 channels it hopes for a fourth, and then saves registers by waiting for each operand by itself (2000 tokens,
// 8 heads: 20.6 us, so 21.4).
template <int D, int SHARE, bool CAUSAL, typename OutT>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, D == 64 ? 3 : 2))) attention_prompt_kernel(PromptArgs a, int by_head) {
    constexpr int WAVES = 4, BN = TILE_KEYS, KEYS = BN / SHARE;
    using Block = RowBlock<D, KEYS>;
    constexpr int BM = 32 * WAVES / SHARE, ROW = Block::ROW, PIECES = Block::PIECES, TILE = Block::TILE, RPC = Block::RPC;
    constexpr int DT = Block::DT, KT = Block::KT;
    constexpr int COPIES = TILE / 1024 / WAVES;                  // of 64 lanes x 16 bytes, per wavefront for each of K and V
    // K 0, V 0, K 1, V 1; first Q, from K 1 on; at last O, from K 0 on, and behind it what is to be joined
    __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * TILE];
    static_assert(BM * ROW <= 2 * TILE && (SHARE == 1 || BM * ROW + BM * (2 * ROW + 8) <= 4 * TILE), "what goes there");
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int band = wave / SHARE, part = wave % SHARE;          // this wavefront's 32 rows and keys of a tile
    const int group = a.q_heads / a.kv_heads;

    // by_head: every XCD keeps to its own key heads, whose keys and values then stay in its L2; a tile's query heads that share a
    // key head run side by side.
    int t, head;
    if (by_head) {
        const int x = blockIdx.x % XCDS_A, i = blockIdx.x / XCDS_A;
        const int heads_x = a.kv_heads / XCDS_A * group;
        t = i / heads_x;
        const int h = i - t * heads_x;
        head = (h / group * XCDS_A + x) * group + h % group;
    } else {
        t = blockIdx.x / a.q_heads;
        head = blockIdx.x - t * a.q_heads;
    }
    const int kv_head = head / group;
    int seq_start, len, tile;
    if (!find_tile<BM>(a.starts, a.n_seqs, a.T, t, seq_start, len, tile)) return;
    const int q0 = tile * BM, row = q0 + 32 * band + col;        // this lane's row of the sequence
    const int key_end = CAUSAL ? min(len, q0 + BM) : len;
    const int n_tiles = (key_end + BN - 1) / BN;

    const uint8_t* kbase = reinterpret_cast<const uint8_t*>(a.k + (int64_t)seq_start * a.ldk + (int64_t)kv_head * D);
    const uint8_t* vbase = reinterpret_cast<const uint8_t*>(a.v + (int64_t)seq_start * a.ldv + (int64_t)kv_head * D);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    uint32_t k_from[COPIES], v_from[COPIES];                     // where this lane's 16 bytes of its copies come from, within a tile
#pragma unroll
    for (int q = 0; q < COPIES; ++q) {
        const int r = (wave * COPIES + q) * RPC + lane / PIECES;
        const uint32_t piece = (uint32_t)(((lane % PIECES) ^ swizzle<D>(r)) * 16);
        k_from[q] = (uint32_t)r * (uint32_t)(a.ldk * 2) + piece;
        v_from[q] = (uint32_t)r * (uint32_t)(a.ldv * 2) + piece;
    }
    int walk = PLAIN;
    auto copy_tile = [&](int kt, int buffer) {
        const uint8_t* kt_base = kbase + (int64_t)kt * BN * a.ldk * 2;
        const uint8_t* vt_base = vbase + (int64_t)kt * BN * a.ldv * 2;
        const uint32_t to = lds_base + 2 * buffer * TILE + wave * COPIES * 1024;
        const int left = len - kt * BN;
        if (left >= BN && walk == PLAIN) {
#pragma unroll
            for (int q = 0; q < COPIES; ++q) {
                lds_dma_16(kt_base, k_from[q], to + q * 1024);
                lds_dma_16(vt_base, v_from[q], to + TILE + q * 1024);
            }
            return;
        }
#pragma unroll 1
        for (int q = 0; q < COPIES; ++q) {
            const int r = (wave * COPIES + q) * RPC + lane / PIECES, from = min(r, left - 1);   // behind the sequence's last row: that one again
            const uint32_t piece = (uint32_t)(((lane % PIECES) ^ swizzle<D>(r)) * 16);
            const uint32_t v_at = (uint32_t)from * (uint32_t)(a.ldv * 2) + piece, here = (uint32_t)uniform((int)(to + q * 1024));
            lds_dma_16(kt_base, (uint32_t)from * (uint32_t)(a.ldk * 2) + piece, here);
            if (walk == PLAIN) {
                lds_dma_16(vt_base, v_at, here + TILE);
            } else {
                u32x4 v = *reinterpret_cast<const u32x4*>(vt_base + v_at);
                const SeenBy seen(walk);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = seen.two(v[i]);
                lds_write(here + TILE + lane * 16, v);
            }
        }
    };
    Block rows(lds_base, lane, KEYS * part);
    {
        const uint8_t* from = reinterpret_cast<const uint8_t*>(a.q + (int64_t)(seq_start + q0) * a.ldq + (int64_t)head * D);
#pragma unroll
        for (int q = 0; q < 32 / RPC; ++q) {
            const int r = 32 * band + q * RPC + lane / PIECES;
            lds_dma_16(from, (uint32_t)min(r, len - 1 - q0) * (uint32_t)(a.ldq * 2) + (uint32_t)(((lane % PIECES) ^ swizzle<D>(r)) * 16),
                       lds_base + 2 * TILE + (32 * band + q * RPC) * ROW);
        }
        copy_tile(0, 0);                                         // on its way together with them
        lds_dma_wait_all();                                      // a wavefront copies its own rows (those that share them, the same bytes)
        rows.read_q(2 * TILE + (32 * band - KEYS * part) * ROW);
    }

    // A weight of zero takes a key out of the sums, unless its value is no number.  So if an output is none, the rows are walked again with zeros
    // for such values, and then to mark the outputs that see one: all weights are one there, and every row counts the ones it sees.  PLUS and MINUS leave
    // out scores of -infinity, whose weights are zero by definition and not for want of bits; such a weight makes NaN of an infinity, so ANY
    // counts under these scores alone.  Scores that are NaN or +infinity are NaN there: such a row's outputs are NaN already, its counts too, and
    // no value changes that.
    uint64_t marked = 0;                                         // outputs of this lane that see +infinity or NaN
    for (;; ++walk) {
    rows.clear();
    if (walk != PLAIN) copy_tile(0, 0);
    auto step = [&](int kt, auto buffer_c) {
        constexpr int buffer = decltype(buffer_c)::value;
        lds_dma_wait_all();
        __syncthreads();
        if (kt + 1 < n_tiles) copy_tile(kt + 1, buffer ^ 1);
        const int key0 = kt * BN + KEYS * part;
        if (CAUSAL && key0 > q0 + 32 * band + 31) return;        // (wave-uniform) no row of this wavefront sees its keys of the tile
        v16f s[KT];
        rows.template scores<buffer>(s);
        const bool masked = key0 + KEYS > len || (CAUSAL && key0 + KEYS - 1 > q0 + 32 * band);
        const int seen = CAUSAL ? min(len, row + 1) : len;       // keys below this one
        // a loop of at most one pass: as a branch the compiler turns it into 32 comparisons and selects in every tile
        int changes = uniform(masked || walk >= PLUS);
        while (changes) {
            int edge = seen - key0 - 4 * half, now = walk;
            asm volatile("" : "+v"(edge), "+s"(now));
            if (now >= PLUS) {
                const float at_inf = now == ANY ? 0.0f : NEG_INF, else_at = now == ANY ? NEG_INF : 0.0f;
#pragma unroll
                for (int k = 0; k < KT; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[k][r] = s[k][r] == NEG_INF ? at_inf : fmaf(s[k][r], 0.0f, else_at);
            }
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * k + (r & 3) + 8 * (r >> 2) >= edge) s[k][r] = NEG_INF;
            asm volatile("s_mov_b32 %0, 0" : "=s"(changes));
        }
        uint32_t p[KT][8];
        rows.weights(s, a.scale_log2, p);
        rows.template add_values<buffer>(p);
    };
    for (int kt = 0; kt < n_tiles; kt += 2) {
        step(kt, std::integral_constant<int, 0>{});
        if (kt + 1 < n_tiles) step(kt + 1, std::integral_constant<int, 1>{});
    }
    float none = 0.0f;                                           // NaN if any output is no number
    if (walk == PLAIN) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) none = fmaf(rows.o[d][r], 0.0f, none);
    }
    if (__builtin_expect(uniform(__syncthreads_or(none != 0.0f)), 0)) continue;
    // O^T to rows of bf16 through this wavefront's part of LDS (all are past the barrier above), so that whole rows go to memory
    float total = sum_over_32(rows.l);
    if (SHARE == 2) {                                            // the two halves of the keys joined, by the wavefront of the first
        const uint32_t theirs = lds_base + BM * ROW + band * 32 * (2 * ROW + 8) + lane * 16, ml = theirs + 32 * 2 * ROW - lane * 8;
        if (part == 1) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    lds_write(theirs + (d * 4 + r / 4) * 1024, v4f{rows.o[d][r], rows.o[d][r + 1], rows.o[d][r + 2], rows.o[d][r + 3]});
            if (half == 0) lds_write(ml, v2f{rows.m, total});
        }
        __syncthreads();
        if (part == 0) {
            const v2f other = lds_read<v2f>(half ? ml - 256 : ml);
            const float top = fmaxf(rows.m, other[0]);
            const float mine = rows.m == NEG_INF ? 0.0f : exp2_fast(rows.m - top), more = other[0] == NEG_INF ? 0.0f : exp2_fast(other[0] - top);
            total = fmaf(total, mine, other[1] * more);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const v4f x = lds_read<v4f>(theirs + (d * 4 + r / 4) * 1024);
#pragma unroll
                    for (int i = 0; i < 4; ++i) rows.o[d][r + i] = fmaf(rows.o[d][r + i], mine, x[i] * more);
                }
        }
    }
    // (every row sees itself: a sum of zero is one of scores of -infinity alone, NaN like 0 / 0.  In a mark's walk a row may count nothing)
    const float inv = walk >= PLUS ? 1.0f : 1.0f / total;
    const uint32_t slab = lds_base + band * 32 * ROW;
    if (part == 0) {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            lds_write(slab + col * ROW + (uint32_t)(((4 * d + (r >> 2)) ^ swizzle<D>(col)) << 4) + 8 * half,
                      u32x2{pack_bf16(rows.o[d][r] * inv, rows.o[d][r + 1] * inv), pack_bf16(rows.o[d][r + 2] * inv, rows.o[d][r + 3] * inv)});
    wave_lds_fence();
    constexpr bool BYTES = sizeof(OutT) == 1;
    constexpr int LANES = BYTES ? PIECES / 2 : PIECES;           // per row, 16 bytes of the output each
    constexpr int EACH = 16 / (int)sizeof(OutT);
    const int piece = lane % LANES;
    OutT* y = static_cast<OutT*>(a.y) + (int64_t)(seq_start + q0 + 32 * band) * a.ldy + (int64_t)head * D + piece * EACH;
    const Bf16Quantizer quant(BYTES ? *a.y_scale : 1.0f);
#pragma unroll
    for (int n = 0; n < LANES / 2; ++n) {
        const int r = n * (64 / LANES) + lane / LANES;
        const uint32_t from = slab + r * ROW;
        u32x4 out;
        if (BYTES) {
            const u32x4 lo = lds_read<u32x4>(from + (uint32_t)(((2 * piece) ^ swizzle<D>(r)) << 4));
            const u32x4 hi = lds_read<u32x4>(from + (uint32_t)(((2 * piece + 1) ^ swizzle<D>(r)) << 4));
            out = u32x4{quant_bf16(lo[0], lo[1], quant), quant_bf16(lo[2], lo[3], quant), quant_bf16(hi[0], hi[1], quant), quant_bf16(hi[2], hi[3], quant)};
        } else {
            out = lds_read<u32x4>(from + (uint32_t)((piece ^ swizzle<D>(r)) << 4));
        }
        if (q0 + 32 * band + r < len && walk <= NUMBERS) stream_out(y + (int64_t)r * a.ldy, out);
    }
    if (walk >= PLUS) {                                          // the outputs that see an infinity or NaN become it
        for (int i = 0; i < 16 * D / 32; ++i) {
            const int r = i / EACH * (64 / LANES) + lane / LANES, c = piece * EACH + i % EACH;
            const uint16_t count = lds_read<uint16_t>(slab + r * ROW + (uint32_t)(((c / 8) ^ swizzle<D>(r)) << 4) + c % 8 * 2);
            if (count == 0 || (count & 0x7FFFu) > 0x7F80u || q0 + 32 * band + r >= len) continue;
            const float becomes = walk == PLUS ? -NEG_INF : walk == ANY || (marked >> i & 1) ? __builtin_nanf("") : NEG_INF;
            if (walk == PLUS) marked |= (uint64_t)1 << i;
            y[(int64_t)r * a.ldy + i % EACH] = BYTES ? (OutT)quantize_one(becomes, quant.s) : (OutT)(__float_as_uint(becomes) >> 16);
        }
    }
    }
    if (walk == PLAIN || walk == ANY) break;
    __syncthreads();                                             // all have read what the next walk's tiles replace
    }
}

template <int D, int SHARE, bool CAUSAL>
void launch_tile(const PromptArgs& a, hipStream_t st) {
    constexpr int BM = 128 / SHARE;
    const int64_t tiles = a.n_seqs == 1 ? (a.T + BM - 1) / BM : a.T / BM + a.n_seqs;   // at most
    const int by_head = a.kv_heads % XCDS_A == 0;
    const dim3 grid((unsigned)(tiles * a.q_heads)), block(256);
    if (a.y_scale) hipLaunchKernelGGL((attention_prompt_kernel<D, SHARE, CAUSAL, uint8_t>), grid, block, 0, st, a, by_head);
    else hipLaunchKernelGGL((attention_prompt_kernel<D, SHARE, CAUSAL, uint16_t>), grid, block, 0, st, a, by_head);
}

// Workgroups of 128 rows read least; but a wavefront's way through a tile is one chain of instructions that wait for each other, and with
// hardly more than one workgroup per compute unit nothing else fills those waits.  Then 64 rows a workgroup, two wavefronts on each 32: one
// prompt of 512 tokens, 32 heads, 14.0 -> 12.4 us (128 workgroups of 128 rows), of 1100 26.5 -> 23.1 (288), of 1536 34.2 -> 31.2 (384), of 2000 on 8
// heads of 64 channels 27.7 -> 20.8 (128).  Of 1700 (448) it would gain still, 38.7 -> 37.3, but three sequences of 700 .. 1500 on 16 heads of 64
// channels, both ways (432), lose, 34.4 -> 40.5, and 40 of 1 .. 300 (1505) 43.7 -> 56.6.
constexpr int FEW = 384;
template <int D, bool CAUSAL>
void launch_rows(const PromptArgs& a, hipStream_t st) {
    if ((a.T + 127) / 128 * a.q_heads <= FEW) launch_tile<D, 2, CAUSAL>(a, st);
    else launch_tile<D, 1, CAUSAL>(a, st);
}

}  // namespace

int launch_attention_prompt(const PromptArgs& a, hipStream_t st) {
    if (a.head_dim == 128) {
        if (a.causal) launch_rows<128, true>(a, st);
        else launch_rows<128, false>(a, st);
    } else {
        if (a.causal) launch_rows<64, true>(a, st);
        else launch_rows<64, false>(a, st);
    }
    return launch_status();
}

}  // namespace w4a8
