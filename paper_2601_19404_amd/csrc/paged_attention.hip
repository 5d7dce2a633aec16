// Attention over a paged cache outside a batch, with a sliding window and sinks, and the attention weight that every cached
// token receives.
//
// Row i of a sequence's chunk sits at slot t = slot0 + i and sees the slots j <= t of which j < sinks or j > t - window.
//   out = sum_j p_j v_j,  p_j = exp(scale q.k_j - lse),  lse = ln sum_j exp(scale q.k_j)
// A row that sees nothing leaves zeros and an lse of -infinity.
//
//  * attn_tile_kernel: chunks, head_dim 32, 64 or 128, bf16 or fp32.  Four waves of 16 or 32 query columns (row x head of a KV
//    head) each; keys and values go through LDS in tiles of 64 (32) tokens, straight from the pages, double buffered.
//  * attn_few_kernel: up to 16 query columns per KV head (single tokens).  Every wave streams tokens of its own from the pages
//    into the operand registers of the matrix instructions; the four waves' results are joined in LDS.
//  * attn_join_kernel: joins the pieces of tokens that were split over workgroups.
//  * score_tile_kernel, score_few_kernel: the weights summed over the query columns, keys in registers.
//  * attn_rows_kernel, score_rows_kernel: any head_dim, one wave per (row, head), one workgroup per 32 tokens.
//
// Both element types go through the same code: a fragment is 16 bytes of a row per lane, which one 16x16x32 bf16 or four
// 16x16x4 fp32 instructions multiply.  Scores are computed transposed, S^T = K Q^T, so that a lane holds scores of one query
// column and its maximum and sum need two lane swaps; and the rows of K are dealt to the instruction such that the weights a
// lane ends with are eight (four) consecutive tokens, which is how a page keeps the values: they are read as they lie.
#include <type_traits>

#include "kernels.hpp"

namespace rpo {

namespace {

// Whether a row at slot t sees slot j.
__device__ inline bool sees(int t, int j, int window, int sinks) {
    return j <= t && (window == 0 || j < sinks || t - j < window);
}

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;

template <typename T>
struct Mat;
template <>
struct Mat<bf16> {
    static constexpr int kGroup = 32;  // tokens of one product of weights and values
    static constexpr int kLaneTok = 8;  // of which a lane holds so many, side by side
    // token of row c (0..15) of 16-token block mb: blocks 2 k and 2 k + 1 share 32 tokens, such that lane group g's rows
    // 4 g .. 4 g + 3 of both are the tokens 8 g .. 8 g + 7
    static __host__ __device__ constexpr int token(int mb, int c) { return 32 * (mb >> 1) + 8 * (c >> 2) + 4 * (mb & 1) + (c & 3); }
    static __device__ constexpr int row_c(int r) { return 4 * ((r >> 3) & 3) + (r & 3); }  // the c of a token
    static __device__ inline f32x4_t mma(u32x4_t a, u32x4_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    }
    // weights of 32 tokens as an operand: rounded to bf16 once
    static __device__ inline u32x4_t weights(const f32x4_t* s) {
        bf16x8_t p;
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = (__bf16)s[0][i], p[4 + i] = (__bf16)s[1][i];
        return __builtin_bit_cast(u32x4_t, p);
    }
    static __device__ inline u32x4_t times(u32x4_t p, float f) {
        bf16x8_t x = __builtin_bit_cast(bf16x8_t, p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (__bf16)((float)x[i] * f);
        return __builtin_bit_cast(u32x4_t, x);
    }
    // 16-byte unit of a values tile [octets][channels][8] that holds lane group g's tokens of group kk
    static __device__ inline int unit(int kk, int g, int dh, int ch) { return (4 * kk + g) * dh + ch; }
    // dword d of an operand that holds 2 where bit i of bits is set and 0 elsewhere
    static __device__ inline uint32_t twos(uint32_t bits, int d) {
        return (bits >> (2 * d) & 1) * 0x4000u | (bits >> (2 * d + 1) & 1) * 0x40000000u;
    }
    // values without those that are not finite; up: the largest number where +infinity or NaN was, down: the smallest where
    // -infinity or NaN was
    static __device__ inline uint32_t finite(uint32_t x, uint32_t& up, uint32_t& down) {
        constexpr uint32_t k1 = 0x00010001u;
        const uint32_t odd = ((x & 0x7f807f80u) + 0x00800080u) >> 15 & k1, nan = ((x & 0x007f007fu) + 0x007f007fu) >> 7, neg = x >> 15;
        up = (odd & (nan | ~neg)) * 0x7f7fu;
        down = (odd & (nan | neg)) * 0xff7fu;
        return x & ~(odd * 0xffffu);
    }
};
template <>
struct Mat<float> {
    static constexpr int kGroup = 16;
    static constexpr int kLaneTok = 4;
    static __host__ __device__ constexpr int token(int mb, int c) { return 16 * mb + c; }
    static __device__ constexpr int row_c(int r) { return r & 15; }
    static __device__ inline f32x4_t mma(u32x4_t a, u32x4_t b, f32x4_t c) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
        return c;
    }
    static __device__ inline u32x4_t weights(const f32x4_t* s) { return __builtin_bit_cast(u32x4_t, s[0]); }
    static __device__ inline u32x4_t times(u32x4_t p, float f) { return __builtin_bit_cast(u32x4_t, __builtin_bit_cast(f32x4_t, p) * f); }
    static __device__ inline int unit(int kk, int g, int dh, int ch) { return ((2 * kk + (g >> 1)) * dh + ch) * 2 + (g & 1); }
    static __device__ inline uint32_t twos(uint32_t bits, int d) { return (bits >> d & 1) * 0x40000000u; }
    static __device__ inline uint32_t finite(uint32_t x, uint32_t& up, uint32_t& down) {
        const uint32_t odd = ((x & 0x7f800000u) + 0x00800000u) >> 31, nan = ((x & 0x007fffffu) + 0x007fffffu) >> 23, neg = x >> 31;
        up = (odd & (nan | ~neg)) * 0x7f7fffffu;
        down = (odd & (nan | neg)) * 0xff7fffffu;
        return x & (odd - 1);
    }
};

// 16-byte pieces of a row, and where piece p of a row lies in LDS: permuted so that the 16 rows that a fragment reads at the
// same piece fall on different banks (the LDS serves lanes 0-3, 12-15, 20-23 and 24-27 together)
template <typename T, int DH>
struct Row {
    static constexpr int kBytes = DH * (int)sizeof(T), kPieces = kBytes / 16, kFrags = kPieces / 4;
    static constexpr int kElems = 16 / (int)sizeof(T);  // elements of a piece
    static __device__ inline int turn(int c) { return kPieces >= 16 ? c : kPieces == 8 ? c >> 1 : (4 - (c >> 2)) & 3; }
};

// in every lane the maximum (sum) over the four lanes that share l % 16
template <typename F>
__device__ inline float over_lane_groups(float v, F f) {
    typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
    u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max_over_lane_groups(float v) {
    return over_lane_groups(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float sum_over_lane_groups(float v) {
    return over_lane_groups(v, [](float a, float b) { return a + b; });
}
__device__ inline int wave_min_int(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ inline int wave_max_int(int v) { return -wave_min_int(-v); }
// The same address in every lane, in scalar registers, for a load written as assembly: scalar registers that a vector
// instruction has written may be read by a memory instruction five wait states later, which the compiler sees to only where
// it knows the instruction.
template <typename T>
__device__ inline const T* uniform(const T* p) {
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    uint64_t u = (uint64_t)hi << 32 | lo;
    asm volatile("s_nop 4" : "+s"(u));
    return (const T*)(uintptr_t)u;
}

// The slots that a set of rows sees any of, in steps of `step` tokens: [0, sink) and then [lo, hi), cut into pieces.
struct Span {
    int hi, lo, sinks;   // slots: seen if < hi and (< sinks or >= lo)
    int sink_steps, lo_step, n;
    __device__ Span(int t_first, int t_last, int window, int sinks_, int step) {
        hi = max(t_last + 1, 0);
        lo = window ? max(0, t_first - window + 1) : 0;
        sinks = window ? min(sinks_, hi) : 0;
        lo_step = lo / step;
        sink_steps = min((sinks + step - 1) / step, lo_step);
        n = sink_steps + max(0, (hi + step - 1) / step - lo_step);
    }
    __device__ int step_at(int i) const { return i < sink_steps ? i : lo_step + i - sink_steps; }
    __device__ bool any(int j) const { return j < hi && (j < sinks || j >= lo); }
    __device__ bool any_of(int j, int n) const { return j < hi && (j < sinks || j + n > lo); }  // any of n slots
};

// the lowest n bits (n below 0: none, above 32: all)
__device__ inline uint32_t low_bits(int n) { return (uint32_t)((1ull << min(max(n, 0), 32)) - 1); }

// A weight of 0 keeps a token from a row, but 0 times NaN or infinity is NaN: values that are not finite reach every column that
// a wave computes with one that sees them.  A wave asks for that in the end, of its sums alone (a question in the loop, a product
// of the values with zeros in every step that has a mask, cost 3 to 5 %): whether a column's sums are not finite though its
// weights' sum is.
template <int DH>
__device__ inline bool only_values_not_finite(const f32x4_t (&ot)[DH / 16], float sum) {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) x = __builtin_fmaf(ot[i][e], 0.f, x);
    return x != x && sum - sum == 0.f;
}
// Then it multiplies once more, the weights by what their sums are relative to, and without the values that are not finite:
// those come in as products of the largest numbers with 2 for the columns that see them, which overflow to an infinity of
// either sign; both make a NaN.  Straight from the pages, a step of M::kGroup tokens at a time, with no loads ahead: 4 x 4352
// rows of 7B heads with NaN among the values 2.5 ms.  Without any, its registers cost the loops about 1 %: 576 -> 584 us.
template <typename T, int DH, int NC, typename F>
__device__ __forceinline__ void multiply_again(const PagedKv& kv, int s, int kh, const Span& span, int n_steps, F first_token,
                                               const u32x4_t (&bq)[NC][Row<T, DH>::kFrags], const int (&limit)[NC],
                                               const int (&from)[NC], float scale_log2, const float (&minus_ref)[NC],
                                               f32x4_t (&ot)[NC][DH / 16]) {
    using R = Row<T, DH>;
    using M = Mat<T>;
    constexpr int KS = M::kGroup, MB = KS / 16;
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4, mask = (1 << kv.shift) - 1;
    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    const u32x4_t none = {0, 0, 0, 0};
    const T* const pool = (const T*)kv.pool;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) ot[c][i] = zero4;
#pragma unroll 1
    for (int x = 0; x < n_steps; ++x) {
        const int tok = first_token(x);
        int page[MB];
        uint32_t there = 0;  // bit r: token r's page is
#pragma unroll
        for (int u = 0; u < MB; ++u) {
            page[u] = tok + 16 * u < span.hi ? kv.page(s, tok + 16 * u) : -1;
            there |= page[u] >= 0 ? 0xffffu << (16 * u) : 0u;
        }
        // what is not there is read from the first page, and cleared
        f32x4_t sc[NC][MB];
        {
            const int r = M::token(0, c16), p = MB > 1 && r >> 4 ? page[MB - 1] : page[0];
            const T* k = pool + kv.k_at(max(p, 0), kh) + (int64_t)((tok + r) & mask) * DH + g * R::kElems;
            const uint32_t keep = ~(uint32_t)(p >> 31);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int j = 0; j < R::kFrags; ++j) {
                    const u32x4_t a = *(const u32x4_t*)(k + (M::token(mb, 0) - M::token(0, 0)) * DH + 4 * j * R::kElems) & keep;
#pragma unroll
                    for (int c = 0; c < NC; ++c) sc[c][mb] = M::mma(a, bq[c][j], j == 0 ? zero4 : sc[c][mb]);
                }
        }
        u32x4_t w[NC], view[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint32_t seen = low_bits(limit[c] - tok) & (low_bits(span.sinks - tok) | ~low_bits(from[c] - tok)) & there;
            const uint32_t mine = seen >> (M::kLaneTok * g);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[c][mb][i], scale_log2, minus_ref[c]));
                    sc[c][mb][i] = __uint_as_float(__float_as_uint(x) & (uint32_t)__builtin_amdgcn_sbfe((int)mine, M::token(mb, i), 1));
                }
            w[c] = M::weights(sc[c]);
#pragma unroll
            for (int d = 0; d < 4; ++d) view[c][d] = M::twos(mine, d);
        }
        const int slot = tok + M::kLaneTok * g, p = MB > 1 && g >> 1 ? page[MB - 1] : page[0];
        const T* v = pool + kv.v_at(max(p, 0), kh) + ((int64_t)((slot & mask) >> 3) * DH + c16) * 8 + (slot & 7);
        const uint32_t keep = ~(uint32_t)(p >> 31);
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) {
            u32x4_t a = *(const u32x4_t*)(v + 16 * 8 * i) & keep, ups, downs;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                uint32_t up, down;
                a[d] = M::finite(a[d], up, down);
                ups[d] = up, downs[d] = down;
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                // (each in a sum of its own: a product added to an infinity does not overflow before the sum does)
                const f32x4_t high = M::mma(ups, view[c], zero4), low = M::mma(downs, view[c], zero4);
                ot[c][i] = M::mma(a, w[c], ot[c][i]) + high + low;
            }
        }
    }
}

// ---------------------------------------------------------------------------
// chunks.  A wave multiplies every fragment that it reads from LDS with two column tiles (32 columns), which takes the LDS to
// half of the matrix units' time; 64 columns would need the registers of the second workgroup of a CU, whose waves fill each
// other's gaps.  Direct loads leave the registers to the pipeline below; K is permuted on the way, V needs no permutation.
// Bound by matrix and vector units about equally (products 1024 cycles, exponentials and their fma, sum and conversion 800
// for a wave and a tile) and by what their taking turns leaves open: prefill of 4 x 4352 rows of 7B heads 555 to 580 us (by box
// and clock) = 0.95 PFLOP/s, where a large library product reaches 1.12.  Steps, on the box of the time: one after the other in a
// tile 667 us; pipelined, fragments read just before their products 613; read ahead 604; the maximum checked by lane and moved
// past 2^8 only 570; masks as bits, values cleared in registers 545; the two sums below 563.
// Registers: with 128 channels and 128 columns bf16 puts 24 to 42 of them away before the loop and fetches them behind it; fp32
// fetches some of 44 to 46 in the loop, and so does bf16 with 32 channels on pages of 16 tokens (80 bytes a lane).
// Weights are rounded to bf16 before they meet the values, which takes the matrix units' full rate; the output is divided by
// the sum of the weights as they were rounded, so that it is a mean of the values with weights a little off and a row that sees
// equal values (or one) returns them.  Divided by the unrounded sum it is off by the largest weight's rounding too: 1.4e-3
// instead of 0 for rows that see one token, 2.3e-3 instead of 2.15e-3 over 512 to 4352 tokens, the result's own rounding 1.7e-3
// among it.  That sum comes from a product with ones (as a sum of converted weights 588 us), the unrounded one, which the
// log-sum-exp needs, is added up only where it is asked for (563 us, without 543).
// ---------------------------------------------------------------------------
struct TileGeom {
    int combos;   // n_seqs * Hkv
    int n_split;  // pieces that the tokens are cut into
    float* part;  // n_split > 1: [row, head, piece][DH] sums, then [row, head, piece] PieceSums
};
// Of a piece's weights: what they are relative to (log2 domain; -infinity if nothing is seen), the sum that divides the output, the
// sum that the log-sum-exp is made of.
struct alignas(16) PieceSums {
    float top, sum, lse_sum, unused;
};
template <int DH>
__device__ inline PieceSums* piece_sums(const PagedAttnArgs& a, const TileGeom& geo) {
    return (PieceSums*)(geo.part + (int64_t)a.n_rows * a.Hq * geo.n_split * DH);
}

template <typename T, int DH, int NC, bool WIDE, bool LSE>
__global__ __launch_bounds__(256, 2) void attn_tile_kernel(PagedAttnArgs a, TileGeom geo) {
    using R = Row<T, DH>;
    using M = Mat<T>;
    constexpr int KS = M::kGroup, KT = 2 * KS;         // tokens of a half tile (one step) and of a tile
    constexpr int MB = KS / 16;                        // 16-token blocks of a step
    constexpr int U = WIDE ? 1 : KT / 16;              // units of a tile that lie in one page: the tile, or 16 tokens
    constexpr int kTileBytes = KT * R::kBytes, kChunks = kTileBytes / 1024 / 4;  // 1 KiB loads per wave and tile
    constexpr int kTok = 1024 / R::kBytes;             // tokens (of keys or of values) of a 1 KiB load
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * kTileBytes];  // keys, keys, values, values
    const PagedKv& kv = a.kv;
    const int combo = blockIdx.x % geo.combos, rest = blockIdx.x / geo.combos;
    const int split = rest % geo.n_split, kh = combo % kv.Hkv, s = combo / kv.Hkv;
    const ChunkRows cr = chunk_rows(kv, a.cu, s, a.n_rows, a.max_new);
    const int hpk = a.Hq / kv.Hkv;
    constexpr int kCols = 64 * NC;
    const int n_cols = cr.n * hpk, n_qt = (n_cols + kCols - 1) / kCols;
    const int qt = n_qt - 1 - rest / geo.n_split;      // the longest contexts first
    if (qt < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;

    // this lane's query columns
    int limit[NC], from[NC];     // sees slots < limit that are >= from or sinks
    u32x4_t bq[NC][R::kFrags];
    int lim_min = 0x7fffffff, from_max = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = qt * kCols + (wave * NC + c) * 16 + c16;
        const bool real = col < n_cols;
        const int i = real ? col / hpk : 0, hq = kh * hpk + (real ? col % hpk : 0);
        const int t = cr.slot0 + i;
        limit[c] = real ? t + 1 : 0x7fffffff;
        from[c] = real && a.window ? max(0, t - a.window + 1) : 0;
        if (real) lim_min = min(lim_min, t + 1), from_max = max(from_max, from[c]);
        const T* q = (const T*)a.q + (int64_t)(cr.row0 + i) * a.q_stride + (int64_t)hq * DH;
#pragma unroll
        for (int j = 0; j < R::kFrags; ++j) bq[c][j] = real ? *(const u32x4_t*)(q + (4 * j + g) * R::kElems) : u32x4_t{0, 0, 0, 0};
    }
    lim_min = wave_min_int(lim_min), from_max = wave_max_int(from_max);

    const int first_row = qt * kCols / hpk, last_row = (min(n_cols, (qt + 1) * kCols) - 1) / hpk;
    const Span span(cr.slot0 + first_row, cr.slot0 + last_row, a.window, a.sinks, KT);
    const int per = (span.n + geo.n_split - 1) / geo.n_split;
    const int it0 = min(span.n, split * per), n = min(span.n - it0, per);  // this workgroup's tiles: it0 .. it0 + n - 1

    f32x4_t ot[NC][DH / 16];
    // weights are 2^(scale_log2 score + minus_ref), minus_ref a whole number; it moves when a score passes bound (-infinity
    // before the first one)
    float minus_ref[NC], bound[NC], l[NC];  // l: a lane's share of the sum of the weights before they are rounded
    f32x4_t lr[NC];                         // every element: the sum of a column's weights as they are multiplied (bf16)
    constexpr bool kRounds = sizeof(T) == 2;
    static_assert(LSE || kRounds, "without roundings there is one sum");
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) ot[c][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        minus_ref[c] = 0.f;
        bound[c] = -INFINITY;
        l[c] = 0.f;
        lr[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const int64_t to_values = (int64_t)kv.Hkv * kv.block() * (int64_t)sizeof(T);
    // byte offset of a lane's piece of keys from the unit's first token (WIDE), or from the first token of the 1 KiB load
    int key_off[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int at = (i * 4 + wave) * 1024 + lane * 16, r = at / R::kBytes, slot = at % R::kBytes / 16;
        key_off[i] = (WIDE ? r : r % kTok) * R::kBytes + ((slot ^ (R::turn(M::row_c(r)) & (R::kPieces - 1))) << 4);
    }
    // page of every unit of a tile, -1: not there.  Left in a vector register for a tile's time before it is looked at.
    const int32_t* const table = kv.table + (int64_t)s * kv.table_stride;
    auto pages = [&](int x, int (&page)[U]) {
        const int slot = span.step_at(it0 + x) * KT;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = x < n && slot + 16 * u < span.hi ? table[(slot + 16 * u) >> kv.shift] : -1;
            page[u] = (unsigned)p < (unsigned)kv.n_pages ? p : -1;
        }
    };
    // addresses of the units' first keys, 0: not there
    const char* const pool = (const char*)kv.pool + kh * kv.block() * (int64_t)sizeof(T);
    const int64_t page_bytes = kv.page_stride * (int64_t)sizeof(T);
    auto bases = [&](int x, const int (&raw)[U], const char* (&base)[U]) {
        const int slot = span.step_at(it0 + x) * KT;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = __builtin_amdgcn_readfirstlane(raw[u]);
            base[u] = p < 0 ? nullptr : pool + p * page_bytes + (int64_t)((slot + 16 * u) & ((1 << kv.shift) - 1)) * R::kBytes;
        }
    };
    auto load_tile = [&](const char* const (&base)[U], bool values, uint32_t to) {
        to += wave * 1024;
        if constexpr (WIDE) {
            if (!base[0]) return;  // uniform; what LDS holds there is masked, its values are cleared
            const char* p = uniform(base[0] + (values ? to_values : 0));
#pragma unroll
            for (int i = 0; i < kChunks; ++i) dma_load16_at<false>(p, values ? (i * 4 + wave) * 1024 + lane * 16 : key_off[i], to, i * 4096);
        } else {
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                const int first = (i * 4 + wave) * kTok, u = first >> 4;
                const char* p = base[0];
#pragma unroll
                for (int y = 1; y < U; ++y) p = u == y ? base[y] : p;
                if (!p) continue;
                p = uniform(p + (first & 15) * R::kBytes + (values ? to_values : 0));
                dma_load16_at<false>(p, values ? lane * 16 : key_off[i], to, i * 4096);
            }
        }
    };
    auto gone_bits = [&](const char* const (&base)[U]) {  // bit u: unit u is not there
        int bits = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) bits |= (base[u] == nullptr) << u;
        return bits;
    };
    const float scale_log2 = a.scale * kLog2e, inv_scale = 1.0f / scale_log2;
    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};

    // A half tile's fragments of keys and of values are read well before they are multiplied: a read from LDS takes longer
    // than a few products.
    u32x4_t kf[MB][R::kFrags], vf[DH / 16];
    auto read_keys = [&](const unsigned char* ks, int half) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int j = 0; j < R::kFrags; ++j)
                kf[mb][j] = *(const u32x4_t*)(ks + M::token(half * MB + mb, c16) * R::kBytes +
                                              (((4 * j + g) ^ (R::turn(c16) & (R::kPieces - 1))) << 4));
    };
    auto read_values = [&](const unsigned char* vs, int half) {
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) vf[i] = *(const u32x4_t*)(vs + (M::unit(half, g, DH, 16 * i + c16) << 4));
    };
    auto scores = [&](f32x4_t (&sc)[NC][MB]) {
#pragma unroll
        for (int j = 0; j < R::kFrags; ++j)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int c = 0; c < NC; ++c) sc[c][mb] = M::mma(kf[mb][j], bq[c][j], j == 0 ? zero4 : sc[c][mb]);
    };
    auto add_values = [&](const u32x4_t (&p)[NC]) {
#pragma unroll
        for (int i = 0; i < DH / 16; ++i)
#pragma unroll
            for (int c = 0; c < NC; ++c) ot[c][i] = M::mma(vf[i], p[c], ot[c][i]);
        if constexpr (kRounds) {
            constexpr uint32_t kOnes = 0x3f803f80u;  // two of bf16
#pragma unroll
            for (int c = 0; c < NC; ++c) lr[c] = M::mma(u32x4_t{kOnes, kOnes, kOnes, kOnes}, p[c], lr[c]);
        }
    };
    auto gone_mask = [&](int gone) -> uint32_t {  // bit r: token r of a half tile is not there
        return WIDE ? (gone ? ~0u : 0u) : (gone & 1 ? 0xffffu : 0u) | (gone & 2 ? 0xffff0000u : 0u);
    };
    // Values that no row here sees may be anything, and 0 x NaN must not reach a sum: they are cleared on their way.
    auto clear_unseen = [&](int tok, int gone) {
        if (!gone && tok + KS <= span.hi && (tok >= span.lo || tok + KS <= span.sinks)) return;
        const uint32_t seen = low_bits(span.hi - tok) & (low_bits(span.sinks - tok) | ~low_bits(span.lo - tok)) & ~gone_mask(gone);
        const int mine = (int)(seen >> (M::kLaneTok * g));
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe(mine, sizeof(T) == 2 ? 2 * d : d, 1);
            if (sizeof(T) == 2) keep = (keep & 0xffffu) | ((uint32_t)__builtin_amdgcn_sbfe(mine, 2 * d + 1, 1) & 0xffff0000u);
#pragma unroll
            for (int i = 0; i < DH / 16; ++i) vf[i][d] &= keep;
        }
    };
    // Before the exponentials of a step: what is not seen goes to -infinity, and ref moves up where a score is more than 2^8
    // above it (rarely: weights up to 2^8 lose nothing).  A whole step 2^-k is exact, also for weights `due` that are
    // rounded already and not yet multiplied with the values.
    auto settle = [&](f32x4_t (&sc)[NC][MB], int tok, int gone, u32x4_t (&due)[NC]) {
        if (gone || tok + KS > lim_min || (tok < from_max && tok + KS > span.sinks)) {
            const uint32_t sink = low_bits(span.sinks - tok), there = ~gone_mask(gone);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                // bit r: the column sees the step's token r; a lane's tokens are M::kLaneTok * g + token(mb, i)
                const uint32_t seen = low_bits(limit[c] - tok) & (sink | ~low_bits(from[c] - tok)) & there;
                const uint32_t mine = seen >> (M::kLaneTok * g);
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)mine, M::token(mb, i), 1);
                        sc[c][mb][i] = __uint_as_float((keep & __float_as_uint(sc[c][mb][i])) | (~keep & 0xff800000u));
                    }
            }
        }
        float top[NC];
        bool up = false;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            top[c] = -INFINITY;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i) top[c] = fmaxf(top[c], sc[c][mb][i]);
            up |= top[c] > bound[c];
        }
        if (__builtin_amdgcn_ballot_w64(up) == 0) return;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const float high = max_over_lane_groups(top[c]);  // the same decision in the four lanes of a column
            const bool move = high > bound[c];
            const float next = move ? __builtin_ceilf(high * scale_log2) : -minus_ref[c];
            const float down = move && bound[c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(-next - minus_ref[c]);
            minus_ref[c] = -next;
            bound[c] = move ? (next + 8.f) * inv_scale : bound[c];
            l[c] *= down;
            lr[c][0] *= down;
#pragma unroll
            for (int i = 0; i < DH / 16; ++i) ot[c][i] *= down;
            due[c] = M::times(due[c], down);
        }
    };
    auto weights = [&](f32x4_t (&sc)[NC][MB], u32x4_t (&p)[NC]) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[c][mb][i], scale_log2, minus_ref[c]));
                    sc[c][mb][i] = w;
                    if constexpr (LSE) l[c] += w;
                }
            p[c] = M::weights(sc[c]);
        }
    };

    // Products and exponentials take turns, so that matrix and vector units both have something to do.
    auto interleave = [&](u32x4_t (&p)[NC]) {
#pragma unroll
        for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(p[c]));  // the weights belong to this step, not to their use
        constexpr int kMma = NC * (DH / 16) * (sizeof(T) == 2 ? 1 : 4), kExp = NC * MB * 4, kPer = (kMma + kExp - 1) / kExp;
#pragma unroll
        for (int i = 0; i < kExp; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, kPer, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
        }
    };

    // A pipeline over half tiles: while one half's exponentials run on the vector units, the matrix units multiply the half
    // before with its values and the queries with the half after.  At tile x: values of x, keys of x + 1 are read; the
    // loads of keys x + 2 and values x + 1 are on their way.
    f32x4_t s0[NC][MB], s1[NC][MB];
    u32x4_t p0[NC], p1[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) p1[c] = u32x4_t{0, 0, 0, 0};
    int raw[U];
    const char *base_k[U], *base_v[U];  // units of the tile whose keys (values) are loaded next
    pages(0, raw);
    bases(0, raw, base_v);
    if (n > 0) load_tile(base_v, false, lds0);
    int gone_next = 0, gone = 0;  // units of tiles x + 1 and x that are not there
    pages(1, raw);
    constexpr int kHalfUnits = WIDE ? 1 : KS / 16;
    auto half_bits = [&](int bits, int half) { return WIDE ? (bits ? -1 : 0) : (bits >> (half * kHalfUnits)) & ((1 << kHalfUnits) - 1); };

    // Start of tile x: waits for its keys and values' loads, starts the next ones.
    auto turn = [&](int x) {
        const int b = (x + 1) & 1;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();  // keys x + 1 and values x are there, and nobody reads keys x and values x - 1 any more
        asm volatile("" ::: "memory");
        bases(x + 2, raw, base_k);
        gone = gone_next;
        gone_next = gone_bits(base_v);
        if (x + 2 < n) load_tile(base_k, false, lds0 + (b ^ 1) * kTileBytes);
        if (x + 1 < n) load_tile(base_v, true, lds0 + (2 + b) * kTileBytes);
#pragma unroll
        for (int u = 0; u < U; ++u) base_v[u] = base_k[u];
        pages(x + 3, raw);
    };
    if (n > 0) {
        turn(-1);
        read_keys(smem, 0);
        scores(s0);
        read_keys(smem, 1);
        settle(s0, span.step_at(it0) * KT, half_bits(gone_next, 0), p1);
        weights(s0, p0);
        scores(s1);
        for (int x = 0; x + 1 < n; ++x) {
            turn(x);
            const unsigned char *ks = smem + ((x + 1) & 1) * kTileBytes, *vs = smem + (2 + (x & 1)) * kTileBytes;
            read_values(vs, 0);
            __builtin_amdgcn_sched_barrier(0);
            const int tok = span.step_at(it0 + x) * KT;
            settle(s1, tok + KS, half_bits(gone, 1), p0);
            clear_unseen(tok, half_bits(gone, 0));
            read_keys(ks, 0);
            __builtin_amdgcn_sched_barrier(0);
            weights(s1, p1);
            add_values(p0);
            interleave(p1);
            __builtin_amdgcn_sched_barrier(0);
            read_values(vs, 1);
            __builtin_amdgcn_sched_barrier(0);
            scores(s0);
            __builtin_amdgcn_sched_barrier(0);
            settle(s0, span.step_at(it0 + x + 1) * KT, half_bits(gone_next, 0), p1);
            clear_unseen(tok + KS, half_bits(gone, 1));
            read_keys(ks, 1);
            __builtin_amdgcn_sched_barrier(0);
            weights(s0, p0);
            add_values(p1);
            interleave(p0);
            __builtin_amdgcn_sched_barrier(0);
            scores(s1);
        }
        turn(n - 1);
        const unsigned char* vs = smem + (2 + ((n - 1) & 1)) * kTileBytes;
        const int tok = span.step_at(it0 + n - 1) * KT;
        read_values(vs, 0);
        settle(s1, tok + KS, half_bits(gone, 1), p0);
        clear_unseen(tok, half_bits(gone, 0));
        weights(s1, p1);
        add_values(p0);
        read_values(vs, 1);
        clear_unseen(tok + KS, half_bits(gone, 1));
        add_values(p1);
    }
    float total[NC], sum[NC];
    bool again = false;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        total[c] = LSE ? sum_over_lane_groups(l[c]) : lr[c][0];
        sum[c] = kRounds ? lr[c][0] : total[c];
        again |= only_values_not_finite<DH>(ot[c], sum[c]);
    }
    if (__builtin_amdgcn_ballot_w64(again) != 0) {
        multiply_again<T, DH, NC>(
            kv, s, kh, span, 2 * n, [&](int x) { return span.step_at(it0 + (x >> 1)) * KT + (x & 1) * KS; }, bq, limit, from, scale_log2,
            minus_ref, ot);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        int col = qt * kCols + (wave * NC + c) * 16 + c16;
        asm volatile("" : "+v"(col));  // worked out again rather than kept in registers for the whole loop
        if (col >= n_cols) continue;
        const int64_t row = cr.row0 + col / hpk;
        const int head = kh * hpk + col % hpk;
        if (geo.n_split > 1) {
            const int64_t piece = (row * a.Hq + head) * geo.n_split + split;
            if (g == 0) piece_sums<DH>(a, geo)[piece] = {sum[c] != 0.f ? -minus_ref[c] : -INFINITY, sum[c], total[c], 0.f};
#pragma unroll
            for (int i = 0; i < DH / 16; ++i) *(f32x4_t*)(geo.part + piece * DH + 16 * i + 4 * g) = ot[c][i];
            continue;
        }
        const float inv = sum[c] != 0.f ? 1.0f / sum[c] : 0.f;
        T* out = (T*)a.out + row * a.out_stride + (int64_t)head * DH;
#pragma unroll
        for (int i = 0; i < DH / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) out[16 * i + 4 * g + e] = from_f32<T>(ot[c][i][e] * inv);
        if (a.lse && g == 0) a.lse[row * a.Hq + head] = sum[c] != 0.f ? -minus_ref[c] * (1.0f / kLog2e) + logf(total[c]) : -INFINITY;
    }
}

// ---------------------------------------------------------------------------
// up to 16 query columns per KV head.  The keys and values are used once, so they go to registers directly; a wave has the
// next step's 16 KiB on their way while it multiplies.  Bound by memory: 128 sequences of 4250 tokens of 7B heads 197 us =
// 5.7 TB/s (of 6.15 that a kernel which only reads reaches); one token over 2176 7.9 us, four rounds of dependent loads.
// ---------------------------------------------------------------------------
template <typename T, int DH>
__global__ __launch_bounds__(256, 2) void attn_few_kernel(PagedAttnArgs a, TileGeom geo) {
    using R = Row<T, DH>;
    using M = Mat<T>;
    constexpr int KS = M::kGroup, MB = KS / 16;  // tokens of a step
    __shared__ __attribute__((aligned(16))) float os[4][16][DH];
    __shared__ float ms[4][16], ls[4][16];
    const PagedKv& kv = a.kv;
    const int combo = blockIdx.x % geo.combos, split = blockIdx.x / geo.combos;
    const int kh = combo % kv.Hkv, s = combo / kv.Hkv, hpk = a.Hq / kv.Hkv;
    const ChunkRows cr = chunk_rows(kv, a.cu, s, a.n_rows, a.max_new);
    const int n_cols = cr.n * hpk;  // <= 16
    if (n_cols == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const Span span(cr.slot0, cr.slot0 + cr.n - 1, a.window, a.sinks, KS);
    const int per = (span.n + geo.n_split - 1) / geo.n_split;
    const int it0 = min(span.n, split * per), it1 = min(span.n, it0 + per);

    const bool real = c16 < n_cols;
    const int i_row = real ? c16 / hpk : 0, hq = kh * hpk + (real ? c16 % hpk : 0), t = cr.slot0 + i_row;
    const int limit = t + 1, from = a.window ? max(0, t - a.window + 1) : 0;
    u32x4_t cols[1][R::kFrags];
    auto& bq = cols[0];
    {
        const T* q = (const T*)a.q + (int64_t)(cr.row0 + i_row) * a.q_stride + (int64_t)hq * DH;
#pragma unroll
        for (int j = 0; j < R::kFrags; ++j) bq[j] = *(const u32x4_t*)(q + (4 * j + g) * R::kElems);
    }
    // a lane's share of a step: a fragment of each 16-token block's keys, a unit of every 16 channels' values.  bf16 has
    // both 16-token units of the pages in play, the one of the lane's key rows and the one of its values' octet.
    const int key_tok = M::token(0, c16), key_unit = key_tok >> 4, val_unit = sizeof(T) == 2 ? g >> 1 : 0;
    const int mask = (1 << kv.shift) - 1;
    const T* pool = (const T*)kv.pool;
    const int64_t to_values = (int64_t)kv.Hkv * kv.block();
    auto page_of = [&](int it, int u) {
        const int slot = span.step_at(it) * KS + 16 * u;
        return it < it1 && slot < span.hi ? kv.page(s, slot) : -1;
    };
    u32x4_t ak[2][MB][R::kFrags] = {}, av[2][DH / 16] = {};
    constexpr int kTok = M::kLaneTok;  // tokens of a lane's values; its keys are of the same many at most
    auto load = [&](int it, int pk, int pv, u32x4_t (&k)[MB][R::kFrags], u32x4_t (&v)[DH / 16]) {
        const int tok0 = span.step_at(it) * KS;
        // What is not there or not seen is not read (it is masked); at the edges of a window and of the sinks that counts:
        // 512 tokens and 4 sinks lie in 18 steps of 32 (512 rows of 1.5B heads 62.9 us with whole steps, 60.4 without).
        bool want_k = pk >= 0, want_v = pv >= 0;
        if (tok0 + KS > span.hi || (tok0 < span.lo && tok0 + KS > span.sinks)) {
            want_k = want_k && span.any_of(tok0 + key_tok / kTok * kTok, kTok);
            want_v = want_v && span.any_of(tok0 + kTok * g, kTok);
        }
        const T* kp = pool + kv.k_at(max(pk, 0), kh) + (int64_t)((tok0 + key_tok) & mask) * DH + g * R::kElems;
        const T* vp = pool + kv.k_at(max(pv, 0), kh) + to_values + (int64_t)((tok0 + 16 * val_unit) & mask) * DH;
        // units of values from there: as M::unit counts them, less the 16-token units before
        const int u0 = M::unit(0, g, DH, c16) - val_unit * 2 * DH;
        if (want_k) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int j = 0; j < R::kFrags; ++j)
                    k[mb][j] = *(const u32x4_t*)(kp + (M::token(mb, 0) - M::token(0, 0)) * DH + 4 * j * R::kElems);
        }
        if (want_v) {
#pragma unroll
            for (int i = 0; i < DH / 16; ++i)
                v[i] = *(const u32x4_t*)(vp + (int64_t)(u0 + (sizeof(T) == 2 ? 16 : 32) * i) * R::kElems);
        }
    };
    f32x4_t acc[1][DH / 16];
    auto& ot = acc[0];
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) ot[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const float scale_log2 = a.scale * kLog2e;
    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    const int lim_min = wave_min_int(limit), from_max = wave_max_int(from);

    auto step = [&](int it, int pk, int pv, u32x4_t (&k)[MB][R::kFrags], u32x4_t (&v)[DH / 16]) {
        const int tok0 = span.step_at(it) * KS;
        f32x4_t sc[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int j = 0; j < R::kFrags; ++j) sc[mb] = M::mma(k[mb][j], bq[j], j == 0 ? zero4 : sc[mb]);
        const uint64_t gone_k = __builtin_amdgcn_ballot_w64(pk < 0), gone_v = __builtin_amdgcn_ballot_w64(pv < 0);
        if (gone_k || gone_v || tok0 + KS > lim_min || (tok0 < from_max && tok0 + KS > span.sinks)) {
            // lanes 0-7 hold the first unit's page, 8-15 the second's (fp32: the only one's)
            const int gone = (int)(gone_k & 1) | (int)(gone_k >> 8 & 1) << 1;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = M::token(mb, 4 * g + i), j = tok0 + r;
                    const bool seen = j < limit && (j >= from || j < span.sinks) && !(gone >> (r >> 4) & 1);
                    sc[mb][i] = seen ? sc[mb][i] : -INFINITY;
                }
            // values that no row sees may be anything
            const int first = tok0 + kTok * g;
#pragma unroll
            for (int i = 0; i < DH / 16; ++i) {
                T e[kTok];
                *(u32x4_t*)e = v[i];
#pragma unroll
                for (int y = 0; y < kTok; ++y)
                    if (pv < 0 || !span.any(first + y)) e[y] = T{};
                v[i] = *(const u32x4_t*)e;
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[mb][i]);
        const float mnew = fmaxf(m, max_over_lane_groups(top));
        const float ref = mnew == -INFINITY ? 0.f : mnew;
        const float alpha = __builtin_amdgcn_exp2f((m - ref) * scale_log2), nb = -ref * scale_log2;
        float sum = 0.f;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[mb][i], scale_log2, nb));
                sc[mb][i] = w;
                sum += w;
            }
        l = l * alpha + sum;
        m = mnew;
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
            for (int i = 0; i < DH / 16; ++i) ot[i] *= alpha;
        }
        const u32x4_t p = M::weights(sc);
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) ot[i] = M::mma(v[i], p, ot[i]);
    };

    // wave w takes steps it0 + w, it0 + w + 4, ...; the next step's fragments are on their way while one is multiplied
    int it = it0 + wave;
    int pk = page_of(it, key_unit), pv = page_of(it, val_unit);
    int pk2 = page_of(it + 4, key_unit), pv2 = page_of(it + 4, val_unit);
    if (it < it1) load(it, pk, pv, ak[0], av[0]);
    while (it < it1) {
        if (it + 4 < it1) load(it + 4, pk2, pv2, ak[1], av[1]);
        int pk3 = page_of(it + 8, key_unit), pv3 = page_of(it + 8, val_unit);
        step(it, pk, pv, ak[0], av[0]);
        it += 4;
        if (it >= it1) break;
        if (it + 4 < it1) load(it + 4, pk3, pv3, ak[0], av[0]);
        pk = page_of(it + 8, key_unit), pv = page_of(it + 8, val_unit);
        step(it, pk2, pv2, ak[1], av[1]);
        pk2 = pk, pv2 = pv;
        pk = pk3, pv = pv3;
        it += 4;
    }
    // join the four waves
    const float wave_l = sum_over_lane_groups(l);
    if (cr.n > 1 && __builtin_amdgcn_ballot_w64(only_values_not_finite<DH>(ot, wave_l)) != 0) {  // the columns of one row see the same
        const int limits[1] = {limit}, froms[1] = {from};
        const float minus_ref[1] = {m == -INFINITY ? 0.f : -m * scale_log2};
        multiply_again<T, DH, 1>(
            kv, s, kh, span, (it1 - it0 - wave + 3) >> 2, [&](int x) { return span.step_at(it0 + wave + 4 * x) * KS; }, cols, limits, froms,
            scale_log2, minus_ref, acc);
    }
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) *(f32x4_t*)&os[wave][c16][16 * i + 4 * g] = ot[i];
    if (g == 0) ms[wave][c16] = m * scale_log2, ls[wave][c16] = wave_l;
    __syncthreads();
    for (int x = tid; x < n_cols * (DH / 4); x += 256) {
        const int c = x / (DH / 4), ch = x % (DH / 4) * 4;
        float top = -INFINITY, total = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, ms[w][c]);
        f32x4_t o = zero4;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float wgt = ms[w][c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms[w][c] - top);
            total += wgt * ls[w][c];
            o += wgt * *(const f32x4_t*)&os[w][c][ch];
        }
        const int i = c / hpk;
        const int64_t row = cr.row0 + i, head = kh * hpk + c % hpk, at = row * a.Hq + head;
        if (geo.n_split > 1) {
            const int64_t piece = at * geo.n_split + split;
            *(f32x4_t*)(geo.part + piece * DH + ch) = o;
            // A piece is empty if its sum is 0.  Scores that are all NaN have no maximum (fmaxf passes them over), but their sum,
            // a NaN, has to reach the join.
            const float ref = total == 0.f ? -INFINITY : top == -INFINITY ? 0.f : top;
            if (ch == 0) piece_sums<DH>(a, geo)[piece] = {ref, total, total, 0.f};
            continue;
        }
        const float inv = total != 0.f ? 1.0f / total : 0.f;
        T* out = (T*)a.out + row * a.out_stride + head * DH + ch;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = from_f32<T>(o[e] * inv);
        if (a.lse && ch == 0) a.lse[at] = total != 0.f ? top * (1.0f / kLog2e) + logf(total) : -INFINITY;
    }
}

// A thread takes four channels of a head of a row of sequence blockIdx.y; threads are dealt to (row, head, channels) in order, so
// that a workgroup may hold several rows, or parts of two.  Pieces are weighed by what their sums are relative to.
template <typename T, int DH>
__global__ __launch_bounds__(256) void attn_join_kernel(PagedAttnArgs a, TileGeom geo) {
    const int s = blockIdx.y, n_split = geo.n_split;
    const ChunkRows cr = chunk_rows(a.kv, a.cu, s, a.n_rows, a.max_new);
    const int per_row = a.Hq * (DH / 4);
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int i = (int)(x / per_row);
    if (i >= cr.n) return;
    const int head = (int)(x % per_row) / (DH / 4), ch = (int)(x % (DH / 4)) * 4;
    const int64_t row = cr.row0 + i, at = row * a.Hq + head, piece = at * n_split;
    const PieceSums* sums = piece_sums<DH>(a, geo) + piece;
    const float* po = geo.part + piece * DH + ch;
    // eight pieces' loads at once: what counts is the number of times that memory is waited for
    constexpr int kAtOnce = 8;
    float top = -INFINITY, total = 0.f, lse_total = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < n_split; p0 += kAtOnce) {
        PieceSums of[kAtOnce];
        f32x4_t v[kAtOnce];
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) {
            const int p = min(p0 + y, n_split - 1);
            of[y] = sums[p];
            v[y] = *(const f32x4_t*)(po + (int64_t)p * DH);
        }
        float next = top;
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) next = fmaxf(next, of[y].top);
        if (next == -INFINITY) continue;  // nothing seen so far
        const float down = __builtin_amdgcn_exp2f(top - next);
        top = next;
        total *= down;
        lse_total *= down;
        o *= down;
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) {
            if (p0 + y >= n_split || of[y].top == -INFINITY) continue;  // a piece that saw nothing holds anything
            const float wgt = __builtin_amdgcn_exp2f(of[y].top - top);
            total += wgt * of[y].sum;
            lse_total += wgt * of[y].lse_sum;
            o += wgt * v[y];
        }
    }
    const float inv = total != 0.f ? 1.0f / total : 0.f;
    T* out = (T*)a.out + row * a.out_stride + (int64_t)head * DH + ch;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = from_f32<T>(o[e] * inv);
    if (a.lse && ch == 0) a.lse[at] = total != 0.f ? top * (1.0f / kLog2e) + logf(lse_total) : -INFINITY;
}

// ---------------------------------------------------------------------------
// scores: the weights of a token summed over the query columns.  Products the other way round, S = Q K^T, so that a lane
// holds scores of one token and its sum stays in one register; the keys of a wave's tokens stay in registers throughout.
// Chunks are bound by vector and matrix units together (64 exponentials, fma and sums a lane and tile against 64 products):
// 4 x 4352 rows of 7B heads 303 us = 0.9 PFLOP/s.  Single tokens by memory: 512 rows over 2100 tokens 113 us = 5.0 TB/s.
// ---------------------------------------------------------------------------
struct ScoreGeom {
    int combos;
    int n_split;  // pieces that the query columns are cut into
    float* part;  // n_split > 1: [piece, sequence, KV head][max_len] sums
};

// 16-token blocks of a wave: 64 VGPRs of keys at 128 channels
template <typename T>
constexpr int kScoreBlocks = sizeof(T) == 2 ? 4 : 2;

// A wave's keys as operands; bit mb of the result: block mb is not there.
template <typename T, int DH>
__device__ inline int load_keys(const PagedKv& kv, int s, int kh, int tok0, int len, u32x4_t (&k)[kScoreBlocks<T>][Row<T, DH>::kFrags]) {
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4, mask = (1 << kv.shift) - 1;
    int gone = 0;
#pragma unroll
    for (int mb = 0; mb < kScoreBlocks<T>; ++mb) {
        const int slot = tok0 + 16 * mb;
        const int page = slot < len ? __builtin_amdgcn_readfirstlane(kv.page(s, slot)) : -1;
        const T* at = (const T*)kv.pool + kv.k_at(max(page, 0), kh) + (int64_t)((slot & mask) + c16) * DH + g * Row<T, DH>::kElems;
        gone |= (page < 0) << mb;
#pragma unroll
        for (int j = 0; j < Row<T, DH>::kFrags; ++j)
            k[mb][j] = page < 0 ? u32x4_t{0, 0, 0, 0} : *(const u32x4_t*)(at + 4 * j * Row<T, DH>::kElems);
    }
    return gone;
}

// A lane's token of the wave's, and where its score so far comes from; the lanes beyond the tokens have none.
struct ScoreSlot {
    int64_t at;
    bool there;
    float before;
    __device__ ScoreSlot(const PagedScoreArgs& b, int combo, int tok0, int n_tok, int len) {
        const int lane = threadIdx.x & 63;
        at = combo * b.score_stride + tok0 + lane;
        there = lane < n_tok && tok0 + lane < len;
        before = there && b.score_in ? b.score_in[at] : 0.f;
    }
};
// The sums of a wave's tokens to where they go: lane l writes token l.
template <int MB>
__device__ inline void store_scores(const PagedScoreArgs& b, const ScoreGeom& geo, int combo, int split, const ScoreSlot& slot, int tok0,
                                    int gone, const float (&acc)[MB]) {
    const int g = (threadIdx.x & 63) >> 4;
    float sum = 0.f;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const float x = sum_over_lane_groups(acc[mb]);  // of token 16 mb + lane % 16
        if (g == mb && !(gone >> mb & 1)) sum = x;
    }
    if (!slot.there) return;
    if (geo.n_split > 1)
        geo.part[((int64_t)split * geo.combos + combo) * b.at.max_len + tok0 + (threadIdx.x & 63)] = sum;
    else
        b.score_out[slot.at] = slot.before + sum;
}

template <typename T, int DH>
__global__ __launch_bounds__(256) void score_few_kernel(PagedScoreArgs b, ScoreGeom geo) {
    using R = Row<T, DH>;
    using M = Mat<T>;
    constexpr int MB = kScoreBlocks<T>;
    const PagedAttnArgs& a = b.at;
    const PagedKv& kv = a.kv;
    const int combo = blockIdx.x % geo.combos, kh = combo % kv.Hkv, s = combo / kv.Hkv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    const int tok0 = (blockIdx.x / geo.combos * 4 + wave) * 16 * MB;
    const int len = min((int)min((int64_t)kv.length(s), b.score_stride), a.max_len);
    if (tok0 >= len) return;
    const ChunkRows cr = chunk_rows(kv, a.cu, s, a.n_rows, a.max_new);
    const int hpk = a.Hq / kv.Hkv, n_cols = cr.n * hpk;
    const Span span(cr.slot0, cr.slot0 + cr.n - 1, a.window, a.sinks, 16);
    const bool some = n_cols > 0 && tok0 < span.hi && (tok0 < span.sinks || tok0 + 16 * MB > span.lo);
    if (!some && b.score_in == b.score_out) return;
    float acc[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) acc[mb] = 0.f;
    int gone = 0;
    u32x4_t k[MB][R::kFrags], q[R::kFrags];
    if (some) gone = load_keys<T, DH>(kv, s, kh, tok0, len, k);
    const ScoreSlot slot(b, combo, tok0, 16 * MB, len);
    if (some) {
        const int col = c16 < n_cols ? c16 : 0;
        const T* qp = (const T*)a.q + (int64_t)(cr.row0 + col / hpk) * a.q_stride + (int64_t)(kh * hpk + col % hpk) * DH;
#pragma unroll
        for (int j = 0; j < R::kFrags; ++j) q[j] = *(const u32x4_t*)(qp + (4 * j + g) * R::kElems);
        int t[4];
        float shift[4];  // -lse in the log2 domain
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = 4 * g + i, y = x < n_cols ? x : 0;
            const float lse = b.lse_in[(int64_t)(cr.row0 + y / hpk) * a.Hq + kh * hpk + y % hpk];
            // what gives nothing sits below slot 0 and sees nothing: its product may be NaN
            t[i] = x < n_cols && lse != -INFINITY ? cr.slot0 + y / hpk : -1;
            shift[i] = -lse * kLog2e;
        }
        const float scale_log2 = a.scale * kLog2e;
        const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            f32x4_t sc;
#pragma unroll
            for (int j = 0; j < R::kFrags; ++j) sc = M::mma(q[j], k[mb][j], j == 0 ? zero4 : sc);
            const int tok = tok0 + 16 * mb + c16;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], scale_log2, shift[i]));
                acc[mb] += sees(t[i], tok, a.window, a.sinks) ? w : 0.f;
            }
        }
    }
    store_scores<MB>(b, geo, combo, 0, slot, tok0, gone, acc);
}

template <typename T, int DH>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) void score_tile_kernel(PagedScoreArgs b, ScoreGeom geo) {
    using R = Row<T, DH>;
    using M = Mat<T>;
    constexpr int MB = kScoreBlocks<T>, QT = 64;      // query columns of a tile
    constexpr int kTileBytes = QT * R::kBytes, kChunks = kTileBytes / 4096;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * kTileBytes];
    __shared__ __attribute__((aligned(16))) float shifts[2][QT];
    __shared__ __attribute__((aligned(16))) int slots[2][QT];
    __shared__ int idle[2];  // whether a tile has columns that give nothing
    const PagedAttnArgs& a = b.at;
    const PagedKv& kv = a.kv;
    const int combo = blockIdx.x % geo.combos, rest = blockIdx.x / geo.combos, split = rest % geo.n_split;
    const int kh = combo % kv.Hkv, s = combo / kv.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, g = lane >> 4;
    const int wg0 = rest / geo.n_split * 64 * MB, tok0 = wg0 + wave * 16 * MB, tok1 = tok0 + 16 * MB;  // first blocks: most rows
    const int len = min((int)min((int64_t)kv.length(s), b.score_stride), a.max_len);
    if (wg0 >= len) return;
    const ChunkRows cr = chunk_rows(kv, a.cu, s, a.n_rows, a.max_new);
    const int hpk = a.Hq / kv.Hkv;
    // columns whose rows see any of the workgroup's tokens
    const int first = min(cr.n, max(0, wg0 - cr.slot0));
    const int64_t past = a.window && wg0 >= a.sinks ? (int64_t)wg0 + 64 * MB - 1 + a.window - cr.slot0 : cr.n;
    const int last = (int)min((int64_t)cr.n, max(past, (int64_t)first));
    const int tile0 = first * hpk / QT, n_tiles = first < last ? (last * hpk + QT - 1) / QT - tile0 : 0;
    const int per = (n_tiles + geo.n_split - 1) / geo.n_split;
    const int it0 = tile0 + min(n_tiles, split * per), it1 = min(tile0 + n_tiles, it0 + per);

    u32x4_t k[MB][R::kFrags];
    const int gone = load_keys<T, DH>(kv, s, kh, tok0, len, k);
    float acc[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) acc[mb] = 0.f;

    // a lane's column in the wave's i-th load: row and head, moved on by QT columns from tile to tile
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const int row_step = QT / hpk, head_step = QT % hpk;
    int ci[kChunks], ch[kChunks], piece[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int at = (i * 4 + wave) * 1024 + lane * 16, c = at / R::kBytes, p = at % R::kBytes / 16;
        ci[i] = (it0 * QT + c) / hpk;
        ch[i] = (it0 * QT + c) % hpk;
        piece[i] = (p ^ (R::turn(c & 15) & (R::kPieces - 1))) << 4;
    }
    int si = (it0 * QT + lane) / hpk, sh = (it0 * QT + lane) % hpk;  // wave 0: the column whose lse it fetches
    float shift_next = 0.f;
    int slot_next = 0, idle_next = 0;
    auto load_tile = [&](int it, int buf) {
        const int base = min(it * QT / hpk, cr.n - 1);
        const T* q = uniform((const T*)a.q + (int64_t)(cr.row0 + base) * a.q_stride + (int64_t)kh * hpk * DH);
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int x = min(ci[i], cr.n - 1);  // columns behind the last row: any that exist
            const uint32_t off = (uint32_t)((x - base) * (int)a.q_stride + ch[i] * DH) * (uint32_t)sizeof(T) + piece[i];
            dma_load16_at<false>(q, off, lds0 + buf * kTileBytes + wave * 1024, i * 4096);
            ci[i] += row_step, ch[i] += head_step;
            if (ch[i] >= hpk) ch[i] -= hpk, ++ci[i];
        }
        if (wave == 0) {
            const int x = min(si, cr.n - 1);
            const float lse = b.lse_in[(int64_t)(cr.row0 + x) * a.Hq + kh * hpk + sh];
            // a column behind the last row or with an lse of -infinity sits below slot 0 and sees nothing: its product may be NaN
            const bool gives = si < cr.n && lse != -INFINITY;
            shift_next = -lse * kLog2e;
            slot_next = gives ? cr.slot0 + x : -1;
            idle_next = __builtin_amdgcn_ballot_w64(!gives) != 0;
            si += row_step, sh += head_step;
            if (sh >= hpk) sh -= hpk, ++si;
        }
    };
    const float scale_log2 = a.scale * kLog2e;
    const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
    auto keep_next = [&](int buf) {
        if (wave == 0) shifts[buf][lane] = shift_next, slots[buf][lane] = slot_next, idle[buf] = idle_next;
    };
    if (it0 < it1) {
        load_tile(it0, 0);
        keep_next(0);
    }
    for (int it = it0; it < it1; ++it) {
        const int buf = (it - it0) & 1;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();  // the tile is there, and nobody reads the other buffer any more
        asm volatile("" ::: "memory");
        const bool more = it + 1 < it1;
        if (more) load_tile(it + 1, buf ^ 1);
        const int t_min = cr.slot0 + it * QT / hpk, t_max = cr.slot0 + min(cr.n - 1, (it * QT + QT - 1) / hpk);
        // rows of this tile that see any of the wave's tokens, and whether all see all
        const bool some = t_max >= tok0 && (!a.window || t_min - (tok1 - 1) < a.window || tok0 < a.sinks) && tok0 < len;
        const bool all = __builtin_amdgcn_readfirstlane(idle[buf]) == 0 && t_min >= tok1 - 1 && (!a.window || t_max - tok0 < a.window || tok1 <= a.sinks);
        if (some) {
#pragma unroll
            for (int cg = 0; cg < QT / 16; ++cg) {
                u32x4_t q[R::kFrags];
#pragma unroll
                for (int j = 0; j < R::kFrags; ++j)
                    q[j] = *(const u32x4_t*)(smem + buf * kTileBytes + (cg * 16 + c16) * R::kBytes +
                                             (((4 * j + g) ^ (R::turn(c16) & (R::kPieces - 1))) << 4));
                const f32x4_t shift = *(const f32x4_t*)&shifts[buf][cg * 16 + 4 * g];
                f32x4_t sc[MB];
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int j = 0; j < R::kFrags; ++j) sc[mb] = M::mma(q[j], k[mb][j], j == 0 ? zero4 : sc[mb]);
                if (all) {
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[mb] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[mb][i], scale_log2, shift[i]));
                } else {
                    int t[4];
                    *(u32x4_t*)t = *(const u32x4_t*)&slots[buf][cg * 16 + 4 * g];
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[mb][i], scale_log2, shift[i]));
                            acc[mb] += sees(t[i], tok0 + 16 * mb + c16, a.window, a.sinks) ? w : 0.f;
                        }
                }
            }
        }
        if (more) keep_next(buf ^ 1);
    }
    store_scores<MB>(b, geo, combo, split, ScoreSlot(b, combo, tok0, 16 * MB, len), tok0, gone, acc);
}

__global__ __launch_bounds__(256) void score_join_kernel(PagedScoreArgs b, ScoreGeom geo) {
    const int combo = blockIdx.y, s = combo / b.at.kv.Hkv, j = blockIdx.x * 256 + threadIdx.x;
    if (j >= min(min((int64_t)b.at.kv.length(s), b.score_stride), (int64_t)b.at.max_len)) return;
    float sum = 0.f;
    for (int p = 0; p < geo.n_split; ++p) sum += geo.part[((int64_t)p * geo.combos + combo) * b.at.max_len + j];
    const int64_t at = combo * b.score_stride + j;
    b.score_out[at] = (b.score_in ? b.score_in[at] : 0.f) + sum;
}

// ---------------------------------------------------------------------------
// any head_dim: a wave streams 64 tokens at a time, a lane to a token for the scores, a lane to a channel for the values
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(64) void attn_rows_kernel(PagedAttnArgs a) {
    __shared__ float qs[256], ps[64];
    __shared__ int64_t vs[64];
    const PagedKv& kv = a.kv;
    const int i = blockIdx.x, hq = blockIdx.y, s = blockIdx.z, lane = threadIdx.x;
    const ChunkRows c = chunk_rows(kv, a.cu, s, a.n_rows, a.max_new);
    if (i >= c.n) return;
    const int dh = kv.dh, kh = hq / (a.Hq / kv.Hkv), mask = (1 << kv.shift) - 1;
    const int64_t row = c.row0 + i;
    const int t = c.slot0 + i;
    const T* pool = (const T*)kv.pool;
    for (int d = lane; d < dh; d += 64) qs[d] = to_f32<T>(((const T*)a.q)[row * a.q_stride + (int64_t)hq * dh + d]);
    __syncthreads();
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const int lo = a.window ? max(0, t - a.window + 1) : 0;
    for (int c0 = 0; c0 <= t; c0 += 64) {
        if (c0 >= a.sinks && c0 + 64 <= lo) continue;  // nothing visible here
        const int j = c0 + lane;
        const int page = j <= t && sees(t, j, a.window, a.sinks) ? kv.page(s, j) : -1;
        float x = -INFINITY;
        if (page >= 0) {
            const T* kp = pool + kv.k_at(page, kh) + (int64_t)(j & mask) * dh;
            float dot = 0.f;
            for (int d = 0; d < dh; ++d) dot = fmaf(qs[d], to_f32<T>(kp[d]), dot);
            x = dot * a.scale;
        }
        const float mnew = fmaxf(m, wave_max(x));
        const float ref = mnew == -INFINITY ? 0.f : mnew;
        const float p = page >= 0 ? expf(x - ref) : 0.f, alpha = expf(m - ref);
        l = l * alpha + wave_sum(p);
        m = mnew;
        __syncthreads();
        ps[lane] = p;
        vs[lane] = page >= 0 ? kv.v_at(page, kh) + (int64_t)((j & mask) >> 3) * dh * 8 + (j & 7) : -1;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int d = lane + 64 * u;
            float acc = o[u] * alpha;
            if (d < dh)
                for (int x = 0; x < 64; ++x)
                    if (vs[x] >= 0) acc = fmaf(ps[x], to_f32<T>(pool[vs[x] + (int64_t)d * 8]), acc);
            o[u] = acc;
        }
    }
    const float inv = l != 0.f ? 1.0f / l : 0.f;
    T* out = (T*)a.out + row * a.out_stride + (int64_t)hq * dh;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int d = lane + 64 * u;
        if (d < dh) out[d] = from_f32<T>(o[u] * inv);
    }
    if (a.lse && lane == 0) a.lse[row * a.Hq + hq] = l != 0.f ? m + logf(l) : -INFINITY;
}

// ---------------------------------------------------------------------------
// any head_dim: 32 keys in LDS, the rows that see any of them dealt to eight groups of 32 threads
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void score_rows_kernel(PagedScoreArgs b) {
    __shared__ float ks[32][257];
    __shared__ float part[8][32];
    const PagedAttnArgs& a = b.at;
    const PagedKv& kv = a.kv;
    const int kh = blockIdx.y, s = blockIdx.z, j0 = blockIdx.x * 32, tid = threadIdx.x;
    const int len = min((int)min((int64_t)kv.length(s), b.score_stride), a.max_len);
    if (j0 >= len) return;
    const int dh = kv.dh, hpk = a.Hq / kv.Hkv, mask = (1 << kv.shift) - 1;
    const ChunkRows c = chunk_rows(kv, a.cu, s, a.n_rows, a.max_new);
    for (int x = tid; x < 32 * dh; x += 256) {
        const int j = j0 + x / dh, d = x % dh;
        const int page = j < len ? kv.page(s, j) : -1;
        ks[x / dh][d] = page >= 0 ? to_f32<T>(((const T*)kv.pool)[kv.k_at(page, kh) + (int64_t)(j & mask) * dh + d]) : 0.f;
    }
    __syncthreads();
    const int tok = tid & 31, grp = tid >> 5, j = j0 + tok;
    const bool there = j < len && kv.page(s, j) >= 0;
    const int i0 = max(0, j0 - c.slot0);  // rows before it see none of these tokens
    float sum = 0.f;
    for (int x = i0 * hpk + grp; x < c.n * hpk; x += 8) {
        const int i = x / hpk, hq = kh * hpk + x % hpk;
        if (!there || !sees(c.slot0 + i, j, a.window, a.sinks)) continue;
        const int64_t row = c.row0 + i;
        const float lse = b.lse_in[row * a.Hq + hq];
        if (lse == -INFINITY) continue;  // a row that sees nothing gives nothing
        const T* q = (const T*)a.q + row * a.q_stride + (int64_t)hq * dh;
        float dot = 0.f;
        for (int d = 0; d < dh; ++d) dot = fmaf(to_f32<T>(q[d]), ks[tok][d], dot);
        sum += expf(dot * a.scale - lse);
    }
    part[grp][tok] = sum;
    __syncthreads();
    if (tid < 32 && j0 + tid < len) {
        float all = 0.f;
        for (int g = 0; g < 8; ++g) all += part[g][tid];
        const int64_t at = ((int64_t)s * kv.Hkv + kh) * b.score_stride + j0 + tid;
        b.score_out[at] = (b.score_in ? b.score_in[at] : 0.f) + all;
    }
}

constexpr int64_t kMaxGrid = 0xffffff;  // workgroups of 256 threads: a launch has fewer than 2^32 threads in a row

// Whether the matrix kernels take a call: fragments are 16 aligned bytes, offsets inside a tile of rows 32 bits.
bool tiles_take(const PagedAttnArgs& a) {
    const int es = (int)dtype_size(a.kv.dtype);
    return a.path != 1 && (a.kv.dh == 32 || a.kv.dh == 64 || a.kv.dh == 128) && (uintptr_t)a.q % 16 == 0 && a.q_stride * es % 16 == 0;
}
// Up to 16 columns per KV head go to the kernel that streams tokens to registers: us a call, tiles / it, one token over
// 4 x 8000 19.1 / 14.7, over 32 x 1750 in fp32 43.6 / 27.7; 14 columns over 2 x 4000 13.6 / 15.1.
int64_t n_cols(const PagedAttnArgs& a) { return (int64_t)a.max_new * (a.Hq / a.kv.Hkv); }
bool few_take(const PagedAttnArgs& a) { return n_cols(a) <= 16; }
// Columns of a tile: 64 where they hold a chunk (128 / 64: 64 x 8 rows of 1.5B heads over 2100 tokens 36.4 / 31.4 us, 26 x 9
// rows in fp32 over 80 tokens 26.7 / 14.9), else 128, which read every fragment of keys and values for twice the columns.
int tile_cols(const PagedAttnArgs& a) { return n_cols(a) <= 64 ? 64 : 128; }
int64_t attn_tiles(const PagedAttnArgs& a) { return few_take(a) ? 1 : ceil_div64(n_cols(a), tile_cols(a)); }

// Slots that the rows of a chunk see at most.
int most_seen(const PagedAttnArgs& a) {
    const int64_t w = a.window ? (int64_t)a.window + a.max_new + a.sinks : a.max_len;
    return (int)(w < a.max_len ? w : a.max_len);
}

// Pieces that the tokens of a sequence are cut into: as many as the two workgroups that a CU holds leave room for (one more
// round for the rest costs more than it gives: fp32, 8 sequences of 200 rows, 304 workgroups, in two pieces 250 us, whole 190),
// but none so short that the partial sums, 4 bytes a channel and query column, outweigh the tokens: eight steps of the
// few-column kernel (two a wave; with four, a token over 2176 took 10.8 instead of 10.4 us), two tokens for every column of a
// tile (7B heads, 2 x 20 rows over 4000 tokens: 128 / 256 / 512 tokens for 128 columns 20.0 / 19.4 / 22.8 us).
int attn_splits(const PagedAttnArgs& a) {
    if (a.kv.n_seqs < 1 || a.max_new < 1 || a.max_len < 1 || !tiles_take(a)) return 1;
    const bool few = few_take(a);
    const int64_t groups = (int64_t)a.kv.n_seqs * a.kv.Hkv * attn_tiles(a);
    const int step = few ? 8 * (a.kv.dtype == kF32 ? Mat<float>::kGroup : Mat<bf16>::kGroup) : 2 * tile_cols(a);
    const int64_t room = 512 / groups, cap = most_seen(a) / step;
    const int64_t n = room < cap ? room : cap;
    return (int)(n < 1 ? 1 : n < 64 ? n : 64);
}

// Workgroups that join a sequence's rows.
int64_t join_groups(const PagedAttnArgs& a) { return ceil_div64((int64_t)a.max_new * a.Hq * (a.kv.dh / 4), 256); }

template <typename T, int DH>
hipError_t launch_tiles(const PagedAttnArgs& a, hipStream_t s) {
    TileGeom geo;
    geo.combos = a.kv.n_seqs * a.kv.Hkv;
    geo.n_split = a.ws ? attn_splits(a) : 1;
    geo.part = (float*)a.ws;
    const int64_t grid = attn_tiles(a) * geo.combos * geo.n_split, join = join_groups(a);
    const bool wide = (1 << a.kv.shift) >= 2 * Mat<T>::kGroup, small = tile_cols(a) == 64;
    auto tiles = [&](auto lse) {
        return wide ? (small ? attn_tile_kernel<T, DH, 1, true, lse.value> : attn_tile_kernel<T, DH, 2, true, lse.value>)
                    : (small ? attn_tile_kernel<T, DH, 1, false, lse.value> : attn_tile_kernel<T, DH, 2, false, lse.value>);
    };
    auto kernel = few_take(a) ? attn_few_kernel<T, DH>
                  : a.lse     ? tiles(std::true_type{})
                              : tiles(std::bool_constant<sizeof(T) == 4>{});  // fp32 has one sum for both
    kernel<<<(unsigned)grid, 256, 0, s>>>(a, geo);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || geo.n_split == 1) return e;
    attn_join_kernel<T, DH><<<dim3((unsigned)join, a.kv.n_seqs), 256, 0, s>>>(a, geo);
    return hipGetLastError();
}

// Offsets of a tile's query rows from its first one are 32 bits.
bool score_tiles_take(const PagedScoreArgs& b) {
    return tiles_take(b.at) && b.at.q_stride < ((int64_t)1 << 30) / 66 / (int)dtype_size(b.at.kv.dtype);
}

// Pieces that the query columns are cut into: about four workgroups per CU (two: 7B heads, 1 x 8000 rows 448 instead of 279 us,
// for want of balance between the first and the last tokens), none of fewer than three tiles (eight / three: 8 x 150 rows of
// 1.5B heads over 2100 tokens 44.7 / 23.7 us, 500 rows over 4000 32.5 / 26.0).
int score_splits(const PagedScoreArgs& b) {
    const PagedAttnArgs& a = b.at;
    if (a.kv.n_seqs < 1 || a.max_new < 1 || a.max_len < 1 || !score_tiles_take(b) || few_take(a)) return 1;
    const int64_t rows = a.window && a.window + (int64_t)256 < a.max_new ? a.window + 256 : a.max_new;
    const int64_t tiles = ceil_div64(rows * (a.Hq / a.kv.Hkv), 64);
    const int64_t groups = (int64_t)a.kv.n_seqs * a.kv.Hkv * ceil_div(a.max_len, a.kv.dtype == kF32 ? 128 : 256);
    const int64_t want = ceil_div64(1024, groups), cap = tiles / 3 > 0 ? tiles / 3 : 1;
    const int64_t n = want < cap ? want : cap;
    return (int)(n < 16 ? n : 16);
}

template <typename T, int DH>
hipError_t launch_score_tiles(const PagedScoreArgs& b, hipStream_t s) {
    const PagedAttnArgs& a = b.at;
    ScoreGeom geo;
    geo.combos = a.kv.n_seqs * a.kv.Hkv;
    geo.n_split = a.ws ? score_splits(b) : 1;
    geo.part = (float*)a.ws;
    const int64_t grid = (int64_t)ceil_div(a.max_len, 64 * kScoreBlocks<T>) * geo.combos * geo.n_split;
    if (few_take(a))
        score_few_kernel<T, DH><<<(unsigned)grid, 256, 0, s>>>(b, geo);
    else
        score_tile_kernel<T, DH><<<(unsigned)grid, 256, 0, s>>>(b, geo);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || geo.n_split == 1) return e;
    score_join_kernel<<<dim3(ceil_div(a.max_len, 256), geo.combos), 256, 0, s>>>(b, geo);
    return hipGetLastError();
}

}  // namespace

bool paged_attn_fits(const PagedAttnArgs& a) {
    if (!tiles_take(a)) return true;  // its grid has three dimensions
    const int n = a.ws ? attn_splits(a) : 1;
    return attn_tiles(a) * a.kv.n_seqs * a.kv.Hkv * n <= kMaxGrid && (n == 1 || join_groups(a) <= kMaxGrid);
}
bool paged_score_fits(const PagedScoreArgs& b) {
    const PagedAttnArgs& a = b.at;
    if (!score_tiles_take(b)) return ceil_div(a.max_len, 32) <= kMaxGrid;
    const int tokens = a.kv.dtype == kF32 ? 64 * kScoreBlocks<float> : 64 * kScoreBlocks<bf16>;
    return (int64_t)ceil_div(a.max_len, tokens) * a.kv.n_seqs * a.kv.Hkv * (a.ws ? score_splits(b) : 1) <= kMaxGrid;
}

size_t paged_attn_ws_bytes(const PagedAttnArgs& a) {
    const int n = attn_splits(a);
    return n == 1 ? 0 : (size_t)a.n_rows * a.Hq * n * (a.kv.dh * 4 + sizeof(PieceSums));
}
size_t paged_score_ws_bytes(const PagedScoreArgs& b) {
    const int n = score_splits(b);
    return n == 1 ? 0 : (size_t)n * b.at.kv.n_seqs * b.at.kv.Hkv * b.at.max_len * 4;
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
    if (a.n_rows <= 0 || a.kv.n_seqs <= 0 || a.max_new <= 0) return hipSuccess;
    if (tiles_take(a)) {
        const bool f32 = a.kv.dtype == kF32;
        if (a.kv.dh == 128) return f32 ? launch_tiles<float, 128>(a, s) : launch_tiles<bf16, 128>(a, s);
        if (a.kv.dh == 64) return f32 ? launch_tiles<float, 64>(a, s) : launch_tiles<bf16, 64>(a, s);
        return f32 ? launch_tiles<float, 32>(a, s) : launch_tiles<bf16, 32>(a, s);
    }
    const dim3 grid(a.max_new, a.Hq, a.kv.n_seqs);
    if (a.kv.dtype == kF32)
        attn_rows_kernel<float><<<grid, 64, 0, s>>>(a);
    else
        attn_rows_kernel<bf16><<<grid, 64, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_score(const PagedScoreArgs& b, hipStream_t s) {
    const PagedAttnArgs& a = b.at;
    if (a.kv.n_seqs <= 0 || a.max_len <= 0) return hipSuccess;
    if (score_tiles_take(b)) {
        const bool f32 = a.kv.dtype == kF32;
        if (a.kv.dh == 128) return f32 ? launch_score_tiles<float, 128>(b, s) : launch_score_tiles<bf16, 128>(b, s);
        if (a.kv.dh == 64) return f32 ? launch_score_tiles<float, 64>(b, s) : launch_score_tiles<bf16, 64>(b, s);
        return f32 ? launch_score_tiles<float, 32>(b, s) : launch_score_tiles<bf16, 32>(b, s);
    }
    const dim3 grid(ceil_div(a.max_len, 32), a.kv.Hkv, a.kv.n_seqs);
    if (a.kv.dtype == kF32)
        score_rows_kernel<float><<<grid, 256, 0, s>>>(b);
    else
        score_rows_kernel<bf16><<<grid, 256, 0, s>>>(b);
    return hipGetLastError();
}

}  // namespace rpo
