// A paged cache outside a batch: new tokens into pages, and the eviction of the tokens that have received the least
// attention weight.
//
//  * append_kernel: rows of keys and values to the last slots of their sequences.  A workgroup takes the eight slots of one
//    octet, in which a page keeps its values, so that a full octet leaves as one 16- or 32-byte unit per channel.
//  * evict_select_kernel: which slots stay, per (sequence, KV head): a search for the score of the last one that the budget
//    has room for, then one pass that lists the slots in order.
//  * evict_move_kernel: the kept tokens' keys and values to the first slots of other pages.
#include <algorithm>

#include "kernels.hpp"

namespace rpo {

namespace {

template <typename T>
struct alignas(sizeof(T) * 8) Octet {  // one channel of eight tokens: what a page keeps together
    T t[8];
};

// ---------------------------------------------------------------------------
// append: bytes only.  Row by row the keys move in 16-byte pieces; a thread collects a channel's eight values, the lanes of
// a wave reading neighbouring channels of a row.  Octets that the chunk covers in part are written value by value.
// Bound by memory: 4 x 4352 rows of 7B heads in 13.6 us, 5.2 TB/s; a decode step's 512 rows in 4 us by the launch.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(PagedAppendArgs a, bool wide) {
    const PagedKv& kv = a.kv;
    const int s = blockIdx.y;
    // A row's slot counts from the length as it is given: beyond the table's end there is none.
    ChunkRows c = chunk_rows(kv, a.cu, s, a.n_rows, a.max_new);
    const int cap = kv.table_stride << kv.shift;
    c.slot0 += max(kv.len[s], 0) - kv.length(s);
    const int from = max(c.slot0, 0), to = min(c.slot0 + c.n, cap);  // slots written
    if (from >= to) return;
    const int slot8 = ((from >> 3) + (int)blockIdx.x) * 8;                                    // an octet lies in one page
    const int lo = max(from, slot8), hi = min(to, slot8 + 8);
    if (lo >= hi) return;
    const int page = kv.page(s, slot8);
    if (page < 0) return;
    const int dh = kv.dh, width = kv.Hkv * dh, mask = (1 << kv.shift) - 1;
    T* pool = (T*)kv.pool;
    const T* k = (const T*)a.k;
    const T* v = (const T*)a.v;
    const int64_t row = c.row0 - (int64_t)c.slot0;  // + slot: row of the arrays
    constexpr int kPiece = 16 / sizeof(T);
    if (wide) {
        const int ppr = width / kPiece;
        for (int i = threadIdx.x; i < (hi - lo) * ppr; i += 256) {
            const int slot = lo + i / ppr, x = (i % ppr) * kPiece;
            *(u32x4_t*)(pool + kv.k_at(page, x / dh) + (int64_t)(slot & mask) * dh + x % dh) =
                *(const u32x4_t*)(k + (row + slot) * a.k_stride + x);
        }
    } else {
        for (int i = threadIdx.x; i < (hi - lo) * width; i += 256) {
            const int slot = lo + i / width, x = i % width;
            pool[kv.k_at(page, x / dh) + (int64_t)(slot & mask) * dh + x % dh] = k[(row + slot) * a.k_stride + x];
        }
    }
    for (int x = threadIdx.x; x < width; x += 256) {
        Octet<T>* dst = (Octet<T>*)(pool + kv.v_at(page, x / dh)) + (int64_t)((slot8 & mask) >> 3) * dh + x % dh;
        Octet<T> o;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (slot8 + e >= lo && slot8 + e < hi) o.t[e] = v[(row + slot8 + e) * a.v_stride + x];
        if (hi - lo == 8) {
            *dst = o;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (slot8 + e >= lo && slot8 + e < hi) dst->t[e] = o.t[e];
        }
    }
}

// ---------------------------------------------------------------------------
// select.  A score's rank is that of its bits, turned so that unsigned order is the order of the numbers (NaN lowest,
// -0 equal to 0).  The rank of the last score that the budget has room for lies between the lowest and the highest one; a
// histogram over 2048 equal parts of that range says in which part, and so on until the part is one rank or stays as a
// whole: three passes at most.  (Fixed digits of the rank gather most scores in a few counters, those of the exponents that
// occur.)  Integer counts alone decide, so the result does not depend on any order.
// A wave owns a stretch of the slots, 64 side by side at a time, and counts with ballots.  EACH > 0: that many times 64, which
// stay in registers; 0: longer rows are read again for every pass.
// What bounds it is one CU's time for a row: a row of 16384 takes 14 us (fixed digits, a stretch of slots per thread and the
// row read for every pass: 33), 128 rows of 2100 8 us.
// ---------------------------------------------------------------------------
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64, kBins = 2048;

constexpr uint32_t kAlways = ~0u;

__device__ inline uint32_t rank_bits(float x) {
    if (x != x) return 1;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// exclusive sum over the threads of the workgroup
__device__ inline int scan(int v, int* part) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(inc, o, 64);
        if (lane >= o) inc += x;
    }
    if (lane == 63) part[wave] = inc;
    __syncthreads();
    int base = 0;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) base += w < wave ? part[w] : 0;
    return base + inc - v;
}

template <int EACH>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(PagedEvictArgs a) {
    __shared__ int hist[kBins];
    __shared__ int part[kSelWaves], more[kSelWaves];
    __shared__ uint32_t ends[2][kSelWaves];
    __shared__ int pick[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = blockIdx.x, s = blockIdx.y;
    const int64_t row = (int64_t)s * a.src.Hkv + h;
    const float* score = a.score + row * a.score_stride;
    float* score_out = a.score_out ? a.score_out + row * a.score_out_stride : nullptr;
    int32_t* kept = a.kept + row * a.budget;
    const int L = (int)min((int64_t)a.src.length(s), a.score_stride);
    const int held = min(L, a.budget);
    for (int i = held + tid; i < a.budget; i += kSelThreads) kept[i] = -1;
    if (score_out)
        for (int64_t i = held + tid; i < a.score_out_stride; i += kSelThreads) score_out[i] = 0.f;
    if (L <= a.budget) {
        for (int i = tid; i < L; i += kSelThreads) {
            kept[i] = i;
            if (score_out) score_out[i] = score[i];
        }
        return;
    }
    const int m0 = a.sinks, m1 = L - a.recent;  // the slots that compete
    constexpr int kBlock = EACH ? EACH : 16;    // scores asked for at once
    const int per = EACH ? EACH : (L + kSelThreads - 1) / kSelThreads;
    const int j0 = wave * per * 64 + lane;      // a lane's e-th slot: j0 + 64 e
    // ranks: 0 beyond the row, ~0 for the slots that stay whatever their score, both outside what scores can have
    float v[kBlock];
    uint32_t rank[kBlock];
    auto fetch = [&](int e0) {
#pragma unroll
        for (int e = 0; e < kBlock; ++e) v[e] = e0 + e < per && j0 + 64 * (e0 + e) < L ? score[j0 + 64 * (e0 + e)] : 0.f;
#pragma unroll
        for (int e = 0; e < kBlock; ++e) {
            const int j = j0 + 64 * (e0 + e);
            rank[e] = e0 + e >= per || j >= L ? 0 : j < m0 || j >= m1 ? kAlways : rank_bits(v[e]);
        }
    };
    if constexpr (EACH > 0) fetch(0);
    auto each = [&](auto f) {  // f(slot, rank, score), all lanes together
        for (int e0 = 0; e0 < (EACH ? 1 : per); e0 += kBlock) {
            if constexpr (EACH == 0) fetch(e0);
#pragma unroll
            for (int e = 0; e < kBlock; ++e) f(j0 + 64 * (e0 + e), rank[e], v[e]);
        }
    };
    int need = a.budget - a.sinks - a.recent;  // 0 <= need < m1 - m0
    uint32_t lo = kAlways - 1, hi = 0;  // of the ranks that compete; in the end the rank of the last one kept
    if (need > 0) {
        for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
        each([&](int, uint32_t k, float) {
            if (k - 1 < kAlways - 1) lo = min(lo, k), hi = max(hi, k);
        });
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64)), hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
        if (lane == 0) ends[0][wave] = lo, ends[1][wave] = hi;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSelWaves; ++w) lo = min(lo, ends[0][w]), hi = max(hi, ends[1][w]);
        while (lo < hi) {  // uniform; the range shrinks to a 2048th each time
            const int shift = max(0, 32 - 11 - __builtin_clz(hi - lo));
            each([&](int, uint32_t k, float) {
                if (k - lo <= hi - lo) atomicAdd(&hist[(k - lo) >> shift], 1);
            });
            __syncthreads();
            // from the highest bin down: the bin in which the need-th score lies.  Thread t holds bins 2047 - 2 t and
            // 2046 - 2 t, so that sums over the threads before it are sums over the bins above.
            const int up = hist[kBins - 1 - 2 * tid], down = hist[kBins - 2 - 2 * tid];
            hist[kBins - 1 - 2 * tid] = hist[kBins - 2 - 2 * tid] = 0;
            const int before = scan(up + down, part);
            if (before < need && need <= before + up + down) {
                const bool first = need <= before + up;
                pick[0] = first ? kBins - 1 - 2 * tid : kBins - 2 - 2 * tid;
                pick[1] = first ? before : before + up;
                pick[2] = first ? up : down;
            }
            __syncthreads();
            need -= pick[1];
            lo += (uint32_t)pick[0] << shift;
            if (need == pick[2]) {  // the whole part stays: everything above the rank before it
                --lo, need = 0;
                break;
            }
            hi = min(hi, lo + ((1u << shift) - 1));
        }
    }
    // lo: the threshold; need: how many of the slots at it stay, the lowest ones.  Every wave counts what it keeps for sure
    // and what lies at the threshold, then places its own behind those of the waves before it.
    int n_sure = 0, n_tied = 0;
    each([&](int, uint32_t k, float) {
        n_sure += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k > lo));
        n_tied += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k == lo));
    });
    __syncthreads();
    if (lane == 0) part[wave] = n_sure, more[wave] = n_tied;
    __syncthreads();
    int at = 0, ties = 0;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) at += w < wave ? part[w] : 0, ties += w < wave ? more[w] : 0;
    at += min(ties, need);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    each([&](int j, uint32_t k, float x) {
        const uint64_t t = __builtin_amdgcn_ballot_w64(k == lo);
        const bool keep = k > lo || (k == lo && ties + __builtin_popcountll(t & below) < need);
        const uint64_t m = __builtin_amdgcn_ballot_w64(keep);
        const int to = at + __builtin_popcountll(m & below);
        if (keep) {
            kept[to] = j;
            if (score_out) score_out[to] = x;
        }
        at += __builtin_popcountll(m);
        ties += __builtin_popcountll(t);
    });
}

// ---------------------------------------------------------------------------
// move: a workgroup takes 64 new slots of one KV head.  Keys row by row in 16-byte pieces; a thread collects a channel's
// eight values from as many octets (kept slots are neighbours often enough that they share lines).
// Bound by memory: half of 64 x 2100 tokens of 1.5B heads in 31 us; the octets of the values are read almost whole, so that
// 170 MB move where 136 would do: 5.5 TB/s.  (Four pieces of a thread in flight at once: 31 us as well.)
// ---------------------------------------------------------------------------
constexpr int kMoveSlots = 64;

template <typename T>
__global__ __launch_bounds__(256) void evict_move_kernel(PagedEvictArgs a, bool wide) {
    __shared__ int64_t from_k[kMoveSlots], from_v[kMoveSlots];  // element offsets in the source, -1: nothing
    const int tid = threadIdx.x, h = blockIdx.y, s = blockIdx.z, i0 = blockIdx.x * kMoveSlots;
    const int dh = a.src.dh;
    if (blockIdx.x == 0 && h == 0 && tid == 0)
        a.len_out[s] = (int)min(min((int64_t)a.src.length(s), a.score_stride), (int64_t)a.budget);
    if (tid < kMoveSlots) {
        int64_t k = -1, v = -1;
        const int j = i0 + tid < a.budget ? a.kept[((int64_t)s * a.src.Hkv + h) * a.budget + i0 + tid] : -1;
        const int page = j >= 0 ? a.src.page(s, j) : -1;
        if (page >= 0) {
            const int at = j & ((1 << a.src.shift) - 1);
            k = a.src.k_at(page, h) + (int64_t)at * dh;
            v = a.src.v_at(page, h) + (int64_t)(at >> 3) * dh * 8 + (at & 7);
        }
        from_k[tid] = k;
        from_v[tid] = v;
    }
    __syncthreads();
    const T* src = (const T*)a.src.pool;
    T* dst = (T*)a.dst.pool;
    const int mask = (1 << a.dst.shift) - 1, n = min(kMoveSlots, a.budget - i0);
    constexpr int kPiece = 16 / sizeof(T);
    const int unit = wide ? kPiece : 1, upr = dh / unit;
    for (int x = tid; x < n * upr; x += 256) {
        const int i = x / upr, d = (x % upr) * unit;
        if (from_k[i] < 0) continue;
        const int page = a.dst.page(s, i0 + i);
        if (page < 0) continue;
        T* to = dst + a.dst.k_at(page, h) + (int64_t)((i0 + i) & mask) * dh + d;
        if (wide)
            *(u32x4_t*)to = *(const u32x4_t*)(src + from_k[i] + d);
        else
            *to = src[from_k[i] + d];
    }
    for (int x = tid; x < (n + 7) / 8 * dh; x += 256) {
        const int i = x / dh * 8, d = x % dh;
        const int page = a.dst.page(s, i0 + i);
        if (page < 0) continue;
        Octet<T> o;
        int have = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t f = from_v[i + e];
            if (f >= 0) o.t[e] = src[f + (int64_t)d * 8], have |= 1 << e;
        }
        Octet<T>* to = (Octet<T>*)(dst + a.dst.v_at(page, h)) + (int64_t)(((i0 + i) & mask) >> 3) * dh + d;
        if (have == 255) {
            *to = o;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (have >> e & 1) to->t[e] = o.t[e];
        }
    }
}

bool aligned16(const void* p, int64_t stride, int dtype) {
    return (uintptr_t)p % 16 == 0 && stride * (int64_t)dtype_size(dtype) % 16 == 0;
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t s) {
    if (a.n_rows <= 0 || a.kv.n_seqs <= 0 || a.max_new <= 0) return hipSuccess;
    // 16-byte pieces of a key row must not leave its head
    const bool wide = aligned16(a.k, a.k_stride, a.kv.dtype) && a.kv.dh * dtype_size(a.kv.dtype) % 16 == 0;
    const dim3 grid((a.max_new + 6) / 8 + 1, a.kv.n_seqs);  // octets that max_new slots can touch
    if (a.kv.dtype == kF32)
        append_kernel<float><<<grid, 256, 0, s>>>(a, wide);
    else
        append_kernel<bf16><<<grid, 256, 0, s>>>(a, wide);
    return hipGetLastError();
}

hipError_t launch_paged_evict(const PagedEvictArgs& a, hipStream_t s) {
    if (a.src.n_seqs <= 0) return hipSuccess;
    const int64_t longest = std::min(a.score_stride, (int64_t)a.src.table_stride << a.src.shift);
    auto select = longest <= 4 * kSelThreads    ? evict_select_kernel<4>
                  : longest <= 16 * kSelThreads ? evict_select_kernel<16>
                  : longest <= 32 * kSelThreads ? evict_select_kernel<32>
                                                : evict_select_kernel<0>;
    select<<<dim3(a.src.Hkv, a.src.n_seqs), kSelThreads, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const bool wide = a.src.dh * dtype_size(a.src.dtype) % 16 == 0;
    const dim3 grid(ceil_div(a.budget, kMoveSlots), a.src.Hkv, a.src.n_seqs);
    if (a.src.dtype == kF32)
        evict_move_kernel<float><<<grid, 256, 0, s>>>(a, wide);
    else
        evict_move_kernel<bf16><<<grid, 256, 0, s>>>(a, wide);
    return hipGetLastError();
}

}  // namespace rpo
