// A paged cache outside a batch: new tokens into pages, and the eviction of the tokens that have received the least
// attention weight.
//
//  * append_kernel: rows of keys and values to the last slots of their sequences.  A workgroup takes the eight slots of one
//    octet, in which a page keeps its values, so that a full octet leaves as one 16- or 32-byte unit per channel.
//  * evict_select_kernel: which slots stay, per (sequence, KV head): the radix select of the budget's last score, then one
//    pass that lists the slots in order.
//  * evict_move_kernel: the kept tokens' keys and values to the first slots of other pages.
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
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(PagedAppendArgs a, bool wide) {
    const PagedKv& kv = a.kv;
    const int s = blockIdx.y;
    const ChunkRows c = chunk_rows(kv, a.cu, s, a.n_rows, a.max_new);
    const int from = max(c.slot0, 0), to = min(c.slot0 + c.n, kv.table_stride << kv.shift);  // slots written
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
// -0 equal to 0).  Three passes of 11, 11 and 10 bits find the bits of the last score that the budget has room for; integer
// counts alone decide, so the result does not depend on any order.  Thread t owns the t-th stretch of the slots, so that one
// scan over the threads gives every stretch the number of ties and of kept slots before it.
// ---------------------------------------------------------------------------
constexpr int kSelThreads = 1024;

__device__ inline uint32_t rank_bits(float x) {
    if (x != x) return 0;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// exclusive sums of two counts over the threads of the workgroup
__device__ inline int2 scan_pairs(int2 v, int2* part) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int2 inc = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(inc.x, o, 64), y = __shfl_up(inc.y, o, 64);
        if (lane >= o) inc.x += x, inc.y += y;
    }
    if (lane == 63) part[wave] = inc;
    __syncthreads();
    int2 base = {0, 0};
    for (int w = 0; w < wave; ++w) base.x += part[w].x, base.y += part[w].y;
    __syncthreads();
    return {base.x + inc.x - v.x, base.y + inc.y - v.y};
}

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(PagedEvictArgs a) {
    __shared__ int hist[2048];
    __shared__ int2 part[kSelThreads / 64];
    __shared__ int pick[2];
    const int tid = threadIdx.x, h = blockIdx.x, s = blockIdx.y;
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
    int need = a.budget - a.sinks - a.recent;   // 0 <= need < m1 - m0
    uint32_t prefix = 0;
    int done = 0;  // leading bits of the threshold known
    if (need > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int bits = pass < 2 ? 11 : 10, shift = 32 - done - bits;
            for (int i = tid; i < 2048; i += kSelThreads) hist[i] = 0;
            __syncthreads();
            for (int j = m0 + tid; j < m1; j += kSelThreads) {
                const uint32_t key = rank_bits(score[j]);
                if (done == 0 || (key >> (32 - done)) == prefix) atomicAdd(&hist[(key >> shift) & ((1 << bits) - 1)], 1);
            }
            __syncthreads();
            // from the highest bin down: the bin in which the need-th score lies.  Thread t holds bins 2047 - 2 t and
            // 2046 - 2 t, so that sums over the threads before it are sums over the bins above.
            const int hi = hist[2047 - 2 * tid], lo = hist[2046 - 2 * tid];
            const int before = scan_pairs({hi + lo, 0}, part).x;
            if (before < need && need <= before + hi + lo) {
                const bool first = need <= before + hi;
                pick[0] = first ? 2047 - 2 * tid : 2046 - 2 * tid;
                pick[1] = first ? before : before + hi;
            }
            __syncthreads();
            prefix = (prefix << bits) | (uint32_t)pick[0];
            need -= pick[1];
            done += bits;
            __syncthreads();
        }
    }
    // prefix: the threshold; need: how many of the slots at it stay, the lowest ones
    const bool any = a.budget > a.sinks + a.recent;
    const int per = (L + kSelThreads - 1) / kSelThreads;
    const int j0 = min(tid * per, L), j1 = min(j0 + per, L);
    int2 cnt = {0, 0};  // kept for sure, at the threshold
    for (int j = j0; j < j1; ++j) {
        if (j < m0 || j >= m1) {
            ++cnt.x;
        } else if (any) {
            const uint32_t key = rank_bits(score[j]);
            cnt.x += key > prefix;
            cnt.y += key == prefix;
        }
    }
    const int2 base = scan_pairs(cnt, part);
    int ties = base.y, at = base.x + min(base.y, need);
    for (int j = j0; j < j1; ++j) {
        bool keep = j < m0 || j >= m1;
        if (!keep && any) {
            const uint32_t key = rank_bits(score[j]);
            keep = key > prefix || (key == prefix && ties++ < need);
        }
        if (keep) {
            kept[at] = j;
            if (score_out) score_out[at] = score[j];
            ++at;
        }
    }
}

// ---------------------------------------------------------------------------
// move: a workgroup takes 64 new slots of one KV head.  Keys row by row in 16-byte pieces; a thread collects a channel's
// eight values from as many octets (kept slots are neighbours often enough that they share lines).
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
    evict_select_kernel<<<dim3(a.src.Hkv, a.src.n_seqs), kSelThreads, 0, s>>>(a);
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
