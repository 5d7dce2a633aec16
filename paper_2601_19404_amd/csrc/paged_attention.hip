// Attention over a paged cache outside a batch, with a sliding window and sinks, and the attention weight that every cached
// token receives.
//
// Row i of a sequence's chunk sits at slot t = slot0 + i and sees the slots j <= t of which j < sinks or j > t - window.
//   out = sum_j p_j v_j,  p_j = exp(scale q.k_j - lse),  lse = ln sum_j exp(scale q.k_j)
// A row that sees nothing leaves zeros and an lse of -infinity.
//
//  * attn_rows_kernel: one wave per (row, query head), any head_dim.
//  * score_rows_kernel: one workgroup per 32 tokens of a KV head, any head_dim.
#include "kernels.hpp"

namespace rpo {

namespace {

// Whether a row at slot t sees slot j.
__device__ inline bool sees(int t, int j, int window, int sinks) {
    return j <= t && (window == 0 || j < sinks || t - j < window);
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
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    T* out = (T*)a.out + row * a.out_stride + (int64_t)hq * dh;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int d = lane + 64 * u;
        if (d < dh) out[d] = from_f32<T>(o[u] * inv);
    }
    if (a.lse && lane == 0) a.lse[row * a.Hq + hq] = l > 0.f ? m + logf(l) : -INFINITY;
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
    const int len = (int)min((int64_t)kv.length(s), b.score_stride);
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

}  // namespace

size_t paged_attn_ws_bytes(const PagedAttnArgs&) { return 0; }
size_t paged_score_ws_bytes(const PagedScoreArgs&) { return 0; }

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
    if (a.n_rows <= 0 || a.kv.n_seqs <= 0 || a.max_new <= 0) return hipSuccess;
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
    const dim3 grid(ceil_div(a.max_len, 32), a.kv.Hkv, a.kv.n_seqs);
    if (a.kv.dtype == kF32)
        score_rows_kernel<float><<<grid, 256, 0, s>>>(b);
    else
        score_rows_kernel<bf16><<<grid, 256, 0, s>>>(b);
    return hipGetLastError();
}

}  // namespace rpo
