// Scores of token ids: log probability, entropy, rank and top alternatives of every row of logits, and the gradient.
//
// With m the row's largest logit, a the scale, d_j = a (x_j - m) <= 0:  s = sum exp d,  u = sum d exp d,
//   lse = a m + ln s,   ln p_t = d_t - ln s,   entropy = ln s - u / s.
// Nothing cancels: ln s >= 0 and -u / s >= 0.
#pragma once
#include "tt_host.cuh"
#include <cuda_bf16.h>
#include <cuda_fp16.h>

constexpr int SCORE_THREADS = 256;
constexpr int SCORE_TOP_MAX = 32;
// Below this d the exponential is 0 in 32 bits; it stands for -inf where d is a factor of a product with it.
constexpr float SCORE_LOW = -1000.0f;

struct ScoreParams {
    const void* logits;
    unsigned long long n_rows, stride;
    u32 n_vocab, top_k;
    float scale;
    const int32_t* ids;
    const long long* ids_off;      // null: row i is asked for ids[i]
    unsigned long long n_docs;
    float* logprob; float* lse; float* entropy; int32_t* rank; int32_t* top_ids; float* top_lp;
    int32_t* status_out;
};

struct ScoreGradParams {
    const void* logits;
    unsigned long long n_rows, stride, grad_stride;
    u32 n_vocab;
    float scale;
    const int32_t* ids;
    const long long* ids_off;
    unsigned long long n_docs;
    const float* lse; const float* entropy; const float* g; const float* h;
    void* grad;
    int32_t* status_out;
};

__device__ __forceinline__ float score_f32(float x) { return x; }
__device__ __forceinline__ float score_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float score_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void score_put(float* p, float v) { *p = v; }
__device__ __forceinline__ void score_put(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void score_put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// The status of the call, by one CTA: the offsets, and the ids that rows are asked for.
template <int NT>
__device__ void score_check(const int32_t* ids, unsigned long long n_rows, u32 n_vocab, const long long* off, unsigned long long n_docs, int32_t* status_out) {
    bool bad_off = false, bad_id = false;
    unsigned long long total = n_rows;
    if (off) {
        const long long t = __ldcg(off + n_docs);
        for (unsigned long long d = threadIdx.x; d < n_docs; d += NT) bad_off |= __ldcg(off + d) > __ldcg(off + d + 1);
        bad_off |= __ldcg(off) != 0 || t < 0;
        if (t > 0 && (unsigned long long)t > n_rows) { if (threadIdx.x == 0) *status_out = 5 /* TT_ERR_CAPACITY */; return; }
        total = t < 0 ? 0 : (unsigned long long)t;
    }
    if (__syncthreads_or(bad_off)) { if (threadIdx.x == 0) *status_out = 1 /* TT_ERR_ARG */; return; }
    // the first id of a document is asked for by no row: of the others, each that is out of range counts
    for (unsigned long long i = threadIdx.x; i < total; i += NT) {
        const int32_t id = __ldcg(ids + i);
        if (off ? (u32)id < n_vocab : id < (long long)n_vocab) continue;
        bool asked = true;
        if (off) {
            unsigned long long lo = 0, hi = n_docs;                    // is i the beginning of a document?
            while (lo < hi) { const unsigned long long mid = (lo + hi) / 2; if (__ldcg(off + mid) < (long long)i) lo = mid + 1; else hi = mid; }
            asked = __ldcg(off + lo) != (long long)i;
        }
        bad_id |= asked;
    }
    if (__syncthreads_or(bad_id)) { if (threadIdx.x == 0) *status_out = 8 /* TT_ERR_BAD_IDS */; }
    else if (threadIdx.x == 0) *status_out = 0;
}

// The id that row i is asked for, -1 for none; in_use = false: the row is behind the last document.
__device__ __forceinline__ int32_t score_target(const int32_t* ids, unsigned long long n_rows, u32 n_vocab, const long long* off, unsigned long long n_docs, unsigned long long i, bool& in_use) {
    unsigned long long at = i;
    in_use = true;
    if (off) {
        const long long total = __ldcg(off + n_docs);
        in_use = total <= (long long)n_rows && (long long)i < total;
        if (!in_use || (long long)(i + 1) >= total) return -1;
        unsigned long long lo = 0, hi = n_docs;                        // the first offset behind i
        while (lo < hi) { const unsigned long long mid = (lo + hi) / 2; if (__ldcg(off + mid) <= (long long)i) lo = mid + 1; else hi = mid; }
        if (__ldcg(off + lo) == (long long)(i + 1)) return -1;         // token i ends its document
        at = i + 1;
    }
    const int32_t id = __ldcg(ids + at);
    return id >= 0 && (u32)id < n_vocab ? id : -1;
}

template <int NT>
__device__ __forceinline__ float cta_sum(float x, float* buf) {
    __syncthreads();
    buf[threadIdx.x] = x;
    __syncthreads();
    for (int o = NT / 2; o; o >>= 1) { if ((int)threadIdx.x < o) buf[threadIdx.x] += buf[threadIdx.x + o]; __syncthreads(); }
    return buf[0];
}
// A logit in the order of the entries: larger logits have larger keys, of equal ones the lower index; never 0.
__device__ __forceinline__ u64 score_key(float x, u32 j) {
    const u32 b = __float_as_uint(x + 0.0f);
    return (u64)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (u32)~j;
}

// A CTA a row, one pass for the maximum, one for the sums, one for each alternative.
template <typename T>
__global__ void __launch_bounds__(SCORE_THREADS)
k_logprobs(const __grid_constant__ ScoreParams P) {
    __shared__ float buf[SCORE_THREADS];
    __shared__ u64 keys[SCORE_THREADS];
    cudaGridDependencySynchronize();
    if (blockIdx.x == P.n_rows) { score_check<SCORE_THREADS>(P.ids, P.n_rows, P.n_vocab, P.ids_off, P.n_docs, P.status_out); return; }
    const unsigned long long row = blockIdx.x;
    const T* x = reinterpret_cast<const T*>(P.logits) + row * P.stride;
    bool in_use;
    const int32_t t = score_target(P.ids, P.n_rows, P.n_vocab, P.ids_off, P.n_docs, row, in_use);
    if (!in_use) return;
    const int tid = threadIdx.x;
    const auto first = [&](u64 below) {                                // the first entry behind the one with key `below`
        u64 best = 0;
        for (u32 j = tid; j < P.n_vocab; j += SCORE_THREADS) { const u64 k = score_key(score_f32(x[j]), j); if (k < below && k > best) best = k; }
        __syncthreads();
        keys[tid] = best;
        __syncthreads();
        for (int o = SCORE_THREADS / 2; o; o >>= 1) { if (tid < o && keys[tid + o] > keys[tid]) keys[tid] = keys[tid + o]; __syncthreads(); }
        return keys[0];
    };
    float m = -INFINITY;
    for (u32 j = tid; j < P.n_vocab; j += SCORE_THREADS) m = fmaxf(m, score_f32(x[j]));
    buf[tid] = m;
    __syncthreads();
    for (int o = SCORE_THREADS / 2; o; o >>= 1) { if (tid < o) buf[tid] = fmaxf(buf[tid], buf[tid + o]); __syncthreads(); }
    m = buf[0];
    const bool nothing = m == -INFINITY;
    const float ref = nothing ? 0.0f : m, xt = t >= 0 ? score_f32(x[t]) : 0.0f;
    float s = 0, u = 0;
    u32 before = 0;
    for (u32 j = tid; j < P.n_vocab; j += SCORE_THREADS) {
        const float v = score_f32(x[j]), d = P.scale * (v - ref), e = expf(d);
        s += e; u += e * fmaxf(d, SCORE_LOW);
        before += v > xt || (v == xt && (int32_t)j < t);
    }
    s = cta_sum<SCORE_THREADS>(s, buf);
    u = cta_sum<SCORE_THREADS>(u, buf);
    u32 rank = 0;
    {
        u32 w = before;
        for (int o = 16; o; o >>= 1) w += __shfl_xor_sync(0xFFFFFFFFu, w, o);
        __syncthreads();
        if ((tid & 31) == 0) buf[tid >> 5] = __uint_as_float(w);
        __syncthreads();
        for (int w2 = 0; w2 < SCORE_THREADS / 32; w2++) rank += __float_as_uint(buf[w2]);
    }
    const bool bad = s != s;
    const float ls = logf(s);
    if (tid == 0) {
        P.logprob[row] = t < 0 ? 0.0f : bad ? s : nothing ? -INFINITY : P.scale * (xt - m) - ls;
        if (P.lse) P.lse[row] = bad ? s : nothing ? -INFINITY : P.scale * m + ls;
        if (P.entropy) P.entropy[row] = bad ? s : nothing ? 0.0f : ls - u / s;
        if (P.rank) P.rank[row] = t < 0 || bad ? 0 : (int32_t)(rank + 1);
    }
    u64 below = ~0ull;
    for (u32 k = 0; k < P.top_k; k++) {
        if (!bad) below = first(below);
        if (tid == 0) {
            const u32 j = ~(u32)below;
            P.top_ids[row * P.top_k + k] = bad ? -1 : (int32_t)j;
            P.top_lp[row * P.top_k + k] = bad ? s : nothing ? -INFINITY : P.scale * (score_f32(x[j]) - m) - ls;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(SCORE_THREADS)
k_logprobs_grad(const __grid_constant__ ScoreGradParams P) {
    cudaGridDependencySynchronize();
    if (blockIdx.x == P.n_rows) { score_check<SCORE_THREADS>(P.ids, P.n_rows, P.n_vocab, P.ids_off, P.n_docs, P.status_out); return; }
    const unsigned long long row = blockIdx.x;
    bool in_use;
    const int32_t t = score_target(P.ids, P.n_rows, P.n_vocab, P.ids_off, P.n_docs, row, in_use);
    if (!in_use) return;
    const T* x = reinterpret_cast<const T*>(P.logits) + row * P.stride;
    T* dx = reinterpret_cast<T*>(P.grad) + row * P.grad_stride;
    const float lse = P.lse[row], ent = P.h ? P.entropy[row] : 0.0f, g = t < 0 ? 0.0f : P.g[row], h = P.h ? P.h[row] : 0.0f;
    const bool zeros = (g == 0.0f && h == 0.0f) || lse == -INFINITY;
    for (u32 j = threadIdx.x; j < P.n_vocab; j += SCORE_THREADS) {
        float v = 0.0f;
        if (!zeros) {
            const float lp = fmaf(P.scale, score_f32(x[j]), -lse), p = expf(lp);
            v = P.scale * (((int32_t)j == t ? g : 0.0f) - p * fmaf(h, fmaxf(lp, SCORE_LOW) + ent, g));
        }
        score_put(dx + j, v);
    }
}
