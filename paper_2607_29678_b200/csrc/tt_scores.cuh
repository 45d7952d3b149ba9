// Scores of token ids: log probability, entropy, rank and top alternatives of every row of logits, and the gradient.
//
// With m the row's largest logit, a the scale, d_j = a (x_j - m) <= 0:  s = sum exp d,  u = sum d exp d,
//   lse = a m + ln s,   ln p_t = d_t - ln s,   entropy = ln s - u / s.
// ln s >= 0 and -u / s >= 0: nothing cancels.  The kernel takes its sums against m a / ln 2 rounded (see ScoreSum): each of the two is off by up to 2^-5, the
// same for both, which drops out of the entropy but for some 2^-29 of rounding; a sure row's is made 0 where that left less.
#pragma once
#include "tt_host.cuh"
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cstring>

constexpr int SCORE_TOP_MAX = 32;
// Below this d the exponential is 0 in 32 bits; it stands for -inf where d is a factor of a product with it.
constexpr float SCORE_LOW = -1000.0f, SCORE_LOW2 = -1500.0f;       // (of the natural exponential, of powers of two)

struct ScoreParams {
    const void* logits;
    unsigned long long n_rows, stride;
    u32 n_vocab, top_k, log_ctas;  // CTAs of a row: 2^log_ctas
    float scale, scale2;           // scale2 = scale / ln 2
    const int32_t* ids;
    const long long* ids_off;      // null: row i is asked for ids[i]
    unsigned long long n_docs;
    float* logprob; float* lse; float* entropy; int32_t* rank; int32_t* top_ids; float* top_lp;
    int32_t* status_out;
};

struct ScoreGradParams {
    const void* logits;
    unsigned long long n_rows, stride, grad_stride;
    u32 n_vocab, parts, rounds;    // CTAs of a row, batches of each
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
// A logit that is read once.  The 16-bit types are loaded as integers: the loads that
// cuda_fp16.hpp and cuda_bf16.hpp define for them are assembly without `volatile`, which the compiler may take out of the condition it stands under
// (entries behind the last row were read, and now and then lay behind the mapped memory).
__device__ __forceinline__ float score_raw(const float* p) { return __ldcg(p); }
__device__ __forceinline__ __half score_raw(const __half* p) { return __ushort_as_half(__ldcg(reinterpret_cast<const unsigned short*>(p))); }
__device__ __forceinline__ __nv_bfloat16 score_raw(const __nv_bfloat16* p) { return __ushort_as_bfloat16(__ldcg(reinterpret_cast<const unsigned short*>(p))); }
template <typename T> __device__ __forceinline__ float score_ld(const T* p) { return score_f32(score_raw(p)); }
__device__ __forceinline__ void score_put(float* p, float v) { *p = v; }
__device__ __forceinline__ void score_put(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void score_put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// The status of the call, by one CTA (the first, so that it runs beside the rows): the offsets, and the ids that rows are asked for.  Eight loads
// of a thread are on their way at once.
template <int NT>
__device__ void score_check(const int32_t* ids, unsigned long long n_rows, u32 n_vocab, const long long* off, unsigned long long n_docs, int32_t* status_out) {
    constexpr int AT_ONCE = 8;
    bool bad_off = false, bad_id = false;
    unsigned long long total = n_rows;
    if (off) {
        const long long t = __ldcg(off + n_docs);
        if (t > 0 && (unsigned long long)t > n_rows) { if (threadIdx.x == 0) *status_out = 5 /* TT_ERR_CAPACITY */; return; }
        for (unsigned long long d0 = threadIdx.x; d0 < n_docs; d0 += NT * AT_ONCE) {
            long long a[AT_ONCE], b[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; i++) {
                const unsigned long long d = d0 + i * NT;
                a[i] = d < n_docs ? __ldcg(off + d) : 0;
                b[i] = d < n_docs ? __ldcg(off + d + 1) : 0;
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; i++) bad_off |= a[i] > b[i];
        }
        bad_off |= __ldcg(off) != 0 || t < 0;
        total = t < 0 ? 0 : (unsigned long long)t;
    }
    if (__syncthreads_or(bad_off)) { if (threadIdx.x == 0) *status_out = 1 /* TT_ERR_ARG */; return; }
    // the first id of a document is asked for by no row: of the others, each that is out of range counts
    for (unsigned long long i0 = threadIdx.x; i0 < total; i0 += NT * AT_ONCE) {
        int32_t id[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; k++) id[k] = i0 + k * NT < total ? __ldcg(ids + i0 + k * NT) : 0;
        bool any = false;
#pragma unroll
        for (int k = 0; k < AT_ONCE; k++) any |= off ? (u32)id[k] >= n_vocab : id[k] >= (long long)n_vocab;
        if (any && !bad_id) {
            for (int k = 0; k < AT_ONCE; k++) {
                const unsigned long long i = i0 + k * NT;
                if (i >= total) break;
                const int32_t x = __ldcg(ids + i);
                if (off ? (u32)x < n_vocab : x < (long long)n_vocab) continue;
                bool asked = true;
                if (off) {
                    unsigned long long lo = 0, hi = n_docs;            // is i the beginning of a document?
                    while (lo < hi) { const unsigned long long mid = (lo + hi) / 2; if (__ldcg(off + mid) < (long long)i) lo = mid + 1; else hi = mid; }
                    asked = __ldcg(off + lo) != (long long)i;
                }
                bad_id |= asked;
            }
        }
    }
    if (__syncthreads_or(bad_id)) { if (threadIdx.x == 0) *status_out = 8 /* TT_ERR_BAD_IDS */; }
    else if (threadIdx.x == 0) *status_out = 0;
}

// The id that row i is asked for, -1 for none, and its logit; in_use = false: the row is behind the last document.  Called by whole warps: 32
// offsets are looked at in each step of the search (two steps for a thousand documents), while the id and its logit are on their way.
template <typename T>
__device__ __forceinline__ int32_t score_target(const int32_t* ids, unsigned long long n_rows, u32 n_vocab, const long long* off, unsigned long long n_docs, unsigned long long i,
                                                const T* x, bool& in_use, float& xt) {
    const bool shifted = off != nullptr;
    int32_t id = !shifted || i + 1 < n_rows ? __ldcg(ids + i + shifted) : -1;
    if (id < 0 || (u32)id >= n_vocab) id = -1;
    xt = x && id >= 0 ? score_ld(x + id) : INFINITY;
    in_use = true;
    if (shifted) {
        const long long total = __ldcg(off + n_docs);
        long long end = total;                                         // off[hi]
        unsigned long long lo = 0, hi = n_docs;                        // off[lo] <= i < off[hi], if the row is in use
        while (hi - lo > 1) {
            const unsigned long long step = (hi - lo + 31) / 32, at = lo + ((threadIdx.x & 31) + 1) * step;
            const long long o = at >= hi ? end : __ldcg(off + at);
            const u32 k = __ffs(__ballot_sync(0xFFFFFFFFu, at >= hi || o > (long long)i)) - 1;
            end = __shfl_sync(0xFFFFFFFFu, o, k);
            hi = min(hi, lo + (k + 1) * step);
            lo += k * step;
        }
        in_use = total <= (long long)n_rows && (long long)i < total;
        if ((long long)(i + 1) >= total || end == (long long)(i + 1)) id = -1;       // token i ends its document
        if (id < 0) xt = INFINITY;
    }
    return id;
}

// ---- arithmetic on pairs ------------------------------------------------------------------------------------------
// Two floats in a 64-bit register: one instruction for both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float a, float b) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void pair_to(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 pair_add(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 pair_mul(f32x2 a, f32x2 b) { f32x2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 pair_fma(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ float exp2_hw(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

// A 16-byte vector of a type: its values, its largest one, how many of it are below a pivot.
template <typename T> struct ScoreVec;
template <> struct ScoreVec<float> {
    static constexpr int N = 4;
    typedef float Pivot;
    struct Count { u32 n = 0; };
    __device__ static float at(const uint4& r, int e) { return __uint_as_float(e == 0 ? r.x : e == 1 ? r.y : e == 2 ? r.z : r.w); }
    __device__ static f32x2 pair(const uint4& r, int p) { return p == 0 ? pair_of(at(r, 0), at(r, 1)) : pair_of(at(r, 2), at(r, 3)); }
    typedef float Most;
    __device__ static Most most(const uint4& r) { return fmaxf(fmaxf(at(r, 0), at(r, 1)), fmaxf(at(r, 2), at(r, 3))); }
    __device__ static Most larger(Most a, Most b) { return fmaxf(a, b); }
    __device__ static float value(Most m) { return m; }
    __device__ static uint4 lowest() { const u32 w = 0xFF800000u; return make_uint4(w, w, w, w); }
    static constexpr float LOW = -1e37f;                       // stands for lower values and -inf, see `masked`
    __device__ static u32 raised(u32 w) { return __float_as_uint(__uint_as_float(w) < LOW ? LOW : __uint_as_float(w)); }
    __device__ static uint4 raised(const uint4& r) { return make_uint4(raised(r.x), raised(r.y), raised(r.z), raised(r.w)); }
    __device__ static Pivot pivot(float x) { return x; }
    // the next larger value
    __device__ static Pivot above(float x) {
        const u32 b = __float_as_uint(x + 0.0f);
        return __uint_as_float(b == 0 ? 1u : b & 0x80000000u ? b - 1 : b + 1);
    }
    __device__ static void below(Count& c, const uint4& r, Pivot p) {
#pragma unroll
        for (int e = 0; e < N; e++) c.n += at(r, e) < p;
    }
    __device__ static u32 take(Count& c) { const u32 n = c.n; c.n = 0; return n; }
};
// The 16-bit types: a word is two values; counts are sums of 1.0 in the type itself, exact up to 256.
template <typename T2> __device__ __forceinline__ T2 as_two(u32 w) { T2 v; memcpy(&v, &w, 4); return v; }
template <typename T, typename T2, u32 LOWEST, u32 LOWER> struct ScoreVec16 {         // bits of -inf, and of what stands for it
    static constexpr int N = 8;
    typedef T2 Pivot;
    struct Count { T2 n = as_two<T2>(0); };
    __device__ static u32 word(const uint4& r, int p) { return p == 0 ? r.x : p == 1 ? r.y : p == 2 ? r.z : r.w; }
    typedef T2 Most;
    __device__ static Most most(const uint4& r) { return __hmax2(__hmax2(as_two<T2>(r.x), as_two<T2>(r.y)), __hmax2(as_two<T2>(r.z), as_two<T2>(r.w))); }
    __device__ static Most larger(Most a, Most b) { return __hmax2(a, b); }
    __device__ static float value(Most m) { return fmaxf(score_f32(m.x), score_f32(m.y)); }
    __device__ static uint4 lowest() { const u32 w = LOWEST << 16 | LOWEST; return make_uint4(w, w, w, w); }
    __device__ static u32 raised(u32 w) { const T2 v = __hmax2_nan(as_two<T2>(w), as_two<T2>(LOWER << 16 | LOWER)); u32 o; memcpy(&o, &v, 4); return o; }
    __device__ static uint4 raised(const uint4& r) { return make_uint4(raised(r.x), raised(r.y), raised(r.z), raised(r.w)); }
    __device__ static Pivot bits_pivot(u32 h) { return as_two<T2>(h << 16 | h); }
    __device__ static void below(Count& c, const uint4& r, Pivot p) {
#pragma unroll
        for (int i = 0; i < 4; i++) c.n = __hadd2(c.n, __hlt2(as_two<T2>(word(r, i)), p));
    }
    __device__ static u32 take(Count& c) { const u32 n = (u32)(score_f32(c.n.x) + score_f32(c.n.y)); c.n = as_two<T2>(0); return n; }
    __device__ static u32 next_bits(u32 b) { return (b & 0x7FFF) == 0 ? 1u : b & 0x8000 ? b - 1 : b + 1; }
};
template <> struct ScoreVec<__nv_bfloat16> : ScoreVec16<__nv_bfloat16, __nv_bfloat162, 0xFF80u, 0xFCF0u> {
    static constexpr float LOW = -9.969209968386869e36f;       // 0xFCF0
    __device__ static float at(const uint4& r, int e) { const u32 w = word(r, e >> 1); return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16); }
    __device__ static f32x2 pair(const uint4& r, int p) { const u32 w = word(r, p); return pair_of(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    __device__ static u32 bits(float x) { return __float_as_uint(x) >> 16; }
    __device__ static Pivot pivot(float x) { return bits_pivot(bits(x)); }
    __device__ static Pivot above(float x) { return bits_pivot(next_bits(bits(x))); }
};
template <> struct ScoreVec<__half> : ScoreVec16<__half, __half2, 0xFC00u, 0xFBFFu> {
    static constexpr float LOW = -65504.0f;
    __device__ static float at(const uint4& r, int e) { const __half2 h = as_two<__half2>(word(r, e >> 1)); return __half2float(e & 1 ? h.y : h.x); }
    __device__ static f32x2 pair(const uint4& r, int p) { const float2 f = __half22float2(as_two<__half2>(word(r, p))); return pair_of(f.x, f.y); }
    __device__ static u32 bits(float x) { return __half_as_ushort(__float2half_rn(x)); }
    __device__ static Pivot pivot(float x) { return bits_pivot(bits(x)); }
    __device__ static Pivot above(float x) { return bits_pivot(next_bits(bits(x))); }
};

// The order of the entries as a number: larger logits have larger keys, of equal ones the lower index; never 0.
__device__ __forceinline__ u32 score_order(float x) {
    const u32 b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float score_unorder(u32 o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ u64 score_key(float x, u32 j) { return (u64)score_order(x) << 32 | (u32)~j; }

// Largest logit m seen and, relative to it and in powers of two, the sums: s of 2^y, u of y 2^y with y = x c - M, c = scale / ln 2, M = m c
// rounded: one multiply-add a logit.  What the rounding of M leaves, rho = M - m c, takes part in every step from one m to another and in the end, so
// that nothing is lost by it.  Where m c is too large for that (2^20: rho stays below 2^-4), M is a NaN and rho 0: the sums of such a batch are
// NaNs, and it is worked out again as y = (x - m) c - rho, as are batches with a y of -inf (masked logits), whose product with 2^y is a NaN.
// m starts at the lowest number, so that rows of -inf leave s = 0 and no difference of infinities arises.
// A difference (x - m) c is (x / 2 - m / 2) 2 c: x - m may pass 32 bits where its product with a small c does not; both halves (but for
// subnormal numbers, whose distances count at no scale) and 2 c are exact.
struct ScoreSum { float m, s, u; };
constexpr float SCORE_NONE = -3.402823466e38f, SCORE_LARGE = 1048576.0f;
__device__ __forceinline__ float score_ref(float m, float c) { const float M = m * c; return fabsf(M) < SCORE_LARGE ? M : NAN; }
__device__ __forceinline__ float score_rho(float m, float c) { const float M = m * c; return fabsf(M) < SCORE_LARGE ? -fmaf(m, c, -M) : 0.0f; }
__device__ __forceinline__ float score_half(float x, float m) { return fmaf(x, 0.5f, -0.5f * m); }
__device__ __forceinline__ void score_raise(ScoreSum& a, float m, float c) {      // to a reference m >= a.m
    const float y = fmaf(score_half(a.m, m), 2.0f * c, score_rho(a.m, c) - score_rho(m, c)), f = exp2_hw(y);
    a.u = f * fmaf(fmaxf(y, SCORE_LOW2), a.s, a.u);
    a.s *= f;
    a.m = m;
}

// A vector's terms, for any logits.
template <typename V>
__device__ __forceinline__ void score_add(const uint4& r, float m, float c, float rho, float& s, float& u) {
#pragma unroll
    for (int e = 0; e < V::N; e++) {
        const float y = fmaf(score_half(V::at(r, e), m), 2.0f * c, -rho), w = exp2_hw(y);
        s += w;
        u = fmaf(w, fmaxf(y, SCORE_LOW2), u);
    }
}

// A row goes to a cluster of CTAs, a stretch of its 16-byte vectors to each; thread i of a CTA takes every NT-th of them from the i-th on, SCORE_U
// at a time (a batch).  One pass over the row keeps the sums and counts what lies before the row's id.  For the alternatives each thread also
// keeps the largest value among its vectors, the first vector that has it, and the largest value of its other batches.  The top_k-th of the largest
// values of 64 groups of threads, with the end of its vector, is a bound that at least top_k entries reach; what reaches it is then looked up
// again: in the one batch of each thread whose largest value does, and in the whole share of the few threads with a second batch that does.
//   Bound by the bytes of the logits while the clock is high: 4,015 rows of 200,000 bf16 252 us, 6.4 TB/s (98 % of a copy's rate).  A long run of such
// calls meets the power limit; at 1.6 GHz the exponentials (16 a clock and SM: 212 us) and the rest of the arithmetic bound it, 305 us.
//   SCORE_PLACES threads of 80 registers are on an SM at once: with 64 registers, for 1,024 threads, the loop spills (4,096 rows of 100,256 bf16 logits
// with twenty alternatives 252 us, so 173).
constexpr int SCORE_U = 4, SCORE_CAND = 512, SCORE_CLUSTER = 8, SCORE_PLACES = 768;

template <int SCORE_NT>
struct ScoreShared {
    ScoreSum part[SCORE_NT / 32];
    u32 before[SCORE_NT / 32];
    ScoreSum sum;                       // of this CTA
    u32 n_before;
    u64 bound;
    u32 n_cand, n_scan;
    u64 best[SCORE_TOP_MAX];            // of this CTA, in order; 0: it has fewer
    u64 heads[64];
    union {
        u64 keys[SCORE_NT];
        u64 cand[SCORE_CAND];
    };
    u32 scan[SCORE_NT];                 // threads whose whole share is looked up
    u32 first[SCORE_NT];                // the vector of each thread's largest value
    // what the CTAs of a cluster leave with its first one
    ScoreSum all_sum[SCORE_CLUSTER];
    u32 all_before[SCORE_CLUSTER];
    u64 all_best[SCORE_CLUSTER * SCORE_TOP_MAX];
};

// The n distinct keys at `from` in order (0: none), the first k of them to `to`: four threads count what is larger than a key.
template <int SCORE_NT>
__device__ __forceinline__ void score_rank(const u64* from, u32 n, u64* to, u32 k) {
    for (u32 i0 = 0; i0 < n; i0 += SCORE_NT / 4) {
        const u32 i = i0 + threadIdx.x / 4;
        const u64 mine = i < n ? from[i] : 0;
        u32 before = 0;
#pragma unroll 4
        for (u32 o = threadIdx.x % 4; o < n; o += 4) before += from[o] > mine;
        before += __shfl_xor_sync(0xFFFFFFFFu, before, 1);
        before += __shfl_xor_sync(0xFFFFFFFFu, before, 2);
        if (mine && before < k && threadIdx.x % 4 == 0) to[before] = mine;
    }
}

template <typename T, bool TOP, bool RANK, int NT>
__global__ void __launch_bounds__(NT, SCORE_PLACES / NT)
k_logprobs(const __grid_constant__ ScoreParams P) {
    typedef ScoreVec<T> V;
    constexpr int N = V::N, U = SCORE_U, GROUPS = 64;
    __shared__ ScoreShared<NT> sh;
    __shared__ uint4 ring[2][U][NT];
    const u32 ctas = 1u << P.log_ctas, cta = blockIdx.x & (ctas - 1);
    if (ctas > 1) cluster_arrive();                            // (the first CTA's memory may be written once it runs)
    cudaGridDependencySynchronize();
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const unsigned long long row = (unsigned long long)(blockIdx.x >> P.log_ctas) - 1;
    if (blockIdx.x < ctas) {
        if (cta == 0) score_check<NT>(P.ids, P.n_rows, P.n_vocab, P.ids_off, P.n_docs, P.status_out);
        if (ctas > 1) cluster_wait();
        return;
    }
    const T* x = reinterpret_cast<const T*>(P.logits) + row * P.stride;
    // the vectors of the row, between the entries in front of the first 16-byte boundary and those behind the last
    const u32 lead = min(P.n_vocab, (u32)((16 - ((uintptr_t)x & 15)) & 15) / (u32)sizeof(T));
    const u32 n_vec = (P.n_vocab - lead) / N, behind = P.n_vocab - lead - n_vec * N;
    const uint4* vec = reinterpret_cast<const uint4*>(x + lead);
    const u32 v0 = (u32)((u64)n_vec * cta >> P.log_ctas), v1 = (u32)((u64)n_vec * (cta + 1) >> P.log_ctas);
    // Two batches are on their way to the thread's own places in shared memory, so that the loads of one run under the arithmetic of the other (and
    // the first two while the row's id is looked up).
    const auto fetch = [&](u32 stage, u32 v) {                  // (fewer than 2^29 vectors: no sum passes 32 bits)
        if (v + (U - 1) * NT < v1) {
#pragma unroll
            for (int i = 0; i < U; i++) copy_async(&ring[stage][i][tid], vec + v + i * NT);
        } else {
#pragma unroll
            for (int i = 0; i < U; i++) if (v + i * NT < v1) copy_async(&ring[stage][i][tid], vec + v + i * NT);
        }
        copy_commit();
    };
    fetch(0, v0 + tid);
    fetch(1, v0 + tid + U * NT);
    bool in_use;
    float xt;
    const int32_t t = score_target(P.ids, P.n_rows, P.n_vocab, P.ids_off, P.n_docs, row, x, in_use, xt);
    if (!in_use) { copy_wait<0>(); if (ctas > 1) cluster_wait(); return; }
    const float c = P.scale2;
    const f32x2 c2 = pair_of(c, c);
    // entries before the row's id: those not below it in the vectors in front of the id's, those not below the next larger value in the others, and
    // the equal ones in front of it in its own vector, which one thread counts here (by one load: entry by entry it took 2 us)
    const u32 vt = t < (int32_t)lead ? 0 : min(n_vec, ((u32)t - lead) / N);
    ScoreSum a = {SCORE_NONE, 0.0f, 0.0f};
    float ref = NAN;
    u32 n_before = 0;
    if (RANK && tid == NT - 1 && t >= (int32_t)lead && vt >= v0 && vt < v1) {
        const uint4 w = __ldcg(vec + vt);
#pragma unroll
        for (int e = 0; e < N; e++) n_before += lead + vt * N + e < (u32)t && V::at(w, e) == xt;
    }
    float most1 = -INFINITY, most2 = -INFINITY;
    u32 first = v0 + tid;                                      // (of a thread that has vectors; none of -inf alone is passed over)
    const auto top = [&](float bm) {                           // a batch's largest value: does it raise the thread's?
        most2 = fmaxf(most2, fminf(most1, bm));
        const bool up = bm > most1;
        if (up) most1 = bm;
        return up;
    };
    u32 stage = 0, v = v0 + tid;
    bool masked = false;                                       // a batch held masked logits
    for (; v + (U - 1) * NT < v1; v += U * NT, stage ^= 1) {
        copy_wait<1>();
        uint4 r[U];
        typename V::Most vm[U], h;
#pragma unroll
        for (int i = 0; i < U; i++) { r[i] = ring[stage][i][tid]; vm[i] = V::most(r[i]); h = i ? V::larger(h, vm[i]) : vm[i]; }
        const float bm = V::value(h);
        asm volatile("" :: "f"(bm) : "memory");                // (all of the batch is in registers: its place is free)
        fetch(stage, v + 2 * U * NT);
        if (TOP && top(bm)) {
            first = v + (U - 1) * NT;
#pragma unroll
            for (int i = U - 2; i >= 0; i--) if (V::value(vm[i]) == bm) first = v + i * NT;
        }
        if (bm > a.m) { score_raise(a, bm, c); ref = score_ref(bm, c); }
        // Once a thread has met masked logits a low number stands for -inf, whose terms are 0 without a NaN: where the largest logit is far above it, so
        // that its terms are 0, too, and the id's is above it, so that the count below is the same.
        if (masked && score_half(V::LOW, a.m) * (2.0f * c) < SCORE_LOW && xt > V::LOW) {
#pragma unroll
            for (int i = 0; i < U; i++) r[i] = V::raised(r[i]);
        }
        const f32x2 ref2 = pair_of(-ref, -ref);
        f32x2 s2 = pair_of(0.0f, 0.0f), u2 = s2;
#pragma unroll
        for (int i = 0; i < U; i++) {
#pragma unroll
            for (int p = 0; p < N / 2; p++) {
                const f32x2 y = pair_fma(V::pair(r[i], p), c2, ref2);
                float y0, y1;
                pair_to(y, y0, y1);
                const f32x2 e = pair_of(exp2_hw(y0), exp2_hw(y1));
                s2 = pair_add(s2, e);
                u2 = pair_fma(e, y, u2);
            }
        }
        float s0, s1, u0, u1;
        pair_to(s2, s0, s1); pair_to(u2, u0, u1);
        s0 += s1; u0 += u1;
        if (u0 != u0) {                                        // masked logits, or some beyond the range of a product
            masked = true;
            s0 = u0 = 0.0f;
            const float rho = score_rho(a.m, c);
#pragma unroll
            for (int i = 0; i < U; i++) score_add<V>(r[i], a.m, c, rho, s0, u0);
        }
        a.s += s0; a.u += u0;
        if (RANK && bm >= xt) {
            const typename V::Pivot piv0 = V::pivot(xt), piv1 = V::above(xt);
            typename V::Count cnt;
#pragma unroll
            for (int i = 0; i < U; i++) V::below(cnt, r[i], v + i * NT < vt ? piv0 : piv1);
            n_before += U * N - V::take(cnt);
        }
    }
    if (v < v1) {                                              // the last batch, vector by vector
        copy_wait<1>();
        float bm = -INFINITY;
#pragma unroll 1
        for (u32 i = 0, w = v; w < v1; i++, w += NT) {
            const uint4 r = ring[stage][i][tid];
            const float vm = V::value(V::most(r));
            if (TOP && vm > fmaxf(most1, bm)) first = w;
            bm = fmaxf(bm, vm);
            if (vm > a.m) score_raise(a, vm, c);
            score_add<V>(r, a.m, c, score_rho(a.m, c), a.s, a.u);
            if (RANK && vm >= xt) {
                typename V::Count cnt;
                V::below(cnt, r, w < vt ? V::pivot(xt) : V::above(xt));
                n_before += N - V::take(cnt);
            }
        }
        if (TOP) top(bm);
    }
    // the entries outside the vectors
    const u32 loose = cta == 0 ? lead + behind : 0;
    if ((u32)tid < loose) {
        const u32 j = (u32)tid < lead ? tid : n_vec * N + tid;
        const float e = score_ld(x + j);
        if (e > a.m) score_raise(a, e, c);
        const float y = fmaf(score_half(e, a.m), 2.0f * c, -score_rho(a.m, c)), w = exp2_hw(y);
        a.s += w;
        a.u = fmaf(w, fmaxf(y, SCORE_LOW2), a.u);
        if (RANK) n_before += e > xt || (e == xt && (int32_t)j < t);
    }
    // sums of the CTA
    const auto join = [&](ScoreSum& b, u32& nb) {              // over a warp
        float m = b.m;
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        score_raise(b, m, c);
#pragma unroll
        for (int o = 16; o; o >>= 1) { b.s += __shfl_xor_sync(0xFFFFFFFFu, b.s, o); b.u += __shfl_xor_sync(0xFFFFFFFFu, b.u, o); }
        if (RANK) nb = __reduce_add_sync(0xFFFFFFFFu, nb);
    };
    const bool has = v0 + tid < v1;
    join(a, n_before);
    if (lane == 0) { sh.part[wid] = a; sh.before[wid] = n_before; }
    if (TOP) {
        sh.keys[tid] = has ? (u64)score_order(most1) << 32 | (u32)~first : 0;
        sh.first[tid] = first;
        if (tid == 0) { sh.bound = 0; sh.n_cand = 0; sh.n_scan = 0; }
        if (tid < SCORE_TOP_MAX) sh.best[tid] = 0;
    }
    __syncthreads();
    if (wid == NT / 32 - 1) {
        a = lane < NT / 32 ? sh.part[lane] : ScoreSum{SCORE_NONE, 0.0f, 0.0f};
        n_before = lane < NT / 32 ? sh.before[lane] : 0;
        join(a, n_before);
        if (lane == 0) { sh.sum = a; sh.n_before = n_before; }
    }
    if (TOP) {
        // the groups' largest values in order
        if (tid < GROUPS) {
            u64 head = 0;
#pragma unroll
            for (int q = 0; q < NT / GROUPS; q++) head = max(head, sh.keys[tid + q * GROUPS]);
            sh.heads[tid] = head;
        }
        __syncthreads();
        {
            constexpr int S = NT / GROUPS;                     // threads that look for the place of a group's
            const u64 head = sh.heads[tid / S];
            u32 before = 0;
#pragma unroll
            for (int o = 0; o < GROUPS / S; o++) before += sh.heads[tid % S + S * o] > head;
#pragma unroll
            for (int o = 1; o < S; o <<= 1) before += __shfl_xor_sync(0xFFFFFFFFu, before, o);
            if (head && before == P.top_k - 1) sh.bound = score_key(score_unorder((u32)(head >> 32)), lead + ~(u32)head * N + N - 1);
        }
        __syncthreads();
        // (not where there is a NaN; again where more entries reach the bound than there is room for: each time with a bound that fewer reach)
        while (sh.sum.s == sh.sum.s) {
            const u64 bound = sh.bound;
            const u32 bv = (u32)(bound >> 32), bj = ~(u32)bound;
            const auto look = [&](const uint4& r, u32 w) {
                if (score_order(V::value(V::most(r))) < bv) return;
#pragma unroll
                for (int e = 0; e < N; e++) {
                    const u64 key = score_key(V::at(r, e), lead + w * N + e);
                    if (key >= bound) { const u32 n = atomicAdd(&sh.n_cand, 1u); if (n < SCORE_CAND) sh.cand[n] = key; }
                }
            };
            const u32 ov = score_order(most1), b0 = (first - v0 - tid) / (U * NT) * (U * NT) + v0;       // the batch: vectors b0 + tid + i * NT
            const bool hot = has && (bound == 0 || ov > bv || (ov == bv && lead + first * N <= bj));
            // others of this thread's batches: all of them, or, where only entries equal to the bound's are left, those in front of it
            if (hot && (bound == 0 || (score_order(most2) >= bv && (ov > bv || lead + (b0 + U * NT) * N <= bj)))) sh.scan[atomicAdd(&sh.n_scan, 1u)] = tid;
            uint4 r[U];                                        // (on its way while the list becomes complete and is worked off)
#pragma unroll
            for (int i = 0; i < U; i++) r[i] = hot && b0 + tid + i * NT < v1 ? __ldcg(vec + b0 + tid + i * NT) : V::lowest();
            if ((u32)tid < loose) {
                const u32 j = (u32)tid < lead ? tid : n_vec * N + tid;
                const u64 key = score_key(score_ld(x + j), j);
                if (key >= bound) { const u32 n = atomicAdd(&sh.n_cand, 1u); if (n < SCORE_CAND) sh.cand[n] = key; }
            }
            __syncthreads();
            const u32 n_scan = sh.n_scan;
            for (u32 i = wid; i < n_scan; i += NT / 32) {
                const u32 o = sh.scan[i], skip = (sh.first[o] - v0 - o) / (U * NT);
                for (u32 n0 = lane; v0 + o + n0 * NT < v1; n0 += 32 * U) {
                    uint4 q[U];
#pragma unroll
                    for (int k = 0; k < U; k++) { const u32 w = v0 + o + (n0 + 32 * k) * NT; q[k] = w < v1 ? __ldcg(vec + w) : V::lowest(); }
#pragma unroll
                    for (int k = 0; k < U; k++) { const u32 w = v0 + o + (n0 + 32 * k) * NT; if (w < v1 && (n0 + 32 * k) / U != skip) look(q[k], w); }
                }
            }
            if (hot) {
#pragma unroll
                for (int i = 0; i < U; i++) if (b0 + tid + i * NT < v1) look(r[i], b0 + tid + i * NT);
            }
            __syncthreads();
            const u32 n_cand = sh.n_cand;
            score_rank<NT>(sh.cand, min(n_cand, (u32)SCORE_CAND), sh.best, P.top_k);
            __syncthreads();
            if (n_cand <= SCORE_CAND) break;
            if (tid == 0) { sh.bound = sh.best[P.top_k - 1]; sh.n_cand = 0; sh.n_scan = 0; }
            __syncthreads();
        }
    } else __syncthreads();
    // the row's from its CTAs'
    ScoreSum sum = sh.sum;
    n_before = sh.n_before;
    if (ctas > 1) {
        cluster_wait();
        if (tid == 0) {
            const u32 at = cluster_map(&sh.all_sum[cta], 0);
            cluster_put(at, sum.m); cluster_put(at + 4, sum.s); cluster_put(at + 8, sum.u);
            cluster_put(cluster_map(&sh.all_before[cta], 0), __uint_as_float(n_before));
        }
        if (TOP && (u32)tid < P.top_k) cluster_put(cluster_map(&sh.all_best[cta * P.top_k + tid], 0), sh.best[tid]);
        cluster_arrive();
        cluster_wait();
        if (cta != 0) return;
        sum = (u32)lane < ctas ? sh.all_sum[lane] : ScoreSum{SCORE_NONE, 0.0f, 0.0f};
        n_before = (u32)lane < ctas ? sh.all_before[lane] : 0;
        join(sum, n_before);
        if (TOP) { score_rank<NT>(sh.all_best, ctas * P.top_k, sh.best, P.top_k); __syncthreads(); }
    }
    const bool bad = sum.s != sum.s, nothing = sum.s == 0.0f;
    const float ln = logf(sum.s), ls = fmaf(score_rho(sum.m, c), 0.6931471806f, ln);       // ls: relative to m itself
    // (what rounding leaves of a probability of 1 is not above it, and no entropy is below 0)
    const auto log_p = [&](float e) { return bad ? sum.s : nothing ? -INFINITY : fminf(fmaf(score_half(e, sum.m), 2.0f * P.scale, -ls), 0.0f); };
    if (tid == 0) {
        P.logprob[row] = t < 0 ? 0.0f : log_p(xt);
        if (P.lse) P.lse[row] = bad ? sum.s : nothing ? -INFINITY : fmaf(P.scale, sum.m, ls);
        if (P.entropy) P.entropy[row] = bad ? sum.s : nothing ? 0.0f : fmaxf(ln - 0.6931471806f * (sum.u / sum.s), 0.0f);
        if (RANK) P.rank[row] = t < 0 || bad ? 0 : (int32_t)(n_before + 1);
    }
    if (TOP && (u32)tid < P.top_k) {
        const u64 key = sh.best[tid];
        P.top_ids[row * P.top_k + tid] = bad ? -1 : (int32_t)~(u32)key;
        P.top_lp[row * P.top_k + tid] = log_p(score_unorder((u32)(key >> 32)));
    }
}

// The gradient: with L = scale x_j - lse,  dx_j = exp(L) (A + B L) + [j = t] scale g,  A = -scale (g + h entropy), B = -scale h.
// Reads a row once and writes it once; a CTA takes a stretch of SCORE_GRAD_NT * SCORE_U * rounds vectors of a row.  Bound by those bytes: 4,015 rows
// of 200,000 bf16 logits 477-489 us, 6.6-6.7 TB/s (a copy that reads and writes as much: 497); in a long run of calls, at the power limit, 515.
constexpr int SCORE_GRAD_NT = 256;
// -2^60: an lse below it, -inf or rounded to 2^37, does not tell a row's probabilities.  (A row of nothing but the lowest value has such a one in bf16 and fp32, but for scales
// below 2^-67; in fp16 only at scales above 2^44.)
constexpr float SCORE_NOTHING = -1.152921504606847e18f;

struct ScoreGradRow { float scale, lse, A, B, hot; int32_t t; };
__device__ __forceinline__ float score_not_above_0(float x) { float r; asm("min.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(x)); return r; }
template <bool ENT>
__device__ __forceinline__ void score_grad_pair(const ScoreGradRow& R, f32x2 x, float& a, float& b) {
    float l0, l1;
    pair_to(pair_fma(x, pair_of(R.scale, R.scale), pair_of(-R.lse, -R.lse)), l0, l1);
    l0 = score_not_above_0(l0); l1 = score_not_above_0(l1);    // (an lse in the millions is off by more than 1 from rounding alone)
    float y0, y1;
    pair_to(pair_mul(pair_of(l0, l1), pair_of(1.44269504f, 1.44269504f)), y0, y1);
    const f32x2 p = pair_of(exp2_hw(y0), exp2_hw(y1));
    f32x2 f = pair_of(R.A, R.A);
    if (ENT) f = pair_fma(pair_of(R.B, R.B), pair_of(fmaxf(l0, SCORE_LOW), fmaxf(l1, SCORE_LOW)), f);
    pair_to(pair_mul(p, f), a, b);
}
template <bool ENT>
__device__ __forceinline__ float score_grad_one(const ScoreGradRow& R, float x, u32 j) {
    float a, b;
    score_grad_pair<ENT>(R, pair_of(x, x), a, b);
    return (int32_t)j == R.t ? a + R.hot : a;
}
template <typename T> struct ScorePut;
template <> struct ScorePut<float> {
    __device__ static uint4 vec(const float (&v)[4]) { return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])); }
};
template <> struct ScorePut<__nv_bfloat16> {
    __device__ static u32 two(float a, float b) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); u32 w; memcpy(&w, &h, 4); return w; }
    __device__ static uint4 vec(const float (&v)[8]) { return make_uint4(two(v[0], v[1]), two(v[2], v[3]), two(v[4], v[5]), two(v[6], v[7])); }
};
template <> struct ScorePut<__half> {
    __device__ static u32 two(float a, float b) { const __half2 h = __floats2half2_rn(a, b); u32 w; memcpy(&w, &h, 4); return w; }
    __device__ static uint4 vec(const float (&v)[8]) { return make_uint4(two(v[0], v[1]), two(v[2], v[3]), two(v[4], v[5]), two(v[6], v[7])); }
};

template <typename T, bool ENT>
__global__ void __launch_bounds__(SCORE_GRAD_NT, 5)
k_logprobs_grad(const __grid_constant__ ScoreGradParams P) {
    typedef ScoreVec<T> V;
    constexpr int N = V::N, U = SCORE_U, NT = SCORE_GRAD_NT;
    cudaGridDependencySynchronize();
    const unsigned long long row = (blockIdx.x - 1) / P.parts;
    const u32 part = (blockIdx.x - 1) % P.parts, tid = threadIdx.x;
    if (blockIdx.x == 0) { score_check<NT>(P.ids, P.n_rows, P.n_vocab, P.ids_off, P.n_docs, P.status_out); return; }
    const T* x = reinterpret_cast<const T*>(P.logits) + row * P.stride;
    T* dx = reinterpret_cast<T*>(P.grad) + row * P.grad_stride;
    ScoreGradRow R;
    bool in_use;
    float unused;
    R.t = score_target(P.ids, P.n_rows, P.n_vocab, P.ids_off, P.n_docs, row, (const T*)nullptr, in_use, unused);
    if (!in_use) return;
    const float g = R.t < 0 ? 0.0f : __ldcg(P.g + row), h = ENT ? __ldcg(P.h + row) : 0.0f;
    R.lse = __ldcg(P.lse + row);
    R.scale = P.scale; R.A = -P.scale * (ENT ? fmaf(h, __ldcg(P.entropy + row), g) : g); R.B = -P.scale * h; R.hot = P.scale * g;
    const bool zeros = (g == 0.0f && h == 0.0f) || R.lse < SCORE_NOTHING;
    // 16-byte vectors where rows of both lie alike in memory; else the logits are read entry by entry
    const u32 lead = min(P.n_vocab, (u32)((16 - ((uintptr_t)dx & 15)) & 15) / (u32)sizeof(T));
    const u32 n_vec = (P.n_vocab - lead) / N;
    const bool alike = (((uintptr_t)x ^ (uintptr_t)dx) & 15) == 0;
    const u32 share = P.rounds * U * NT;                       // vectors of a CTA
    uint4* out = reinterpret_cast<uint4*>(dx + lead);
    const uint4* in = reinterpret_cast<const uint4*>(x + lead);
    // By way of L1, its lines the first to be replaced: the wait above makes what the kernel before wrote visible there, too, even where this CTA and old lines
    // of the logits were on the SM before they were written.  Past L1 (__ldcg) 1,000 rows of 64 KB with entropies take 26.6 us, so 24.7.
    const auto load = [&](u32 v) {
        if (alike) return __ldcs(in + v);
        const T* e = x + lead + (size_t)v * N;
        uint4 r; T w[N];
#pragma unroll
        for (int i = 0; i < N; i++) w[i] = score_raw(e + i);
        memcpy(&r, w, 16);
        return r;
    };
    const u32 vt = R.t < (int32_t)lead ? 0xFFFFFFFFu : ((u32)R.t - lead) / N;
    const auto put = [&](const uint4& r, u32 v) {
        float d[N];
#pragma unroll
        for (int p = 0; p < N / 2; p++) score_grad_pair<ENT>(R, V::pair(r, p), d[2 * p], d[2 * p + 1]);
        if (v == vt) {
#pragma unroll
            for (int e = 0; e < N; e++) if ((int32_t)(lead + v * N + e) == R.t) d[e] += R.hot;
        }
        __stcs(out + v, ScorePut<T>::vec(d));
    };
    const u32 v1 = min(n_vec, (part + 1) * share);             // (fewer than 2^29 vectors, a share of at most 2^12: no sum passes 32 bits)
    u32 v = part * share + tid;
    if (zeros) {
        for (; v < v1; v += NT) __stcs(out + v, make_uint4(0, 0, 0, 0));
    } else {
        for (; v + (U - 1) * NT < v1; v += U * NT) {
            uint4 r[U];
#pragma unroll
            for (int i = 0; i < U; i++) r[i] = load(v + i * NT);
#pragma unroll
            for (int i = 0; i < U; i++) put(r[i], v + i * NT);
        }
        if (v < v1) {
            uint4 r[U];
#pragma unroll
            for (int i = 0; i < U; i++) if (v + i * NT < v1) r[i] = load(v + i * NT);
#pragma unroll
            for (int i = 0; i < U; i++) if (v + i * NT < v1) put(r[i], v + i * NT);
        }
    }
    const u32 loose = lead + (P.n_vocab - lead - n_vec * N);
    if (part == 0 && tid < loose) {
        const u32 j = tid < lead ? tid : n_vec * N + tid;
        score_put(dx + j, zeros ? 0.0f : score_grad_one<ENT>(R, score_ld(x + j), j));
    }
}
