// Block tables: blocks for the new tokens of every request, their slots in the paged cache, and blocks that go back.
//
// With c_r tokens of request r in the cache and n_r new ones (release: c_r and the k_r that stay) the request's blocks change by
//   ceil((c_r + n_r) / B) - ceil(c_r / B)      (release: ceil(c_r / B) - ceil(k_r / B)),
// and an exclusive sum over the requests says which entries of the free list each of them gets (or fills).
// The first kernel reads all lengths, decides whether the call can be done, and only then writes the new state; the second one
// works from what it left in the workspace, so that the new state may lie in the buffers of the old one.
#pragma once
#include "tt_host.cuh"

constexpr int BLOCKS_THREADS = 1024;

struct BlocksPlan {                    // workspace: a head, then per request (tokens in the cache, blocks of the requests before)
    long long n_free;                  // before the call
    long long total;                   // blocks taken or given back
    int status, pad;
};
struct BlocksParams {
    const long long* new_off;          // extend
    const int32_t* keep;               // release
    const int32_t* seq_len;
    u32 n_req, block, width;
    int32_t* table;
    int32_t* free_blocks;
    unsigned long long free_cap;
    const long long* n_free;
    long long* slots; unsigned long long slots_cap;
    int32_t* pos; int32_t* req;
    int32_t* seq_out; long long* n_free_out; int32_t* status_out;
    BlocksPlan* plan; int2* per;       // (tokens in the cache, blocks before)
};

__device__ __forceinline__ u32 blocks_of(u32 tokens, u32 block) { return tokens / block + (tokens % block != 0); }

// One request: the change of its blocks and its new length; `bad` collects the status bits (1 argument, 2 capacity).
template <bool EXTEND>
__device__ __forceinline__ u32 blocks_change(const BlocksParams& P, u32 r, int32_t& c, int32_t& c_new, u32& bad) {
    c = __ldcg(P.seq_len + r);
    c_new = c;
    if (c < 0) { bad |= 1; return 0; }
    if constexpr (EXTEND) {
        const long long a = __ldcg(P.new_off + r), b = __ldcg(P.new_off + r + 1);
        if (b < a || a < 0 || (r == 0 && a != 0)) { bad |= 1; return 0; }
        if (b - a > (long long)0x7FFFFFFF - c) { bad |= 2; return 0; }
        c_new = c + (int32_t)(b - a);
        const u32 have = blocks_of((u32)c, P.block), want = blocks_of((u32)c_new, P.block);
        if (want > P.width) { bad |= 2; return 0; }
        return want - have;
    } else {
        const int32_t k = __ldcg(P.keep + r);
        if (k < 0 || k > c) { bad |= 1; return 0; }
        c_new = k;
        const u32 have = blocks_of((u32)c, P.block);
        if (have > P.width) { bad |= 2; return 0; }
        return have - blocks_of((u32)k, P.block);
    }
}

template <bool EXTEND>
__global__ void __launch_bounds__(BLOCKS_THREADS)
k_blocks_plan(const __grid_constant__ BlocksParams P) {
    __shared__ long long s_sum[BLOCKS_THREADS];
    cudaGridDependencySynchronize();
    const int tid = threadIdx.x;
    const long long n_free = __ldcg(P.n_free);
    u32 bad = 0;
    if (n_free < 0 || (unsigned long long)n_free > P.free_cap) bad |= 1;
    if (EXTEND) {
        const long long t = P.n_req ? __ldcg(P.new_off + P.n_req) : 0;
        if (t > 0 && (unsigned long long)t > P.slots_cap) bad |= 2;
    }
    long long carry = 0;
    for (u32 r0 = 0; r0 < P.n_req; r0 += BLOCKS_THREADS) {
        const u32 r = r0 + tid;
        int32_t c = 0, c_new = 0;
        const long long mine = r < P.n_req ? blocks_change<EXTEND>(P, r, c, c_new, bad) : 0;
        __syncthreads();
        s_sum[tid] = mine;
        __syncthreads();
        for (int o = 1; o < BLOCKS_THREADS; o <<= 1) {
            const long long t = tid >= o ? s_sum[tid - o] : 0;
            __syncthreads();
            s_sum[tid] += t;
            __syncthreads();
        }
        if (r < P.n_req) P.per[r] = make_int2(c, (int)(u32)(carry + s_sum[tid] - mine));
        carry += s_sum[BLOCKS_THREADS - 1];
    }
    if (carry > (EXTEND ? n_free : (long long)P.free_cap - n_free)) bad |= 2;
    const int any1 = __syncthreads_or(bad & 1), any2 = __syncthreads_or(bad & 2);
    const int status = any1 ? 1 /* TT_ERR_ARG */ : any2 ? 5 /* TT_ERR_CAPACITY */ : 0;
    for (u32 r = tid; r < P.n_req; r += BLOCKS_THREADS) {              // (every length has been read: the new ones may lie over them)
        const int32_t c = P.per[r].x;
        int32_t c_new = c;
        if (status == 0) c_new = EXTEND ? c + (int32_t)(__ldcg(P.new_off + r + 1) - __ldcg(P.new_off + r)) : __ldcg(P.keep + r);
        P.seq_out[r] = c_new;
    }
    if (tid == 0) {
        BlocksPlan q; q.n_free = n_free; q.total = carry; q.status = status; q.pad = 0;
        *P.plan = q;
        *P.n_free_out = status ? n_free : EXTEND ? n_free - carry : n_free + carry;
        *P.status_out = status;
    }
}

// Blocks into the table, then a token a thread.
__global__ void __launch_bounds__(256)
k_blocks_extend(const __grid_constant__ BlocksParams P) {
    cudaGridDependencySynchronize();
    if (P.plan->status != 0) return;
    const long long n_free = P.plan->n_free;
    const unsigned long long step = (unsigned long long)gridDim.x * blockDim.x, first = (unsigned long long)blockIdx.x * blockDim.x + threadIdx.x;
    for (unsigned long long r = first / 32; r < P.n_req; r += step / 32) {                  // a warp a request
        const int2 q = P.per[r];
        const u32 have = blocks_of((u32)q.x, P.block), want = blocks_of((u32)q.x + (u32)(P.new_off[r + 1] - P.new_off[r]), P.block);
        for (u32 b = have + (threadIdx.x & 31); b < want; b += 32) P.table[r * P.width + b] = P.free_blocks[n_free - 1 - ((long long)q.y + (b - have))];
    }
    const unsigned long long total = (unsigned long long)P.new_off[P.n_req];
    for (unsigned long long i = first; i < total; i += step) {
        u32 lo = 0, hi = P.n_req;                                      // the first offset behind i
        while (lo < hi) { const u32 mid = (lo + hi) / 2; if (__ldg(P.new_off + mid) <= (long long)i) lo = mid + 1; else hi = mid; }
        const u32 r = lo - 1;
        const int2 q = P.per[r];
        const u32 have = blocks_of((u32)q.x, P.block), p = (u32)q.x + (u32)((long long)i - P.new_off[r]), b = p / P.block;
        const int32_t id = b < have ? P.table[(unsigned long long)r * P.width + b] : P.free_blocks[n_free - 1 - ((long long)q.y + (b - have))];
        P.slots[i] = (long long)id * P.block + p % P.block;
        if (P.pos) P.pos[i] = (int32_t)p;
        if (P.req) P.req[i] = (int32_t)r;
    }
}

__global__ void __launch_bounds__(256)
k_blocks_release(const __grid_constant__ BlocksParams P) {
    cudaGridDependencySynchronize();
    if (P.plan->status != 0) return;
    const long long end = P.plan->n_free + P.plan->total;
    const unsigned long long step = (unsigned long long)gridDim.x * blockDim.x, first = (unsigned long long)blockIdx.x * blockDim.x + threadIdx.x;
    for (unsigned long long r = first / 32; r < P.n_req; r += step / 32) {
        const int2 q = P.per[r];
        const u32 have = blocks_of((u32)q.x, P.block), left = blocks_of((u32)P.keep[r], P.block);
        for (u32 b = left + (threadIdx.x & 31); b < have; b += 32) P.free_blocks[end - 1 - ((long long)q.y + (b - left))] = P.table[r * P.width + b];
    }
}
