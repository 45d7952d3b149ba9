// Block tables: blocks for the new tokens of every request, their slots in the paged cache, and blocks that go back.
//
// With c_r tokens of request r in the cache and n_r new ones (release: c_r and the k_r that stay) the request's blocks change by
//   ceil((c_r + n_r) / B) - ceil(c_r / B)      (release: ceil(c_r / B) - ceil(k_r / B)),
// and an exclusive sum over the requests says which entries of the free list each of them gets (or fills).
// What earlier kernels wrote is read behind the wait for them (cudaGridDependencySynchronize), and past L1, since it is read once.
// All lengths are read and the call decided on before anything of the new state is written, so that it may lie in the buffers of the old one.
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
    u32 div_mul, div_shift;            // x / block = x * div_mul >> div_shift for x < 2^31
    int32_t* table;
    int32_t* free_blocks;
    unsigned long long free_cap;
    const long long* n_free;
    long long* slots; unsigned long long slots_cap;
    int32_t* pos; int32_t* req;
    int32_t* seq_out; long long* n_free_out; int32_t* status_out;
    BlocksPlan* plan; int2* per;       // (tokens in the cache, blocks before)
};

// With 2^(s-1) < block <= 2^s and mul = ceil(2^(31+s) / block): mul block - 2^(31+s) < block <= 2^s, so that x * mul >> 31 + s is x / block rounded down.
__device__ __forceinline__ u32 blocks_div(const BlocksParams& P, u32 x) { return (u32)((u64)x * P.div_mul >> P.div_shift); }
__device__ __forceinline__ u32 blocks_of(const BlocksParams& P, u32 tokens) { const u32 b = blocks_div(P, tokens); return b + (b * P.block != tokens); }

// One request's lengths (nothing depends on a load here, so that those of all of a thread's requests are on their way at once), and the change of its
// blocks and its new length; `bad` collects the status bits (1 argument, 2 capacity).
struct BlocksLen { int32_t c; long long a, b; };                       // tokens in the cache; extend: offsets of the new ones and behind them; release: a = tokens kept
template <bool EXTEND>
__device__ __forceinline__ BlocksLen blocks_len(const BlocksParams& P, u32 r) {
    BlocksLen l;
    l.c = __ldcg(P.seq_len + r);
    l.a = EXTEND ? __ldcg(P.new_off + r) : __ldcg(P.keep + r);
    l.b = EXTEND ? __ldcg(P.new_off + r + 1) : 0;
    return l;
}
template <bool EXTEND>
__device__ __forceinline__ u32 blocks_change(const BlocksParams& P, u32 r, const BlocksLen& l, int32_t& c_new, u32& bad) {
    c_new = l.c;
    if (l.c < 0) { bad |= 1; return 0; }
    if constexpr (EXTEND) {
        if (l.b < l.a || l.a < 0 || (r == 0 && l.a != 0)) { bad |= 1; return 0; }
        if (l.b - l.a > (long long)0x7FFFFFFF - l.c) { bad |= 2; return 0; }
        c_new = l.c + (int32_t)(l.b - l.a);
        const u32 have = blocks_of(P, (u32)l.c), want = blocks_of(P, (u32)c_new);
        if (want > P.width) { bad |= 2; return 0; }
        return want - have;
    } else {
        if (l.a < 0 || l.a > l.c) { bad |= 1; return 0; }
        c_new = (int32_t)l.a;
        const u32 have = blocks_of(P, (u32)l.c);
        if (have > P.width) { bad |= 2; return 0; }
        return have - blocks_of(P, (u32)l.a);
    }
}

// Exclusive sum of x over the CTA in front of this thread, `total` over all of it.  Two barriers; the buffer may be used again after the next one.
__device__ __forceinline__ long long blocks_scan(long long x, long long* buf, long long& total) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    long long sum = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xFFFFFFFFu, sum, o); if (lane >= o) sum += t; }
    if (lane == 31) buf[wid] = sum;
    __syncthreads();
    long long w = buf[lane];                                           // (32 warps)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xFFFFFFFFu, w, o); if (lane >= o) w += t; }
    total = __shfl_sync(0xFFFFFFFFu, w, 31);
    const long long before = __shfl_sync(0xFFFFFFFFu, w, wid ? wid - 1 : 0);
    __syncthreads();
    return (wid ? before : 0) + sum - x;
}

// What the lengths alone do not say: the free list's count, room for the tokens; then the sum of the changes against the list.
__device__ __forceinline__ u32 blocks_bad(const BlocksParams& P, long long n_free, long long tokens) {
    return (n_free < 0 || (unsigned long long)n_free > P.free_cap ? 1 : 0) | (tokens > 0 && (unsigned long long)tokens > P.slots_cap ? 2 : 0);
}
template <bool EXTEND>
__device__ __forceinline__ long long blocks_tokens(const BlocksParams& P) { return EXTEND && P.n_req ? __ldcg(P.new_off + P.n_req) : 0; }
template <bool EXTEND>
__device__ __forceinline__ int blocks_status(const BlocksParams& P, u32 bad, long long n_free, long long total) {
    if (total > (EXTEND ? n_free : (long long)P.free_cap - n_free)) bad |= 2;
    const int arg = __syncthreads_or(bad & 1), cap = __syncthreads_or(bad & 2);
    return arg ? 1 /* TT_ERR_ARG */ : cap ? 5 /* TT_ERR_CAPACITY */ : 0;
}

// Few requests: one kernel.  Every CTA of the cluster (one, or BLOCKS_CLUSTER of them) works out the whole plan in its shared memory, and they
// wait for each other between the reading of the old state and the writing of the new one, which may lie in the same place.  256 requests of
// one token 3.3 us, a chain of dependent loads.
constexpr int BLOCKS_FEW = 2048, BLOCKS_CLUSTER = 8;
template <bool EXTEND>
__global__ void __launch_bounds__(BLOCKS_THREADS)
k_blocks_few(const __grid_constant__ BlocksParams P) {
    __shared__ int s_c[BLOCKS_FEW], s_before[BLOCKS_FEW];              // tokens in the cache, blocks of the requests before
    __shared__ int s_at[BLOCKS_FEW];                                   // extend: offset of the new tokens; release: tokens kept
    __shared__ long long s_scan[32];
    const u32 ctas = gridDim.x, cta = blockIdx.x, tid = threadIdx.x;
    cudaGridDependencySynchronize();
    const long long n_free = __ldcg(P.n_free), all = blocks_tokens<EXTEND>(P);
    BlocksLen l[2] = {};
    int32_t c_new[2] = {0, 0};
    u32 change[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; i++) if (2 * tid + i < P.n_req) l[i] = blocks_len<EXTEND>(P, 2 * tid + i);
    u32 bad = blocks_bad(P, n_free, all);
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const u32 r = 2 * tid + i;
        if (r >= P.n_req) continue;
        change[i] = blocks_change<EXTEND>(P, r, l[i], c_new[i], bad);
        s_c[r] = l[i].c;
        s_at[r] = (int)l[i].a;
    }
    long long total;
    const long long before = blocks_scan((long long)change[0] + change[1], s_scan, total);
    if (2 * tid < P.n_req) s_before[2 * tid] = (int)before;
    if (2 * tid + 1 < P.n_req) s_before[2 * tid + 1] = (int)(before + change[0]);
    const int status = blocks_status<EXTEND>(P, bad, n_free, total);
    if (ctas > 1) { cluster_arrive(); cluster_wait(); }                // the old state has been read
    if (cta == 0) {
#pragma unroll
        for (int i = 0; i < 2; i++) if (2 * tid + i < P.n_req) P.seq_out[2 * tid + i] = status ? l[i].c : c_new[i];
        if (tid == 0) { *P.n_free_out = status ? n_free : EXTEND ? n_free - total : n_free + total; *P.status_out = status; }
    }
    if (status) return;
    const u32 n = (u32)(EXTEND ? all : total);
    const int* at = EXTEND ? s_at : s_before;
    for (u32 i = cta * BLOCKS_THREADS + tid; i < n; i += ctas * BLOCKS_THREADS) {
        u32 lo = 0, hi = P.n_req - 1;                                  // the last request that begins at i or before
        while (lo < hi) { const u32 mid = (lo + hi + 1) / 2; if (at[mid] <= (int)i) lo = mid; else hi = mid - 1; }
        const u32 r = lo;
        const unsigned long long row = (unsigned long long)r * P.width;
        if constexpr (EXTEND) {
            const u32 have = blocks_of(P, (u32)s_c[r]), p = (u32)s_c[r] + (i - s_at[r]), b = blocks_div(P, p), o = p - b * P.block;
            const int32_t id = b < have ? __ldcg(P.table + row + b) : __ldcg(P.free_blocks + (n_free - 1 - ((long long)s_before[r] + (b - have))));
            if (o == 0 && b >= have) P.table[row + b] = id;            // (every new block has a new token at its beginning)
            P.slots[i] = (long long)id * P.block + o;
            if (P.pos) P.pos[i] = (int32_t)p;
            if (P.req) P.req[i] = (int32_t)r;
        } else {
            P.free_blocks[n_free + total - 1 - i] = __ldcg(P.table + row + blocks_of(P, (u32)s_at[r]) + (i - s_before[r]));
        }
    }
}

// Many requests or many tokens: the plan by one CTA, four requests a thread, into the workspace; the rest by the whole GPU.
template <bool EXTEND>
__global__ void __launch_bounds__(BLOCKS_THREADS)
k_blocks_plan(const __grid_constant__ BlocksParams P) {
    constexpr int EACH = 4;
    __shared__ long long s_scan[32];
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    const u32 tid = threadIdx.x;
    const long long n_free = __ldcg(P.n_free);
    u32 bad = blocks_bad(P, n_free, blocks_tokens<EXTEND>(P));
    long long carry = 0;
    BlocksLen l[EACH] = {};
    int32_t c_new[EACH] = {};
    for (unsigned long long r0 = 0; r0 < P.n_req; r0 += EACH * BLOCKS_THREADS) {
        u32 change[EACH];
        long long mine = 0, total;
#pragma unroll
        for (int i = 0; i < EACH; i++) if (r0 + EACH * tid + i < P.n_req) l[i] = blocks_len<EXTEND>(P, (u32)(r0 + EACH * tid + i));
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            const unsigned long long r = r0 + EACH * tid + i;
            change[i] = r < P.n_req ? blocks_change<EXTEND>(P, (u32)r, l[i], c_new[i], bad) : 0;
            mine += change[i];
        }
        long long at = carry + blocks_scan(mine, s_scan, total);
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            const unsigned long long r = r0 + EACH * tid + i;
            if (r < P.n_req) P.per[r] = make_int2(l[i].c, (int)(u32)at);
            at += change[i];
        }
        carry += total;
    }
    const int status = blocks_status<EXTEND>(P, bad, n_free, carry);
    // every length has been read: the new ones may lie over them
    if (P.n_req <= EACH * BLOCKS_THREADS) {
#pragma unroll
        for (int i = 0; i < EACH; i++) if (EACH * tid + i < P.n_req) P.seq_out[EACH * tid + i] = status ? l[i].c : c_new[i];
    } else {
        for (u32 r = tid; r < P.n_req; r += BLOCKS_THREADS) {
            const int32_t c = P.per[r].x;
            P.seq_out[r] = status ? c : EXTEND ? c + (int32_t)(__ldcg(P.new_off + r + 1) - __ldcg(P.new_off + r)) : __ldcg(P.keep + r);
        }
    }
    if (tid == 0) {
        BlocksPlan q; q.n_free = n_free; q.total = carry; q.status = status; q.pad = 0;
        *P.plan = q;
        *P.n_free_out = status ? n_free : EXTEND ? n_free - carry : n_free + carry;
        *P.status_out = status;
    }
}

// The last of lo .. hi whose `at` is at most i, where at(lo) is; by a whole warp, 32 at a time (two steps for a thousand requests).
template <typename F>
__device__ __forceinline__ u32 blocks_find(u32 lo, u32 hi, long long i, const F& at) {
    while (lo < hi) {
        const u32 step = (hi - lo + 31) / 32;
        const unsigned long long mid = lo + (unsigned long long)((threadIdx.x & 31) + 1) * step;
        const u32 k = __popc(__ballot_sync(0xFFFFFFFFu, mid <= hi && at((u32)mid) <= i));
        lo += k * step;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}

// Slots and maps: a CTA takes a stretch of tiles of BLOCKS_TILE tokens, four neighbouring tokens a thread, so that each map is written 16 bytes
// at a time.  The request of a tile is searched for only where it changes; of a tile with several requests their offsets and plans go to shared
// memory, where every token looks for its own.  What all CTAs read is read by one warp of each: by every warp of the GPU it was a queue at one
// slice of L2 (the blocks of 256 long requests back into the list 34 us).  Bound by the 16 bytes a token that it writes:
// 22.7 million tokens of 256 requests 68 us behind a plan of 4, 5.3 TB/s.
constexpr int BLOCKS_WRITE_NT = 256, BLOCKS_WRITE_CTAS = 5, BLOCKS_TILE = 4 * BLOCKS_WRITE_NT, BLOCKS_STAGED = 1024;
struct BlocksHead { long long n_free, total; int status; u32 r, last; };

__device__ __forceinline__ void blocks_head(const BlocksParams& P, BlocksHead& head, bool extend) {
    if (threadIdx.x == 0) {
        head.status = __ldcg(&P.plan->status);
        head.n_free = __ldcg(&P.plan->n_free);
        head.total = extend ? __ldcg(P.new_off + P.n_req) : __ldcg(&P.plan->total);
    }
    __syncthreads();
}
__global__ void __launch_bounds__(BLOCKS_WRITE_NT, 5)
k_blocks_extend(const __grid_constant__ BlocksParams P) {
    __shared__ long long s_off[BLOCKS_STAGED + 1];
    __shared__ int2 s_per[BLOCKS_STAGED];
    __shared__ BlocksHead head;
    cudaGridDependencySynchronize();
    blocks_head(P, head, true);
    if (head.status != 0) return;
    const long long n_free = head.n_free, total = head.total, tiles = (total + BLOCKS_TILE - 1) / BLOCKS_TILE;
    const long long t0 = tiles * blockIdx.x / gridDim.x, t1 = tiles * (blockIdx.x + 1) / gridDim.x;
    const bool wide = (((uintptr_t)P.slots | (uintptr_t)P.pos | (uintptr_t)P.req) & 15) == 0;
    const auto off = [&](u32 r) { return __ldcg(P.new_off + r); };
    u32 r = 0, last = 0;
    bool staged = false;
    long long r_off = 0, r_end = -1;                                   // off[r], off[r + 1]
    int2 r_per = make_int2(0, 0);
    for (long long t = t0; t < t1; t++) {
        const long long first = t * BLOCKS_TILE, i0 = first + 4 * threadIdx.x, behind = min(total, first + BLOCKS_TILE);
        if (behind > r_end) {                                          // not all of the request that the tile before ended in
            __syncthreads();                                           // (the tile before is done with the shared memory)
            if (threadIdx.x < 32) {
                const u32 q = blocks_find(r, P.n_req - 1, first, off), e = blocks_find(q, P.n_req - 1, behind - 1, off);
                if (threadIdx.x == 0) { head.r = q; head.last = e; }
            }
            __syncthreads();
            r = head.r; last = head.last;
            staged = last - r < BLOCKS_STAGED;
            if (staged) for (u32 k = threadIdx.x; k <= last - r + 1; k += BLOCKS_WRITE_NT) { s_off[k] = off(r + k); if (k <= last - r) s_per[k] = __ldcg(P.per + r + k); }
            __syncthreads();
            r_off = staged ? s_off[0] : off(r); r_end = staged ? s_off[1] : off(r + 1); r_per = staged ? s_per[0] : __ldcg(P.per + r);
        } else last = r;
        long long slot[4];
        int pos[4], req[4];
        u32 q = r, have = 0, b = 0, o = 0;
        long long q_end = -1;
        int before = 0;
        int32_t id = 0;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const long long i = i0 + k;
            if (i >= total) break;
            if (i >= q_end) {                                          // the thread's first token, or the first of another request
                long long at = r_off;
                int2 per = r_per;
                q_end = r_end;
                if (last != r) {
                    u32 hi = last;
                    while (q < hi) { const u32 mid = q + (hi - q + 1) / 2; if ((staged ? s_off[mid - r] : off(mid)) <= i) q = mid; else hi = mid - 1; }
                    at = staged ? s_off[q - r] : off(q);
                    q_end = staged ? s_off[q - r + 1] : off(q + 1);
                    per = staged ? s_per[q - r] : __ldcg(P.per + q);
                }
                const u32 p = (u32)per.x + (u32)(i - at);
                before = per.y;
                have = blocks_of(P, (u32)per.x);
                b = blocks_div(P, p); o = p - b * P.block;
                id = b < have ? __ldcg(P.table + (unsigned long long)q * P.width + b) : __ldcg(P.free_blocks + (n_free - 1 - ((long long)before + (b - have))));
            } else if (o == P.block) {                                 // a new block: one in the cache has no room for a beginning
                o = 0; b++;
                id = __ldcg(P.free_blocks + (n_free - 1 - ((long long)before + (b - have))));
            }
            if (o == 0 && b >= have) P.table[(unsigned long long)q * P.width + b] = id;              // (every new block has a new token at its beginning)
            slot[k] = (long long)id * P.block + o;
            pos[k] = (int)(b * P.block + o);
            req[k] = (int)q;
            o++;
        }
        if (wide && i0 + 4 <= total) {
            __stcs(reinterpret_cast<longlong2*>(P.slots + i0), make_longlong2(slot[0], slot[1]));
            __stcs(reinterpret_cast<longlong2*>(P.slots + i0 + 2), make_longlong2(slot[2], slot[3]));
            if (P.pos) __stcs(reinterpret_cast<int4*>(P.pos + i0), make_int4(pos[0], pos[1], pos[2], pos[3]));
            if (P.req) __stcs(reinterpret_cast<int4*>(P.req + i0), make_int4(req[0], req[1], req[2], req[3]));
        } else {
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (i0 + k < total) { P.slots[i0 + k] = slot[k]; if (P.pos) P.pos[i0 + k] = pos[k]; if (P.req) P.req[i0 + k] = req[k]; }
        }
    }
}

// Blocks back into the list: a CTA takes a stretch of them, four a thread side by side in the row of the table.
__global__ void __launch_bounds__(BLOCKS_WRITE_NT, 6)
k_blocks_release(const __grid_constant__ BlocksParams P) {
    __shared__ int s_before[BLOCKS_STAGED], s_left[BLOCKS_STAGED];
    __shared__ BlocksHead head;
    cudaGridDependencySynchronize();
    blocks_head(P, head, false);
    if (head.status != 0) return;
    const long long total = head.total, end = head.n_free + total, tiles = (total + BLOCKS_TILE - 1) / BLOCKS_TILE;
    const long long t0 = tiles * blockIdx.x / gridDim.x, t1 = tiles * (blockIdx.x + 1) / gridDim.x;
    const auto before = [&](u32 r) { return (long long)(u32)__ldcg(&P.per[r].y); };
    const auto left = [&](u32 r) { return blocks_of(P, (u32)__ldcg(P.keep + r)); };
    u32 r = 0;
    for (long long t = t0; t < t1; t++) {
        const long long first = t * BLOCKS_TILE, behind = min(total, first + BLOCKS_TILE);
        __syncthreads();                                               // (the tile before is done with the shared memory)
        if (threadIdx.x < 32) {
            const u32 q = blocks_find(r, P.n_req - 1, first, before), e = blocks_find(q, P.n_req - 1, behind - 1, before);
            if (threadIdx.x == 0) { head.r = q; head.last = e; }
        }
        __syncthreads();
        r = head.r;
        const u32 last = head.last;
        const bool staged = last - r < BLOCKS_STAGED;
        if (staged) for (u32 k = threadIdx.x; k <= last - r; k += BLOCKS_WRITE_NT) { s_before[k] = (int)before(r + k); s_left[k] = (int)left(r + k); }
        __syncthreads();
        int32_t id[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const long long i = first + k * BLOCKS_WRITE_NT + threadIdx.x;
            if (i >= total) break;
            u32 q = r, hi = last;
            while (q < hi) { const u32 mid = q + (hi - q + 1) / 2; if ((staged ? (long long)(u32)s_before[mid - r] : before(mid)) <= i) q = mid; else hi = mid - 1; }
            const u32 at = staged ? (u32)s_left[q - r] + ((u32)i - (u32)s_before[q - r]) : left(q) + (u32)(i - before(q));
            id[k] = __ldcg(P.table + (unsigned long long)q * P.width + at);
        }
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const long long i = first + k * BLOCKS_WRITE_NT + threadIdx.x;
            if (i < total) P.free_blocks[end - 1 - i] = id[k];
        }
    }
}
