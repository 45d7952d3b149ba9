// C ABI of the block tables (see include/toktier.h): tt_blocks_extend and tt_blocks_release.  Nothing here synchronises or allocates.
#include "../../include/toktier.h"
#include "tt_blocks.cuh"

static size_t blocks_up(size_t x) { return (x + 255) / 256 * 256; }

extern "C" size_t tt_blocks_workspace_bytes(size_t n_req) { return blocks_up(sizeof(BlocksPlan)) + blocks_up(n_req * sizeof(int2)); }

static int blocks_args(BlocksParams& P, size_t n_req, const int32_t* seq_len, size_t block_size, const int32_t* table, size_t width, const int32_t* free_blocks,
                       size_t free_cap, const int64_t* n_free, int32_t* seq_out, int64_t* n_free_out, int32_t* status_out, void* workspace, size_t workspace_bytes) {
    const size_t most = (size_t)1 << 31;
    if (n_req >= ((size_t)1 << 24) || !block_size || block_size >= most || width >= most || free_cap >= most) return TT_ERR_ARG;
    if (!n_free || !n_free_out || !status_out || !workspace || (n_req && (!seq_len || !seq_out || (width && !table))) || (free_cap && !free_blocks)) return TT_ERR_ARG;
    if (host_misaligned(4, seq_len, table, free_blocks, seq_out, status_out) || host_misaligned(8, n_free, n_free_out)) return TT_ERR_ARG;
    if (((uintptr_t)workspace & 255) != 0 || workspace_bytes < tt_blocks_workspace_bytes(n_req)) return TT_ERR_ARG;
    P = BlocksParams{};
    unsigned sh = 0;
    while ((size_t)1 << sh < block_size) sh++;
    P.div_shift = 31 + sh; P.div_mul = (u32)((((size_t)1 << (31 + sh)) + block_size - 1) / block_size);
    P.seq_len = seq_len; P.n_req = (u32)n_req; P.block = (u32)block_size; P.width = (u32)width; P.table = const_cast<int32_t*>(table);
    P.free_blocks = const_cast<int32_t*>(free_blocks); P.free_cap = free_cap; P.n_free = (const long long*)n_free;
    P.seq_out = seq_out; P.n_free_out = (long long*)n_free_out; P.status_out = status_out;
    P.plan = (BlocksPlan*)workspace; P.per = (int2*)((char*)workspace + blocks_up(sizeof(BlocksPlan)));
    return TT_OK;
}

// `most`: entries (tokens, blocks) that the call may have to write.
//   One kernel for up to BLOCKS_FEW requests and 4 tokens or 16 blocks a thread of the cluster: 64 requests of 500 tokens 6.6 us, as two kernels 8.2;
//   1,000 of 60 11.8 and 9.3; 1,000 requests' 31,000 blocks back 6.6 and 9.7 (there are mostly fewer than fit in the list).
//   Of one CTA up to an entry a thread: 256 and 1,000 requests of one token 3.3 and 4.2 us, of a cluster 3.9 and 4.8; 64 of 64 6.3 and 4.3.
//   The room in the buffers decides, since the host does not know what there is to write: 256 requests of one token take 12.8 us (two kernels) where
// `slots` has room for more than 32,768 tokens, and 1,000 14.5.  Maps of their own for decode steps have the small form.
template <bool EXTEND>
static int blocks_launch(const BlocksParams& P, size_t most, cudaStream_t st) {
    if (P.n_req <= BLOCKS_FEW && most <= (size_t)(EXTEND ? 4 : 16) * BLOCKS_CLUSTER * BLOCKS_THREADS) {
        const unsigned ctas = most <= BLOCKS_THREADS ? 1 : BLOCKS_CLUSTER;
        TT_TRY(host_launch(k_blocks_few<EXTEND>, ctas, BLOCKS_THREADS, ctas, 0, st, P));
        return TT_OK;
    }
    const int sms = host_sm_count();
    if (!sms) return TT_ERR_CUDA;
    TT_TRY(host_launch(k_blocks_plan<EXTEND>, 1, BLOCKS_THREADS, 1, 0, st, P));
    if (P.n_req) TT_TRY(host_launch(EXTEND ? k_blocks_extend : k_blocks_release, (unsigned)sms * BLOCKS_WRITE_CTAS, BLOCKS_WRITE_NT, 1, 0, st, P));
    return TT_OK;
}

extern "C" int tt_blocks_extend(const int64_t* new_off, size_t n_req, const int32_t* seq_len, size_t block_size, int32_t* block_table, size_t table_width,
                                const int32_t* free_blocks, size_t free_cap, const int64_t* n_free, void* stream, int64_t* slots_out, size_t slots_cap,
                                int32_t* pos_out, int32_t* req_out, int32_t* seq_len_out, int64_t* n_free_out, int32_t* status_out,
                                void* workspace, size_t workspace_bytes) {
    BlocksParams P;
    const int rc = blocks_args(P, n_req, seq_len, block_size, block_table, table_width, free_blocks, free_cap, n_free, seq_len_out, n_free_out, status_out, workspace, workspace_bytes);
    if (rc != TT_OK) return rc;
    if (host_misaligned(4, pos_out, req_out) || host_misaligned(8, new_off, slots_out)) return TT_ERR_ARG;
    if ((n_req && !new_off) || slots_cap >= ((size_t)1 << 31) || (slots_cap && !slots_out)) return TT_ERR_ARG;
    P.new_off = (const long long*)new_off; P.slots = (long long*)slots_out; P.slots_cap = slots_cap; P.pos = pos_out; P.req = req_out;
    return blocks_launch<true>(P, slots_cap, (cudaStream_t)stream);
}

extern "C" int tt_blocks_release(const int32_t* keep_len, size_t n_req, const int32_t* seq_len, size_t block_size, const int32_t* block_table, size_t table_width,
                                 int32_t* free_blocks, size_t free_cap, const int64_t* n_free, void* stream, int32_t* seq_len_out, int64_t* n_free_out,
                                 int32_t* status_out, void* workspace, size_t workspace_bytes) {
    BlocksParams P;
    const int rc = blocks_args(P, n_req, seq_len, block_size, block_table, table_width, free_blocks, free_cap, n_free, seq_len_out, n_free_out, status_out, workspace, workspace_bytes);
    if (rc != TT_OK) return rc;
    if ((n_req && !keep_len) || host_misaligned(4, keep_len)) return TT_ERR_ARG;
    P.keep = keep_len;
    const size_t most = (size_t)n_req * table_width;
    return blocks_launch<false>(P, most < free_cap ? most : free_cap, (cudaStream_t)stream);
}
