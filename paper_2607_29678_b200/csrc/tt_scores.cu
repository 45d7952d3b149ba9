// C ABI of the scores of token ids (see include/toktier.h): tt_logprobs and its gradient.  Nothing here synchronises or allocates.
#include "../../include/toktier.h"
#include "tt_scores.cuh"

static size_t score_size(int dtype) { return dtype == TT_FP32 ? 4 : 2; }

// What both entry points check of their arguments.
static int score_args(const void* logits, int dtype, size_t n_rows, size_t n_vocab, size_t row_stride, float scale, const int32_t* ids,
                      const int64_t* ids_off, size_t n_docs, const int32_t* status_out) {
    if (dtype != TT_BF16 && dtype != TT_FP16 && dtype != TT_FP32) return TT_ERR_ARG;
    if (!status_out || (n_rows && (!logits || !ids)) || !n_vocab || n_vocab >= ((size_t)1 << 31) || n_rows >= ((size_t)1 << 24)) return TT_ERR_ARG;
    if (row_stride < n_vocab || row_stride >= ((size_t)1 << 38)) return TT_ERR_ARG;
    if (host_misaligned(score_size(dtype), logits) || host_misaligned(4, ids, status_out) || host_misaligned(8, ids_off)) return TT_ERR_ARG;
    if (!(scale > 0.0f && scale <= 0x1p100f) || (ids_off == nullptr && n_docs != 0) || n_docs >= ((size_t)1 << 31)) return TT_ERR_ARG;
    return TT_OK;
}

template <typename T, int NT>
static cudaError_t launch_logprobs_nt(const ScoreParams& P, cudaStream_t st) {
    const auto kernel = P.top_k ? (P.rank ? k_logprobs<T, true, true, NT> : k_logprobs<T, true, false, NT>) : P.rank ? k_logprobs<T, false, true, NT> : k_logprobs<T, false, false, NT>;
    return host_launch(kernel, ((unsigned)P.n_rows + 1) << P.log_ctas, NT, 1u << P.log_ctas, 0, st, P);
}
// Threads of a CTA and CTAs of a row.  An SM has places for SCORE_PLACES threads.
//   Short rows, many of them: CTAs of 64 (4,096 rows of 8.7 KB: 64 threads 17 us, with alternatives 32, 128 threads 23 and 38, 256 39 and 59).
//   Up to one row for each SM 256 threads, otherwise 128 (4,096 rows of 200 KB: 64 threads 139 us, 128 133, 256 141; with alternatives 218, 169, 182).
//   But between half a round and one and a half of CTAs of 128 threads, where the SMs get one or two more or less: long 16-bit rows, bound by arithmetic
//   too, take 256 (1,024 rows of 400 KB: 64 threads 86 us, 128 85, 256 73; with alternatives 124, 100, 93), others behind a full round 64, all at
//   once (1,000 rows of 400 KB in 32 bits: 66, 90, 74; 1,100 of 64 KB: 27, 28, 30).
//   These borders lie between sizes that were measured, 8.7 and 64 KB for the first, 64 and 400 KB for the second, and some rows outside them would gain by another form: 2,200 of
// 400 KB with alternatives 128 threads 189 us, 256 175; 600 without 256 threads 51.7, 128 in clusters of two 48.3.
//   Fewer rows: a cluster for a row as long as its CTAs have places and 48 KB each (one row of 200 KB: 1 CTA 11.6 us, 4 7.7; 64 rows of 400 KB:
//   1 CTA 21, 4 14.9, 8 24; 300 of 400 KB: 42, of 2 CTAs 36, 4 37, 8 46; 64 rows of 64 KB: 1 CTA 8.8, 2 9.2, 8 15.7).
template <typename T>
static cudaError_t launch_logprobs(ScoreParams& P, size_t sms, cudaStream_t st) {
    const size_t bytes = (size_t)P.n_vocab * sizeof(T), places = sms * SCORE_PLACES, half = places / 256, full = places / 128;
    P.log_ctas = 0;
    if (P.n_rows > half && bytes <= 16384) return launch_logprobs_nt<T, 64>(P, st);
    if (P.n_rows > half && P.n_rows <= full * 3 / 2) {
        if (sizeof(T) == 2 && bytes >= 131072) return launch_logprobs_nt<T, 256>(P, st);
        if (P.n_rows > full) return launch_logprobs_nt<T, 64>(P, st);
    }
    const size_t nt = P.n_rows <= sms ? 256 : 128;
    while (2u << P.log_ctas <= SCORE_CLUSTER && (P.n_rows * nt << (P.log_ctas + 1)) <= places && bytes >> (P.log_ctas + 1) >= 49152) P.log_ctas++;
    return nt == 256 ? launch_logprobs_nt<T, 256>(P, st) : launch_logprobs_nt<T, 128>(P, st);
}

extern "C" int tt_logprobs(const void* logits, int dtype, size_t n_rows, size_t n_vocab, size_t row_stride, float scale, const int32_t* ids,
                           const int64_t* ids_off, size_t n_docs, size_t top_k, void* stream, float* logprob_out, float* lse_out, float* entropy_out,
                           int32_t* rank_out, int32_t* top_ids_out, float* top_logprob_out, int32_t* status_out) {
    const int rc = score_args(logits, dtype, n_rows, n_vocab, row_stride, scale, ids, ids_off, n_docs, status_out);
    if (rc != TT_OK) return rc;
    if ((n_rows && !logprob_out) || top_k > TT_TOP_MAX || top_k > n_vocab) return TT_ERR_ARG;
    if (host_misaligned(4, logprob_out, lse_out, entropy_out, rank_out, top_ids_out, top_logprob_out)) return TT_ERR_ARG;
    if (top_k ? n_rows && (!top_ids_out || !top_logprob_out) : top_ids_out || top_logprob_out) return TT_ERR_ARG;
    ScoreParams P;
    P.logits = logits; P.n_rows = n_rows; P.stride = row_stride; P.n_vocab = (u32)n_vocab; P.top_k = (u32)top_k; P.scale = scale;
    P.ids = ids; P.ids_off = (const long long*)ids_off; P.n_docs = n_docs;
    P.logprob = logprob_out; P.lse = lse_out; P.entropy = entropy_out; P.rank = rank_out; P.top_ids = top_ids_out; P.top_lp = top_logprob_out;
    P.status_out = status_out;
    P.scale2 = (float)((double)scale * 1.4426950408889634);
    const int sms = host_sm_count();
    if (!sms) return TT_ERR_CUDA;
    TT_TRY(dtype == TT_BF16 ? launch_logprobs<__nv_bfloat16>(P, sms, (cudaStream_t)stream) : dtype == TT_FP16 ? launch_logprobs<__half>(P, sms, (cudaStream_t)stream)
                            : launch_logprobs<float>(P, sms, (cudaStream_t)stream));
    return TT_OK;
}

template <typename T>
static cudaError_t launch_logprobs_grad(const ScoreGradParams& P, cudaStream_t st) {
    return host_launch(P.h ? k_logprobs_grad<T, true> : k_logprobs_grad<T, false>, (unsigned)(P.n_rows * P.parts + 1), SCORE_GRAD_NT, 1, 0, st, P);
}

extern "C" int tt_logprobs_grad(const void* logits, int dtype, size_t n_rows, size_t n_vocab, size_t row_stride, float scale, const int32_t* ids,
                                const int64_t* ids_off, size_t n_docs, const float* lse, const float* entropy, const float* grad_logprob,
                                const float* grad_entropy, void* stream, void* grad_out, size_t grad_stride, int32_t* status_out) {
    const int rc = score_args(logits, dtype, n_rows, n_vocab, row_stride, scale, ids, ids_off, n_docs, status_out);
    if (rc != TT_OK) return rc;
    if ((n_rows && (!lse || !grad_logprob || !grad_out)) || (grad_entropy != nullptr) != (entropy != nullptr)) return TT_ERR_ARG;
    if (grad_stride < n_vocab || grad_stride >= ((size_t)1 << 38)) return TT_ERR_ARG;
    if (host_misaligned(score_size(dtype), grad_out) || host_misaligned(4, lse, entropy, grad_logprob, grad_entropy)) return TT_ERR_ARG;
    if (n_rows && grad_out == logits && grad_stride != row_stride) return TT_ERR_ARG;
    ScoreGradParams P;
    P.logits = logits; P.n_rows = n_rows; P.stride = row_stride; P.grad_stride = grad_stride; P.n_vocab = (u32)n_vocab; P.scale = scale;
    P.ids = ids; P.ids_off = (const long long*)ids_off; P.n_docs = n_docs;
    P.lse = lse; P.entropy = entropy; P.g = grad_logprob; P.h = grad_entropy; P.grad = grad_out; P.status_out = status_out;
    const int sms = host_sm_count();
    if (!sms) return TT_ERR_CUDA;
    // a CTA takes up to four batches of 16 KB, so that a row's scalars are looked up for more of it, fewer where that makes less than four rounds of CTAs
    // (five on an SM): 1,000 rows of 64 KB with one batch 24.7 us, with four 25.7
    const size_t batch = (size_t)SCORE_GRAD_NT * SCORE_U * 16, bytes = n_vocab * score_size(dtype), places = (size_t)sms * 5 * 4;
    size_t rounds = 4;
    while (rounds > 1 && n_rows * ((bytes + rounds * batch - 1) / (rounds * batch)) < places) rounds /= 2;
    if (n_rows * ((bytes + rounds * batch - 1) / (rounds * batch)) >= (size_t)0x7FFFFFFF) return TT_ERR_ARG;
    P.rounds = (u32)rounds; P.parts = (u32)((bytes + rounds * batch - 1) / (rounds * batch));
    TT_TRY(dtype == TT_BF16 ? launch_logprobs_grad<__nv_bfloat16>(P, (cudaStream_t)stream) : dtype == TT_FP16 ? launch_logprobs_grad<__half>(P, (cudaStream_t)stream)
                            : launch_logprobs_grad<float>(P, (cudaStream_t)stream));
    return TT_OK;
}
