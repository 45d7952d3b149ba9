// C ABI of the scores of token ids (see include/toktier.h): tt_logprobs and its gradient.  Nothing here synchronises or allocates.
#include "../../include/toktier.h"
#include "tt_scores.cuh"

static size_t score_size(int dtype) { return dtype == TT_FP32 ? 4 : 2; }

// What both entry points check of their arguments.
static int score_args(const void* logits, int dtype, size_t n_rows, size_t n_vocab, size_t row_stride, float scale, const int32_t* ids,
                      const int64_t* ids_off, size_t n_docs, const int32_t* status_out) {
    if (dtype != TT_BF16 && dtype != TT_FP16 && dtype != TT_FP32) return TT_ERR_ARG;
    if (!status_out || (n_rows && (!logits || !ids)) || !n_vocab || n_vocab >= ((size_t)1 << 31) || n_rows >= ((size_t)1 << 24)) return TT_ERR_ARG;
    if (row_stride < n_vocab || row_stride >= ((size_t)1 << 38) || ((uintptr_t)logits & (score_size(dtype) - 1)) != 0) return TT_ERR_ARG;
    if (!(scale > 0.0f && scale <= 0x1p100f) || (ids_off == nullptr && n_docs != 0) || n_docs >= ((size_t)1 << 31)) return TT_ERR_ARG;
    return TT_OK;
}

template <typename T>
static cudaError_t launch_logprobs(const ScoreParams& P, unsigned ctas, cudaStream_t st) {
    const auto kernel = P.top_k ? (P.rank ? k_logprobs<T, true, true> : k_logprobs<T, true, false>) : P.rank ? k_logprobs<T, false, true> : k_logprobs<T, false, false>;
    return host_launch(kernel, ((unsigned)P.n_rows + 1) * ctas, SCORE_NT, ctas, 0, st, P);
}

extern "C" int tt_logprobs(const void* logits, int dtype, size_t n_rows, size_t n_vocab, size_t row_stride, float scale, const int32_t* ids,
                           const int64_t* ids_off, size_t n_docs, size_t top_k, void* stream, float* logprob_out, float* lse_out, float* entropy_out,
                           int32_t* rank_out, int32_t* top_ids_out, float* top_logprob_out, int32_t* status_out) {
    const int rc = score_args(logits, dtype, n_rows, n_vocab, row_stride, scale, ids, ids_off, n_docs, status_out);
    if (rc != TT_OK) return rc;
    if ((n_rows && !logprob_out) || top_k > TT_TOP_MAX || top_k > n_vocab) return TT_ERR_ARG;
    if (top_k ? n_rows && (!top_ids_out || !top_logprob_out) : top_ids_out || top_logprob_out) return TT_ERR_ARG;
    ScoreParams P;
    P.logits = logits; P.n_rows = n_rows; P.stride = row_stride; P.n_vocab = (u32)n_vocab; P.top_k = (u32)top_k; P.scale = scale;
    P.ids = ids; P.ids_off = (const long long*)ids_off; P.n_docs = n_docs;
    P.logprob = logprob_out; P.lse = lse_out; P.entropy = entropy_out; P.rank = rank_out; P.top_ids = top_ids_out; P.top_lp = top_logprob_out;
    P.status_out = status_out;
    P.scale2 = (float)((double)scale * 1.4426950408889634);
    const int sms = host_sm_count();
    if (!sms) return TT_ERR_CUDA;
    // CTAs of a row: as many as fill the GPU's places, while each has 16 KB of the row
    unsigned ctas = 1;
    while (ctas < SCORE_CLUSTER && (size_t)ctas * 2 * n_rows <= (size_t)sms * SCORE_CTAS && n_vocab * score_size(dtype) >= (size_t)ctas * 2 * 16384) ctas *= 2;
    TT_TRY(dtype == TT_BF16 ? launch_logprobs<__nv_bfloat16>(P, ctas, (cudaStream_t)stream) : dtype == TT_FP16 ? launch_logprobs<__half>(P, ctas, (cudaStream_t)stream)
                            : launch_logprobs<float>(P, ctas, (cudaStream_t)stream));
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
    if (grad_stride < n_vocab || grad_stride >= ((size_t)1 << 38) || ((uintptr_t)grad_out & (score_size(dtype) - 1)) != 0) return TT_ERR_ARG;
    if (n_rows && grad_out == logits && grad_stride != row_stride) return TT_ERR_ARG;
    ScoreGradParams P;
    P.logits = logits; P.n_rows = n_rows; P.stride = row_stride; P.grad_stride = grad_stride; P.n_vocab = (u32)n_vocab; P.scale = scale;
    P.ids = ids; P.ids_off = (const long long*)ids_off; P.n_docs = n_docs;
    P.lse = lse; P.entropy = entropy; P.g = grad_logprob; P.h = grad_entropy; P.grad = grad_out; P.status_out = status_out;
    const int sms = host_sm_count();
    if (!sms) return TT_ERR_CUDA;
    // a CTA takes up to four batches of 16 KB, fewer where that leaves places on the GPU (five CTAs on an SM) empty
    const size_t batch = (size_t)SCORE_GRAD_NT * SCORE_U * 16, bytes = n_vocab * score_size(dtype), places = (size_t)sms * 5;
    size_t rounds = 4;
    while (rounds > 1 && n_rows * ((bytes + rounds * batch - 1) / (rounds * batch)) < places) rounds /= 2;
    P.rounds = (u32)rounds; P.parts = (u32)((bytes + rounds * batch - 1) / (rounds * batch));
    TT_TRY(dtype == TT_BF16 ? launch_logprobs_grad<__nv_bfloat16>(P, (cudaStream_t)stream) : dtype == TT_FP16 ? launch_logprobs_grad<__half>(P, (cudaStream_t)stream)
                            : launch_logprobs_grad<float>(P, (cudaStream_t)stream));
    return TT_OK;
}
