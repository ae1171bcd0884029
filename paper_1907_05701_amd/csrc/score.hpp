// Row operators of scoring (score.hip), as the heads launch them.
#pragma once

#include "common.hpp"

// What is asked of rows of K classes, or what their gradient is taken from; BLSTM_OK or an error code (message set).
int check_scores(const softmax_scores* q, int32_t K, const char* fn);
int check_score_grads(const softmax_score_grads* g, int32_t K, const char* fn);

// The same for rows from r0 on.
softmax_scores scores_from(const softmax_scores& q, int64_t r0);
softmax_score_grads score_grads_from(const softmax_score_grads& g, int64_t r0);

// M rows of logits (type TI).
template <typename TI>
int score_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, const softmax_scores& q, hipStream_t stream);

// dlogits (type TO) of M rows; `pad` columns behind K are set to 0.
template <typename TI, typename TO>
int score_grad_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, const softmax_score_grads& g, TO* dlogits,
                    int64_t ldd, int32_t pad, hipStream_t stream);
