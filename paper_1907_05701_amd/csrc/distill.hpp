// Row operators of distillation (distill.hip), as the head launches them.
#pragma once

#include "common.hpp"

// Arguments of either operator for rows of K classes; BLSTM_OK or an error code (message set).
int check_teacher(const softmax_teacher* t, int32_t K, const char* fn);
int check_top(int32_t k, int32_t K, float temperature, const char* fn);

// top, idx, rest of M rows of logits (type TI).
template <typename TI>
int topk_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, int32_t k, float temperature, float* top,
              int32_t* idx, float* rest, hipStream_t stream);

// row losses and dlogits (type TO) of M rows; `pad` columns behind K are set to 0.
template <typename TI, typename TO>
int distill_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, const softmax_teacher* teacher, float loss_scale,
                 float* row_loss, TO* dlogits, int64_t ldd, int32_t pad, hipStream_t stream);
