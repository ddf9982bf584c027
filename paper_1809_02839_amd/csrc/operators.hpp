// The operators of the public interface that stand by themselves (rotary
// positions, masked attention, 8-bit activation checkpoints, linear layers in 8
// bits): argument checks and launches. Failures are thrown as StageError.
#pragma once

#include "stage.hpp"

namespace spx {

void run_rotary(const spectrain_rotary_desc* d, const void* x, const int32_t* positions, int inverse, void* out,
                hipStream_t s);

size_t attention_workspace(const spectrain_attention_desc* d, bool backward);
// The checks that a forward or backward makes of its masks.
void check_attention_masks(const spectrain_attention_desc* d, const spectrain_attention_masks* masks);
void run_attention_forward(const spectrain_attention_desc* d, const spectrain_attention_masks* masks, const void* q,
                           const void* k, const void* v, void* out, float* lse, void* ws, size_t ws_bytes,
                           hipStream_t s);
void run_attention_backward(const spectrain_attention_desc* d, const spectrain_attention_masks* masks, const void* q,
                            const void* k, const void* v, const void* out, const float* lse, const void* dout,
                            void* dq, void* dk, void* dv, void* ws, size_t ws_bytes, hipStream_t s);

// x given: pack; out given: restore.
void run_checkpoint(int dtype, int64_t rows, int64_t cols, const void* x, int64_t ld, uint8_t* codes, uint8_t* scales,
                    void* out, hipStream_t s);

void run_blocks_pack(const spectrain_blocks_desc* d, const void* x, uint8_t* codes, uint8_t* scales, uint8_t* t_codes,
                     uint8_t* t_scales, hipStream_t s);
void run_blocks_restore(const spectrain_blocks_desc* d, const uint8_t* codes, const uint8_t* scales, void* out,
                        hipStream_t s);

size_t rms_norm_workspace(const spectrain_rms_norm_desc* d);
void run_rms_norm_forward(const spectrain_rms_norm_desc* d, const void* x, const void* residual, const void* weight,
                          void* sum, void* y, uint8_t* codes, uint8_t* scales, float* rstd, hipStream_t s);
void run_rms_norm_backward(const spectrain_rms_norm_desc* d, const void* dy, const void* h, const void* weight,
                           const float* rstd, const void* dsum, void* dx, float* dweight, void* ws, size_t ws_bytes,
                           hipStream_t s);

size_t product_workspace(const spectrain_product_desc* d);
void run_product(const spectrain_product_desc* d, const uint8_t* a_codes, const uint8_t* a_scales,
                 const uint8_t* b_codes, const uint8_t* b_scales, const void* bias, const void* mask, void* out,
                 void* ws, size_t ws_bytes, hipStream_t s);

}  // namespace spx
