// Rows of 8-bit integers: layout and packing shared by the translation units that hold and multiply them.  The format is described in include/galv.h.
#pragma once

#include "galv_mx.cuh"

constexpr float kI8Least = 7.888609052210118e-31f;        // 2^-100: a row's largest magnitude counts as this at least, so that its scale's inverse is a number
inline int64_t i8_pitch(int64_t cols) { return (cols + 15) / 16 * 16; }      // bytes of a row of codes
// The same where a product packs its tokens for itself: whole sectors.  Bulk copies of rows that start in the middle of one take longer (2711 x 7803, 5008 columns: 101 us, 5024 84).
inline int64_t i8_pitch_within(int64_t cols) { return (cols + 31) / 32 * 32; }

cudaError_t galv_i8_pack_launch(int num_sms, int64_t rows, int64_t cols, const void* x, int64_t stride, int32_t dtype, int8_t* codes, int64_t pitch, float* scales, cudaStream_t st);
