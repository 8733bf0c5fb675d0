// What the kernels on rows and weights in 8-bit integers share.
//
// An element is a code c = -127..127 and stands for s c, with one fp32 scale s for a row of activations or the weights of an output.
// Products are exact sums of 32-bit integers, whatever their order: |c c'| <= 2^14 (codes of the caller's own may be -128), below 2^17 inputs.
//
// v_mfma_i32_16x16x64_i8 (D = A[16x64] B[64x16] + C), lane (r = l % 16, g = l / 16): A: row r, k = 16 g .. 16 g + 15 (16 bytes); B: the same of
// column r; D: rows 4 g .. 4 g + 3 of column r. The first operand is weights (a row is an output), the second rows of activations: a lane's
// four results are neighbours in memory.
#pragma once

#include "four_bit.h"

namespace laser {

typedef int int4_t __attribute__((ext_vector_type(4)));

constexpr int kQ8Pad = 128;                          // rows of codes lie multiples of this many bytes apart
constexpr int kQ8MaxK = (1 << 17) - 1;
constexpr int kQ8MaxRows = 65535 * 32;

__device__ inline int4_t mfma_i8(const u32x4& a, const u32x4& b, int4_t c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(int4_t, a), __builtin_bit_cast(int4_t, b), c, 0, 0, 0);
}

// A launch without the configuration stack of <<<>>>: 2.2 us of the host's time instead of 2.4. What went wrong is for hipGetLastError.
template <class... P, class... A>
inline void launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t stream, A... args) {
    static_assert(sizeof...(P) == sizeof...(A));
    [&](P... p) {
        void* at[] = {(void*)&p...};
        (void)hipLaunchKernel((const void*)kernel, grid, block, at, 0, stream);
    }(args...);
}

// Rows into 8 bits, with or without the norm before it; arguments have been checked.
struct Q8Args {
    const void* x; const void* res; void* res_out;   // res, res_out: NULL without a residual
    const float* gain;                               // NULL: no norm
    int8_t* codes; float* scales;
    int64_t x_stride, res_stride, res_out_stride, codes_stride;      // elements
    int64_t part_stride;                             // x is the sum of n_part fp32 arrays, this many elements apart (1: one array of any type)
    int M, N, n_part;
    float eps;
};
int launch_q8(const Q8Args& a, int dtype, int res_dtype, hipStream_t stream);

// A matrix of 8-bit weights: fragments of 16 outputs x 64 inputs, a kilobyte each as the lanes of a wave hold it (16 bytes of lane 0, of lane 1, ..),
// [Kp / 64][rows / 16], Kp = Kd rounded up to 256; then the scales of the rows. Rows are outputs, up to a multiple of 16 with zeros; of a gated
// matrix 16 gate outputs, the 16 up outputs that belong to them, and so on.
struct W8 { int N, Kd, gated, outs, rows, Kp; uint8_t* codes; float* scales; int far; };   // outs: columns of a result; far: see w8_few.h
// dtype: of the results, [M][outs]
int launch_w8(const W8* w, const int8_t* x, int64_t x_stride, const float* x_scales, int M, int dtype, void* out, int64_t out_stride, hipStream_t stream);

// Whether M rows of a_row bytes every a_step bytes share no byte with M rows of b_row bytes every b_step.
bool rows_apart(const void* a, int64_t a_row, int64_t a_step, const void* b, int64_t b_row, int64_t b_step, int64_t M);

}  // namespace laser
