// Argument blocks and launchers of the operators in 8-bit integers (see cats.h for what they compute).
#pragma once
#include "common.hpp"

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- rows in 8 bits
// What a row is before it is quantised: ROWS_PLAIN the source row; ROWS_NORM (src + delta) normalised and
// times gain; ROWS_SWIGLU silu(first half of the source row) * second half.
enum { ROWS_PLAIN = 0, ROWS_NORM = 1, ROWS_SWIGLU = 2 };
struct QuantRowsArgs {
    const void* src;       // float32 or bf16 (ROWS_NORM: float32)
    const void* delta;     // ROWS_NORM, optional
    const bf16_t* gain;    // ROWS_NORM: [cols]
    float* x_out;          // ROWS_NORM with delta: the updated rows (may be src)
    int8_t* q;
    float* scale;          // [rows]
    int64_t src_ld, delta_ld, x_out_ld, q_ld;   // elements from one row to the next
    int rows, cols;
    float eps;
    int src_type, delta_type;   // CATS_F32, CATS_BF16
};
// kind: ROWS_*.  Nothing is enqueued for no rows.
void launch_quant_rows(const QuantRowsArgs& a, int kind, int n_cus, hipStream_t st);

// ---------------------------------------------------------------- product
// Packed 8-bit weights: rows in blocks of 16 and columns in chunks of 64, both filled up with zeros; the kilobyte
// of block rb and chunk c starts at (rb * chunks + c) * 1024 and holds, for lane l < 64, the 16 values
// W[16 rb + l % 16][64 c + 16 (l / 16) .. + 15]: a wave's operand of the 16x16x64 matrix instruction in one load.
constexpr int QPACK_ROWS = 16, QPACK_COLS = 64, QPACK_FRAG = QPACK_ROWS * QPACK_COLS;
struct QuantLinearArgs {
    const int8_t* x;       // [rows][x_ld]
    const float* x_scale;  // [rows]
    const int8_t* w;       // packed
    const float* w_scale;  // [cols]
    void* y;               // [rows][y_ld], float32 or bf16
    int64_t x_ld, y_ld;
    int rows, cols, inner;
    int chunks;            // inner in chunks of 64
    int y_type;
};
void launch_quant_linear(const QuantLinearArgs& a, int n_cus, hipStream_t st);

// Compute units of the current device (0: it could not be asked).
int quant_cus();
