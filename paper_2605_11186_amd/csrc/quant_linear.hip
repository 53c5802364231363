// Product of 8-bit integers with a scale for each row of X and each output column:
//   y[t][n] = (sum over k of X[t][k] W[n][k]) * x_scale[t] * w_scale[n].
// The sums are whole numbers in 32 bits and exact (inner <= CATS_QUANT_MAX_INNER), so neither the order of the
// summation nor the split of the work changes a result.
#include <algorithm>

#include "quant.hpp"

namespace {

// Operands of the 16x16x64 matrix instruction: lane l supplies row l % 16 and the 16 values from 16 (l / 16) on, of both
// operands; register r of lane l of the result is D[row 4 (l / 16) + r of the first][row l % 16 of the second].  The
// weights are the first operand: a lane's four results are neighbouring columns of y.

// A workgroup owns a tile of 16 MB rows and 16 NB columns; its waves split the chunks of k among them and add up their
// sums through LDS.
template <int MB, int NB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void cats_quant_linear_rows(QuantLinearArgs a, int m_tiles) {
    __shared__ i32x4 s_acc[WAVES][MB * NB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int mt = blockIdx.x % m_tiles, nt = blockIdx.x / m_tiles;
    const int n_rb = (a.cols + QPACK_ROWS - 1) / QPACK_ROWS;
    const int k_last = (a.inner - 1) / 16 * 16;
    const int8_t* xp[MB];
    const int8_t* wp[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) xp[i] = a.x + min((mt * MB + i) * 16 + (lane & 15), a.rows - 1) * a.x_ld;
#pragma unroll
    for (int i = 0; i < NB; ++i)
        wp[i] = a.w + static_cast<int64_t>(min(nt * NB + i, n_rb - 1)) * a.chunks * QPACK_FRAG + lane * 16;
    i32x4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    for (int c = wave; c < a.chunks; c += WAVES) {
        i32x4 x[MB], w[NB];
        // past the end of a row of X the weights are zeros: any value will do there
        const int k = min(c * QPACK_COLS + (lane >> 4) * 16, k_last);
#pragma unroll
        for (int i = 0; i < NB; ++i) w[i] = *reinterpret_cast<const i32x4*>(wp[i] + static_cast<int64_t>(c) * QPACK_FRAG);
#pragma unroll
        for (int i = 0; i < MB; ++i) x[i] = *reinterpret_cast<const i32x4*>(xp[i] + k);
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j], x[i], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) s_acc[wave][i * NB + j][lane] = acc[i][j];
    __syncthreads();
    for (int f = wave; f < MB * NB; f += WAVES) {
        i32x4 sum = s_acc[0][f][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += s_acc[w][f][lane];
        const i32x4 one[1][1] = {{sum}};
        quant_store_tile<1, 1>(a, (mt * MB + f / NB) * 16 + (lane & 15), (nt * NB + f % NB) * 16 + 4 * (lane >> 4), one);
    }
}

template <int MB, int NB, int WAVES>
void launch_rows(const QuantLinearArgs& a, hipStream_t st) {
    const int m_tiles = (a.rows + 16 * MB - 1) / (16 * MB), n_tiles = (a.cols + 16 * NB - 1) / (16 * NB);
    hipLaunchKernelGGL((cats_quant_linear_rows<MB, NB, WAVES>), dim3(static_cast<unsigned>(m_tiles) * n_tiles),
                       dim3(64 * WAVES), 0, st, a, m_tiles);
}

// One wave moves one kilobyte: rows of 64 values in, an operand of the matrix instruction out.
__global__ __launch_bounds__(256) void cats_quant_pack(const int8_t* src, int64_t ld, int8_t* dst, int rows, int cols, int chunks,
                                                      int64_t frags) {
    const int lane = threadIdx.x & 63;
    for (int64_t f = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); f < frags; f += static_cast<int64_t>(gridDim.x) * 4) {
        const int rb = static_cast<int>(f / chunks), c = static_cast<int>(f - static_cast<int64_t>(rb) * chunks);
        const int n = rb * QPACK_ROWS + (lane & 15), k = c * QPACK_COLS + (lane >> 4) * 16;
        uint32_t v[4] = {0, 0, 0, 0};
        if (n < rows) {
            const int8_t* p = src + n * ld;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (k + e < cols) v[e >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(p[k + e])) << 8 * (e & 3);
        }
        *reinterpret_cast<u32x4*>(dst + f * QPACK_FRAG + lane * 16) = u32x4{v[0], v[1], v[2], v[3]};
    }
}

int64_t frags_of(int32_t rows, int32_t cols) {
    return (static_cast<int64_t>(rows) + QPACK_ROWS - 1) / QPACK_ROWS * qpack_chunks(cols);
}
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool aligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

}  // namespace

void launch_quant_linear(const QuantLinearArgs& a, int n_cus, hipStream_t st) {
    if (a.rows < 1) return;
    if (a.rows <= 16)
        launch_rows<1, 1, 8>(a, st);
    else if (a.rows >= 256 && a.x_ld < (1 << 23))
        launch_quant_linear_tiles(a, n_cus, st);
    else
        launch_rows<4, 2, 4>(a, st);
}

extern "C" {

size_t cats_packed_quantized_bytes(int32_t rows, int32_t cols) {
    return rows < 1 || cols < 1 ? 0 : static_cast<size_t>(frags_of(rows, cols)) * QPACK_FRAG;
}

int cats_pack_quantized_matrix(const int8_t* src, int64_t src_ld, int32_t rows, int32_t cols, int8_t* dst, void* stream) {
    if (!src || !dst || !aligned16(dst) || rows < 1 || cols < 1 || src_ld < cols) return CATS_EINVAL;
    if (cols > CATS_QUANT_MAX_INNER || rows > CATS_QUANT_MAX_ROWS) return CATS_ECAPACITY;
    const int64_t frags = frags_of(rows, cols);
    hipLaunchKernelGGL(cats_quant_pack, dim3(static_cast<unsigned>(std::min<int64_t>((frags + 3) / 4, 1 << 16))), dim3(256), 0, static_cast<hipStream_t>(stream),
                       src, src_ld, dst, rows, cols, qpack_chunks(cols), frags);
    return hipGetLastError() == hipSuccess ? CATS_OK : CATS_EHIP;
}

int cats_quantized_linear(const int8_t* x, int64_t x_ld, const float* x_scale, const int8_t* w_packed, const float* w_scale,
                          void* y, int32_t y_type, int64_t y_ld, int32_t rows, int32_t cols, int32_t inner, void* stream) {
    if (!x || !x_scale || !w_packed || !w_scale || !y) return CATS_EINVAL;
    if (y_type != CATS_F32 && y_type != CATS_BF16) return CATS_EINVAL;
    if (rows < 0 || cols < 1 || inner < 1 || x_ld < inner || x_ld % 16 != 0 || y_ld < cols) return CATS_EINVAL;
    if (!aligned16(x) || !aligned16(w_packed) || !aligned4(x_scale) || !aligned4(w_scale) ||
        reinterpret_cast<uintptr_t>(y) % (y_type == CATS_F32 ? 4 : 2) != 0)
        return CATS_EINVAL;
    if (inner > CATS_QUANT_MAX_INNER || rows > CATS_QUANT_MAX_ROWS || cols > CATS_QUANT_MAX_ROWS ||
        static_cast<int64_t>(rows) * cols > (int64_t{1} << 33))   // threads of a launch: fewer than 2^32
        return CATS_ECAPACITY;
    if (rows == 0) return CATS_OK;
    const int n_cus = quant_cus();
    if (!n_cus) return CATS_EHIP;
    QuantLinearArgs a{};
    a.x = x;
    a.x_ld = x_ld;
    a.x_scale = x_scale;
    a.w = w_packed;
    a.w_scale = w_scale;
    a.y = y;
    a.y_type = y_type;
    a.y_ld = y_ld;
    a.rows = rows;
    a.cols = cols;
    a.inner = inner;
    a.chunks = qpack_chunks(inner);
    launch_quant_linear(a, n_cus, static_cast<hipStream_t>(stream));
    return hipGetLastError() == hipSuccess ? CATS_OK : CATS_EHIP;
}

}  // extern "C"
