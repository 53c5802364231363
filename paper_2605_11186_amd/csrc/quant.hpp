// Argument blocks and launchers of the operators in 8-bit integers (see cats.h for what they compute).
#pragma once
#include "common.hpp"
#include "fast_div.hpp"

typedef int i32x4 __attribute__((ext_vector_type(4)));

// CATS_EHIP; cats_strerror then gives the text of e.  Hidden: a name like any other's, which another library must not take the place of.
__attribute__((visibility("hidden"))) int hip_fail(hipError_t e);
// The status behind a launch.
inline int launch_status() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CATS_OK : hip_fail(e);
}

// ---------------------------------------------------------------- rows in 8 bits
// What a row is before it is quantised: ROWS_PLAIN the source row; ROWS_NORM (src + delta) normalised and
// times gain; ROWS_SWIGLU silu(first half of the source row) * second half; ROWS_MERGED the single row that the chunks of a
// single query's attention make (see DecodeAttnArgs), rounded to bf16.
enum { ROWS_PLAIN = 0, ROWS_NORM = 1, ROWS_SWIGLU = 2, ROWS_MERGED = 3 };
struct QuantRowsArgs {
    const void* src;       // float32 or bf16 (ROWS_NORM: float32; ROWS_MERGED: DecodeAttnArgs.po)
    const void* delta;     // ROWS_NORM, optional
    int delta_pieces;      // more than one: float32 [delta_pieces][rows][delta_ld], to be added up first (QuantLinearArgs.pieces)
    const bf16_t* gain;    // ROWS_NORM: [cols]
    float* x_out;          // ROWS_NORM with delta: the updated rows (may be src)
    int8_t* q;
    float* scale;          // [rows]
    int64_t src_ld, delta_ld, x_out_ld, q_ld;   // elements from one row to the next
    int rows, cols;
    float eps;
    int src_type, delta_type;   // CATS_F32, CATS_BF16
    const float* ml;       // ROWS_MERGED: DecodeAttnArgs.pml
    int n_chunks, head_dim;
};
// kind: ROWS_*.  Nothing is enqueued for no rows.
void launch_quant_rows(const QuantRowsArgs& a, int kind, hipStream_t st);

// ---------------------------------------------------------------- product
// Packed 8-bit weights: rows in blocks of 16 and columns in chunks of 64, a multiple of four of them, filled up with zeros; the
// kilobyte of block rb and chunk c starts at (rb * chunks + c) * 1024 and holds, for lane l < 64, the 16 values
// W[16 rb + l % 16][64 c + 16 (l / 16) .. + 15]: a wave's operand of the 16x16x64 matrix instruction in one load.
constexpr int QPACK_ROWS = 16, QPACK_COLS = 64, QPACK_FRAG = QPACK_ROWS * QPACK_COLS;
inline int qpack_chunks(int cols) { return static_cast<int>((static_cast<int64_t>(cols) + 255) / 256 * 4); }
struct QuantLinearArgs {
    const int8_t* x;       // [rows][x_ld]
    const float* x_scale;  // [rows]
    const int8_t* w;       // packed
    const float* w_scale;  // [cols]
    void* y;               // [rows][y_ld], float32 or bf16
    int64_t x_ld, y_ld;
    int rows, cols, inner;
    int chunks;            // packed chunks of 64 along inner, a multiple of four
    int y_type;
    int pieces = 1;        // of the inner length, the sums of each times the scales in y + piece * rows * y_ld; float32, at most
                           // QUANT_MAX_PIECES, and only with a tile of cats_quant_linear_split (quant_choice)
    int tile = -1;         // one of QUANT_TILES, or -1: the best for one piece
    bool cold = false;     // the caller reads more weights than the caches hold before it reads these again
};
constexpr int QUANT_MAX_PIECES = 3;
void launch_quant_linear(const QuantLinearArgs& a, int n_cus, hipStream_t st);
void launch_quant_tiles(const QuantLinearArgs& a, int n_cus, hipStream_t st);               // tiles of 256 x 256
void launch_quant_tiles_narrow(const QuantLinearArgs& a, int n_cus, hipStream_t st);        // of 256 rows x 192 columns
void launch_quant_tiles_half(const QuantLinearArgs& a, int n_cus, hipStream_t st);          // of 128 rows x 256 columns
void launch_quant_tiles_half_narrow(const QuantLinearArgs& a, int n_cus, hipStream_t st);   // of 128 rows x 192 columns

// 64 lanes copy 16 bytes each from base + their own offset to 1024 consecutive bytes of LDS (at byte `lds`), with no
// register between.  Counted in vmcnt like a load; the compiler does not see it and waits for nothing on its account.
// ONCE: of bytes that are not wanted again soon and that the caches need not keep.
template <bool ONCE = false>
__device__ __forceinline__ void copy_to_lds(const int8_t* base, uint32_t offset, uint32_t lds) {
    if constexpr (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}

// The tiles of a launch, n_tiles of them side by side for each piece, and what they are divided by.
constexpr int QUANT_BAND = 4;
struct QuantGrid {
    int m_tiles, n_tiles, all;         // all: m_tiles * n_tiles * pieces
    int band;                          // tiles of a band of QUANT_BAND row tiles
    FastDiv by_band, by_last, by_n;    // by_last: the row tiles of the last band, if it has fewer
};
inline QuantGrid quant_grid(int rows, int cols, int pieces, int bm, int bn) {
    QuantGrid g;
    g.m_tiles = (rows + bm - 1) / bm;
    g.n_tiles = (cols + bn - 1) / bn;
    g.all = g.m_tiles * g.n_tiles * pieces;
    g.band = QUANT_BAND * g.n_tiles * pieces;
    g.by_band = make_fast_div(g.band);
    g.by_last = make_fast_div(g.m_tiles % QUANT_BAND);
    g.by_n = make_fast_div(g.n_tiles);
    return g;
}
// Tile number `index` (of a launch's workgroups).  Workgroup b runs on XCD b % 8: an XCD takes a run of tiles, in bands of 4 row
// tiles (a run of tiles of one band shares rows of X and of W in the XCD's L2).
__device__ __forceinline__ void quant_tile_of(const QuantGrid& g, int index, int& mt, int& nt) {
    const int xcd = index & 7;
    const int id = xcd * (g.all >> 3) + min(xcd, g.all & 7) + (index >> 3);
    const int band = fast_div(id, g.by_band), in_band = id - band * g.band;
    const int band_rows = min(QUANT_BAND, g.m_tiles - band * QUANT_BAND);
    nt = band_rows == QUANT_BAND ? in_band / QUANT_BAND : static_cast<int>(fast_div(in_band, g.by_last));
    mt = __builtin_amdgcn_readfirstlane(band * QUANT_BAND + in_band - nt * band_rows);
    nt = __builtin_amdgcn_readfirstlane(nt);
}

// Four neighbouring columns of y from their sums; sums times the row's scale first, then the columns' ones.
__device__ __forceinline__ f32x4 quant_scaled(i32x4 v, float sx, f32x4 sw) {
    return f32x4{static_cast<float>(v[0]), static_cast<float>(v[1]), static_cast<float>(v[2]), static_cast<float>(v[3])} * sx * sw;
}
// One store where the rows of y keep its alignment and all four columns exist.
__device__ __forceinline__ void quant_store4(const QuantLinearArgs& a, int t, int n, f32x4 y) {
    const int size = a.y_type == CATS_F32 ? 4 : 2;
    const bool whole = ((reinterpret_cast<uintptr_t>(a.y) | static_cast<uint64_t>(a.y_ld) * size) & (4 * size - 1)) == 0;
    char* p = static_cast<char*>(a.y) + (t * a.y_ld + n) * size;
    const uint2 b = make_uint2(pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3]));
    if (whole && n + 4 <= a.cols) {
        if (size == 4)
            *reinterpret_cast<f32x4*>(p) = y;
        else
            *reinterpret_cast<uint2*>(p) = b;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (n + e >= a.cols) break;
        if (size == 4)
            reinterpret_cast<float*>(p)[e] = y[e];
        else
            reinterpret_cast<bf16_t*>(p)[e] = static_cast<bf16_t>((e & 2 ? b.y : b.x) >> 16 * (e & 1));
    }
}
