// Product of 8-bit integers with a scale for each row of X and each output column:
//   y[t][n] = (sum over k of X[t][k] W[n][k]) * x_scale[t] * w_scale[n].
// The sums are whole numbers in 32 bits and exact (inner <= CATS_QUANT_MAX_INNER), so neither the order of the
// summation nor the split of the work changes a result.
#include <algorithm>
#include <atomic>

#include "quant.hpp"
#include "quant_choice.hpp"

namespace {

// Operands of the 16x16x64 matrix instruction: lane l supplies row l % 16 and the 16 values from 16 (l / 16) on, of both
// operands; register r of lane l of the result is D[row 4 (l / 16) + r of the first][row l % 16 of the second].  The
// weights are the first operand: a lane's four results are neighbouring columns of y.

// From one row to some hundreds.  A workgroup owns a tile of 16 MB rows and 16 NB columns; its KW waves take turns at the steps
// of 128 values of k and add up their sums through LDS at the end.  Each wave keeps the rows of NS and the weights of NW of its steps
// in rings of LDS that nobody else touches: it waits for its own copies only, reads a step's fragments, sends for what takes their
// place, and multiplies; there is no barrier before the sums meet.
// Bound by the operands' way into the compute unit: with few rows the weights' from memory (22016 x 4096 weights: 14.7 us with
// one row = 6.1 TB/s, 19.5 with 63 rows), with more the rows' and the weights' from the L2 (see quant_choice.hpp).
// Splitting k over the waves, not over workgroups, needs no scratch memory and no second launch; X and W both go through LDS because
// then every wait is for a count of copies that is known here (a load that the compiler sees in between makes it wait for
// more), and eight lanes copy a whole line of a row of X.
// Two steps in a wave's rings where one tile a compute unit is all there is and its steps are small: more of the weights are under
// way (one row, 4096 x 11008 weights from memory: 10.4 -> 8.9 us; nothing lost from the cache); of the weights alone in the middle
// sizes (63 x 8192 x 11008 from memory 26.2 -> 23.1 us).  One step and more workgroups a compute unit for the larger ones (64 x 64:
// 512 x 4096 x 4096 18.1 against 18.6 us with two steps of weights), unless the weights come past the caches.
// A compute unit takes in rows at 63 GB/s from the L2 and weights at 22 from memory, and the two times add up: its requests come
// back in order.  So 128 x 15360 x 5120 with weights from memory takes 25 us, 64 rows 18.7, one 14.
// ONCE: the weights are copied past the caches (see launch_split).
template <int MB, int NB, int KW, int NS, int NW, bool ONCE>
__global__ __launch_bounds__(64 * KW) void cats_quant_linear_split(QuantLinearArgs a, QuantGrid grid) {
    constexpr int UNDER_WAY = (NS - 1) * 2 * MB + (NW - 1) * 2 * NB;   // copies of 1 KB behind a step's own
    static_assert(NS <= 2 && NW - NS <= 1 && NW >= NS && UNDER_WAY < 64, "counts of the waits");
    constexpr int OWN = (NS * MB + NW * NB) * 2048, RING = KW * OWN;
    // the waves' sums meet in parts of PB row blocks that fit where the ring was
    constexpr int PB = KW * MB * NB * 1024 <= RING ? MB : MB / 2;
    static_assert(KW * PB * NB * 1024 <= RING && MB % PB == 0, "a part of the sums fits the ring");
    __shared__ __align__(1024) int8_t s_lds[RING];
    __shared__ __align__(16) float s_sx[16 * MB], s_sw[16 * NB];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int mt, nt;
    // all arguments at once: loaded where they are used, they are several scalar round trips one behind the other
    asm volatile("" ::"s"(a.x), "s"(a.x_scale), "s"(a.w), "s"(a.w_scale), "s"(a.x_ld), "s"(a.rows), "s"(a.cols), "s"(a.inner), "s"(a.chunks),
                 "s"(a.pieces), "s"(grid.all), "s"(grid.band), "s"(grid.m_tiles));
    quant_tile_of(grid, blockIdx.x, mt, nt);
    const int n_rb = (a.cols + QPACK_ROWS - 1) / QPACK_ROWS;
    const int k_last = (a.inner - 1) / 16 * 16;
    int step0 = 0, steps = (a.inner + 127) >> 7;   // (the packed weights may have one step of zeros more)
    if (a.pieces > 1) {
        const int piece = fast_div(nt, grid.by_n), all = steps;
        nt -= piece * grid.n_tiles;
        step0 = all * piece / a.pieces;
        steps = all * (piece + 1) / a.pieces - step0;
        a.y = static_cast<float*>(a.y) + static_cast<int64_t>(piece) * a.rows * a.y_ld;
    }
    const int mine = (steps - wave + KW - 1) / KW;

    // the scales, for when the sums are ready
    static_assert(MB <= 4 * KW && NB <= 4 * KW, "one of each a thread");
    const int tid = threadIdx.x;
    const float sx_own = a.x_scale[min(mt * 16 * MB + min(tid, 16 * MB - 1), a.rows - 1)];
    const float sw_own = a.w_scale[min(nt * 16 * NB + min(tid, 16 * NB - 1), a.cols - 1)];
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;   // places of X in LDS: see cats_quant_linear_tiles
    const int8_t* x0 = a.x + static_cast<int64_t>(mt) * 16 * MB * a.x_ld;
    uint32_t xo[2 * MB];
#pragma unroll
    for (int i = 0; i < 2 * MB; ++i) xo[i] = min(i * 8 + (lane >> 3), a.rows - 1 - mt * 16 * MB) * static_cast<int>(a.x_ld);
    const int8_t* wp[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) wp[j] = a.w + static_cast<int64_t>(min(nt * NB + j, n_rb - 1)) * a.chunks * QPACK_FRAG;
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&s_lds[0])) + wave * OWN;
    auto fetch_w = [&](int i, int slot) {   // for the i-th of this wave's steps
        const int s = step0 + wave + i * KW;
        const uint32_t to = lds0 + slot * NB * 2048;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            copy_to_lds<ONCE>(wp[j] + s * 2048, lane * 16, to + j * 2048);
            copy_to_lds<ONCE>(wp[j] + s * 2048 + 1024, lane * 16, to + j * 2048 + 1024);
        }
    };
    auto fetch_x = [&](int i, int slot) {
        const int k = min((step0 + wave + i * KW) * 128 + piece, k_last);
        const uint32_t to = lds0 + (NW * NB + slot * MB) * 2048;
#pragma unroll
        for (int p = 0; p < 2 * MB; ++p) copy_to_lds(x0, xo[p] + k, to + p * 1024);
    };
    i32x4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        if (i < mine) fetch_w(i, i);
        if (i < NS && i < mine) fetch_x(i, i);
    }
    int slot = 0, w_slot = 0;
    for (int i = 0; i < mine; ++i) {
        // this step's copies; all behind them are under way until the last steps
        if (mine - 1 - i >= NW - 1)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(UNDER_WAY) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const int8_t* w_from = &s_lds[0] + wave * OWN + w_slot * NB * 2048;
        const int8_t* x_from = &s_lds[0] + wave * OWN + (NW * NB + slot * MB) * 2048;
        i32x4 w[2][NB], x[2][MB];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < NB; ++j) w[h][j] = *reinterpret_cast<const i32x4*>(w_from + j * 2048 + h * 1024 + lane * 16);
#pragma unroll
            for (int b = 0; b < MB; ++b)
                x[h][b] = *reinterpret_cast<const i32x4*>(x_from + (b * 16 + r) * 128 + ((4 * h + g) ^ (r & 7)) * 16);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the fragments are in registers: their place is free
        if (i + NS < mine) fetch_x(i + NS, slot);
        if (i + NW < mine) fetch_w(i + NW, w_slot);
        slot = slot == NS - 1 ? 0 : slot + 1;
        w_slot = w_slot == NW - 1 ? 0 : w_slot + 1;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[b][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[h][j], x[h][b], acc[b][j], 0, 0, 0);
    }
    if (tid < 16 * MB) s_sx[tid] = sx_own;
    if (tid < 16 * NB) s_sw[tid] = sw_own;
    i32x4* sums = reinterpret_cast<i32x4*>(&s_lds[0]);
#pragma unroll
    for (int b0 = 0; b0 < MB; b0 += PB) {
        __syncthreads();   // nobody needs its ring, or the part before, any more
#pragma unroll
        for (int b = 0; b < PB; ++b)
#pragma unroll
            for (int j = 0; j < NB; ++j) sums[(wave * PB * NB + b * NB + j) * 64 + lane] = acc[b0 + b][j];
        __syncthreads();
        for (int f = wave; f < PB * NB; f += KW) {
            i32x4 sum = sums[f * 64 + lane];
#pragma unroll
            for (int q = 1; q < KW; ++q) sum += sums[(q * PB * NB + f) * 64 + lane];
            const int t = 16 * (b0 + f / NB) + r, n = 16 * (f % NB) + 4 * g;   // in the tile
            if (mt * 16 * MB + t < a.rows && nt * 16 * NB + n < a.cols)
                quant_store4(a, mt * 16 * MB + t, nt * 16 * NB + n, quant_scaled(sum, s_sx[t], *reinterpret_cast<const f32x4*>(s_sw + n)));
        }
    }
}

// Weights that will hardly be found in the 256 MB cache in front of the memory by the next call are copied past the caches, which then
// keep other things: a matrix that one row tile reads and that takes a third of that size or more, so that three like it do not stay
// there, and whatever the caller calls cold, also for two tiles of up to 32 rows (which read it side by side; larger pairs lose by
// it).  The size is all that a call knows of its weights' whereabouts; us through the caches -> past them, matrices in turn that
// come from memory | one or two that the cache holds:
//   79 MB (15360 x 5120), below the border: one row 15.6 -> 14.2 | 13.1 -> 12.4 to 13.3, 63 rows 21.2 -> 18.3 | 16.1 -> 16.3 to 17.3,
//     128 rows 28.0 -> 24.5 | 19.7 -> 22.7 to 23.6; three of them, 236 MB, 63 rows 16.1 -> 17.6
//   90 MB (22016 x 4096): one row 17.3 -> 16.0 | 14.7 -> 14.0 to 14.6, 63 rows 22.6 -> 19.8 | 18.5 -> 17.8 to 18.8, 128 rows
//     28.4 -> 25.2 | 22.4 -> 23.3 to 24.1; three of them, 271 MB, even: 63 rows 19.1 -> 19.3
//   205 MB (40000 x 5120): one row 37.3 -> 33.2 | 29.4 -> 31.4, 63 rows 50.7 -> 45.5 | 37.8 -> 43.0
// Smaller ones gain less from memory and lose more from the cache (34 MB, 8192 x 4096, one row 7.7 -> 7.2 | 4.1 -> 5.9).
constexpr int64_t CACHE_BYTES = int64_t{256} << 20;
template <int MB, int NB, int KW, int NS, int NW>
void launch_split(const QuantLinearArgs& a, int, hipStream_t st) {
    const QuantGrid grid = quant_grid(a.rows, a.cols, a.pieces, 16 * MB, 16 * NB);
    const bool once = a.cold ? grid.m_tiles <= (MB <= 2 ? 2 : 1) : grid.m_tiles == 1 && static_cast<int64_t>(a.cols) * a.inner >= CACHE_BYTES / 3;
    // weights that come past the caches, one step further ahead where the LDS holds it (63 x 27648 x 5120 30.0 -> 28.2 us)
    constexpr int ONCE_NW = NW == 1 && MB >= 4 && (MB + 2 * NB) * 2048 * KW < 156 * 1024 ? 2 : NW;
    hipLaunchKernelGGL((once ? cats_quant_linear_split<MB, NB, KW, NS, ONCE_NW, true> : cats_quant_linear_split<MB, NB, KW, NS, NW, false>),
                       dim3(grid.all), dim3(64 * KW), 0, st, a, grid);
}

// One wave moves one kilobyte: rows of 64 values in, an operand of the matrix instruction out.  vec: rows start at multiples of
// 16 bytes.  (22016 x 4096: 108 us byte by byte, 28 us with whole loads.)
__global__ __launch_bounds__(256) void cats_quant_pack(const int8_t* src, int64_t ld, int8_t* dst, int rows, int cols, int chunks,
                                                      int64_t frags, bool vec) {
    const int lane = threadIdx.x & 63;
    for (int64_t f = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); f < frags; f += static_cast<int64_t>(gridDim.x) * 4) {
        const int rb = static_cast<int>(f / chunks), c = static_cast<int>(f - static_cast<int64_t>(rb) * chunks);
        const int n = rb * QPACK_ROWS + (lane & 15), k = c * QPACK_COLS + (lane >> 4) * 16;
        uint32_t v[4] = {0, 0, 0, 0};
        if (n < rows) {
            const int8_t* p = src + n * ld + k;
            if (vec && k + 16 <= cols) {
                const u32x4 whole = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = whole[e];
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k + e < cols) v[e >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(p[e])) << 8 * (e & 3);
            }
        }
        *reinterpret_cast<u32x4*>(dst + f * QPACK_FRAG + lane * 16) = u32x4{v[0], v[1], v[2], v[3]};
    }
}

int64_t frags_of(int32_t rows, int32_t cols) {
    return (static_cast<int64_t>(rows) + QPACK_ROWS - 1) / QPACK_ROWS * qpack_chunks(cols);
}
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool aligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

// Compute units of the current device.
hipError_t quant_cus(int& n) {
    constexpr int MAX_DEVICES = 64;
    static std::atomic<int> known[MAX_DEVICES];   // zero: not asked yet
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const bool keep = dev >= 0 && dev < MAX_DEVICES;
    n = keep ? known[dev].load(std::memory_order_relaxed) : 0;
    if (n) return hipSuccess;
    e = hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev);
    if (e == hipSuccess && n < 1) e = hipErrorInvalidDevice;
    if (e == hipSuccess && keep) known[dev].store(n, std::memory_order_relaxed);
    return e;
}

}  // namespace

void launch_quant_linear(const QuantLinearArgs& a, int n_cus, hipStream_t st) {
    if (a.rows < 1) return;
    static constexpr void (*LAUNCH[])(const QuantLinearArgs&, int, hipStream_t) = {
        launch_split<1, 1, 8, 2, 2>, launch_split<1, 2, 8, 1, 1>, launch_split<1, 3, 8, 1, 1>, launch_split<2, 1, 8, 2, 2>,
        launch_split<2, 2, 8, 2, 2>, launch_split<2, 3, 4, 1, 2>, launch_split<2, 4, 4, 1, 2>, launch_split<2, 6, 4, 1, 2>,
        launch_split<2, 7, 4, 1, 2>, launch_split<2, 8, 4, 1, 2>, launch_split<4, 2, 4, 1, 2>, launch_split<4, 3, 4, 1, 1>,
        launch_split<4, 4, 4, 1, 1>, launch_split<4, 6, 4, 1, 1>, launch_split<4, 7, 4, 1, 1>, launch_split<4, 8, 4, 1, 1>,
        launch_split<6, 6, 4, 1, 1>, launch_split<8, 4, 4, 1, 1>, launch_split<8, 6, 4, 1, 1>, launch_split<6, 8, 4, 1, 1>,
        launch_split<8, 7, 4, 1, 1>, launch_split<8, 8, 4, 1, 1>,
        launch_quant_tiles_half_narrow, launch_quant_tiles_half, launch_quant_tiles_narrow, launch_quant_tiles};
    static_assert(sizeof(LAUNCH) / sizeof(LAUNCH[0]) == N_QUANT_TILES, "one kernel for each tile");
    if (a.tile >= 0) return LAUNCH[a.tile](a, n_cus, st);
    const QuantPlan plan = quant_plan(a.rows, a.cols, a.inner, n_cus);
    QuantLinearArgs part = a;
    part.cols = plan.cols;
    LAUNCH[plan.tile](part, n_cus, st);
    if (plan.cols == a.cols) return;
    part.cols = a.cols - plan.cols;
    part.w = a.w + static_cast<int64_t>(plan.cols / QPACK_ROWS) * a.chunks * QPACK_FRAG;
    part.w_scale = a.w_scale + plan.cols;
    part.y = static_cast<char*>(a.y) + static_cast<int64_t>(plan.cols) * (a.y_type == CATS_F32 ? 4 : 2);
    LAUNCH[plan.rest_tile](part, n_cus, st);
}

extern "C" {

size_t cats_packed_quantized_bytes(int32_t rows, int32_t cols) {
    return rows < 1 || cols < 1 ? 0 : static_cast<size_t>(frags_of(rows, cols)) * QPACK_FRAG;
}

int cats_pack_quantized_matrix(const int8_t* src, int64_t src_ld, int32_t rows, int32_t cols, int8_t* dst, void* stream) {
    if (!src || !dst || !aligned16(dst) || rows < 1 || cols < 1 || src_ld < cols) return CATS_EINVAL;
    if (cols > CATS_QUANT_MAX_INNER || rows > CATS_QUANT_MAX_ROWS) return CATS_ECAPACITY;
    const int64_t frags = frags_of(rows, cols);
    const unsigned groups = static_cast<unsigned>(std::min<int64_t>((frags + 3) / 4, 1 << 16));
    hipLaunchKernelGGL(cats_quant_pack, dim3(groups), dim3(256), 0, static_cast<hipStream_t>(stream), src, src_ld, dst, rows, cols,
                       qpack_chunks(cols), frags, aligned16(src) && src_ld % 16 == 0);
    return launch_status();
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
        x_ld >= CATS_QUANT_MAX_LD ||                             // offsets inside a tile of X: fewer than 2^31
        static_cast<int64_t>(rows) * cols > (int64_t{1} << 33))   // threads of a launch: fewer than 2^32
        return CATS_ECAPACITY;
    if (rows == 0) return CATS_OK;
    int n_cus = 0;
    const hipError_t e = quant_cus(n_cus);
    if (e != hipSuccess) {
        (void)hipGetLastError();   // the next launch is not to blame for it
        return hip_fail(e);
    }
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
    return launch_status();
}

}  // extern "C"
