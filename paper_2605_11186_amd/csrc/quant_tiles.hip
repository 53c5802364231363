// The product of 8-bit integers for many rows (prompts): bound by the matrix instructions.  4096 x 4096 x 11008 takes 139 us =
// 2.65 Pop/s on tiles of 256 x 256 (the library's product of 8-bit integers 147 to 152 us; the bare instruction, fed from registers,
// reaches 4.0 Pop/s at the clock that this power allows).  The matrix units are busy two thirds of the time; what they wait for
// is operands from the L2: timing copies without the weight loads take 13 % less, without the copies of X 12 %, without the step's
// barrier or the reads from LDS as long.  With operands of zeros it takes 130 us: the rest of the way is the clock.
#include <algorithm>
#include <type_traits>

#include "quant.hpp"

namespace {

// A workgroup of WM x WN waves takes tiles of BM = 16 WM MB rows of X and BN = 16 WN NB columns one after the other, a wave MB x NB
// blocks of 16 x 16 of each.  X passes through LDS in steps of 128 values of k, NS - 1 steps ahead; W's packed fragments go
// straight from memory into the registers of the matrix instruction: both through LDS would take all of its 128 bytes a cycle.
// Eight waves, two a SIMD: four waves of 128 x 128 each read less from LDS but wait alone (157 against 146 us), and the
// 32x32x32 instruction, whose operands are runs of 256 bytes of the packed weights, is slower under load (153 against 144 us).
template <int WM, int WN, int MB, int NB, int NS, int WS>
__global__ __launch_bounds__(64 * WM * WN) void cats_quant_linear_tiles(QuantLinearArgs a, QuantGrid grid) {
    constexpr int WAVES = WM * WN, BM = 16 * WM * MB, BN = 16 * WN * NB;
    constexpr int COPIES = BM / 8 / WAVES;   // of a wave and step: 8 rows of 128 bytes each
    static_assert(4 % WS == 0, "places of W come round again after a pair of steps");
    static_assert(MB >= NB && 2 * MB % COPIES == 0, "requests dealt evenly");
    static_assert(COPIES * 8 * WAVES == BM, "rows dealt evenly");
    constexpr int ROW = 16 * NB * 2 + 16;   // bytes of a row of y on its way out: data and 16, so that rows start at different banks
    __shared__ __align__(1024) int8_t s_x[NS][BM * 128];
    __shared__ __align__(16) int8_t s_y[WAVES][16 * ROW];
    __shared__ __align__(16) float s_sx[2][BM], s_sw[2][BN];   // by parity of the tile
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int steps = a.chunks >> 1;
    const int k_last = (a.inner - 1) / 16 * 16;
    const int n_rb = (a.cols + QPACK_ROWS - 1) / QPACK_ROWS;

    // ---- the tile whose operands are requested
    int mt, nt;
    // X: lane l copies piece (l % 8) ^ (l / 8) of row l / 8 of its eight rows: piece p of row r lies at place p ^ (r % 8) of
    // the row's 128 bytes, so that the eight lanes that read neighbouring rows at once find different banks
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const int8_t* x0;
    uint32_t xo[COPIES];   // (a tile of X spans less than 2^31 bytes: CATS_QUANT_MAX_LD)
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&s_x[0][0])) + wave * COPIES * 1024;
    auto copy_piece = [&](int s, int slot, int i) {
        // past the end of a row of X the weights are zeros: any value will do there
        copy_to_lds(x0, xo[i] + min(s * 128 + piece, k_last), lds0 + slot * (BM * 128) + i * 1024);
    };
    // W (row blocks and chunks that do not exist are read from the last ones: their products are not stored, or not made)
    __amdgpu_buffer_rsrc_t w_buf;
    int w_at[NB];
    i32x4 w[WS][NB];   // chunk c in place c % WS, WS - 1 chunks ahead
    auto load_w = [&](int c, int j) {
        return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(w_buf, lane * 16, w_at[j] + min(c, a.chunks - 1) * QPACK_FRAG, 0));
    };
    // the scales, for when the sums are ready
    static_assert(BM <= 64 * WAVES && BN <= 64 * WAVES, "one of each a thread");
    float sx_own, sw_own;
    auto enter = [&](int index) {
        quant_tile_of(grid, index, mt, nt);
        sx_own = a.x_scale[min(mt * BM + min(tid, BM - 1), a.rows - 1)];
        sw_own = a.w_scale[min(nt * BN + min(tid, BN - 1), a.cols - 1)];
        x0 = a.x + static_cast<int64_t>(mt) * BM * a.x_ld;
#pragma unroll
        for (int i = 0; i < COPIES; ++i)
            xo[i] = min((wave * COPIES + i) * 8 + (lane >> 3), a.rows - 1 - mt * BM) * static_cast<int>(a.x_ld);
        const int rb0 = min(nt * (BN / 16) + wn * NB, n_rb - 1);
        const int w_bytes = __builtin_amdgcn_readfirstlane(min(NB, n_rb - rb0) * a.chunks * QPACK_FRAG);
        w_buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(a.w + static_cast<int64_t>(rb0) * a.chunks * QPACK_FRAG), 0,
                                                  w_bytes, 0x00020000);
#pragma unroll
        for (int j = 0; j < NB; ++j) w_at[j] = __builtin_amdgcn_readfirstlane(min(j, n_rb - 1 - rb0) * a.chunks * QPACK_FRAG);
        // What the first step needs comes first: X of step 0, W of its chunks, X of step 1.
        auto load_chunk = [&](int c) {
#pragma unroll
            for (int j = 0; j < NB; ++j) w[c][j] = load_w(c, j);
        };
        static_assert(NS == 4 && WS == 4, "order and counts of the first requests");
#pragma unroll
        for (int i = 0; i < COPIES; ++i) copy_piece(0, 0, i);
        load_chunk(0);
        load_chunk(1);
#pragma unroll
        for (int i = 0; i < COPIES; ++i) copy_piece(1, 1, i);
        load_chunk(2);
#pragma unroll
        for (int i = 0; i < COPIES; ++i) copy_piece(2, 2, i);
    };

    i32x4 acc[MB][NB];
    const int r = lane & 15, g = lane >> 4;
    const int8_t* xs = &s_x[0][0] + (wm * MB * 16 + r) * 128;
    // fragment f of a step: block f % MB of rows, chunk f / MB
    const int at[2] = {(g ^ (r & 7)) * 16, ((4 + g) ^ (r & 7)) * 16};
    auto read_x = [&](int slot, int f) { return *reinterpret_cast<const i32x4*>(xs + slot * (BM * 128) + (f % MB) * 2048 + at[f / MB]); };
    constexpr int AHEAD = 4;   // fragments of X read ahead of their products, across the steps' border
    i32x4 x[AHEAD];
    auto next_slot = [](int slot) { return slot == NS - 1 ? 0 : slot + 1; };
    // u: parity of the step
    auto step = [&](int s, int slot, auto u_) {
        constexpr int u = decltype(u_)::value;
        // Requests are dealt out over the step, one between some products each: issued together they hold up the products
        // behind them (49 -> 43 us for 256 x 4096 x 4096).
        // What step s - 1 issued may be under way; all before it, the copies for step s + 1 among it, has come.  Then everybody's
        // copies are there, and nobody reads the slot of step s - 1 any more: the copies for step s + NS - 1 go there (those of
        // steps that do not exist are read by nobody).
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)" ::"n"(COPIES + 2 * NB), "n"(AHEAD) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int slot1 = next_slot(slot);
#pragma unroll
        for (int f = 0; f < 2 * MB; ++f) {
            const int i = f % MB, h = f / MB;
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (i == j * MB / NB) w[(2 * u + h + WS - 1) % WS][j] = load_w(2 * s + h + WS - 1, j);
            if (f % (2 * MB / COPIES) == 1) copy_piece(s + NS - 1, slot == 0 ? NS - 1 : slot - 1, f / (2 * MB / COPIES));
            const i32x4 xf = x[f % AHEAD];
            x[f % AHEAD] = f + AHEAD < 2 * MB ? read_x(slot, f + AHEAD) : read_x(slot1, f + AHEAD - 2 * MB);
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[(2 * u + h) % WS][j], xf, acc[i][j], 0, 0, 0);
        }
        // the order of the step: a fragment of X for each that is multiplied, the requests for W between them
#pragma unroll
        for (int f = 0; f < 2 * MB; ++f) {
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (f % MB == j * MB / NB) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, NB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
    };
    enter(blockIdx.x);
    for (int index = blockIdx.x, parity = 0;; parity ^= 1) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES + NB) : "memory");
        if (tid < BM) s_sx[parity][tid] = sx_own;
        if (tid < BN) s_sw[parity][tid] = sw_own;
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) x[f] = read_x(0, f);
        int slot = 0;
        for (int s = 0; s < steps; s += 2) {   // packed weights end with a whole pair of steps
            step(s, slot, std::integral_constant<int, 0>{});
            slot = next_slot(slot);
            step(s + 1, slot, std::integral_constant<int, 1>{});
            slot = next_slot(slot);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no copy may land after the workgroup's end, or in the next tile's X
        __syncthreads();
        // the next tile's operands come while this one's y leaves
        const int t0 = mt * BM + wm * MB * 16, n0 = nt * BN + wn * NB * 16;
        const bool inside = nt * BN + BN <= a.cols;
        index += gridDim.x;
        const bool more = index < grid.all;
        if (more) enter(index);
        // Four columns a lane are short runs of a row in bf16: a row block goes through LDS (each wave has its own place) and leaves
        // as eight columns a lane, whole lines of y.  With the scales read ahead: 4096 x 4096 x 256 16.6 -> 12.7 us.
        int8_t* mine = &s_y[wave][0];
        const bool wide = a.y_type == CATS_BF16 && ((reinterpret_cast<uintptr_t>(a.y) | static_cast<uint64_t>(a.y_ld) * 2) & 15) == 0 && inside;
        f32x4 sw[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) sw[j] = *reinterpret_cast<const f32x4*>(&s_sw[parity][wn * NB * 16 + 16 * j + 4 * g]);
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            const float sx = s_sx[parity][(wm * MB + i) * 16 + r];
            const int t = t0 + 16 * i;
            f32x4 y[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) y[j] = quant_scaled(acc[i][j], sx, sw[j]);
            if (wide) {
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    *reinterpret_cast<uint2*>(mine + r * ROW + 32 * j + 8 * g) = make_uint2(pack_bf2(y[j][0], y[j][1]), pack_bf2(y[j][2], y[j][3]));
                __builtin_amdgcn_wave_barrier();
                constexpr int LANES = 2 * NB;   // of a row
#pragma unroll
                for (int k = 0; k < (16 * LANES + 63) / 64; ++k) {
                    const int row = (k * 64 + lane) / LANES, at16 = (k * 64 + lane) % LANES;
                    if (16 * LANES % 64 != 0 && row >= 16) break;
                    const u32x4 v = *reinterpret_cast<const u32x4*>(mine + row * ROW + at16 * 16);
                    if (t + row < a.rows) *reinterpret_cast<u32x4*>(static_cast<bf16_t*>(a.y) + (t + row) * a.y_ld + n0 + at16 * 8) = v;
                }
                __builtin_amdgcn_wave_barrier();
            } else if (t + r < a.rows) {
#pragma unroll
                for (int j = 0; j < NB; ++j) quant_store4(a, t + r, n0 + 16 * j + 4 * g, y[j]);
            }
        }
        if (!more) return;
    }
}

template <int WM, int WN, int MB, int NB, int NS, int WS>
void launch_tiles(const QuantLinearArgs& a, int n_cus, hipStream_t st) {
    constexpr int BM = 16 * WM * MB, BN = 16 * WN * NB;
    const QuantGrid grid = quant_grid(a.rows, a.cols, 1, BM, BN);
    hipLaunchKernelGGL((cats_quant_linear_tiles<WM, WN, MB, NB, NS, WS>), dim3(std::min(grid.all, n_cus)),
                       dim3(64 * WM * WN), 0, st, a, grid);
}

}  // namespace

void launch_quant_tiles(const QuantLinearArgs& a, int n_cus, hipStream_t st) { launch_tiles<2, 4, 8, 4, 4, 4>(a, n_cus, st); }
void launch_quant_tiles_narrow(const QuantLinearArgs& a, int n_cus, hipStream_t st) { launch_tiles<2, 4, 8, 3, 4, 4>(a, n_cus, st); }
void launch_quant_tiles_half(const QuantLinearArgs& a, int n_cus, hipStream_t st) { launch_tiles<2, 4, 4, 4, 4, 4>(a, n_cus, st); }
void launch_quant_tiles_half_narrow(const QuantLinearArgs& a, int n_cus, hipStream_t st) { launch_tiles<2, 4, 4, 3, 4, 4>(a, n_cus, st); }
