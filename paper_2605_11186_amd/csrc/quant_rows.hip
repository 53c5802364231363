// Rows in 8-bit integers with one scale each, and the steps of a decoder layer that end in such rows:
//   q = rint(127 v / max|v|) (ties to even),  scale = max|v| / 127 (at least 2^-126)
// for v = a source row, v = rmsnorm(x + delta) * gain, v = silu(gate) * up, or v = the merged chunks of a single query's attention.
//
// One pass: a row is read once, held in the registers of the threads that share it (8 values a thread and piece)
// until its maximum (for the norm its sum of squares first) is known, and written as bytes.  There is no matrix work and no more
// than 20 instructions a value: the kernel is bound by memory with many rows and by its chain of loads, two reductions and
// stores with few, every instruction of it counts.  8192 x 5120 with a bf16 delta 85 us, 32000 x 4096 from bf16 68 us, SwiGLU of 4096 x
// 13824 52 us: 5.4 to 5.8 TB/s, where a large copy reaches 5.2; 63 rows of 4096 2.0 to 2.5 us, where an empty launch takes 1.6.
#include <type_traits>

#include "quant.hpp"

namespace {

typedef double none_t;   // the type of a delta that is not there
struct pieces_t {        // a delta of several pieces
    float v;
};

constexpr float SCALE_MIN = 0x1p-126f;   // smallest normal number: 1 / scale stays finite

// Largest of a wave's unsigned values, in all lanes (see sum_lanes for the moves).
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_moved_u(uint32_t x) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t wave_max64(uint32_t v) {
    const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max(p[0], p[1]);
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(r[0], r[1]);
    v = max(v, dpp_moved_u<0x128>(v));
    v = max(v, dpp_moved_u<0x124>(v));
    v = max(v, dpp_moved_u<0x4E>(v));
    return max(v, dpp_moved_u<0xB1>(v));
}

// 1 / sqrt(x) for x > 0, to 1 ulp: the hardware's, which takes no numbers below the normal ones.
__device__ __forceinline__ float inverse_sqrt(float x) {
    const bool small = x < 0x1p-96f;
    return __builtin_amdgcn_rsqf(small ? x * 0x1p96f : x) * (small ? 0x1p48f : 1.f);
}

// silu(g) * u for gates below CLOSED, where 1 + exp(g) is 1: g exp(g) u in two halves, exp(g / 2) each, which stay normal numbers down
// to g = -174 (1 + exp(-g) passes 2^126, above which the hardware's reciprocal is zero, at g = -87).  The rounding of g log2(e) / 2,
// which as an exponent counts |g| times, is made good.
constexpr float CLOSED = -20.f;
__device__ __forceinline__ float closed_gate(float g, float u) {
    constexpr float HALF_LOG2E = 0.72134751f, HALF_LOG2E_LOW = 9.6298117e-9f, LN2 = 0.69314718f;
    const float t = g * HALF_LOG2E;
    const float h = __builtin_amdgcn_exp2f(t) * fmaf(fmaf(g, HALF_LOG2E_LOW, fmaf(g, HALF_LOG2E, -t)), LN2, 1.f);
    return (g * h) * (u * h);
}

// Eight values as they lie in memory: whole pieces of 16 bytes (VEC) or one by one.
template <class T, bool VEC>
struct Raw;
template <>
struct Raw<float, true> {
    f32x4 v[2];
    __device__ __forceinline__ float get(int e) const { return v[e >> 2][e & 3]; }
};
template <>
struct Raw<bf16_t, true> {
    u32x4 v;
    __device__ __forceinline__ float get(int e) const {
        return __uint_as_float(e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16);
    }
};
template <>
struct Raw<float, false> {
    float v[8];
    __device__ __forceinline__ float get(int e) const { return v[e]; }
};
template <>
struct Raw<bf16_t, false> {
    bf16_t v[8];
    __device__ __forceinline__ float get(int e) const { return bf2f(v[e]); }
};

// Places of a thread's values: piece j, value e.  VEC: eight neighbours; else neighbouring threads hold neighbouring
// values, so that a wave's load of one value each is still one run of memory.
template <int TPR, bool VEC>
__device__ __forceinline__ int place(int tid, int j, int e) {
    return VEC ? (j * TPR + tid) * 8 + e : (j * 8 + e) * TPR + tid;
}
// A row as a buffer of its own: what lies behind it reads as zero and is not written (the buffer's range check), so that the
// loads and stores need no branch and the values no select.  VEC only; else places behind the row read its last value, which counts
// for nothing.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const void* row, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(row), 0, bytes, 0x00020000);
}
template <class T, int TPR, bool VEC>
__device__ __forceinline__ Raw<T, VEC> load8(const T* row, int tid, int j, int cols) {
    Raw<T, VEC> r;
    if constexpr (VEC) {
        const __amdgpu_buffer_rsrc_t buf = row_buffer(row, cols * static_cast<int>(sizeof(T)));
        const int at = place<TPR, VEC>(tid, j, 0) * static_cast<int>(sizeof(T));
        if constexpr (sizeof(T) == 4) {
            r.v[0] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, at, 0, 0));
            r.v[1] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, at + 16, 0, 0));
        } else {
            r.v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, at, 0, 0));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = row[min(place<TPR, VEC>(tid, j, e), cols - 1)];
    }
    return r;
}

// ROWS_MERGED: columns k .. k + 7 belong to head k / head_dim, whose chunks are merged in index order, CH chunks' loads in flight
// at a time, rescaled to the running maximum between groups.  One workgroup reads it all at some 60 GB/s (32 heads of 128: 16 KB
// a chunk); the row's maximum leaves no work for more.
template <int TPR, int NC>
__device__ __forceinline__ void merge_chunks(const QuantRowsArgs& a, int tid, float (&v)[NC][8]) {
    constexpr int CH = 8;
    const float* po[NC];
    const float* ml[NC];
    float den[NC], top[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int k = min(place<TPR, true>(tid, j, 0), a.cols - 8), h = k / a.head_dim;
        po[j] = static_cast<const float*>(a.src) + static_cast<size_t>(h) * a.n_chunks * a.head_dim + (k - h * a.head_dim);
        ml[j] = a.ml + static_cast<size_t>(h) * a.n_chunks * 2;
        den[j] = 0.f;
        top[j] = -1e30f;   // where a chunk's maximum starts, too
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
    }
    for (int c0 = 0; c0 < a.n_chunks; c0 += CH) {
        f32x4 x[NC][CH][2];
        float mc[NC][CH], lc[NC][CH];
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int c = min(c0 + i, a.n_chunks - 1);   // (clamped repeats do not change the maximum and do not count)
                mc[j][i] = ml[j][2 * c];
                lc[j][i] = ml[j][2 * c + 1];
                const f32x4* p = reinterpret_cast<const f32x4*>(po[j] + static_cast<size_t>(c) * a.head_dim);
                x[j][i][0] = p[0];
                x[j][i][1] = p[1];
            }
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            float most = top[j];
#pragma unroll
            for (int i = 0; i < CH; ++i) most = fmaxf(most, mc[j][i]);
            const float before = __builtin_amdgcn_exp2f(top[j] - most);
            top[j] = most;
            den[j] *= before;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] *= before;
#pragma unroll
            for (int i = 0; i < CH; ++i)
                if (c0 + i < a.n_chunks) {
                    const float w = __builtin_amdgcn_exp2f(mc[j][i] - most);
                    den[j] = fmaf(w, lc[j][i], den[j]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[j][e] = fmaf(w, x[j][i][e >> 2][e & 3], v[j][e]);
                }
        }
    }
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] *= 1.f / den[j];
}

// TPR threads share a row (64: four rows a workgroup), NC pieces of 8 values each.  T: type of the source.
// D: type of delta (none_t: none).
template <int KIND, class T, class D, int TPR, int NC, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void cats_quantize_rows_kernel(QuantRowsArgs a) {
    constexpr int ROWS_WG = TPR < 256 ? 256 / TPR : 1;
    constexpr int WAVES = TPR / 64;
    constexpr bool HAS_DELTA = !std::is_same<D, none_t>::value;
    const int tid = threadIdx.x % TPR;
    const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * ROWS_WG + threadIdx.x / TPR);   // (a wave's threads share a row)
    // all arguments at once: loaded where they are used, they are several scalar round trips one behind the other
    asm volatile("" ::"s"(a.src), "s"(a.src_ld), "s"(a.q), "s"(a.q_ld), "s"(a.scale), "s"(a.rows), "s"(a.cols));
    if constexpr (KIND == ROWS_NORM) asm volatile("" ::"s"(a.gain), "s"(a.eps));
    if constexpr (HAS_DELTA) asm volatile("" ::"s"(a.delta), "s"(a.delta_ld), "s"(a.x_out), "s"(a.x_out_ld));
    if (t >= a.rows) return;   // whole waves, and no barrier where a workgroup has several rows
    const int cols = a.cols;
    const T* src = static_cast<const T*>(a.src) + t * a.src_ld;
    // 64 values a thread leave no registers for all that they are made of: that is read piece by piece.  (Read at once it is put by in
    // memory, 340 to 650 bytes a thread: 63 rows of 20001 columns, norm with a float32 delta 70 us, 15 by piece; SwiGLU from float32 27 and 12.)
    constexpr bool BY_PIECE = NC > 4 && (!VEC || sizeof(T) == 4) && (KIND == ROWS_SWIGLU || (KIND == ROWS_NORM && !VEC));
    auto end_of_piece = [] {
        if constexpr (BY_PIECE) __builtin_amdgcn_sched_barrier(0);
    };

    Raw<T, VEC> r0[NC];
    float v[NC][8];
    bool in[NC][VEC ? 1 : 8];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        if constexpr (KIND != ROWS_MERGED && !BY_PIECE) r0[j] = load8<T, TPR, VEC>(src, tid, j, cols);
#pragma unroll
        for (int e = 0; e < (VEC ? 1 : 8); ++e) in[j][e] = place<TPR, VEC>(tid, j, e) < cols;
    }
    if constexpr (KIND == ROWS_PLAIN) {
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = VEC || in[j][e] ? r0[j].get(e) : 0.f;
    } else if constexpr (KIND == ROWS_MERGED) {
        merge_chunks<TPR, NC>(a, tid, v);
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = in[j][0] ? bf2f(f2bf(v[j][e])) : 0.f;
    } else if constexpr (KIND == ROWS_SWIGLU) {
        Raw<T, VEC> r1[NC];
#pragma unroll
        for (int j = 0; j < NC; ++j)
            if constexpr (!BY_PIECE) r1[j] = load8<T, TPR, VEC>(src + cols, tid, j, cols);
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            if constexpr (BY_PIECE) {
                r0[j] = load8<T, TPR, VEC>(src, tid, j, cols);
                r1[j] = load8<T, TPR, VEC>(src + cols, tid, j, cols);
            }
            float lowest = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = r0[j].get(e);
                lowest = fminf(lowest, g);
                // (the hardware's reciprocal, 1 ulp: a division's ten instructions more cost half a microsecond in rows of 11008)
                v[j][e] = g * __builtin_amdgcn_rcpf(1.f + __expf(-g)) * r1[j].get(e);
            }
            // few rows have such gates: a wave whose values have none goes past
            if (__builtin_amdgcn_ballot_w64(lowest < CLOSED) != 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[j][e] = r0[j].get(e) < CLOSED ? closed_gate(r0[j].get(e), r1[j].get(e)) : v[j][e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = VEC || in[j][e] ? v[j][e] : 0.f;
            end_of_piece();
        }
    } else {
        Raw<bf16_t, VEC> rg[NC];
        float ss = 0.f;
        if constexpr (HAS_DELTA) {
            // PIECES loads of each value at once; those of pieces that are not there are the last one's again, and do not count
            constexpr bool PIECED = std::is_same<D, pieces_t>::value;
            constexpr int PIECES = PIECED ? QUANT_MAX_PIECES : 1;
            using E = typename std::conditional<PIECED, float, D>::type;
            Raw<E, VEC> r1[PIECES][NC];
            const E* delta = static_cast<const E*>(a.delta) + t * a.delta_ld;
            float* out = a.x_out + t * a.x_out_ld;
            auto load_delta = [&](int p, int j) {
                r1[p][j] = load8<E, TPR, VEC>(delta + (PIECED ? min(p, a.delta_pieces - 1) * (a.rows * a.delta_ld) : 0), tid, j, cols);
            };
            if constexpr (!BY_PIECE) {
#pragma unroll
                for (int p = 0; p < PIECES; ++p)
#pragma unroll
                    for (int j = 0; j < NC; ++j) load_delta(p, j);
#pragma unroll
                for (int j = 0; j < NC; ++j) rg[j] = load8<bf16_t, TPR, VEC>(a.gain, tid, j, cols);
            }
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                if constexpr (BY_PIECE) {
                    r0[j] = load8<T, TPR, VEC>(src, tid, j, cols);
#pragma unroll
                    for (int p = 0; p < PIECES; ++p) load_delta(p, j);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float sum = r1[0][j].get(e);
#pragma unroll
                    for (int p = 1; p < PIECES; ++p)
                        if (p < a.delta_pieces) sum += r1[p][j].get(e);
                    v[j][e] = VEC || in[j][e] ? r0[j].get(e) + sum : 0.f;
                }
                if constexpr (VEC) {
                    const __amdgpu_buffer_rsrc_t buf = row_buffer(out, cols * 4);
                    const int at = place<TPR, VEC>(tid, j, 0) * 4;
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[j][0], v[j][1], v[j][2], v[j][3]}), buf, at, 0, 0);
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[j][4], v[j][5], v[j][6], v[j][7]}), buf, at + 16, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (in[j][e]) out[place<TPR, VEC>(tid, j, e)] = v[j][e];
                }
                end_of_piece();
            }
        } else {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                if constexpr (BY_PIECE)
                    r0[j] = load8<T, TPR, VEC>(src, tid, j, cols);
                else
                    rg[j] = load8<bf16_t, TPR, VEC>(a.gain, tid, j, cols);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[j][e] = VEC || in[j][e] ? r0[j].get(e) : 0.f;
                end_of_piece();
            }
        }
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(v[j][e], v[j][e], ss);
        ss = wave_sum64(ss);
        if constexpr (WAVES > 1) {
            __shared__ float s_sum[WAVES];
            if ((tid & 63) == 0) s_sum[tid >> 6] = ss;
            __syncthreads();
            ss = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) ss += s_sum[w];
        }
        // a sum of squares beyond float32 makes the row not a number, as an infinity in it does
        const float r = ss < INFINITY ? inverse_sqrt(ss * (1.f / static_cast<float>(cols)) + a.eps) : NAN;
        // (values that are not there are zeros, and NaN only where r or the last gains make the row's last values so, too)
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            if constexpr (BY_PIECE) {
                int again = tid;   // (or else the places of all values are kept since the loads of x)
                asm volatile("" : "+v"(again));
                rg[j] = load8<bf16_t, TPR, VEC>(a.gain, again, j, cols);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = v[j][e] * r * rg[j].get(e);
            end_of_piece();
        }
    }

    // the largest |v|, as bits: ordered like the numbers, infinity above them and NaN above infinity
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[j][e]) & 0x7FFFFFFFu);
    top = wave_max64(top);
    if constexpr (WAVES > 1) {
        __shared__ uint32_t s_top[WAVES];
        if ((tid & 63) == 0) s_top[tid >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = max(top, s_top[w]);
    }
    const bool finite = top < 0x7F800000u;
    const float most = fmaxf(__uint_as_float(top), 127.f * SCALE_MIN);
    // y + 1.5 * 2^23: the sum's last bits are the whole number nearest to y in two's complement (ties to even)
    constexpr float WHOLE = 12582912.f;
    // Plain and merged rows: 127 v / most is rounded as the exact quotient is.  By the power of two p, most p lies in [1, 4) and no
    // product leaves the range.
    // Values of bf16: their quotients are ties (one in some thousands) or 2^-17 of themselves away, and a correctly rounded quotient y (one
    // correction) tells which.
    // Values of float32: 127 v p = z + low exactly.  whole is the whole number n next to z / den or, next to a tie, one of the two, and
    // rest = z - n den, which is exact, tells whether it is: low is at most 2^-17 den.  If so, |rest| is so near half of den that their difference is
    // exact as well, and over has the sign of the exact remainder's distance from half (0: a tie).  A wave without such values, most
    // are, goes past (a row of 4096: 1.75 us, 2.35 without the branch; in rows of bf16 the ties make it 2.05 against the quotient's 1.8).
    // Computed rows have no ties worth either.
    const float p = __uint_as_float(max(0x7F000000u - (__float_as_uint(most) & 0x7F800000u), 0x00800000u));
    constexpr bool TIES = KIND == ROWS_PLAIN || KIND == ROWS_MERGED, EXACT = KIND == ROWS_PLAIN && std::is_same<T, float>::value;
    const float den = most * p, rden = TIES ? 1.f / den : __builtin_amdgcn_rcpf(den), mul = 127.f * p * (TIES ? 1.f : rden);
    int8_t* q = a.q + t * a.q_ld;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        uint32_t b[8];
        if constexpr (EXACT) {
            float furthest = 0.f;
            auto remainder = [&](float z, float whole) { return fmaf(WHOLE - whole, den, z); };
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = v[j][e] * mul, whole = fmaf(z, rden, WHOLE);
                b[e] = __float_as_uint(whole);
                furthest = fmaxf(furthest, fabsf(remainder(z, whole)));
            }
            if (__builtin_amdgcn_ballot_w64(furthest > den * (0.5f - 0x1p-15f)) != 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = v[j][e] * mul, low = fmaf(v[j][e], mul, -z), rest = remainder(z, __uint_as_float(b[e]));
                    const uint32_t sign = __float_as_uint(rest) & 0x80000000u;
                    const float over = fabsf(rest) - 0.5f * den + __uint_as_float(__float_as_uint(low) ^ sign);
                    // (as whole numbers: negative, 0 or positive, like over; n's last bit tells the odd one of two)
                    const bool other = static_cast<int>(__float_as_uint(over) + (b[e] & 1)) > 0;
                    b[e] += other ? (sign ? -1 : 1) : 0;
                }
            }
        } else if constexpr (TIES) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = v[j][e] * mul, y = z * rden;
                b[e] = __float_as_uint(fmaf(fmaf(-y, den, z), rden, y) + WHOLE);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(fmaf(v[j][e], mul, WHOLE));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = finite ? b[e] & 0xFFu : 0u;
        if constexpr (VEC) {
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            __builtin_amdgcn_raw_buffer_store_b64(u32x2{b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24, b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24},
                                                  row_buffer(q, cols), place<TPR, VEC>(tid, j, 0), 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (in[j][e]) q[place<TPR, VEC>(tid, j, e)] = static_cast<int8_t>(b[e]);
        }
    }
    if (tid == 0) a.scale[t] = finite ? most / 127.f : NAN;
}

template <int KIND, class T, class D, int TPR, int NC, bool VEC>
void launch(const QuantRowsArgs& a, hipStream_t st) {
    constexpr int ROWS_WG = TPR < 256 ? 256 / TPR : 1;
    hipLaunchKernelGGL((cats_quantize_rows_kernel<KIND, T, D, TPR, NC, VEC>), dim3((a.rows + ROWS_WG - 1) / ROWS_WG),
                       dim3(TPR < 256 ? 256 : TPR), 0, st, a);
}

// Threads a row: few threads with a few pieces each wait for one another the least (two barriers a row) as long as a row's loads
// are all under way at once.  Norm of 63 rows: 4096 columns 2.5 us with 256 threads, 2.6 with 512; 11008 columns 4.4 with 512 and
// three pieces, 5.0 with 1024 and two; 5120 columns 2.9 with 256 and three pieces, 3.25 with 512 and two.
template <int KIND, class T, class D, bool VEC>
void by_size(const QuantRowsArgs& a, hipStream_t st) {
    const int pieces = (a.cols + 7) / 8;   // of 8 values
    if (pieces <= 64) return launch<KIND, T, D, 64, 1, VEC>(a, st);
    if (pieces <= 256) return launch<KIND, T, D, 256, 1, VEC>(a, st);
    if (pieces <= 512) return launch<KIND, T, D, 256, 2, VEC>(a, st);
    if (pieces <= 768) return launch<KIND, T, D, 256, 3, VEC>(a, st);
    if (pieces <= 1024 || std::is_same<D, pieces_t>::value) return launch<KIND, T, D, 512, 2, VEC>(a, st);
    if constexpr (!std::is_same<D, pieces_t>::value) {   // (a delta of several pieces has the columns of a model's hidden rows, at most 8192)
        if (pieces <= 1536) return launch<KIND, T, D, 512, 3, VEC>(a, st);
        if (pieces <= 2048) return launch<KIND, T, D, 512, 4, VEC>(a, st);
        return launch<KIND, T, D, 1024, 8, VEC>(a, st);
    }
}
static_assert(CATS_QUANT_MAX_ROWS <= (1 << 21), "threads of a launch: fewer than 2^32");
static_assert(CATS_QUANT_MAX_COLS == 1024 * 8 * 8, "the longest row fills the largest workgroup's registers");

// Whole pieces of 8 values: no row starts or ends inside one, and rows stay aligned.
bool whole_pieces(const void* p, int64_t ld, size_t size) {
    const size_t piece = size == 4 ? 16 : 8 * size;   // float32 pieces are two loads of 16 bytes
    return (reinterpret_cast<uintptr_t>(p) | static_cast<uint64_t>(ld) * size) % piece == 0;
}

template <int KIND, class T, class D>
void by_alignment(const QuantRowsArgs& a, hipStream_t st) {
    bool vec = a.cols % 8 == 0 && whole_pieces(a.src, a.src_ld, sizeof(T)) && whole_pieces(a.q, a.q_ld, 1);
    if (KIND == ROWS_NORM) vec = vec && whole_pieces(a.gain, 0, 2);
    if (KIND == ROWS_NORM && !std::is_same<D, none_t>::value)
        vec = vec && whole_pieces(a.delta, a.delta_ld, sizeof(D)) && whole_pieces(a.x_out, a.x_out_ld, 4);
    if (vec)
        by_size<KIND, T, D, true>(a, st);
    else
        by_size<KIND, T, D, false>(a, st);
}

bool type_ok(int32_t t) { return t == CATS_F32 || t == CATS_BF16; }
bool aligned(const void* p, int32_t type) { return reinterpret_cast<uintptr_t>(p) % (type == CATS_F32 ? 4 : 2) == 0; }

// The checks that every entry point with quantised rows shares.
int check_rows(int32_t rows, int32_t cols, const int8_t* q, int64_t q_ld, const float* scale) {
    if (!q || !scale || rows < 0 || cols < 1 || q_ld < cols || !aligned(scale, CATS_F32)) return CATS_EINVAL;
    return cols > CATS_QUANT_MAX_COLS || rows > CATS_QUANT_MAX_ROWS ? CATS_ECAPACITY : CATS_OK;
}
int enqueue(const QuantRowsArgs& a, int kind, void* stream) {
    if (a.rows == 0) return CATS_OK;
    launch_quant_rows(a, kind, static_cast<hipStream_t>(stream));
    return launch_status();
}

}  // namespace

void launch_quant_rows(const QuantRowsArgs& a, int kind, hipStream_t st) {
    if (a.rows < 1) return;
    if (kind == ROWS_MERGED) {
        const int pieces = a.cols / 8;
        if (pieces <= 64) return launch<ROWS_MERGED, float, none_t, 64, 1, true>(a, st);
        if (pieces <= 256) return launch<ROWS_MERGED, float, none_t, 256, 1, true>(a, st);
        if (pieces <= 512) return launch<ROWS_MERGED, float, none_t, 512, 1, true>(a, st);
        return launch<ROWS_MERGED, float, none_t, 1024, 1, true>(a, st);
    }
    const bool f32 = a.src_type == CATS_F32;
    if (kind == ROWS_PLAIN)
        return f32 ? by_alignment<ROWS_PLAIN, float, none_t>(a, st) : by_alignment<ROWS_PLAIN, bf16_t, none_t>(a, st);
    if (kind == ROWS_SWIGLU)
        return f32 ? by_alignment<ROWS_SWIGLU, float, none_t>(a, st) : by_alignment<ROWS_SWIGLU, bf16_t, none_t>(a, st);
    if (!a.delta) return by_alignment<ROWS_NORM, float, none_t>(a, st);
    if (a.delta_pieces > 1) return by_alignment<ROWS_NORM, float, pieces_t>(a, st);
    return a.delta_type == CATS_F32 ? by_alignment<ROWS_NORM, float, float>(a, st)
                                    : by_alignment<ROWS_NORM, float, bf16_t>(a, st);
}

extern "C" {

int cats_quantize_rows(const void* src, int32_t src_type, int64_t src_ld, int32_t rows, int32_t cols, int8_t* q,
                       int64_t q_ld, float* scale, void* stream) {
    if (!src || !type_ok(src_type) || !aligned(src, src_type)) return CATS_EINVAL;
    const int rc = check_rows(rows, cols, q, q_ld, scale);
    if (rc != CATS_OK) return rc;
    if (src_ld < cols) return CATS_EINVAL;
    QuantRowsArgs a{};
    a.src = src;
    a.src_type = src_type;
    a.src_ld = src_ld;
    a.rows = rows;
    a.cols = cols;
    a.q = q;
    a.q_ld = q_ld;
    a.scale = scale;
    return enqueue(a, ROWS_PLAIN, stream);
}

int cats_rmsnorm_quantize(const float* x, int64_t x_ld, const void* delta, int32_t delta_type, int64_t delta_ld,
                          const void* gain, float eps, int32_t rows, int32_t cols, float* x_out, int64_t x_out_ld,
                          int8_t* q, int64_t q_ld, float* scale, void* stream) {
    if (!x || !gain || !aligned(x, CATS_F32) || !aligned(gain, CATS_BF16) || !(eps > 0.f && eps < INFINITY)) return CATS_EINVAL;
    if ((delta == nullptr) != (x_out == nullptr)) return CATS_EINVAL;
    const int rc = check_rows(rows, cols, q, q_ld, scale);
    if (rc != CATS_OK) return rc;
    if (x_ld < cols) return CATS_EINVAL;
    if (delta && (!type_ok(delta_type) || !aligned(delta, delta_type) || !aligned(x_out, CATS_F32) || delta_ld < cols ||
                  x_out_ld < cols || (x_out == x && x_out_ld != x_ld)))
        return CATS_EINVAL;
    QuantRowsArgs a{};
    a.src = x;
    a.src_type = CATS_F32;
    a.src_ld = x_ld;
    a.delta = delta;
    a.delta_type = delta_type;
    a.delta_ld = delta_ld;
    a.gain = static_cast<const bf16_t*>(gain);
    a.eps = eps;
    a.rows = rows;
    a.cols = cols;
    a.x_out = x_out;
    a.x_out_ld = x_out_ld;
    a.q = q;
    a.q_ld = q_ld;
    a.scale = scale;
    return enqueue(a, ROWS_NORM, stream);
}

int cats_swiglu_quantize(const void* gate_up, int32_t type, int64_t ld, int32_t rows, int32_t cols, int8_t* q,
                         int64_t q_ld, float* scale, void* stream) {
    if (!gate_up || !type_ok(type) || !aligned(gate_up, type)) return CATS_EINVAL;
    const int rc = check_rows(rows, cols, q, q_ld, scale);
    if (rc != CATS_OK) return rc;
    if (ld < 2 * static_cast<int64_t>(cols)) return CATS_EINVAL;
    QuantRowsArgs a{};
    a.src = gate_up;
    a.src_type = type;
    a.src_ld = ld;
    a.rows = rows;
    a.cols = cols;
    a.q = q;
    a.q_ld = q_ld;
    a.scale = scale;
    return enqueue(a, ROWS_SWIGLU, stream);
}

}  // extern "C"
