// quantize.hip -- matrices to 8 bits with one scale per block of 128, and back.
//
//   s = 2^e, the smallest power of two >= 2^-126 with max|x| / s <= 448
//   q = e4m3(x / s), to nearest, ties to even         x' = q s
//
// A power of two divides exactly, so an element is rounded once, and the
// matrix instruction takes the exponent byte as its own block scale.
// Dividing by max|x| / 448 itself would use up to one more bit of the
// format's range, not of its precision.
//
// All kernels are bound by memory: each element is read once and written in
// one byte, also when both orders of a matrix are asked for at once.
#include <type_traits>

#include "operators.hpp"

namespace rs {
namespace {

constexpr float kInf = __builtin_huge_valf();

// Largest of a value over the 16 lanes of a row, in each of them.
__device__ inline float max16(float x) {
    auto turn = [&](auto ctrl) {
        const int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, false);
        x = fmaxf(x, __int_as_float(y));
    };
    turn(std::integral_constant<int, 0x128>{});  // lanes turned by 8, 4, 2 and 1
    turn(std::integral_constant<int, 0x124>{});
    turn(std::integral_constant<int, 0x122>{});
    turn(std::integral_constant<int, 0x121>{});
    return x;
}

// |x| where x is finite, else 0: NaN and infinities do not widen their block's
// scale.  The maximum leaves NaN out by itself, so this is needed only where
// a block's comes out infinite.
__device__ inline float finite_abs(float x) {
    const float a = fabsf(x);
    return a < kInf ? a : 0.0f;
}

// Biased exponent of the block's scale: adding 0x1fffff carries into the
// exponent where the mantissa is above that of 1.75 (448 = 1.75 * 2^8).
__device__ inline int scale_code(float amax) {
    const int e = int((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8;
    return amax > 0 ? (e > 1 ? e : 1) : 127;
}

__device__ inline float inverse_of(int code) { return __int_as_float((254 - code) << 23); }

// Four codes of x / s.  e4m3 has no infinity: the conversion makes NaN of one,
// which so is not lost.
__device__ inline uint32_t to_codes(float a, float b, float c, float d, float inv) {
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, r, true));
}

__device__ inline void store_scale(void *scales, int64_t at, int code, bool e8m0) {
    if (e8m0) static_cast<uint8_t *>(scales)[at] = uint8_t(code);
    else static_cast<float *>(scales)[at] = __int_as_float(code << 23);
}

// Eight elements, zeros past the n that exist.
template <typename T>
struct Eight {
    Pack<T> p[8 / kVec<T>];

    __device__ void load(const T *at, int64_t n) {
#pragma unroll
        for (int h = 0; h < 8 / kVec<T>; ++h) p[h] = load_pack(at + h * kVec<T>, n - h * kVec<T>);
    }
    __device__ float operator[](int i) const { return float(p[i / kVec<T>].e[i % kVec<T>]); }
};

__device__ inline void store_codes(uint8_t *p, uint2 c, int64_t n) {
    if (n >= 8) {
        store_any(p, c);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = uint8_t((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
}

struct QuantArgs {
    const void *x;
    uint8_t *q, *qt;
    void *scales, *scales_t;
    int64_t rows, cols, x_pitch, q_pitch, qt_pitch, scales_pitch, scales_t_pitch;
    int e8m0;
};

constexpr int kUnits = 4;  // blocks of 128 that 16 lanes take, loaded before the first is reduced

// Blocks of one row: 16 lanes hold a block, eight elements each, so that loads
// and stores are whole lines and the maximum needs four moves.  Bound by
// memory: 16384 x 12288 bf16 in 106 us, 5.7 TB/s read and written.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs a, uint32_t per_row) {
    const uint32_t first = blockIdx.x * (16 * kUnits), row0 = first / per_row, b0 = first - row0 * per_row;
    const int lane = threadIdx.x % 16;
    Eight<T> v[kUnits];
    int64_t row[kUnits], col[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const uint32_t b = b0 + u * 16 + threadIdx.x / 16;
        row[u] = row0 + b / per_row;  // at most 2^29 blocks: 32-bit divisions, a tenth of 64-bit ones
        col[u] = int64_t(b % per_row) * kBlock + lane * 8;
        const int64_t n = row[u] < a.rows ? a.cols - col[u] : 0;
        v[u].load(static_cast<const T *>(a.x) + row[u] * a.x_pitch + col[u], n);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        float m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[u][i]));
        if (__any(m == kInf)) {
            m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(v[u][i]));
        }
        const int code = scale_code(max16(m));
        if (row[u] >= a.rows) continue;
        const float inv = inverse_of(code);
        const uint2 c = make_uint2(to_codes(v[u][0], v[u][1], v[u][2], v[u][3], inv),
                                   to_codes(v[u][4], v[u][5], v[u][6], v[u][7], inv));
        store_codes(a.q + row[u] * a.q_pitch + col[u], c, a.cols - col[u]);
        if (lane == 0) store_scale(a.scales, row[u] * a.scales_pitch + col[u] / kBlock, code, a.e8m0);
    }
}

// A 128 x 128 tile a workgroup, read once: the row-wise codes straight from
// the registers, the transposed ones through 16 KiB of LDS.  A thread holds 8
// consecutive rows of 8 columns, so that 8 codes of one column are one
// 8-byte word of the transposed tile.  Word `g` of column c lies in slot
// g ^ (c / 8), which spreads the 16 columns that a row of lanes writes at once
// over all banks.  TILE: one scale for the whole tile, else one per row of it
// (row-wise codes) and one per column (transposed).
// Bound by what three waves a SIMD (64 elements a thread) keep in flight: 8192 x
// 16384 bf16 in 141 us with a scale per row and column, 3.8 TB/s, in 110 us with
// tiles' scales; registers for four waves spilled and took 187.
template <typename T, bool TILE>
__global__ __launch_bounds__(256) void quantize_tile_kernel(QuantArgs a, uint32_t tiles_across) {
    __shared__ uint2 words[kBlock][16];
    __shared__ float part[4][kBlock];
    const uint32_t down = blockIdx.x / tiles_across;
    const int64_t tr = down, tc = blockIdx.x - down * tiles_across;
    const int g = threadIdx.x / 16, lane = threadIdx.x % 16, wave = threadIdx.x / kWave;
    const int64_t r0 = tr * kBlock + g * 8, c0 = tc * kBlock + lane * 8;
    Eight<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        raw[i].load(static_cast<const T *>(a.x) + (r0 + i) * a.x_pitch + c0, r0 + i < a.rows ? a.cols - c0 : 0);
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = raw[i][j];

    float rmax[8], cmax[8];
    auto largest = [&](auto magnitude) {
#pragma unroll
        for (int i = 0; i < 8; ++i) rmax[i] = cmax[i] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float m = magnitude(v[i][j]);
                rmax[i] = fmaxf(rmax[i], m);
                cmax[j] = fmaxf(cmax[j], m);
            }
    };
    largest([](float x) { return fabsf(x); });
    float any = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) any = fmaxf(any, rmax[i]);
    if (__any(any == kInf)) largest([](float x) { return finite_abs(x); });
    if constexpr (TILE) {
        float m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, rmax[i]);
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
        if (threadIdx.x % kWave == 0) part[wave][0] = m;
        __syncthreads();
        m = fmaxf(fmaxf(part[0][0], part[1][0]), fmaxf(part[2][0], part[3][0]));
#pragma unroll
        for (int i = 0; i < 8; ++i) rmax[i] = cmax[i] = m;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) rmax[i] = max16(rmax[i]);
        if (a.qt) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                cmax[j] = fmaxf(cmax[j], __shfl_xor(cmax[j], 16, kWave));
                cmax[j] = fmaxf(cmax[j], __shfl_xor(cmax[j], 32, kWave));
                if (g % 4 == 0) part[wave][lane * 8 + j] = cmax[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = lane * 8 + j;
                cmax[j] = fmaxf(fmaxf(part[0][c], part[1][c]), fmaxf(part[2][c], part[3][c]));
            }
        }
    }

    if (a.q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i >= a.rows) break;
            const int code = scale_code(rmax[i]);
            const float inv = inverse_of(code);
            const uint2 c = make_uint2(to_codes(v[i][0], v[i][1], v[i][2], v[i][3], inv),
                                       to_codes(v[i][4], v[i][5], v[i][6], v[i][7], inv));
            store_codes(a.q + (r0 + i) * a.q_pitch + c0, c, a.cols - c0);
            if (!TILE && lane == 0) store_scale(a.scales, (r0 + i) * a.scales_pitch + tc, code, a.e8m0);
        }
        if (TILE && threadIdx.x == 0) store_scale(a.scales, tr * a.scales_pitch + tc, scale_code(rmax[0]), a.e8m0);
    }
    if (!a.qt) return;  // the same for the whole launch
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int code = scale_code(cmax[j]);
        const float inv = inverse_of(code);
        words[lane * 8 + j][g ^ lane] = make_uint2(to_codes(v[0][j], v[1][j], v[2][j], v[3][j], inv),
                                                   to_codes(v[4][j], v[5][j], v[6][j], v[7][j], inv));
        if (!TILE && g == 0 && c0 + j < a.cols) store_scale(a.scales_t, (c0 + j) * a.scales_t_pitch + tr, code, a.e8m0);
    }
    if (TILE && threadIdx.x == 0) store_scale(a.scales_t, tc * a.scales_t_pitch + tr, scale_code(cmax[0]), a.e8m0);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {  // 16 lanes write the 128 codes of a column
        const int c = i * 16 + g;
        const int64_t col = tc * kBlock + c, row = tr * kBlock + lane * 8;
        if (col < a.cols) store_codes(a.qt + col * a.qt_pitch + row, words[c][lane ^ (c / 8)], a.rows - row);
    }
}

struct DequantArgs {
    const uint8_t *q;
    const void *scales;
    void *y;
    int64_t rows, cols, q_pitch, scales_pitch, y_pitch;
    int e8m0, row_shift;  // rows that share a scale: 1 << row_shift
    bool past_cache;      // y is larger than the last-level cache
};

// code * s as a float32 whose rounding to 16 bits is that of the product
// itself: where the product (28 bits at most) lies between two floats, the odd
// one of them, which no 16-bit value or midpoint of two is.  `off` is the
// product less p, exact, and NaN beside an infinity, which stays.
template <typename F>
__device__ inline float odd_of(float p, F off) {
    const uint32_t bits = __float_as_uint(p);
    if (!(off < 0 || off > 0) || bits & 1) return p;
    return __uint_as_float((off < 0) == (bits >> 31 != 0) ? bits + 1 : bits - 1);
}

__device__ inline void products_to_odd(float (&v)[8], float s) {
    if (fabsf(s) < 0x1p-90f) {  // `off` may be below float32's subnormals
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            const double exact = double(v[i]) * double(s);
            const float p = float(exact);
            v[i] = odd_of(p, exact - double(p));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float p = v[i] * s;
        v[i] = odd_of(p, fmaf(v[i], s, -p));
    }
}

// Bound by memory: 16384 x 12288 to bf16 in 106 us, 5.7 TB/s.  TO_ODD: scales
// of any value into 16 bits (104 us); a power of two multiplies exactly.
template <typename T, bool TO_ODD>
__global__ __launch_bounds__(256) void dequantize_kernel(DequantArgs a, uint32_t per_row) {
    const uint32_t first = blockIdx.x * (16 * kUnits), row0 = first / per_row, b0 = first - row0 * per_row;
    const int lane = threadIdx.x % 16;
    uint2 c[kUnits];
    float s[kUnits];
    int64_t row[kUnits], col[kUnits], n[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const uint32_t b = b0 + u * 16 + threadIdx.x / 16;
        row[u] = row0 + b / per_row;
        col[u] = int64_t(b % per_row) * kBlock + lane * 8;
        n[u] = row[u] < a.rows ? a.cols - col[u] : 0;
        c[u] = make_uint2(0, 0);
        s[u] = 0;
        if (n[u] <= 0) continue;
        const uint8_t *p = a.q + row[u] * a.q_pitch + col[u];
        if (n[u] >= 8) {
            c[u] = load_any<uint2>(p);
        } else {
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n[u]) w[i / 4] |= uint32_t(p[i]) << (8 * (i & 3));
            c[u] = make_uint2(w[0], w[1]);
        }
        const int64_t at = (row[u] >> a.row_shift) * a.scales_pitch + col[u] / kBlock;
        s[u] = a.e8m0 ? e8m0_value(static_cast<const uint8_t *>(a.scales)[at]) : static_cast<const float *>(a.scales)[at];
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        if (n[u] <= 0) continue;
        typedef float pair __attribute__((ext_vector_type(2)));
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int w = int(h ? c[u].y : c[u].x);
            const pair lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            v[4 * h] = lo.x;
            v[4 * h + 1] = lo.y;
            v[4 * h + 2] = hi.x;
            v[4 * h + 3] = hi.y;
        }
        if constexpr (TO_ODD) {
            products_to_odd(v, s[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= s[u];
        }
        T *y = static_cast<T *>(a.y) + row[u] * a.y_pitch + col[u];
#pragma unroll
        for (int h = 0; h < 8; h += kVec<T>) {
            Pack<T> r;
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) r.e[i] = T(v[h + i]);
            if (a.past_cache && n[u] >= h + kVec<T>) store_past(y + h, r.v);
            else if (n[u] > h) store_pack(y + h, r, n[u] - h);
        }
    }
}

template <typename T>
reshard_status_t launch_quantize(const QuantArgs &a, bool tile, hipStream_t s) {
    const char *what = "quantize launch";
    const int64_t across = ceil_div(a.cols, kBlock);
    if (!tile && !a.qt) {
        const int64_t wgs = ceil_div(a.rows * across, 16 * kUnits);
        return launch(what, quantize_rows_kernel<T>, dim3(unsigned(wgs)), 256, 0, s, a, across);
    }
    const dim3 grid(unsigned(across * ceil_div(a.rows, kBlock)));
    return launch(what, tile ? quantize_tile_kernel<T, true> : quantize_tile_kernel<T, false>, grid, 256, 0, s, a, across);
}

// Extents of a blocked matrix that one launch of 2^32 threads holds.
reshard_status_t check_blocks(int64_t rows, int64_t cols, int block_rows, reshard_dtype_t scale_dtype) {
    reshard_status_t st = check_extent("rows", rows);
    if (st == RESHARD_OK) st = check_extent("cols", cols);
    if (st != RESHARD_OK) return st;
    if (block_rows != 1 && block_rows != kBlock) return fail(RESHARD_EINVAL, "block_rows must be 1 or 128");
    if (scale_dtype != RESHARD_E8M0 && scale_dtype != RESHARD_F32)
        return fail(RESHARD_EINVAL, "scale_dtype must be E8M0 or F32");
    const int64_t across = ceil_div(cols, kBlock);
    if (across > 0 && (rows > (int64_t(1) << 29) / across || ceil_div(rows, kBlock) > (int64_t(1) << 23) / across))
        return fail(RESHARD_EUNSUPPORTED, "more than 2^29 blocks of 128 elements or 2^23 tiles of 128 x 128");
    return RESHARD_OK;
}

}  // namespace
}  // namespace rs

using rs::fail;

extern "C" reshard_status_t reshard_quantize(int64_t rows, int64_t cols, const void *x, int64_t x_pitch,
                                             reshard_dtype_t dtype, int block_rows, reshard_dtype_t scale_dtype,
                                             void *q, int64_t q_pitch, void *scales, int64_t scales_pitch, void *qt,
                                             int64_t qt_pitch, void *scales_t, int64_t scales_t_pitch, void *stream) {
    return rs::guarded([&]() -> reshard_status_t {
        using namespace rs;
        reshard_status_t st = check_blocks(rows, cols, block_rows, scale_dtype);
        if (st != RESHARD_OK) return st;
        if (!is_float_type(dtype)) return fail(RESHARD_EINVAL, "dtype must be F16, BF16 or F32");
        const int64_t ss = scale_dtype == RESHARD_F32 ? 4 : 1;
        const int64_t across = ceil_div(cols, kBlock), down = ceil_div(rows, kBlock);
        if (rows > 0 && cols > 0 && !q && !qt) return fail(RESHARD_EINVAL, "q and qt are both NULL");
        st = check_matrix("x", x, rows, cols, x_pitch, dtype == RESHARD_F32 ? 4 : 2);
        if (st == RESHARD_OK && q) st = check_matrix("q", q, rows, cols, q_pitch, 1);
        if (st == RESHARD_OK && q)
            st = check_matrix("scales", scales, block_rows == 1 ? rows : down, across, scales_pitch, ss);
        if (st == RESHARD_OK && qt) st = check_matrix("qt", qt, cols, rows, qt_pitch, 1);
        if (st == RESHARD_OK && qt)
            st = check_matrix("scales_t", scales_t, block_rows == 1 ? cols : across, down, scales_t_pitch, ss);
        if (st != RESHARD_OK || rows == 0 || cols == 0) return st;
        const QuantArgs a{x,       static_cast<uint8_t *>(q), static_cast<uint8_t *>(qt), scales,
                          scales_t, rows, cols, x_pitch, q_pitch, qt_pitch, scales_pitch, scales_t_pitch,
                          scale_dtype == RESHARD_E8M0};
        const hipStream_t s = static_cast<hipStream_t>(stream);
        const bool tile = block_rows == kBlock;
        if (dtype == RESHARD_F32) return launch_quantize<float>(a, tile, s);
        return dtype == RESHARD_BF16 ? launch_quantize<bf16>(a, tile, s) : launch_quantize<f16>(a, tile, s);
    });
}

extern "C" reshard_status_t reshard_dequantize(int64_t rows, int64_t cols, const void *q, int64_t q_pitch,
                                               int block_rows, const void *scales, int64_t scales_pitch,
                                               reshard_dtype_t scale_dtype, void *y, int64_t y_pitch,
                                               reshard_dtype_t dtype, void *stream) {
    return rs::guarded([&]() -> reshard_status_t {
        using namespace rs;
        reshard_status_t st = check_blocks(rows, cols, block_rows, scale_dtype);
        if (st != RESHARD_OK) return st;
        if (!is_float_type(dtype)) return fail(RESHARD_EINVAL, "dtype must be F16, BF16 or F32");
        const int64_t across = ceil_div(cols, kBlock);
        st = check_matrix("q", q, rows, cols, q_pitch, 1);
        if (st == RESHARD_OK)
            st = check_matrix("scales", scales, block_rows == 1 ? rows : ceil_div(rows, kBlock), across, scales_pitch,
                              scale_dtype == RESHARD_F32 ? 4 : 1);
        if (st == RESHARD_OK) st = check_matrix("y", y, rows, cols, y_pitch, dtype == RESHARD_F32 ? 4 : 2);
        if (st != RESHARD_OK || rows == 0 || cols == 0) return st;
        const DequantArgs a{static_cast<const uint8_t *>(q), scales, y, rows, cols, q_pitch, scales_pitch, y_pitch,
                            scale_dtype == RESHARD_E8M0, block_rows == 1 ? 0 : 7,
                            rows * cols * (dtype == RESHARD_F32 ? 4 : 2) >= int64_t(256) << 20};
        const hipStream_t s = static_cast<hipStream_t>(stream);
        const dim3 grid(unsigned(ceil_div(rows * across, 16 * kUnits)));
        auto run = [&](auto kernel) { return launch("dequantize launch", kernel, grid, 256, 0, s, a, across); };
        if (dtype == RESHARD_F32) return run(dequantize_kernel<float, false>);
        if (dtype == RESHARD_BF16) return run(a.e8m0 ? dequantize_kernel<bf16, false> : dequantize_kernel<bf16, true>);
        return run(a.e8m0 ? dequantize_kernel<f16, false> : dequantize_kernel<f16, true>);
    });
}
