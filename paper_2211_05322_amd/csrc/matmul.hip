// matmul.hip -- product of two 8-bit matrices with a scale per block of 128
// along the reduction:
//
//   out[i, j] = sum_b sa[i, b] sb[j, b] sum_{l in block b} A[i, l] B[j, l]
//
// One step of the reduction is one block of 128.  Into 16-bit results the
// 8-bit instruction 16 x 16 x 128 multiplies a whole block; it takes E8M0
// scales itself, and float scales are applied to its result, which then
// starts from zero in every step.  Inside it, eight neighbouring products are
// aligned to the largest of them and cut 13 bits below it before they enter
// the float32 sum (measured: 2^16 + 2^3 is kept, 2^16 + 2^2 is not, eight
// places away both are).  A group is so off by at most 2^-10 of its largest
// product, typically 1e-5 to 2e-4 of the sum: below the rounding of a 16-bit
// result, but not of a float32 one.  Float32 results are therefore summed by
// the bf16 instruction, into which codes convert exactly, at half the rate.
//
// B's rows are the instruction's rows and A's its columns: a lane's four
// results are then neighbours in a row of `out`, and they share A's scale.
#include <algorithm>
#include <type_traits>

#include "operators.hpp"

namespace rs {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

// How a block's products are summed.
enum Sum {
    kScaled,  // 8-bit instruction with E8M0 scales
    kFloat,   // 8-bit instruction, scales applied to its result
    kExact    // bf16 instruction, scales applied to its result
};

// 32 codes of a row: a lane's share of a block, for the 8-bit instruction as
// they are, for the bf16 one (four steps of 8) converted.
union Codes {
    uint4 h[2];
    uint32_t w[8];
    i32x8 v;
};
struct Wide {
    union {
        bf16x8 v[4];
        bf16x2 p[16];
    };
    __device__ explicit Wide(const Codes &c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.w[i], 1.0f, false);
            p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.w[i], 1.0f, true);
        }
    }
};

__device__ inline f32x4 block_product(const Wide &b, const Wide &a) {
    f32x4 p{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < 4; ++s) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[s], a.v[s], p, 0, 0, 0);
    return p;
}

__device__ inline f32x4 block_product(const Codes &b, const Codes &a) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}

struct Operand {
    const uint8_t *q;
    const void *scales;
    int64_t rows, pitch, scales_pitch;
    int row_shift;  // rows that share a scale: 1 << row_shift
};

struct MatmulArgs {
    Operand a, b;
    void *out;
    int64_t k, out_pitch;
    int out_dtype, accumulate, e8m0;
};

__device__ inline int scale_code(const Operand &o, int64_t row, int64_t block) {
    return static_cast<const uint8_t *>(o.scales)[(row >> o.row_shift) * o.scales_pitch + block];
}

__device__ inline float scale_value(const Operand &o, int e8m0, int64_t row, int64_t block) {
    if (e8m0) return e8m0_value(uint8_t(scale_code(o, row, block)));
    return static_cast<const float *>(o.scales)[(row >> o.row_shift) * o.scales_pitch + block];
}

// 16 codes of a row from l on, zeros past its k.
__device__ inline uint4 load_codes(const Operand &o, int64_t row, int64_t l, int64_t k) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (row >= o.rows || l >= k) return v;
    const uint8_t *p = o.q + row * o.pitch + l;
    if (l + 16 <= k) return load_any<uint4>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (l + i < k) w[i / 4] |= uint32_t(p[i]) << (8 * (i & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__device__ inline void store_out(const MatmulArgs &g, int64_t i, int64_t j, f32x4 v) {
    T *p = static_cast<T *>(g.out) + i * g.out_pitch + j;
    const int64_t n = g.b.rows - j;
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (n >= 4) {
        if (g.accumulate) {
            const T4 o = load_any<T4>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += float(o[e]);
        }
        T4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = T(v[e]);
        store_any(p, r);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) p[e] = T(g.accumulate ? float(p[e]) + v[e] : v[e]);
    }
}

__device__ inline void store_any_type(const MatmulArgs &g, int64_t i, int64_t j, f32x4 v) {
    if (g.out_dtype == RESHARD_F32) store_out<float>(g, i, j, v);
    else if (g.out_dtype == RESHARD_BF16) store_out<bf16>(g, i, j, v);
    else store_out<f16>(g, i, j, v);
}

// 128 x 128 of `out` a workgroup, 64 x 64 a wave.  A row of the LDS tiles is
// one block, eight 16-byte words; word w of row r lies in slot w ^ (r % 8).
template <Sum SUM>
__global__ __launch_bounds__(256) void matmul_kernel(MatmulArgs g, uint32_t tiles_n) {
    __shared__ uint4 sa[128][8], sb[128][8];
    const int64_t i0 = int64_t(blockIdx.x / tiles_n) * 128, j0 = int64_t(blockIdx.x % tiles_n) * 128;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int wi = (wave / 2) * 64, wj = (wave % 2) * 64, r16 = lane % 16, quad = lane / 16;
    f32x4 acc[4][4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[x][y] = f32x4{0, 0, 0, 0};
    const int64_t steps = ceil_div(g.k, kBlock);
    for (int64_t s = 0; s < steps; ++s) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int w = u * 256 + threadIdx.x, r = w / 8, c = w % 8;
            sa[r][c ^ (r & 7)] = load_codes(g.a, i0 + r, s * kBlock + c * 16, g.k);
            sb[r][c ^ (r & 7)] = load_codes(g.b, j0 + r, s * kBlock + c * 16, g.k);
        }
        __syncthreads();
        Codes fa[4], fb[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int ra = wi + x * 16 + r16, rb = wj + x * 16 + r16;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fa[x].h[h] = sa[ra][(quad * 2 + h) ^ (ra & 7)];
                fb[x].h[h] = sb[rb][(quad * 2 + h) ^ (rb & 7)];
            }
        }
        if constexpr (SUM == kScaled) {
            int ka[4], kb[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int64_t i = i0 + wi + x * 16 + r16, j = j0 + wj + x * 16 + r16;
                ka[x] = i < g.a.rows ? scale_code(g.a, i, s) : 127;
                kb[x] = j < g.b.rows ? scale_code(g.b, j, s) : 127;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    acc[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[y].v, fa[x].v, acc[x][y], 0, 0, 0,
                                                                                 kb[y], 0, ka[x]);
        } else {
            float ka[4], kb[4][4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int64_t i = i0 + wi + x * 16 + r16;
                ka[x] = i < g.a.rows ? scale_value(g.a, g.e8m0, i, s) : 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t j = j0 + wj + x * 16 + quad * 4 + e;
                    kb[x][e] = j < g.b.rows ? scale_value(g.b, g.e8m0, j, s) : 0.0f;
                }
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const typename std::conditional<SUM == kExact, Wide, Codes>::type b(fb[y]);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const typename std::conditional<SUM == kExact, Wide, Codes>::type a(fa[x]);
                    const f32x4 p = block_product(b, a);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[x][y][e] = fmaf(p[e], ka[x] * kb[y][e], acc[x][y][e]);
                }
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int64_t i = i0 + wi + x * 16 + r16;
        if (i >= g.a.rows) continue;
#pragma unroll
        for (int y = 0; y < 4; ++y) store_any_type(g, i, j0 + wj + y * 16 + quad * 4, acc[x][y]);
    }
}

reshard_status_t check_operand(const char *name, const char *scales_name, const void *q, int64_t rows, int64_t k,
                               int64_t pitch, int block_rows, const void *scales, int64_t scales_pitch,
                               reshard_dtype_t scale_dtype) {
    if (block_rows != 1 && block_rows != kBlock)
        return fail(RESHARD_EINVAL, std::string(name) + "_block_rows must be 1 or 128");
    reshard_status_t st = check_matrix(name, q, rows, k, pitch, 1);
    if (st != RESHARD_OK) return st;
    return check_matrix(scales_name, scales, block_rows == 1 ? rows : ceil_div(rows, kBlock), ceil_div(k, kBlock),
                        scales_pitch, scale_dtype == RESHARD_F32 ? 4 : 1);
}

}  // namespace
}  // namespace rs

using rs::fail;

extern "C" int64_t reshard_matmul_workspace(int64_t m, int64_t n, int64_t k) {
    if (m < 0 || n < 0 || k < 0) return -1;
    return 0;
}

extern "C" reshard_status_t reshard_matmul(int64_t m, int64_t n, int64_t k, const void *a, int64_t a_pitch,
                                           int a_block_rows, const void *a_scales, int64_t a_scales_pitch,
                                           const void *b, int64_t b_pitch, int b_block_rows, const void *b_scales,
                                           int64_t b_scales_pitch, reshard_dtype_t scale_dtype, void *out,
                                           int64_t out_pitch, reshard_dtype_t out_dtype, int accumulate,
                                           void *workspace, int64_t workspace_bytes, void *stream) {
    return rs::guarded([&]() -> reshard_status_t {
        using namespace rs;
        reshard_status_t st = check_extent("m", m);
        if (st == RESHARD_OK) st = check_extent("n", n);
        if (st == RESHARD_OK) st = check_extent("k", k);
        if (st != RESHARD_OK) return st;
        if (scale_dtype != RESHARD_E8M0 && scale_dtype != RESHARD_F32)
            return fail(RESHARD_EINVAL, "scale_dtype must be E8M0 or F32");
        if (!is_float_type(out_dtype)) return fail(RESHARD_EINVAL, "out_dtype must be F16, BF16 or F32");
        if (accumulate & ~1) return fail(RESHARD_EINVAL, "accumulate must be 0 or 1");
        st = check_operand("a", "a_scales", a, m, k, a_pitch, a_block_rows, a_scales, a_scales_pitch, scale_dtype);
        if (st == RESHARD_OK)
            st = check_operand("b", "b_scales", b, n, k, b_pitch, b_block_rows, b_scales, b_scales_pitch, scale_dtype);
        if (st == RESHARD_OK)
            st = check_matrix("out", out, m, n, out_pitch, out_dtype == RESHARD_F32 ? 4 : 2);
        if (st != RESHARD_OK || m == 0 || n == 0) return st;
        const int64_t tiles_m = ceil_div(m, 128), tiles_n = ceil_div(n, 128);
        if (tiles_n > (int64_t(1) << 23) / tiles_m)
            return fail(RESHARD_EUNSUPPORTED, "out has more than 2^23 tiles of 128 x 128");
        MatmulArgs g{};
        g.a = Operand{static_cast<const uint8_t *>(a), a_scales, m, a_pitch, a_scales_pitch, a_block_rows == 1 ? 0 : 7};
        g.b = Operand{static_cast<const uint8_t *>(b), b_scales, n, b_pitch, b_scales_pitch, b_block_rows == 1 ? 0 : 7};
        g.out = out;
        g.k = k;
        g.out_pitch = out_pitch;
        g.out_dtype = int(out_dtype);
        g.accumulate = accumulate;
        g.e8m0 = scale_dtype == RESHARD_E8M0;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        const dim3 grid(unsigned(tiles_m * tiles_n));
        if (out_dtype == RESHARD_F32) matmul_kernel<kExact><<<grid, 256, 0, s>>>(g, uint32_t(tiles_n));
        else if (g.e8m0) matmul_kernel<kScaled><<<grid, 256, 0, s>>>(g, uint32_t(tiles_n));
        else matmul_kernel<kFloat><<<grid, 256, 0, s>>>(g, uint32_t(tiles_n));
        return launched("matmul launch");
    });
}
