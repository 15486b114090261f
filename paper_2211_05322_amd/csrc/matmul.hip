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
#include <utility>

#include "operators.hpp"

namespace rs {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

// How a block's products are summed.
enum Sum {
    kScaled,   // 8-bit instruction with E8M0 scales
    kFloat,    // 8-bit instruction, scales applied to its result
    kUniform,  // the same where all of a wave's rows of B share a scale
    kExact,    // bf16 instruction, scales applied to its result
    kWide      // bf16 instruction, E8M0 scales applied as codes are converted
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
    // times a power of two (its exponent 0 stands for 2^-127, 255 gives NaN, as in E8M0)
    __device__ explicit Wide(const Codes &c, float scale = 1.0f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.w[i], scale, false);
            p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.w[i], scale, true);
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
    float *parts;  // [parts of the reduction][m][n], where it is split
    int64_t k, out_pitch;
    int out_dtype, accumulate, e8m0;
};

__device__ inline int scale_code(const Operand &o, int64_t row, int64_t block) {
    return static_cast<const uint8_t *>(o.scales)[(row >> o.row_shift) * o.scales_pitch + block];
}

__device__ inline f32x16 zeros() {
    f32x16 z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0;
    return z;
}

// The same for half a block and tiles of 32 x 32, added to p.
template <Sum SUM>
__device__ inline f32x16 block_product(const Wide &b, const Wide &a, f32x16 p) {
#pragma unroll
    for (int s = 0; s < 4; ++s) p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.v[s], a.v[s], p, 0, 0, 0);
    return p;
}

template <Sum SUM>
__device__ inline f32x16 block_product(const Codes &b, const Codes &a, f32x16 p) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b.v, a.v, p, 0, 0, 0, 0, 0, 0);
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

// Operands whose rows start anywhere, or lie too far apart for the tile
// kernel's 32-bit offsets: codes go through registers, a step ahead, 128 x 128
// of `out` a workgroup, 64 x 64 a wave.  Bound by those loads, which straddle
// cache lines, and two barriers a step: 8192 x 8192 x 4096 with rows 4097 apart
// takes 692 us (249 in tiles on 16-byte boundaries), 811 into float32 (463; this
// instantiation spills 3 registers).
// A row of the LDS tiles is one block, eight 16-byte words; word w of row r
// lies in slot w ^ (r % 8).
template <Sum SUM>
__global__ __launch_bounds__(256, 2) void matmul_kernel(MatmulArgs g, uint32_t tiles_n) {
    using Scale = typename std::conditional<SUM == kScaled, int, float>::type;
    __shared__ uint4 sa[128][8], sb[128][8];
    __shared__ __align__(16) Scale sk[256];  // of A's rows, then of B's
    const int64_t i0 = int64_t(blockIdx.x / tiles_n) * 128, j0 = int64_t(blockIdx.x % tiles_n) * 128;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int wi = (wave / 2) * 64, wj = (wave % 2) * 64, r16 = lane % 16, quad = lane / 16;
    f32x4 acc[4][4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[x][y] = f32x4{0, 0, 0, 0};
    const int64_t steps = ceil_div(g.k, kBlock), whole = g.k / kBlock;
    // A thread's words of a block, loaded while the block before is multiplied;
    // rows past a matrix's end repeat its last, whose results are not stored.
    const int row0 = threadIdx.x / 8, word = threadIdx.x % 8;
    uint4 a_next[4], b_next[4];
    Scale k_next;
    const Operand &mine = threadIdx.x < 128 ? g.a : g.b;
    const int64_t k_row = min((threadIdx.x < 128 ? i0 : j0 - 128) + threadIdx.x, mine.rows - 1);
    auto load = [&](int64_t s) {
        const int64_t l = s * kBlock + word * 16;
        if constexpr (SUM == kScaled) k_next = scale_code(mine, k_row, s);
        else k_next = scale_value(mine, g.e8m0, k_row, s);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t i = min(i0 + row0 + u * 32, g.a.rows - 1), j = min(j0 + row0 + u * 32, g.b.rows - 1);
            if (s < whole) {
                a_next[u] = load_any<uint4>(g.a.q + i * g.a.pitch + l);
                b_next[u] = load_any<uint4>(g.b.q + j * g.b.pitch + l);
            } else {
                a_next[u] = load_codes(g.a, i, l, g.k);
                b_next[u] = load_codes(g.b, j, l, g.k);
            }
        }
    };
    if (steps > 0) load(0);
    for (int64_t s = 0; s < steps; ++s) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = row0 + u * 32;
            sa[r][word ^ (r & 7)] = a_next[u];
            sb[r][word ^ (r & 7)] = b_next[u];
        }
        sk[threadIdx.x] = k_next;
        __syncthreads();
        if (s + 1 < steps) load(s + 1);
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
                ka[x] = sk[wi + x * 16 + r16];
                kb[x] = sk[128 + wj + x * 16 + r16];
            }
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    acc[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[y].v, fa[x].v, acc[x][y], 0, 0, 0,
                                                                                 kb[y], 0, ka[x]);
        } else {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const typename std::conditional<SUM == kExact, Wide, Codes>::type b(fb[y]);
                const f32x4 kb = *reinterpret_cast<const f32x4 *>(&sk[128 + wj + y * 16 + quad * 4]);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const typename std::conditional<SUM == kExact, Wide, Codes>::type a(fa[x]);
                    const f32x4 p = block_product(b, a);
                    const float ka = sk[wi + x * 16 + r16];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[x][y][e] = fmaf(p[e], ka * kb[e], acc[x][y][e]);
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

// Eight neighbouring results.
template <typename T>
__device__ inline void store_eight(const MatmulArgs &g, int64_t i, int64_t j, f32x4 lo, f32x4 hi) {
    T *p = static_cast<T *>(g.out) + i * g.out_pitch + j;
    const int64_t n = g.b.rows - j;
    typedef T T8 __attribute__((ext_vector_type(8)));
    float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    if (n >= 8) {
        T8 r;
        if (g.accumulate) r = load_any<T8>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = T(g.accumulate ? float(r[e]) + v[e] : v[e]);
        store_any(p, r);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = T(g.accumulate ? float(p[e]) + v[e] : v[e]);
    }
}

__device__ inline void store_run(const MatmulArgs &g, int64_t i, int64_t j, f32x4 lo, f32x4 hi) {
    if (g.out_dtype == RESHARD_F32) store_eight<float>(g, i, j, lo, hi);
    else if (g.out_dtype == RESHARD_BF16) store_eight<bf16>(g, i, j, lo, hi);
    else store_eight<f16>(g, i, j, lo, hi);
}

struct Tile {
    uint32_t i, j;
};

// Workgroups start on the 8 XCDs in turn.  Each XCD takes a contiguous run of
// the tiles, ordered in bands of kBand rows of tiles, column by column, so
// that the tiles in flight there share rows of A and of B in its L2.
constexpr uint32_t kBand = 8;
__device__ inline Tile tile_of(uint32_t wg, uint32_t tiles, uint32_t tiles_n) {
    const uint32_t xcd = wg % 8, each = tiles / 8, more = tiles % 8;
    const uint32_t p = xcd * each + min(xcd, more) + wg / 8;
    const uint32_t band = p / (kBand * tiles_n), r = p - band * (kBand * tiles_n);
    const uint32_t rows = min(kBand, tiles / tiles_n - band * kBand), j = r / rows;
    return Tile{uint32_t(__builtin_amdgcn_readfirstlane(band * kBand + (r - j * rows))),
                uint32_t(__builtin_amdgcn_readfirstlane(j))};
}

template <typename F, int... I>
__device__ inline void each(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}

// f(0), f(1), ..., f(N - 1) with constants.
template <int N, typename F>
__device__ inline void unrolled(F &&f) {
    each(f, std::make_integer_sequence<int, N>{});
}

// The large products: a WM x WN grid of waves, each TM x TN instruction tiles
// of 32 x 32.  A block of both operands' rows goes from memory into LDS
// without passing through registers, while the block before it is multiplied
// (two LDS buffers).
//
// An instruction takes half a block, so a step has two phases.  While one is
// multiplied, row of tiles by row of tiles, the fragments of the next are
// read: B's and the last rows' of A beside those in use, the first rows' of A
// in place of them once they are done.  The step's one barrier lies between
// its phases: there a wave holds the rest of its block in registers, so that
// the block two steps ahead can be loaded over it, and the next block, loaded
// since the last barrier, can be read.
//
// LDS rows are 128 bytes, eight 16-byte words, word w of row r in slot
// w ^ (r / 2 % 8): lanes that read at once fall on different banks.  The loads
// write LDS in order, so the order of words is set by the addresses they read.
//
// With E8M0 scales bound by the matrix instructions, and by the power they take:
// 16384 x 12288 x 12288 in 256 x 256 tiles runs at 2620 to 2650 TFLOP/s (on
// zeros, which take less power, at 2920); in 8192 x 4096 x 16384 the instruction
// is busy 73 % of the cycles.  Waves of 128 x 128, which read a third less from
// LDS, measured the same.  Float scales cost an operation an element and block
// beside it: 1540 to 1810 TFLOP/s with a scale per tile of B, 1460 to 1490 with
// one per row.  There neither unit is the bound (matrix instructions busy 43 %
// and vector ones 36 % of the cycles, per row 34 and 45) but that they overlap
// little.  Float32 results cost the conversion and the bf16 instruction's half
// rate: 1280 TFLOP/s with E8M0 scales, 1020 to 1040 with float ones.  kWide in
// 256 x 256 tiles spills 21 registers and is faster than 128 x 128 all the same.
template <int ROWS>
struct Stage {
    uint4 words[ROWS * 8];
};

template <Sum SUM, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(WM *WN *kWave, 2) void matmul_tile_kernel(MatmulArgs g, uint32_t tiles_n, int32_t blocks) {
    constexpr int THREADS = WM * WN * kWave, BM = WM * TM * 32, BN = WN * TN * 32;
    constexpr int LA = BM * 8 / THREADS, LB = BN * 8 / THREADS;  // 16-byte loads a thread and step
    constexpr int ROWS_AT_ONCE = THREADS / 8;
    constexpr int SROWS = (BM + BN) / THREADS;  // scales a thread and step
    constexpr bool E8M0 = SUM == kScaled || SUM == kWide;  // else the block's sum is scaled
    using Scale = typename std::conditional<E8M0, uint8_t, float>::type;
    __shared__ Stage<BM> a_lds0, a_lds1;
    __shared__ Stage<BN> b_lds0, b_lds1;
    __shared__ __align__(16) Scale s_lds[3][BM + BN];  // three: a step's may be read while those two ahead are written

    const Tile at = tile_of(blockIdx.x, gridDim.x, tiles_n);
    const int64_t i0 = int64_t(at.i) * BM, j0 = int64_t(at.j) * BN;
    const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
    const int r32 = lane % 32, half = lane / 32, wi = wave / WN, wj = wave % WN;
    if (gridDim.y > 1) {  // this workgroup's part of the reduction, to a place of its own
        const int64_t first = int64_t(blockIdx.y) * blocks;
        g.a.q += first * kBlock;
        g.b.q += first * kBlock;
        g.a.scales = static_cast<const Scale *>(g.a.scales) + first;
        g.b.scales = static_cast<const Scale *>(g.b.scales) + first;
        g.k = min(g.k - first * kBlock, int64_t(blocks) * kBlock);
        g.out = g.parts + int64_t(blockIdx.y) * g.a.rows * g.b.rows;
        g.out_pitch = g.b.rows;
        g.out_dtype = RESHARD_F32;
        g.accumulate = 0;
    }
    const int32_t steps = int32_t(ceil_div(g.k, kBlock));
    const int32_t paired = int32_t(g.k / (2 * kBlock)) * 2;  // whole blocks, two at a time

    // rows past a matrix's end are read as zeros
    const int lrow = t / 8, lword = (t % 8) ^ ((lrow / 2) % 8);
    const uint32_t a_off = lrow * uint32_t(g.a.pitch) + lword * 16, b_off = lrow * uint32_t(g.b.pitch) + lword * 16;
    const uint32_t a_next_rows = ROWS_AT_ONCE * uint32_t(g.a.pitch), b_next_rows = ROWS_AT_ONCE * uint32_t(g.b.pitch);
    const __amdgpu_buffer_rsrc_t a_base =
        bytes_from(g.a.q + i0 * g.a.pitch, (g.a.rows - 1 - i0) * g.a.pitch + g.k);
    const __amdgpu_buffer_rsrc_t b_base =
        bytes_from(g.b.q + j0 * g.b.pitch, (g.b.rows - 1 - j0) * g.b.pitch + g.k);
    auto stage_one = [&](int32_t s, auto &a_lds, auto &b_lds, auto u_) {
        constexpr int u = decltype(u_)::value;
        if constexpr (u < LA)
            load_to_lds(a_base, a_off + (u * a_next_rows + s * kBlock), &a_lds.words[u * THREADS + wave * kWave]);
        else
            load_to_lds(b_base, b_off + ((u - LA) * b_next_rows + s * kBlock),
                        &b_lds.words[(u - LA) * THREADS + wave * kWave]);
    };
    auto stage = [&](int32_t s, auto &a_lds, auto &b_lds) {
        unrolled<LA + LB>([&](auto u) { stage_one(s, a_lds, b_lds, u); });
    };

    // A row's scales lie a row apart from the next row's, so each load of them
    // touches as many cache lines as it has lanes: two steps' at once.
    using Two = typename std::conditional<E8M0, uint16_t, uint64_t>::type;
    const Scale *s_at[SROWS];
    int s_to[SROWS];
    Two s_held[SROWS], s_next[SROWS];
#pragma unroll
    for (int u = 0; u < SROWS; ++u) {
        const int r = t + u * THREADS;
        const bool is_a = r < BM;
        const Operand &o = is_a ? g.a : g.b;
        const int rr = is_a ? r : r - BM, T = is_a ? TM : TN;
        const int64_t row = min((is_a ? i0 : j0) + rr, o.rows - 1);
        s_at[u] = static_cast<const Scale *>(o.scales) + (row >> o.row_shift) * o.scales_pitch;
        // [wave's row][r32][tile]: a lane's scales of all tiles lie together
        s_to[u] = is_a || E8M0 ? (is_a ? 0 : BM) + rr / (T * 32) * (T * 32) + rr % 32 * T + rr / 32 % T : r;
    }
    // Of blocks s and s + 1; past the last, any.  Nothing is computed from
    // what is loaded before it is put into LDS, so that nothing waits for it.
    auto load_scales = [&](int32_t s, Two (&to)[SROWS]) {
#pragma unroll
        for (int u = 0; u < SROWS; ++u) to[u] = load_any<Two>(s_at[u] + min(s, steps - 2));
    };
    auto put_scales = [&](int buf, int32_t s, int32_t block) {  // block's, from those loaded for s and s + 1
        const int shift = block > min(s, steps - 2) ? 4 * int(sizeof(Two)) : 0;
#pragma unroll
        for (int u = 0; u < SROWS; ++u) {
            const Two w = Two(s_held[u] >> shift);
            __builtin_memcpy(&s_lds[buf][s_to[u]], &w, sizeof(Scale));
        }
    };

    // A lane's share of 32 rows' half block: words half and half + 2 of a row,
    // or half + 4 and half + 6.  Which element of the block is which of the
    // instruction's does not matter, as long as A and B agree.  One address a
    // word and operand, with the tile and the buffer in the instruction's
    // offset: left to itself, the compiler keeps a register for each.
    uint32_t a_word[4], b_word[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t word = r32 * 8 + ((half + 2 * p) ^ ((r32 / 2) % 8));
        a_word[p] = wi * TM * 256 + word;
        b_word[p] = wj * TN * 256 + word;
        asm("" : "+v"(a_word[p]), "+v"(b_word[p]));
    }
    auto read = [&](auto &lds, const uint32_t (&word)[4], int part, int tile) {
        Codes c;
        c.h[0] = lds.words[word[2 * part] + tile * 256];
        c.h[1] = lds.words[word[2 * part + 1] + tile * 256];
        return c;
    };

    f32x16 acc[TM][TN], sum[TM][TN];  // sum: of the block at hand, where its scales are applied to it
    unrolled<TM>([&](auto x) { unrolled<TN>([&](auto y) { acc[x][y] = zeros(); }); });
    constexpr int TWO = TM / 2;  // rows of tiles from here on have two sets of registers
    Codes fa[TM], fa_odd[TM - TWO], fb[2][TN];
    auto frag_a = [&](auto part, auto x) -> Codes & {
        if constexpr (decltype(part)::value == 1 && decltype(x)::value >= TWO) return fa_odd[decltype(x)::value - TWO];
        else return fa[decltype(x)::value];
    };
    int ka[2], kb[2];  // E8M0: the tiles' exponents, a byte each
    float kf[2][TM];   // else: A's scales (kUniform: times B's)
    auto read_scales = [&](const Scale *sc, int into) {
        if constexpr (E8M0) {
            using Bytes_m = typename std::conditional<TM == 4, uint32_t, uint16_t>::type;
            using Bytes_n = typename std::conditional<TN == 4, uint32_t, uint16_t>::type;
            ka[into] = *reinterpret_cast<const Bytes_m *>(&sc[wi * TM * 32 + r32 * TM]);
            kb[into] = *reinterpret_cast<const Bytes_n *>(&sc[BM + wj * TN * 32 + r32 * TN]);
        } else {
#pragma unroll
            for (int x = 0; x < TM; ++x) {
                kf[into][x] = sc[wi * TM * 32 + r32 * TM + x];
                if constexpr (SUM == kUniform) kf[into][x] *= sc[BM + wj * TN * 32];
            }
        }
    };

    constexpr std::integral_constant<int, 0> low{};
    constexpr std::integral_constant<int, 1> high{};
    int sbuf = 0;  // the step's scales, of three
    auto product = [&](auto cur_, auto part, auto x_, auto y_) {
        constexpr int cur = decltype(cur_)::value, x = decltype(x_)::value, y = decltype(y_)::value;
        const Codes &a = frag_a(part, x_), &b = fb[part][y];
        if constexpr (SUM == kScaled) {
            acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b.v, a.v, acc[x][y], 0, 0, y, kb[cur], x, ka[cur]);
        } else if constexpr (SUM == kWide) {
            auto scale = [](int codes, int i) { return __uint_as_float((uint32_t(codes) >> (8 * i) & 255) << 23); };
            acc[x][y] = block_product<SUM>(Wide(b, scale(kb[cur], y)), Wide(a, scale(ka[cur], x)), acc[x][y]);
        } else {
            const f32x16 before = decltype(part)::value ? sum[x][y] : zeros();
            if constexpr (SUM == kExact) sum[x][y] = block_product<SUM>(Wide(b), Wide(a), before);
            else sum[x][y] = block_product<SUM>(b, a, before);
        }
    };
    // A row of tiles' sums over the block, scaled, to the results.
    auto scale_row = [&](auto cur_, auto x_) {
        constexpr int cur = decltype(cur_)::value, x = decltype(x_)::value;
        unrolled<TN>([&](auto y) {
            unrolled<4>([&](auto q_) {
                constexpr int q = decltype(q_)::value;
                f32x4 k{kf[cur][x], kf[cur][x], kf[cur][x], kf[cur][x]};
                if constexpr (SUM != kUniform)
                    k *= *reinterpret_cast<const f32x4 *>(&s_lds[sbuf][BM + (wj * TN + y) * 32 + q * 8 + half * 4]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[x][y][q * 4 + e] = fmaf(sum[x][y][q * 4 + e], k[e], acc[x][y][q * 4 + e]);
            });
        });
    };
    // One phase: a_from and b_from are the buffers that the other part's
    // fragments are read from, and load(x) what else is done beside a row.
    auto phase = [&](auto cur, auto part, auto &a_from, auto &b_from, auto &&load) {
        constexpr std::integral_constant<int, decltype(part)::value ^ 1> other{};
        unrolled<TM>([&](auto x_) {
            constexpr int x = decltype(x_)::value;
            if constexpr (x == 0) {
                unrolled<TN>([&](auto y) { fb[other][y] = read(b_from, b_word, other, y); });
            }
            if constexpr (x > 0 && x <= TWO) {
                frag_a(other, std::integral_constant<int, x - 1>{}) = read(a_from, a_word, other, x - 1);
            }
            if constexpr (x < TM - TWO) {
                frag_a(other, std::integral_constant<int, TWO + x>{}) = read(a_from, a_word, other, TWO + x);
            }
            load(x_);
            unrolled<TN>([&](auto y) { product(cur, part, x_, y); });
            // the row before this one, whose products are done by now
            if constexpr (!E8M0 && decltype(part)::value == 1 && x > 0)
                scale_row(cur, std::integral_constant<int, x - 1>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (!E8M0 && decltype(part)::value == 1) scale_row(cur, std::integral_constant<int, TM - 1>{});
    };
    auto step = [&](auto cur_, int32_t s, auto &a_cur, auto &b_cur, auto &a_next, auto &b_next) {
        constexpr int cur = decltype(cur_)::value, EACH = (LA + LB + TM - 1) / TM;
        const int snext = sbuf == 2 ? 0 : sbuf + 1;
        const int32_t ahead = min(s + 2, paired - 1);
        phase(cur_, low, a_cur, b_cur, [](auto) {});
        // the last step's reads ahead find an older block, which is not used
        put_scales(snext, s + 1 - cur, s + 1);
        loads_done();
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        read_scales(s_lds[snext], cur ^ 1);
        if constexpr (cur == 1) {  // those of s + 2 and s + 3 were loaded two steps ago
#pragma unroll
            for (int u = 0; u < SROWS; ++u) s_held[u] = s_next[u];
            load_scales(s + 4, s_next);
        }
        phase(cur_, high, a_next, b_next, [&](auto x) {
            unrolled<EACH>([&](auto e) {
                constexpr int u = decltype(x)::value * EACH + decltype(e)::value;
                if constexpr (u < LA + LB) stage_one(ahead, a_cur, b_cur, std::integral_constant<int, u>{});
            });
        });
        sbuf = snext;
    };

    if (paired > 0) {
        load_scales(0, s_held);
        stage(0, a_lds0, b_lds0);
        put_scales(0, 0, 0);
        load_scales(1, s_held);
        load_scales(3, s_next);
        loads_done();
        stage(1, a_lds1, b_lds1);
        __syncthreads();
        read_scales(s_lds[0], 0);
        unrolled<TM>([&](auto x) { fa[x] = read(a_lds0, a_word, 0, x); });
        unrolled<TN>([&](auto y) { fb[0][y] = read(b_lds0, b_word, 0, y); });
        for (int32_t s = 0; s < paired; s += 2) {
            step(low, s, a_lds0, b_lds0, a_lds1, b_lds1);
            step(high, s + 1, a_lds1, b_lds1, a_lds0, b_lds0);
        }
        loads_done();
        __syncthreads();
    }
    // An odd block, and a short one, whose missing codes are zeros.  (An odd one in the pipeline above would save 3 %
    // where there are 15 and cost all others 1 %, in spilled registers.)
#pragma unroll 1
    for (int32_t s = paired; s < steps; ++s) {
        const int64_t l = int64_t(s) * kBlock + lword * 16;
#pragma unroll 1
        for (int u = 0; u < LA; ++u)
            a_lds0.words[u * THREADS + t] = load_codes(g.a, i0 + lrow + u * ROWS_AT_ONCE, l, g.k);
#pragma unroll 1
        for (int u = 0; u < LB; ++u)
            b_lds0.words[u * THREADS + t] = load_codes(g.b, j0 + lrow + u * ROWS_AT_ONCE, l, g.k);
#pragma unroll
        for (int u = 0; u < SROWS; ++u) s_lds[0][s_to[u]] = s_at[u][s];
        sbuf = 0;
        __syncthreads();
        read_scales(s_lds[0], 0);
        unrolled<TM>([&](auto x) { fa[x] = read(a_lds0, a_word, 0, x); });
        unrolled<TN>([&](auto y) { fb[0][y] = read(b_lds0, b_word, 0, y); });
        phase(low, low, a_lds0, b_lds0, [](auto) {});
        phase(low, high, a_lds0, b_lds0, [](auto) {});
        __syncthreads();
    }

    // Each wave turns its results, 32 rows of one column of tiles at a time,
    // through its part of LDS (float32, 16-byte word w of row r in slot
    // w ^ (r % 8)), so that lanes store runs of a row.
    f32x4 *turn = reinterpret_cast<f32x4 *>(a_lds0.words) + wave * 256;
    static_assert(WM * WN * 256 * sizeof(f32x4) <= sizeof(a_lds0.words), "LDS for the results");
    unrolled<TM>([&](auto x) {
        unrolled<TN>([&](auto y) {
            unrolled<4>([&](auto q_) {
                constexpr int q = decltype(q_)::value;
                turn[r32 * 8 + ((q * 2 + half) ^ (r32 % 8))] =
                    f32x4{acc[x][y][q * 4], acc[x][y][q * 4 + 1], acc[x][y][q * 4 + 2], acc[x][y][q * 4 + 3]};
            });
#pragma unroll 1
            for (int r = lane / 4; r < 32; r += 16) {
                const int w = lane % 4 * 2;
                const f32x4 lo = turn[r * 8 + (w ^ (r % 8))], hi = turn[r * 8 + ((w + 1) ^ (r % 8))];
                const int64_t i = i0 + (wi * TM + x) * 32 + r, j = j0 + (wj * TN + y) * 32 + w * 4;
                if (i < g.a.rows) store_run(g, i, j, lo, hi);
            }
        });
    });
}

// Adds the parts of a split reduction, in order: eight neighbouring results a
// thread, parts from the caches.  Four parts of 64 x 15360 in 4.4 us.
__global__ __launch_bounds__(256) void matmul_join_kernel(MatmulArgs g, int parts) {
    const uint32_t across = uint32_t(ceil_div(g.b.rows, 8)), total = uint32_t(g.a.rows) * across;  // at most 2^31
    for (uint32_t at = blockIdx.x * 256 + threadIdx.x; at < total; at += gridDim.x * 256) {
        const int64_t i = at / across, j = int64_t(at % across) * 8;
        const float *p = g.parts + i * g.b.rows + j;
        f32x4 lo{0, 0, 0, 0}, hi{0, 0, 0, 0};
        for (int s = 0; s < parts; ++s, p += g.a.rows * g.b.rows) {
            const Pack<float> x = load_pack(p, g.b.rows - j), y = load_pack(p + 4, g.b.rows - j - 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] += x.e[e];
                hi[e] += y.e[e];
            }
        }
        store_run(g, i, j, lo, hi);
    }
}

// Few rows of A: the weights' bytes are the work.  A workgroup takes 16 rows
// of B and all of A's (at most 16); its waves deal the blocks of the reduction
// among them, load DEPTH blocks' fragments at once straight into registers,
// and add their sums through LDS.  Bound by memory: 1 x 12288 x 12288 in 30 us,
// 5.0 TB/s of weights, and in 31 with float scales; eight rows in 38 and 41.
template <Sum SUM, int WAVES, int DEPTH>
__global__ __launch_bounds__(WAVES *kWave) void matmul_few_kernel(MatmulArgs g) {
    __shared__ f32x4 part[WAVES][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, r16 = lane % 16, quad = lane / 16;
    const int64_t j0 = int64_t(blockIdx.x) * 16;
    const int32_t steps = int32_t(ceil_div(g.k, kBlock)), full = int32_t(g.k / kBlock);
    // rows past a matrix's end repeat its last, whose results are not stored
    const int64_t i = min(int64_t(r16), g.a.rows - 1), j = min(j0 + r16, g.b.rows - 1);
    const uint8_t *a_at = g.a.q + i * g.a.pitch + quad * 16, *b_at = g.b.q + j * g.b.pitch + quad * 16;
    f32x4 acc{0, 0, 0, 0};

    // blocks s0, s0 + WAVES, ..., `depth` of them; `whole`: none is the short one at the end
    auto blocks = [&](int32_t s0, auto depth, auto whole) {
        constexpr int D = decltype(depth)::value;
        Codes fa[D], fb[D];
        float ka[D], kb[D][4];
        int ea[D], eb[D];
        auto load = [&](const Operand &o, const uint8_t *at, int64_t row, int64_t s) {
            Codes c;
            if constexpr (decltype(whole)::value) {
                c.h[0] = load_any<uint4>(at + s * kBlock);
                c.h[1] = load_any<uint4>(at + s * kBlock + 64);
            } else {
                c.h[0] = load_codes(o, row, s * kBlock + quad * 16, g.k);
                c.h[1] = load_codes(o, row, s * kBlock + quad * 16 + 64, g.k);
            }
            return c;
        };
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int64_t s = s0 + d * WAVES;
            fb[d] = load(g.b, b_at, j, s);
            fa[d] = load(g.a, a_at, i, s);
            if constexpr (SUM == kScaled) {
                eb[d] = scale_code(g.b, j, s);
                ea[d] = scale_code(g.a, i, s);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    kb[d][e] = scale_value(g.b, 0, min(j0 + quad * 4 + e, g.b.rows - 1), s);
                ka[d] = scale_value(g.a, 0, i, s);
            }
        }
#pragma unroll
        for (int d = 0; d < D; ++d) {
            if constexpr (SUM == kScaled) {
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[d].v, fa[d].v, acc, 0, 0, 0, eb[d], 0, ea[d]);
            } else {
                const f32x4 p = block_product(fb[d], fa[d]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e], ka[d] * kb[d][e], acc[e]);
            }
        }
    };
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::integral_constant<bool, true> whole{};
    int32_t s = wave;
    for (; s + (DEPTH - 1) * WAVES < full; s += DEPTH * WAVES) blocks(s, std::integral_constant<int, DEPTH>{}, whole);
    for (; s < full; s += WAVES) blocks(s, one, whole);
    if (s < steps) blocks(s, one, std::integral_constant<bool, false>{});

    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) acc += part[w][lane];
        if (r16 < g.a.rows && j0 + quad * 4 < g.b.rows) store_any_type(g, r16, j0 + quad * 4, acc);
    }
}

// How a product is launched: up to 8 rows of A into 16-bit results by its
// weights' rows alone (1 x 12288 x 12288: 31 us against 37 in tiles; 8 x 5120 x
// 5120: 11 against 15; but 16 x 15360 x 5120: 29 against 23); otherwise in tiles
// of 256 x 256 (E8M0 operands, where there are enough of them: 16384 x 4096 x
// 8192 into float32 861 us against 934, 4098 x 5130 x 2047 136 against 124) or
// 128 x 128, and where those are too few for the 256 CUs, the reduction split
// into parts that are joined.  (The times are those that the rules were set by;
// the kernels' present ones stand with them.)
struct Launch {
    bool few, large;
    int64_t tile, tiles_m, tiles_n;
    int32_t parts, blocks;  // parts of the reduction, and the blocks of each
};

// At most 2^20 tiles of 128 x 128 in `out`.  Extents up to 2^40 have as many
// tiles as 64 bits do not count, so this comes before launch_of.
bool too_many_tiles(int64_t m, int64_t n) { return ceil_div(n, 128) > (int64_t(1) << 20) / ceil_div(m, 128); }

Launch launch_of(int64_t m, int64_t n, int64_t k, Sum sum) {
    Launch p{};
    p.few = m <= 8 && (sum == kScaled || sum == kFloat);
    const int64_t steps = ceil_div(k, kBlock);
    auto tiles = [&](int64_t side) { return ceil_div(m, side) * ceil_div(n, side); };
    // rounds over the CUs: one tile of 256 x 256 on each, or two of 128 x 128 in the measured share of its time,
    // 2/3 with scaled 8-bit instructions and 7/13 with bf16 ones (half, if both sizes ran equally well)
    const int64_t large = ceil_div(tiles(256), 256), small = ceil_div(tiles(128), 512);
    p.large = sum == kScaled ? large * 3 <= small * 2 : sum == kWide && large * 13 <= small * 7;
    p.tile = p.large ? 256 : 128;
    p.tiles_m = ceil_div(m, p.tile);
    p.tiles_n = ceil_div(n, p.tile);
    p.parts = 1;
    if (!p.few && tiles(128) <= 256) {
        const int64_t most = std::min<int64_t>(std::max<int64_t>(1, steps / 8), 32);
        p.parts = int32_t(std::min(most, std::max<int64_t>(1, 512 / tiles(128))));
    }
    p.blocks = int32_t(ceil_div(ceil_div(std::max<int64_t>(steps, 1), p.parts), 2) * 2);
    p.parts = int32_t(ceil_div(std::max<int64_t>(steps, 1), p.blocks));
    return p;
}

Sum sum_for(reshard_dtype_t scale_dtype, reshard_dtype_t out_dtype) {
    if (out_dtype == RESHARD_F32) return scale_dtype == RESHARD_E8M0 ? kWide : kExact;
    return scale_dtype == RESHARD_E8M0 ? kScaled : kFloat;
}

constexpr const char *kLaunch = "matmul launch";

template <Sum SUM>
reshard_status_t launch_few(const MatmulArgs &g, hipStream_t s) {
    const dim3 grid(unsigned(ceil_div(g.b.rows, 16)));
    if (grid.x >= 256) return launch(kLaunch, matmul_few_kernel<SUM, 4, 8>, grid, 4 * kWave, 0, s, g);
    // more waves a row where rows are few
    return launch(kLaunch, matmul_few_kernel<SUM, 16, 2>, grid, 16 * kWave, 0, s, g);
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

extern "C" int64_t reshard_matmul_workspace(int64_t m, int64_t n, int64_t k, reshard_dtype_t scale_dtype,
                                            reshard_dtype_t out_dtype) {
    if (m < 0 || n < 0 || k < 0 || m > int64_t(1) << 40 || n > int64_t(1) << 40 || k > int64_t(1) << 36) return -1;
    if (m == 0 || n == 0) return 0;
    if (rs::too_many_tiles(m, n)) return -1;
    const rs::Launch p = rs::launch_of(m, n, k, rs::sum_for(scale_dtype, out_dtype));
    return p.parts > 1 ? int64_t(p.parts) * m * n * int64_t(sizeof(float)) : 0;
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
        if (too_many_tiles(m, n))
            return fail(RESHARD_EUNSUPPORTED, "out has more than 2^20 tiles of 128 x 128");
        if (k > int64_t(1) << 36) return fail(RESHARD_EUNSUPPORTED, "k is above 2^36");
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
        const Sum sum = sum_for(scale_dtype, out_dtype);
        const Launch p = launch_of(m, n, k, sum);
        if (p.few) return sum == kScaled ? launch_few<kScaled>(g, s) : launch_few<kFloat>(g, s);
        // the tile kernel's loads into LDS: whole 16-byte words, 32-bit offsets within a tile's rows
        const bool aligned = (reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | uintptr_t(a_pitch) |
                              uintptr_t(b_pitch)) % 16 == 0 &&
                             a_pitch <= 1 << 22 && b_pitch <= 1 << 22 && k <= 1 << 22;
        if (!aligned) {
            const dim3 grid(unsigned(ceil_div(m, 128) * ceil_div(n, 128)));
            const uint32_t tiles_n = uint32_t(ceil_div(n, 128));
            auto run = [&](auto kernel) { return launch(kLaunch, kernel, grid, 256, 0, s, g, tiles_n); };
            if (sum == kExact || sum == kWide) return run(matmul_kernel<kExact>);
            return run(sum == kScaled ? matmul_kernel<kScaled> : matmul_kernel<kFloat>);
        }
        if (p.parts > 1) {
            const int64_t need = int64_t(p.parts) * m * n * int64_t(sizeof(float));
            if (!workspace || workspace_bytes < need)
                return fail(RESHARD_EINVAL, "the product needs a workspace of " + std::to_string(need) +
                                                " bytes, got " + std::to_string(workspace ? workspace_bytes : 0));
            if (reinterpret_cast<uintptr_t>(workspace) % 16)
                return fail(RESHARD_EINVAL, "workspace is not aligned to 16 bytes");
            g.parts = static_cast<float *>(workspace);
        }
        const dim3 grid(unsigned(p.tiles_m * p.tiles_n), unsigned(p.parts));
        auto run = [&](auto kernel, unsigned threads) {
            return launch(kLaunch, kernel, grid, threads, 0, s, g, p.tiles_n, p.blocks);
        };
        if (sum == kWide && p.large) st = run(matmul_tile_kernel<kWide, 4, 2, 2, 4>, 512);
        else if (sum == kWide) st = run(matmul_tile_kernel<kWide, 2, 2, 2, 2>, 256);
        else if (sum == kExact) st = run(matmul_tile_kernel<kExact, 2, 2, 2, 2>, 256);
        else if (sum == kFloat && b_block_rows == kBlock) st = run(matmul_tile_kernel<kUniform, 2, 2, 2, 2>, 256);
        else if (sum == kFloat) st = run(matmul_tile_kernel<kFloat, 2, 2, 2, 2>, 256);
        else if (p.large) st = run(matmul_tile_kernel<kScaled, 4, 2, 2, 4>, 512);
        else st = run(matmul_tile_kernel<kScaled, 2, 2, 2, 2>, 256);
        if (st != RESHARD_OK || p.parts == 1) return st;
        const int64_t wgs = std::min<int64_t>(ceil_div(m * ceil_div(n, 8), 256), 4096);
        return launch("matmul join launch", matmul_join_kernel, dim3(unsigned(wgs)), 256, 0, s, g, p.parts);
    });
}
