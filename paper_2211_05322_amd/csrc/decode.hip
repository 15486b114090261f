// decode.hip -- attention of one new token of each sequence over a paged cache.
//
//   out = softmax(scale q k^T) v,  k and v the sequence's `length` slots
//
// Bound by memory: the cache is read once, and each of its elements is used by
// the few query heads that share it.  So the work is dealt by what is read: the
// tiles of 128 tokens of all sequences and key heads lie in one line, which the
// workgroups cut into equal runs, whatever the lengths.  A run may end inside
// a sequence; its part (weighted values, their sum, the maximum) then goes to
// the workspace, and a second kernel joins parts in their order.
#include <algorithm>

#include "attention.hpp"

namespace rs {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kWaveKeys = 32, kTileKeys = kWaves * kWaveKeys;  // a wave's and a workgroup's tokens of a tile
constexpr int kQueries = 16;                                   // heads of a group that one pass takes
constexpr float kLowest = -3.402823466e38f;

struct PagedArgs {
    Heads q, out;
    Cache cache;
    const int32_t *pages, *lengths;
    int64_t pages_pitch;
    int64_t *line;  // [sequences + 1]: tiles before each sequence, of one key head
    float *parts;   // [workgroups][2][group's rows up to 16][dim + 2]
    int sequences, width, kv_heads, group, passes, dim, rows;
    uint32_t magic, magic_shift;  // slot / page_length
    float scale2;
};

__device__ inline int64_t tiles_of(const PagedArgs &a, int s) {
    const int64_t most = int64_t(a.width) * a.cache.page_length;
    const int64_t n = min(int64_t(max(a.lengths[s], 0)), most);
    return (n + kTileKeys - 1) / kTileKeys;
}

// The number of tiles before each thread's share of the sequences, and of all.
__device__ inline int64_t scan(int64_t mine, int64_t *total, int64_t *part) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int64_t sum = mine;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int64_t other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    if (lane == kWave - 1) part[wave] = sum;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before += w < wave ? part[w] : 0;
        all += part[w];
    }
    *total = all;
    return before + sum - mine;
}

// A wave's keys are the instruction's rows and the group's queries its columns:
// a lane has 8 scores of one query, whose weights then go into the second
// product as they are.  Keys come straight into the operands' registers; values
// pass through LDS, where the transposing load finds their columns, in a part
// that is the wave's own.  The next tile's are on their way meanwhile.
template <typename T, int DP>
__global__ __launch_bounds__(kThreads, 2) void paged_kernel(PagedArgs a) {
    constexpr int STEPS = DP / 32, BLOCKS = DP / 16, WORDS = TileShape<DP>::words;
    constexpr int ROWS_AT_ONCE = kWave / WORDS, VALUES = kWaveKeys / ROWS_AT_ONCE;
    __shared__ uint4 values[kWaves][kWaveKeys * WORDS];
    __shared__ float maxima[kWaves][kQueries], sums[kWaves][kQueries];
    __shared__ int64_t part[kWaves], found[2];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, column = lane % 16, quarter = lane / 16;
    const int units = a.kv_heads * a.passes;

    // this workgroup's run of the line
    const int share = (a.sequences + kThreads - 1) / kThreads;
    const int from_s = min(int(threadIdx.x) * share, a.sequences), to_s = min(from_s + share, a.sequences);
    int64_t mine = 0, total;
    for (int s = from_s; s < to_s; ++s) mine += tiles_of(a, s);
    int64_t before = scan(mine, &total, part);
    const int64_t all = total * units, runs = min(all, int64_t(gridDim.x));
    if (blockIdx.x == 0) {  // for the joining kernel
        int64_t n = before;
        for (int s = from_s; s < to_s; ++s) {
            a.line[s] = n;
            n += tiles_of(a, s);
        }
        if (threadIdx.x == 0) a.line[a.sequences] = total;
    }
    if (blockIdx.x >= runs) return;
    const int64_t at = all * blockIdx.x / runs, end = all * (blockIdx.x + 1) / runs;
    if (mine > 0 && before * units <= at && at < (before + mine) * units) {
        int s = from_s;
        for (int64_t n; (before + (n = tiles_of(a, s))) * units <= at; ++s) before += n;
        found[0] = s;
        found[1] = before;
    }
    __syncthreads();
    int s = int(found[0]);
    int64_t line = found[1] * units, tiles = tiles_of(a, s);

    for (int64_t tile = at; tile < end;) {
        while (tile >= line + tiles * units) {
            line += tiles * units;
            tiles = tiles_of(a, ++s);
        }
        const int unit = int((tile - line) / tiles);
        const int64_t unit_at = line + unit * tiles;
        const int first = int(tile - unit_at), last = int(min(tiles, end - unit_at));  // of the unit's tiles
        const int head = unit / a.passes, pass = unit - head * a.passes;
        const int group0 = pass * kQueries, rows = min(kQueries, a.group - group0);
        const int length = int(min(int64_t(a.lengths[s]), int64_t(a.width) * a.cache.page_length));
        const int32_t *table = a.pages + s * a.pages_pitch;

        Operand8<T> q[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int d = i * 32 + quarter * 8;
            q[i].w = make_uint4(0, 0, 0, 0);
            if (column < rows && d < a.dim)
                q[i].w = load_any<uint4>(a.q.template at<const T>(s, int64_t(head) * a.group + group0 + column) + d);
        }
        // where a lane's token of a tile lies (-1: nowhere)
        auto page_of = [&](int t) {
            const int key = t * kTileKeys + wave * kWaveKeys + lane % kWaveKeys;
            if (t >= last || key >= length) return -1;
            return int(table[(__umulhi(a.magic, uint32_t(key)) + uint32_t(key)) >> a.magic_shift]);
        };
        auto offset_of = [&](int t, int page) -> int64_t {
            const int key = t * kTileKeys + wave * kWaveKeys + lane % kWaveKeys;
            if (t >= last || key >= length || page < 0 || page >= a.cache.pages) return -1;
            const uint32_t number = (__umulhi(a.magic, uint32_t(key)) + uint32_t(key)) >> a.magic_shift;
            return page * a.cache.page_pitch + (key - int(number) * a.cache.page_length) * a.cache.slot_pitch +
                   head * a.cache.head_pitch;
        };
        auto of_lane = [](int64_t x, int l) -> int64_t {
            const uint32_t lo = uint32_t(__shfl(int(x), l)), hi = uint32_t(__shfl(int(x >> 32), l));
            return int64_t(uint64_t(hi) << 32 | lo);
        };
        Operand8<T> k[2][STEPS];
        uint4 v[VALUES];
        const T *keys = static_cast<const T *>(a.cache.keys), *vals = static_cast<const T *>(a.cache.values);
        auto load_keys = [&](int64_t offset) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int64_t o = of_lane(offset, b * 16 + column);
#pragma unroll
                for (int i = 0; i < STEPS; ++i) {
                    const int d = i * 32 + quarter * 8;
                    k[b][i].w = make_uint4(0, 0, 0, 0);
                    if (o >= 0 && d < a.dim) k[b][i].w = load_any<uint4>(keys + o + d);
                }
            }
        };
        auto load_values = [&](int64_t offset) {
#pragma unroll
            for (int u = 0; u < VALUES; ++u) {
                const int64_t o = of_lane(offset, u * ROWS_AT_ONCE + lane / WORDS);
                const int d = lane % WORDS * 8;
                v[u] = make_uint4(0, 0, 0, 0);
                if (o >= 0 && d < a.dim) v[u] = load_any<uint4>(vals + o + d);
            }
        };

        f32x4 o[BLOCKS];
#pragma unroll
        for (int d = 0; d < BLOCKS; ++d) o[d] = f32x4{0, 0, 0, 0};
        float m = kLowest, l = 0;
        int64_t now = offset_of(first, page_of(first)), next = offset_of(first + 1, page_of(first + 1));
        load_keys(now);
        load_values(now);
        for (int t = first; t < last; ++t) {
            const int page = page_of(t + 2);
            f32x4 x[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                x[b] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < STEPS; ++i) x[b] = mfma(k[b][i], q[i], x[b]);
            }
            load_keys(next);
            const uint64_t there = __builtin_amdgcn_ballot_w64(now >= 0);  // bit j: token j of the wave's 32
            float top = kLowest;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (!(there >> (b * 16 + quarter * 4 + r) & 1)) x[b][r] = -INFINITY;
                    top = fmaxf(top, x[b][r] * a.scale2);
                }
            if (__builtin_amdgcn_ballot_w64(top > m + 8)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                top = fmaxf(top, m);
                const float shrink = __builtin_amdgcn_exp2f(m - top);
                m = top;
                l *= shrink;
#pragma unroll
                for (int d = 0; d < BLOCKS; ++d) o[d] *= shrink;
            }
            Operand8<T> p;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(x[b][r], a.scale2, -m));
                    l += e;
                    p.e[b * 4 + r] = T(e);
                }
#pragma unroll
            for (int u = 0; u < VALUES; ++u)
                values[wave][TileShape<DP>::at(u * ROWS_AT_ONCE + lane / WORDS, lane % WORDS)] = v[u];
            load_values(next);
            now = next;
            next = offset_of(t + 2, page);
            __builtin_amdgcn_wave_barrier();  // a wave's LDS accesses are done in their order
#pragma unroll
            for (int d = 0; d < BLOCKS; ++d) {
                typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                Operand8<T> vv;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int row = b * 16 + quarter * 4 + column / 4;
                    const char *from =
                        reinterpret_cast<const char *>(&values[wave][TileShape<DP>::at(row, d * 2 + column % 4 / 2)]);
                    vv.half[b] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(from + column % 2 * 8));
                }
                o[d] = mfma(vv, p, o[d]);
            }
            __builtin_amdgcn_wave_barrier();
        }
        // the waves' parts, one query a lane of 16 and 4 elements a block
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        __syncthreads();
        float *mine_o = reinterpret_cast<float *>(values[wave]);  // [queries][DP / 2 of it]: half the elements at a time
        if (quarter == 0) {
            maxima[wave][column] = m;
            sums[wave][column] = l;
        }
        const bool whole = first == 0 && last == tiles;
        float *to = a.parts + ((int64_t(blockIdx.x) * 2 + (first == 0)) * a.rows) * (a.dim + 2);
        constexpr int HALF = DP / 2;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            __syncthreads();
#pragma unroll
            for (int d = 0; d < BLOCKS / 2; ++d)
                *reinterpret_cast<f32x4 *>(mine_o + column * HALF + d * 16 + quarter * 4) = o[h * (BLOCKS / 2) + d];
            __syncthreads();
            for (int i = threadIdx.x; i < rows * HALF; i += kThreads) {
                const int r = i / HALF, d = i - r * HALF;
                float top = maxima[0][r];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) top = fmaxf(top, maxima[w][r]);
                float sum = 0, value = 0;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float f = __builtin_amdgcn_exp2f(maxima[w][r] - top);
                    sum = fmaf(f, sums[w][r], sum);
                    value = fmaf(f, reinterpret_cast<const float *>(values[w])[i], value);
                }
                if (h * HALF + d >= a.dim) continue;
                if (whole) {
                    a.out.template at<T>(s, int64_t(head) * a.group + group0 + r)[h * HALF + d] =
                        T(sum == 0 ? 0.0f : value / sum);
                } else {
                    float *row = to + r * (a.dim + 2);
                    row[h * HALF + d] = value;
                    if (h == 0 && d == 0) {
                        row[a.dim] = top;
                        row[a.dim + 1] = sum;
                    }
                }
            }
        }
        __syncthreads();
        tile = unit_at + last;
    }
}

// Joins the parts of each unit that more than one workgroup had, and writes the
// zeros of sequences without tokens.  A workgroup a sequence and key head and pass.
template <typename T>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(PagedArgs a, uint32_t workgroups) {
    const int units = a.kv_heads * a.passes, s = blockIdx.x / units, unit = blockIdx.x - s * units;
    const int head = unit / a.passes, group0 = (unit - head * a.passes) * kQueries, rows = min(kQueries, a.group - group0);
    const int64_t tiles = a.line[s + 1] - a.line[s], all = a.line[a.sequences] * units;
    const int64_t at = a.line[s] * units + unit * tiles;
    int64_t w0 = 0, w1 = -1;
    if (tiles > 0) {
        // the workgroup whose run holds tile x: the last w with all * w / runs <= x; no run is empty
        const int64_t runs = min(all, int64_t(workgroups));
        w0 = ((at + 1) * runs - 1) / all;
        w1 = ((at + tiles) * runs - 1) / all;
        if (w0 == w1) return;
    }
    const int stride = a.dim + 2;
    for (int i = threadIdx.x; i < rows * a.dim; i += kThreads) {
        const int r = i / a.dim, d = i - r * a.dim;
        float top = kLowest, sum = 0, value = 0;
        for (int64_t w = w0; w <= w1; ++w)
            top = fmaxf(top, a.parts[((w * 2 + (w == w0)) * a.rows + r) * stride + a.dim]);
        for (int64_t w = w0; w <= w1; ++w) {
            const float *row = a.parts + ((w * 2 + (w == w0)) * a.rows + r) * stride;
            const float f = __builtin_amdgcn_exp2f(row[a.dim] - top);
            sum = fmaf(f, row[a.dim + 1], sum);
            value = fmaf(f, row[d], value);
        }
        a.out.template at<T>(s, int64_t(head) * a.group + group0 + r)[d] = T(sum == 0 ? 0.0f : value / sum);
    }
}

// Two workgroups a CU, or one a tile where there are fewer.
int64_t workgroups_of(int64_t sequences, int64_t kv_heads, int64_t passes, int64_t slots) {
    const int64_t tiles = ceil_div(slots, kTileKeys), most = 512;
    if (tiles == 0) return 1;
    return std::max<int64_t>(1, tiles >= most ? most : std::min(most, sequences * kv_heads * passes * tiles));
}

}  // namespace
}  // namespace rs

extern "C" int64_t reshard_attention_paged_workspace(int64_t sequences, int64_t heads, int64_t kv_heads, int64_t dim,
                                                     int64_t pages_a_sequence, int64_t page_length) {
    using namespace rs;
    if (sequences < 0 || sequences > 0x7fffffff || heads < 1 || heads > kMaxHeads || kv_heads < 1 || heads % kv_heads ||
        dim < 1 || dim > kMaxDim || pages_a_sequence < 0 || page_length < 1 || page_length > 0x7fffffff ||
        pages_a_sequence > 0x7fffffff / page_length)
        return -1;
    const int64_t group = heads / kv_heads, passes = ceil_div(group, kQueries);
    const int64_t n = workgroups_of(sequences, kv_heads, passes, pages_a_sequence * page_length);
    return (sequences + 2) / 2 * 16 + n * 2 * std::min<int64_t>(group, kQueries) * (dim + 2) * 4;
}

extern "C" reshard_status_t reshard_attention_paged(int64_t sequences, int64_t heads, int64_t kv_heads, int64_t dim,
                                                    reshard_dtype_t dtype, const reshard_heads_t *q,
                                                    const reshard_cache_t *cache, const int32_t *pages,
                                                    int64_t pages_a_sequence, int64_t pages_pitch,
                                                    const int32_t *lengths, double scale, const reshard_heads_t *out,
                                                    void *workspace, int64_t workspace_bytes, void *stream) {
    return rs::guarded([&]() -> reshard_status_t {
        using namespace rs;
        reshard_status_t st = check_head_counts(heads, kv_heads);
        if (st != RESHARD_OK) return st;
        if (sequences < 0 || pages_a_sequence < 0)
            return fail(RESHARD_EINVAL, "sequences or pages_a_sequence is negative");
        if (heads % kv_heads) return fail(RESHARD_EINVAL, "heads must be a multiple of kv_heads");
        if (dim < 1) return fail(RESHARD_EINVAL, "dim must be >= 1");
        if (dim % 8 || dim > kMaxDim)
            return fail(RESHARD_EUNSUPPORTED, "dim must be a multiple of 8 up to " + std::to_string(kMaxDim));
        if (dtype != RESHARD_F16 && dtype != RESHARD_BF16) return fail(RESHARD_EINVAL, "dtype must be F16 or BF16");
        if (!(scale > 0 && scale < 1e30)) return fail(RESHARD_EINVAL, "scale must be positive and finite");
        if (!cache) return fail(RESHARD_EINVAL, "cache is NULL");
        PagedArgs a{};
        st = check_heads("q", q, sequences, heads, dim, 2, false, &a.q);
        if (st == RESHARD_OK) st = check_heads("out", out, sequences, heads, dim, 2, true, &a.out);
        if (st == RESHARD_OK) st = check_cache(cache, kv_heads, dim, 2, &a.cache);
        if (st == RESHARD_OK) st = check_matrix("pages", pages, sequences, pages_a_sequence, pages_pitch, 4);
        if (st == RESHARD_OK) st = check_matrix("lengths", lengths, 1, sequences, sequences, 4);
        if (st != RESHARD_OK) return st;
        const int64_t group = heads / kv_heads, passes = ceil_div(group, kQueries);
        if (pages_a_sequence > 0x7fffffff / cache->page_length || sequences * kv_heads * passes > int64_t(1) << 30)
            return fail(RESHARD_EUNSUPPORTED, "a sequence's pages hold 2^31 tokens or more, or above 2^30 sequences and heads");
        const int64_t need = reshard_attention_paged_workspace(sequences, heads, kv_heads, dim, pages_a_sequence,
                                                               cache->page_length);
        if (sequences == 0) return RESHARD_OK;
        st = check_workspace("the parts of long sequences need", workspace, workspace_bytes, need);
        if (st != RESHARD_OK) return st;
        a.pages = pages;
        a.lengths = lengths;
        a.pages_pitch = pages_pitch;
        a.line = static_cast<int64_t *>(workspace);
        a.parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + (sequences + 2) / 2 * 16);
        a.sequences = int(sequences);
        a.width = int(pages_a_sequence);
        a.kv_heads = int(kv_heads);
        a.group = int(group);
        a.passes = int(passes);
        a.dim = int(dim);
        a.rows = int(std::min<int64_t>(group, kQueries));
        // x / d = (hi(magic * x) + x) >> shift for x < 2^31, with 2^shift the first power of two not below d
        // (Granlund and Montgomery, 1994)
        const uint64_t d = uint64_t(cache->page_length);
        uint32_t shift = 0;
        while ((uint64_t(1) << shift) < d) ++shift;
        a.magic = uint32_t((uint64_t(1) << 32) * ((uint64_t(1) << shift) - d) / d + 1);
        a.magic_shift = shift;
        a.scale2 = float(scale) * kLog2e;
        const unsigned n = unsigned(workgroups_of(sequences, kv_heads, passes, pages_a_sequence * cache->page_length));
        const hipStream_t s = static_cast<hipStream_t>(stream);
        auto go = [&](auto zero) {
            using T = decltype(zero);
            auto *kernel = dim <= 32 ? paged_kernel<T, 32> : dim <= 64 ? paged_kernel<T, 64>
                                   : dim <= 96 ? paged_kernel<T, 96> : paged_kernel<T, 128>;
            reshard_status_t status = launch("paged attention launch", kernel, dim3(n), kThreads, 0, s, a);
            if (status != RESHARD_OK) return status;
            return launch("paged attention join launch", paged_join_kernel<T>,
                          dim3(unsigned(sequences * kv_heads * passes)), kThreads, 0, s, a, n);
        };
        return dtype == RESHARD_BF16 ? go(bf16{}) : go(f16{});
    });
}
