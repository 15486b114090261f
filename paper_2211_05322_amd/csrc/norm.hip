// norm.hip -- layer norm of rows and its gradients.
//
//   mean = sum_c x / C      rstd = 1 / sqrt(sum_c (x - mean)^2 / C + eps)
//   xhat = (x - mean) rstd  y = xhat w + b
//   g = dy w                dx = rstd (g - mean_c(g) - xhat mean_c(g xhat))
//   dw = sum_r dy xhat      db = sum_r dy
//
// Both are bound by memory: the forward pass reads and writes each element
// once, the backward pass reads two and writes one.  A row's elements stay in
// registers between the reductions and the result, so the second moment is
// taken about the mean (no cancellation) without a second read.
#include <algorithm>
#include <type_traits>

#include "operators.hpp"

namespace rs {
namespace {

// Sum of N values over the THREADS threads that share a row: a wave by
// shuffles; more waves through `part`, which every call site owns a part of.
template <int THREADS, int N>
__device__ inline void row_sum(float (&v)[N], float *part) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (THREADS > kWave) {
        constexpr int W = THREADS / kWave;
        const int wave = threadIdx.x / kWave;
        if (threadIdx.x % kWave == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) part[i * W + wave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) s += part[i * W + w];
            v[i] = s;
        }
    }
}

// A thread's columns of a row: NV vectors, the k-th the (k * THREADS + t)-th
// of the row.  NV is the fewest that cover the row, so only the last can pass
// the row's end; it is moved back to end there, and its first `skip` elements
// are another vector's.  Both compute the same values for those.
template <typename T, int THREADS, int NV>
struct Columns {
    static constexpr int V = kVec<T>;
    int64_t last;
    int first, skip;

    __device__ Columns(int64_t cols, int t) {
        const int64_t c = int64_t((NV - 1) * THREADS + t) * V;
        last = min(c, cols - V);
        skip = int(min(c - last, int64_t(V)));
        first = t * V;
    }
    __device__ int64_t at(int k) const { return k == NV - 1 ? last : int64_t(k) * (THREADS * V) + first; }
    __device__ bool mine(int k, int i) const { return k < NV - 1 || i >= skip; }
    __device__ bool any(int k) const { return k < NV - 1 || skip < V; }
};

// Between a reduction and the next use of a row: elements are converted again
// there.  Without it the compiler keeps both forms of them in registers
// across the barrier, and spills.
template <typename T, int NV>
__device__ inline void packed(Pack<T> (&p)[NV]) {
#pragma unroll
    for (int k = 0; k < NV; ++k) asm("" : "+v"(p[k].v.x), "+v"(p[k].v.y), "+v"(p[k].v.z), "+v"(p[k].v.w));
}

struct NormArgs {
    const void *x, *weight, *bias;
    void *y;
    float *mean, *rstd;
    int64_t rows, cols, x_pitch, y_pitch;
    float eps;
    int weight_dtype;
    bool past_cache;  // y is larger than the last-level cache
};

// THREADS threads hold a row, 256 / THREADS rows a workgroup where a wave
// holds one.  A workgroup keeps its columns' weights in registers over the
// rows that it takes in turn (read for every row they were three times the
// row's bytes, from L2), and loads each row while the one before is reduced.
// Bound by memory: 16384 x 12288 bf16 in 153 us, 5.2 TB/s; 8192 x 4096 fp16 in
// 24 us.
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_kernel(NormArgs a) {
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
    constexpr int V = kVec<T>;
    constexpr bool AHEAD = THREADS * NV < 4096;  // registers for two rows
    __shared__ float part[2][THREADS / kWave];
    const int t = threadIdx.x % THREADS;
    const Columns<T, THREADS, NV> my(a.cols, t);
    const float cols = float(a.cols);
    const int64_t stride = int64_t(gridDim.x) * ROWS;
    int64_t row = int64_t(blockIdx.x) * ROWS + threadIdx.x / THREADS;
    Pack<T> next[NV];
    auto load = [&](int64_t r) {
        const T *x = static_cast<const T *>(a.x) + min(r, a.rows - 1) * a.x_pitch;
#pragma unroll
        for (int k = 0; k < NV; ++k) next[k].v = load_any<uint4>(x + my.at(k));
    };
    if (AHEAD) load(row);  // before the weights, which few rows would wait for too
    float w[NV][V], b[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_as_float<V>(a.weight, a.weight_dtype, my.at(k), a.cols, 1.0f, w[k]);
        load_as_float<V>(a.bias, a.weight_dtype, my.at(k), a.cols, 0.0f, b[k]);
    }
    for (; row < a.rows; row += stride) {
        if (!AHEAD) load(row);
        Pack<T> p[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) p[k] = next[k];
        if (AHEAD) load(row + stride);
        float s[1] = {0}, q[1] = {0};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += my.mine(k, i) ? float(p[k].e[i]) : 0.0f;
        row_sum<THREADS>(s, part[0]);
        packed(p);
        const float mean = s[0] / cols;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = float(p[k].e[i]) - mean;
                q[0] += my.mine(k, i) ? d * d : 0.0f;
            }
        row_sum<THREADS>(q, part[1]);
        packed(p);
        const float rstd = 1.0f / sqrtf(q[0] / cols + a.eps);
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        T *y = static_cast<T *>(a.y) + row * a.y_pitch;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            Pack<T> r;
#pragma unroll
            for (int i = 0; i < V; ++i) r.e[i] = T((float(p[k].e[i]) - mean) * rstd * w[k][i] + b[k][i]);
            if (!my.any(k)) continue;
            if (a.past_cache) store_past(y + my.at(k), r.v);
            else store_any(y + my.at(k), r.v);
        }
    }
}

// Rows too long for registers, or shorter than one vector: read once for each
// moment and once for the result, the second and third time mostly from L2.
// 4096 x 33000 bf16 in 176 us, 3.1 TB/s of its input and output.
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float part[2][1024 / kWave];
    const float cols = float(a.cols);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_pitch;
        T *y = static_cast<T *>(a.y) + row * a.y_pitch;
        float s[1] = {0}, q[1] = {0};
        for (int64_t c = int64_t(threadIdx.x) * V; c < a.cols; c += 1024 * V) {
            const Pack<T> p = load_pack(x + c, a.cols - c);
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += float(p.e[i]);
        }
        row_sum<1024>(s, part[0]);
        const float mean = s[0] / cols;
        for (int64_t c = int64_t(threadIdx.x) * V; c < a.cols; c += 1024 * V) {
            const Pack<T> p = load_pack(x + c, a.cols - c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = float(p.e[i]) - mean;
                q[0] += c + i < a.cols ? d * d : 0.0f;
            }
        }
        row_sum<1024>(q, part[1]);
        const float rstd = 1.0f / sqrtf(q[0] / cols + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (int64_t c = int64_t(threadIdx.x) * V; c < a.cols; c += 1024 * V) {
            const Pack<T> p = load_pack(x + c, a.cols - c);
            float w[V], b[V];
            load_as_float<V>(a.weight, a.weight_dtype, c, a.cols, 1.0f, w);
            load_as_float<V>(a.bias, a.weight_dtype, c, a.cols, 0.0f, b);
            Pack<T> r;
#pragma unroll
            for (int i = 0; i < V; ++i) r.e[i] = T((float(p.e[i]) - mean) * rstd * w[i] + b[i]);
            store_pack(y + c, r, a.cols - c);
        }
    }
}

struct NormGradArgs {
    const void *dy, *x, *weight;
    const float *mean, *rstd;
    void *dx;
    float *partial;  // [workgroups][2][cols]: sums of dy xhat, then of dy, over a workgroup's rows
    int64_t rows, cols, dy_pitch, x_pitch, dx_pitch;
    int weight_dtype;
};

// Each group of THREADS threads takes every groups-th row and keeps its
// columns' sums in registers over all of them, loading each row while the one
// before is reduced; no atomics, so the gradients of the weights are the same
// in every run.  The weights, as float32, lie in LDS: with them the registers
// would not hold two rows and the sums.  Bound by memory where rows are long
// (16384 x 12288 bf16 in 245 us, 4.9 TB/s; 16376 x 12300, off 16-byte boundaries,
// in 262), by the 20 operations an element at two waves a SIMD where they are
// shorter (8192 x 4096 fp16 in 50 us, 4.1 TB/s), by 22 spilled registers in float32
// rows over 12288 (8192 x 16384 in 378 us, 4.3 TB/s; 8192 x 12288 in 229, 5.3).
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_grad_kernel(NormGradArgs a) {
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
    constexpr int V = kVec<T>;
    constexpr bool AHEAD = THREADS < 1024;
    __shared__ float part[2][2 * (THREADS / kWave)];
    extern __shared__ float weights[];  // cols, a whole number of vectors
    const int t = threadIdx.x % THREADS;
    const Columns<T, THREADS, NV> my(a.cols, t);
    const int64_t group = int64_t(blockIdx.x) * ROWS + threadIdx.x / THREADS;
    const int64_t groups = int64_t(gridDim.x) * ROWS;
    const float cols = float(a.cols);
    float dw[NV][V], db[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = 0;
    Pack<T> next_x[NV], next_g[NV];
    float next_mean, next_rstd;
    auto load = [&](int64_t r) {
        r = min(r, a.rows - 1);
        const T *x = static_cast<const T *>(a.x) + r * a.x_pitch, *dy = static_cast<const T *>(a.dy) + r * a.dy_pitch;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            next_x[k].v = load_any<uint4>(x + my.at(k));
            next_g[k].v = load_any<uint4>(dy + my.at(k));
        }
        next_mean = a.mean[r];
        next_rstd = a.rstd[r];
    };
    if (AHEAD) load(group);
    for (int64_t c = threadIdx.x * V; c < a.cols; c += blockDim.x * V) {
        float w[V];
        load_as_float<V>(a.weight, a.weight_dtype, c, a.cols, 1.0f, w);
#pragma unroll
        for (int i = 0; i < V; ++i) weights[c + i] = w[i];
    }
    __syncthreads();
    int turn = 0;  // rows in turn use the two halves of `part`: one barrier a row
    for (int64_t row = group; row < a.rows; row += groups, turn ^= 1) {
        if (!AHEAD) load(row);
        Pack<T> px[NV], pg[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            px[k] = next_x[k];
            pg[k] = next_g[k];
        }
        const float mean = next_mean, rstd = next_rstd;
        // xhat; x * rstd - mean * rstd would save an operation and lose digits where x is near the mean
        auto normal = [&](T x) { return (float(x) - mean) * rstd; };
        if (AHEAD) load(row + groups);
        float s[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const float *w = weights + my.at(k);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = float(pg[k].e[i]), h = normal(px[k].e[i]);
                const float g = my.mine(k, i) ? d * w[i] : 0.0f;
                dw[k][i] = fmaf(d, h, dw[k][i]);
                db[k][i] += d;
                s[0] += g;
                s[1] = fmaf(g, h, s[1]);
            }
        }
        row_sum<THREADS>(s, part[turn]);
        packed(px);
        packed(pg);
        if (a.dx) {
            const float c0 = -rstd * (s[0] / cols), c1 = -rstd * (s[1] / cols);
            T *dx = static_cast<T *>(a.dx) + row * a.dx_pitch;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const float *w = weights + my.at(k);
                Pack<T> r;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    r.e[i] = T(fmaf(normal(px[k].e[i]), c1, fmaf(float(pg[k].e[i]) * w[i], rstd, c0)));
                if (my.any(k)) store_any(dx + my.at(k), r.v);
            }
        }
    }
    if (!a.partial) return;
    float *out = a.partial + int64_t(blockIdx.x) * 2 * a.cols;
    if constexpr (ROWS > 1) {  // the waves of a workgroup add up in LDS, one after the other
        float *sums = weights + ceil_div(a.cols, V) * V;
        for (int r = 0; r < ROWS; ++r) {
            __syncthreads();
            if (threadIdx.x / THREADS != r) continue;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (!my.mine(k, i)) continue;
                    float *w = sums + my.at(k) + i, *b = w + a.cols;
                    *w = r ? *w + dw[k][i] : dw[k][i];
                    *b = r ? *b + db[k][i] : db[k][i];
                }
        }
        __syncthreads();
        for (int64_t c = threadIdx.x; c < 2 * a.cols; c += blockDim.x) out[c] = sums[c];
        return;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (my.any(k)) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {  // elements that are another's have the same sums
                store_any(out + my.at(k) + i, make_float4(dw[k][i], dw[k][i + 1], dw[k][i + 2], dw[k][i + 3]));
                store_any(out + a.cols + my.at(k) + i, make_float4(db[k][i], db[k][i + 1], db[k][i + 2], db[k][i + 3]));
            }
        }
    }
}

// Rows too long for registers, or shorter than one vector: dx, reading the
// row twice (with the columns' sums, a third time: 4096 x 33000 bf16 in 386 us).
template <typename T>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormGradArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float part[2][2 * (1024 / kWave)];
    const float cols = float(a.cols);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_pitch;
        const T *dy = static_cast<const T *>(a.dy) + row * a.dy_pitch;
        T *dx = static_cast<T *>(a.dx) + row * a.dx_pitch;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s[2] = {0, 0};
        for (int64_t c = int64_t(threadIdx.x) * V; c < a.cols; c += 1024 * V) {
            const Pack<T> px = load_pack(x + c, a.cols - c), pg = load_pack(dy + c, a.cols - c);
            float w[V];
            load_as_float<V>(a.weight, a.weight_dtype, c, a.cols, 1.0f, w);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float g = float(pg.e[i]) * w[i];
                s[0] += g;
                s[1] += g * ((float(px.e[i]) - mean) * rstd);
            }
        }
        row_sum<1024>(s, part[turn]);
        const float c0 = s[0] / cols, c1 = s[1] / cols;
        for (int64_t c = int64_t(threadIdx.x) * V; c < a.cols; c += 1024 * V) {
            const Pack<T> px = load_pack(x + c, a.cols - c), pg = load_pack(dy + c, a.cols - c);
            float w[V];
            load_as_float<V>(a.weight, a.weight_dtype, c, a.cols, 1.0f, w);
            Pack<T> r;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float h = (float(px.e[i]) - mean) * rstd;
                r.e[i] = T(rstd * (float(pg.e[i]) * w[i] - c0 - h * c1));
            }
            store_pack(dx + c, r, a.cols - c);
        }
    }
}

// The columns' sums for such rows: a thread holds one vector's columns over
// the rows of its group.
template <typename T>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormGradArgs a) {
    constexpr int V = kVec<T>;
    const int64_t c = (int64_t(blockIdx.x) * 256 + threadIdx.x) * V;
    if (c >= a.cols) return;
    float dw[V], db[V];
#pragma unroll
    for (int i = 0; i < V; ++i) dw[i] = db[i] = 0;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const Pack<T> px = load_pack(static_cast<const T *>(a.x) + row * a.x_pitch + c, a.cols - c);
        const Pack<T> pg = load_pack(static_cast<const T *>(a.dy) + row * a.dy_pitch + c, a.cols - c);
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = float(pg.e[i]);
            dw[i] += d * ((float(px.e[i]) - mean) * rstd);
            db[i] += d;
        }
    }
    float *out = a.partial + int64_t(blockIdx.y) * 2 * a.cols + c;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (c + i < a.cols) {
            out[i] = dw[i];
            out[a.cols + i] = db[i];
        }
    }
}

// Joins the workgroups' sums: 64 columns a workgroup, the parts dealt to its 16
// waves, whose sums are then added in a fixed order.  256 parts of 12300 columns
// in 6 us, mostly from the last-level cache; of 1024 in 3 us, the launch.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float *partial, int64_t groups, int64_t cols, float *dw,
                                                         float *db, int accumulate) {
    __shared__ float part[16][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t j = int64_t(blockIdx.x) * kWave + lane;
    float s = 0;
    if (j < 2 * cols) {
#pragma unroll 8
        for (int64_t g = wave; g < groups; g += 16) s += partial[g * 2 * cols + j];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && j < 2 * cols) {
        s = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) s += part[w][lane];
        float *out = j < cols ? dw : db;
        const int64_t c = j < cols ? j : j - cols;
        if (out) out[c] = accumulate ? out[c] + s : s;
    }
}

constexpr int64_t kMaxGrid = int64_t(1) << 21;  // workgroups; rows beyond are taken in turn

reshard_status_t check_norm(int64_t rows, int64_t cols, reshard_dtype_t dtype, reshard_dtype_t weight_dtype,
                            bool weights) {
    reshard_status_t st = check_extent("rows", rows);
    if (st == RESHARD_OK) st = check_extent("cols", cols);
    if (st != RESHARD_OK) return st;
    if (cols == 0) return fail(RESHARD_EINVAL, "cols must be >= 1: a row without elements has no mean");
    if (cols > int64_t(1) << 24) return fail(RESHARD_EUNSUPPORTED, "cols is above 2^24");
    if (!is_float_type(dtype)) return fail(RESHARD_EINVAL, "dtype must be F16, BF16 or F32");
    if (weights && !is_float_type(weight_dtype))
        return fail(RESHARD_EINVAL, "weight_dtype must be F16, BF16 or F32");
    return RESHARD_OK;
}

// Calls f(THREADS, NV), as constants, for rows of nv vectors; false where no
// registers hold such rows.  A wave a row up to 2 vectors a lane; then as many
// waves as keep a thread at `each` vectors at most.
template <int V, int EACH, int MOST, typename F>
bool with_columns(int64_t cols, F &&f) {
    const int64_t nv = ceil_div(cols, V);
    if (cols < V || nv > MOST) return false;
    bool done = false;
    auto offer = [&](auto threads, auto n) {
        constexpr int THREADS = decltype(threads)::value, NV = decltype(n)::value;
        // 1024 threads only for rows that 512 do not hold
        if constexpr (THREADS * NV <= MOST && NV <= (THREADS == 512 ? EACH : 4) &&
                      (THREADS < 1024 || THREADS * NV > 512 * EACH)) {
            if (!done && nv <= THREADS * NV) {
                f(threads, n);
                done = true;
            }
        }
    };
    using std::integral_constant;
    constexpr integral_constant<int, 1> n1{};
    constexpr integral_constant<int, 2> n2{};
    constexpr integral_constant<int, 3> n3{};
    constexpr integral_constant<int, 4> n4{};
    offer(integral_constant<int, 64>{}, n1);
    offer(integral_constant<int, 64>{}, n2);
    offer(integral_constant<int, 256>{}, n1);
    offer(integral_constant<int, 256>{}, n2);
    offer(integral_constant<int, 256>{}, n3);
    offer(integral_constant<int, 512>{}, n2);
    offer(integral_constant<int, 512>{}, n3);
    offer(integral_constant<int, 512>{}, n4);
    offer(integral_constant<int, 1024>{}, n2);
    offer(integral_constant<int, 1024>{}, n3);
    offer(integral_constant<int, 1024>{}, n4);
    return done;
}

template <typename T>
reshard_status_t launch_norm(const NormArgs &a, hipStream_t s) {
    reshard_status_t st = RESHARD_OK;
    const bool done = with_columns<kVec<T>, 3, 4096>(a.cols, [&](auto threads, auto n) {
        constexpr int THREADS = decltype(threads)::value, ROWS = THREADS < 256 ? 256 / THREADS : 1;
        const int64_t most = 256 * 2048 / (THREADS < 256 ? 256 : THREADS);  // what the CUs hold at once
        const dim3 grid(unsigned(std::min(ceil_div(a.rows, ROWS), most)));
        st = launch("layer norm launch", norm_kernel<T, THREADS, decltype(n)::value>, grid,
                    THREADS < 256 ? 256 : THREADS, 0, s, a);
    });
    if (done) return st;
    return launch("layer norm launch", norm_long_kernel<T>, dim3(unsigned(std::min(a.rows, kMaxGrid))), 1024, 0, s, a);
}

// Workgroups of the backward pass, whose column sums are kept apart until the
// join: two a CU; one where a row takes 512 threads, of which a CU holds one
// workgroup (8192 x 8192 bf16: 97 us against 103), or rows are few and the sums
// weigh more (1024 x 4096: 19 against 22; but 8192 x 4096: 62 against 51).
int64_t norm_groups(int64_t rows, int64_t cols) {
    return std::min<int64_t>(rows, cols > 6144 || rows < 4096 ? 256 : 512);
}

template <typename T>
reshard_status_t launch_norm_grad(const NormGradArgs &a, int64_t groups, hipStream_t s) {
    const char *what = "layer norm gradient launch";
    reshard_status_t st = RESHARD_OK;
    // 16384 columns: the sums of more do not fit
    const bool done = with_columns<kVec<T>, 4, 16384 / kVec<T>>(a.cols, [&](auto threads, auto n) {
        constexpr int THREADS = decltype(threads)::value, ROWS = THREADS < 256 ? 256 / THREADS : 1;
        const dim3 grid{unsigned(groups)};
        const size_t padded = size_t(ceil_div(a.cols, kVec<T>)) * kVec<T>;
        const size_t lds = (padded + (ROWS > 1 ? 2 * a.cols : 0)) * sizeof(float);
        st = launch(what, norm_grad_kernel<T, THREADS, decltype(n)::value>, grid, THREADS < 256 ? 256 : THREADS, lds, s, a);
    });
    if (done) return st;
    // the sums first: dx may take dy's place
    if (a.partial)
        st = launch(what, norm_columns_kernel<T>,
                    dim3(unsigned(ceil_div(ceil_div(a.cols, kVec<T>), 256)), unsigned(groups)), 256, 0, s, a);
    if (st != RESHARD_OK || !a.dx) return st;
    return launch(what, norm_grad_long_kernel<T>, dim3(unsigned(std::min(a.rows, kMaxGrid))), 1024, 0, s, a);
}

}  // namespace
}  // namespace rs

using rs::fail;

extern "C" reshard_status_t reshard_layer_norm(int64_t rows, int64_t cols, const void *x, int64_t x_pitch,
                                               reshard_dtype_t dtype, const void *weight, const void *bias,
                                               reshard_dtype_t weight_dtype, double eps, void *y, int64_t y_pitch,
                                               float *mean, float *rstd, void *stream) {
    return rs::guarded([&]() -> reshard_status_t {
        using namespace rs;
        reshard_status_t st = check_norm(rows, cols, dtype, weight_dtype, weight || bias);
        const int64_t es = dtype == RESHARD_F32 ? 4 : 2, ws = weight_dtype == RESHARD_F32 ? 4 : 2;
        if (st == RESHARD_OK && !(eps >= 0)) st = fail(RESHARD_EINVAL, "eps must be >= 0");
        if (st == RESHARD_OK) st = check_matrix("x", x, rows, cols, x_pitch, es);
        if (st == RESHARD_OK) st = check_matrix("y", y, rows, cols, y_pitch, es);
        if (st == RESHARD_OK && weight) st = check_matrix("weight", weight, 1, cols, cols, ws);
        if (st == RESHARD_OK && bias) st = check_matrix("bias", bias, 1, cols, cols, ws);
        if (st == RESHARD_OK && mean) st = check_matrix("mean", mean, 1, rows, rows, 4);
        if (st == RESHARD_OK && rstd) st = check_matrix("rstd", rstd, 1, rows, rows, 4);
        if (st != RESHARD_OK || rows == 0) return st;
        const NormArgs a{x, weight, bias, y, mean, rstd, rows, cols, x_pitch, y_pitch, float(eps), int(weight_dtype),
                         rows * cols * es >= int64_t(256) << 20};
        const hipStream_t s = static_cast<hipStream_t>(stream);
        if (dtype == RESHARD_F32) return launch_norm<float>(a, s);
        return dtype == RESHARD_BF16 ? launch_norm<bf16>(a, s) : launch_norm<f16>(a, s);
    });
}

extern "C" int64_t reshard_layer_norm_backward_workspace(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1 || cols > int64_t(1) << 24) return -1;
    return rs::norm_groups(rows, cols) * 2 * cols * int64_t(sizeof(float));
}

extern "C" reshard_status_t reshard_layer_norm_backward(int64_t rows, int64_t cols, const void *dy, int64_t dy_pitch,
                                                        const void *x, int64_t x_pitch, reshard_dtype_t dtype,
                                                        const void *weight, reshard_dtype_t weight_dtype,
                                                        const float *mean, const float *rstd, void *dx,
                                                        int64_t dx_pitch, float *dweight, float *dbias, int accumulate,
                                                        void *workspace, int64_t workspace_bytes, void *stream) {
    return rs::guarded([&]() -> reshard_status_t {
        using namespace rs;
        reshard_status_t st = check_norm(rows, cols, dtype, weight_dtype, weight != nullptr);
        const int64_t es = dtype == RESHARD_F32 ? 4 : 2, ws = weight_dtype == RESHARD_F32 ? 4 : 2;
        if (st == RESHARD_OK) st = check_matrix("dy", dy, rows, cols, dy_pitch, es);
        if (st == RESHARD_OK) st = check_matrix("x", x, rows, cols, x_pitch, es);
        if (st == RESHARD_OK && weight) st = check_matrix("weight", weight, 1, cols, cols, ws);
        if (st == RESHARD_OK) st = check_matrix("mean", mean, 1, rows, rows, 4);
        if (st == RESHARD_OK) st = check_matrix("rstd", rstd, 1, rows, rows, 4);
        if (st == RESHARD_OK && dx) st = check_matrix("dx", dx, rows, cols, dx_pitch, es);
        if (st == RESHARD_OK && dweight) st = check_matrix("dweight", dweight, 1, cols, cols, 4);
        if (st == RESHARD_OK && dbias) st = check_matrix("dbias", dbias, 1, cols, cols, 4);
        if (st == RESHARD_OK && (accumulate & ~1)) st = fail(RESHARD_EINVAL, "accumulate must be 0 or 1");
        if (st != RESHARD_OK) return st;
        const bool sums = dweight || dbias;
        const int64_t need = reshard_layer_norm_backward_workspace(rows, cols);
        if (sums && rows > 0) {
            if (!workspace || workspace_bytes < need)
                return fail(RESHARD_EINVAL, "the gradients of the weights need a workspace of " +
                                                std::to_string(need) + " bytes, got " +
                                                std::to_string(workspace ? workspace_bytes : 0));
            if (reinterpret_cast<uintptr_t>(workspace) % 16)
                return fail(RESHARD_EINVAL, "workspace is not aligned to 16 bytes");
        }
        const hipStream_t s = static_cast<hipStream_t>(stream);
        const int64_t groups = norm_groups(rows, cols);
        if (rows > 0 && (dx || sums)) {
            const NormGradArgs a{dy,   x,    weight,   mean,    rstd,     dx, sums ? static_cast<float *>(workspace) : nullptr,
                                 rows, cols, dy_pitch, x_pitch, dx_pitch, int(weight_dtype)};
            if (dtype == RESHARD_F32) st = launch_norm_grad<float>(a, groups, s);
            else st = dtype == RESHARD_BF16 ? launch_norm_grad<bf16>(a, groups, s) : launch_norm_grad<f16>(a, groups, s);
            if (st != RESHARD_OK) return st;
        }
        if (!sums || (rows == 0 && accumulate)) return RESHARD_OK;
        // no rows: the sums are zeros (0 groups to join)
        return launch("layer norm gradient join launch", norm_join_kernel, dim3(unsigned(ceil_div(2 * cols, kWave))), 1024,
                      0, s, static_cast<const float *>(workspace), groups, cols, dweight, dbias, accumulate);
    });
}
