// operators.hpp -- what the kernels at a stage's edge (norm.hip,
// quantize.hip, matmul.hip) share: element types, vectors that may start at
// any element, reductions, argument checks and launch errors.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>
#include <tuple>
#include <type_traits>

#include "../../include/reshard.h"
#include "status.hpp"

namespace rs {

constexpr int kWave = 64;
constexpr int kBlock = 128;  // elements that share one scale

using bf16 = __bf16;
using f16 = _Float16;

// 16 or 8 bytes at an address of any element's alignment: global memory takes
// such accesses in one instruction, so rows of any pitch need no second path.
template <typename V>
__device__ inline V load_any(const void *p) {
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}

template <typename V>
__device__ inline void store_any(void *p, V v) {
    __builtin_memcpy(p, &v, sizeof(V));
}

// A store that is not kept in the caches: for outputs that they could not hold
// until their reader comes.
__device__ inline void store_past(void *p, uint4 v) {
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2), may_alias));
    __builtin_nontemporal_store(words{v.x, v.y, v.z, v.w}, static_cast<words *>(p));
}

template <typename T>
constexpr int kVec = 16 / int(sizeof(T));  // elements of one 16-byte vector

template <typename T>
union Pack {
    uint4 v;
    T e[kVec<T>];
};

// Up to kVec<T> elements from p, zeros past the n that exist.
template <typename T>
__device__ inline Pack<T> load_pack(const T *p, int64_t n) {
    Pack<T> r;
    if (n >= kVec<T>) {
        r.v = load_any<uint4>(p);
        return r;
    }
    r.v = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
        if (i < n) r.e[i] = p[i];
    return r;
}

template <typename T>
__device__ inline void store_pack(T *p, const Pack<T> &x, int64_t n) {
    if (n >= kVec<T>) {
        store_any(p, x.v);
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
        if (i < n) p[i] = x.e[i];
}

// N elements of a run-time type from column c on as float32; `fill` past the
// end or without an array.  The branch is the same for every lane.
template <int N>
__device__ inline void load_as_float(const void *base, int dtype, int64_t c, int64_t cols, float fill, float *out) {
    if (!base) {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = fill;
    } else if (dtype == RESHARD_F32) {
        const float *p = static_cast<const float *>(base) + c;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const Pack<float> x = load_pack(p + i, cols - c - i);
#pragma unroll
            for (int j = 0; j < 4; ++j) out[i + j] = x.e[j];
        }
    } else if (dtype == RESHARD_BF16) {
        const bf16 *p = static_cast<const bf16 *>(base) + c;
        const Pack<bf16> x = load_pack(p, cols - c);
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = float(x.e[i]);
    } else {
        const f16 *p = static_cast<const f16 *>(base) + c;
        const Pack<f16> x = load_pack(p, cols - c);
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = float(x.e[i]);
    }
}

// The wave's sum, in every lane.  Within rows of 16 lanes and then from row to
// row by data-parallel moves, which cost an addition each; shuffles go through
// LDS and would be most of a short row's time.
__device__ inline float wave_sum(float x) {
    auto moved = [&](auto ctrl, auto rows) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value,
                                                          decltype(rows)::value, 0xf, true));
    };
    using std::integral_constant;
    constexpr integral_constant<int, 0xf> all{};
    x += moved(integral_constant<int, 0x111>{}, all);  // right by 1, 2, 4 and 8: lane 15 has its row's sum
    x += moved(integral_constant<int, 0x112>{}, all);
    x += moved(integral_constant<int, 0x114>{}, all);
    x += moved(integral_constant<int, 0x118>{}, all);
    x += moved(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});  // lane 15 to the next row
    x += moved(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});  // lane 31 to rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), kWave - 1));
}

// A descriptor for `bytes` bytes from p, the same in every lane.  Loads from an
// offset past the end give zeros.
__device__ inline __amdgpu_buffer_rsrc_t bytes_from(const void *p, int64_t bytes) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    const uint64_t lo = uint32_t(__builtin_amdgcn_readfirstlane(int(a)));
    const uint64_t hi = uint32_t(__builtin_amdgcn_readfirstlane(int(a >> 32)));
    const int n = __builtin_amdgcn_readfirstlane(int(bytes < 0xffffffff ? uint32_t(bytes) : 0xffffffffu));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(hi << 32 | lo), 0, n, 0x00020000);
}

// 16 bytes of a lane's straight into LDS, from `base` + its offset; lane l's
// go to `to` + 16 l, `to` being the wave's.  The whole offset is the lane's:
// the instruction's scalar offset is subtracted from the descriptor's size in
// the range check, which past a matrix's last rows would be below zero.
__device__ inline void load_to_lds(__amdgpu_buffer_rsrc_t base, uint32_t offset, uint4 *to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(base, (__attribute__((address_space(3))) void *)to, 16, offset, 0, 0, 0);
}

// Before a barrier behind which other waves read what this one loaded into
// LDS: the barrier itself waits for LDS accesses, not for such loads.
__device__ inline void loads_done() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt(0)

__device__ inline float e8m0_value(uint8_t code) {
    // 2^(code - 127); code 0 is 2^-127, a subnormal, and 255 NaN
    return code == 255 ? __builtin_nanf("") : code ? __uint_as_float(uint32_t(code) << 23) : __uint_as_float(0x400000u);
}

inline bool is_float_type(reshard_dtype_t t) { return t == RESHARD_F16 || t == RESHARD_BF16 || t == RESHARD_F32; }

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// One operand of an operator: `rows` rows of `cols` elements, `pitch`
// elements from one row to the next.
inline reshard_status_t check_matrix(const char *name, const void *p, int64_t rows, int64_t cols, int64_t pitch,
                                     int64_t elem_bytes) {
    if (rows > 0 && cols > 0 && !p) return fail(RESHARD_EINVAL, std::string(name) + " is NULL");
    if (rows > 1 && pitch < cols)
        return fail(RESHARD_EINVAL, std::string(name) + ": a pitch of " + std::to_string(pitch) +
                                        " is less than the row's " + std::to_string(cols) + " elements");
    if (pitch < 0 || (rows > 0 && pitch > (int64_t(1) << 56) / (rows * elem_bytes)))
        return fail(RESHARD_EUNSUPPORTED, std::string(name) + " spans more than 2^56 bytes");
    if (reinterpret_cast<uintptr_t>(p) % uintptr_t(elem_bytes))
        return fail(RESHARD_EINVAL, std::string(name) + " is not aligned to its " + std::to_string(elem_bytes) +
                                        "-byte elements");
    return RESHARD_OK;
}

inline reshard_status_t check_extent(const char *name, int64_t n) {
    if (n < 0) return fail(RESHARD_EINVAL, std::string(name) + " is negative");
    if (n > int64_t(1) << 40) return fail(RESHARD_EUNSUPPORTED, std::string(name) + " is above 2^40");
    return RESHARD_OK;
}

// Launches a kernel and reports that launch's error alone: the thread's last
// error, which <<<>>> leaves to be asked for, may be another call's.
template <typename... P, typename... A>
reshard_status_t launch(const char *what, void (*kernel)(P...), dim3 grid, unsigned threads, size_t lds, hipStream_t s,
                        const A &...a) {
    std::tuple<P...> args(static_cast<P>(a)...);
    const hipError_t e = std::apply(
        [&](P &...p) {
            void *argv[] = {&p...};
            return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(threads), argv, lds, s);
        },
        args);
    if (e == hipSuccess) return RESHARD_OK;
    return fail(RESHARD_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace rs
