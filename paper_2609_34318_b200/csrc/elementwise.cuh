// What the memory-bound kernels that move rows of bf16 share (mla_ops.cu, paged_ops.cu): vectors of 16 or 32 bytes, division by
// a number known on the host, the rotary angle.
#pragma once
#include <cuda_bf16.h>

#include <initializer_list>

#include "hydra_internal.h"
#include "sm100_ptx.cuh"

namespace hydra {
namespace {

constexpr int kVecThreads = 256;

__device__ __forceinline__ float2 bf2_to_f2(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t f2_to_bf2(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

inline bool aligned16_all(std::initializer_list<const void*> ptrs)
{
    uintptr_t bits = 0;
    for (const void* p : ptrs) bits |= reinterpret_cast<uintptr_t>(p);
    return (bits & 15u) == 0;
}

inline bool all_aligned32(std::initializer_list<const void*> ptrs)
{
    uintptr_t bits = 0;
    for (const void* p : ptrs) bits |= reinterpret_cast<uintptr_t>(p);
    return (bits & 31u) == 0;
}

// kWords 32-bit words (pairs of bf16) per thread and access: 4 (16 bytes), or 8 (32 bytes) where the element
// count and the buffers allow it. Half as many threads then share the loop and address arithmetic.
template <int kWords>
struct Words { uint32_t w[kWords]; };
template <int kWords>
__device__ __forceinline__ Words<kWords> ld_words(const void* base, int64_t i)
{
    Words<kWords> v;
    if constexpr (kWords == 8) {
        const Words<8>* p = static_cast<const Words<8>*>(base) + i;
        asm volatile("ld.global.nc.L1::no_allocate.v8.u32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]),
                       "=r"(v.w[6]), "=r"(v.w[7])
                     : "l"(p));
    } else {
        const uint4 t = static_cast<const uint4*>(base)[i];
        v.w[0] = t.x; v.w[1] = t.y; v.w[2] = t.z; v.w[3] = t.w;
    }
    return v;
}
// the same from memory that this kernel writes
template <int kWords>
__device__ __forceinline__ Words<kWords> ld_words_coherent(const void* base, int64_t i)
{
    Words<kWords> v;
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const Words<kWords>*>(base) + i);
#pragma unroll
    for (int j = 0; j < kWords / 4; ++j) {
        const uint4 t = p[j];
        v.w[4 * j] = t.x; v.w[4 * j + 1] = t.y; v.w[4 * j + 2] = t.z; v.w[4 * j + 3] = t.w;
    }
    return v;
}
template <int kWords>
__device__ __forceinline__ void st_words(void* base, int64_t i, const Words<kWords>& v)
{
    if constexpr (kWords == 8) {
        st_global_v8(static_cast<Words<8>*>(base) + i, v.w);
    } else {
        static_cast<uint4*>(base)[i] = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    }
}

// n / d for n * d < 2^32: the error of n * m / 2^32, m = floor(2^32 / d) + 1, is under 1 / d
struct Div {
    uint32_t d, m;
    explicit Div(uint32_t div) : d(div), m(div > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / div) + 1 : 0) {}
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return m ? __umulhi(n, m) : n; }
};

// cos / sin of position * freq, the angle reduced as in rope_table. The reduced angle, up to 2 pi, is rounded to 32 bits (2^-22 at most):
// that and the single-precision functions leave cosine and sine off by some 2^-21, where the row is rounded to bf16 by 2^-8.
__device__ __forceinline__ void rope_angle(int32_t pos, double freq, float& cs, float& sn)
{
    double ang = static_cast<double>(pos) * freq;
    // The whole turns are the floor of ang / 2 pi. Multiplied by 1 / 2 pi it is off by less than 3 * 2^-53 of at most 2^31 / 2 pi turns,
    // 1.2e-7: the division itself is needed only next to a whole number.
    const double turns = ang * 0.15915494309189533576889;
    double whole = floor(turns);
    if (const double part = turns - whole; part < 1e-6 || part > 1.0 - 1e-6) whole = floor(ang / 6.283185307179586476925);
    ang -= 6.283185307179586476925 * whole;
    sincosf(static_cast<float>(ang), &sn, &cs);
}

template <int kWords>
__device__ __forceinline__ Words<kWords> rotate_vec(const Words<kWords>& w, const float* cp, const float* sp)
{
    Words<kWords> out;
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        const float2 v = bf2_to_f2(w.w[j]);
        out.w[j] = f2_to_bf2(v.x * cp[j] - v.y * sp[j], v.x * sp[j] + v.y * cp[j]);
    }
    return out;
}

// n vectors of a block: load(e) gives vector e and where it goes, store(at, v) puts it there
template <int kWords, int kVecUnroll, class Load, class Store>
__device__ __forceinline__ void move_vecs(uint32_t n, Load load, Store store)
{
    for (uint32_t e0 = threadIdx.x; e0 < n; e0 += kVecUnroll * kVecThreads) {
        Words<kWords> v[kVecUnroll];
        uint32_t at[kVecUnroll];
#pragma unroll
        for (int u = 0; u < kVecUnroll; ++u)
            if (e0 + u * kVecThreads < n) v[u] = load(e0 + u * kVecThreads, at[u]);
#pragma unroll
        for (int u = 0; u < kVecUnroll; ++u)
            if (e0 + u * kVecThreads < n) store(at[u], v[u]);
    }
}

// kWords of the vector kernels that the dimensions and buffers admit: 8, 4 or 0 (the four-byte kernels)
inline int words_for(std::initializer_list<int32_t> dims, std::initializer_list<const void*> ptrs)
{
    int32_t bits = 0;
    for (int32_t d : dims) bits |= d;
    if (bits % 16 == 0 && all_aligned32(ptrs)) return 8;
    return bits % 8 == 0 && aligned16_all(ptrs) ? 4 : 0;
}

}  // namespace
}  // namespace hydra
