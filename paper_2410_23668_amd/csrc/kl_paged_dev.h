// Device helpers of the paged KV cache's kernels.
#pragma once

#include "kl_paged.h"
#include "kl_step_impl.h"

namespace kl {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void flag_error(int32_t *error, int bits) {
    if (error) __hip_atomic_fetch_or(error, bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// 2^(s - 127) from its exponent bits (s in 1..254)
__device__ __forceinline__ float pow2_of(unsigned s) { return __uint_as_float(s << 23); }

// 16 bytes of a caller's elements (16-bit ones, or floats), as one word where
// it is aligned; Once: non-temporal.
template <bool Once, class E>
__device__ __forceinline__ u32x4 load_16B(const E *p, bool vec) {
    if (vec) {
        if constexpr (Once) return ld_stream_16B(p);
        else return *reinterpret_cast<const u32x4 *>(p);
    }
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 4) w[i] = __builtin_bit_cast(unsigned, p[i]);
        else w[i] = p[2 * i] | ((unsigned)p[2 * i + 1] << 16);
    }
    return w;
}
// 8 elements from their words (of 16-bit elements: the first four).
__device__ __forceinline__ void words_to_f32(u32x4 a, u32x4 b, int type, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (type == KL_DTYPE_FP32) {
            x[i] = __uint_as_float(a[i]);
            x[i + 4] = __uint_as_float(b[i]);
        } else if (type == KL_DTYPE_BF16) {
            x[2 * i] = bf_lo(a[i]);
            x[2 * i + 1] = bf_hi(a[i]);
        } else {
            x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)a[i]);
            x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(a[i] >> 16));
        }
    }
}

// 16 bytes that this call does not read again: non-temporal (rows read back,
// e4m3 to fp32: 61 -> 42 us at 24402 rows of 8 heads of 128).
template <class V>
__device__ __forceinline__ void store_16B(void *p, V v) {
    static_assert(sizeof(V) == 16, "one word");
    __builtin_nontemporal_store(v, reinterpret_cast<V *>(p));
}

// 8 consecutive elements of a caller's row as floats, and back.  (16-bit rows
// are read once, non-temporal; a lane's two words of an fp32 row lie in lines
// that other lanes' words are in: 71 us against 73 so at 32768 rows, where 16-bit
// ones take 47 against 50.)
__device__ __forceinline__ void load8(const void *p, int type, bool vec, float (&x)[8]) {
    const float *f = reinterpret_cast<const float *>(p);
    if (type == KL_DTYPE_FP32)
        words_to_f32(load_16B<false>(f, vec), load_16B<false>(f + 4, vec), type, x);
    else
        words_to_f32(load_16B<true>(reinterpret_cast<const uint16_t *>(p), vec), u32x4{}, type, x);
}

// The 16-bit pattern of x in type (bf16 or fp16), nearest even.
__device__ __forceinline__ uint16_t bits16(float x, int type) {
    return type == KL_DTYPE_BF16 ? f2bf(x) : __builtin_bit_cast(uint16_t, (_Float16)x);
}

__device__ __forceinline__ void store8(void *p, int type, bool vec, const float (&x)[8]) {
    if (type == KL_DTYPE_FP32) {
        float *f = reinterpret_cast<float *>(p);
        if (vec) {
            store_16B(f, f32x4{x[0], x[1], x[2], x[3]});
            store_16B(f + 4, f32x4{x[4], x[5], x[6], x[7]});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = x[i];
        }
        return;
    }
    uint16_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = bits16(x[i], type);
    if (vec) {
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = h[2 * i] | ((unsigned)h[2 * i + 1] << 16);
        store_16B(p, a);
    } else {
        uint16_t *o = reinterpret_cast<uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = h[i];
    }
}

// Two floats written and read as one device-coherent word (8-byte aligned).
__device__ __forceinline__ void st_dev_f2(float *p, float a, float b) {
    st_dev_u64(reinterpret_cast<unsigned long long *>(p),
               (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a));
}
__device__ __forceinline__ f32x2 ld_dev_f2(const float *p) {
    const unsigned long long v = ld_dev_u64(p);
    return f32x2{__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32))};
}

}  // namespace kl
