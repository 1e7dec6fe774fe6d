// Device code of the paged KV cache (kl_paged_* in include/kl.h): rows written
// to and read from pages, and the attention of one new token per sequence.

#include <algorithm>

#include "kl_paged.h"
#include "kl_step_impl.h"

namespace kl {

typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void flag_error(int32_t *error, int bits) {
    if (error) __hip_atomic_fetch_or(error, bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// 2^(s - 127) from its exponent bits (s in 1..254)
__device__ __forceinline__ float pow2_of(unsigned s) { return __uint_as_float(s << 23); }

// ---------------------------------------------------------------- rows

// 8 consecutive elements of a caller's row as floats, and back.
__device__ __forceinline__ void load8(const void *p, int type, bool vec, float (&x)[8]) {
    if (type == KL_DTYPE_FP32) {
        const float *f = reinterpret_cast<const float *>(p);
        if (vec) {
            const f32x4 a = *reinterpret_cast<const f32x4 *>(f);
            const f32x4 b = *reinterpret_cast<const f32x4 *>(f + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = a[i], x[i + 4] = b[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = f[i];
        }
        return;
    }
    unsigned u[4];
    if (vec) {
        const u32x4 a = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = a[i];
    } else {
        const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = h[2 * i] | ((unsigned)h[2 * i + 1] << 16);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (type == KL_DTYPE_BF16) {
            x[2 * i] = bf_lo(u[i]);
            x[2 * i + 1] = bf_hi(u[i]);
        } else {
            x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)u[i]);
            x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(u[i] >> 16));
        }
    }
}

// The 16-bit pattern of x in type (bf16 or fp16), nearest even.
__device__ __forceinline__ uint16_t bits16(float x, int type) {
    return type == KL_DTYPE_BF16 ? f2bf(x) : __builtin_bit_cast(uint16_t, (_Float16)x);
}

__device__ __forceinline__ void store8(void *p, int type, bool vec, const float (&x)[8]) {
    if (type == KL_DTYPE_FP32) {
        float *f = reinterpret_cast<float *>(p);
        if (vec) {
            *reinterpret_cast<f32x4 *>(f) = f32x4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<f32x4 *>(f + 4) = f32x4{x[4], x[5], x[6], x[7]};
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
        *reinterpret_cast<u32x4 *>(p) = a;
    } else {
        uint16_t *o = reinterpret_cast<uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = h[i];
    }
}

// The pool row of (row r of the call, head): its index among the layer's rows
// of heads, -1 for a padding row, -2 for a bad one.
__device__ __forceinline__ long long slot_row(const RowParams &p, long long r, int head) {
    const int pos = p.positions[r];
    if (pos < 0) return -1;
    const long long b = p.seq ? p.seq[r] : r;
    if (b < 0 || b >= p.t.batch || (pos >> p.c.page_log2) >= p.t.max_pages) {
        flag_error(p.error, KL_DEVERR_POSITION);
        return -2;
    }
    const int page = p.t.pages[b * p.t.stride + (pos >> p.c.page_log2)];
    if (page < 0 || page >= p.c.n_pages) {
        flag_error(p.error, KL_DEVERR_PAGE);
        return -2;
    }
    return (((long long)page * p.c.nkv + head) << p.c.page_log2) +
           (pos & ((1 << p.c.page_log2) - 1));
}

// 8 lanes (head_dim 64) or 16 (128) have a row of a head, 8 elements each: one
// 16-byte load of 16-bit values.  A row's largest magnitude is a maximum of
// bit patterns (monotonic for magnitudes, and an infinity or a NaN is above
// every number), by DPP within the row's lanes.
template <int D>
__global__ void __launch_bounds__(256) kl_paged_append_kernel(RowParams p) {
    constexpr int LR = D / 8;
    const long long items = p.rows * p.c.nkv * 2;
    const int j = threadIdx.x % LR;
    for (long long it = (long long)blockIdx.x * (256 / LR) + threadIdx.x / LR; it < items;
         it += (long long)gridDim.x * (256 / LR)) {
        const bool is_v = it & 1;
        const int head = (int)((it >> 1) % p.c.nkv);
        const long long r = (it >> 1) / p.c.nkv;
        const long long row = slot_row(p, r, head);
        if (row < 0) continue;
        const int type = is_v ? p.v_type : p.k_type;
        const long long at = (is_v ? r * p.v_row + head * p.v_head : r * p.k_row + head * p.k_head) + 8 * j;
        float x[8];
        load8(reinterpret_cast<const uint8_t *>(is_v ? p.v : p.k) + at * (type == KL_DTYPE_FP32 ? 4 : 2),
              type, is_v ? p.v_vec : p.k_vec, x);
        uint8_t *pool = is_v ? p.c.v : p.c.k;
        if (!p.c.e4m3) {
            store8(pool + (row * D + 8 * j) * 2, KL_DTYPE_BF16, true, x);
            continue;
        }
        unsigned a = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
        for (int o = 1; o < LR; o <<= 1) a = max(a, (unsigned)__shfl_xor((int)a, o));
        // a = 1.f 2^E <= 448 2^e = 1.75 2^(e + 8): e = E - 8, one more past 1.75
        const bool bad = a >= 0x7f800000u;
        const int e = max((int)(a >> 23) - 127 - 8 + ((a & 0x7fffffu) > 0x600000u), -126);
        const float inv = pow2_of(bad ? 127 : 127 - e);
        int w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, w[i], false);
            w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, w[i], true);
        }
        if (bad) w[0] = w[1] = 0x7f7f7f7f;   // (NaN)
        *reinterpret_cast<int2 *>(pool + row * D + 8 * j) = make_int2(w[0], w[1]);
        if (j == 0) (is_v ? p.c.vs : p.c.ks)[row] = (uint8_t)(bad ? 127 : e + 127);
    }
}

template <int D>
__global__ void __launch_bounds__(256) kl_paged_read_kernel(RowParams p) {
    constexpr int LR = D / 8;
    const long long items = p.rows * p.c.nkv * 2;
    const int j = threadIdx.x % LR;
    for (long long it = (long long)blockIdx.x * (256 / LR) + threadIdx.x / LR; it < items;
         it += (long long)gridDim.x * (256 / LR)) {
        const bool is_v = it & 1;
        const int head = (int)((it >> 1) % p.c.nkv);
        const long long r = (it >> 1) / p.c.nkv;
        const long long row = slot_row(p, r, head);
        if (row == -1) continue;
        float x[8];
        if (row < 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_nanf("");
        } else if (!p.c.e4m3) {
            load8((is_v ? p.c.v : p.c.k) + (row * D + 8 * j) * 2, KL_DTYPE_BF16, true, x);
        } else {
            const int2 w = *reinterpret_cast<const int2 *>((is_v ? p.c.v : p.c.k) + row * D + 8 * j);
            const float s = pow2_of((is_v ? p.c.vs : p.c.ks)[row]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int u = i ? w.y : w.x;
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(u, false);
                const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
                x[4 * i] = lo[0] * s, x[4 * i + 1] = lo[1] * s;
                x[4 * i + 2] = hi[0] * s, x[4 * i + 3] = hi[1] * s;
            }
        }
        const int type = is_v ? p.v_type : p.k_type;
        const long long at = (is_v ? r * p.v_row + head * p.v_head : r * p.k_row + head * p.k_head) + 8 * j;
        store8(reinterpret_cast<uint8_t *>(is_v ? p.v : p.k) + at * (type == KL_DTYPE_FP32 ? 4 : 2),
               type, is_v ? p.v_vec : p.k_vec, x);
    }
}

static int row_blocks(const RowParams &p) {
    const long long per = 256 / (p.c.d / 8), items = p.rows * p.c.nkv * 2;
    return (int)std::min<long long>((items + per - 1) / per, 1 << 20);
}

hipError_t launch_paged_append(const RowParams &p, hipStream_t stream) {
    if (p.c.d == 128)
        hipLaunchKernelGGL(kl_paged_append_kernel<128>, dim3(row_blocks(p)), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(kl_paged_append_kernel<64>, dim3(row_blocks(p)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_paged_read(const RowParams &p, hipStream_t stream) {
    if (p.c.d == 128)
        hipLaunchKernelGGL(kl_paged_read_kernel<128>, dim3(row_blocks(p)), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(kl_paged_read_kernel<64>, dim3(row_blocks(p)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

// ---------------------------------------------------------------- attention

__device__ __forceinline__ float load1(const void *p, int type, long long i) {
    if (type == KL_DTYPE_FP32) return reinterpret_cast<const float *>(p)[i];
    const uint16_t h = reinterpret_cast<const uint16_t *>(p)[i];
    return type == KL_DTYPE_BF16 ? bf2f(h) : (float)__builtin_bit_cast(_Float16, h);
}
__device__ __forceinline__ void store1(void *p, int type, long long i, float x) {
    if (type == KL_DTYPE_FP32) reinterpret_cast<float *>(p)[i] = x;
    else reinterpret_cast<uint16_t *>(p)[i] = bits16(x, type);
}

// Element i of a pool's row.
__device__ __forceinline__ float pool1(const PagedLayer &c, const uint8_t *p, const uint8_t *scale,
                                       long long row, int D, int i) {
    if (!c.e4m3) return bf2f(reinterpret_cast<const uint16_t *>(p)[row * D + i]);
    return __builtin_amdgcn_cvt_f32_fp8(p[row * D + i], 0) * pow2_of(scale[row]);
}

// One workgroup per (sequence, query head), its four waves every fourth
// position each with a running maximum and sum, joined at the end.
template <int D>
__global__ void __launch_bounds__(256) kl_paged_attention_kernel(AttnParams p) {
    constexpr int E = D / 64;
    __shared__ float wm[4], wl[4], wo[4][D];
    const int b = blockIdx.x / p.nq, h = blockIdx.x % p.nq, g = h / p.group;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int ps = 1 << p.c.page_log2;
    int len = p.lengths[b];
    bool bad = len < 0 || (long long)len > (long long)p.t.max_pages * ps;
    if (bad) {
        flag_error(p.error, KL_DEVERR_POSITION);
        len = 0;
    }
    float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        q[i] = load1(p.q, p.q_type, b * p.q_row + h * p.q_head + lane * E + i);
        o[i] = 0.f;
    }
    for (int j = (p.window > 0 ? max(0, len - p.window) : 0) + wave; j < len; j += 4) {
        const int page = p.t.pages[(long long)b * p.t.stride + (j >> p.c.page_log2)];
        if (page < 0 || page >= p.c.n_pages) {
            flag_error(p.error, KL_DEVERR_PAGE);
            bad = true;
            break;
        }
        const long long row = (((long long)page * p.c.nkv + g) << p.c.page_log2) + (j & (ps - 1));
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) s = fmaf(q[i], pool1(p.c, p.c.k, p.c.ks, row, D, lane * E + i), s);
        s = wave_sum(s) * p.scale;
        const float mn = fmaxf(m, s), a = __expf(m - mn), w = __expf(s - mn);
        l = l * a + w;
#pragma unroll
        for (int i = 0; i < E; ++i)
            o[i] = o[i] * a + w * pool1(p.c, p.c.v, p.c.vs, row, D, lane * E + i);
        m = mn;
    }
    if (bad) l = __builtin_nanf("");
    wm[wave] = m;
    wl[wave] = l;
#pragma unroll
    for (int i = 0; i < E; ++i) wo[wave][lane * E + i] = o[i];
    __syncthreads();
    const float M = fmaxf(fmaxf(wm[0], wm[1]), fmaxf(wm[2], wm[3]));
    float L = 0.f;
    for (int w = 0; w < 4; ++w) L += wl[w] * (wm[w] == -INFINITY && !isnan(wl[w]) ? 0.f : __expf(wm[w] - M));
    if (isnan(wl[0]) || isnan(wl[1]) || isnan(wl[2]) || isnan(wl[3])) L = __builtin_nanf("");
    for (int i = threadIdx.x; i < D; i += 256) {
        float O = 0.f;
        for (int w = 0; w < 4; ++w) O += wm[w] == -INFINITY ? 0.f : wo[w][i] * __expf(wm[w] - M);
        store1(p.out, p.out_type, b * p.out_row + h * p.out_head + i, L == 0.f ? 0.f : O / L);
    }
    if (p.lse && threadIdx.x == 0) p.lse[(long long)b * p.nq + h] = L == 0.f ? -INFINITY : M + logf(L);
}

hipError_t launch_paged_attention(const AttnParams &p, hipStream_t stream) {
    const dim3 grid(p.t.batch * p.nq);
    if (p.c.d == 128)
        hipLaunchKernelGGL(kl_paged_attention_kernel<128>, grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(kl_paged_attention_kernel<64>, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace kl
