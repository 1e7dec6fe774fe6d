// Device code of the paged KV cache (kl_paged_* in include/kl.h): rows written
// to and read from pages, and the choice of the attention kernel.

#include <algorithm>

#include "kl_paged_dev.h"

namespace kl {

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


hipError_t launch_paged_attention(const AttnParams &p, hipStream_t stream) {
    return p.c.d == 128 ? launch_paged_attention_d128(p, stream)
                        : launch_paged_attention_d64(p, stream);
}

}  // namespace kl
