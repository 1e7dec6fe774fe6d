// Device code of the paged KV cache (kl_paged_* in include/kl.h): rows written
// to and read from pages, and the choice of the attention kernel.

#include <algorithm>

#include "kl_paged_dev.h"

namespace kl {

// Rows.  A group of lanes, 8 for head_dim 64 and 16 for 128 (8 elements each),
// has R rows of the call, of one head and of K or V.  Its first R lanes look up
// a row's slot each; all R rows are in flight together, and their scale bytes
// move in one access, a byte per lane.  Both kernels are bound by HBM (32768
// rows of 8 heads of 128, bf16 to e4m3: 47 us, 4.3 TB/s; 24402 rows e4m3 to fp32:
// 40 us, 6.3 TB/s; with R = 1 66 and 73, with R = 8 51 and 42).  How many rows a
// group takes: many_rows below.

// The pool row of (row r of the call, head): its index among the layer's rows
// of heads, -1 for a padding row (or none), -2 for a bad one.
__device__ __forceinline__ long long slot_row(const RowParams &p, long long r, int head) {
    if (r >= p.rows) return -1;
    const int pos = p.positions[r];
    const long long b = p.seq ? p.seq[r] : r;
    if (pos < 0) return -1;
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

// a group's lane i's value of a 64-bit integer (width: lanes of a group)
__device__ __forceinline__ long long of_lane(long long v, int i, int width) {
    const int lo = __shfl((int)v, i, width), hi = __shfl((int)(v >> 32), i, width);
    return ((long long)hi << 32) | (unsigned)lo;
}

template <int W>
__device__ __forceinline__ unsigned max_lanes(unsigned v) {   // over aligned groups of W lanes
    const auto step = [&](auto ctrl) {
        v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, false));
    };
    step(std::integral_constant<int, 0xB1>());    // quad_perm [1,0,3,2]
    step(std::integral_constant<int, 0x4E>());    // quad_perm [2,3,0,1]
    step(std::integral_constant<int, 0x141>());   // row_half_mirror
    if constexpr (W == 16) step(std::integral_constant<int, 0x140>());   // row_mirror
    return v;
}

// A group's place: its rows' block, K or V, its head (heads first, so that a
// wave reads neighbouring ones).
struct RowItem { long long row0; int head; bool is_v; };
template <int R>
__device__ __forceinline__ RowItem row_item(const RowParams &p, long long it) {
    const int head = (int)(it % p.c.nkv);
    const long long rest = it / p.c.nkv;
    return RowItem{(rest >> 1) * R, head, (rest & 1) != 0};
}
template <int R>
__device__ __forceinline__ long long row_items(const RowParams &p) {
    return (p.rows + R - 1) / R * 2 * p.c.nkv;
}

// A row's largest magnitude is a maximum of bit patterns: monotonic for
// magnitudes, and an infinity or a NaN is above every number.
template <int D, int R>
__global__ void __launch_bounds__(256) kl_paged_append_kernel(RowParams p) {
    constexpr int LR = D / 8;
    static_assert(R <= LR, "a lane for every row");
    const int j = threadIdx.x % LR;
    const long long items = row_items<R>(p);
    for (long long it = (long long)blockIdx.x * (256 / LR) + threadIdx.x / LR; it < items;
         it += (long long)gridDim.x * (256 / LR)) {
        const RowItem m = row_item<R>(p, it);
        const int type = m.is_v ? p.v_type : p.k_type;
        const bool vec = m.is_v ? p.v_vec : p.k_vec;
        const uint8_t *src = reinterpret_cast<const uint8_t *>(m.is_v ? p.v : p.k);
        const long long stride = m.is_v ? p.v_row : p.k_row;
        const long long col = m.head * (m.is_v ? p.v_head : p.k_head) + 8 * j;
        const int bytes = type == KL_DTYPE_FP32 ? 4 : 2;
        float x[R][8];
#pragma unroll
        for (int i = 0; i < R; ++i)   // (rows past the last: the last again)
            load8(src + (min(m.row0 + i, p.rows - 1) * stride + col) * bytes, type, vec, x[i]);
        const long long own = j < R ? slot_row(p, m.row0 + j, m.head) : -1;
        uint8_t *pool = m.is_v ? p.c.v : p.c.k;
        unsigned scale = 0;   // of lane j's row
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long row = of_lane(own, i, LR);
            if (!p.c.e4m3) {
                if (row >= 0) store8(pool + (row * D + 8 * j) * 2, KL_DTYPE_BF16, true, x[i]);
                continue;
            }
            unsigned a = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) a = max(a, __float_as_uint(x[i][k]) & 0x7fffffffu);
            a = max_lanes<LR>(a);
            // a = 1.f 2^E <= 448 2^e = 1.75 2^(e + 8): e = E - 8, one more past 1.75
            const bool bad = a >= 0x7f800000u;
            const int e = max((int)(a >> 23) - 127 - 8 + ((a & 0x7fffffu) > 0x600000u), -126);
            const float inv = pow2_of(bad ? 127 : 127 - e);
            int w[2] = {0, 0};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float *y = x[i] + 4 * k;
                w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * inv, y[1] * inv, w[k], false);
                w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * inv, y[3] * inv, w[k], true);
            }
            if (bad) w[0] = w[1] = 0x7f7f7f7f;   // (NaN)
            if (row >= 0)
                __builtin_nontemporal_store(u32x2{(unsigned)w[0], (unsigned)w[1]},
                                            reinterpret_cast<u32x2 *>(pool + row * D + 8 * j));
            if (j == i) scale = bad ? 127 : e + 127;
        }
        if (p.c.e4m3 && own >= 0) (m.is_v ? p.c.vs : p.c.ks)[own] = (uint8_t)scale;
    }
}

// Wide: both outputs are fp32; a lane has 4 elements in each half of the row, so
// that a store covers contiguous memory.
template <int D, int R, bool Wide>
__global__ void __launch_bounds__(256) kl_paged_read_kernel(RowParams p) {
    constexpr int LR = D / 8;
    static_assert(R <= LR, "a lane for every row");
    const int j = threadIdx.x % LR;
    const int e0 = Wide ? 4 * j : 8 * j, e1 = Wide ? D / 2 + 4 * j : 8 * j + 4;
    const long long items = row_items<R>(p);
    for (long long it = (long long)blockIdx.x * (256 / LR) + threadIdx.x / LR; it < items;
         it += (long long)gridDim.x * (256 / LR)) {
        const RowItem m = row_item<R>(p, it);
        const long long own = j < R ? slot_row(p, m.row0 + j, m.head) : -1;
        const uint8_t *pool = m.is_v ? p.c.v : p.c.k;
        unsigned scale = 0;
        if (p.c.e4m3 && own >= 0) scale = (m.is_v ? p.c.vs : p.c.ks)[own];
        u32x2 w[R][2];   // 4 elements each (e4m3: one word of each pair)
        long long row[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            row[i] = of_lane(own, i, LR);
            const long long at = max(row[i], 0ll) * D;
            if (p.c.e4m3) {
                w[i][0][0] = *reinterpret_cast<const unsigned *>(pool + at + e0);
                w[i][1][0] = *reinterpret_cast<const unsigned *>(pool + at + e1);
            } else {
                w[i][0] = *reinterpret_cast<const u32x2 *>(pool + (at + e0) * 2);
                w[i][1] = *reinterpret_cast<const u32x2 *>(pool + (at + e1) * 2);
            }
        }
        const int type = m.is_v ? p.v_type : p.k_type;
        const bool vec = m.is_v ? p.v_vec : p.k_vec;
        uint8_t *dst = reinterpret_cast<uint8_t *>(m.is_v ? p.v : p.k);
        const long long stride = m.is_v ? p.v_row : p.k_row;
        const long long col = m.head * (m.is_v ? p.v_head : p.k_head);
        const int bytes = type == KL_DTYPE_FP32 ? 4 : 2;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float s = pow2_of((unsigned)__shfl((int)scale, i, LR));
            if (row[i] == -1) continue;
            float x[8];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (p.c.e4m3) {
                    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i][k][0], false);
                    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i][k][0], true);
                    x[4 * k] = lo[0] * s, x[4 * k + 1] = lo[1] * s;
                    x[4 * k + 2] = hi[0] * s, x[4 * k + 3] = hi[1] * s;
                } else {
                    x[4 * k] = bf_lo(w[i][k][0]), x[4 * k + 1] = bf_hi(w[i][k][0]);
                    x[4 * k + 2] = bf_lo(w[i][k][1]), x[4 * k + 3] = bf_hi(w[i][k][1]);
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = row[i] < 0 ? __builtin_nanf("") : x[k];
            uint8_t *out = dst + ((m.row0 + i) * stride + col) * bytes;
            if constexpr (Wide) {
                float *o0 = reinterpret_cast<float *>(out) + e0, *o1 = reinterpret_cast<float *>(out) + e1;
                if (vec) {
                    store_16B(o0, f32x4{x[0], x[1], x[2], x[3]});
                    store_16B(o1, f32x4{x[4], x[5], x[6], x[7]});
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) o0[k] = x[k], o1[k] = x[4 + k];
                }
            } else {
                store8(out + 8 * j * bytes, type, vec, x);
            }
        }
    }
}

// A group takes 4 rows where the groups then still make 8 waves for each of 256
// compute units, else one.
static bool many_rows(const RowParams &p) {
    return (p.rows / 4 * 2 * p.c.nkv) * (p.c.d / 8) >= 256 * 8 * 64;
}
template <class Kernel>
static hipError_t launch_rows(Kernel kernel, const RowParams &p, int R, hipStream_t stream) {
    const long long items = (p.rows + R - 1) / R * 2 * p.c.nkv, per = 256 / (p.c.d / 8);
    const int blocks = (int)std::min<long long>((items + per - 1) / per, 1 << 20);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, stream, p);
    return hipGetLastError();
}

template <int D>
static hipError_t append_for(const RowParams &p, hipStream_t stream) {
    return many_rows(p) ? launch_rows(kl_paged_append_kernel<D, 4>, p, 4, stream)
                        : launch_rows(kl_paged_append_kernel<D, 1>, p, 1, stream);
}
template <int D, bool Wide>
static hipError_t read_for(const RowParams &p, hipStream_t stream) {
    return many_rows(p) ? launch_rows(kl_paged_read_kernel<D, 4, Wide>, p, 4, stream)
                        : launch_rows(kl_paged_read_kernel<D, 1, Wide>, p, 1, stream);
}

hipError_t launch_paged_append(const RowParams &p, hipStream_t stream) {
    return p.c.d == 128 ? append_for<128>(p, stream) : append_for<64>(p, stream);
}

hipError_t launch_paged_read(const RowParams &p, hipStream_t stream) {
    const bool wide = p.k_type == KL_DTYPE_FP32 && p.v_type == KL_DTYPE_FP32;
    if (p.c.d == 128) return wide ? read_for<128, true>(p, stream) : read_for<128, false>(p, stream);
    return wide ? read_for<64, true>(p, stream) : read_for<64, false>(p, stream);
}

// One workgroup per sequence: 8.6 us at 262144 positions in pages of 16, whose
// step took 20 us more with one wave.
__global__ void __launch_bounds__(256) kl_paged_step_rows_kernel(StepRowsParams p) {
    const int b = blockIdx.x;
    const int t = p.tokens[b], pos = p.positions[b];
    const bool in = pos >= 0 && pos < p.cap;
    bool bad = false;
    if (in)
        for (int i = threadIdx.x; i <= pos >> p.page_log2; i += 256) {
            const int page = p.t.pages[(long long)b * p.t.stride + i];
            bad = bad || page < 0 || page >= p.n_pages;
        }
    bad = __syncthreads_or(bad);
    if (threadIdx.x != 0) return;
    if (bad) flag_error(p.error, KL_DEVERR_PAGE);
    const bool ok = in && !bad && t >= 0 && t < p.vocab;
    p.step_pos[b] = bad ? -1 : pos;
    p.append_pos[b] = ok ? pos : -1;
    p.lengths[b] = ok ? pos + 1 : 0;
}

hipError_t launch_paged_step_rows(const StepRowsParams &p, hipStream_t stream) {
    hipLaunchKernelGGL(kl_paged_step_rows_kernel, dim3(p.batch), dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_paged_attention(const AttnParams &p, hipStream_t stream) {
    return p.c.d == 128 ? launch_paged_attention_d128(p, stream)
                        : launch_paged_attention_d64(p, stream);
}

}  // namespace kl
