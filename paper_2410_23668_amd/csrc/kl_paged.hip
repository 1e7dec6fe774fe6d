// Device code of the paged KV cache (kl_paged_* in include/kl.h): rows written
// to and read from pages, and the attention of one new token per sequence.

#include <algorithm>
#include <atomic>

#include "kl_paged.h"
#include "kl_paged_shares.h"
#include "kl_step_impl.h"

namespace kl {

typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void flag_error(int32_t *error, int bits) {
    if (error) __hip_atomic_fetch_or(error, bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// 2^(s - 127) from its exponent bits (s in 1..254)
__device__ __forceinline__ float pow2_of(unsigned s) { return __uint_as_float(s << 23); }

// ---------------------------------------------------------------- rows

// 16 bytes of a caller's elements (16-bit ones, or floats), as one word where
// it is aligned.
template <class E>
__device__ __forceinline__ u32x4 load_16B(const E *p, bool vec) {
    if (vec) return *reinterpret_cast<const u32x4 *>(p);
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

// 8 consecutive elements of a caller's row as floats, and back.
__device__ __forceinline__ void load8(const void *p, int type, bool vec, float (&x)[8]) {
    const float *f = reinterpret_cast<const float *>(p);
    if (type == KL_DTYPE_FP32)
        words_to_f32(load_16B(f, vec), load_16B(f + 4, vec), type, x);
    else
        words_to_f32(load_16B(reinterpret_cast<const uint16_t *>(p), vec), u32x4{}, type, x);
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
//
// Split-K flash decoding over pages.  A unit is a (sequence, KV head); its
// attended positions are cut into tiles of 16 KiB of keys and values, and the
// tiles of all units, one unit after the other, are dealt in equal contiguous
// shares to the workgroups and within one to its eight waves, so that lengths
// of any kind load every wave alike.  A wave goes through its tiles with a
// running maximum and sum; a unit that lies inside its share it writes out,
// of a unit cut by the share's ends it leaves its part (maximum, sum,
// unnormalised output) in LDS.  The workgroup joins the parts there; what is
// part of a unit of several workgroups goes to the workspace, and the last of
// them to arrive (a counter per unit) joins all in workgroup order.
//
// All query heads of a KV head share one pass over its keys and values on the
// matrix cores, in layouts that need no exchange between lanes:
//   S^T = K Q^T  v_mfma_f32_16x16x32_bf16: A = 16 key rows, B = the queries as
//                columns.  The rows of two such products, t = 0 and 1, are the
//                positions 8 (r / 4) + 4 t + r % 4 of a block of 32, so that
//                lane (k4, n) ends up with the scores of head n and positions
//                8 k4 .. 8 k4 + 7: what the second product wants of it.
//   O^T = V^T P^T  A = V^T: lane (k4, r) has loaded elements EV r .. EV r +
//                EV - 1 (EV = d / 16) of the 8 positions, one load a position
//                that covers the whole row; product m takes element m of each,
//                pairs of positions put together by byte permutes.
// e4m3 rows become bf16 (exactly) on the way, keys with their row's scale,
// values without: theirs goes into the probabilities.  Queries of 32 or 16
// bits that bf16 cannot hold, and the probabilities, are taken as several bf16
// terms: three are all 24 bits of a float; two, 16 bits, where the output has
// 16 bits (the weights are off by 2^-17, an eighth of its fp16 half-step at
// most).  Softmax and sums are fp32; the maximum moves only when a score passes
// it by 2^8, so the loop has no cross-lane step.

constexpr int kAttnWaves = 8;
constexpr int kAttnThreads = kAttnWaves * 64;

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float load1(const void *p, int type, long long i) {
    if (type == KL_DTYPE_FP32) return reinterpret_cast<const float *>(p)[i];
    const uint16_t h = reinterpret_cast<const uint16_t *>(p)[i];
    return type == KL_DTYPE_BF16 ? bf2f(h) : (float)__builtin_bit_cast(_Float16, h);
}
__device__ __forceinline__ void store1(void *p, int type, long long i, float x) {
    if (type == KL_DTYPE_FP32) reinterpret_cast<float *>(p)[i] = x;
    else reinterpret_cast<uint16_t *>(p)[i] = bits16(x, type);
}

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(unsigned, v);
}
// NT bf16 terms of 8 floats (x is left as what the terms do not hold)
template <int NT>
__device__ __forceinline__ void split_terms(float (&x)[8], bf16x8 (&t)[NT]) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
            if (i + 1 < NT) {
                x[2 * j] -= bf_lo(w[j]);
                x[2 * j + 1] -= bf_hi(w[j]);
            }
        }
        t[i] = __builtin_bit_cast(bf16x8, w);
    }
}

// Adds the first n (at most NB) of the parts that get(j, output, maximum, sum)
// reads, all of them at once, to (O, M, L).
template <int NB, class Get>
__device__ __forceinline__ void join_parts(int n, float &O, float &M, float &L, Get &&get) {
    float o[NB], m[NB], l[NB], mn = M;
#pragma unroll
    for (int j = 0; j < NB; ++j) get(j, o[j], m[j], l[j]);
#pragma unroll
    for (int j = 0; j < NB; ++j) mn = j < n ? fmaxf(mn, m[j]) : mn;
    const float a = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);   // (none yet: 0)
    L *= a;
    O *= a;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const float w = __builtin_amdgcn_exp2f(m[j] - mn);
        L = j < n ? fmaf(l[j], w, L) : L;
        O = j < n ? fmaf(o[j], w, O) : O;
    }
    M = mn;
}

template <int D, bool F8, bool Full>
__global__ void __launch_bounds__(kAttnThreads, 2) kl_paged_attention_kernel(AttnParams p) {
    constexpr int ES = F8 ? 1 : 2;
    constexpr int NK = paged_tile(D, ES), NS = NK / 32;   // positions of a tile; blocks of 32
    constexpr int RB = D * ES;                  // bytes of a row
    constexpr int NC = RB / 64;                 // 16-byte loads of a key row per lane
    constexpr int EV = D / 16, VW = EV * ES / 4;   // value elements, words per lane and position
    constexpr int ST = D / 32;                  // steps of the first product
    constexpr int QT = Full ? 3 : 1, PT = Full ? 3 : 2;   // terms of queries, probabilities
    constexpr int WD = D + 2;                   // floats of a part of one head
    constexpr int NE = 2 * kAttnWaves;          // parts in LDS

    const int G = p.group, nkv = p.c.nkv, B = p.t.batch;
    float *const part = reinterpret_cast<float *>(kl_smem);      // [NE][G][WD]
    int *const unit = reinterpret_cast<int *>(part + NE * G * WD);   // [NE]: unit, -1: none
    int *const ubeg = unit + NE, *const uend = ubeg + NE;        // its tiles
    int *const wsum = uend + NE;                                 // [kAttnWaves + 1]
    int *const last = wsum + kAttnWaves + 1;                     // [2]
    int *const pre = last + 2;                                   // [B + 1] tiles of earlier sequences

    const int tid = threadIdx.x, lane = tid & 63, k4 = lane >> 4, n = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int psl = p.c.page_log2, psm = (1 << psl) - 1;
    const long long cap = (long long)p.t.max_pages << psl;

    // a length's tiles; a length out of range counts as empty
    auto length_of = [&](int b, bool &bad) {
        const int len = p.lengths[b];
        bad = len < 0 || (long long)len > cap;
        return bad ? 0 : len;
    };
    // Tiles of the sequences up to each: one per lane of every wave, where the
    // wave has lanes for all (no wait for the other waves: 1 us less), else in LDS.
    const bool few = B <= 64;
    if (lane < 2) unit[2 * wave + lane] = -1;   // (read behind a barrier)
    int len_own = 0, upto = 0, most = 0, T;
    bool bad_own = false;
    auto wave_scan = [&](int v) {   // inclusive sum over the lanes
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = from_lane(v, max(lane - off, 0));
            v += lane >= off ? o : 0;
        }
        return v;
    };
    if (few) {
        if (lane < B) len_own = length_of(lane, bad_own);
        const int own = lane < B ? paged_tiles(len_own, p.window, NK) : 0;
        upto = wave_scan(own);
        most = (int)wave_max((float)own);   // (below 2^24: cap and NK)
        T = __builtin_amdgcn_readlane(upto, 63) * nkv;
    } else {
        if (tid == 0) pre[0] = 0;
        int base = 0;
        for (int b0 = 0; b0 < B; b0 += kAttnThreads) {
            const int b = b0 + tid;
            bool bad;
            const int s = wave_scan(b < B ? paged_tiles(length_of(b, bad), p.window, NK) : 0);
            if (lane == 63) wsum[wave] = s;
            __syncthreads();
            int add = base;
#pragma unroll
            for (int w = 0; w < kAttnWaves; ++w) {
                if (w < wave) add += wsum[w];
                base += wsum[w];
            }
            if (b < B) pre[b + 1] = add + s;
            __syncthreads();
        }
        T = __builtin_amdgcn_readfirstlane(base) * nkv;
    }
    // tiles (of one KV head) of the sequences before b
    auto before = [&](int b) {
        if (few) return b > 0 ? __builtin_amdgcn_readlane(upto, b - 1) : 0;
        return __builtin_amdgcn_readfirstlane(pre[b]);
    };
    // the workgroup's share [X0, X1): a unit of its own (unit_shares), or an
    // equal share, with a workgroup for every kAttnWaves tiles
    const int wg = blockIdx.x;
    const bool by_unit = few && unit_shares(B * nkv, gridDim.x, most, T, kAttnWaves);
    const Shares sh(T, by_unit ? B * nkv : min((int)gridDim.x, (T + kAttnWaves - 1) / kAttnWaves));
    if (wg >= sh.np) return;
    int X0, X1;
    if (by_unit) {
        const int b = wg / nkv, g = wg % nkv, nt = before(b + 1) - before(b);
        X0 = before(b) * nkv + g * nt;
        X1 = X0 + nt;
    } else {
        X0 = sh.first(wg);
        X1 = sh.first(wg + 1);
    }
    int x = X0 + (((X1 - X0) * wave) / kAttnWaves);
    const int x1 = X0 + (((X1 - X0) * (wave + 1)) / kAttnWaves);

    // A place in the row of tiles.
    struct At {
        int b, g, t, nt;     // sequence, KV head, tile of the unit, its tiles
        int len, start, t0;  // positions attended: [start, len); first tile
        bool bad;
    };
    auto enter = [&](At &a, int b) {
        a.b = b;
        a.nt = before(b + 1) - before(b);
        if (few) {
            a.len = __builtin_amdgcn_readlane(len_own, b);
            a.bad = __builtin_amdgcn_readlane((int)bad_own, b) != 0;
        } else {
            a.len = __builtin_amdgcn_readfirstlane(length_of(b, a.bad));
        }
        a.start = paged_start(a.len, p.window);
        a.t0 = paged_first_tile(a.len, p.window, NK);
    };
    auto find = [&](int i) {
        int lo = 0;   // before(lo) nkv <= i < before(lo + 1) nkv
        if (few) {
            lo = __popcll(__ballot(lane < B && upto * nkv <= i));
        } else {
            for (int hi = B; hi - lo > 1;) {
                const int mid = (lo + hi) >> 1;
                if (before(mid) * nkv <= i) lo = mid;
                else hi = mid;
            }
        }
        At a;
        enter(a, lo);
        const int r = i - before(lo) * nkv;
        a.g = r / a.nt;
        a.t = r % a.nt;
        return a;
    };
    auto next = [&](At a) {
        if (++a.t == a.nt) {
            a.t = 0;
            if (++a.g == nkv) {
                a.g = 0;
                enter(a, a.b + 1);
            }
        }
        return a;
    };

    // The pages of a tile, entry of the tile's i-th group of 8 positions in
    // lane i (positions outside the attended ones: the nearest one's).
    auto load_pages = [&](const At &a) {
        if (a.len == 0) return 0;
        const int pos = (a.t0 + a.t) * NK + 8 * (lane % (NK / 8));
        return p.t.pages[(long long)a.b * p.t.stride +
                         (min(max(pos, a.start), a.len - 1) >> psl)];
    };
    u32x4 kr[NS][2][NC];
    unsigned vr[NS][8][VW];
    u32x2 ksr[NS], vsr[NS];
    bool page_bad = false;   // of the tile whose keys were asked for last
    auto tile_inside = [&](const At &a) {
        const int key0 = (a.t0 + a.t) * NK;
        return key0 >= a.start && key0 + NK <= a.len;
    };
    // byte offset of the page's rows of head g, for the group of positions of
    // lane 'from' of pages
    auto page_row = [&](const At &a, int pages, int from) {
        const int page = from_lane(pages, from);
        return ((long long)page * nkv + a.g) << psl;
    };
    auto load_keys = [&](const At &a, int &pages) {
        if (a.len == 0) return;
        page_bad = __any((unsigned)pages >= (unsigned)p.c.n_pages);
        if ((unsigned)pages >= (unsigned)p.c.n_pages) pages = 0;
        const int key0 = (a.t0 + a.t) * NK;
        if (tile_inside(a)) {
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const int key = key0 + 32 * s + 8 * (n >> 2);
                const long long r0 = page_row(a, pages, 4 * s + (n >> 2)) + (key & psm);
                const uint8_t *src = p.c.k + (r0 + (n & 3)) * RB + 16 * k4;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int c = 0; c < NC; ++c) kr[s][t][c] = ld_stream_16B(src + 4 * t * RB + 64 * c);
                if constexpr (F8) ksr[s] = *reinterpret_cast<const u32x2 *>(p.c.ks + r0);
            }
            return;
        }
        // (rows outside the attended positions: the nearest attended one's)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int gk = key0 + 32 * s + 8 * (n >> 2);
            const long long r0 = page_row(a, pages, 4 * s + (n >> 2));
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int key = min(max(gk + 4 * t + (n & 3), a.start), a.len - 1);
                const uint8_t *src = p.c.k + (r0 + (key & psm)) * RB + 16 * k4;
#pragma unroll
                for (int c = 0; c < NC; ++c) kr[s][t][c] = ld_stream_16B(src + 64 * c);
            }
            if constexpr (F8)
                ksr[s] = *reinterpret_cast<const u32x2 *>(
                    p.c.ks + r0 + (min(max(gk, a.start), a.len - 1) & psm & ~7));
        }
    };
    auto load_value = [&](const uint8_t *src, unsigned (&v)[VW]) {
        if constexpr (VW == 4) {
            const u32x4 w = ld_stream_16B(src);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = w[i];
        } else if constexpr (VW == 2) {
            const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(src));
            v[0] = w[0];
            v[1] = w[1];
        } else {
            v[0] = __builtin_nontemporal_load(reinterpret_cast<const unsigned *>(src));
        }
    };
    auto load_values = [&](const At &a, int pages) {
        if (a.len == 0) return;
        const int key0 = (a.t0 + a.t) * NK;
        if (tile_inside(a)) {
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const int key = key0 + 32 * s + 8 * k4;
                const long long r0 = page_row(a, pages, 4 * s + k4) + (key & psm);
                const uint8_t *src = p.c.v + r0 * RB + n * (EV * ES);
#pragma unroll
                for (int j = 0; j < 8; ++j) load_value(src + j * RB, vr[s][j]);
                if constexpr (F8) vsr[s] = *reinterpret_cast<const u32x2 *>(p.c.vs + r0);
            }
            return;
        }
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int gk = key0 + 32 * s + 8 * k4;
            const long long r0 = page_row(a, pages, 4 * s + k4);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int key = min(max(gk + j, a.start), a.len - 1);
                load_value(p.c.v + (r0 + (key & psm)) * RB + n * (EV * ES), vr[s][j]);
            }
            if constexpr (F8)
                vsr[s] = *reinterpret_cast<const u32x2 *>(
                    p.c.vs + r0 + (min(max(gk, a.start), a.len - 1) & psm & ~7));
        }
    };

    // The queries of a unit as columns of the first product: asked for as they
    // are, and taken apart into terms when they are needed.
    constexpr int QW = Full ? 2 : 1;   // 16-byte words of 8 elements, at most
    bf16x8 q[QT][ST];
    auto ask_q = [&](const At &a, u32x4 (&raw)[ST][QW]) {
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            const int d0 = F8 ? 64 * (s / 2) + 16 * k4 + 8 * (s & 1) : 32 * s + 8 * k4;
            // (columns past the group: head 0 again, masked below)
            const long long at = a.b * p.q_row + (a.g * G + (n < G ? n : 0)) * p.q_head + d0;
            const float *f = reinterpret_cast<const float *>(p.q) + at;
            if (Full && p.q_type == KL_DTYPE_FP32) {
                raw[s][0] = load_16B(f, p.q_vec);
                raw[s][QW - 1] = load_16B(f + 4, p.q_vec);
            } else {
                raw[s][0] = load_16B(reinterpret_cast<const uint16_t *>(p.q) + at, p.q_vec);
                if (Full) raw[s][QW - 1] = raw[s][0];
            }
        }
    };
    const float sign = p.scale > 0.f ? 1.f : p.scale < 0.f ? -1.f : 0.f;
    auto take_q = [&](const u32x4 (&raw)[ST][QW]) {
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            if constexpr (Full) {
                float v[8];
                words_to_f32(raw[s][0], raw[s][QW - 1], p.q_type, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = n < G ? v[j] * sign : 0.f;
                bf16x8 t[QT];
                split_terms(v, t);
#pragma unroll
                for (int i = 0; i < QT; ++i) q[i][s] = t[i];
            } else {   // (bf16 queries are their own term)
                u32x4 w = raw[s][0];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = n < G && sign != 0.f ? w[i] ^ (sign < 0.f ? 0x80008000u : 0u) : 0u;
                q[0][s] = __builtin_bit_cast(bf16x8, w);
            }
        }
    };

    const int out_bytes = p.out_type == KL_DTYPE_FP32 ? 4 : 2;
    // head h of the group, of maximum M (log2 units) and sum L
    auto write_lse = [&](int b, int g, int h, float M, float L) {
        p.lse[(long long)b * p.nq + g * G + h] = (M + __log2f(L)) * 0.69314718055994531f;
    };
    // its element dd, O unnormalised
    auto write_out = [&](int b, int g, int h, int dd, float O, float M, float L) {
        store1(p.out, p.out_type, b * p.out_row + (g * G + h) * p.out_head + dd, O / L);
        if (p.lse && dd == 0) write_lse(b, g, h, M, L);
    };

    if (x < x1) {
        // scores are c S^T in log2 units, c > 0: a negative scale's sign is in
        // the queries, as is a zero scale
        const float c = p.scale == 0.f ? 1.f : fabsf(p.scale) * 1.4426950408889634f;
        const int first = x;
        At a = find(x), an, ann;
        int pg = load_pages(a), pgn = 0, pgnn = 0;
        bool more = x + 1 < x1;
        if (more) {
            an = next(a);
            pgn = load_pages(an);
        }
        {
            u32x4 raw[ST][QW];
            ask_q(a, raw);
            load_keys(a, pg);
            load_values(a, pg);
            take_q(raw);
        }
        bool bad = a.bad || (a.len > 0 && page_bad);
        float m = -INFINITY, l = 0.f;
        f32x4 o[EV];
#pragma unroll
        for (int i = 0; i < EV; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (;;) {
            const bool inside = tile_inside(a);
            const int key0 = (a.t0 + a.t) * NK;
            float s[NS][8];
            if (a.len > 0) {
#pragma unroll
                for (int sb = 0; sb < NS; ++sb) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
                        if constexpr (F8) {
                            const float ks = pow2_of((ksr[sb][t] >> (8 * (n & 3))) & 255u);
#pragma unroll
                            for (int e = 0; e < ST; ++e) {
                                u32x4 w;
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    const unsigned u = kr[sb][t][e / 2][2 * (e & 1) + i];
                                    w[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, ks, false));
                                    w[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, ks, true));
                                }
#pragma unroll
                                for (int i = QT - 1; i >= 0; --i)
                                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                        __builtin_bit_cast(bf16x8, w), q[i][e], acc, 0, 0, 0);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < ST; ++e)
#pragma unroll
                                for (int i = QT - 1; i >= 0; --i)
                                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                        __builtin_bit_cast(bf16x8, kr[sb][t][e]), q[i][e], acc, 0, 0, 0);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[sb][4 * t + i] = acc[i];
                    }
                }
            }
            if (more) {
                load_keys(an, pgn);
                if (x + 2 < x1) {
                    ann = next(an);
                    pgnn = load_pages(ann);
                }
            }
            if (a.len > 0) {
                if (!inside) {
#pragma unroll
                    for (int sb = 0; sb < NS; ++sb)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int key = key0 + 32 * sb + 8 * k4 + j;
                            const bool out = key < a.start || key >= a.len;
                            if (out) s[sb][j] = -INFINITY;
#pragma unroll
                            for (int i = 0; i < VW; ++i) vr[sb][j][i] = out ? 0u : vr[sb][j][i];
                        }
                }
                float mx = s[0][0];
#pragma unroll
                for (int sb = 0; sb < NS; ++sb)
#pragma unroll
                    for (int j = 0; j < 8; ++j) mx = fmaxf(mx, s[sb][j]);
                mx *= c;
                if (__any(mx > m + 8.f)) {
                    const float mn = fmaxf(m, max_16_32(mx));
                    const float al = __builtin_amdgcn_exp2f(m - mn);
                    l *= al;
#pragma unroll
                    for (int i = 0; i < EV; ++i) o[i] *= al;
                    m = mn;
                }
#pragma unroll
                for (int sb = 0; sb < NS; ++sb) {
                    float pr[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        pr[j] = __builtin_amdgcn_exp2f(fmaf(s[sb][j], c, -m));
                        l += pr[j];
                    }
                    if constexpr (F8) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float vs = pow2_of((vsr[sb][j / 4] >> (8 * (j & 3))) & 255u);
                            if (!inside && s[sb][j] == -INFINITY) vs = 0.f;
                            pr[j] *= vs;
                        }
                    }
                    bf16x8 pt[PT];
                    split_terms(pr, pt);
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        constexpr int EW = F8 ? 4 : 2;   // elements per word
                        u32x4 e[EW];   // element i of the word, positions in pairs
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const unsigned v0 = vr[sb][2 * j][w], v1 = vr[sb][2 * j + 1][w];
                            if constexpr (F8) {
                                const unsigned u0 = __builtin_amdgcn_perm(v1, v0, 0x05010400);
                                const unsigned u1 = __builtin_amdgcn_perm(v1, v0, 0x07030602);
                                e[0][j] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u0, 1.f, false));
                                e[1][j] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u0, 1.f, true));
                                e[2][j] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u1, 1.f, false));
                                e[3][j] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u1, 1.f, true));
                            } else {
                                e[0][j] = __builtin_amdgcn_perm(v1, v0, 0x05040100);
                                e[1][j] = __builtin_amdgcn_perm(v1, v0, 0x07060302);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < EW; ++i)
#pragma unroll
                            for (int t = PT - 1; t >= 0; --t)
                                o[EW * w + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                    __builtin_bit_cast(bf16x8, e[i]), pt[t], o[EW * w + i], 0, 0, 0);
                    }
                }
            }
            if (more) load_values(an, pgn);
            const bool ends = a.t + 1 == a.nt;
            if (ends || !more) {
                // the unit's first tile, in the row of all
                const int u0 = x - a.t;
                if (bad) {
                    l = __builtin_nanf("");
                    if (lane == 0) flag_error(p.error, a.bad ? KL_DEVERR_POSITION : KL_DEVERR_PAGE);
                }
                const float L = sum_16_32(l);
                // into LDS: a unit's part, or a whole unit on its way out (in
                // the place of the part that the wave may end with)
                const bool whole = ends && u0 >= first;
                const int slot = 2 * wave + (u0 >= first);
                float *const w = part + slot * G * WD;
                if (n < G) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < EV; ++e) w[n * WD + EV * (4 * k4 + i) + e] = o[e][i];
                    if (k4 == 0) {
                        w[n * WD + D] = m;
                        w[n * WD + D + 1] = a.len == 0 && !bad ? 1.f : L;
                    }
                }
                if (whole) {
                    __builtin_amdgcn_wave_barrier();   // (a wave's LDS accesses are in order)
                    for (int i = 8 * lane; i < G * D; i += 512) {
                        const int h = i / D, dd = i % D;
                        const float *const r = w + h * WD;
                        const float inv = 1.f / r[D + 1];
                        float v[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = r[dd + j] * inv;
                        store8(reinterpret_cast<uint8_t *>(p.out) +
                                   (a.b * p.out_row + (a.g * G + h) * p.out_head + dd) * out_bytes,
                               p.out_type, p.out_vec, v);
                        if (p.lse && dd == 0) write_lse(a.b, a.g, h, r[D], r[D + 1]);
                    }
                } else if (lane == 0) {
                    unit[slot] = a.b * nkv + a.g;
                    ubeg[slot] = u0;
                    uend[slot] = u0 + a.nt;
                }
                if (!more) break;
                m = -INFINITY;
                l = 0.f;
                bad = false;
#pragma unroll
                for (int i = 0; i < EV; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (an.len > 0) {
                    u32x4 raw[ST][QW];
                    ask_q(an, raw);
                    take_q(raw);
                }
            }
            ++x;
            a = an;
            pg = pgn;
            bad = bad || a.bad || (a.len > 0 && page_bad);
            an = ann;
            pgn = pgnn;
            more = x + 1 < x1;
        }
    }
    __syncthreads();

    // join the parts in LDS, run by run of one unit's (lane i: part i)
    // units handed on and their workgroups: one that began earlier, one that goes on
    int sent0 = -1, sent1 = -1, count0 = 0, count1 = 0;
    const int own_unit = lane < NE ? unit[lane] : -1;
    unsigned left = (unsigned)__ballot(own_unit >= 0);
    while (left) {
        const int e = __builtin_ctz(left);
        const int u = __builtin_amdgcn_readlane(own_unit, e);
        const unsigned run = (unsigned)__ballot(own_unit == u);
        left &= ~run;
        const int b0 = __builtin_amdgcn_readfirstlane(ubeg[e]);
        const int b1 = __builtin_amdgcn_readfirstlane(uend[e]);
        const bool whole = b0 >= X0 && b1 <= X1;
        const int z = b0 >= X0;
        if (!whole) {
            const int nw = sh.of(b1 - 1) - sh.of(b0) + 1;
            if (z) sent1 = u, count1 = nw;
            else sent0 = u, count0 = nw;
        }
        for (int i = tid; i < G * D; i += kAttnThreads) {
            const int h = i / D, dd = i % D;
            constexpr int NB = 8;   // parts read together (a run has 9 at most)
            float M = -INFINITY, L = 0.f, O = 0.f;
            for (unsigned r = run; r;) {
                int k[NB], nk = 0;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    k[j] = r ? __builtin_ctz(r) : e;
                    nk += r != 0;
                    r &= r - 1;
                }
                join_parts<NB>(nk, O, M, L, [&](int j, float &o, float &m, float &l) {
                    const float *w = part + (k[j] * G + h) * WD;
                    m = w[D];
                    l = w[D + 1];
                    o = w[dd];
                });
            }
            if (whole) {
                write_out(u / nkv, u % nkv, h, dd, O, M, L);
            } else {
                float *w = p.parts + ((size_t)(wg * 2 + z) * G + h) * WD;
                st_dev(w + dd, O);
                if (dd == 0) {
                    st_dev(w + D, M);
                    st_dev(w + D + 1, L);
                }
            }
        }
    }
    if (sent0 < 0 && sent1 < 0) return;

    // arrive with what was handed on; the last to arrive joins a unit's parts
    wait_stores();
    __syncthreads();
    if (tid < 2) {
        const int u = tid ? sent1 : sent0, nw = tid ? count1 : count0;
        int mine = 0;
        if (u >= 0)
            mine = __hip_atomic_fetch_add(p.arrived + u, 1u, __ATOMIC_RELAXED,
                                          __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(nw - 1);
        if (mine)
            __hip_atomic_store(p.arrived + u, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last[tid] = mine;
    }
    __syncthreads();
    for (int z = 0; z < 2; ++z) {
        if (!__builtin_amdgcn_readfirstlane(last[z])) continue;
        const int u = z ? sent1 : sent0, nw = z ? count1 : count0;
        const int b = u / nkv, g = u % nkv;
        const int f = sh.of(before(b) * nkv + g * (before(b + 1) - before(b)));
        for (int i = tid; i < G * D; i += kAttnThreads) {
            const int h = i / D, dd = i % D;
            constexpr int NB = 16;   // parts whose loads are issued together
            float M = -INFINITY, L = 0.f, O = 0.f;
            for (int k0 = 0; k0 < nw; k0 += NB)
                join_parts<NB>(nw - k0, O, M, L, [&](int j, float &o, float &m, float &l) {
                    const int k = min(k0 + j, nw - 1);
                    const float *w = p.parts + ((size_t)((f + k) * 2 + (k == 0)) * G + h) * WD;
                    m = ld_dev(w + D);
                    l = ld_dev(w + D + 1);
                    o = ld_dev(w + dd);
                });
            write_out(b, g, h, dd, O, M, L);
        }
    }
}

template <int D, bool F8, bool Full>
static hipError_t launch_attention(const AttnParams &p, hipStream_t stream) {
    const auto kernel = kl_paged_attention_kernel<D, F8, Full>;
    const int lds = 4 * (2 * kAttnWaves * (p.group * (D + 2) + 3) + kAttnWaves + 3 + p.t.batch + 1);
    // (more than the default 64 KiB: once per device)
    if (lds > 65536) {
        static std::atomic<unsigned long long> done{0};
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        const unsigned long long bit = 1ull << (dev & 63);
        if (!(done.load(std::memory_order_relaxed) & bit)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                    hipFuncAttributeMaxDynamicSharedMemorySize, kLdsMost);
            if (e != hipSuccess) return e;
            done.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    // at most a workgroup for every kAttnWaves tiles that the table has room for
    const long long tiles = (((long long)p.t.max_pages << p.c.page_log2) + paged_tile(D, F8 ? 1 : 2) - 1) /
                            paged_tile(D, F8 ? 1 : 2) * p.t.batch * p.c.nkv;
    // (or for every unit)
    const int grid = (int)std::min<long long>(
        std::max<long long>((tiles + kAttnWaves - 1) / kAttnWaves, (long long)p.t.batch * p.c.nkv),
        kPagedGroups);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kAttnThreads), lds, stream, p);
    return hipGetLastError();
}

hipError_t launch_paged_attention(const AttnParams &p, hipStream_t stream) {
    const bool full = p.q_type != KL_DTYPE_BF16 || p.out_type == KL_DTYPE_FP32;
    const int which = (p.c.d == 128 ? 4 : 0) + (p.c.e4m3 ? 2 : 0) + (full ? 1 : 0);
    switch (which) {
        case 0: return launch_attention<64, false, false>(p, stream);
        case 1: return launch_attention<64, false, true>(p, stream);
        case 2: return launch_attention<64, true, false>(p, stream);
        case 3: return launch_attention<64, true, true>(p, stream);
        case 4: return launch_attention<128, false, false>(p, stream);
        case 5: return launch_attention<128, false, true>(p, stream);
        case 6: return launch_attention<128, true, false>(p, stream);
        default: return launch_attention<128, true, true>(p, stream);
    }
}

}  // namespace kl
