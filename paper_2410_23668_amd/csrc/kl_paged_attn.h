// The paged cache's attention kernel (kl_paged_attention in include/kl.h),
// included by the translation units that instantiate it (kl_paged_d*.hip).
#pragma once

#include <algorithm>
#include <atomic>

#include "kl_paged_dev.h"
#include "kl_paged_shares.h"

namespace kl {

// out_h = sum_j p_j v_j / sum_j p_j, p_j = 2^(c (s_j - m) - 8), s_j = q_h . k_j,
// c = scale log2 e, m the largest s_j of the attended positions j, or up to 8 / c
// less.
//
// Split-K flash decoding over pages, bound by HBM: at 262144 positions of 8 KV
// heads 6.1 TB/s bf16, 5.6 e4m3 and, e4m3 at head dimension 64, 5.0 (a read stream:
// 6.8), and 6.4 TB/s for what is added to a long sequence; about 9 us stand
// before the first tile (three round trips: lengths, pages, rows) and behind the
// last (joins, two more).
//
// A unit is a (sequence, KV head); its attended positions are cut into tiles of
// 16 KiB of keys and values, and the tiles of all units, one unit after the
// other, are dealt in equal contiguous shares to the workgroups and within one
// to its eight waves, so that lengths of any kind load every wave alike (few
// units: kl_paged_shares.h).  A wave goes through its tiles with a running
// maximum and sum; a unit that lies inside its share it writes out, of a unit
// cut by the share's ends it leaves its part (m, sum, unnormalised output)
// in LDS.  The workgroup joins the parts there; what is part of a unit of several
// workgroups goes to the workspace, and the last of them to arrive (a counter
// per unit) joins all in workgroup order.
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
// A group of up to 8 or 4 heads has its columns 2 or 4 times (column n: head
// n % (16 / C), copy n / (16 / C)), which costs the products nothing: each copy
// goes on with its own 8 / C of the lane's 8 scores, so that the softmax's
// vector instructions are spent on a fourth of what 16 columns would need,
// and the copies' outputs are added at the unit's end.
// e4m3 rows become bf16 on the way, with their row's scale (exactly, but for
// multiples of 2^-135 and 2^-134 at scale bytes 1 and 2: bf16's are 2^-133).  In the
// probabilities the values' scales would take 1 % less time (64.2 us against 64.9,
// batch 32, 8 KV heads of 128), but a small one leaves their terms below bf16's
// range.
// Queries and probabilities are taken as bf16 terms that hold all their bits:
// bf16 queries are one, fp16 ones two, fp32 ones three, and so are probabilities,
// whatever the output's type: of two terms a weight would be off by up to 2^-17 of
// itself, and where values cancel a 16-bit output by many of its own half-steps
// (two take 1 % less time: 49.7 us against 50.2 at batch 48, 32 KV heads of 64,
// e4m3, fp16).  Softmax and sums are fp32; m moves only when a score is more than 8
// / c above it, so the loop has no cross-lane step and no weight is above 1.  It is
// taken from the scores before they are multiplied: c s - m would carry the
// rounding of a product, more than 8 where scores are above 2^27.

constexpr int kAttnWaves = 8;
constexpr int kAttnThreads = kAttnWaves * 64;

__device__ __forceinline__ void store1(void *p, int type, long long i, float x) {
    if (type == KL_DTYPE_FP32) reinterpret_cast<float *>(p)[i] = x;
    else reinterpret_cast<uint16_t *>(p)[i] = bits16(x, type);
}

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(unsigned, v);
}
// NT bf16 terms of 8 floats (x is left as what the terms do not hold), each cut
// off towards zero: three hold all 24 bits as rounded ones would, but none has the
// other sign or is larger than x, so that a product with a term overflows only
// where the one with x does, and to the same side.
template <int NT>
__device__ __forceinline__ void split_terms(float (&x)[8], bf16x8 (&t)[NT]) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = __builtin_amdgcn_perm(__float_as_uint(x[2 * j + 1]), __float_as_uint(x[2 * j]),
                                         0x07060302);
            if (i + 1 < NT) {
                x[2 * j] -= bf_lo(w[j]);
                x[2 * j + 1] -= bf_hi(w[j]);
            }
        }
        t[i] = __builtin_bit_cast(bf16x8, w);
    }
}

// m where no score has been seen: below every one, and finite, so that there is
// no difference of infinities.
constexpr float kNoScore = -3.402823466e38f;

// Two neighbouring outputs of a head, unnormalised, with their m and sum.
struct Joined { float o0 = 0.f, o1 = 0.f, m = kNoScore, l = 0.f; };
// Adds the first n (at most NB) of the parts that get(j, outputs, (m, sum))
// reads, all of them at once.
template <int NB, class Get>
__device__ __forceinline__ void join_parts(int n, float c, Joined &a, Get &&get) {
    f32x2 o[NB], ml[NB];
    float mn = a.m;
#pragma unroll
    for (int j = 0; j < NB; ++j) get(j, o[j], ml[j]);
#pragma unroll
    for (int j = 0; j < NB; ++j) mn = j < n ? fmaxf(mn, ml[j][0]) : mn;
    const float al = __builtin_amdgcn_exp2f((a.m - mn) * c);
    a.l *= al;
    a.o0 *= al;
    a.o1 *= al;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const float w = __builtin_amdgcn_exp2f((ml[j][0] - mn) * c);
        a.l = j < n ? fmaf(ml[j][1], w, a.l) : a.l;
        a.o0 = j < n ? fmaf(o[j][0], w, a.o0) : a.o0;
        a.o1 = j < n ? fmaf(o[j][1], w, a.o1) : a.o1;
    }
    a.m = mn;
}

// The i-th of 8 scale bytes.
__device__ __forceinline__ unsigned scale_byte(u32x2 w, int i) { return (w[i / 4] >> (8 * (i & 3))) & 255u; }

// Two of a word's four e4m3 codes (the upper two: Hi) as bf16, times a power of two.
template <bool Hi>
__device__ __forceinline__ unsigned fp8_to_bf16(unsigned w, float scale) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, Hi));
}

// op over the C columns (of 16) that a head has; every one of them gets it.
struct MaxOp { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct AddOp { __device__ float operator()(float a, float b) const { return a + b; } };
template <int C, class Op>
__device__ __forceinline__ float over_copies(float v, Op op) {
    if constexpr (C >= 2) v = op(v, dpp<0x128>(v));   // row_ror:8
    if constexpr (C >= 4) v = op(v, dpp<0x124>(v));   // row_ror:4
    return v;
}

// Floats of LDS for the waves' parts (and, at the end, for four floats a thread).
__host__ __device__ constexpr int attn_part_floats(int group, int d) {
    return 2 * kAttnWaves * group * (d + 2) > 4 * kAttnThreads ? 2 * kAttnWaves * group * (d + 2)
                                                               : 4 * kAttnThreads;
}

template <int D, bool F8, int QT, int C>
__global__ void __launch_bounds__(kAttnThreads, 2) kl_paged_attention_kernel(AttnParams p) {
    constexpr int ES = F8 ? 1 : 2;
    constexpr int NK = paged_tile(D, ES), NS = NK / 32;   // positions of a tile; blocks of 32
    constexpr int RB = D * ES;                  // bytes of a row
    constexpr int NC = RB / 64;                 // 16-byte loads of a key row per lane
    constexpr int EV = D / 16, VW = EV * ES / 4;   // value elements, words per lane and position
    constexpr int ST = D / 32;                  // steps of the first product
    constexpr int PT = 3;                       // terms of probabilities
    constexpr bool kIsBf16 = QT == 1;           // queries: bf16, fp16, fp32 in 1, 2, 3 terms
    constexpr int NV = 8 / C;                   // scores of a block that a lane goes on with
    constexpr int WD = D + 2;                   // floats of a part of one head
    constexpr int NE = 2 * kAttnWaves;          // parts in LDS

    const int G = p.group, nkv = p.c.nkv, B = p.t.batch;
    float *const part = reinterpret_cast<float *>(kl_smem);      // [NE][G][WD]
    int *const unit = reinterpret_cast<int *>(part + attn_part_floats(G, D));   // [NE]: unit, -1: none
    int *const wsum = unit + NE;                                 // [kAttnWaves]
    int *const last = wsum + kAttnWaves;                         // [2]
    int *const pre = last + 2;                                   // [B + 1] tiles of earlier sequences

    const int tid = threadIdx.x, lane = tid & 63, k4 = lane >> 4, n = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int head = n % (16 / C), copy = n / (16 / C);   // of this lane's column
    const int psl = p.c.page_log2, psm = (1 << psl) - 1;
    const long long cap = (long long)p.t.max_pages << psl;

    const auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    // the length of sequence b, -1 where it is out of range (tiles: as for 0)
    auto checked = [&](int len) { return len < 0 || (long long)len > cap ? -1 : len; };
    auto tiles_of = [&](int len) { return paged_tiles(max(len, 0), p.window, NK); };
    // Tiles of the sequences up to each: one per lane of every wave, where the
    // wave has lanes for all (no wait for the other waves: 1 us less), else in LDS.
    const bool few = B <= 64;
    if (lane < 2) unit[2 * wave + lane] = -1;   // (read behind a barrier)
    int len_own = 0, tiles_own = 0, upto = 0, T;
    auto wave_scan = [&](int v) {   // inclusive sum over the first B lanes
        for (int off = 1; off < 64 && off < B; off <<= 1) {
            const int o = from_lane(v, max(lane - off, 0));
            v += lane >= off ? o : 0;
        }
        return v;
    };
    if (few) {
        if (lane < B) len_own = checked(p.lengths[lane]);
        tiles_own = lane < B ? tiles_of(len_own) : 0;
        upto = wave_scan(tiles_own);
        T = __builtin_amdgcn_readlane(upto, B - 1) * nkv;
    } else {
        if (tid == 0) pre[0] = 0;
        int base = 0;
        for (int b0 = 0; b0 < B; b0 += kAttnThreads) {
            const int b = b0 + tid;
            const int s = wave_scan(b < B ? tiles_of(checked(p.lengths[b])) : 0);
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
        T = uni(base) * nkv;
    }
    // tiles (of one KV head) of the sequences before b
    auto before = [&](int b) {
        if (few) return b > 0 ? __builtin_amdgcn_readlane(upto, b - 1) : 0;
        return uni(pre[b]);
    };
    // (through the scalar cache: a vector load would have to be waited for
    // behind the tiles in flight)
    auto length_at = [&](int b) {
        if (few) return __builtin_amdgcn_readlane(len_own, b);
        return checked(reinterpret_cast<const KL_KARG int32_t *>(
            reinterpret_cast<uint64_t>(p.lengths))[b]);
    };
    // The workgroup's share [X0, X1): of one unit (unit_groups), or an equal
    // share, with a workgroup for every kAttnWaves tiles.  Units of several
    // workgroups: the one that the share begins inside of, and the one that
    // begins in the share and goes on behind it; their numbers of workgroups,
    // and the first one's first.
    const int wg = blockIdx.x, groups = gridDim.x;
    int X0 = 0, X1 = 0, sent0 = -1, sent1 = -1, from0 = 0, count0 = 0, count1 = 0;
    bool by_unit = false;
    if (few && B * nkv <= groups) {
        const int equal = uni(equal_rounds(T, groups, kAttnWaves));
        const int most = uni((int)wave_max((float)tiles_own));   // (exact where it matters: below 2^24)
        int own = 0, to = 0;   // workgroups of one unit of sequence 'lane'; up to it
        const auto fits = [&](int per) {
            own = unit_groups(tiles_own, per);
            to = wave_scan(own);
            return __builtin_amdgcn_readlane(to, B - 1) * nkv <= groups;
        };
        by_unit = half_shares(most, equal, kAttnWaves) && fits(kHalfShare);
        if (!by_unit) by_unit = fits(equal * kAttnWaves);
        if (by_unit) {
            if (wg >= __builtin_amdgcn_readlane(to, B - 1) * nkv) return;
            const int b = __popcll(__ballot(lane < B && to * nkv <= wg));
            const int n = __builtin_amdgcn_readlane(own, b), nt = __builtin_amdgcn_readlane(tiles_own, b);
            const int i = wg - (__builtin_amdgcn_readlane(to, b) - n) * nkv;
            const int g = n == 1 ? i : uni(i / n), j = i - g * n;
            X0 = before(b) * nkv + g * nt;
            X1 = X0 + nt;
            if (n > 1) {
                const Shares unit_sh(nt, n);
                X1 = uni(X0 + unit_sh.first(j + 1));
                X0 = uni(X0 + unit_sh.first(j));
            }
            if (j > 0) sent0 = b * nkv + g, from0 = wg - j, count0 = n;
            else if (n > 1) sent1 = b * nkv + g, count1 = n;
        }
    }
    Shares sh(1, 1);
    if (!by_unit) {
        sh = Shares(T, min(groups, (T + kAttnWaves - 1) / kAttnWaves));
        if (wg >= sh.np) return;
        X0 = uni(sh.first(wg));
        X1 = uni(sh.first(wg + 1));
    }
    int x = X0 + (((X1 - X0) * wave) / kAttnWaves);
    const int x1 = X0 + (((X1 - X0) * (wave + 1)) / kAttnWaves);

    // A place in the row of tiles.
    struct At {
        int b, g, t, nt;     // sequence, KV head, tile of the unit, its tiles
        int len, start;      // positions attended: [start, len); len -1: a bad length
        int t0;              // the unit's first tile, counted from position 0
    };
    auto enter = [&](At &a, int b) {
        a.b = b;
        a.nt = before(b + 1) - before(b);
        a.len = length_at(b);
        a.start = paged_start(a.len, p.window);
        a.t0 = paged_first_tile(max(a.len, 0), p.window, NK);
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
        a.g = uni(r / a.nt);
        a.t = r - a.g * a.nt;
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

    // Loads, non-temporal: 94 us where ordinary ones take 104 (batch 16, 8192
    // positions, 64 heads on 8 of 128, bf16), but for values of 64-byte rows: 51.8 us
    // against 53.3 (batch 48, 32 KV heads of 64, e4m3).
    //
    // Every tile is asked for in the same way, without branches (behind a branch
    // around loads the compiler has to wait for all that may be in flight): a
    // group of 8 positions without an attended one reads the nearest group that
    // has one, a sequence without positions page 0, and what is not attended is
    // masked when it is used.
    //
    // The pages of a tile: lane i has that of the tile's i-th group of 8 positions.
    auto nearest = [&](const At &a, int pos) { return max(min(max(pos, a.start), a.len - 1), 0); };
    auto ask_pages = [&](const At &a) {
        const int pos = nearest(a, (a.t0 + a.t) * NK + 8 * (lane % (NK / 8)));
        return p.t.pages[(long long)a.b * p.t.stride + (pos >> psl)];
    };
    u32x4 kr[NS][2][NC];
    unsigned vr[NS][8][VW];
    u32x2 ksr[NS], vsr[NS];
    typedef unsigned VWord __attribute__((ext_vector_type(VW)));
    bool page_bad = false;   // of the tile whose keys were asked for last
    // the first row of the group of positions at 'key', whose page lane 'from' of pages has
    auto group_row = [&](const At &a, int pages, int from, int key) {
        return (((long long)from_lane(pages, from) * nkv + a.g) << psl) +
               (nearest(a, key) & psm & ~7);
    };
    auto ask_keys = [&](const At &a, int &pages) {
        if (a.len <= 0) pages = 0;
        page_bad = __any((unsigned)pages >= (unsigned)p.c.n_pages);
        pages = (unsigned)pages < (unsigned)p.c.n_pages ? pages : 0;
        const int key0 = (a.t0 + a.t) * NK;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const long long r0 = group_row(a, pages, 4 * s + (n >> 2), key0 + 32 * s + 8 * (n >> 2));
            const uint8_t *src = p.c.k + (r0 + (n & 3)) * RB + 16 * k4;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int c = 0; c < NC; ++c) kr[s][t][c] = ld_stream_16B(src + 4 * t * RB + 64 * c);
            if constexpr (F8) ksr[s] = *reinterpret_cast<const u32x2 *>(p.c.ks + r0);
        }
    };
    auto ask_values = [&](const At &a, int pages) {
        const int key0 = (a.t0 + a.t) * NK;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const long long r0 = group_row(a, pages, 4 * s + k4, key0 + 32 * s + 8 * k4);
            const uint8_t *src = p.c.v + r0 * RB + n * (EV * ES);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // (two 64-byte rows share a cache line: the second load finds it)
                const VWord *at = reinterpret_cast<const VWord *>(src + j * RB);
                const VWord w = RB < 128 ? *at : __builtin_nontemporal_load(at);
#pragma unroll
                for (int i = 0; i < VW; ++i) vr[s][j][i] = w[i];
            }
            if constexpr (F8) vsr[s] = *reinterpret_cast<const u32x2 *>(p.c.vs + r0);
        }
    };

    // The queries of a unit as columns of the first product: asked for as they
    // are, and taken apart into terms when they are needed.
    constexpr int QW = QT < 3 ? 1 : 2;   // 16-byte words of 8 elements
    bf16x8 q[QT][ST];
    auto ask_q = [&](const At &a, u32x4 (&raw)[ST][QW]) {
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            const int d0 = F8 ? 64 * (s / 2) + 16 * k4 + 8 * (s & 1) : 32 * s + 8 * k4;
            // (columns past the group: head 0 again, masked below)
            const long long at = a.b * p.q_row + (a.g * G + (head < G ? head : 0)) * p.q_head + d0;
            if constexpr (QT == 3) {
                const float *f = reinterpret_cast<const float *>(p.q) + at;
                raw[s][0] = load_16B<false>(f, p.q_vec);
                raw[s][1] = load_16B<false>(f + 4, p.q_vec);
            } else {
                raw[s][0] = load_16B<false>(reinterpret_cast<const uint16_t *>(p.q) + at, p.q_vec);
            }
        }
    };
    const float sign = p.scale > 0.f ? 1.f : p.scale < 0.f ? -1.f : 0.f;
    auto take_q = [&](const u32x4 (&raw)[ST][QW]) {
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            if constexpr (!kIsBf16) {
                float v[8];
                words_to_f32(raw[s][0], raw[s][QW - 1], QT == 3 ? KL_DTYPE_FP32 : KL_DTYPE_FP16, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = head < G ? v[j] * sign : 0.f;
                bf16x8 t[QT];
                split_terms(v, t);
#pragma unroll
                for (int i = 0; i < QT; ++i) q[i][s] = t[i];
            } else {   // (bf16 queries are their own term)
                u32x4 w = raw[s][0];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = head < G && sign != 0.f ? w[i] ^ (sign < 0.f ? 0x80008000u : 0u) : 0u;
                q[0][s] = __builtin_bit_cast(bf16x8, w);
            }
        }
    };

    const int out_bytes = p.out_type == KL_DTYPE_FP32 ? 4 : 2;
    // scores are c S^T in log2 units, c > 0: a negative scale's sign is in the
    // queries, as is a zero scale
    const float abs_scale = p.scale == 0.f ? 1.f : fabsf(p.scale), c = abs_scale * 1.4426950408889634f;
    // head h of the group, of m M and sum L
    auto write_lse = [&](int b, int g, int h, float M, float L) {
        p.lse[(long long)b * p.nq + g * G + h] =
            fmaf(M, abs_scale, (8.f + __log2f(L)) * 0.69314718055994531f);
    };
    // its elements dd and dd + 1
    auto write_pair = [&](int b, int g, int h, int dd, const Joined &a) {
        const long long at = b * p.out_row + (g * G + h) * p.out_head + dd;
        const float inv = 1.f / a.l, x0 = a.o0 * inv, x1 = a.o1 * inv;
        if (p.out_type == KL_DTYPE_FP32 && p.out_vec) {
            *reinterpret_cast<f32x2 *>(reinterpret_cast<float *>(p.out) + at) = f32x2{x0, x1};
        } else if (p.out_vec) {
            *reinterpret_cast<unsigned *>(reinterpret_cast<uint16_t *>(p.out) + at) =
                bits16(x0, p.out_type) | ((unsigned)bits16(x1, p.out_type) << 16);
        } else {
            store1(p.out, p.out_type, at, x0);
            store1(p.out, p.out_type, at + 1, x1);
        }
        if (QT == 3 && p.out_lo) {
            store1(p.out_lo, KL_DTYPE_BF16, at, x0 - bf2f(f2bf(x0)));
            store1(p.out_lo, KL_DTYPE_BF16, at + 1, x1 - bf2f(f2bf(x1)));
        }
        if (p.lse && dd == 0) write_lse(b, g, h, a.m, a.l);
    };

    float m = kNoScore, l = 0.f;    // the column's m, this lane's share of its sum
    f32x4 o[EV];                    // O^T: element EV (4 k4 + i) + e of head n in o[e][i]
    auto clear = [&]() {
        m = kNoScore;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < EV; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    };

    // the scores of the tile in kr that this lane goes on with
    auto scores = [&](float (&s)[NS][NV]) {
#pragma unroll
        for (int sb = 0; sb < NS; ++sb) {
            f32x4 st[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
                float ks = 1.f;
                if constexpr (F8) ks = pow2_of((ksr[sb][t] >> (8 * (n & 3))) & 255u);
#pragma unroll
                for (int e = 0; e < ST; ++e) {
                    u32x4 w;
                    if constexpr (F8) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const unsigned u = kr[sb][t][e / 2][2 * (e & 1) + i];
                            w[2 * i] = fp8_to_bf16<false>(u, ks);
                            w[2 * i + 1] = fp8_to_bf16<true>(u, ks);
                        }
                    } else {
                        w = kr[sb][t][e];
                    }
#pragma unroll
                    for (int i = QT - 1; i >= 0; --i)
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w),
                                                                      q[i][e], acc, 0, 0, 0);
                }
                st[t] = acc;
            }
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if constexpr (C == 1) {
                    s[sb][v] = st[v / 4][v & 3];
                } else if constexpr (C == 2) {
                    s[sb][v] = copy ? st[1][v] : st[0][v];
                } else {
                    const float lo = copy & 1 ? st[0][v + 2] : st[0][v];
                    const float hi = copy & 1 ? st[1][v + 2] : st[1][v];
                    s[sb][v] = copy & 2 ? hi : lo;
                }
            }
        }
    };
    // tile a's share of m, l and o, from its scores and the values in vr
    auto weigh = [&](const At &a, float (&s)[NS][NV]) {
        const int key0 = (a.t0 + a.t) * NK;
        const bool inside = key0 >= a.start && key0 + NK <= a.len;
        if (!inside) {
            // what is masked may hold anything: its scores, values and scales go (of a
            // scale byte of 255 a zero code, too, would be NaN)
#pragma unroll
            for (int sb = 0; sb < NS; ++sb) {
                const int k0 = key0 + 32 * sb + 8 * k4;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int key = k0 + NV * copy + v;
                    if (key < a.start || key >= a.len) s[sb][v] = -INFINITY;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool out = k0 + j < a.start || k0 + j >= a.len;
#pragma unroll
                    for (int i = 0; i < VW; ++i) vr[sb][j][i] = out ? 0u : vr[sb][j][i];
                    if constexpr (F8) vsr[sb][j / 4] &= out ? ~(255u << (8 * (j & 3))) : ~0u;
                }
            }
        }
        float mx = s[0][0];
#pragma unroll
        for (int sb = 0; sb < NS; ++sb)
#pragma unroll
            for (int v = 0; v < NV; ++v) mx = fmaxf(mx, s[sb][v]);
        if (__any((mx - m) * c > 8.f)) {
            const float mn = fmaxf(m, over_copies<C>(max_16_32(mx), MaxOp()));
            const float al = __builtin_amdgcn_exp2f((m - mn) * c);
            l *= al;
#pragma unroll
            for (int i = 0; i < EV; ++i) o[i] *= al;
            m = mn;
        }
#pragma unroll
        for (int sb = 0; sb < NS; ++sb) {
            float pr[NV];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                pr[v] = __builtin_amdgcn_exp2f(fmaf(s[sb][v] - m, c, -8.f));
                l += pr[v];
            }
            // this lane's column has the weights of its own positions and
            // zeros for the other copies'
            bf16x8 pt[PT];
#pragma unroll
            for (int t = 0; t < PT; ++t) {
                u32x4 w;
                unsigned pk[NV / 2];
#pragma unroll
                for (int i = 0; i < NV / 2; ++i) {
                    pk[i] = pack_bf16(pr[2 * i], pr[2 * i + 1]);
                    if (t + 1 < PT) {
                        pr[2 * i] -= bf_lo(pk[i]);
                        pr[2 * i + 1] -= bf_hi(pk[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = C == 1 || copy == i / (NV / 2) ? pk[i % (NV / 2)] : 0u;
                pt[t] = __builtin_bit_cast(bf16x8, w);
            }
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                constexpr int EW = F8 ? 4 : 2;   // elements per word
                u32x4 e[EW];   // element i of the word, positions in pairs
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned v0 = vr[sb][2 * j][w], v1 = vr[sb][2 * j + 1][w];
                    if constexpr (F8) {
                        const float s0 = pow2_of(scale_byte(vsr[sb], 2 * j));
                        const float s1 = pow2_of(scale_byte(vsr[sb], 2 * j + 1));
                        const unsigned a0 = fp8_to_bf16<false>(v0, s0), a1 = fp8_to_bf16<true>(v0, s0);
                        const unsigned b0 = fp8_to_bf16<false>(v1, s1), b1 = fp8_to_bf16<true>(v1, s1);
                        e[0][j] = __builtin_amdgcn_perm(b0, a0, 0x05040100);
                        e[1][j] = __builtin_amdgcn_perm(b0, a0, 0x07060302);
                        e[2][j] = __builtin_amdgcn_perm(b1, a1, 0x05040100);
                        e[3][j] = __builtin_amdgcn_perm(b1, a1, 0x07060302);
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
    };

    auto find_shared = [&]() {   // (equal shares: sent0 and what goes with it)
        if (by_unit) return;
        const At h = find(X0), e = find(X1 - 1);
        const int hb = X0 - h.t, eb = X1 - 1 - e.t;
        if (h.t > 0) {
            sent0 = h.b * nkv + h.g;
            from0 = uni(sh.of(hb));
            count0 = uni(sh.of(hb + h.nt - 1)) - from0 + 1;
        }
        if (eb >= X0 && eb + e.nt > X1) {
            sent1 = e.b * nkv + e.g;
            count1 = uni(sh.of(eb + e.nt - 1)) - wg + 1;
        }
    };

    if (x < x1) {
        const int first = x;
        clear();
        At a = find(x);
        // The unit of tile a ends here, or the wave's share does: a unit that is
        // the wave's own goes out, of another the part is left in LDS.
        bool bad = false;
        auto flush = [&](bool ends, auto &&between) {
            const int u0 = x - a.t;   // the unit's first tile, in the row of all
            if (bad) {
                l = __builtin_nanf("");
                if (lane == 0) flag_error(p.error, a.len < 0 ? KL_DEVERR_POSITION : KL_DEVERR_PAGE);
            }
            float L = over_copies<C>(sum_16_32(l), AddOp());
            if constexpr (C > 1) {
#pragma unroll
                for (int e = 0; e < EV; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[e][i] = over_copies<C>(o[e][i], AddOp());
            }
            if (a.len == 0) {   // (nothing attended: what was computed is void)
                clear();
                m = -INFINITY;
                L = 1.f;
            }
            // into LDS: a unit's part, or a whole unit on its way out (in the
            // place of the part that the wave may end with)
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
                    w[n * WD + D + 1] = L;
                }
            }
            between();
            if (whole) {
                __builtin_amdgcn_wave_barrier();   // (a wave's LDS accesses are in order)
                for (int i = 8 * lane; i < G * D; i += 512) {
                    const int h = i / D, dd = i % D;
                    const float *const r = w + h * WD;
                    const float inv = 1.f / r[D + 1];
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = r[dd + j] * inv;
                    const long long at = a.b * p.out_row + (a.g * G + h) * p.out_head + dd;
                    store8(reinterpret_cast<uint8_t *>(p.out) + at * out_bytes, p.out_type,
                           p.out_vec, v);
                    if (QT == 3 && p.out_lo) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] -= bf2f(f2bf(v[j]));
                        store8(p.out_lo + at, KL_DTYPE_BF16, p.out_vec, v);
                    }
                    if (p.lse && dd == 0) write_lse(a.b, a.g, h, r[D], r[D + 1]);
                }
                __builtin_amdgcn_wave_barrier();
            } else if (lane == 0) {
                unit[slot] = a.b * nkv + a.g;
            }
        };
        int pg = ask_pages(a);
        At an = a;
        if (x + 1 < x1) an = next(a);
        int pgn = ask_pages(an);
        {
            u32x4 raw[ST][QW];
            ask_q(a, raw);
            ask_keys(a, pg);
            // (values behind keys, here as in the loop: what waits for keys then
            // need not wait for values)
            __builtin_amdgcn_sched_barrier(0);
            ask_values(a, pg);
            find_shared();   // (while the loads run)
            take_q(raw);
        }
        bad = a.len < 0 || page_bad;
        // While a tile is worked on the next one's loads run: its keys are asked
        // for once this one's are used, its values likewise, its pages a tile
        // earlier.
        for (; x + 1 < x1; ++x) {
            float s[NS][NV];
            scores(s);
            ask_keys(an, pgn);
            At ann = an;
            if (x + 2 < x1) ann = next(an);
            const int pgnn = ask_pages(ann);
            weigh(a, s);
            ask_values(an, pgn);
            if (a.t + 1 == a.nt) {
                u32x4 raw[ST][QW];
                ask_q(an, raw);
                // (taken before the results are stored: no later wait for loads
                // then waits for stores)
                flush(true, [&]() { take_q(raw); });
                clear();
                bad = false;
            }
            bad = bad || an.len < 0 || page_bad;
            a = an;
            an = ann;
            pgn = pgnn;
        }
        float s[NS][NV];
        scores(s);
        weigh(a, s);
        flush(a.t + 1 == a.nt, []() {});
    } else {
        find_shared();
    }
    __syncthreads();

    // join the parts in LDS, run by run of one unit's (lane i: part i), a pair of
    // outputs per thread; several runs at a time, of as many waves each
    const int pairs = G * D / 2;
    const int own_unit = lane < NE ? unit[lane] : -1;
    const auto for_runs = [&](auto &&f) {
        int k = 0;
        for (unsigned left = (unsigned)__ballot(own_unit >= 0); left; ++k) {
            const int u = __builtin_amdgcn_readlane(own_unit, __builtin_ctz(left));
            const unsigned run = (unsigned)__ballot(own_unit == u);
            left &= ~run;
            f(k, u, run);
        }
        return k;
    };
    const int runs = for_runs([](int, int, unsigned) {});
    const int team = runs >= 8 ? 1 : runs >= 4 ? 2 : runs >= 2 ? 4 : 8;   // waves per run
    for_runs([&](int k, int u, unsigned run) {
        if ((k & (kAttnWaves / team - 1)) != wave / team) return;
        const int e = __builtin_ctz(run), nr = __builtin_popcount(run);
        const bool whole = u != sent0 && u != sent1;
        for (int i = (wave & (team - 1)) * 64 + lane; i < pairs; i += team * 64) {
            const int h = i / (D / 2), dd = 2 * (i % (D / 2));
            Joined a;
            // (each wave has one part of a unit at most)
            unsigned r = run;
            join_parts<kAttnWaves>(nr, c, a, [&](int, f32x2 &o, f32x2 &ml) {
                const float *w = part + ((r ? __builtin_ctz(r) : e) * G + h) * WD;
                r &= r - 1;
                o = *reinterpret_cast<const f32x2 *>(w + dd);
                ml = *reinterpret_cast<const f32x2 *>(w + D);
            });
            if (whole) {
                write_pair(u / nkv, u % nkv, h, dd, a);
            } else {
                float *w = p.parts + ((size_t)(wg * 2 + (u == sent1)) * G + h) * WD;
                st_dev_f2(w + dd, a.o0, a.o1);
                if (dd == 0) st_dev_f2(w + D, a.m, a.l);
            }
        }
    });
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
    constexpr int NB = 16;   // parts whose loads are issued together
    for (int z = 0; z < 2; ++z) {
        if (!uni(last[z])) continue;
        const int u = z ? sent1 : sent0, nw = z ? count1 : count0, f = z ? wg : from0;
        // (where there are more parts, and a group's pairs leave threads over,
        // S times as many threads take every S-th part: a round trip less, for
        // an exchange in LDS)
        const int S = nw > NB ? max(1, min(uni(kAttnThreads / pairs), (nw + NB - 1) / NB)) : 1;
        const int sub = S > 1 ? tid / pairs : 0;
        for (int i0 = 0; i0 < pairs; i0 += kAttnThreads) {
            const int i = S > 1 ? tid - sub * pairs : i0 + tid;
            const int h = i / (D / 2), dd = 2 * (i % (D / 2));
            Joined a;
            if (sub < S && i < pairs) {
                for (int k0 = sub; k0 < nw; k0 += S * NB)
                    join_parts<NB>((nw - k0 + S - 1) / S, c, a, [&](int j, f32x2 &o, f32x2 &ml) {
                        const int k = min(k0 + j * S, nw - 1);
                        const float *w = p.parts + ((size_t)((f + k) * 2 + (k == 0)) * G + h) * WD;
                        o = ld_dev_f2(w + dd);
                        ml = ld_dev_f2(w + D);
                    });
            }
            if (S > 1) {
                f32x4 *const x = reinterpret_cast<f32x4 *>(part);
                x[tid] = f32x4{a.o0, a.o1, a.m, a.l};
                __syncthreads();
                if (sub == 0) {
                    for (int k = 1; k < min(S, nw); ++k)
                        join_parts<1>(1, c, a, [&](int, f32x2 &o, f32x2 &ml) {
                            const f32x4 v = x[tid + k * pairs];
                            o = f32x2{v[0], v[1]};
                            ml = f32x2{v[2], v[3]};
                        });
                }
                __syncthreads();
            }
            if (sub == 0 && i < pairs) write_pair(u / nkv, u % nkv, h, dd, a);
        }
    }
}

template <int D, bool F8, int QT, int C>
static hipError_t launch_attention(const AttnParams &p, hipStream_t stream) {
    const auto kernel = kl_paged_attention_kernel<D, F8, QT, C>;
    const int lds = 4 * (attn_part_floats(p.group, D) + 2 * kAttnWaves + kAttnWaves + 2 + p.t.batch + 1);
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
    // for as many tiles as the table has room for
    constexpr int NK = paged_tile(D, F8 ? 1 : 2);
    const long long most = (((long long)p.t.max_pages << p.c.page_log2) + NK - 1) / NK;
    const long long units = (long long)p.t.batch * p.c.nkv;
    const int grid = (int)std::min<long long>(wanted_groups(most, units, kAttnWaves), kPagedGroups);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kAttnThreads), lds, stream, p);
    return hipGetLastError();
}

// The instance for the pool's type, the queries' terms and the group's copies.
template <int D, bool F8, int QT>
static hipError_t launch_copies(const AttnParams &p, hipStream_t stream) {
    if (p.group <= 4) return launch_attention<D, F8, QT, 4>(p, stream);
    if (p.group <= 8) return launch_attention<D, F8, QT, 2>(p, stream);
    return launch_attention<D, F8, QT, 1>(p, stream);
}
template <int D, bool F8>
static hipError_t launch_terms(const AttnParams &p, hipStream_t stream) {
    if (p.q_type == KL_DTYPE_FP32) return launch_copies<D, F8, 3>(p, stream);
    return p.q_type == KL_DTYPE_FP16 ? launch_copies<D, F8, 2>(p, stream)
                                     : launch_copies<D, F8, 1>(p, stream);
}
template <int D>
static hipError_t launch_attention_for(const AttnParams &p, hipStream_t stream) {
    return p.c.e4m3 ? launch_terms<D, true>(p, stream) : launch_terms<D, false>(p, stream);
}

}  // namespace kl
