// Shares of the paged attention's work: which tiles a sequence has, which of
// all tiles a workgroup and a wave take, and which workgroups share a unit.
// Shared by the device code and by the CPU test (compiled there with KL_HD
// defined empty).
#pragma once

#ifndef KL_HD
#define KL_HD __host__ __device__
#endif

namespace kl {

// A tile is 16 KiB of keys and values of one KV head: this many positions.
KL_HD constexpr int paged_tile(int d, int element_bytes) { return 8192 / (d * element_bytes); }

// First attended position of a sequence of 'len' positions.
KL_HD inline int paged_start(int len, int window) {
    return window > 0 && len > window ? len - window : 0;
}
// The first tile, and the number of tiles, of its attended positions (tiles
// start at multiples of NK positions); at least one tile, which is empty where
// there is no position.
KL_HD inline int paged_first_tile(int len, int window, int NK) {
    return paged_start(len, window) / NK;
}
KL_HD inline int paged_tiles(int len, int window, int NK) {
    const int n = (int)(((long long)len + NK - 1) / NK) - paged_first_tile(len, window, NK);
    return n > 1 ? n : 1;
}

// The tiles of all units (sequence, KV head), T in a row, are dealt to np
// workgroups in contiguous shares, equal but for one tile: the first T % np
// have one more.  Workgroup i has [first(i), first(i + 1)).  (In 32 bits: the
// 64-bit division of T i / np took 0.4 us at a kernel's start.)
struct Shares {
    int np, each, more;   // workgroups; tiles of a share; shares with one more
    KL_HD Shares(int T, int n) : np(n), each(T / n), more(T % n) {}
    KL_HD int first(int i) const { return each * i + (i < more ? i : more); }
    // the workgroup that has tile x
    KL_HD int of(int x) const {
        const int big = (each + 1) * more;
        return x < big ? x / (each + 1) : more + (x - big) / each;
    }
};

// Where it can be had at no cost, a workgroup has tiles of one unit only: each
// unit gets whole workgroups, as many as make shares of at most 'per' tiles.  A
// workgroup then hands on one part and not two, and a unit of one workgroup
// needs no part in memory at all, which is worth about 4 us.
//   per = equal rounds   the rounds (a tile for each of the workgroup's waves)
//                        that an equal share has, in tiles;
//   per = kHalfShare     half a round, where no unit fits into one workgroup
//                        anyway: twice the workgroups, and less for each to
//                        load and join, as long as a unit's parts are read in
//                        one go (kHalfParts of them).
// 32 heads on 8 of 128, bf16, one sequence, half rounds against whole: 1024
// positions 10.9 us against 12.3, 2048 11.6 against 12.5; 4096, 32 parts, 14.7
// against 13.6; shares of 2 tiles: 1024 11.2, 2048, 32 parts, 13.8.
constexpr int kHalfShare = 4, kHalfParts = 16;
KL_HD inline int equal_rounds(int T, int groups, int waves) {
    const int each = (T + groups - 1) / groups;
    return (each + waves - 1) / waves;
}
// workgroups of a unit of nt tiles (one round is the usual case, and a division
// takes 0.1 us)
KL_HD inline int unit_groups(int nt, int per) {
    return per == 8 ? (nt + 7) / 8 : (nt + per - 1) / per;
}
// whether half rounds are tried, for units of at most 'most' tiles
KL_HD inline bool half_shares(int most, int equal, int waves) {
    return most > equal * waves && most <= kHalfParts * kHalfShare;
}
// Workgroups to launch for units of up to 'most' tiles each: one for every
// round, one for every half round that may be taken, and one for every unit.
KL_HD inline long long wanted_groups(long long most, long long units, int waves) {
    const long long round = (most * units + waves - 1) / waves;
    const long long capped = most < kHalfParts * kHalfShare ? most : kHalfParts * kHalfShare;
    const long long half = (capped + kHalfShare - 1) / kHalfShare * units;
    return round > half ? round : half;   // (half >= units: most >= 1)
}

}  // namespace kl
