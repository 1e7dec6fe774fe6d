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

// Where a workgroup can have a unit to itself, the parts need not meet in
// memory (about 4 us), for at most kUnitRounds more rounds of its waves than
// an equal share has (a round, a tile for each wave, is about 2 us).
constexpr int kUnitRounds = 2;
KL_HD inline bool unit_shares(int units, int groups, int most, int T, int waves) {
    const int np = (T + waves - 1) / waves < groups ? (T + waves - 1) / waves : groups;
    const int equal = ((T + np - 1) / np + waves - 1) / waves;
    return units <= groups && (most + waves - 1) / waves <= equal + kUnitRounds;
}

}  // namespace kl
