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
// workgroups in equal contiguous shares: workgroup i has [first(i), first(i + 1)).
KL_HD inline int share_first(int T, int np, int i) { return (int)((long long)T * i / np); }
// the workgroup that has tile x
KL_HD inline int share_of(int T, int np, int x) {
    return (int)((((long long)x + 1) * np - 1) / T);
}

}  // namespace kl
