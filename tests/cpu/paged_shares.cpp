// The shares of the paged attention (kl_paged_shares.h): every tile of every
// unit is worked on once, a wave leaves at most two parts, a unit's parts are
// where its last workgroup looks for them, and as many workgroups arrive at a
// unit's counter as its count says.
// Prints "paged shares OK" and exits 0, else prints the failures and exits 1.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <set>
#include <vector>

#include "kl_paged_shares.h"

using namespace kl;

namespace {

int g_fail = 0;
void check(bool ok, const char *what, long long a, long long b) {
    if (ok || ++g_fail > 20) return;
    std::fprintf(stderr, "FAIL: %s (%lld, %lld)\n", what, a, b);
}

constexpr int kWaves = 8;

// The kernel's walk for a batch, with 'grid' workgroups launched.
void walk(const std::vector<int> &lengths, int nkv, int window, int NK, int grid, bool may_by_unit) {
    const int B = (int)lengths.size();
    std::vector<int> nt, first_of;   // by unit
    int T = 0, most = 0;
    for (int b = 0; b < B; ++b)
        for (int g = 0; g < nkv; ++g) {
            const int n = paged_tiles(lengths[b], window, NK), t0 = paged_first_tile(lengths[b], window, NK);
            check(n >= 1, "a tile at least", lengths[b], window);
            // the tiles hold the attended positions, and each of them holds one
            const int lo = paged_start(lengths[b], window), hi = lengths[b];
            check((long long)t0 * NK <= lo && (hi == 0 || ((long long)t0 + n) * NK >= hi), "tiles cover", lo, hi);
            check(hi == 0 || (((long long)t0 + 1) * NK > lo && ((long long)t0 + n - 1) * NK < hi), "no empty tile", lo, hi);
            first_of.push_back(T);
            nt.push_back(n);
            T += n;
            if (n > most) most = n;
        }
    const int units = B * nkv, equal = equal_rounds(T, grid, kWaves);
    bool by_unit = false;
    std::vector<int> unit_wg, part_wg, groups_of(units);   // by workgroup; by unit
    const bool half = half_shares(most, equal, kWaves);
    for (int per = half ? kHalfShare : equal * kWaves; may_by_unit && units <= grid; per = equal * kWaves) {
        int need = 0;
        for (int u = 0; u < units; ++u) {
            need += groups_of[u] = unit_groups(nt[u], per);
            check(per != kHalfShare || groups_of[u] <= kHalfParts, "parts", u, groups_of[u]);
        }
        by_unit = need <= grid;
        if (!by_unit && per == kHalfShare) continue;
        if (by_unit)
            for (int u = 0; u < units; ++u)
                for (int j = 0; j < groups_of[u]; ++j) {
                    unit_wg.push_back(u);
                    part_wg.push_back(j);
                }
        break;
    }
    const int want = (T + kWaves - 1) / kWaves < grid ? (T + kWaves - 1) / kWaves : grid;
    const Shares sh(T, want);
    const int np = by_unit ? (int)unit_wg.size() : sh.np;
    check(np <= grid, "workgroups", np, grid);
    std::vector<int> unit_of(T);
    for (int u = 0; u < units; ++u)
        for (int i = 0; i < nt[u]; ++i) unit_of[first_of[u] + i] = u;

    std::vector<int> seen(T, 0);
    std::map<int, std::set<std::pair<int, int>>> parts;   // unit -> (workgroup, slot) in memory
    std::map<int, int> arrivals, counts, writes;          // unit -> ...
    std::vector<int> first_wg(units, -1);   // of units of several workgroups
    for (int wg = 0; wg < np; ++wg) {
        int X0 = 0, X1 = 0;
        int sent0 = -1, sent1 = -1, from0 = 0, count0 = 0, count1 = 0;
        if (by_unit) {
            const int u = unit_wg[wg], j = part_wg[wg], n = groups_of[u];
            const Shares s(nt[u], n);
            X0 = first_of[u] + s.first(j);
            X1 = first_of[u] + s.first(j + 1);
            if (j > 0) sent0 = u, from0 = wg - j, count0 = n;
            else if (n > 1) sent1 = u, count1 = n;
        } else {
            X0 = sh.first(wg), X1 = sh.first(wg + 1);
        }
        check(X1 > X0, "a share", wg, np);
        if (!by_unit) {
            const int hu = unit_of[X0], eu = unit_of[X1 - 1];
            const int hb = first_of[hu], eb = first_of[eu];
            if (X0 > hb) {
                sent0 = hu;
                from0 = sh.of(hb);
                count0 = sh.of(hb + nt[hu] - 1) - from0 + 1;
            }
            if (eb >= X0 && eb + nt[eu] > X1) {
                sent1 = eu;
                count1 = sh.of(eb + nt[eu] - 1) - wg + 1;
            }
            check(sent0 < 0 || sent0 != sent1, "two units", sent0, sent1);
            for (int x = X0; x < X1; ++x) check(sh.of(x) == wg, "of", x, wg);
        }
        std::set<int> in_lds;
        for (int w = 0; w < kWaves; ++w) {
            const int x0 = X0 + (X1 - X0) * w / kWaves, x1 = X0 + (X1 - X0) * (w + 1) / kWaves;
            std::map<int, int> slot;   // LDS slot -> unit
            for (int x = x0; x < x1; ++x) {
                ++seen[x];
                const int u = unit_of[x], u0 = first_of[u];
                const bool ends = x + 1 == u0 + nt[u];
                if (!ends && x + 1 < x1) continue;
                if (ends && u0 >= x0) {
                    ++writes[u];
                } else {
                    const int k = u0 >= x0;
                    check(!slot.count(k), "an LDS slot twice", x, k);
                    slot[k] = u;
                    in_lds.insert(u);
                }
            }
        }
        for (int u : in_lds) {
            if (u != sent0 && u != sent1) {
                ++writes[u];
                check(first_of[u] >= X0 && first_of[u] + nt[u] <= X1, "a whole unit", u, wg);
            } else {
                parts[u].insert({wg, u == sent1});
            }
        }
        if (sent1 >= 0) first_wg[sent1] = wg;
        if (sent0 >= 0) {
            check(in_lds.count(sent0), "the part of an earlier unit", wg, sent0);
            ++arrivals[sent0];
            const int had = counts.emplace(sent0, count0).first->second;
            check(had == count0, "the same count everywhere", had, count0);
            check(from0 == first_wg[sent0], "first workgroup", from0, wg);
        }
        if (sent1 >= 0) {
            check(in_lds.count(sent1), "the part of a unit that goes on", wg, sent1);
            ++arrivals[sent1];
            const int had = counts.emplace(sent1, count1).first->second;
            check(had == count1, "the same count everywhere", had, count1);
        }
    }
    for (int x = 0; x < T; ++x) check(seen[x] == 1, "a tile once", x, seen[x]);
    for (int u = 0; u < units; ++u) {
        check((writes.count(u) ? writes[u] : 0) + (arrivals.count(u) ? 1 : 0) == 1, "written once", u, 0);
        if (!arrivals.count(u)) continue;
        check(arrivals[u] == counts[u] && counts[u] > 1, "arrivals", arrivals[u], counts[u]);
        const int f = first_wg[u];
        for (int k = 0; k < counts[u]; ++k)
            check(parts[u].count({f + k, k == 0}) == 1, "a part where it is looked for", u, k);
        check((int)parts[u].size() == counts[u], "parts", (long long)parts[u].size(), counts[u]);
    }
}

}  // namespace

int main() {
    check(paged_tile(128, 2) == 32 && paged_tile(64, 2) == 64 && paged_tile(128, 1) == 64 &&
              paged_tile(64, 1) == 128, "tile", 0, 0);
    // (no 32-bit overflow at the longest sequences)
    check(paged_tiles(1 << 30, 0, 32) == 1 << 25 && paged_tiles((1 << 30) - 1, 1000, 128) >= 8, "long", 0, 0);
    for (int T : {1, 2, 7, 8, 9, 255, 256, 257, 2047, 100003, 1 << 30})
        for (int n : {1, 2, 3, 7, 128, 255, 256}) {
            if (n > T) continue;
            const Shares s(T, n);
            check(s.first(0) == 0 && s.first(n) == T, "ends", T, n);
            for (int i = 0; i < n; ++i) {
                const int a = s.first(i), b = s.first(i + 1);
                check(b > a && b - a <= T / n + 1, "share", T, i);
                check(s.of(a) == i && s.of(b - 1) == i, "of", T, i);
            }
        }
    check(wanted_groups(1, 7, 8) == 7 && wanted_groups(3, 8, 8) == 8 && wanted_groups(64, 1, 8) == 16 &&
              wanted_groups(65, 1, 8) == 16 && wanted_groups(1000, 2, 8) == 250, "launched", 0, 0);
    std::srand(7);
    const int grids[] = {1, 2, 5, 64, 256};
    for (int it = 0; it < 3000; ++it) {
        const int B = 1 + std::rand() % (it % 10 == 0 ? 90 : 7), nkv = 1 + std::rand() % 8;
        const int NK = 32 << (std::rand() % 3), window = std::rand() % 3 ? 0 : 1 + std::rand() % 300;
        const int top = it % 3 == 0 ? 20000 : it % 3 == 1 ? 700 : 60;
        std::vector<int> n(B);
        for (int &x : n) x = std::rand() % 6 ? std::rand() % (top + 1) : 0;
        walk(n, nkv, window, NK, grids[std::rand() % 5], B <= 64);
    }
    for (int n : {1, 31, 32, 33, 4095, 4096, 4097, 131072}) walk({n}, 8, 0, 32, 256, true);
    if (g_fail) return 1;
    std::puts("paged shares OK");
    return 0;
}
