// How the attention over a paged cache shares its work out, behind a C interface (test-only).
#include <algorithm>
#include <cstring>

#include "../paper_2609_14507_b200/csrc/paged.h"

using namespace ipkvi;

extern "C" {
int shim_paged_most_units(int capacity, int window, int first, int unit) { return int(paged_most_units(capacity, window, first, unit)); }
int shim_paged_cluster(int pairs, int most_units, int group, int ctas) { return paged_cluster(pairs, most_units, group, paged_sixteens(group), ctas); }
int shim_paged_group(int group, int* groups_per_kv, int* rows_per_part, int* sixteens) {
    *groups_per_kv = paged_groups_per_kv(group); *rows_per_part = paged_rows_per_part(group); *sixteens = paged_sixteens(group);
    return paged_rows(group);
}
// seen[t] for the slots 0 .. cap - 1, as the units show them; the number of units
int shim_paged_seen(int n, int window, int first, int unit, int cap, unsigned char* seen) {
    const PagedSeen s = paged_seen(n, window, first, unit);
    std::memset(seen, 0, size_t(cap));
    for (int j = 0; j < s.units; ++j)
        for (int t = s.unit(j) * unit; t < (s.unit(j) + 1) * unit; ++t)
            if (t < cap && s.sees(t)) ++seen[t];
    for (int a = 0; a < cap; a += 16) {
        int some = 0, all = 1;
        for (int t = a; t < a + 16; ++t) { some |= s.sees(t); all &= s.sees(t); }
        if (some != s.sees_any(a, a + 16) || all != s.sees_all(a, a + 16)) return -1;
    }
    return s.units;
}
// Plays a launch: parts as the CTAs take them, partials as the join finds them.  0: every unit once, every result once, every partial where it
// is looked for; else what is wrong.  *most: the most units that a CTA takes; *ways: the share.
int shim_paged_play(const int* n, int n_rows, int n_gh, int window, int first, int unit, int teams, int ctas, int* most, int* ways) {
    static int32_t units[kPagedRowsPerLaunch], cum[kPagedRowsPerLaunch + 1];
    static int32_t taken[1 << 16], owner[2 * 4096];
    int64_t all = 0, pairs = 0;
    for (int r = 0; r < n_rows; ++r) {
        units[r] = paged_seen(n[r], window, first, unit).units;
        all += units[r]; pairs += units[r] > 0 ? n_gh : 0;
    }
    PagedShare s{0, 0, 0};
    for (int i = 0; i < 32 && pairs <= ctas && s.share == 0; ++i) {
        const int share = paged_share_tried(int32_t(all * n_gh), 1.f / float(ctas), teams, i);
        int64_t parts = 0;
        for (int r = 0; r < n_rows; ++r) parts += (units[r] + share - 1) / share;
        if (parts * n_gh <= ctas) s.share = share;
    }
    if (s.share > 0 && !paged_share_wins(s.share, int32_t(all * n_gh), int32_t(pairs), 1.f / float(ctas))) s.share = 0;
    cum[0] = 0;
    for (int r = 0; r < n_rows; ++r) cum[r + 1] = cum[r] + paged_cost(units[r], s);
    if (s.share == 0) { s.cost = cum[n_rows] * n_gh; s.ctas = std::min(ctas, s.cost); }
    *ways = s.share; *most = 0;
    std::fill(owner, owner + 2 * ctas, -1);
    static int32_t results[1 << 14];
    std::fill(results, results + n_rows * n_gh, 0);
    int64_t base = 0;
    static int64_t at[kPagedRowsPerLaunch];
    for (int r = 0; r < n_rows; ++r) { at[r] = base; base += int64_t(units[r]) * n_gh; }
    if (base > int64_t(sizeof(taken) / 4)) return -1;
    std::fill(taken, taken + base, 0);
    for (int c = 0; c < ctas; ++c) {
        PagedParts parts{cum, n, s, n_rows, n_gh, window, first, unit, c, 0, 0};
        PagedPart x;
        int mine = 0;
        for (bool more = parts.begin(x); more; more = parts.next(x)) {
            if (x.row < 0 || x.row >= n_rows || x.gh < 0 || x.gh >= n_gh || x.u0 < 0 || x.u1 < x.u0 || x.u1 > units[x.row]) return 1;
            for (int t = x.u0; t < x.u1; ++t) ++taken[at[x.row] + int64_t(x.gh) * units[x.row] + t];
            mine += x.u1 - x.u0;
            if (x.u0 == x.u1) { if (x.whole) return 2; continue; }
            if (x.whole) { ++results[x.row * n_gh + x.gh]; continue; }
            if (x.place < 0 || x.place >= 2 * ctas || owner[x.place] != -1) return 3;
            owner[x.place] = x.row * n_gh + x.gh;
        }
        *most = std::max(*most, mine);
    }
    for (int64_t i = 0; i < base; ++i)
        if (taken[i] != 1) return 4;
    int used = 0;
    for (int r = 0; r < n_rows; ++r)
        for (int g = 0; g < n_gh; ++g) {
            const int32_t cost = cum[r + 1] - cum[r];
            if ((cost == 0) != (units[r] == 0)) return 5;
            if (cost == 0) continue;
            const PagedPartials of = paged_partials(s, cum[r], cost, n_gh, g);
            if (of.n < 1 || (of.n == 1) != (results[r * n_gh + g] == 1)) return 6;
            for (int i = 0; of.n > 1 && i < of.n; ++i, ++used)
                if (owner[2 * (of.c0 + i) + (i == 0 ? of.odd : 0)] != r * n_gh + g) return 7;
        }
    for (int i = 0; i < 2 * ctas; ++i) used -= owner[i] != -1;
    return used ? 8 : 0;
}
}
