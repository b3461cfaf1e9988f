// Host build of csrc/paged_index.hpp, driven by tests/test_paged_host.py: reads one request a line, answers one a line.
//   row n_pages n_kv shift page head pos           -> row
//   len len max_len                                 -> length
//   cut workers least n tiles_1 .. tiles_n          -> ok, or what is wrong with the cut of these pairs over the workers
#include <cstdio>
#include <cstring>
#include <map>
#include <vector>

#include "../paper_2601_11676_amd/csrc/paged_index.hpp"

using namespace halo;

// Walks every workgroup's shares as the first launch does and every pair as the second does; both have to agree.
static const char *check_cut(int workers, int least, const std::vector<int> &tiles)
{
    int total = 0;
    std::vector<int> offset;
    for (int n : tiles) {
        offset.push_back(total);
        total += n;
    }
    const int per = tiles_per_worker(total, workers, least);
    if (per < least || (int64_t)per * workers < total) return "share";
    std::map<int64_t, size_t> slots;                             // slot -> pair
    std::vector<int> seen(tiles.size(), 0), out(tiles.size(), 0);
    for (int team = 0; team * kTeam < workers; ++team) {
        int key[kTeam], got[kTeam];
        for (int i = 0; i < kTeam; ++i) {
            const int w = team * kTeam + i;
            key[i] = -1;
            const int64_t from = (int64_t)w * per;
            if (w >= workers || from >= total) continue;
            const int to = from + per < total ? (int)from + per : total;
            for (size_t p = 0; p < tiles.size(); ++p) {
                const int b = from > offset[p] ? (int)from : offset[p], e = to < offset[p] + tiles[p] ? to : offset[p] + tiles[p];
                if (b >= e) continue;
                seen[p] += e - b;
                if (e - b == tiles[p]) {
                    out[p]++;
                } else if (e < to) {                             // goes on
                    if (slots.count(2 * w)) return "slot";
                    slots[2 * w] = p;
                } else {
                    key[i] = (int)p;
                    got[i] = e - b;
                }
            }
        }
        for (int i = 0; i < kTeam; ++i) {
            if (key[i] < 0 || (i && key[i - 1] == key[i])) continue;
            int have = 0;
            for (int j = i; j < kTeam && key[j] == key[i]; ++j) have += got[j];
            if (have == tiles[key[i]]) {
                out[key[i]]++;
            } else {
                if (slots.count(2 * (team * kTeam + i) + 1)) return "slot";
                slots[2 * (team * kTeam + i) + 1] = key[i];
            }
        }
    }
    for (size_t p = 0; p < tiles.size(); ++p) {
        if (seen[p] != tiles[p]) return "cover";
        if (tiles[p] == 0) continue;
        const Cut c(offset[p], tiles[p], per, total);
        int mine = 0;
        for (const auto &s : slots) mine += s.second == p;
        if (out[p] != (c.whole || c.in_team)) return "out";
        if (out[p]) {
            if (mine) return "both";
            continue;
        }
        if (mine != c.parts()) return "count";
        for (int k = 0; k < c.parts(); ++k) {
            if (c.slot(k) >= 2 * (int64_t)workers || !slots.count(c.slot(k)) || slots[c.slot(k)] != p) return "join";
            if (k && c.slot(k) <= c.slot(k - 1)) return "order";
        }
    }
    return "ok";
}

int main()
{
    char what[8];
    while (std::scanf("%7s", what) == 1) {
        if (!std::strcmp(what, "row")) {
            int n, kv, shift, page, head, pos;
            if (std::scanf("%d %d %d %d %d %d", &n, &kv, &shift, &page, &head, &pos) != 6) return 1;
            std::printf("%lld\n", (long long)paged_row(PagePool{n, kv, shift}, page, head, pos));
        } else if (!std::strcmp(what, "len")) {
            int len, most;
            if (std::scanf("%d %d", &len, &most) != 2) return 1;
            std::printf("%d\n", paged_length(len, most));
        } else {
            int workers, least, n;
            if (std::scanf("%d %d %d", &workers, &least, &n) != 3) return 1;
            std::vector<int> tiles(n);
            for (int &t : tiles)
                if (std::scanf("%d", &t) != 1) return 1;
            std::printf("%s\n", check_cut(workers, least, tiles));
        }
    }
    return 0;
}
