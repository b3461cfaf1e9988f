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

// Walks every worker's share as the first launch does and every pair as the second does; both have to agree.
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
    std::map<std::pair<int, size_t>, int64_t> slots;             // (worker, pair) -> slot
    std::map<int64_t, int> used;
    std::vector<int> seen(tiles.size(), 0), whole(tiles.size(), 0);
    for (int w = 0; w < workers; ++w) {
        const int64_t from = (int64_t)w * per;
        if (from >= total) break;
        const int to = from + per < total ? (int)from + per : total;
        for (size_t i = 0; i < tiles.size(); ++i) {
            const int b = from > offset[i] ? (int)from : offset[i], e = to < offset[i] + tiles[i] ? to : offset[i] + tiles[i];
            if (b >= e) continue;
            seen[i] += e - b;
            if (e - b == tiles[i]) {
                whole[i] = 1;
                continue;
            }
            const int64_t s = partial_slot(w, per, offset[i]);
            if (s < 0 || s >= 2 * (int64_t)workers || used[s]++) return "slot";
            slots[{w, i}] = s;
        }
    }
    for (size_t i = 0; i < tiles.size(); ++i) {
        if (seen[i] != tiles[i]) return "cover";
        if (tiles[i] == 0) continue;
        const int w0 = first_worker(offset[i], per), w1 = last_worker(offset[i], tiles[i], per);
        if ((w0 == w1) != (whole[i] != 0)) return "whole";
        if (w0 == w1) continue;
        size_t mine = 0;
        for (const auto &kv : slots) mine += kv.first.second == i;
        if (mine != (size_t)(w1 - w0 + 1)) return "count";
        for (int w = w0; w <= w1; ++w)
            if (!slots.count({w, i}) || slots[{w, i}] != partial_slot(w, per, offset[i])) return "join";
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
