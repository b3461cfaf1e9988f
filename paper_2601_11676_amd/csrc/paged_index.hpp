// Where a token of a sequence lies in a paged cache, and which wave attends over which tokens: integer arithmetic only, compiled
// for the kernels and, by tests/test_paged_host.py, for the host.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define HALO_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define HALO_HOST_DEVICE inline
#endif

namespace halo {

// A pool of pages is [n_pages][n_kv_heads][1 << page_shift][head_dim]: a head's tokens of one page are consecutive rows.
struct PagePool {
    int n_pages, n_kv, page_shift;
};

HALO_HOST_DEVICE bool page_exists(const PagePool &p, int page) { return (unsigned)page < (unsigned)p.n_pages; }

// Row of the token at position `pos` of a sequence whose page number pos >> page_shift is `page`; -1 if that page does not exist.
// 64 bits: a pool passes 2^31 elements, and may pass 2^31 rows.
HALO_HOST_DEVICE int64_t paged_row(const PagePool &p, int page, int head, int pos)
{
    if (!page_exists(p, page)) return -1;
    const int in_page = pos & ((1 << p.page_shift) - 1);
    return (((int64_t)page * p.n_kv + head) << p.page_shift) + in_page;
}

// What a length counts for: nothing below 0, no more than the caller's bound and the page table's row hold.
HALO_HOST_DEVICE int paged_length(int len, int max_len) { return len < 0 ? 0 : len < max_len ? len : max_len; }

// Split attention.  The tiles of all (sequence, unit) pairs that have work stand in one line, sequence by sequence, each pair's tiles in
// order; worker w (a wave) takes the tiles [w * per, (w + 1) * per) of it.  kTeam consecutive workers are a workgroup.  A pair whose tiles all
// fall to one worker is written out by it.  Of any other pair each worker has a part: its share ends inside the pair (or with it), or goes on after it.
// Parts of the first kind meet at the end of a workgroup, which joins those of one pair; if they are all of the pair, it is written out there.
// What is left is at most two partial results a worker: slot 2w + 1 for the joined ones, where w is the first of the workers joined, and
// slot 2w for a share that goes on.
constexpr int kTeam = 4;

HALO_HOST_DEVICE int tiles_per_worker(int total, int workers, int least)
{
    const int even = total / workers + (total % workers != 0);
    return even > least ? even : least;
}

// A pair's tiles [offset, offset + tiles), tiles > 0, of a line of `total` cut into shares of `per`.
struct Cut {
    int w0, w1;                                      // its first and last worker
    int last;                                        // the last one whose share ends inside it: w1 or w1 - 1
    bool whole, in_team;                             // all with one worker; all with workers of one workgroup that end inside it

    HALO_HOST_DEVICE Cut(int offset, int tiles, int per, int total)
    {
        const int end = offset + tiles;
        w0 = offset / per;
        w1 = (end - 1) / per;
        const int64_t share_end = (int64_t)(w1 + 1) * per;
        last = (share_end < total ? share_end : total) <= end ? w1 : w1 - 1;
        whole = w0 == w1;
        in_team = last == w1 && w0 / kTeam == w1 / kTeam;
    }
    // partial results of a pair that is neither whole nor in_team, in order
    HALO_HOST_DEVICE int parts() const { return last / kTeam - w0 / kTeam + 1 + (last < w1); }
    HALO_HOST_DEVICE int64_t slot(int part) const
    {
        const int team = w0 / kTeam + part;
        if (team > last / kTeam) return 2 * (int64_t)w1;
        return 2 * (int64_t)(part == 0 ? w0 : team * kTeam) + 1;
    }
};

}  // namespace halo
