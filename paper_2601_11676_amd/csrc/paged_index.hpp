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
// order; worker w (a wave) takes the tiles [w * per, (w + 1) * per) of it.  A pair whose tiles all fall to one worker is written out by it.
// Of any other pair every worker keeps a partial result, in slot 0 of the worker if the pair is the first in its share, in slot 1 if not
// (then it is the share's last): a worker never has more than these two.
HALO_HOST_DEVICE int tiles_per_worker(int total, int workers, int least)
{
    const int even = total / workers + (total % workers != 0);
    return even > least ? even : least;
}
HALO_HOST_DEVICE int first_worker(int offset, int per) { return offset / per; }
HALO_HOST_DEVICE int last_worker(int offset, int tiles, int per) { return (offset + tiles - 1) / per; }
// slot of worker w's partial result of the pair that begins at `offset`
HALO_HOST_DEVICE int64_t partial_slot(int w, int per, int offset) { return 2 * (int64_t)w + ((int64_t)w * per >= offset ? 0 : 1); }

}  // namespace halo
