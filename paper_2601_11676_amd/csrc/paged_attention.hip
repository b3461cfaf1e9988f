// Attention of one new token of each of T sequences over a paged cache (halo_paged_attention):
//     o_h = sum_j p_j V_j,  p = softmax_j(scale q_h . K_j),  j < len
// one pass over the rows with the running maximum and sum of the softmax.  Bytes bound it: a cached element meets `group` queries,
// 4 * group / 2 operations a byte in bf16, where this card has about 200 to spare.
//
// A wave is the worker.  The queries of one cache head (up to 16, over large caches 32: a unit) are the columns of the matrix instruction, so that grouped heads
// share what is read; with one query a column of 16 is used, and the matrix cores still outrun the stream.
//   S^T = K Q^T      rows = tokens, columns = queries.  A lane (c = lane & 15, g = lane >> 4) wants pieces (16 bytes) of token c's row; loaded
//                    like that, an instruction touches 16 rows.  So whole rows are loaded, and pass through a part of LDS that is the wave's own.
//                    The result leaves the lane with query c's scores of the tokens 4g .. 4g+3 of each 16.
//   O^T += V^T P^T   the sum over tokens may take them in any order, so the operand P^T is what the lane already holds: its own
//                    scores' exponentials.  V^T then wants, in lane (c, g), those tokens' values of one dimension.  The lane loads
//                    whole 16-byte pieces of the same tokens' rows (piece c: coalesced) and pairs up halves of registers; the dimension
//                    that row c of instruction j stands for is c * VEC + j, which only the place of the results in memory has to know.
// Maximum and sum of a query then live in its column's lanes, as do its outputs: rescaling needs no exchange.
//
// How the work is cut: with short caches one workgroup takes a (sequence, unit) pair, its waves the tokens, joined in LDS (one launch).  Otherwise every wave of
// a grid that fills the card takes an even share of all tiles of all pairs (paged_index.hpp), whatever the lengths, and a second launch joins
// the pairs that were cut.
#include "paged_attention.hpp"

namespace halo {
namespace {

inline size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Queries of a unit: all of a cache head up to `most`; of more, as even parts as that gives.
inline int rows_of_unit(const halo_paged_shape &s, int most)
{
    const int group = s.n_heads / s.n_kv_heads, units = (group + most - 1) / most;
    return (group + units - 1) / units;
}
// The most there are for any call: with heads of up to 128 two times 16 (longer rows have no registers for it).
inline int most_rows(const halo_paged_shape &s) { return s.head_dim <= 128 ? 2 * kCols : kCols; }

// Bytes of a call's cache, as far as the host knows.
inline int64_t most_bytes(const halo_paged_shape &s, int T, int max_len, bool codes)
{
    return (int64_t)T * s.n_kv_heads * max_len * 2 * (codes ? s.head_dim + 4 : s.head_dim * (s.dtype == HALO_F32 ? 4 : 2));
}

struct PagedWorkspace {
    size_t plan = 0, stats = 0, part = 0, bytes = 0;
    PagedWorkspace(const halo_paged_shape &s, int T)
    {
        const size_t rows = rows_of_unit(s, most_rows(s));       // no call has more
        const size_t slots = 2 * (size_t)kMaxWorkers;
        stats = align256(((size_t)T + 2) * sizeof(int32_t));
        part = stats + align256(slots * rows * 2 * sizeof(float));
        bytes = part + align256(slots * rows * s.head_dim * sizeof(float));
    }
};

}  // namespace

int launch_attend_bf16(const AttendArgs &a, hipStream_t s) { return launch_dim<CoreBf16One>(a, s); }

int check_paged_shape(const halo_paged_shape *s)
{
    if (!s) return HALO_ERR_NULL;
    if (s->dtype != HALO_F32 && s->dtype != HALO_BF16) return HALO_ERR_DTYPE;
    if (s->n_kv_heads < 1 || s->n_heads < s->n_kv_heads || s->n_heads > 256 || s->n_heads % s->n_kv_heads) return HALO_ERR_SHAPE;
    if (s->head_dim < 16 || s->head_dim > 256 || s->head_dim % 16) return HALO_ERR_SHAPE;
    if (s->page_size < 16 || s->page_size > 4096 || (s->page_size & (s->page_size - 1))) return HALO_ERR_SHAPE;
    if (s->n_pages < 1 || s->max_pages < 1 || (int64_t)s->max_pages * s->page_size > (1 << 30)) return HALO_ERR_SHAPE;
    return HALO_OK;
}

}  // namespace halo

extern "C" size_t halo_paged_workspace_bytes(const halo_paged_shape *shape, int32_t T)
{
    using namespace halo;
    if (check_paged_shape(shape) != HALO_OK || T < 0 || T > kMaxSeqs) return 0;
    return PagedWorkspace(*shape, T).bytes;
}

namespace halo {
namespace {

int attend(const halo_paged_shape *shape, int32_t T, const void *q, int64_t q_stride, const void *k, const float *k_scale, const void *v, const float *v_scale,
           bool codes, const int32_t *page_table, const int32_t *lens, int32_t max_len, const uint8_t *mask, float scale, void *out, void *workspace,
           size_t ws_bytes, void *stream)
{
    if (const int rc = check_paged_shape(shape)) return rc;
    if (T < 0 || T > kMaxSeqs) return HALO_ERR_ARG;
    if (T == 0) return HALO_OK;
    if (!q || !k || !v || !page_table || !lens || !out || (codes && (!k_scale || !v_scale))) return HALO_ERR_NULL;
    const halo_paged_shape &s = *shape;
    const int size = s.dtype == HALO_F32 ? 4 : 2;
    auto odd = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; };
    if (max_len < 1 || max_len > s.max_pages * s.page_size || !std::isfinite(scale)) return HALO_ERR_ARG;
    if (q_stride < (int64_t)s.n_heads * s.head_dim || q_stride * size % 16 || odd(q) || odd(k) || odd(v) || odd(out) ||
        odd(workspace) || (reinterpret_cast<uintptr_t>(page_table) & 3u) || (reinterpret_cast<uintptr_t>(lens) & 3u) ||
        ((reinterpret_cast<uintptr_t>(k_scale) | reinterpret_cast<uintptr_t>(v_scale)) & 3u))
        return HALO_ERR_ARG;
    const PagedWorkspace ws(s, T);
    if (!workspace || ws_bytes < ws.bytes) return HALO_ERR_WORKSPACE;

    AttendArgs a{};
    a.q = q; a.k = k; a.v = v; a.k_scale = k_scale; a.v_scale = v_scale; a.table = page_table; a.lens = lens; a.mask = mask; a.out = out;
    char *w = static_cast<char *>(workspace);
    a.plan = reinterpret_cast<int32_t *>(w + ws.plan);
    a.stats = reinterpret_cast<float *>(w + ws.stats);
    a.part = reinterpret_cast<float *>(w + ws.part);
    a.q_stride = q_stride;
    a.pool = PagePool{s.n_pages, s.n_kv_heads, __builtin_ctz((unsigned)s.page_size)};
    a.T = T; a.n_heads = s.n_heads; a.group = s.n_heads / s.n_kv_heads;
    a.bytes = most_bytes(s, T, max_len, codes);
    // More than 16 queries a cache head: 32 at once read the cache once, 16 at a time have more workgroups.  us, 32 / 16, lengths from half of the longest on: 16 sequences of up to
    // 8000, 8 cache heads with 20 queries (524 MB at the longest) 77 / 134; 30 of up to 5000, 2 with 20, heads of 96 (115 MB) 27.5 / 36.7; 8 of up to 700, 2 with 20 (6 MB)
    // 12.3 / 8.3.  Float, 8 cache heads with 20 queries: 24 of up to 5000 150 / 243; 4 of up to 4000 (131 MB) 31.8 / 40.6; 4 of up to 1000 (33 MB) 20.6 / 20.2; 1 of 1000
    // 18.8 / 14.4.
    a.rows = rows_of_unit(s, a.bytes > (64 << 20) && !(codes && s.dtype == HALO_F32) ? most_rows(s) : kCols);
    a.n_qt = (a.group + a.rows - 1) / a.rows;
    a.n_units = s.n_kv_heads * a.n_qt;
    a.D = s.head_dim; a.max_pages = s.max_pages; a.max_len = max_len;
    a.scale2 = scale * 1.44269504088896341f;
    if ((int64_t)((max_len + 15) / 16) * T * a.n_units > (1 << 30)) return HALO_ERR_ARG;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (codes) return s.dtype == HALO_F32 ? launch_attend_q8_f32(a, st) : a.rows <= kCols ? launch_attend_q8(a, st) : launch_attend_q8_32(a, st);
    if (s.dtype == HALO_BF16) return a.rows <= kCols ? launch_attend_bf16(a, st) : launch_attend_bf16_32(a, st);
    return a.rows <= 4 ? launch_attend_f32_4(a, st) : a.rows <= kCols ? launch_attend_f32(a, st) : launch_attend_f32_32(a, st);
}

}  // namespace
}  // namespace halo

extern "C" int halo_paged_attention(const halo_paged_shape *shape, int32_t T, const void *q, int64_t q_stride, const void *k_pages,
                                    const void *v_pages, const int32_t *page_table, const int32_t *lens, int32_t max_len,
                                    const uint8_t *mask, float scale, void *out, void *workspace, size_t ws_bytes, void *stream)
{
    return halo::attend(shape, T, q, q_stride, k_pages, nullptr, v_pages, nullptr, false, page_table, lens, max_len, mask, scale, out, workspace, ws_bytes,
                        stream);
}

extern "C" int halo_paged_attention_q8(const halo_paged_shape *shape, int32_t T, const void *q, int64_t q_stride, const int8_t *k_codes,
                                       const float *k_scales, const int8_t *v_codes, const float *v_scales, const int32_t *page_table,
                                       const int32_t *lens, int32_t max_len, const uint8_t *mask, float scale, void *out, void *workspace,
                                       size_t ws_bytes, void *stream)
{
    return halo::attend(shape, T, q, q_stride, k_codes, k_scales, v_codes, v_scales, true, page_table, lens, max_len, mask, scale, out, workspace, ws_bytes,
                        stream);
}
