// New tokens' queries and keys rotated by their positions, keys and values written to the pages of their sequences (halo_paged_append).
//     (a, b) -> (a cos - b sin, b cos + a sin)
// Moves each element once and reads a token's angles once: bytes bound it, and with few tokens the launch and two round trips (position, page; then
// the store).  A workgroup takes a token, or some of its heads where there are few tokens.  A thread keeps one place in the head -- two
// pieces of eight elements that hold whole pairs -- and walks over the heads with it, so that its eight angles are read once.
#include "../../include/halo.h"

#include <cmath>

#include "kernels.hpp"
#include "paged_index.hpp"

namespace halo {

int check_paged_shape(const halo_paged_shape *s);

namespace {

constexpr int kAppendThreads = 256;

struct AppendArgs {
    const void *q, *k, *v;
    void *q_out, *k_pages, *v_pages;
    const int32_t *pos, *seq, *table;
    const float *rope;
    int64_t q_stride, k_stride, v_stride;
    PagePool pool;
    int n_heads, D, max_pages, n_seq, max_pos, rotary, pairs;
};

template <typename T>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a)
{
    const int token = blockIdx.x, places = a.D / 16, heads_at_once = kAppendThreads / places;
    const int place = threadIdx.x % places, first = threadIdx.x / places + blockIdx.y * heads_at_once;
    const int rows = (a.q ? a.n_heads : 0) + 2 * a.pool.n_kv, k_from = a.q ? a.n_heads : 0, v_from = k_from + a.pool.n_kv;
    if ((int)threadIdx.x >= heads_at_once * places) return;

    const int seq = a.seq ? a.seq[token] : token, pos = a.pos[token];
    int page = -1;
    if ((unsigned)seq < (unsigned)a.n_seq && (unsigned)pos < (unsigned)a.max_pos)
        page = a.table[(int64_t)seq * a.max_pages + (pos >> a.pool.page_shift)];
    const bool there = page_exists(a.pool, page);    // else padding

    // the two pieces of this place: a pair's elements face each other in them, or follow one another
    const bool turned = a.rope && place * 16 < a.rotary, facing = turned && !a.pairs;
    const int e0 = facing ? place * 8 : place * 16, e1 = facing ? place * 8 + a.rotary / 2 : place * 16 + 8;
    float cs[8], sn[8];
    if (turned && there) {
        const float *angles = a.rope + (int64_t)pos * a.rotary + place * 8;
        load8(angles, cs);
        load8(angles + a.rotary / 2, sn);
    }
    for (int row = first; row < rows; row += heads_at_once * gridDim.y) {
        const T *from;
        T *to;
        if (row < k_from) {
            from = static_cast<const T *>(a.q) + token * a.q_stride + row * a.D;
            to = static_cast<T *>(a.q_out) + ((int64_t)token * a.n_heads + row) * a.D;
        } else {
            const bool key = row < v_from;
            const int head = row - (key ? k_from : v_from);
            from = static_cast<const T *>(key ? a.k : a.v) + token * (key ? a.k_stride : a.v_stride) + head * a.D;
            if (!there) continue;
            to = static_cast<T *>(key ? a.k_pages : a.v_pages) + paged_row(a.pool, page, head, pos) * a.D;
        }
        Piece8<T> p0, p1;
        p0.load(from + e0);
        p1.load(from + e1);
        if (!there) {
            p0.zero();
            p1.zero();
        }
        float x[8], y[8];
        p0.get(x);
        p1.get(y);
        if (turned && there && row < v_from) {
            float u[8], w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // pair i of this place: (x[i], y[i]) facing, else elements 2i and 2i + 1 of x followed by y
                const float p = facing ? x[i] : i < 4 ? x[(2 * i) & 7] : y[(2 * i) & 7];
                const float q = facing ? y[i] : i < 4 ? x[(2 * i + 1) & 7] : y[(2 * i + 1) & 7];
                u[i] = p * cs[i] - q * sn[i];
                w[i] = q * cs[i] + p * sn[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = facing ? u[i] : i & 1 ? w[i / 2] : u[i / 2];
                y[i] = facing ? w[i] : i & 1 ? w[4 + i / 2] : u[4 + i / 2];
            }
        }
        store8(to + e0, x);
        store8(to + e1, y);
    }
}

}  // namespace
}  // namespace halo

extern "C" int halo_rope_table(int32_t n_pos, int32_t rotary_dim, double theta, float *table)
{
    if (!table) return HALO_ERR_NULL;
    if (n_pos < 0 || rotary_dim < 2 || rotary_dim % 2 || !(theta > 0.0) || !std::isfinite(theta)) return HALO_ERR_ARG;
    const int half = rotary_dim / 2;
    for (int i = 0; i < half; ++i) {
        const double step = std::pow(theta, -2.0 * i / rotary_dim);
        for (int32_t p = 0; p < n_pos; ++p) {
            const double angle = p * step;
            table[((size_t)p * 2) * half + i] = (float)std::cos(angle);
            table[((size_t)p * 2 + 1) * half + i] = (float)std::sin(angle);
        }
    }
    return HALO_OK;
}

extern "C" int halo_paged_append(const halo_paged_shape *shape, int32_t N, const void *q, int64_t q_stride, const void *k,
                                 int64_t k_stride, const void *v, int64_t v_stride, const int32_t *pos, const int32_t *seq,
                                 int32_t n_seq, const int32_t *page_table, const float *rope, int32_t rope_len, int32_t rotary_dim,
                                 int32_t rope_pairs, void *q_out, void *k_pages, void *v_pages, void *stream)
{
    using namespace halo;
    if (const int rc = check_paged_shape(shape)) return rc;
    if (!k || !v || !pos || !page_table || !k_pages || !v_pages || !q != !q_out) return HALO_ERR_NULL;
    const halo_paged_shape &s = *shape;
    const int size = s.dtype == HALO_F32 ? 4 : 2;
    auto odd = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; };
    auto bad_stride = [&](int64_t stride, int heads) { return stride < (int64_t)heads * s.head_dim || stride * size % 16; };
    if (N < 0 || n_seq < 1 || (q && (q == q_out || bad_stride(q_stride, s.n_heads))) || bad_stride(k_stride, s.n_kv_heads) ||
        bad_stride(v_stride, s.n_kv_heads))
        return HALO_ERR_ARG;
    if (odd(q) || odd(k) || odd(v) || odd(q_out) || odd(k_pages) || odd(v_pages) || odd(rope) ||
        ((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(seq) | reinterpret_cast<uintptr_t>(page_table)) & 3u))
        return HALO_ERR_ARG;
    if (rope && (rope_len < 1 || rotary_dim < 16 || rotary_dim % 16 || rotary_dim > s.head_dim)) return HALO_ERR_ARG;
    if (N == 0) return HALO_OK;

    AppendArgs a{};
    a.q = q; a.k = k; a.v = v; a.q_out = q_out; a.k_pages = k_pages; a.v_pages = v_pages;
    a.pos = pos; a.seq = seq; a.table = page_table; a.rope = rope;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.pool = PagePool{s.n_pages, s.n_kv_heads, __builtin_ctz((unsigned)s.page_size)};
    a.n_heads = s.n_heads; a.D = s.head_dim; a.max_pages = s.max_pages; a.n_seq = n_seq;
    a.max_pos = s.max_pages * s.page_size;
    if (rope && rope_len < a.max_pos) a.max_pos = rope_len;
    a.rotary = rope ? rotary_dim : 0;
    a.pairs = rope_pairs != 0;
    const int at_once = kAppendThreads / (s.head_dim / 16), rows = (q ? s.n_heads : 0) + 2 * s.n_kv_heads;
    const int parts = N < 512 ? (rows + at_once - 1) / at_once : 1;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (s.dtype == HALO_F32)
        append_kernel<float><<<dim3(N, parts), dim3(kAppendThreads), 0, st>>>(a);
    else
        append_kernel<bf16_t><<<dim3(N, parts), dim3(kAppendThreads), 0, st>>>(a);
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}
