// New tokens' queries and keys rotated by their positions, keys and values written to the pages of their sequences (halo_paged_append).
//     (a, b) -> (a cos - b sin, b cos + a sin)
// Moves each element once: bytes bound it, and with few tokens the launch and two round trips (position and page; then
// the rows).  A workgroup takes a token, or as many of its heads as have room in it; a thread takes two pieces of 16 bytes of a head that hold whole pairs,
// so that neighbouring threads' pieces are neighbours in memory, loaded and stored as runs of half a head.  (Two pieces of eight elements whatever their
// type, walking over the heads with a token's angles in registers, left holes between a float head's stores: 394 MB 100 us, now 68.)
// PASS: stores with the non-temporal hint, where they fill whole 64-byte parts of lines and are many: 208 MB 41 -> 36 us (5.8 TB/s, a copy of 8 GiB
// reaches 4.8), 112 MB of float 21.9 -> 18.3; runs of 80 bytes (heads of 80, bf16) 12.3 -> 15.5, so these do without it.
#include "../../include/halo.h"

#include <algorithm>
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
    int first;                                       // token of the launch's first workgroup
};

// 16 bytes of a head
template <typename T> struct Piece {
    static constexpr int kElems = 16 / sizeof(T);
    u32x4 v;
    __device__ __forceinline__ void get(float (&o)[kElems]) const
    {
        if constexpr (sizeof(T) == 2) {
            unpack8(v, o);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(v[i]);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[kElems])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2)
                v[i] = (uint32_t)f32_to_bf16(x[2 * i]) | ((uint32_t)f32_to_bf16(x[2 * i + 1]) << 16);
            else
                v[i] = __float_as_uint(x[i]);
        }
    }
};

template <typename T, bool PASS>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a)
{
    constexpr int E = Piece<T>::kElems;
    const int token = a.first + blockIdx.x, places = a.D / (2 * E), heads_at_once = kAppendThreads / places;
    const int place = threadIdx.x % places, row = threadIdx.x / places + blockIdx.y * heads_at_once;
    const int k_from = a.q ? a.n_heads : 0, v_from = k_from + a.pool.n_kv, rows = v_from + a.pool.n_kv;
    if ((int)threadIdx.x >= heads_at_once * places || row >= rows) return;

    const int seq = a.seq ? a.seq[token] : token, pos = a.pos[token];
    int page = -1;
    if ((unsigned)seq < (unsigned)a.n_seq && (unsigned)pos < (unsigned)a.max_pos)
        page = a.table[(int64_t)seq * a.max_pages + (pos >> a.pool.page_shift)];
    const bool there = page_exists(a.pool, page);    // else padding

    // The two pieces of this place.  Elements that face each other in their pairs: place p < rotary / (2 E) has p and the piece that faces it, the other places
    // share the rest of the head like this; else, and for values, piece p of either half of the head.
    const bool query = row < k_from, value = row >= v_from, facing = a.rope && !a.pairs && !value;
    const int from = facing ? a.rotary : 0, p = facing ? place - a.rotary / (2 * E) : place;
    const bool faced = facing && p < 0;
    const int e0 = faced ? place * E : from + p * E, e1 = faced ? e0 + a.rotary / 2 : e0 + (a.D - from) / 2;

    const T *row_in;
    T *row_out;
    if (query) {
        row_in = static_cast<const T *>(a.q) + token * a.q_stride + row * a.D;
        row_out = static_cast<T *>(a.q_out) + ((int64_t)token * a.n_heads + row) * a.D;
    } else {
        const int head = row - (value ? v_from : k_from);
        row_in = static_cast<const T *>(value ? a.v : a.k) + token * (value ? a.v_stride : a.k_stride) + head * a.D;
        if (!there) return;
        row_out = static_cast<T *>(value ? a.v_pages : a.k_pages) + paged_row(a.pool, page, head, pos) * a.D;
    }
    Piece<T> p0, p1;
    p0.v = *reinterpret_cast<const u32x4 *>(row_in + e0);
    p1.v = *reinterpret_cast<const u32x4 *>(row_in + e1);
    if (!there) {
        p0.v = p1.v = u32x4{0u, 0u, 0u, 0u};
    } else if (faced) {
        const float *angles = a.rope + (int64_t)pos * a.rotary + e0;
        float x[E], y[E], u[E], w[E];
        p0.get(x);
        p1.get(y);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float cs = angles[i], sn = angles[i + a.rotary / 2];
            u[i] = x[i] * cs - y[i] * sn;
            w[i] = y[i] * cs + x[i] * sn;
        }
        p0.set(u);
        p1.set(w);
    } else if (a.rope && a.pairs && !value) {
        auto turn = [&](Piece<T> &piece, int e) {
            if (e >= a.rotary) return;
            const float *angles = a.rope + (int64_t)pos * a.rotary + e / 2;
            float x[E], u[E];
            piece.get(x);
#pragma unroll
            for (int i = 0; i < E; i += 2) {
                const float cs = angles[i / 2], sn = angles[i / 2 + a.rotary / 2];
                u[i] = x[i] * cs - x[i + 1] * sn;
                u[i + 1] = x[i + 1] * cs + x[i] * sn;
            }
            piece.set(u);
        };
        turn(p0, e0);
        turn(p1, e1);
    }
    if constexpr (PASS) {
        __builtin_nontemporal_store(p0.v, reinterpret_cast<u32x4 *>(row_out + e0));
        __builtin_nontemporal_store(p1.v, reinterpret_cast<u32x4 *>(row_out + e1));
    } else {
        *reinterpret_cast<u32x4 *>(row_out + e0) = p0.v;
        *reinterpret_cast<u32x4 *>(row_out + e1) = p1.v;
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
    if (N < 0) return HALO_ERR_ARG;
    if (N == 0) return HALO_OK;
    if (!k || !v || !pos || !page_table || !k_pages || !v_pages || !q != !q_out) return HALO_ERR_NULL;
    const halo_paged_shape &s = *shape;
    const int size = s.dtype == HALO_F32 ? 4 : 2;
    auto odd = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; };
    auto bad_stride = [&](int64_t stride, int heads) { return stride < (int64_t)heads * s.head_dim || stride * size % 16; };
    if (n_seq < 1 || (q && (q == q_out || bad_stride(q_stride, s.n_heads))) || bad_stride(k_stride, s.n_kv_heads) ||
        bad_stride(v_stride, s.n_kv_heads))
        return HALO_ERR_ARG;
    if (odd(q) || odd(k) || odd(v) || odd(q_out) || odd(k_pages) || odd(v_pages) || odd(rope) ||
        ((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(seq) | reinterpret_cast<uintptr_t>(page_table)) & 3u))
        return HALO_ERR_ARG;
    if (rope && (rope_len < 1 || rotary_dim < 16 || rotary_dim % 16 || rotary_dim > s.head_dim)) return HALO_ERR_ARG;

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
    const int at_once = kAppendThreads / (s.head_dim * size / 32), rows = (q ? s.n_heads : 0) + 2 * s.n_kv_heads;
    const int faced = rope && !rope_pairs ? rotary_dim : 0;
    const bool runs = (faced / 2 * size | (s.head_dim - faced) / 2 * size | s.head_dim / 2 * size) % 64 == 0;
    const bool pass = runs && (int64_t)N * rows * s.head_dim * size >= (4 << 20);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    // one launch, of tokens whose workgroups number less than 2^32 threads; of more tokens one after the other
    constexpr int64_t kRun = 0xffffffffu / kAppendThreads;
    for (int64_t first = 0; first < N; first += kRun) {
        a.first = (int)first;
        const dim3 grid((unsigned)std::min(kRun, N - first), (rows + at_once - 1) / at_once), threads(kAppendThreads);
        if (s.dtype == HALO_F32) {
            if (pass) append_kernel<float, true><<<grid, threads, 0, st>>>(a);
            else append_kernel<float, false><<<grid, threads, 0, st>>>(a);
        } else {
            if (pass) append_kernel<bf16_t, true><<<grid, threads, 0, st>>>(a);
            else append_kernel<bf16_t, false><<<grid, threads, 0, st>>>(a);
        }
    }
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}
