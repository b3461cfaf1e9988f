// New tokens' queries and keys normed head by head and rotated by their positions, keys and values written to the pages (halo_paged_append_norm), or as codes of
// eight bits with a scale for each row of a head (halo_paged_append_q8); what such rows stand for (halo_paged_read_q8).
//     n(z) = z / sqrt(mean(z^2) + eps) * w,  then  (a, b) -> (a cos - b sin, b cos + a sin)
//     s = max|x| / 127,  c = rint(x / s),  standing for s c
// Each element moves once and its row's sum or maximum is exchanged between the lanes that hold it; few tokens are a launch and two round trips (3.2 us, of codes 5.0).  A row of
// a head is 2^n neighbouring lanes of a wave, two pieces of 16 bytes each (a head of 80 leaves lanes idle).  Bytes bound the rows: 4099 tokens of 64 + 8 + 8 heads of 128, 170 MB, 35 us
// with the call's gap, 4.9 TB/s (a copy of 4 GiB reaches 4.7).  The codes are bound by their instructions: 3001 tokens of 120 heads, 154 MB, 51 us, the VALU issuing 78 % of it.
//
// A code is a decision: next to the border of two of them an error of the last bit moves the value by a whole step.  So what becomes a code is computed in double from
// the inputs on; rows that come as they are, values among them, are exact as floats; what does not become a code is computed in float, rounded once.
// (us, 3001 tokens as above with the read: all in double, with the compiler's roots and quotients, 86; queries in float and Newton's steps 79; results packed by one instruction 76; several tokens a workgroup, 99 to 105.)
#include "../../include/halo.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.hpp"
#include "paged_index.hpp"

namespace halo {

int check_paged_shape(const halo_paged_shape *s);

namespace {

constexpr int kThreads = 256;

struct NormAppendArgs {
    const void *q, *k, *v, *w_q, *w_k;
    void *q_out, *k_pages, *v_pages;                 // pages of rows, or of codes
    float *k_scales, *v_scales;
    const int32_t *pos, *seq, *table;
    const float *rope;
    int64_t q_stride, k_stride, v_stride;
    PagePool pool;
    int n_heads, D, max_pages, n_seq, max_pos, rotary, pairs, norm;
    int lanes, lanes_log;                            // of a row, a power of two
    float eps;
    int first;                                       // token of the launch's first workgroup
};

template <typename T> constexpr int kElems = 16 / (int)sizeof(T);

template <typename T, typename C>
__device__ __forceinline__ void load_piece(const T *p, C (&x)[kElems<T>])
{
    const u32x4 v = *reinterpret_cast<const u32x4 *>(p);
    if constexpr (sizeof(T) == 2) {
        float f[8];
        unpack8(v, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = f[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
    }
}

template <bool PASS, typename T, typename C>
__device__ __forceinline__ void store_piece(T *p, const C (&x)[kElems<T>])
{
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2)
            v[i] = __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)(float)x[2 * i], (__bf16)(float)x[2 * i + 1]});      // one instruction, to nearest even
        else
            v[i] = __float_as_uint((float)x[i]);
    }
    if constexpr (PASS)
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
    else
        *reinterpret_cast<u32x4 *>(p) = v;
}

__device__ __forceinline__ float over_row(float v, int lanes)
{
    if (lanes > 1) v = xor_add<1>(v);
    if (lanes > 2) v = xor_add<2>(v);
    if (lanes > 4) v = xor_add<4>(v);
    if (lanes > 8) v = xor_add<8>(v);
    if (lanes > 16) v = xor_add<16>(v);
    return v;
}
__device__ __forceinline__ double over_row(double v, int lanes)
{
    for (int d = 1; d < lanes; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
// 1 / sqrt(v) and 1 / v of a positive number: the hardware's estimates and two steps of Newton's method each, within a few units of 2^-53.  (sqrt and division by the compiler are some 50
// instructions each, and a lane has 16 elements.)
__device__ __forceinline__ float root_inverse(float v) { return 1.0f / sqrtf(v); }
__device__ __forceinline__ double root_inverse(double v)
{
    double r = __builtin_amdgcn_rsq(v);
    if (!(v > 1e-300 && v < 1e300)) return 1.0 / sqrt(v);            // 0, the ends of the numbers, NaN
#pragma unroll
    for (int i = 0; i < 2; ++i) r = r + r * 0.5 * __builtin_fma(-v * r, r, 1.0);
    return r;
}
__device__ __forceinline__ double inverse(double v)
{
    double r = __builtin_amdgcn_rcp(v);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = __builtin_fma(r, __builtin_fma(-v, r, 1.0), r);
    return r;
}
__device__ __forceinline__ float top_of_row(float v, int lanes)
{
    auto as_f = [](int i) { return __builtin_bit_cast(float, i); };
    auto other = [&](float f, auto ctrl) { return as_f(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, f), decltype(ctrl)::value, 0xf, 0xf, true)); };
    if (lanes > 1) v = fmaxf(v, other(v, std::integral_constant<int, 0xB1>{}));          // lane ^ 1, 2 (quad permutations), 4 (half a row's mirror, quads reversed), 8
    if (lanes > 2) v = fmaxf(v, other(v, std::integral_constant<int, 0x4E>{}));
    if (lanes > 4) v = fmaxf(v, other(other(v, std::integral_constant<int, 0x141>{}), std::integral_constant<int, 0x1B>{}));
    if (lanes > 8) v = fmaxf(v, other(v, std::integral_constant<int, 0x128>{}));
    if (lanes > 16) v = fmaxf(v, __shfl_xor(v, 16));
    return v;
}
__device__ __forceinline__ double top_of_row(double v, int lanes)
{
    for (int d = 1; d < lanes; d <<= 1) v = fmax(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ float nearest(float v) { return rintf(v); }
__device__ __forceinline__ double nearest(double v) { return rint(v); }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ float size(float v) { return fabsf(v); }
__device__ __forceinline__ double size(double v) { return fabs(v); }

// A head's row in registers: pieces at elements e0 and e1 of lane `place`, normed and turned.
template <typename T, typename C>
struct HeadRow {
    static constexpr int E = kElems<T>;
    C x[E], y[E];

    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = y[i] = (C)0;
    }
    __device__ __forceinline__ void load(const T *row, int e0, int e1)
    {
        load_piece(row + e0, x);
        load_piece(row + e1, y);
    }
    __device__ __forceinline__ void norm(const NormAppendArgs &a, const T *w, int e0, int e1, bool in)
    {
        C sum = (C)0;
#pragma unroll
        for (int i = 0; i < E; ++i) sum += x[i] * x[i] + y[i] * y[i];
        const C by = root_inverse(over_row(sum, a.lanes) * ((C)1 / (C)a.D) + (C)a.eps);
        C u[E], v[E];
#pragma unroll
        for (int i = 0; i < E; ++i) u[i] = v[i] = (C)1;
        if (w && in) {
            load_piece(w + e0, u);
            load_piece(w + e1, v);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            x[i] = x[i] * by * u[i];
            y[i] = y[i] * by * v[i];
        }
    }
    __device__ __forceinline__ void turn(const NormAppendArgs &a, int pos, int e0, int e1, bool faced)
    {
        if (a.pairs) {
            auto turn2 = [&](C (&z)[E], int e) {
                if (e >= a.rotary) return;
                const float *angles = a.rope + (int64_t)pos * a.rotary + e / 2;
#pragma unroll
                for (int i = 0; i < E; i += 2) {
                    const C cs = angles[i / 2], sn = angles[i / 2 + a.rotary / 2], p = z[i], r = z[i + 1];
                    z[i] = p * cs - r * sn;
                    z[i + 1] = r * cs + p * sn;
                }
            };
            turn2(x, e0);
            turn2(y, e1);
        } else if (faced) {
            const float *angles = a.rope + (int64_t)pos * a.rotary + e0;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const C cs = angles[i], sn = angles[i + a.rotary / 2], p = x[i], r = y[i];
                x[i] = p * cs - r * sn;
                y[i] = r * cs + p * sn;
            }
        }
    }
    // As codes.  A product with 127 / max says which, unless it lies so near the border of two that its error decides: within 2e-5 in float (two roundings of a number
    // up to 127, 127 * 2^-23) and 1e-6 in double.  A lane that has one of those takes quotients 127 x / max, rounded once: of rows that came as floats 127 x is exact, and of such
    // numbers no quotient that is no tie lies within 2^-35 of one, so that ties, and they alone, go to even.
    __device__ __forceinline__ void store_codes(int8_t *row, float *scale, int lanes, int e0, int e1, bool in, bool first) const
    {
        C top = (C)0, odd = (C)0;                    // 0 times an infinity or NaN is NaN
#pragma unroll
        for (int i = 0; i < E; ++i) {
            top = larger(top, larger(size(x[i]), size(y[i])));
            odd += x[i] * (C)0 + y[i] * (C)0;
        }
        top = top_of_row(odd == (C)0 ? top : (C)INFINITY, lanes);
        const bool number = top < (C)INFINITY, few = !(top >= (C)0x1p-100);      // few: a product could overflow
        const double step = (double)top * (1.0 / 127.0);
        const C by = few || !number ? (C)0 : (C)(127.0 * inverse((double)top)), border = sizeof(C) == 4 ? (C)(0.5 - 2e-5) : (C)(0.5 - 1e-6);
        C far = (C)0;
        uint32_t w[2][E / 4];
        auto put = [&](const C (&z)[E], uint32_t (&words)[E / 4]) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const C v = z[i] * by, c = nearest(v);
                far = larger(far, size(v - c));
                const uint32_t code = (uint32_t)(uint8_t)(int)c;
                words[i / 4] = i % 4 ? words[i / 4] | code << (8 * (i % 4)) : code;
            }
        };
        put(x, w[0]);
        put(y, w[1]);
        if (!number) {
#pragma unroll
            for (int i = 0; i < E / 4; ++i) w[0][i] = w[1][i] = 0;
        } else if ((far > border || few) && top > (C)0) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint32_t u = (uint32_t)(uint8_t)(int)rint(127.0 * x[i] / (double)top), v = (uint32_t)(uint8_t)(int)rint(127.0 * y[i] / (double)top);
                w[0][i / 4] = i % 4 ? w[0][i / 4] | u << (8 * (i % 4)) : u;
                w[1][i / 4] = i % 4 ? w[1][i / 4] | v << (8 * (i % 4)) : v;
            }
        }
        if (in) {
            if constexpr (E == 8) {
                *reinterpret_cast<uint2 *>(row + e0) = make_uint2(w[0][0], w[0][1]);
                *reinterpret_cast<uint2 *>(row + e1) = make_uint2(w[1][0], w[1][1]);
            } else {
                *reinterpret_cast<uint32_t *>(row + e0) = w[0][0];
                *reinterpret_cast<uint32_t *>(row + e1) = w[1][0];
            }
        }
        if (!first) return;
        float s = number ? (float)step : NAN;
        if (number && 127.0f * s == INFINITY) s = __uint_as_float(__float_as_uint(s) - 1);      // or the largest float would read back as infinity
        *scale = s;
    }
};

template <typename T, bool Q8, bool PASS>
__global__ __launch_bounds__(kThreads) void append_norm_kernel(NormAppendArgs a)
{
    constexpr int E = kElems<T>;
    const int token = a.first + blockIdx.x, places = a.D / (2 * E);
    const int place = threadIdx.x & (a.lanes - 1), row = (threadIdx.x >> a.lanes_log) + blockIdx.y * (kThreads >> a.lanes_log);
    const int k_from = a.q ? a.n_heads : 0, v_from = k_from + a.pool.n_kv, rows = v_from + a.pool.n_kv;
    const bool in = row < rows && place < places;    // the others stay for the exchanges

    const int seq = a.seq ? a.seq[token] : token, pos = a.pos[token];
    int page = -1;
    if ((unsigned)seq < (unsigned)a.n_seq && (unsigned)pos < (unsigned)a.max_pos)
        page = a.table[(int64_t)seq * a.max_pages + (pos >> a.pool.page_shift)];
    const bool there = page_exists(a.pool, page);    // else padding: the same for the whole workgroup

    // the two pieces of this place: with pairs that face each other, place p < rotary / (2 E) has p and the piece that faces it, the others share
    // the rest of the head like this; else, and for values, piece p of either half of the head
    const bool query = row < k_from, value = row >= v_from, facing = a.rope && !a.pairs && !value;
    const int from = facing ? a.rotary : 0, p = facing ? place - a.rotary / (2 * E) : place;
    const bool faced = facing && p < 0;
    const int e0 = faced ? place * E : from + p * E, e1 = faced ? e0 + a.rotary / 2 : e0 + (a.D - from) / 2;

    const int head = query ? row : row - (value ? v_from : k_from);
    T *q_out = static_cast<T *>(a.q_out) + ((int64_t)token * a.n_heads + head) * a.D;
    const T *source = query   ? static_cast<const T *>(a.q) + token * a.q_stride + head * a.D
                      : value ? static_cast<const T *>(a.v) + token * a.v_stride + head * a.D
                              : static_cast<const T *>(a.k) + token * a.k_stride + head * a.D;
    if (!there) {
        if (in && query) {
            HeadRow<T, float> zero;
            zero.zero();
            store_piece<false>(q_out + e0, zero.x);
            store_piece<false>(q_out + e1, zero.y);
        }
        return;
    }
    const int64_t cell = paged_row(a.pool, page, head, pos);
    auto compute = [&](auto &r, const T *w) {        // of a query or a key
        r.zero();
        if (in) r.load(source, e0, e1);
        if (a.norm) r.norm(a, w, e0, e1, in);
        if (a.rope && in) r.turn(a, pos, e0, e1, faced);
    };
    // all lanes of a row take the same way
    if (query || !Q8) {
        HeadRow<T, float> r;
        if (value) {
            r.zero();
            if (in) r.load(source, e0, e1);
        } else {
            compute(r, static_cast<const T *>(query ? a.w_q : a.w_k));
        }
        T *to = query ? q_out : static_cast<T *>(value ? a.v_pages : a.k_pages) + cell * a.D;
        if (in) {
            store_piece<PASS>(to + e0, r.x);
            store_piece<PASS>(to + e1, r.y);
        }
    } else {
        int8_t *to = static_cast<int8_t *>(value ? a.v_pages : a.k_pages) + cell * a.D;
        float *scale = (value ? a.v_scales : a.k_scales) + cell;
        if (value || (!a.norm && !a.rope)) {         // rows as they came, exact as floats
            HeadRow<T, float> r;
            r.zero();
            if (in) r.load(source, e0, e1);
            r.store_codes(to, scale, a.lanes, e0, e1, in, in && place == 0);
        } else {
            HeadRow<T, double> r;
            compute(r, static_cast<const T *>(a.w_k));
            r.store_codes(to, scale, a.lanes, e0, e1, in, in && place == 0);
        }
    }
}

struct ReadArgs {
    const int8_t *k_codes, *v_codes;
    const float *k_scales, *v_scales;
    const int32_t *pos, *seq, *table;
    void *k_out, *v_out;
    PagePool pool;
    int D, max_pages, n_seq, first;
    int lanes_log;                                   // 2^lanes_log neighbouring lanes have a row
};

template <typename T>
__global__ __launch_bounds__(kThreads) void read_q8_kernel(ReadArgs a)
{
    constexpr int E = kElems<T>;
    const int token = a.first + blockIdx.x, row = (threadIdx.x >> a.lanes_log) + blockIdx.y * (kThreads >> a.lanes_log);
    const int e = (threadIdx.x & ((1 << a.lanes_log) - 1)) * E;
    if (row >= 2 * a.pool.n_kv || e >= a.D) return;
    const bool value = row >= a.pool.n_kv;
    const int head = value ? row - a.pool.n_kv : row;
    const int seq = a.seq ? a.seq[token] : token, pos = a.pos[token];
    int page = -1;
    if ((unsigned)seq < (unsigned)a.n_seq && (unsigned)pos < (unsigned)(a.max_pages << a.pool.page_shift))
        page = a.table[(int64_t)seq * a.max_pages + (pos >> a.pool.page_shift)];
    const int64_t cell = paged_row(a.pool, page, head, pos);
    float x[E];
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = 0.0f;
    if (cell >= 0) {
        const float s = (value ? a.v_scales : a.k_scales)[cell];
        const int8_t *c = (value ? a.v_codes : a.k_codes) + cell * a.D + e;
        uint32_t w[E / 4];
#pragma unroll
        for (int i = 0; i < E / 4; ++i) w[i] = reinterpret_cast<const uint32_t *>(c)[i];
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = s * (float)(int8_t)(w[i / 4] >> (8 * (i % 4)));
    }
    store_piece<false>(static_cast<T *>(value ? a.v_out : a.k_out) + ((int64_t)token * a.pool.n_kv + head) * a.D + e, x);
}

bool off(const void *p, unsigned by) { return (reinterpret_cast<uintptr_t>(p) & (by - 1)) != 0; }

// tokens whose workgroups number less than 2^32 threads
constexpr int64_t kRun = 0xffffffffu / kThreads;

int append(const halo_paged_shape *shape, int32_t N, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
           const int32_t *pos, const int32_t *seq, int32_t n_seq, const int32_t *table, int32_t norm, const void *w_q, const void *w_k, float eps,
           const float *rope, int32_t rope_len, int32_t rotary_dim, int32_t rope_pairs, void *q_out, void *k_pages, float *k_scales, void *v_pages,
           float *v_scales, bool codes, void *stream)
{
    if (const int rc = check_paged_shape(shape)) return rc;
    if (N < 0) return HALO_ERR_ARG;
    if (N == 0) return HALO_OK;
    if (!k || !v || !pos || !table || !k_pages || !v_pages || !q != !q_out || (codes && (!k_scales || !v_scales))) return HALO_ERR_NULL;
    const halo_paged_shape &s = *shape;
    const int size = s.dtype == HALO_F32 ? 4 : 2;
    auto bad_stride = [&](int64_t stride, int heads) { return stride < (int64_t)heads * s.head_dim || stride * size % 16; };
    if (n_seq < 1 || (q && (q == q_out || bad_stride(q_stride, s.n_heads))) || bad_stride(k_stride, s.n_kv_heads) ||
        bad_stride(v_stride, s.n_kv_heads))
        return HALO_ERR_ARG;
    if (off(q, 16) || off(k, 16) || off(v, 16) || off(q_out, 16) || off(k_pages, 16) || off(v_pages, 16) || off(rope, 16) || off(pos, 4) ||
        off(seq, 4) || off(table, 4) || off(k_scales, 4) || off(v_scales, 4))
        return HALO_ERR_ARG;
    if (norm && (off(w_q, 16) || off(w_k, 16) || !(eps >= 0.0f) || !std::isfinite(eps))) return HALO_ERR_ARG;
    if (rope && (rope_len < 1 || rotary_dim < 16 || rotary_dim % 16 || rotary_dim > s.head_dim)) return HALO_ERR_ARG;

    NormAppendArgs a{};
    a.q = q; a.k = k; a.v = v; a.q_out = q_out; a.k_pages = k_pages; a.v_pages = v_pages; a.k_scales = k_scales; a.v_scales = v_scales;
    a.w_q = norm ? w_q : nullptr; a.w_k = norm ? w_k : nullptr; a.norm = norm != 0; a.eps = eps;
    a.pos = pos; a.seq = seq; a.table = table; a.rope = rope;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.pool = PagePool{s.n_pages, s.n_kv_heads, __builtin_ctz((unsigned)s.page_size)};
    a.n_heads = s.n_heads; a.D = s.head_dim; a.max_pages = s.max_pages; a.n_seq = n_seq;
    a.max_pos = s.max_pages * s.page_size;
    if (rope && rope_len < a.max_pos) a.max_pos = rope_len;
    a.rotary = rope ? rotary_dim : 0;
    a.pairs = rope_pairs != 0;
    a.lanes = 1;
    while (a.lanes * 32 < s.head_dim * size) a.lanes *= 2, ++a.lanes_log;
    const int at_once = kThreads / a.lanes, rows = (q ? s.n_heads : 0) + 2 * s.n_kv_heads;
    // stores with the non-temporal hint where they fill whole 64-byte parts of lines and are many, as in paged_append.hip
    const int faced = rope && !rope_pairs ? rotary_dim : 0;
    const bool runs = (faced / 2 * size | (s.head_dim - faced) / 2 * size | s.head_dim / 2 * size) % 64 == 0;
    const bool pass = runs && (int64_t)N * rows * s.head_dim * size >= (4 << 20);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    for (int64_t first = 0; first < N; first += kRun) {
        a.first = (int)first;
        const dim3 grid((unsigned)std::min(kRun, N - first), (rows + at_once - 1) / at_once), threads(kThreads);
        auto launch = [&](auto kernel) { kernel<<<grid, threads, 0, st>>>(a); };
        if (s.dtype == HALO_F32) {
            if (codes) launch(pass ? append_norm_kernel<float, true, true> : append_norm_kernel<float, true, false>);
            else launch(pass ? append_norm_kernel<float, false, true> : append_norm_kernel<float, false, false>);
        } else {
            if (codes) launch(pass ? append_norm_kernel<bf16_t, true, true> : append_norm_kernel<bf16_t, true, false>);
            else launch(pass ? append_norm_kernel<bf16_t, false, true> : append_norm_kernel<bf16_t, false, false>);
        }
    }
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}

}  // namespace
}  // namespace halo

extern "C" int halo_paged_append_norm(const halo_paged_shape *shape, int32_t N, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                                      const void *v, int64_t v_stride, const int32_t *pos, const int32_t *seq, int32_t n_seq,
                                      const int32_t *page_table, const void *w_q, const void *w_k, float eps, const float *rope, int32_t rope_len,
                                      int32_t rotary_dim, int32_t rope_pairs, void *q_out, void *k_pages, void *v_pages, void *stream)
{
    return halo::append(shape, N, q, q_stride, k, k_stride, v, v_stride, pos, seq, n_seq, page_table, 1, w_q, w_k, eps, rope, rope_len, rotary_dim, rope_pairs,
                        q_out, k_pages, nullptr, v_pages, nullptr, false, stream);
}

extern "C" int halo_paged_append_q8(const halo_paged_shape *shape, int32_t N, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                                    const void *v, int64_t v_stride, const int32_t *pos, const int32_t *seq, int32_t n_seq,
                                    const int32_t *page_table, int32_t qk_norm, const void *w_q, const void *w_k, float eps, const float *rope,
                                    int32_t rope_len, int32_t rotary_dim, int32_t rope_pairs, void *q_out, int8_t *k_codes, float *k_scales,
                                    int8_t *v_codes, float *v_scales, void *stream)
{
    return halo::append(shape, N, q, q_stride, k, k_stride, v, v_stride, pos, seq, n_seq, page_table, qk_norm, w_q, w_k, eps, rope, rope_len, rotary_dim,
                        rope_pairs, q_out, k_codes, k_scales, v_codes, v_scales, true, stream);
}

extern "C" int halo_paged_read_q8(const halo_paged_shape *shape, int32_t N, const int32_t *pos, const int32_t *seq, int32_t n_seq,
                                  const int32_t *page_table, const int8_t *k_codes, const float *k_scales, const int8_t *v_codes,
                                  const float *v_scales, void *k_out, void *v_out, void *stream)
{
    using namespace halo;
    if (const int rc = check_paged_shape(shape)) return rc;
    if (N < 0) return HALO_ERR_ARG;
    if (N == 0) return HALO_OK;
    if (!pos || !page_table || !k_codes || !k_scales || !v_codes || !v_scales || !k_out || !v_out) return HALO_ERR_NULL;
    if (n_seq < 1 || off(k_codes, 16) || off(v_codes, 16) || off(k_out, 16) || off(v_out, 16) || off(k_scales, 4) || off(v_scales, 4) || off(pos, 4) ||
        off(seq, 4) || off(page_table, 4))
        return HALO_ERR_ARG;
    const halo_paged_shape &s = *shape;
    ReadArgs a{};
    a.k_codes = k_codes; a.v_codes = v_codes; a.k_scales = k_scales; a.v_scales = v_scales;
    a.pos = pos; a.seq = seq; a.table = page_table; a.k_out = k_out; a.v_out = v_out;
    a.pool = PagePool{s.n_pages, s.n_kv_heads, __builtin_ctz((unsigned)s.page_size)};
    a.D = s.head_dim; a.max_pages = s.max_pages; a.n_seq = n_seq;
    while ((1 << a.lanes_log) * (s.dtype == HALO_F32 ? 4 : 8) < s.head_dim) ++a.lanes_log;
    const int at_once = kThreads >> a.lanes_log;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    for (int64_t first = 0; first < N; first += kRun) {
        a.first = (int)first;
        const dim3 grid((unsigned)std::min(kRun, N - first), (2 * s.n_kv_heads + at_once - 1) / at_once), threads(kThreads);
        if (s.dtype == HALO_F32) read_q8_kernel<float><<<grid, threads, 0, st>>>(a);
        else read_q8_kernel<bf16_t><<<grid, threads, 0, st>>>(a);
    }
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}
