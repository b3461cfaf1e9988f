// The kernels and launch rules of halo_paged_chunk_attention (paged_chunk.hip, where their mathematics stands), for the files that make them for one kind of
// cache each.
#pragma once
#include "../../include/halo.h"

#include <cmath>
#include <type_traits>

#include "kernels.hpp"
#include "paged_index.hpp"

namespace halo {

struct ChunkArgs {
    const void *q, *k, *v;
    const float *k_scale, *v_scale;                  // of a cache of codes
    const int32_t *starts, *table, *lens;
    const uint8_t *mask;
    void *out;
    float *part, *stats;                             // partial results of cut blocks: [slot][rows][D], [slot][rows][max, sum]
    int64_t q_stride;
    PagePool pool;
    int N, n_seq, n_heads, group, D, max_pages, max_len;
    int most;                                        // parts that a call may have, whatever its lengths (more: starts that go back)
    int slots;                                       // the same where blocks are cut: partial results that the workspace holds; else 0
    float scale2;                                    // scale * log2(e): the softmax is computed in powers of two
};

namespace {

constexpr int kCol = 32;                             // columns of the matrix instruction: rows of a block, that is queries
constexpr int kParts = 512;                          // parts that few blocks are cut into, about
constexpr int kLeast = 2;                            // tiles of a part at least
constexpr int kDies = 8;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// What a cache holds and how it goes to the matrix cores: an element as the sum of so many bf16 parts (three hold a float), of which products i * j
// with i + j < 3 are taken, what is left out is 2^-24 of a product.  kP: of a probability.
struct KindBf16 {
    typedef bf16_t Row, Cell;                        // queries and results; the cache
    static constexpr int kQ = 1, kC = 1, kP = 1;
    static constexpr bool kScaled = false, kCheckAll = false;
};
struct KindF32 {
    typedef float Row, Cell;
    static constexpr int kQ = 3, kC = 3, kP = 3;
    static constexpr bool kScaled = false, kCheckAll = true;
};
struct KindQ8 {
    typedef bf16_t Row;
    typedef int8_t Cell;
    static constexpr int kQ = 1, kC = 1, kP = 1;
    static constexpr bool kScaled = true, kCheckAll = false;
};
struct KindQ8F32 {
    typedef float Row;
    typedef int8_t Cell;
    static constexpr int kQ = 3, kC = 1, kP = 3;
    static constexpr bool kScaled = true, kCheckAll = false;
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// Eight floats as P bf16 parts each: a part is what the ones before leave, rounded.
template <int P>
__device__ __forceinline__ void parts_of(const float (&x)[8], u32x4 (&out)[P])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            out[p][i] = pack_bf16(a, b);
            if (p + 1 < P) {
                a -= bf16_lo(out[p][i]);
                b -= bf16_hi(out[p][i]);
            }
        }
    }
}

// Eight elements of the cache, as loaded; as bf16 parts.
template <typename Cell> struct Eight;
template <> struct Eight<bf16_t> {
    u32x4 v;
    __device__ __forceinline__ void load(const bf16_t *p) { v = *reinterpret_cast<const u32x4 *>(p); }
    __device__ __forceinline__ void zero() { v = u32x4{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ void parts(u32x4 (&out)[1]) const { out[0] = v; }
    // those that are no finite numbers become 0; whether there were any
    __device__ __forceinline__ bool mend()
    {
        bool any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool lo = (v[i] & 0x7f80u) == 0x7f80u, hi = (v[i] & 0x7f800000u) == 0x7f800000u;
            any = any || lo || hi;
            v[i] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
        }
        return any;
    }
};
template <> struct Eight<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float *p)
    {
        a = *reinterpret_cast<const f32x4 *>(p);
        b = *reinterpret_cast<const f32x4 *>(p + 4);
    }
    __device__ __forceinline__ void zero() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ void parts(u32x4 (&out)[3]) const
    {
        const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        parts_of<3>(x, out);
    }
    __device__ __forceinline__ bool mend()
    {
        bool any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // the largest floats, which round to infinity as bf16, count with the infinities: they are added as they are too
            const bool x = !(fabsf(a[i]) < 0x1.fep127f), y = !(fabsf(b[i]) < 0x1.fep127f);
            any = any || x || y;
            a[i] = x ? 0.0f : a[i];
            b[i] = y ? 0.0f : b[i];
        }
        return any;
    }
};
template <> struct Eight<int8_t> {
    u32x2 v;
    __device__ __forceinline__ void load(const int8_t *p) { v = *reinterpret_cast<const u32x2 *>(p); }
    __device__ __forceinline__ void zero() { v = u32x2{0u, 0u}; }
    __device__ __forceinline__ void parts(u32x4 (&out)[1]) const    // whole numbers up to 127 are bf16 numbers: a float's upper half
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = v[i >> 1] >> (16 * (i & 1));
            const float lo = (float)(int8_t)w, hi = (float)(int8_t)(w >> 8);
            out[0][i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        }
    }
    __device__ __forceinline__ bool mend() { return false; }
};

// Wave-wide scans: a lane stands for a sequence.
__device__ __forceinline__ int upto(int v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}
__device__ __forceinline__ int64_t over_lanes(int64_t v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor((long long)v, d);
    return v;
}
__device__ __forceinline__ int same(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A sequence of the call: its new tokens [first, first + fresh) of the batch, the last `fresh` of its `len` positions.
struct Sequence {
    int first, fresh, len;
    __device__ __forceinline__ int blocks(int group, int rows) const { return (fresh * group + rows - 1) / rows; }
    __device__ __forceinline__ int tiles(int tile) const { return (len + tile - 1) / tile; }
    __device__ __forceinline__ int parts(int tile, int per) const { return per ? max(1, (tiles(tile) + per - 1) / per) : 1; }
};
__device__ __forceinline__ Sequence sequence(const ChunkArgs &a, int s)
{
    Sequence r;
    r.first = min(max(a.starts[s], 0), a.N);
    r.fresh = max(min(a.starts[s + 1], a.N) - r.first, 0);
    r.len = paged_length(a.lens[s], a.max_len);
    return r;
}

// The line of all parts of all blocks of rows of one cache head, sequence by sequence, the blocks that see the most first.
template <int kRows, int kTile>
struct Line {
    int per, items;                                  // tiles of a part at most (0: nothing is cut); parts of a cache head
    Sequence seq;                                    // what find() found
    int block, part, parts;

    __device__ __forceinline__ Line(const ChunkArgs &a, int lane) : per(0), items(0)
    {
        if (a.slots > 0) {
            int64_t all = 0;
            for (int base = 0; base < a.n_seq; base += 64)
                if (base + lane < a.n_seq) {
                    const Sequence s = sequence(a, base + lane);
                    all += (int64_t)s.blocks(a.group, kRows) * s.tiles(kTile);
                }
            all = over_lanes(all) * a.pool.n_kv;
            per = same((int)max((all + kParts - 1) / kParts, (int64_t)kLeast));
        }
        for (int base = 0; base < a.n_seq; base += 64) {
            int mine = 0;
            if (base + lane < a.n_seq) {
                const Sequence s = sequence(a, base + lane);
                mine = s.blocks(a.group, kRows) * s.parts(kTile, per);
            }
            items = min(items + __builtin_amdgcn_readlane(upto(mine, lane), 63), a.most);
        }
    }
    // the n-th, n < items; all wave-uniform.  Returns its sequence's number.
    __device__ __forceinline__ int find(const ChunkArgs &a, int n, int lane)
    {
        for (int base = 0;; base += 64) {
            int mine = 0;
            const Sequence s = sequence(a, min(base + lane, a.n_seq - 1));
            if (base + lane < a.n_seq) mine = s.blocks(a.group, kRows) * s.parts(kTile, per);
            const int end = upto(mine, lane), all = __builtin_amdgcn_readlane(end, 63);
            if (n >= all && base + 64 < a.n_seq) {
                n -= all;
                continue;
            }
            const int at = min((int)__popcll(__ballot(end <= n)), 63);
            n -= __builtin_amdgcn_readlane(end - mine, at);
            seq.first = __builtin_amdgcn_readlane(s.first, at);
            seq.fresh = __builtin_amdgcn_readlane(s.fresh, at);
            seq.len = __builtin_amdgcn_readlane(s.len, at);
            parts = seq.parts(kTile, per);
            block = max(seq.blocks(a.group, kRows) - 1 - n / parts, 0);
            part = n % parts;
            return base + at;
        }
    }
};

// The place of a workgroup in a line of `all`: a die takes neighbours, which read the same rows.  -1: none.
__device__ __forceinline__ int place_of(int block, int all)
{
    const int per = (all + kDies - 1) / kDies, slot = block / kDies, at = block % kDies * per + slot;
    return slot < per && at < all ? at : -1;
}

__device__ __forceinline__ void store_four(float *p, const float (&v)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store_four(bf16_t *p, const float (&v)[4])
{
    *reinterpret_cast<uint2 *>(p) = make_uint2((uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
                                               (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
}

// A workgroup of WR * WK waves takes 32 WR rows of a cache head's queries; tiles of TT tokens, of which each of the WK waves of the same rows has
// every WK-th 32.
template <typename Kind, int DP, int WR, int WK>
struct Layout {
    static constexpr int kRows = WR * kCol, kWaves = WR * WK, kThreads = kWaves * 64;
    static constexpr int TT = WK > 1 ? WK * 32 : DP * Kind::kC > 384 ? 32 : 64;
    static constexpr int kUnits = DP / 8, kEach = TT * kUnits / kThreads;     // pieces of eight elements of a row; pieces of a thread
    static constexpr int kPlane = TT * DP * 2, kTileBytes = Kind::kC * kPlane, kJoin = (WK - 1) * kRows * (DP + 2) * 4;
    static constexpr int kLds = 2 * kTileBytes > kJoin ? 2 * kTileBytes : kJoin;
    static_assert(TT * kUnits % kThreads == 0 && kThreads % kUnits == 0, "whole pieces");
};

template <typename Kind, int DP, bool EXACT, int WR, int WK>
__global__ __launch_bounds__(WR * WK * 64) void chunk_attend(ChunkArgs a)
{
    typedef Layout<Kind, DP, WR, WK> L;
    typedef typename Kind::Row Row;
    typedef typename Kind::Cell Cell;
    constexpr int QS = DP / 16, DB = DP / 32, TT = L::TT;
    __shared__ __align__(16) char s_tile[L::kLds];
    __shared__ float s_scale[2][TT];
    __shared__ int s_page[2][TT / 16];               // of the tile's parts of 16 tokens
    __shared__ int s_bad;                            // values of the tile that are no finite numbers
    char *const s_k = s_tile, *const s_v = s_tile + L::kTileBytes;
    const int tid = threadIdx.x, lane = tid & 63, wave = same(tid >> 6), wr = wave / WK, wk = wave % WK;
    const int c = lane & 31, h = lane >> 5;
    const int D = EXACT ? DP : a.D;

    Line<L::kRows, TT> line(a, lane);
    const int work = place_of(blockIdx.x, (int)min((int64_t)line.items * a.pool.n_kv, (int64_t)a.most));
    if (work < 0) return;
    const int kv = work / line.items;
    const int sq = line.find(a, work % line.items, lane);
    const int *table = a.table + (int64_t)sq * a.max_pages;
    const int rows = line.seq.fresh * a.group, row0 = line.block * L::kRows, past = line.seq.len - line.seq.fresh;

    // the lane's row: a query head of a token, heads first
    const int row = row0 + wr * kCol + c, there = min(row, rows - 1);
    const int token = there / a.group, head = kv * a.group + (there - token * a.group);
    const int64_t at = line.seq.first + token;
    const bool kept = !a.mask || a.mask[at * a.n_heads + head] != 0;
    const int lim = max(past + token + 1, 0);        // positions that it sees
    const int wave_last = min(row0 + (wr + 1) * kCol, rows) - 1, wave_first = min(row0 + wr * kCol, rows - 1);
    const int most = max(past + wave_last / a.group + 1, 0), least = max(past + wave_first / a.group + 1, 0);
    const int block_most = max(past + (min(row0 + L::kRows, rows) - 1) / a.group + 1, 0), block_least = max(past + row0 / a.group + 1, 0);
    int tiles = (block_most + TT - 1) / TT;
    // a block without a row that counts reads nothing
    if (!__syncthreads_or(kept && row < rows)) tiles = 0;
    const int from = (int)((int64_t)tiles * line.part / line.parts), to = (int)((int64_t)tiles * (line.part + 1) / line.parts);

    u32x4 qf[Kind::kQ][QS];
    {
        const Row *q = static_cast<const Row *>(a.q) + at * a.q_stride + head * D;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            const int dim = s * 16 + h * 8;
            u32x4 p[Kind::kQ];
            Eight<Row> e;
            e.load(q + (EXACT || dim < D ? dim : 0));
            e.parts(p);
#pragma unroll
            for (int i = 0; i < Kind::kQ; ++i) qf[i][s] = EXACT || dim < D ? p[i] : u32x4{0u, 0u, 0u, 0u};
        }
    }
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    // the thread's pieces of a tile on their way to LDS: those of row unit_row + i * kStep, columns unit * 8
    constexpr int kStep = L::kThreads / L::kUnits;
    const int unit = tid % L::kUnits, unit_row = tid / L::kUnits;
    Eight<Cell> kp[L::kEach], vp[L::kEach];
    float kps = 0.0f, vps = 0.0f;
    int page16 = 0;
    auto fetch = [&](int t) {
        auto cell = [&](int r) {                     // row of the pools that holds position t * TT + r, or -1
            const int pos = t * TT + r;
            const int page = pos < block_most ? table[pos >> a.pool.page_shift] : -1;
            return paged_row(a.pool, page, kv, pos);
        };
#pragma unroll
        for (int i = 0; i < L::kEach; ++i) {
            const int64_t r = cell(unit_row + i * kStep);
            if (r >= 0 && (EXACT || unit * 8 < D)) {
                kp[i].load(static_cast<const Cell *>(a.k) + r * D + unit * 8);
                vp[i].load(static_cast<const Cell *>(a.v) + r * D + unit * 8);
            } else {
                kp[i].zero();
                vp[i].zero();
            }
        }
        if (Kind::kScaled && tid < TT) {
            const int64_t r = cell(tid);
            kps = r >= 0 ? a.k_scale[r] : 0.0f;
            vps = r >= 0 ? a.v_scale[r] : 0.0f;
        }
        if (tid < TT / 16) page16 = cell(tid * 16) >= 0;
    };
    auto put = [&](int t) {
        const bool check = Kind::kCheckAll || (t + 1) * TT > block_least;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < L::kEach; ++i) {
            const int r = unit_row + i * kStep;
            if (check) bad = vp[i].mend() || bad;
            u32x4 p[Kind::kC];
            kp[i].parts(p);
#pragma unroll
            for (int j = 0; j < Kind::kC; ++j)
                *reinterpret_cast<u32x4 *>(s_k + j * L::kPlane + r * DP * 2 + ((unit ^ (r & (L::kUnits < 16 ? 7 : 15))) << 4)) = p[j];
            vp[i].parts(p);
#pragma unroll
            for (int j = 0; j < Kind::kC; ++j)
                *reinterpret_cast<u32x4 *>(s_v + j * L::kPlane + r * DP * 2 + ((unit ^ ((r & 3) << 1)) << 4)) = p[j];
        }
        if (Kind::kScaled && tid < TT) s_scale[0][tid] = kps, s_scale[1][tid] = vps;
        if (tid < TT / 16) s_page[0][tid] = page16;
        if (bad) s_bad = 1;
    };

    // 32 tokens of a tile, from s0 on, against the wave's rows
    auto step = [&](int t, int s0) {
        const int pos0 = t * TT + s0;
        f32x16 x;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.0f;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            if (!EXACT && s * 16 >= D) continue;
            const int r = s0 + c, piece = s * 2 + h;
#pragma unroll
            for (int j = 0; j < Kind::kC; ++j) {
                const u32x4 kf = *reinterpret_cast<const u32x4 *>(s_k + j * L::kPlane + r * DP * 2 + ((piece ^ (r & (L::kUnits < 16 ? 7 : 15))) << 4));
#pragma unroll
                for (int i = 0; i < Kind::kQ; ++i)
                    if (i + j < 3)
                        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf), __builtin_bit_cast(bf16x8_t, qf[i][s]), x, 0, 0, 0);
            }
        }
        float vs[16];
        if constexpr (Kind::kScaled) {
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const f32x4 ks = *reinterpret_cast<const f32x4 *>(&s_scale[0][s0 + 8 * b + 4 * h]), w = *reinterpret_cast<const f32x4 *>(&s_scale[1][s0 + 8 * b + 4 * h]);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * b + e] *= ks[e], vs[4 * b + e] = w[e];
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= a.scale2;
        bool any = true, whole = pos0 + 32 <= least;
        const int p0 = s_page[0][s0 / 16], p1 = s_page[0][s0 / 16 + 1];
        if (!(whole && p0 && p1)) {
            any = false;
            whole = false;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = 8 * (i / 4) + 4 * h + i % 4;
                const bool sees = pos0 + r < lim && (i < 8 ? p0 : p1);
                any = any || sees;
                x[i] = sees ? x[i] : -INFINITY;
                if (Kind::kScaled) vs[i] = sees ? vs[i] : 0.0f;
            }
        }
        float top = any ? -__FLT_MAX__ : -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, x[i]);
        {
            const unsigned u = __builtin_bit_cast(unsigned, top);
            const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
            top = fmaxf(__builtin_bit_cast(float, (unsigned)both[0]), __builtin_bit_cast(float, (unsigned)both[1]));
        }
        // The maximum only moves when a score passes it by 8 (a factor of 256, which float sums take with ease), so that most steps rescale nothing.
        const bool passed = top > m + 8.0f;
        if (__ballot(passed)) {
            const float next = passed ? top : m;     // a row's own scores decide: its result does not depend on its neighbours
            const float by = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - next);
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= by;
            l *= by;
            m = next;
        }
        const float mm = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(x[i] - mm);
        l += (((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]))) + (((x[8] + x[9]) + (x[10] + x[11])) + ((x[12] + x[13]) + (x[14] + x[15])));
        if (Kind::kScaled)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] *= vs[i];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            u32x4 pp[Kind::kP];
            const float e[8] = {x[8 * ks], x[8 * ks + 1], x[8 * ks + 2], x[8 * ks + 3], x[8 * ks + 4], x[8 * ks + 5], x[8 * ks + 6], x[8 * ks + 7]};
            parts_of<Kind::kP>(e, pp);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                if (!EXACT && d * 32 >= D) continue;
                const int r = s0 + 16 * ks + 4 * h + ((lane & 15) >> 2), dim = d * 32 + (lane & 16) + 4 * (lane & 3);
#pragma unroll
                for (int j = 0; j < Kind::kC; ++j) {
                    auto turned = [&](int token) {
                        typedef __attribute__((address_space(3))) s16x4 Lds;
                        char *p = s_v + j * L::kPlane + token * DP * 2 + (((dim >> 3) ^ ((token & 3) << 1)) << 4) + (dim & 4) * 2;
                        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)p));
                    };
                    const u32x2 lo = turned(r), hi = turned(r + 8);
                    const u32x4 vf = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
                    for (int i = 0; i < Kind::kP; ++i)
                        if (i + j < 3)
                            acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf), __builtin_bit_cast(bf16x8_t, pp[i]), acc[d], 0, 0, 0);
                }
            }
        }
        // Values that are no finite numbers were left out of the products (0 * infinity would reach the rows that do not see them): they are added as they
        // are to the rows that do.
        if constexpr (!Kind::kScaled) {
            if (s_bad)
                for (int tt = 0; tt < 32; ++tt) {
                    const int pos = pos0 + tt, page = pos < block_most ? table[pos >> a.pool.page_shift] : -1;
                    const int64_t r = paged_row(a.pool, page, kv, pos);
                    if (r < 0) continue;
                    const Cell *v = static_cast<const Cell *>(a.v) + r * D;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int dim = d * 32 + 8 * (i / 4) + 4 * h + i % 4;
                            const float w = EXACT || dim < D ? to_float(v[dim]) : 0.0f;
                            if (!(fabsf(w) < (Kind::kC > 1 ? 0x1.fep127f : INFINITY)) && pos < lim) acc[d][i] += w;
                        }
                }
        }
    };

    if (tid == 0) s_bad = 0;
    if (from < to) fetch(from);
    for (int t = from; t < to; ++t) {
        __syncthreads();
        if (tid == 0) s_bad = 0;
        __syncthreads();
        put(t);
        if (t + 1 < to) fetch(t + 1);
        __syncthreads();
#pragma unroll 1
        for (int s0 = wk * 32; s0 < TT; s0 += WK * 32)
            if (t * TT + s0 < most) step(t, s0);
    }
    l = xor_add<32>(l);

    if constexpr (WK > 1) {                          // the waves of the same rows, joined in LDS
        __syncthreads();
        float *const part = reinterpret_cast<float *>(s_tile);
        float *const mine = part + ((wr * (WK - 1) + wk - 1) * kCol + c) * (DP + 2);
        if (wk > 0) {
            if (h == 0) mine[DP] = m, mine[DP + 1] = l;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) mine[d * 32 + 8 * (i / 4) + 4 * h + i % 4] = acc[d][i];
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll 1
        for (int w = 0; w < WK - 1; ++w) {
            const float *o = part + ((wr * (WK - 1) + w) * kCol + c) * (DP + 2);
            const float om = o[DP], ol = o[DP + 1], next = fmaxf(m, om), use = next == -INFINITY ? 0.0f : next;
            const float keep = __builtin_amdgcn_exp2f(m - use), by = __builtin_amdgcn_exp2f(om - use);
            l = l * keep + ol * by;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] = acc[d][i] * keep + o[d * 32 + 8 * (i / 4) + 4 * h + i % 4] * by;
            m = next;
        }
    }
    if (row >= rows) return;
    if (line.parts > 1) {
        const int64_t slot = (int64_t)work * L::kRows + wr * kCol + c;
        if (h == 0) *reinterpret_cast<float2 *>(a.stats + slot * 2) = make_float2(m, l);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int dim = d * 32 + 8 * b + 4 * h;
                const float v[4] = {acc[d][4 * b], acc[d][4 * b + 1], acc[d][4 * b + 2], acc[d][4 * b + 3]};
                if (EXACT || dim < D) store_four(a.part + slot * D + dim, v);
            }
        return;
    }
    Row *out = static_cast<Row *>(a.out) + (at * a.n_heads + head) * D;
    const bool none = !kept || m == -INFINITY;
    const float by = 1.0f / l;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int dim = d * 32 + 8 * b + 4 * h;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = none ? 0.0f : acc[d][4 * b + e] * by;
            if (EXACT || dim < D) store_four(out + dim, v);
        }
}

// Joins the blocks that were cut.  Workgroups stand for the line's parts, of which the first of a block does the work (x), cut by y; a thread stands for four
// dimensions of a row.
template <typename Row, int kRows, int kTile>
__global__ __launch_bounds__(256) void chunk_join(ChunkArgs a)
{
    const int lane = threadIdx.x & 63;
    Line<kRows, kTile> line(a, lane);
    const int work = blockIdx.x;
    if (work >= min((int64_t)line.items * a.pool.n_kv, (int64_t)a.most)) return;
    const int kv = work / line.items;
    line.find(a, work % line.items, lane);
    if (line.part != 0 || line.parts == 1) return;
    const int row0 = line.block * kRows, count = min(line.seq.fresh * a.group - row0, kRows), quads = a.D / 4;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < count * quads; i += gridDim.y * 256) {
        const int r = i / quads, q = i - r * quads;
        float m = -INFINITY, l = 0.0f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p = 0; p < line.parts && work + p < a.slots; ++p) {
            const int64_t slot = (int64_t)(work + p) * kRows + r;
            const float2 ml = *reinterpret_cast<const float2 *>(a.stats + slot * 2);
            const float4 v = *reinterpret_cast<const float4 *>(a.part + slot * a.D + q * 4);
            const float next = fmaxf(m, ml.x), use = next == -INFINITY ? 0.0f : next;
            const float keep = __builtin_amdgcn_exp2f(m - use), by = __builtin_amdgcn_exp2f(ml.x - use);
            l = l * keep + ml.y * by;
            o.x = o.x * keep + v.x * by;
            o.y = o.y * keep + v.y * by;
            o.z = o.z * keep + v.z * by;
            o.w = o.w * keep + v.w * by;
            m = next;
        }
        const int row = row0 + r, token = row / a.group, head = kv * a.group + (row - token * a.group);
        const int64_t at = line.seq.first + token;
        const bool none = m == -INFINITY || (a.mask && !a.mask[at * a.n_heads + head]);
        const float by = 1.0f / l;
        const float v[4] = {none ? 0.0f : o.x * by, none ? 0.0f : o.y * by, none ? 0.0f : o.z * by, none ? 0.0f : o.w * by};
        store_four(static_cast<Row *>(a.out) + (at * a.n_heads + head) * a.D + q * 4, v);
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// Blocks of `rows` rows that a call may have, over all cache heads.
inline int64_t most_blocks(const ChunkArgs &a, int rows)
{
    return ((int64_t)a.N * a.group / rows + (a.n_seq < a.N ? a.n_seq : a.N)) * a.pool.n_kv;
}

template <typename Kind, int DP, bool EXACT, int WR, int WK>
int launch_rows(ChunkArgs a, hipStream_t s)
{
    typedef Layout<Kind, DP, WR, WK> L;
    const int64_t blocks = most_blocks(a, L::kRows);
    int64_t grid = blocks;
    const bool cut = blocks < kParts && a.max_len > kLeast * L::TT;
    if (cut) {
        grid += kParts;                              // a part more than even shares give, for each block
        a.slots = (int)grid;
    }
    a.most = (int)grid;
    grid = (grid + kDies - 1) / kDies * kDies;
    chunk_attend<Kind, DP, EXACT, WR, WK><<<dim3((unsigned)grid), dim3(L::kThreads), 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return HALO_ERR_HIP;
    if (!cut) return HALO_OK;
    chunk_join<typename Kind::Row, L::kRows, L::TT><<<dim3(a.slots, (L::kRows * (a.D / 4) + 1023) / 1024), dim3(256), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}

template <typename Kind, int DP, bool EXACT>
int launch_chunk(const ChunkArgs &a, hipStream_t s)
{
    constexpr int kNarrow = DP * Kind::kC > 512 ? 1 : DP * Kind::kC > 256 ? 2 : 4;      // waves of the same rows that LDS has room for
    if ((int64_t)a.N * a.group <= (int64_t)kCol * a.n_seq) return launch_rows<Kind, DP, EXACT, 1, kNarrow>(a, s);
    return launch_rows<Kind, DP, EXACT, 4, 1>(a, s);
}

template <typename Kind>
int launch_chunk_dim(const ChunkArgs &a, hipStream_t s)
{
    if (a.D == 64) return launch_chunk<Kind, 64, true>(a, s);
    if (a.D == 128) return launch_chunk<Kind, 128, true>(a, s);
    if (a.D == 256) return launch_chunk<Kind, 256, true>(a, s);
    if (a.D < 64) return launch_chunk<Kind, 64, false>(a, s);
    if (a.D < 128) return launch_chunk<Kind, 128, false>(a, s);
    return launch_chunk<Kind, 256, false>(a, s);
}

}  // namespace

// One for each kind of cache and queries, each in a file of its own.
int launch_chunk_bf16(const ChunkArgs &a, hipStream_t s);
int launch_chunk_f32(const ChunkArgs &a, hipStream_t s);
int launch_chunk_q8(const ChunkArgs &a, hipStream_t s);
int launch_chunk_q8_f32(const ChunkArgs &a, hipStream_t s);

}  // namespace halo
