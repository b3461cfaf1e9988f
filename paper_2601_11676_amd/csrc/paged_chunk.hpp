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
    int32_t *kept, *n_kept;                          // with a mask: rows that survive [cache head][N * group] and how many [cache head][sequence] (chunk_rows)
    int64_t q_stride;
    PagePool pool;
    int N, n_seq, n_heads, group, D, max_pages, max_len;
    int most;                                        // parts that a call may have, whatever its lengths (more: starts that go back)
    int slots;                                       // the same where blocks are cut: partial results that the workspace holds; else 0
    float scale2;                                    // scale * log2(e): the softmax is computed in powers of two
};

namespace {

constexpr int kCol = 32;                             // columns of the matrix instruction: rows of a block, that is queries
constexpr int kLeast = 2;                            // tiles of a part at least: a part of one is mostly its beginning (some 8 us until the first product)
constexpr int kDies = 8;
constexpr int kPartRows = 2 * 256 * 8 * kCol;        // rows of partial results: see Layout::kCuts

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// What a cache holds and how it goes to the matrix cores: an element as the sum of so many bf16 parts (three hold a float), of which products i * j
// with i + j < 3 are taken, what is left out is 2^-24 of a product.  kP: of a probability.
struct KindBf16 {
    typedef bf16_t Row, Cell;                        // queries and results; the cache
    static constexpr int kQ = 1, kC = 1, kP = 1;     // of a probability one part: paged_chunk.hip has what two cost
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
            out[p][i] = P > 1 && p == 0 ? pack_bf16(first_part(a), first_part(b)) : pack_bf16(a, b);
            if (p + 1 < P) {
                a -= bf16_lo(out[p][i]);
                b -= bf16_hi(out[p][i]);
            }
        }
    }
}

// 16 bytes of a row of the cache, as loaded, and as bf16 parts in LDS: words of two elements each.
template <typename Cell> struct Piece;
template <> struct Piece<bf16_t> {
    static constexpr int kElems = 8, kWords = 4;
    u32x4 v;
    __device__ __forceinline__ void parts(uint32_t (&out)[1][4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[0][i] = v[i];
    }
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
template <> struct Piece<float> {
    static constexpr int kElems = 4, kWords = 2;
    u32x4 v;
    __device__ __forceinline__ void parts(uint32_t (&out)[3][2]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float a = __uint_as_float(v[2 * i]), b = __uint_as_float(v[2 * i + 1]);
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                out[p][i] = p == 0 ? pack_bf16(first_part(a), first_part(b)) : pack_bf16(a, b);
                a -= bf16_lo(out[p][i]);
                b -= bf16_hi(out[p][i]);
            }
        }
    }
    __device__ __forceinline__ bool mend()
    {
        bool any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool x = !(fabsf(__uint_as_float(v[i])) < INFINITY);
            any = any || x;
            v[i] = x ? 0u : v[i];
        }
        return any;
    }
};
template <> struct Piece<int8_t> {
    static constexpr int kElems = 16, kWords = 8;
    u32x4 v;
    __device__ __forceinline__ void parts(uint32_t (&out)[1][8]) const    // whole numbers up to 127 are bf16 numbers: a float's upper half
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int w = (int)v[i >> 1];
            const float lo = (float)(i & 1 ? (w << 8) >> 24 : (w << 24) >> 24), hi = (float)(i & 1 ? w >> 24 : (w << 16) >> 24);
            out[0][i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        }
    }
    __device__ __forceinline__ bool mend() { return false; }
};

// Eight elements of a query as bf16 parts.
__device__ __forceinline__ void query_parts(const bf16_t *p, u32x4 (&out)[1]) { out[0] = *reinterpret_cast<const u32x4 *>(p); }
__device__ __forceinline__ void query_parts(const float *p, u32x4 (&out)[3])
{
    float x[8];
    load8(p, x);
    parts_of<3>(x, out);
}

// The sum of the lanes up to each one.
__device__ __forceinline__ int upto(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8: within 16 lanes
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast 15, 31: the rows before
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
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

// The line of all parts of all blocks of rows of one cache head: sequence by sequence, long ones first (up to 64 of them; of more in their order), and a sequence's blocks that see
// the most first, so that what begins last is short.  All of a wave-uniform; a lane has a sequence.
template <int kRows, int kTile, int kCuts>
struct Line {
    int per, items;                                  // tiles of a part at most (0: nothing is cut); parts of a cache head
    Sequence own;                                    // up to 64 sequences: of the lane's, in the line's order; its number and the parts up to its end
    int number, end;
    Sequence seq;                                    // what find() found: sequence, block of rows, part of so many
    int block, part, parts;

    __device__ __forceinline__ Line(const ChunkArgs &a, int lane) : per(0), items(0), number(lane), end(0)
    {
        const bool few = a.n_seq <= 64;
        if (few) {
            own = sequence(a, min(lane, a.n_seq - 1));
            if (lane >= a.n_seq) own.fresh = 0, own.len = 0;
            int rank = 0;
            for (int i = 0; i < a.n_seq; ++i) {
                const int other = __builtin_amdgcn_readlane(own.len, i);
                rank += other > own.len || (other == own.len && i < lane);
            }
            const int to = (lane < a.n_seq ? rank : lane) * 4;
            number = __builtin_amdgcn_ds_permute(to, lane);
            own.first = __builtin_amdgcn_ds_permute(to, own.first);
            own.fresh = __builtin_amdgcn_ds_permute(to, own.fresh);
            own.len = __builtin_amdgcn_ds_permute(to, own.len);
        }
        if (a.slots > 0) {
            // tiles of all blocks, and blocks: a part is that share of them that leaves about as many parts as are resident at once (each block's last is half of one)
            float tiles = 0.0f, blocks = 0.0f;
            for (int i = lane; i < a.n_seq; i += 64) {
                const Sequence s = few ? own : sequence(a, i);
                blocks += (float)s.blocks(a.group, kRows);
                tiles += (float)s.blocks(a.group, kRows) * (float)s.tiles(kTile);
            }
            tiles = wave_sum(tiles) * a.pool.n_kv;
            blocks = wave_sum(blocks) * a.pool.n_kv;
            per = same(max((int)fminf(tiles / fmaxf(kCuts - 0.5f * blocks, 0.25f * kCuts), 1e9f) + 1, kLeast));
        }
        if (few) {
            end = upto(own.blocks(a.group, kRows) * own.parts(kTile, per));
            items = __builtin_amdgcn_readlane(end, 63);
        } else {
            for (int base = 0; base < a.n_seq; base += 64) {
                int mine = 0;
                if (base + lane < a.n_seq) {
                    const Sequence s = sequence(a, base + lane);
                    mine = s.blocks(a.group, kRows) * s.parts(kTile, per);
                }
                items = min(items + __builtin_amdgcn_readlane(upto(mine), 63), a.most);
            }
        }
        items = min(items, a.most);
    }
    __device__ __forceinline__ int take(const ChunkArgs &a, const Sequence &s, int mine, int upto_end, int name, int n, int at)
    {
        n -= __builtin_amdgcn_readlane(upto_end - mine, at);
        seq.first = __builtin_amdgcn_readlane(s.first, at);
        seq.fresh = __builtin_amdgcn_readlane(s.fresh, at);
        seq.len = __builtin_amdgcn_readlane(s.len, at);
        parts = seq.parts(kTile, per);
        const int blocks = seq.blocks(a.group, kRows);
        block = max(blocks - 1 - n / parts, 0);
        part = n % parts;
        return __builtin_amdgcn_readlane(name, at);
    }
    // the n-th, n < items.  Returns its sequence's number.
    __device__ __forceinline__ int find(const ChunkArgs &a, int n, int lane)
    {
        if (a.n_seq <= 64) return take(a, own, own.blocks(a.group, kRows) * own.parts(kTile, per), end, number, n, min((int)__popcll(__ballot(end <= n)), 63));
        for (int base = 0;; base += 64) {
            int mine = 0;
            const Sequence s = sequence(a, min(base + lane, a.n_seq - 1));
            if (base + lane < a.n_seq) mine = s.blocks(a.group, kRows) * s.parts(kTile, per);
            const int last = upto(mine), all = __builtin_amdgcn_readlane(last, 63);
            if (n >= all && base + 64 < a.n_seq) {
                n -= all;
                continue;
            }
            return take(a, s, mine, last, base + lane, n, min((int)__popcll(__ballot(last <= n)), 63));
        }
    }
};

// A workgroup's part of the line and cache head: neighbours of the line, all heads of one after those of the other.  Workgroup i runs on die i % 8: where the cache heads are
// a multiple of the dies, each die has heads of its own, whose rows its L2 then serves to all that read them.
__device__ __forceinline__ bool place_of(const ChunkArgs &a, int block, int items, int &item, int &kv)
{
    const int heads = a.pool.n_kv % kDies == 0 ? a.pool.n_kv / kDies : a.pool.n_kv;
    const int slot = heads < a.pool.n_kv ? block / kDies : block;
    item = slot / heads;
    kv = slot - item * heads + (heads < a.pool.n_kv ? block % kDies * heads : 0);
    return item < items && (int64_t)item * a.pool.n_kv + kv < a.most;
}

// The rows of a sequence and cache head that the mask keeps, in order: the i-th of them, or of more the last.
struct Survivors {
    const int32_t *list;
    int rows, last;                                  // rows, and the last row of the sequence
    __device__ __forceinline__ Survivors(const ChunkArgs &a, const Sequence &s, int number, int kv) : list(nullptr), rows(s.fresh * a.group), last(rows - 1)
    {
        if (!a.kept) return;
        list = a.kept + ((int64_t)kv * a.N + s.first) * a.group;
        rows = same(a.n_kept[(int64_t)kv * a.n_seq + number]);
    }
    __device__ __forceinline__ int row(int i) const
    {
        i = min(i, rows - 1);
        return list ? min(list[i], last) : i;        // no further than the sequence, were starts to go back and lists to be one another's
    }
};

__device__ __forceinline__ void store_four(float *p, const float (&v)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store_four(bf16_t *p, const float (&v)[4])
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
}

// A workgroup of WR * WK waves takes 32 WR rows of a cache head's queries; tiles of TT tokens, of which each of the WK waves of the same rows has
// every WK-th 32.  Two tiles in LDS, one being read while the next is written, where they have room beside another workgroup's.
template <typename Kind, int DP, int WR, int WK>
struct Layout {
    typedef typename Kind::Cell Cell;
    static constexpr int kRows = WR * kCol, kWaves = WR * WK, kThreads = kWaves * 64;
    static constexpr int TT = WK > 1 ? WK * 32 : DP * Kind::kC > 128 ? 32 : 64, kSub = TT / 32 / WK;
    static constexpr int kPlane = TT * DP * 2, kTileBytes = 2 * Kind::kC * kPlane, kJoin = (WK - 1) * kRows * (DP + 2) * 4;
    static constexpr int kBufs = kTileBytes <= 65536 && WK < 4 ? 2 : 1, kRowsBytes = kTileBytes / 2;
    static constexpr int kLds = kBufs * kTileBytes > kJoin ? kBufs * kTileBytes : kJoin;
    // loads of a wave, 1 KiB each: of kRowsEach rows, which lie in one part of 16 tokens
    static constexpr int kRowBytes = DP * (int)sizeof(Cell), kRowLanes = kRowBytes / 16, kRowsEach = 64 / kRowLanes, kLoads = TT / kRowsEach;
    static constexpr int kEach = (kLoads + kWaves - 1) / kWaves, kParts16 = TT / 16, kPerPart = kEach * kRowsEach > 16 ? 16 / kRowsEach : kEach;
    static_assert(16 % kRowsEach == 0 && (kLoads % kWaves == 0 || kLoads < kWaves), "whole loads");
    // Waves of a SIMD (two for float heads of 64 too: 4 sequences of 4000 in all, 32 heads, 147 us with one, 137); and the parts that few blocks are cut into, about: what is resident at once.  Their partial results are of a part each and one more for each block, fewer than parts.
    static constexpr int kOnSimd = DP * Kind::kC <= 192 && kLds * (8 / kWaves) <= 163840 ? 2 : 1, kCuts = kOnSimd * 4 > kWaves ? 512 : 256;
    static_assert(2 * kCuts * kRows <= kPartRows, "partial results in the workspace");
};

// Where a lane's 16 bytes lie in LDS: key rows are read 16 bytes a lane, a row a lane; value rows 16 dimensions of four rows at a time.  The pieces of a row change
// places so that neither meets a bank twice.
template <int DP> __device__ __forceinline__ int key_place(int row, int piece) { return row * DP * 2 + ((piece ^ (row & (DP < 128 ? 7 : 15))) << 4); }
template <int DP> __device__ __forceinline__ int value_place(int row, int piece)
{
    const int f = ((row & 3) ^ ((row & 3) << 1)) << 1;
    return row * DP * 2 + ((piece ^ (f & (DP / 8 - 1))) << 4);
}

// Products of parts that are taken.
constexpr int products(int a, int b) { return a * b < 9 ? a * b : 6; }

// The order of a run of matrix instructions and of the loads from LDS of their operands, READS loads an operand: four operands first, then one for each that is used up
// (left to itself the compiler loads one ahead and waits out the latency at every second instruction).
template <int OPERANDS, int MFMAS, int READS>
__device__ __forceinline__ void reads_ahead()
{
    constexpr int kAhead = OPERANDS < 4 ? OPERANDS : 4;
    __builtin_amdgcn_sched_group_barrier(0x100, kAhead * READS, 0);
#pragma unroll
    for (int i = 0; i < OPERANDS - kAhead; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, MFMAS, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kAhead * MFMAS, 0);
}

template <typename Kind, int DP, bool EXACT, int WR, int WK>
__global__ __launch_bounds__(WR * WK * 64, (Layout<Kind, DP, WR, WK>::kOnSimd)) void chunk_attend(ChunkArgs a)
{
    typedef Layout<Kind, DP, WR, WK> L;
    typedef typename Kind::Row Row;
    typedef typename Kind::Cell Cell;
    typedef Piece<Cell> P;
    constexpr int QS = DP / 16, DB = DP / 32, TT = L::TT, NS = L::kSub;
    __shared__ __align__(16) char s_tile[L::kLds];
    __shared__ __align__(16) float s_scale[L::kBufs][2][TT];
    __shared__ int s_bad[L::kBufs];                  // 1 + the tile whose values have some that are no finite numbers
    const int tid = threadIdx.x, lane = tid & 63, wave = same(tid >> 6), wr = wave / WK, wk = wave % WK;
    const int c = lane & 31, h = lane >> 5;
    const int D = EXACT ? DP : a.D;

    Line<L::kRows, TT, L::kCuts> line(a, lane);
    int item, kv;
    if (!place_of(a, blockIdx.x, line.items, item, kv)) return;
    const int sq = line.find(a, item, lane);
    const Survivors survivors(a, line.seq, sq, kv);
    const int rows = survivors.rows, row0 = line.block * L::kRows, past = line.seq.len - line.seq.fresh;
    if (row0 >= rows) return;

    // the lane's row: a query head of a token, heads first
    const int row = row0 + wr * kCol + c, there = survivors.row(row);
    const int token = there / a.group, head = kv * a.group + (there - token * a.group);
    const int64_t at = line.seq.first + token;
    const bool kept = !a.mask || a.kept || a.mask[at * a.n_heads + head] != 0;
    const int lim = max(past + token + 1, 0);        // positions that it sees; of the wave's rows and of the block's, the most and the least
    const int most = row0 + wr * kCol < rows ? __builtin_amdgcn_readlane(lim, 31) : 0, least = __builtin_amdgcn_readlane(lim, 0);      // a wave without rows reads nothing
    const int block_most = same(max(past + survivors.row(row0 + L::kRows - 1) / a.group + 1, 0)), block_least = same(max(past + survivors.row(row0) / a.group + 1, 0));
    int tiles = (block_most + TT - 1) / TT;
    // a block without a row that counts reads nothing
    if (a.mask && !a.kept && !__syncthreads_or(kept && row < rows)) tiles = 0;
    const int from = same((int)((int64_t)tiles * line.part / line.parts)), to = same((int)((int64_t)tiles * (line.part + 1) / line.parts));

    // queries are asked for first, so that they travel while the pages' numbers do
    u32x4 qf[Kind::kQ][QS];
    {
        const Row *q = static_cast<const Row *>(a.q) + at * a.q_stride + head * D;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            const int dim = s * 16 + h * 8;
            u32x4 p[Kind::kQ];
            query_parts(q + (EXACT || dim < D ? dim : 0), p);
#pragma unroll
            for (int i = 0; i < Kind::kQ; ++i) qf[i][s] = EXACT || dim < D ? p[i] : u32x4{0u, 0u, 0u, 0u};
        }
    }
    // page numbers of the parts of 16 tokens, 64 parts at a time, a lane each (-1: no page), and which are pages
    const int32_t *table = a.table + (int64_t)sq * a.max_pages;
    int held = from * L::kParts16, id = 0, id_next = 0;
    uint64_t pages = 0, pages_next = 0;
    auto look = [&](int part) {
        const int64_t pos = (int64_t)(part + lane) * 16;
        int page = pos < block_most ? table[(int)pos >> a.pool.page_shift] : -1;
        return page_exists(a.pool, page) ? page : -1;
    };
    if (from < to) {
        id = look(held), id_next = look(held + 64);
        pages = __ballot(id >= 0), pages_next = __ballot(id_next >= 0);
    }
    // both wave-uniform, of the tile being computed, one before or two after it: a part's page; whether all parts of a tile are pages
    auto page_of = [&](int part) {
        const int n = part - held, p0 = __builtin_amdgcn_readlane(id, n & 63), p1 = __builtin_amdgcn_readlane(id_next, n & 63);
        return n < 64 ? p0 : p1;
    };
    auto all_pages = [&](int t) {                    // 64 is a multiple of a tile's parts
        constexpr uint64_t kAll = (1ull << L::kParts16) - 1;
        const int n = t * L::kParts16 - held;
        return (((n < 64 ? pages : pages_next) >> (n & 63)) & kAll) == kAll;
    };
    auto advance = [&](int part) {                   // nobody asks for parts before this one any more
        if (part - held < 64) return;
        held += 64;
        id = id_next;
        pages = pages_next;
        id_next = look(held + 64);
        pages_next = __ballot(id_next >= 0);
    };

    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    // a tile's rows on their way to LDS: 16 bytes a lane and load
    const int load_row = lane / L::kRowLanes, load_piece = lane % L::kRowLanes;
    const uint32_t voff = EXACT || load_piece * P::kElems < D ? (uint32_t)(load_row * D * (int)sizeof(Cell) + load_piece * 16) : kOutOfRange;
    P kp[L::kEach], vp[L::kEach];
    float kps = 0.0f, vps = 0.0f;
    // Without a condition: rows that are none, and tiles past the last, are descriptors of no bytes (a load that may not be made would have its registers copied, and that
    // waits for it).
    auto fetch = [&](int t) {
        constexpr int kRow = (int)sizeof(Cell);
#pragma unroll
        for (int j = 0; j < L::kEach; j += L::kPerPart) {
            const int r = (wave * L::kEach + j) % L::kLoads * L::kRowsEach, pos = t * TT + r;
            const int page = page_of(t * L::kParts16 + r / 16);
            const int live = page < 0 || t >= to ? 0 : max(0, min(block_most - pos, L::kPerPart * L::kRowsEach));
            const uint64_t row = ((((uint64_t)max(page, 0) * a.pool.n_kv + kv) << a.pool.page_shift) + (pos & ((1 << a.pool.page_shift) - 1))) * (uint64_t)(D * kRow);
            const uint64_t byte = (uint64_t)(uint32_t)same((int)(row >> 32)) << 32 | (uint32_t)same((int)row);
            const int bytes = same(live * D * kRow);
            const auto k_rows = buffer_of(static_cast<const char *>(a.k) + byte, bytes), v_rows = buffer_of(static_cast<const char *>(a.v) + byte, bytes);
#pragma unroll
            for (int i = 0; i < L::kPerPart; ++i) kp[j + i].v = buffer_load16<0>(k_rows, voff + i * L::kRowsEach * D * kRow, 0);
#pragma unroll
            for (int i = 0; i < L::kPerPart; ++i) vp[j + i].v = buffer_load16<0>(v_rows, voff + i * L::kRowsEach * D * kRow, 0);
        }
        if constexpr (Kind::kScaled) {
            if (wave * 64 < TT) {                    // whole waves, of tiles of 32 too: an exchange takes nothing from lanes that are not there
                const int pos = t * TT + tid, part = t * L::kParts16 + tid / 16 - held;
                const int p0 = __shfl(id, part & 63), p1 = __shfl(id_next, part & 63);
                const int page = part < 64 ? p0 : p1;
                const bool in = tid < TT && page >= 0 && pos < block_most && t < to;
                const int64_t r = in ? paged_row(a.pool, page, kv, pos) : 0;
                kps = in ? a.k_scale[r] * a.scale2 : 0.0f;
                vps = in ? a.v_scale[r] : 0.0f;
            }
        }
    };
    auto put_rows = [&](const P (&from)[L::kEach], char *plane, bool value) {
#pragma unroll
        for (int i = 0; i < L::kEach; ++i) {
            if (L::kLoads < L::kWaves && wave >= L::kLoads) break;
            const int r = (wave * L::kEach + i) * L::kRowsEach + load_row;
            {
                uint32_t w[Kind::kC][P::kWords];
                from[i].parts(w);
#pragma unroll
                for (int j = 0; j < Kind::kC; ++j) {
                    if constexpr (P::kWords == 2) {
                        const int piece = load_piece >> 1;
                        char *to = plane + j * L::kPlane + (value ? value_place<DP>(r, piece) : key_place<DP>(r, piece)) + (load_piece & 1) * 8;
                        *reinterpret_cast<uint2 *>(to) = make_uint2(w[j][0], w[j][1]);
                    } else {
#pragma unroll
                        for (int e = 0; e < P::kWords / 4; ++e) {
                            const int piece = load_piece * (P::kWords / 4) + e;
                            char *to = plane + j * L::kPlane + (value ? value_place<DP>(r, piece) : key_place<DP>(r, piece));
                            *reinterpret_cast<u32x4 *>(to) = u32x4{w[j][4 * e], w[j][4 * e + 1], w[j][4 * e + 2], w[j][4 * e + 3]};
                        }
                    }
                }
            }
        }
    };
    auto keys_of = [&](int buf) { return s_tile + buf * L::kRowsBytes; };
    auto values_of = [&](int buf) { return s_tile + (L::kBufs + buf) * L::kRowsBytes; };
    auto put = [&](int t, int buf) {
        put_rows(kp, keys_of(buf), false);
        if (Kind::kScaled && tid < TT) s_scale[buf][0][tid] = kps, s_scale[buf][1][tid] = vps;
        if (Kind::kCheckAll || (!Kind::kScaled && (t + 1) * TT > block_least)) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < L::kEach; ++i) bad = vp[i].mend() || bad;
            if (bad) s_bad[buf] = t + 1;
        }
        put_rows(vp, values_of(buf), true);
    };

    // where the lane reads: 16 bytes of token c's key; four tokens' values of its dimension, as the loads that turn them want it
    int key_at[QS], value_at[DB];
#pragma unroll
    for (int s = 0; s < QS; ++s) key_at[s] = key_place<DP>(c, s * 2 + h);
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const int dim = d * 32 + (lane & 16) + 4 * (lane & 3);
        value_at[d] = value_place<DP>(4 * h + ((lane & 15) >> 2), dim >> 3) + (dim & 4) * 2;
    }

    // the wave's tokens of a tile against its rows: scores, probabilities, products with the values
    float x[NS][16];
    u32x4 pp[NS][2][Kind::kP];
    auto scores = [&](int t, int buf) {
        const char *const s_k = keys_of(buf);
        f32x16 sc[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[n][i] = 0.0f;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            if (!EXACT && s * 16 >= D) continue;
#pragma unroll
            for (int j = 0; j < Kind::kC; ++j)
#pragma unroll
                for (int n = 0; n < NS; ++n) {
                    const u32x4 kf = *reinterpret_cast<const u32x4 *>(s_k + j * L::kPlane + (n * WK + wk) * 32 * DP * 2 + key_at[s]);
#pragma unroll
                    for (int i = 0; i < Kind::kQ; ++i)
                        if (i + j < 3)
                            sc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf), __builtin_bit_cast(bf16x8_t, qf[i][s]), sc[n], 0, 0, 0);
                }
        }
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[n][i] = sc[n][i];
        if constexpr (EXACT) reads_ahead<NS * QS * Kind::kC, products(Kind::kQ, Kind::kC) / Kind::kC, 1>();
    };
    auto soften = [&](int t, int buf) {
        float vs[NS][16];
        if constexpr (Kind::kScaled) {
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                const int s0 = (n * WK + wk) * 32;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const f32x4 ks = *reinterpret_cast<const f32x4 *>(&s_scale[buf][0][s0 + 8 * b + 4 * h]), w = *reinterpret_cast<const f32x4 *>(&s_scale[buf][1][s0 + 8 * b + 4 * h]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[n][4 * b + e] *= ks[e], vs[n][4 * b + e] = w[e];
                }
            }
        }
        // all seen by all rows, and scores whose order the scale keeps: the scale waits for the exponent
        bool whole = (t + 1) * TT <= least && all_pages(t), any = true;
        float by_scale = Kind::kScaled ? 1.0f : a.scale2;
        if (!whole || !(by_scale > 0.0f)) {
            any = false;
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                const int s0 = (n * WK + wk) * 32, part = t * L::kParts16 + s0 / 16;
                const bool p0 = page_of(part) >= 0, p1 = page_of(part + 1) >= 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int r = 8 * (i / 4) + 4 * h + i % 4;
                    const bool sees = t * TT + s0 + r < lim && (i < 8 ? p0 : p1);
                    any = any || sees;
                    x[n][i] = sees ? x[n][i] * by_scale : -INFINITY;
                    if (Kind::kScaled) vs[n][i] = sees ? vs[n][i] : 0.0f;
                }
            }
            by_scale = 1.0f;
        }
        float top = x[0][0];
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[n][i]);
        {
            const unsigned u = __builtin_bit_cast(unsigned, top);
            const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
            top = fmaxf(__builtin_bit_cast(float, (unsigned)both[0]), __builtin_bit_cast(float, (unsigned)both[1]));
        }
        // positions that count lift the maximum to the lowest float at least: -infinity says that a row has none
        if (!whole) any = __builtin_amdgcn_permlane32_swap((unsigned)any, (unsigned)any, false, false)[0] != 0 || __builtin_amdgcn_permlane32_swap((unsigned)any, (unsigned)any, false, false)[1] != 0;
        top = fmaxf(top * by_scale, any ? -__FLT_MAX__ : -INFINITY);
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
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][i], by_scale, -mm));
        if (Kind::kScaled || Kind::kP > 1) {
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int i = 0; i < 16; i += 4) l += (x[n][i] + x[n][i + 1]) + (x[n][i + 2] + x[n][i + 3]);
        }
        if (Kind::kScaled) {
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[n][i] *= vs[n][i];
        }
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const float e[8] = {x[n][8 * ks], x[n][8 * ks + 1], x[n][8 * ks + 2], x[n][8 * ks + 3], x[n][8 * ks + 4], x[n][8 * ks + 5], x[n][8 * ks + 6], x[n][8 * ks + 7]};
                parts_of<Kind::kP>(e, pp[n][ks]);
                if (!Kind::kScaled && Kind::kP == 1) {       // the sum is of what is multiplied: the weights add up to one
#pragma unroll
                    for (int i = 0; i < 4; ++i) l = dot2_bf16(pp[n][ks][0][i], 0x3f803f80u, l);
                }
            }
    };
    auto product = [&](int t, int buf) {
        const char *const s_v = values_of(buf);
        // of a tile with values that are no finite numbers: the lane's probabilities that are 0
        bool bad = false;
        uint32_t none = 0;
        if constexpr (!Kind::kScaled) {
            bad = s_bad[buf] == t + 1;
            if (bad) {
#pragma unroll
                for (int n = 0; n < NS; ++n)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t two = pp[n][i / 4][0][i % 4];
                        none |= (two & 0x7fffu ? 0u : 1u) << (16 * n + 2 * i) | (two & 0x7fff0000u ? 0u : 2u) << (16 * n + 2 * i);
                    }
            }
        }
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const int s0 = (n * WK + wk) * 32;
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    if (!EXACT && d * 32 >= D) continue;
#pragma unroll
                    for (int j = 0; j < Kind::kC; ++j) {
                        auto turned = [&](int token) {
                            typedef __attribute__((address_space(3))) s16x4 Lds;
                            return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)(s_v + j * L::kPlane + token * DP * 2 + value_at[d])));
                        };
                        const u32x2 lo = turned(s0 + 16 * ks), hi = turned(s0 + 16 * ks + 8);
                        const u32x4 vf = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
                        for (int i = 0; i < Kind::kP; ++i)
                            if (i + j < 3)
                                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf), __builtin_bit_cast(bf16x8_t, pp[n][ks][i]), acc[d], 0, 0, 0);
                    }
                }
            }
        if constexpr (EXACT) reads_ahead<NS * 2 * DB * Kind::kC, products(Kind::kP, Kind::kC) / Kind::kC, 2>();
        // Values that are no finite numbers were left out of the products (0 * infinity would reach the rows that do not see them): the rows that do have them added, as
        // products with their probabilities: themselves, or NaN where that is 0.
        if constexpr (!Kind::kScaled) {
            if (bad)
                for (int tt = 0; tt < 32 * NS; ++tt) {
                    const int r0 = (tt / 32 * WK + wk) * 32 + tt % 32, pos = t * TT + r0, page = page_of(t * L::kParts16 + r0 / 16);
                    if (page < 0 || pos >= block_most) continue;
                    const uint32_t bits = (uint32_t)__shfl((int)none, c + (tt & 4) * 8);         // of the lane that has the row's probability of this token
                    const bool zero = bits >> (tt / 32 * 16 + tt % 32 / 8 * 4 + tt % 4) & 1;
                    const Cell *v = static_cast<const Cell *>(a.v) + paged_row(a.pool, page, kv, pos) * D;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int dim = d * 32 + 8 * (i / 4) + 4 * h + i % 4;
                            const float w = EXACT || dim < D ? to_float(v[dim]) : 0.0f;
                            if (!(fabsf(w) < INFINITY) && pos < lim) acc[d][i] += zero ? NAN : w;
                        }
                }
        }
    };

    if (tid < L::kBufs) s_bad[tid] = 0;
    if (from < to) fetch(from);
    __syncthreads();
    auto step = [&](int t, int buf) {
        scores(t, buf);
        soften(t, buf);
        product(t, buf);
    };
    if constexpr (L::kBufs == 2) {
        if (from < to) put(from, 0);
        for (int t = from; t < to; ++t) {
            const int buf = (t - from) & 1;
            __syncthreads();
            advance(t * L::kParts16);
            fetch(t + 1);
            if (t * TT < most) step(t, buf);
            put(t + 1, buf ^ 1);                     // which every wave was done with before the barrier
        }
    } else {
        for (int t = from; t < to; ++t) {
            put(t, 0);
            __syncthreads();
            advance(t * L::kParts16);
            fetch(t + 1);
            if (t * TT < most) step(t, 0);
            __syncthreads();
        }
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
        const int64_t slot = ((int64_t)item * a.pool.n_kv + kv) * L::kRows + wr * kCol + c;
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

// Joins the blocks that were cut.  Workgroups stand for blocks of rows (x), cut by y; a thread stands for four dimensions of a row.
template <typename Row, int kRows, int kTile, int kCuts>
__global__ __launch_bounds__(256) void chunk_join(ChunkArgs a)
{
    const int lane = threadIdx.x & 63, kv = blockIdx.z;
    Line<kRows, kTile, kCuts> line(a, lane);
    // the x-th of those that are cut: the first part of each block is its place in the line
    int n = 0;
    {
        int at = blockIdx.x;
        for (int base = 0; base < a.n_seq; base += 64) {
            const bool few = a.n_seq <= 64, in = base + lane < a.n_seq;
            Sequence s = few ? line.own : sequence(a, min(base + lane, a.n_seq - 1));
            const int parts = s.parts(kTile, line.per), blocks = in || few ? s.blocks(a.group, kRows) : 0;
            const int cut = parts > 1 ? blocks : 0, cut_end = upto(cut), cuts_all = __builtin_amdgcn_readlane(cut_end, 63);
            const int end = upto(blocks * parts);
            if (at < cuts_all) {
                const int l = min((int)__popcll(__ballot(cut_end <= at)), 63);
                n += __builtin_amdgcn_readlane(end - blocks * parts, l) + (at - __builtin_amdgcn_readlane(cut_end - cut, l)) * __builtin_amdgcn_readlane(parts, l);
                at = -1;
                break;
            }
            at -= cuts_all;
            n += __builtin_amdgcn_readlane(end, 63);
        }
        if (at >= 0 || n >= line.items) return;
    }
    const int sq = line.find(a, n, lane);
    const Survivors survivors(a, line.seq, sq, kv);
    // a row is 2^lanes_log neighbouring lanes
    const int row0 = line.block * kRows, count = min(survivors.rows - row0, kRows), quads = a.D / 4, lanes_log = quads > 32 ? 6 : quads > 16 ? 5 : 4;
    const int q = threadIdx.x & ((1 << lanes_log) - 1), at_once = 256 >> lanes_log;
    if (q >= quads) return;
    for (int r = blockIdx.y * at_once + (threadIdx.x >> lanes_log); r < count; r += gridDim.y * at_once) {
        float m = -INFINITY, l = 0.0f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        // no part past the slots, were starts to go back
        const int parts = min(line.parts, (a.most - kv + a.pool.n_kv - 1) / a.pool.n_kv - n);
#pragma unroll 4
        for (int p = 0; p < parts; ++p) {
            const int64_t slot = ((int64_t)(n + p) * a.pool.n_kv + kv) * kRows + r;
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
        const int row = survivors.row(row0 + r), token = row / a.group, head = kv * a.group + (row - token * a.group);
        const int64_t at = line.seq.first + token;
        const bool none = m == -INFINITY || (a.mask && !a.mask[at * a.n_heads + head]);
        const float by = 1.0f / l;
        const float v[4] = {none ? 0.0f : o.x * by, none ? 0.0f : o.y * by, none ? 0.0f : o.z * by, none ? 0.0f : o.w * by};
        store_four(static_cast<Row *>(a.out) + (at * a.n_heads + head) * a.D + q * 4, v);
    }
}

// With a mask, before the others: lists the rows that survive, so that blocks are of those alone, and gives 0 to the rest.  Workgroups stand for a sequence (x) and a cache
// head (y); those of one pair (z) take kScan of its rows each in turn, and count the survivors before them.
constexpr int kScan = 512;
template <typename Row>
__global__ __launch_bounds__(256) void chunk_rows(ChunkArgs a)
{
    constexpr int kEach = kScan / 256;
    __shared__ int s_count[4 * kEach];
    __shared__ uint64_t s_bits[4 * kEach];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kv = blockIdx.y;
    const Sequence s = sequence(a, blockIdx.x);
    const int rows = s.fresh * a.group, pieces = a.D * (int)sizeof(Row) / 16;
    const uint8_t *mask = a.mask + (int64_t)s.first * a.n_heads + kv * a.group;
    int32_t *list = a.kept + ((int64_t)kv * a.N + s.first) * a.group;
    auto kept = [&](int r) {
        if (r >= rows) return false;
        const int token = r / a.group;
        return mask[(int64_t)token * a.n_heads + (r - token * a.group)] != 0;
    };
    if (rows == 0 && blockIdx.z == 0 && tid == 0) a.n_kept[(int64_t)kv * a.n_seq + blockIdx.x] = 0;
    int place = 0, counted = 0;                      // survivors before row `counted`
    for (int row0 = blockIdx.z * kScan; row0 < rows; row0 += gridDim.z * kScan) {
        int before = 0;
#pragma unroll 8
        for (int r = counted + tid; r < row0; r += 256) before += kept(r);
        before = __builtin_amdgcn_readlane(upto(before), 63);
        if (lane == 0) s_count[wave] = before;
        __syncthreads();
        place += s_count[0] + s_count[1] + s_count[2] + s_count[3];
        __syncthreads();
        bool mine[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            mine[i] = kept(row0 + i * 256 + tid);
            const uint64_t bits = __ballot(mine[i]);
            if (lane == 0) s_count[i * 4 + wave] = __popcll(bits), s_bits[i * 4 + wave] = bits;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4 * kEach; ++i) {
            if (i % 4 == wave && mine[i / 4]) list[place + __popcll(s_bits[i] & ((1ull << lane) - 1))] = row0 + i / 4 * 256 + tid;
            place += s_count[i];
        }
        counted = row0 + kScan;
        if (tid == 0 && counted >= rows) a.n_kept[(int64_t)kv * a.n_seq + blockIdx.x] = place;
        const int count = min(rows - row0, kScan);
        for (int r = tid >> 4; r < count; r += 16) { // 16 lanes a row
            if ((s_bits[r / 64] >> (r & 63)) & 1) continue;
            const int token = (row0 + r) / a.group;
            Row *out = static_cast<Row *>(a.out) + ((int64_t)(s.first + token) * a.n_heads + kv * a.group + (row0 + r - token * a.group)) * a.D;
            for (int piece = tid & 15; piece < pieces; piece += 16) reinterpret_cast<u32x4 *>(out)[piece] = u32x4{0u, 0u, 0u, 0u};
        }
        __syncthreads();                             // before the counts are written again
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
    // of a cache head at most: for a call whose starts go back, what is beyond is left out
    const int64_t heads = a.pool.n_kv, blocks = most_blocks(a, L::kRows);
    int64_t grid = blocks;
    const bool cut = blocks < L::kCuts && a.max_len > kLeast * L::TT;
    if (cut) {
        grid += L::kCuts;                              // a part more than even shares give, for each block
        a.slots = (int)grid;
    }
    a.most = (int)grid;
    grid = (grid + kDies - 1) / kDies * kDies;
    // Blocks of the surviving rows alone save their share of the products, and cost a launch and blocks that end where their sequence does more often.  us, without / with the list:
    // 7 sequences of 4099 in all, 40 heads, three quarters of them kept (1.5e8 scores of the longest sequence) 77 / 85; 4 of 4000, 32 heads, half (2e8) 79 / 72; one of 4096 (5e8)
    // 172 / 147, of 8192 564 / 353, with three quarters 540 / 465; 2 of 4000 in all after 2000, 64 heads, 8 cache heads, half 372 / 234, three quarters 355 / 302.  With nearly all kept it costs: 31 of
    // 32 heads, one of 4096 150 / 165, of 8192 550 / 569, 2 of 4000 after 2000 355 / 373.
    if (!a.mask || (int64_t)a.N * a.n_heads * a.max_len < 200000000) {
        a.kept = nullptr;
    } else {
        const int64_t scans = ((int64_t)a.N * a.group + kScan - 1) / kScan, pairs = (int64_t)a.n_seq * heads;
        const int64_t each = pairs < 2048 ? 2048 / pairs : 1;        // eight workgroups a unit
        chunk_rows<typename Kind::Row><<<dim3(a.n_seq, (unsigned)heads, (unsigned)(each < scans ? each : scans)), dim3(256), 0, s>>>(a);
        if (hipGetLastError() != hipSuccess) return HALO_ERR_HIP;
    }
    chunk_attend<Kind, DP, EXACT, WR, WK><<<dim3((unsigned)grid), dim3(L::kThreads), 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return HALO_ERR_HIP;
    if (!cut) return HALO_OK;
    chunk_join<typename Kind::Row, L::kRows, L::TT, L::kCuts><<<dim3((unsigned)(blocks / heads), (L::kRows * (a.D / 4) + 511) / 512, (unsigned)heads), dim3(256), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}

template <typename Kind, int DP, bool EXACT>
int launch_chunk(const ChunkArgs &a, hipStream_t s)
{
    // waves of a wide block: of eight a SIMD has two, 256 registers each, which long rows and rows of three parts pass
    constexpr int kWide = DP * (Kind::kC > Kind::kQ ? Kind::kC : Kind::kQ) > 128 ? 4 : 8;
    const int64_t rows = (int64_t)a.N * a.group;     // against those of all sequences in even blocks
    if constexpr (DP <= 128 && DP * Kind::kC <= 256) {       // four waves that share rows: LDS and registers for 128 tokens
        if (rows <= (int64_t)kCol * a.n_seq) return launch_rows<Kind, DP, EXACT, 1, 4>(a, s);
    }
    if constexpr (kWide == 8) {
        // Blocks of 128 rows, two waves for the same, where rows are few, and where wide blocks would be one round of unequal ones.  us, 256 rows / 128: 16 sequences of 40 new
        // tokens after 3000, 64 heads, 8 cache heads (288 blocks) 101 / 93; one of 2048, 32 heads, half kept (288) 80 / 63; 4 of 4000 in all (620) 79 / 98; 7 of 4099, 40 heads (920)
        // 77 / 103; cut blocks: 4 of 400 in all after 2000 (132) 51 / 55, one of 1024 after 2000 (160) 76 / 72.
        const int64_t wide = most_blocks(a, 8 * kCol);
        if (rows <= (int64_t)4 * kCol * a.n_seq || (wide >= 256 && wide < 512)) return launch_rows<Kind, DP, EXACT, 4, 2>(a, s);
    }
    return launch_rows<Kind, DP, EXACT, kWide, 1>(a, s);
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
