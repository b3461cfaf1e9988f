// Attention of one new token of each of T sequences over a paged cache (halo_paged_attention):
//     o_h = sum_j p_j V_j,  p = softmax_j(scale q_h . K_j),  j < len
// one pass over the rows with the running maximum and sum of the softmax.  Bytes bound it: a cached element meets `group` queries,
// 4 * group / 2 operations a byte in bf16, where this card has about 200 to spare.
//
// A wave is the worker.  The queries of one cache head (up to 16: a unit) are the 16 columns of the matrix instruction, so that grouped heads share
// what is read; with one query a column of 16 is used, and the matrix cores still outrun the stream.  Nothing passes through LDS on the way:
//   S^T = K Q^T      rows = tokens, columns = queries.  A lane (row = lane & 15) holds 16-byte pieces of its token's row as they lie in memory.
//                    The result leaves lane (c = lane & 15, g = lane >> 4) with query c's scores of the tokens 4g .. 4g+3 of each 16.
//   O^T += V^T P^T   the sum over tokens may take them in any order, so the operand P^T is what the lane already holds: its own
//                    scores' exponentials.  V^T then wants, in lane (c, g), those tokens' values of one dimension.  The lane loads
//                    whole 16-byte pieces of the same tokens' rows (piece c: coalesced) and pairs up halves of registers; the dimension
//                    that row c of instruction j stands for is c * VEC + j, which only the place of the results in memory has to know.
// Maximum and sum of a query then live in its column's lanes, as do its outputs: rescaling needs no exchange.
//
// How the work is cut: with short caches one workgroup takes a (sequence, unit) pair, its waves the tokens, joined in LDS (one launch).  Otherwise every wave of
// a grid that fills the card takes an even share of all tiles of all pairs (paged_index.hpp), whatever the lengths, and a second launch joins
// the pairs that were cut.
#include "../../include/halo.h"

#include <cmath>
#include <type_traits>

#include "kernels.hpp"
#include "paged_index.hpp"

namespace halo {
namespace {

constexpr int kCols = 16;                            // queries of a unit at most: columns of the matrix instruction
constexpr int kStreamWaves = 4;                      // waves of a workgroup of the even shares
constexpr int kStreamGrid = 512;                     // two such workgroups on each of 256 compute units
constexpr int kMaxWorkers = kStreamGrid * kStreamWaves;
constexpr int kMaxSeqs = 4096;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct AttendArgs {
    const void *q, *k, *v;
    const int32_t *table, *lens;
    const uint8_t *mask;
    void *out;
    float *part, *stats;                             // partial results of cut pairs: [slot][rows][D], [slot][rows][max, sum]
    int32_t *plan;                                   // [0] tiles per worker, [1 + t] first tile of sequence t
    int64_t q_stride;
    PagePool pool;
    int T, n_heads, group, n_qt, n_units, rows, D, max_pages, max_len;
    float scale2;                                    // scale * log2(e): the softmax is computed in powers of two
    int least;                                       // tiles that a worker takes at least
};

__device__ __forceinline__ float xor_max16_32(float v)
{
    auto as_f = [](unsigned u) { return __builtin_bit_cast(float, u); };
    unsigned u = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    u = __builtin_bit_cast(unsigned, fmaxf(as_f(a[0]), as_f(a[1])));
    const auto b = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(as_f(b[0]), as_f(b[1]));
}

// The running softmax of one unit over bf16 rows: 32 tokens a step.  DP = head dimension, or the next of 64, 128, 256 above it (EXACT false).
template <int DP, bool EXACT>
struct CoreBf16 {
    typedef bf16_t Elem;
    static constexpr int kTile = 32, kSub = 2;       // tokens a step, 16-token rows of the matrix instruction in it
    static constexpr int kItemWaves = DP > 128 ? 4 : 8;     // waves of a workgroup that takes a pair: rows of 256 need more than 256 registers
    static constexpr int KS = DP / 32;               // pieces of a key row in a lane
    static constexpr int VEC = DP >= 128 ? 8 : 4, VH = DP >= 128 ? DP / 128 : 1, kAcc = VEC * VH;
    typedef std::conditional_t<VEC == 8, u32x4, u32x2> VPiece;

    u32x4 qf[KS], kf[2][KS];
    VPiece vf[8][VH];
    f32x4 acc[kAcc], sum;
    float m;
    uint32_t koff[KS], voff[VH];
    bool kin[KS];
    int D, c, g;

    __device__ __forceinline__ void place(int d, int lane)
    {
        D = EXACT ? DP : d;
        c = lane & 15;
        g = lane >> 4;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int dim = s * 32 + g * 8;
            kin[s] = EXACT || dim < D;
            koff[s] = (uint32_t)(c * D + (kin[s] ? dim : 0)) * 2;
        }
#pragma unroll
        for (int h = 0; h < VH; ++h) {
            const int dim = h * 16 * VEC + c * VEC;
            voff[h] = (uint32_t)(g * 4 * D + (EXACT || dim < D ? dim : 0)) * 2;     // past the row's end: not stored
        }
    }
    __device__ __forceinline__ void begin(const bf16_t *q, int nq)
    {
#pragma unroll
        for (int s = 0; s < KS; ++s)
            qf[s] = c < nq && kin[s] ? *reinterpret_cast<const u32x4 *>(q + c * D + s * 32 + g * 8) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        sum = f32x4{0.f, 0.f, 0.f, 0.f};
        m = -INFINITY;
    }
    __device__ __forceinline__ void load_k(const char *const (&base)[kSub])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[i][s] = *reinterpret_cast<const u32x4 *>(base[i] + koff[s]);
    }
    __device__ __forceinline__ void load_v(const char *const (&base)[kSub])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int h = 0; h < VH; ++h)
                vf[i][h] = *reinterpret_cast<const VPiece *>(base[i >> 2] + (i & 3) * D * 2 + voff[h]);
    }
    static __device__ __forceinline__ f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &acc)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    }
    __device__ __forceinline__ void scores(float (&x)[8])
    {
        f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                u32x4 a = kf[i][k];
                if constexpr (!EXACT) a = kin[k] ? a : u32x4{0u, 0u, 0u, 0u};
                s[i] = mfma(a, qf[k], s[i]);
            }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3];
    }
    // token of the lane's e-th score, from the step's first
    __device__ __forceinline__ int token(int e) const { return (e >> 2) * 16 + g * 4 + (e & 3); }
    __device__ __forceinline__ void clear_v(int e)
    {
#pragma unroll
        for (int h = 0; h < VH; ++h) vf[e][h] = VPiece{};
    }
    __device__ __forceinline__ void rescale(float by)
    {
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[j] *= by;
        sum *= by;
    }
    // The probabilities are rounded to bf16 here, and the sum is of the rounded ones: weights that add up to one, so that a row with one
    // dominant token comes out as that token's values.
    __device__ __forceinline__ void accumulate(const float (&p)[8])
    {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        auto pair = [&](float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); };
        const u32x4 pf = {pair(p[0], p[1]), pair(p[2], p[3]), pair(p[4], p[5]), pair(p[6], p[7])};
        const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        sum = mfma(ones, pf, sum);
#pragma unroll
        for (int h = 0; h < VH; ++h)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
                u32x4 a;
#pragma unroll
                for (int t = 0; t < 4; ++t) a[t] = __builtin_amdgcn_perm(vf[2 * t + 1][h][j >> 1], vf[2 * t][h][j >> 1], sel);
                acc[h * VEC + j] = mfma(a, pf, acc[h * VEC + j]);
            }
    }
    __device__ __forceinline__ float total() const { return sum[0]; }
};

// The same over float rows: 16 tokens a step, every operand one float a lane.
template <int DP, bool EXACT>
struct CoreF32 {
    typedef float Elem;
    static constexpr int kTile = 16, kSub = 1;
    static constexpr int kItemWaves = DP > 128 ? 4 : 8;
    static constexpr int KS = DP / 16, VEC = 4, VH = DP / 64, kAcc = VEC * VH;

    f32x4 qf[KS], kf[KS], vf[4][VH], acc[kAcc];
    float m, l;
    uint32_t koff[KS], voff[VH];
    bool kin[KS];
    int D, c, g;

    __device__ __forceinline__ void place(int d, int lane)
    {
        D = EXACT ? DP : d;
        c = lane & 15;
        g = lane >> 4;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            kin[s] = EXACT || s * 16 < D;            // D is a multiple of 16
            koff[s] = (uint32_t)(c * D + (kin[s] ? s * 16 + g * 4 : 0)) * 4;
        }
#pragma unroll
        for (int h = 0; h < VH; ++h) {
            const int dim = h * 64 + c * 4;
            voff[h] = (uint32_t)(g * 4 * D + (EXACT || dim < D ? dim : 0)) * 4;
        }
    }
    __device__ __forceinline__ void begin(const float *q, int nq)
    {
#pragma unroll
        for (int s = 0; s < KS; ++s)
            qf[s] = c < nq && kin[s] ? *reinterpret_cast<const f32x4 *>(q + c * D + s * 16 + g * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        l = 0.0f;
        m = -INFINITY;
    }
    __device__ __forceinline__ void load_k(const char *const (&base)[kSub])
    {
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[s] = *reinterpret_cast<const f32x4 *>(base[0] + koff[s]);
    }
    __device__ __forceinline__ void load_v(const char *const (&base)[kSub])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < VH; ++h) vf[i][h] = *reinterpret_cast<const f32x4 *>(base[0] + i * D * 4 + voff[h]);
    }
    __device__ __forceinline__ void scores(float (&x)[4])
    {
        f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = EXACT || kin[k] ? kf[k][e] : 0.0f;
                s[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, qf[k][e], s[e & 1], 0, 0, 0);
            }
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = s[0][e] + s[1][e];
    }
    __device__ __forceinline__ int token(int e) const { return g * 4 + e; }
    __device__ __forceinline__ void clear_v(int e)
    {
#pragma unroll
        for (int h = 0; h < VH; ++h) vf[e][h] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void rescale(float by)
    {
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[j] *= by;
        l *= by;
    }
    __device__ __forceinline__ void accumulate(const float (&p)[4])
    {
        l += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kAcc; ++j)
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i][j >> 2][j & 3], p[i], acc[j], 0, 0, 0);
    }
    __device__ __forceinline__ float total() const { return xor_add<16>(xor_add<32>(l)); }
};

// The pages of one sequence: 64 entries of its row of the table at a time, one a lane.  All calls are wave-uniform.
struct PageRow {
    const int32_t *row;
    int n, first, id, lane;

    __device__ __forceinline__ PageRow(const AttendArgs &a, int t, int page, int lane)
        : row(a.table + (int64_t)t * a.max_pages), n(a.max_pages), lane(lane)
    {
        fetch(page);
    }
    __device__ __forceinline__ void fetch(int page)
    {
        first = page;
        id = page + lane < n ? row[page + lane] : -1;
        asm volatile("" : "+v"(id));                 // waited for here, and not at every use of a step that fetched nothing
    }
    __device__ __forceinline__ int operator[](int page)
    {
        if (page - first >= kWave) fetch(page);
        return __builtin_amdgcn_readlane(id, page - first);
    }
};

// Where a step's rows are, and whether all of them count.  Rows of a page that does not exist are replaced by the pool's first ones: loads need no
// condition, and what they bring is masked.
template <typename Core>
struct Step {
    const char *k[Core::kSub], *v[Core::kSub];
    int live[Core::kSub];                            // tokens of the 16 that count
    bool whole;

    __device__ __forceinline__ Step(const AttendArgs &a, PageRow &pages, int kv, int len, int tile)
    {
        whole = true;
#pragma unroll
        for (int i = 0; i < Core::kSub; ++i) {
            const int pos = tile * Core::kTile + i * 16;
            const int64_t row = pos < len ? paged_row(a.pool, pages[pos >> a.pool.page_shift], kv, pos) : -1;
            live[i] = row < 0 ? 0 : len - pos < 16 ? len - pos : 16;
            whole = whole && live[i] == 16;
            const int64_t at = (row < 0 ? 0 : row) * a.D * (int)sizeof(typename Core::Elem);
            k[i] = static_cast<const char *>(a.k) + at;
            v[i] = static_cast<const char *>(a.v) + at;
        }
    }
};

// The part of a step between its products: scores -> probabilities, with the running maximum.  The maximum only moves when a score passes it by 8
// (a factor of 256, which float sums take with ease), so that most steps rescale nothing.
template <typename Core, int N>
__device__ __forceinline__ void softmax_step(Core &core, const Step<Core> &st, float scale2, float (&x)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] *= scale2;
    if (!st.whole) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = (core.token(e) & 15) < st.live[e >> 2] ? x[e] : -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
    top = xor_max16_32(top);
    const bool passed = top > core.m + 8.0f;
    if (__ballot(passed)) {
        const float to = passed ? top : core.m;      // a query's own scores decide: its result does not depend on its neighbours
        core.rescale(to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(core.m - to));
        core.m = to;
    }
    const float m = core.m == -INFINITY ? 0.0f : core.m;
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = __builtin_amdgcn_exp2f(x[e] - m);
}

// Tiles [b, e) of sequence t, unit (kv, first query): the next step's keys are asked for as soon as this one's are used up, and its
// values after this one's.
template <typename Core>
__device__ __forceinline__ void attend_tiles(const AttendArgs &a, Core &core, int t, int kv, int len, int b, int e, int lane)
{
    constexpr int N = 4 * Core::kSub;
    PageRow pages(a, t, (b * Core::kTile) >> a.pool.page_shift, lane);
    Step<Core> now(a, pages, kv, len, b);
    core.load_k(now.k);
    core.load_v(now.v);
    auto drop_absent = [&] {                         // probability 0, but whatever the row holds: not even NaN may reach the sums
        if (!now.whole) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if ((core.token(i) & 15) >= now.live[i >> 2]) core.clear_v(i);
        }
    };
    float x[N];
    for (int tile = b; tile + 1 < e; ++tile) {
        const Step<Core> next(a, pages, kv, len, tile + 1);
        core.scores(x);
        core.load_k(next.k);
        softmax_step(core, now, a.scale2, x);
        drop_absent();
        core.accumulate(x);
        core.load_v(next.v);
        now = next;
    }
    core.scores(x);
    softmax_step(core, now, a.scale2, x);
    drop_absent();
    core.accumulate(x);
}

struct Unit {
    int kv, head, nq;                                // cache head, first query head, queries
    __device__ __forceinline__ Unit(const AttendArgs &a, int u)
    {
        kv = u / a.n_qt;
        const int from = (u - kv * a.n_qt) * kCols;
        head = kv * a.group + from;
        nq = a.group - from < kCols ? a.group - from : kCols;
    }
};

__device__ __forceinline__ bool unit_alive(const AttendArgs &a, int t, int u)
{
    if (!a.mask) return true;
    const Unit unit(a, u);
    const uint8_t *m = a.mask + (int64_t)t * a.n_heads + unit.head;
    int any = 0;
    for (int i = 0; i < unit.nq; ++i) any |= m[i];
    return any != 0;
}

__device__ __forceinline__ bool head_alive(const AttendArgs &a, int t, int head)
{
    return !a.mask || a.mask[(int64_t)t * a.n_heads + head] != 0;
}

__device__ __forceinline__ void store_piece(float *p, const float (&v)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store_piece(float *p, const float (&v)[8]) { store8(p, v); }
__device__ __forceinline__ void store_piece(bf16_t *p, const float (&v)[8]) { store8(p, v); }
__device__ __forceinline__ void store_piece(bf16_t *p, const float (&v)[4])
{
    *reinterpret_cast<uint2 *>(p) = make_uint2((uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
                                               (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
}

// A lane's results are runs of VEC dimensions of query c: row 4g + r of instruction (h, j) is dimension h * 16 VEC + (4g + r) * VEC + j.
template <typename Core, typename OT>
__device__ __forceinline__ void store_rows(const Core &core, OT *rows, int nq, float by)
{
    if (core.c >= nq) return;
#pragma unroll
    for (int h = 0; h < Core::VH; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dim = h * 16 * Core::VEC + (core.g * 4 + r) * Core::VEC;
            float v[Core::VEC];
#pragma unroll
            for (int j = 0; j < Core::VEC; ++j) v[j] = by == 0.0f ? 0.0f : core.acc[h * Core::VEC + j][r] * by;
            if (dim < core.D) store_piece(rows + (int64_t)core.c * core.D + dim, v);
        }
}

template <typename Core>
__device__ __forceinline__ void store_out_rows(const AttendArgs &a, const Core &core, int t, const Unit &unit)
{
    const float l = core.total();
    const bool alive = core.c < unit.nq && head_alive(a, t, unit.head + core.c);
    // a sum of 0 is a row without positions; NaN has to come through
    store_rows(core, static_cast<typename Core::Elem *>(a.out) + ((int64_t)t * a.n_heads + unit.head) * core.D, unit.nq,
               !alive || l == 0.0f ? 0.0f : 1.0f / l);
}

// ---------------------------------------------------------------------------
// one workgroup a pair
// ---------------------------------------------------------------------------
template <typename Core>
__global__ __launch_bounds__(Core::kItemWaves * 64) void attend_item(AttendArgs a)
{
    constexpr int kItemWaves = Core::kItemWaves;
    extern __shared__ __align__(16) float s_part[];  // [waves][rows][D], then [waves][16][max, sum]
    float *s_stats = s_part + kItemWaves * a.rows * a.D;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = blockIdx.x / a.n_units, u = blockIdx.x - t * a.n_units;
    const Unit unit(a, u);
    const int len = paged_length(a.lens[t], a.max_len);
    const int tiles = unit_alive(a, t, u) ? (len + Core::kTile - 1) / Core::kTile : 0;
    const int b = tiles * wave / kItemWaves, e = tiles * (wave + 1) / kItemWaves;
    Core core;
    core.place(a.D, lane);
    core.begin(static_cast<const typename Core::Elem *>(a.q) + t * a.q_stride + unit.head * core.D, unit.nq);
    if (b < e) attend_tiles(a, core, t, unit.kv, len, b, e, lane);
    const float l = core.total();
    if (core.g == 0) {
        s_stats[(wave * kCols + core.c) * 2] = core.m;
        s_stats[(wave * kCols + core.c) * 2 + 1] = l;
    }
    if (b < e) store_rows(core, s_part + wave * a.rows * core.D, unit.nq, 1.0f);
    __syncthreads();
    typename Core::Elem *out = static_cast<typename Core::Elem *>(a.out) + ((int64_t)t * a.n_heads + unit.head) * core.D;
    for (int i = threadIdx.x; i < unit.nq * core.D; i += kItemWaves * 64) {
        const int n = i / core.D;
        float top = -INFINITY, sum = 0.0f, o = 0.0f;
#pragma unroll
        for (int w = 0; w < kItemWaves; ++w) top = fmaxf(top, s_stats[(w * kCols + n) * 2]);
        for (int w = 0; w < kItemWaves; ++w) {
            const float ml = s_stats[(w * kCols + n) * 2], ll = s_stats[(w * kCols + n) * 2 + 1];
            if (ll == 0.0f) continue;                // no positions: nothing was stored
            const float by = __builtin_amdgcn_exp2f(ml - top);
            sum += ll * by;
            o += s_part[(w * a.rows) * core.D + i] * by;
        }
        store_out(out + i, sum == 0.0f || !head_alive(a, t, unit.head + n) ? 0.0f : o / sum);
    }
}

// ---------------------------------------------------------------------------
// even shares of all tiles
// ---------------------------------------------------------------------------
// s_base[t] = tiles of the sequences before t, s_base[T] = all.  Called by the whole workgroup.
template <int kTile>
__device__ __forceinline__ void line_up(const AttendArgs &a, int *s_base, int *s_wave)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, threads = kStreamWaves * 64;
    for (int t = tid; t < a.T; t += threads) s_base[t] = a.mask ? 0 : a.n_units;
    __syncthreads();
    if (a.mask) {
        for (int i = tid; i < a.T * a.n_units; i += threads) {
            const int t = i / a.n_units;
            if (unit_alive(a, t, i - t * a.n_units)) atomicAdd(&s_base[t], 1);       // integers: any order gives the same count
        }
        __syncthreads();
    }
    const int each = (a.T + threads - 1) / threads, from = min(tid * each, a.T), to = min(from + each, a.T);
    int mine = 0;
    for (int t = from; t < to; ++t) {
        const int n = s_base[t] * ((paged_length(a.lens[t], a.max_len) + kTile - 1) / kTile);
        s_base[t] = mine;
        mine += n;
    }
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int before = upto - mine;
    for (int w = 0; w < wave; ++w) before += s_wave[w];
    for (int t = from; t < to; ++t) s_base[t] += before;
    if (tid == threads - 1) s_base[a.T] = before + mine;
    __syncthreads();
}

// The surviving units of a sequence in order, 64 of them looked at at a time.
struct AliveUnits {
    uint64_t bits;
    int block;

    __device__ __forceinline__ void look(const AttendArgs &a, int t, int from, int lane)
    {
        block = from;
        const int u = from + lane;
        bits = __ballot(u < a.n_units && unit_alive(a, t, u));
    }
    // the n-th, which exists
    __device__ __forceinline__ void find(const AttendArgs &a, int t, int n, int lane)
    {
        look(a, t, 0, lane);
        for (int c; n >= (c = __popcll(bits)); n -= c) look(a, t, block + 64, lane);
        for (; n > 0; --n) bits &= bits - 1;
    }
    __device__ __forceinline__ int unit() const { return block + __ffsll((unsigned long long)bits) - 1; }
    __device__ __forceinline__ void next(const AttendArgs &a, int t, int lane)
    {
        bits &= bits - 1;
        while (!bits && block + 64 < a.n_units) look(a, t, block + 64, lane);
    }
};

template <typename Core>
__global__ __launch_bounds__(kStreamWaves * 64) void attend_stream(AttendArgs a)
{
    __shared__ int s_base[kMaxSeqs + 1], s_wave[kStreamWaves];
    line_up<Core::kTile>(a, s_base, s_wave);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    auto base = [&](int t) { return __builtin_amdgcn_readfirstlane(s_base[t]); };
    const int total = base(a.T), per = tiles_per_worker(total, gridDim.x * kStreamWaves, a.least);
    if (blockIdx.x == 0) {                           // for the second launch
        for (int t = threadIdx.x; t < a.T; t += kStreamWaves * 64) a.plan[1 + t] = s_base[t];
        if (threadIdx.x == 0) a.plan[0] = per;
    }
    const int worker = blockIdx.x * kStreamWaves + wave;
    if ((int64_t)worker * per >= total) return;
    int at = worker * per;
    const int end = min(at + per, total);
    int lo = 0, hi = a.T;                            // the sequence whose tiles hold `at`: base[lo] <= at < base[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (base(mid) <= at) lo = mid; else hi = mid;
    }
    Core core;
    core.place(a.D, lane);
    AliveUnits units;
    for (int t = lo; at < end; ++t) {
        const int from = base(t), size = base(t + 1) - from;
        if (size == 0) continue;
        const int len = paged_length(__builtin_amdgcn_readfirstlane(a.lens[t]), a.max_len);
        const int tiles = (len + Core::kTile - 1) / Core::kTile;
        int n = (at - from) / tiles;
        units.find(a, t, n, lane);
        for (; at < end && at < from + size; ++n, units.next(a, t, lane)) {
            const Unit unit(a, units.unit());
            const int offset = from + n * tiles, b = at - offset, e = min(tiles, end - offset);
            core.begin(static_cast<const typename Core::Elem *>(a.q) + t * a.q_stride + unit.head * core.D, unit.nq);
            attend_tiles(a, core, t, unit.kv, len, b, e, lane);
            at = offset + e;
            if (b == 0 && e == tiles) {
                store_out_rows(a, core, t, unit);
                continue;
            }
            const int64_t slot = partial_slot(worker, per, offset);
            const float l = core.total();
            if (core.g == 0 && core.c < unit.nq)
                *reinterpret_cast<float2 *>(a.stats + (slot * a.rows + core.c) * 2) = make_float2(core.m, l);
            store_rows(core, a.part + slot * a.rows * core.D, unit.nq, 1.0f);
        }
    }
}

// Joins the pairs that more than one worker had, and gives 0 to those that nobody had.  A workgroup a pair: its threads stand for four
// dimensions of one query each, several of them sharing the partial results where there are threads to spare.
template <typename Core>
__global__ __launch_bounds__(256) void attend_join(AttendArgs a)
{
    __shared__ float4 s_o[256];
    __shared__ float2 s_ml[256];
    typedef typename Core::Elem Elem;
    const int lane = threadIdx.x & 63, tid = threadIdx.x;
    const int t = blockIdx.x / a.n_units, u = blockIdx.x - t * a.n_units;
    const Unit unit(a, u);
    const int per = a.plan[0], from = a.plan[1 + t];
    const int tiles = (paged_length(a.lens[t], a.max_len) + Core::kTile - 1) / Core::kTile;
    int rank = u;
    bool alive = true;
    if (a.mask) {
        rank = 0;
        for (int block = 0; block <= u; block += 64) {
            const uint64_t bits = __ballot(block + lane < a.n_units && unit_alive(a, t, block + lane));
            rank += __popcll(u - block < 64 ? bits & ((1ull << (u - block)) - 1) : bits);
            if (u - block < 64) alive = (bits >> (u - block)) & 1;
        }
    }
    const int offset = from + rank * tiles;
    const bool any = alive && tiles > 0;
    const int w0 = any ? first_worker(offset, per) : 0, w1 = any ? last_worker(offset, tiles, per) : -1;
    if (any && w0 == w1) return;                     // written by that worker
    Elem *out = static_cast<Elem *>(a.out) + ((int64_t)t * a.n_heads + unit.head) * a.D;
    const int quads = unit.nq * (a.D / 4);           // at least 4
    const int parts = quads < 256 ? 256 / quads : 1, part = quads < 256 ? tid / quads : 0;
    for (int block = 0; block < quads; block += 256) {
        const int i = quads < 256 ? tid - part * quads : block + tid;
        const int n = min(i / (a.D / 4), unit.nq - 1);
        float m = -INFINITY, l = 0.0f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < quads && part < parts) {
#pragma unroll 4
            for (int w = w0 + part; w <= w1; w += parts) {
                const int64_t slot = partial_slot(w, per, offset);
                const float2 ml = *reinterpret_cast<const float2 *>(a.stats + (slot * a.rows + n) * 2);
                const float4 p = *reinterpret_cast<const float4 *>(a.part + slot * a.rows * a.D + i * 4);
                const float to = fmaxf(m, ml.x), use = to == -INFINITY ? 0.0f : to;
                const float keep = __builtin_amdgcn_exp2f(m - use), by = __builtin_amdgcn_exp2f(ml.x - use);
                l = l * keep + ml.y * by;
                o.x = o.x * keep + p.x * by;
                o.y = o.y * keep + p.y * by;
                o.z = o.z * keep + p.z * by;
                o.w = o.w * keep + p.w * by;
                m = to;
            }
        }
        if (parts > 1) {                             // the same for every thread
            s_o[tid] = o;
            s_ml[tid] = make_float2(m, l);
            __syncthreads();
            if (part == 0)
                for (int k = 1; k < parts; ++k) {
                    const float2 ml = s_ml[k * quads + tid];
                    const float4 p = s_o[k * quads + tid];
                    const float to = fmaxf(m, ml.x), use = to == -INFINITY ? 0.0f : to;
                    const float keep = __builtin_amdgcn_exp2f(m - use), by = __builtin_amdgcn_exp2f(ml.x - use);
                    l = l * keep + ml.y * by;
                    o.x = o.x * keep + p.x * by;
                    o.y = o.y * keep + p.y * by;
                    o.z = o.z * keep + p.z * by;
                    o.w = o.w * keep + p.w * by;
                    m = to;
                }
        }
        if (part == 0 && i < quads) {
            const bool none = l == 0.0f || !head_alive(a, t, unit.head + n);
            const float v[4] = {none ? 0.0f : o.x / l, none ? 0.0f : o.y / l, none ? 0.0f : o.z / l, none ? 0.0f : o.w / l};
            store_piece(out + i * 4, v);
        }
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
inline size_t align256(size_t n) { return (n + 255) / 256 * 256; }

struct PagedWorkspace {
    size_t plan = 0, stats = 0, part = 0, bytes = 0;
    PagedWorkspace(const halo_paged_shape &s, int T)
    {
        const size_t group = s.n_heads / s.n_kv_heads, rows = group < kCols ? group : kCols;
        const size_t slots = 2 * (size_t)kMaxWorkers;
        stats = align256(((size_t)T + 1) * sizeof(int32_t));
        part = stats + align256(slots * rows * 2 * sizeof(float));
        bytes = part + align256(slots * rows * s.head_dim * sizeof(float));
    }
};

template <typename Core>
int launch_core(const AttendArgs &a, bool one_launch, int bound, hipStream_t s)
{
    if (one_launch) {
        constexpr int kItemWaves = Core::kItemWaves;
        const size_t lds = (size_t)kItemWaves * ((size_t)a.rows * a.D + 2 * kCols) * sizeof(float);
        if (lds > 65536 &&
            hipFuncSetAttribute(reinterpret_cast<const void *>(attend_item<Core>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
            return HALO_ERR_HIP;
        attend_item<Core><<<dim3(a.T * a.n_units), dim3(kItemWaves * 64), lds, s>>>(a);
    } else {
        const int wanted = (bound + kStreamWaves * a.least - 1) / (kStreamWaves * a.least);
        attend_stream<Core><<<dim3(wanted < kStreamGrid ? wanted : kStreamGrid), dim3(kStreamWaves * 64), 0, s>>>(a);
        if (hipGetLastError() != hipSuccess) return HALO_ERR_HIP;
        attend_join<Core><<<dim3(a.T * a.n_units), dim3(256), 0, s>>>(a);
    }
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}

template <template <int, bool> class Core>
int launch_dim(const AttendArgs &a, bool one_launch, int bound, hipStream_t s)
{
    if (a.D == 64) return launch_core<Core<64, true>>(a, one_launch, bound, s);
    if (a.D == 128) return launch_core<Core<128, true>>(a, one_launch, bound, s);
    if (a.D == 256) return launch_core<Core<256, true>>(a, one_launch, bound, s);
    if (a.D < 64) return launch_core<Core<64, false>>(a, one_launch, bound, s);
    if (a.D < 128) return launch_core<Core<128, false>>(a, one_launch, bound, s);
    return launch_core<Core<256, false>>(a, one_launch, bound, s);
}

}  // namespace

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

extern "C" int halo_paged_attention(const halo_paged_shape *shape, int32_t T, const void *q, int64_t q_stride, const void *k_pages,
                                    const void *v_pages, const int32_t *page_table, const int32_t *lens, int32_t max_len,
                                    const uint8_t *mask, float scale, void *out, void *workspace, size_t ws_bytes, void *stream)
{
    using namespace halo;
    if (const int rc = check_paged_shape(shape)) return rc;
    if (!q || !k_pages || !v_pages || !page_table || !lens || !out) return HALO_ERR_NULL;
    const halo_paged_shape &s = *shape;
    const int size = s.dtype == HALO_F32 ? 4 : 2, tile = s.dtype == HALO_F32 ? 16 : 32;
    auto odd = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; };
    if (T < 0 || T > kMaxSeqs || max_len < 1 || max_len > s.max_pages * s.page_size || !std::isfinite(scale)) return HALO_ERR_ARG;
    if (q_stride < (int64_t)s.n_heads * s.head_dim || q_stride * size % 16 || odd(q) || odd(k_pages) || odd(v_pages) || odd(out) ||
        odd(workspace) || (reinterpret_cast<uintptr_t>(page_table) & 3u) || (reinterpret_cast<uintptr_t>(lens) & 3u))
        return HALO_ERR_ARG;
    const PagedWorkspace ws(s, T);
    if (!workspace || ws_bytes < ws.bytes) return HALO_ERR_WORKSPACE;
    if (T == 0) return HALO_OK;

    AttendArgs a{};
    a.q = q; a.k = k_pages; a.v = v_pages; a.table = page_table; a.lens = lens; a.mask = mask; a.out = out;
    char *w = static_cast<char *>(workspace);
    a.plan = reinterpret_cast<int32_t *>(w + ws.plan);
    a.stats = reinterpret_cast<float *>(w + ws.stats);
    a.part = reinterpret_cast<float *>(w + ws.part);
    a.q_stride = q_stride;
    a.pool = PagePool{s.n_pages, s.n_kv_heads, __builtin_ctz((unsigned)s.page_size)};
    a.T = T; a.n_heads = s.n_heads; a.group = s.n_heads / s.n_kv_heads;
    a.n_qt = (a.group + kCols - 1) / kCols;
    a.n_units = s.n_kv_heads * a.n_qt;
    a.rows = a.group < kCols ? a.group : kCols;
    a.D = s.head_dim; a.max_pages = s.max_pages; a.max_len = max_len;
    a.scale2 = scale * 1.44269504088896341f;
    a.least = 4;
    const int64_t tiles = (max_len + tile - 1) / tile, bound = tiles * T * a.n_units;
    if (bound > (1 << 30)) return HALO_ERR_ARG;
    const bool one_launch = max_len <= 1024;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return s.dtype == HALO_F32 ? launch_dim<CoreF32>(a, one_launch, (int)bound, st) : launch_dim<CoreBf16>(a, one_launch, (int)bound, st);
}
