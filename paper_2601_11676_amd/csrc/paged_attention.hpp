// The kernels and launch rules of halo_paged_attention (paged_attention.hip, where their mathematics stands), for the files that make them for one type each.
#pragma once
#include "../../include/halo.h"

#include <cmath>
#include <type_traits>

#include "kernels.hpp"
#include "paged_index.hpp"

namespace halo {

struct AttendArgs {
    const void *q, *k, *v;
    const int32_t *table, *lens;
    const uint8_t *mask;
    void *out;
    float *part, *stats;                             // partial results of cut pairs: [slot][rows][D], [slot][rows][max, sum]
    int32_t *plan;                                   // [0] tiles per worker, [1] all tiles, [2 + t] first tile of sequence t
    int64_t q_stride;
    PagePool pool;
    int T, n_heads, group, n_qt, n_units, rows, D, max_pages, max_len;
    int64_t bytes;                                   // of the cache, for the host's choices
    float scale2;                                    // scale * log2(e): the softmax is computed in powers of two
};

namespace {

constexpr int kCols = 16;                            // columns of the matrix instruction: queries
constexpr int kUnits = 256;                          // compute units
constexpr int kMaxWorkers = 2 * kUnits * kTeam;      // even shares: two workgroups a unit
constexpr int kMaxSeqs = 4096;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// A value that is the same in every lane, said so: what descriptors are made of has to be in scalar registers (or each load becomes a loop over the lanes'
// descriptors).
__device__ __forceinline__ int same(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ float xor_max16_32(float v)
{
    auto as_f = [](unsigned u) { return __builtin_bit_cast(float, u); };
    unsigned u = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    u = __builtin_bit_cast(unsigned, fmaxf(as_f(a[0]), as_f(a[1])));
    const auto b = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(as_f(b[0]), as_f(b[1]));
}

// 16 rows of one page: what a descriptor lets a lane read.  Rows that do not count lie past its end and read as zeros, whatever memory holds there
// (a probability of 0 does not keep NaN out of a sum), and a page that does not exist is a descriptor of no bytes: loads need no condition.
template <typename V, int POLICY>
__device__ __forceinline__ V row_load(__amdgpu_buffer_rsrc_t rows, uint32_t at)
{
    if constexpr (sizeof(V) == 16)
        return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(rows, at, 0, POLICY));
    else
        return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(rows, at, 0, POLICY));
}

// Which of the cache's rows carry the non-temporal hint: none, the values, both.  What passes through once should not push out what stays; with
// caches that fit the dies' L2 the hint costs.  us, by the bytes of the call at its longest length, none / values / both: 33 MB 9.6 / 11.9 / 12.0; 131 MB 19.0 / 18.7 /
// 19.1; 262 MB 38.7 / 33.9 / 34.5; 524 MB 72.4 / 66.1 / 64.6; 885 MB 79.4 / 72.4 / 70.6; 3.2 GB 285 / 283 / 278.
enum { kKeepAll = 0, kPassValues = 1, kPassBoth = 2 };

// Keys on their way from whole rows, as they are loaded, to the lanes that multiply them: 16 rows of DP elements in LDS, piece p of row r at place
// p ^ r (within 16), so that neither side meets a bank twice.  kRows rows a load; the same number of loads as of pieces a lane gets.  (With each lane
// loading its pieces itself, 8 sequences of up to 1000 took 12.8 us, then 9.0.)
template <typename Elem, int DP>
struct KeyPlace {
    static constexpr int kBytes = DP * sizeof(Elem), kPieces = kBytes / 16, kRows = 64 / kPieces;
    static constexpr int kTurn = (kPieces < 16 ? kPieces : 16) - 1;
    uint32_t from, in, out;                          // offset in memory, places in LDS of the first load and of the first piece

    __device__ __forceinline__ void place(int D, int lane)
    {
        const int row = lane / kPieces, piece = lane % kPieces, c = lane & 15, g = lane >> 4;
        from = piece * 16 < D * (int)sizeof(Elem) ? (uint32_t)(row * D * (int)sizeof(Elem) + piece * 16) : kOutOfRange;
        in = row * kBytes + ((piece ^ row) << 4);
        out = c * kBytes + ((g ^ (c & kTurn)) << 4);
    }
    __device__ __forceinline__ uint32_t put(int i) const { return (in ^ ((i * kRows & kTurn) << 4)) + i * kRows * kBytes; }
    __device__ __forceinline__ uint32_t get(int s) const { return out ^ (s << 6); }
};

// Between LDS accesses of lanes that use each other's: the hardware keeps a wave's in order, so that there is nothing to wait for, but the compiler, which
// sees one lane, has to be told.  No instruction comes of it.
__device__ __forceinline__ void wave_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// A step's keys: loaded rows in, the lane's pieces out.
template <typename Core>
__device__ __forceinline__ void turn_keys(Core &core)
{
#pragma unroll
    for (int i = 0; i < Core::kSub; ++i)
#pragma unroll
        for (int s = 0; s < Core::KS; ++s) *reinterpret_cast<u32x4 *>(core.lds + i * 16 * core.keys.kBytes + core.keys.put(s)) = __builtin_bit_cast(u32x4, core.kf[i][s]);
    wave_in_order();
#pragma unroll
    for (int i = 0; i < Core::kSub; ++i)
#pragma unroll
        for (int s = 0; s < Core::KS; ++s) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(core.lds + i * 16 * core.keys.kBytes + core.keys.get(s));
            core.kf[i][s] = __builtin_bit_cast(std::remove_reference_t<decltype(core.kf[i][s])>, v);
        }
    wave_in_order();                                 // before the next step's rows, or the results, take the place
}

// The running softmax of one unit over bf16 rows, kSub times 16 tokens a step.  DP = head dimension, or the next of 64, 128, 256 above it (EXACT false).
template <int DP, bool EXACT, int HINT, int TILES>
struct CoreBf16 {
    typedef bf16_t Elem;
    static constexpr int QT = TILES;                 // times 16 queries: more than one where a cache head has more than 16
    static constexpr int kSub = DP > 64 ? 2 : 4, kTile = kSub * 16;      // rows of 128 and 64: 16 KiB of keys and values a step
    static constexpr int kItemWaves = DP > 128 ? 4 : 8;     // waves of a workgroup that takes a pair: rows of 256 need more than 256 registers
    static constexpr int kWaves = DP > 128 || (DP > 64 && QT > 1) ? 1 : 2;         // on a SIMD, for the same reason
    static constexpr int kSteps = DP > 64 ? 8 : 4, kLeast = DP > 128 ? 4 : 2;     // see launch_cut; tiles a worker takes at least
    static constexpr int kMostRows = QT * kCols * DP * 4, kStage = kTile * DP * 2 > kMostRows ? kTile * DP * 2 : kMostRows;    // LDS of a wave: a step's keys, in the end its part of the results
    static constexpr int KS = DP / 32;               // pieces of a key row in a lane
    static constexpr int VEC = DP > 64 ? 8 : 4, VH = DP > 128 ? 2 : 1, kAcc = VEC * VH;
    typedef std::conditional_t<VEC == 8, u32x4, u32x2> VPiece;

    u32x4 qf[QT][KS], kf[kSub][KS];
    VPiece vf[4 * kSub][VH];
    f32x4 acc[QT][kAcc], sum[QT];
    float m[QT];
    KeyPlace<bf16_t, DP> keys;
    char *lds;                                       // kStage bytes, the wave's own
    uint32_t voff[VH];
    int D, c, g;

    __device__ __forceinline__ void place(int d, int lane, char *own)
    {
        D = EXACT ? DP : d;
        c = lane & 15;
        g = lane >> 4;
        lds = own;
        keys.place(D, lane);
#pragma unroll
        for (int h = 0; h < VH; ++h) {
            const int dim = h * 16 * VEC + c * VEC;
            voff[h] = EXACT || dim < D ? (uint32_t)(g * 4 * D + dim) * 2 : kOutOfRange;
        }
    }
    __device__ __forceinline__ void begin(const bf16_t *q, int nq)
    {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                // columns past the last query repeat it: nobody reads their results
                const int n = min(t * kCols + c, nq - 1), dim = s * 32 + g * 8;
                qf[t][s] = *reinterpret_cast<const u32x4 *>(q + n * D + (EXACT || dim < D ? dim : 0));
                if constexpr (!EXACT) qf[t][s] = dim < D ? qf[t][s] : u32x4{0u, 0u, 0u, 0u};
            }
#pragma unroll
            for (int j = 0; j < kAcc; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[t] = -INFINITY;
        }
    }
    __device__ __forceinline__ void load_k(const __amdgpu_buffer_rsrc_t (&rows)[kSub])
    {
#pragma unroll
        for (int i = 0; i < kSub; ++i)
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[i][s] = row_load<u32x4, HINT == kPassBoth ? kNt : 0>(rows[i], keys.from + s * keys.kRows * D * 2);
    }
    __device__ __forceinline__ void load_v(const __amdgpu_buffer_rsrc_t (&rows)[kSub])
    {
#pragma unroll
        for (int i = 0; i < 4 * kSub; ++i)
#pragma unroll
            for (int h = 0; h < VH; ++h) vf[i][h] = row_load<VPiece, HINT != kKeepAll ? kNt : 0>(rows[i >> 2], voff[h] + (i & 3) * D * 2);
    }
    static __device__ __forceinline__ f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &acc)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    }
    // the lane's scores: 4i + r is token 16i + 4g + r of the step
    __device__ __forceinline__ void scores(float (&x)[QT][4 * kSub])
    {
        turn_keys(*this);
        f32x4 s[QT][kSub];
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int i = 0; i < kSub; ++i) s[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int t = 0; t < QT; ++t)
#pragma unroll
                for (int i = 0; i < kSub; ++i) s[t][i] = mfma(kf[i][k], qf[t][k], s[t][i]);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int e = 0; e < 4 * kSub; ++e) x[t][e] = s[t][e >> 2][e & 3];
    }
    __device__ __forceinline__ void rescale(int t, float by)
    {
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[t][j] *= by;
        sum[t] *= by;
    }
    // A probability goes to the matrix cores as three bf16 values, each what the ones before leave of it, rounded: three times eight bits are all that a float
    // has.  The sum is of the same values, so that the weights add up to one.  (Two of
    // them would leave up to 2^-17 of it.  us, two / three: one sequence of 301 5.1 / 5.3, 8 of up to 1000 9.5 / 9.8, heads of 256 15.1 / 16.4, 192 of up to 600
    // 58.7 / 61.4; large caches, also with 20 queries a cache head, level: the matrix cores have the time.)
    __device__ __forceinline__ void accumulate(const float (&p)[QT][4 * kSub])
    {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        auto pair = [](float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); };
        const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
        for (int o = 0; o < 4 * kSub; o += 8) {
            u32x4 part[QT][3];
#pragma unroll
            for (int q = 0; q < QT; ++q) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    float a = p[q][o + 2 * t], b = p[q][o + 2 * t + 1];
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        part[q][i][t] = pair(a, b);
                        a -= bf16_lo(part[q][i][t]);
                        b -= bf16_hi(part[q][i][t]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 3; ++i) sum[q] = mfma(ones, part[q][i], sum[q]);
            }
#pragma unroll
            for (int h = 0; h < VH; ++h)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
                    u32x4 a;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        a[t] = __builtin_amdgcn_perm(vf[o + 2 * t + 1][h][j >> 1], vf[o + 2 * t][h][j >> 1], sel);
#pragma unroll
                    for (int q = 0; q < QT; ++q)
#pragma unroll
                        for (int i = 0; i < 3; ++i) acc[q][h * VEC + j] = mfma(a, part[q][i], acc[q][h * VEC + j]);
                }
        }
    }
    // The lane's query of each 16, its first token of each 16, whether it is the one to store what several lanes hold; the maximum over a query's lanes; what is left
    // to do after the last step, and the query's sum.
    __device__ __forceinline__ int col() const { return c; }
    __device__ __forceinline__ int row() const { return g * 4; }
    __device__ __forceinline__ bool stores() const { return true; }
    __device__ __forceinline__ float top(float v) const { return xor_max16_32(v); }
    __device__ __forceinline__ void finish(float (&l)[QT])
    {
#pragma unroll
        for (int t = 0; t < QT; ++t) l[t] = sum[t][0];
    }
};

template <int DP, bool EXACT, int HINT> using CoreBf16One = CoreBf16<DP, EXACT, HINT, 1>;
template <int DP, bool EXACT, int HINT> using CoreBf16Two = CoreBf16<DP, EXACT, HINT, 2>;

// The same over float rows: every operand of the matrix instruction is one float a lane.  With 32 queries and rows of 128 one wave a SIMD, which has
// 350 registers; two with 256 each take 163 us where one takes 150 (24 sequences of 2500 to 5000, 8 cache heads of 20 queries; floor 106).  A workgroup that
// takes a pair has eight waves here too, which spill 9 registers with heads of 80 to 112.
template <int DP, bool EXACT, int HINT, int TILES>
struct CoreF32 {
    typedef float Elem;
    static constexpr int QT = TILES;
    static constexpr int kSub = DP > 64 ? 1 : 2, kTile = kSub * 16;
    static constexpr int kSteps = 4, kLeast = DP > 128 ? 4 : 2;
    static constexpr int kItemWaves = DP > 128 ? 4 : 8, kWaves = DP > 128 || (DP > 64 && QT > 1) ? 1 : 2;
    static constexpr int kMostRows = QT * kCols * DP * 4, kStage = kTile * DP * 4 > kMostRows ? kTile * DP * 4 : kMostRows;
    static constexpr int KS = DP / 16, VEC = 4, VH = DP / 64, kAcc = VEC * VH;

    f32x4 qf[QT][KS], kf[kSub][KS], vf[4 * kSub][VH], acc[QT][kAcc];
    float m[QT], l[QT];
    KeyPlace<float, DP> keys;
    char *lds;
    uint32_t voff[VH];
    int D, c, g;

    __device__ __forceinline__ void place(int d, int lane, char *own)
    {
        D = EXACT ? DP : d;
        c = lane & 15;
        g = lane >> 4;
        lds = own;
        keys.place(D, lane);
#pragma unroll
        for (int h = 0; h < VH; ++h) {
            const int dim = h * 64 + c * 4;
            voff[h] = EXACT || dim < D ? (uint32_t)(g * 4 * D + dim) * 4 : kOutOfRange;
        }
    }
    __device__ __forceinline__ void begin(const float *q, int nq)
    {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
#pragma unroll
            for (int s = 0; s < KS; ++s)
                qf[t][s] = EXACT || s * 16 < D ? *reinterpret_cast<const f32x4 *>(q + min(t * kCols + c, nq - 1) * D + s * 16 + g * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < kAcc; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            l[t] = 0.0f;
            m[t] = -INFINITY;
        }
    }
    __device__ __forceinline__ void load_k(const __amdgpu_buffer_rsrc_t (&rows)[kSub])
    {
#pragma unroll
        for (int i = 0; i < kSub; ++i)
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[i][s] = row_load<f32x4, HINT == kPassBoth ? kNt : 0>(rows[i], keys.from + s * keys.kRows * D * 4);
    }
    __device__ __forceinline__ void load_v(const __amdgpu_buffer_rsrc_t (&rows)[kSub])
    {
#pragma unroll
        for (int i = 0; i < 4 * kSub; ++i)
#pragma unroll
            for (int h = 0; h < VH; ++h) vf[i][h] = row_load<f32x4, HINT != kKeepAll ? kNt : 0>(rows[i >> 2], voff[h] + (i & 3) * D * 4);
    }
    __device__ __forceinline__ void scores(float (&x)[QT][4 * kSub])
    {
        turn_keys(*this);
        f32x4 s[QT][kSub][2];
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int i = 0; i < kSub; ++i) s[t][i][0] = s[t][i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int i = 0; i < kSub; ++i)
                        s[t][i][e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i][k][e], qf[t][k][e], s[t][i][e & 1], 0, 0, 0);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int e = 0; e < 4 * kSub; ++e) x[t][e] = s[t][e >> 2][0][e & 3] + s[t][e >> 2][1][e & 3];
    }
    __device__ __forceinline__ void rescale(int t, float by)
    {
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[t][j] *= by;
        l[t] *= by;
    }
    __device__ __forceinline__ void accumulate(const float (&p)[QT][4 * kSub])
    {
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int i = 0; i < 4 * kSub; i += 4) l[t] += (p[t][i] + p[t][i + 1]) + (p[t][i + 2] + p[t][i + 3]);
#pragma unroll
        for (int i = 0; i < 4 * kSub; ++i)
#pragma unroll
            for (int j = 0; j < kAcc; ++j)
#pragma unroll
                for (int t = 0; t < QT; ++t)
                    acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i][j >> 2][j & 3], p[t][i], acc[t][j], 0, 0, 0);
    }
    __device__ __forceinline__ int col() const { return c; }
    __device__ __forceinline__ int row() const { return g * 4; }
    __device__ __forceinline__ bool stores() const { return true; }
    __device__ __forceinline__ float top(float v) const { return xor_max16_32(v); }
    __device__ __forceinline__ void finish(float (&out)[QT])
    {
#pragma unroll
        for (int t = 0; t < QT; ++t) out[t] = xor_add<16>(xor_add<32>(l[t]));
    }
};

template <int DP, bool EXACT, int HINT> using CoreF32One = CoreF32<DP, EXACT, HINT, 1>;
template <int DP, bool EXACT, int HINT> using CoreF32Two = CoreF32<DP, EXACT, HINT, 2>;

// Up to four queries over float rows.  The float matrix instruction is slow enough to bound short caches (a step of 32 tokens, heads of 64: 0.85 us of
// a SIMD), and with few queries most of its 16 columns are empty.  The one of 16 blocks of four rows and four columns does a quarter of the work
// (5 sequences of up to 777, 4 cache heads of 64, three queries each: 12.1 -> 9.2 us; one of 1024, 8 heads 13.8 -> 10.5; 64 of 1024 36.6 -> 34.2):
//   S^T  block (g, m) = rows 4m .. 4m+3 of the 16 tokens, this lane group's pieces of the row; the sum over g is an exchange
//   O^T  block (g, m) = tokens 4m .. 4m+3, dimensions of the pieces 4g .. 4g+3; the sum over m waits until the end
// where lane l = (g, m, j) = (l >> 4, l >> 2 & 3, l & 3), j its row of an operand and its column, a query, of the other and of the results.
template <int DP, bool EXACT, int HINT>
struct CoreF32Few {
    typedef float Elem;
    static constexpr int QT = 1;
    static constexpr int kSub = DP > 64 ? 1 : 2, kTile = kSub * 16;
    static constexpr int kSteps = DP > 128 ? 8 : 6, kLeast = DP > 128 ? 4 : 2;
    static constexpr int kItemWaves = DP > 128 ? 4 : 8, kWaves = DP > 128 ? 1 : 2, kStage = kTile * DP * 4, kMostRows = kCols * DP * 4;
    static constexpr int KS = DP / 16, VEC = 4, VH = DP / 64, kAcc = VEC * VH;

    f32x4 qf[KS], kf[kSub][KS], vf[4 * kSub][VH], acc[1][kAcc];
    float m[1], l;
    KeyPlace<float, DP> keys;
    char *lds;
    uint32_t voff[VH];
    int D, g, quad, j;

    __device__ __forceinline__ void place(int d, int lane, char *own)
    {
        D = EXACT ? DP : d;
        g = lane >> 4;
        quad = lane >> 2 & 3;
        j = lane & 3;
        lds = own;
        keys.place(D, lane);
#pragma unroll
        for (int h = 0; h < VH; ++h) {
            const int dim = h * 64 + (g * 4 + j) * 4;
            voff[h] = EXACT || dim < D ? (uint32_t)(quad * 4 * D + dim) * 4 : kOutOfRange;
        }
    }
    __device__ __forceinline__ void begin(const float *q, int nq)
    {
#pragma unroll
        for (int s = 0; s < KS; ++s)
            qf[s] = EXACT || s * 16 < D ? *reinterpret_cast<const f32x4 *>(q + min(j, nq - 1) * D + s * 16 + g * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kAcc; ++i) acc[0][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        l = 0.0f;
        m[0] = -INFINITY;
    }
    __device__ __forceinline__ void load_k(const __amdgpu_buffer_rsrc_t (&rows)[kSub])
    {
#pragma unroll
        for (int i = 0; i < kSub; ++i)
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[i][s] = row_load<f32x4, HINT == kPassBoth ? kNt : 0>(rows[i], keys.from + s * keys.kRows * D * 4);
    }
    __device__ __forceinline__ void load_v(const __amdgpu_buffer_rsrc_t (&rows)[kSub])
    {
#pragma unroll
        for (int i = 0; i < 4 * kSub; ++i)
#pragma unroll
            for (int h = 0; h < VH; ++h) vf[i][h] = row_load<f32x4, HINT != kKeepAll ? kNt : 0>(rows[i >> 2], voff[h] + (i & 3) * D * 4);
    }
    __device__ __forceinline__ void scores(float (&x)[1][4 * kSub])
    {
        turn_keys(*this);
        f32x4 s[kSub][2];
#pragma unroll
        for (int i = 0; i < kSub; ++i) s[i][0] = s[i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < kSub; ++i)
                    s[i][e & 1] = __builtin_amdgcn_mfma_f32_4x4x1f32(kf[i][k][e], qf[k][e], s[i][e & 1], 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4 * kSub; ++e) x[0][e] = xor_add<16>(xor_add<32>(s[e >> 2][0][e & 3] + s[e >> 2][1][e & 3]));
    }
    __device__ __forceinline__ void rescale(int, float by)
    {
#pragma unroll
        for (int i = 0; i < kAcc; ++i) acc[0][i] *= by;
        l *= by;
    }
    __device__ __forceinline__ void accumulate(const float (&p)[1][4 * kSub])
    {
#pragma unroll
        for (int i = 0; i < 4 * kSub; i += 4) l += (p[0][i] + p[0][i + 1]) + (p[0][i + 2] + p[0][i + 3]);
#pragma unroll
        for (int i = 0; i < 4 * kSub; ++i)
#pragma unroll
            for (int k = 0; k < kAcc; ++k)
                acc[0][k] = __builtin_amdgcn_mfma_f32_4x4x1f32(vf[i][k >> 2][k & 3], p[0][i], acc[0][k], 0, 0, 0);
    }
    __device__ __forceinline__ int col() const { return j; }
    __device__ __forceinline__ int row() const { return quad * 4; }
    __device__ __forceinline__ bool stores() const { return quad == 0; }
    __device__ __forceinline__ float top(float v) const
    {
        auto as_f = [](int i) { return __builtin_bit_cast(float, i); };
        auto other = [&](float f, auto ctrl) { return __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, f), decltype(ctrl)::value, 0xf, 0xf, true); };
        v = fmaxf(v, as_f(other(v, std::integral_constant<int, 0x128>{})));          // row_ror:8: lane ^ 8
        // row_half_mirror and a reversed quad: lane ^ 4
        return fmaxf(v, as_f(other(as_f(other(v, std::integral_constant<int, 0x141>{})), std::integral_constant<int, 0x1B>{})));
    }
    __device__ __forceinline__ void finish(float (&out)[1])
    {
#pragma unroll
        for (int k = 0; k < kAcc; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[0][k][r] = xor_add<8>(xor_add<4>(acc[0][k][r]));
        out[0] = xor_add<8>(xor_add<4>(l));
    }
};

// The tiles first, first + stride, .. (count of them) of one sequence that a wave takes, and the pages of their 16-token parts: 64 parts at a time, one
// a lane.  All calls are wave-uniform.
template <typename Core>
struct Tiles {
    static constexpr int kHeld = kWave / Core::kSub;
    const int32_t *row;
    int max_pages, shift, first, stride, from, id, lane;

    __device__ __forceinline__ Tiles(const AttendArgs &a, int t, int first, int stride, int lane)
        : row(a.table + (int64_t)t * a.max_pages), max_pages(a.max_pages), shift(a.pool.page_shift), first(first), stride(stride), lane(lane)
    {
        fetch(0);
    }
    __device__ __forceinline__ int position(int i) const { return (first + i * stride) * Core::kTile; }
    __device__ __forceinline__ void fetch(int i)
    {
        from = i;
        const int page = (position(i + lane / Core::kSub) + lane % Core::kSub * 16) >> shift;
        id = page < max_pages ? row[page] : -1;
        asm volatile("" : "+v"(id));                 // waited for here, and not at every use of a step that fetched nothing
    }
    __device__ __forceinline__ int page(int i, int part) const { return __builtin_amdgcn_readlane(id, (i - from) * Core::kSub + part); }
};

template <typename Core>
struct Step {
    __amdgpu_buffer_rsrc_t k[Core::kSub], v[Core::kSub];
    int live[Core::kSub];                            // tokens of the 16 that count
    bool whole, any;

    __device__ __forceinline__ Step(const AttendArgs &a, Tiles<Core> &tiles, int kv, int len, int i)
    {
        constexpr int kBytes = sizeof(typename Core::Elem);
        if (i - tiles.from >= Tiles<Core>::kHeld) tiles.fetch(i);
        whole = true;
        any = false;
#pragma unroll
        for (int p = 0; p < Core::kSub; ++p) {
            const int pos = tiles.position(i) + p * 16;
            const int64_t row = paged_row(a.pool, tiles.page(i, p), kv, pos);
            live[p] = same(row < 0 ? 0 : max(0, min(len - pos, 16)));
            whole = whole && live[p] == 16;
            any = any || live[p] > 0;
            const uint64_t bytes = (uint64_t)(row < 0 ? 0 : row) * (a.D * kBytes);
            const uint64_t at = (uint64_t)(uint32_t)same((int)(bytes >> 32)) << 32 | (uint32_t)same((int)bytes);
            k[p] = buffer_of(static_cast<const char *>(a.k) + at, live[p] * a.D * kBytes);
            v[p] = buffer_of(static_cast<const char *>(a.v) + at, live[p] * a.D * kBytes);
        }
    }
};

// The part of a step between its products: scores -> probabilities, with the running maximum.  The maximum only moves when a score passes it by 8
// (a factor of 256, which float sums take with ease), so that most steps rescale nothing.  A step with tokens that count lifts it to the lowest float at least,
// so that one of -infinity says "no positions": a row of scores that are all -infinity has a sum of 0 and gives 0 / 0.
template <typename Core>
__device__ __forceinline__ void softmax_step(Core &core, const Step<Core> &st, float scale2, float (&x)[Core::QT][4 * Core::kSub])
{
    constexpr int N = 4 * Core::kSub;
#pragma unroll
    for (int t = 0; t < Core::QT; ++t) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[t][e] *= scale2;
        if (!st.whole) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[t][e] = core.row() + (e & 3) < st.live[e >> 2] ? x[t][e] : -INFINITY;
        }
        float top = x[t][0];
#pragma unroll
        for (int e = 1; e < N; ++e) top = fmaxf(top, x[t][e]);
        top = fmaxf(core.top(top), st.any ? -__FLT_MAX__ : -INFINITY);
        const bool passed = top > core.m[t] + 8.0f;
        if (__ballot(passed)) {
            const float to = passed ? top : core.m[t];   // a query's own scores decide: its result does not depend on its neighbours
            core.rescale(t, to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(core.m[t] - to));
            core.m[t] = to;
        }
        const float m = core.m[t] == -INFINITY ? 0.0f : core.m[t];
#pragma unroll
        for (int e = 0; e < N; ++e) x[t][e] = __builtin_amdgcn_exp2f(x[t][e] - m);
    }
}

// `count` tiles of a sequence against the queries in `core`: the next step's keys are asked for as soon as this one's are used up, and its
// values after this one's.
template <typename Core>
__device__ __forceinline__ void attend_tiles(const AttendArgs &a, Core &core, Tiles<Core> &tiles, int kv, int len, int count)
{
    float x[Core::QT][4 * Core::kSub];
    Step<Core> now(a, tiles, kv, len, 0);
    core.load_k(now.k);
    core.load_v(now.v);
    for (int i = 1; i < count; ++i) {
        const Step<Core> next(a, tiles, kv, len, i);
        core.scores(x);
        core.load_k(next.k);
        softmax_step(core, now, a.scale2, x);
        core.accumulate(x);
        core.load_v(next.v);
        now = next;
    }
    core.scores(x);
    softmax_step(core, now, a.scale2, x);
    core.accumulate(x);
}

struct Unit {
    int kv, head, nq;                                // cache head, first query head, queries
    __device__ __forceinline__ Unit(const AttendArgs &a, int kv, int part) : kv(kv)
    {
        const int from = part * a.rows;
        head = kv * a.group + from;
        nq = min(a.group - from, a.rows);
    }
    __device__ __forceinline__ Unit(const AttendArgs &a, int u)      // u may differ from lane to lane
        : Unit(a, a.n_qt == 1 ? u : u / a.n_qt, a.n_qt == 1 ? 0 : u % a.n_qt) {}
    static __device__ __forceinline__ Unit of_wave(const AttendArgs &a, int u) { return Unit(a, same(u)).scalars(); }
    __device__ __forceinline__ Unit scalars() const
    {
        Unit r = *this;
        r.kv = same(kv);
        r.head = same(head);
        r.nq = same(nq);
        return r;
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

// A lane's results are runs of VEC dimensions of a query: row 4g + r of instruction (h, j) is dimension h * 16 VEC + (4g + r) * VEC + j.
template <typename Core, typename OT>
__device__ __forceinline__ void store_rows(const Core &core, OT *rows, int nq, const float (&by)[Core::QT])
{
#pragma unroll
    for (int t = 0; t < Core::QT; ++t) {
        const int n = t * kCols + core.col();
        if (n >= nq || !core.stores()) continue;
#pragma unroll
        for (int h = 0; h < Core::VH; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int dim = h * 16 * Core::VEC + (core.g * 4 + r) * Core::VEC;
                float v[Core::VEC];
#pragma unroll
                for (int j = 0; j < Core::VEC; ++j) v[j] = by[t] == 0.0f ? 0.0f : core.acc[t][h * Core::VEC + j][r] * by[t];
                if (dim < core.D) store_piece(rows + (int64_t)n * core.D + dim, v);
            }
    }
}

// The same as partial results, with each query's maximum and sum (l).
template <typename Core>
__device__ __forceinline__ void store_part(const Core &core, float *rows, float2 *stats, int nq, const float (&l)[Core::QT])
{
    float one[Core::QT];
#pragma unroll
    for (int t = 0; t < Core::QT; ++t) {
        const int n = t * kCols + core.col();
        one[t] = 1.0f;
        if (core.g == 0 && core.stores() && n < nq) stats[n] = make_float2(core.m[t], l[t]);
    }
    store_rows(core, rows, nq, one);
}

// ---------------------------------------------------------------------------
// one workgroup a pair
// ---------------------------------------------------------------------------
// What the waves of a workgroup have of one pair, joined from LDS: four dimensions of the pair's rows, the i-th four, of query n.
struct Joined {
    float m, l;
    float4 o;
    __device__ __forceinline__ Joined(const float *part, int part_stride, const float2 *stats, int stats_stride, int waves, int n, int i)
        : m(-INFINITY), l(0.0f), o(make_float4(0.f, 0.f, 0.f, 0.f))
    {
        for (int w = 0; w < waves; ++w) m = fmaxf(m, stats[w * stats_stride + n].x);
        for (int w = 0; w < waves; ++w) {
            const float2 ml = stats[w * stats_stride + n];
            const bool none = ml.x == -INFINITY;     // no positions: nothing was stored
            const float by = none ? 0.0f : __builtin_amdgcn_exp2f(ml.x - m);
            const float4 v = *reinterpret_cast<const float4 *>(part + w * part_stride + i * 4);
            l += ml.y * by;
            o.x += (none ? 0.0f : v.x) * by;
            o.y += (none ? 0.0f : v.y) * by;
            o.z += (none ? 0.0f : v.z) * by;
            o.w += (none ? 0.0f : v.w) * by;
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T *to, bool kept) const
    {
        const bool none = m == -INFINITY || !kept;
        const float by = 1.0f / l;
        const float v[4] = {none ? 0.0f : o.x * by, none ? 0.0f : o.y * by, none ? 0.0f : o.z * by, none ? 0.0f : o.w * by};
        store_piece(to, v);
    }
};

// The waves take every kWaves-th tile, so that where a wave begins, and with it the pages it asks for first, does not wait for the length.
template <typename Core, int kWaves>
__global__ __launch_bounds__(kWaves * 64) void attend_item(AttendArgs a)
{
    __shared__ __align__(16) char s_own[kWaves * Core::kStage];
    constexpr int kMost = Core::QT * kCols;
    __shared__ float2 s_stats[kWaves * kMost];       // maximum and sum
    __shared__ int s_kept[kMost];
    static_assert(Core::kStage >= Core::kMostRows, "a wave's results fit its part");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = blockIdx.z;
    const Unit unit(a, blockIdx.x, blockIdx.y);
    Core core;
    core.place(a.D, lane, s_own + wave * Core::kStage);
    float *const s_part = reinterpret_cast<float *>(s_own);
    constexpr int kPart = Core::kStage / 4;
    // everything that tells where the rows are is asked for at once, none of it behind a condition (without a mask, any byte)
    const uint8_t *marks = a.mask ? a.mask + (int64_t)t * a.n_heads + unit.head : reinterpret_cast<const uint8_t *>(a.lens);
    const int mark = marks[a.mask ? min(lane, unit.nq - 1) : 0];
    const int raw_len = a.lens[t];
    core.begin(static_cast<const typename Core::Elem *>(a.q) + t * a.q_stride + unit.head * core.D, unit.nq);
    Tiles<Core> tiles(a, t, wave, kWaves, lane);
    const bool kept = !a.mask || mark != 0;
    const int len = paged_length(same(raw_len), a.max_len);
    const int all = __ballot(kept) ? (len + Core::kTile - 1) / Core::kTile : 0;
    if (wave == 0 && lane < kMost) s_kept[lane] = kept;
    const int count = (all - wave + kWaves - 1) / kWaves;        // all < wave: none
    if (count > 0) attend_tiles(a, core, tiles, unit.kv, len, count);
    float l[Core::QT];
    core.finish(l);
    if (count > 0) store_part(core, s_part + wave * kPart, s_stats + wave * kMost, unit.nq, l);
    else if (lane < unit.nq) s_stats[wave * kMost + lane] = make_float2(-INFINITY, 0.0f);
    __syncthreads();
    typename Core::Elem *out = static_cast<typename Core::Elem *>(a.out) + ((int64_t)t * a.n_heads + unit.head) * core.D;
    for (int i = threadIdx.x; i < unit.nq * (core.D / 4); i += kWaves * 64) {
        const int n = i / (core.D / 4);
        Joined(s_part, kPart, s_stats, kMost, kWaves, n, i).store(out + i * 4, s_kept[n]);
    }
}

// ---------------------------------------------------------------------------
// even shares of all tiles
// ---------------------------------------------------------------------------
// The line of all tiles: tiles before each sequence and its length.  Up to 64 sequences every wave has it in registers, a sequence a lane, without a mask
// without a barrier; of more it is in LDS.  Made by the whole workgroup.
template <int kTile>
struct Line {
    int *s_base, *s_len;                             // [T + 1], [T]
    int before, len, T;                              // up to 64 sequences: of the lane's
    int total;                                       // all tiles
    bool small;

    __device__ __forceinline__ int tiles(int n) const { return (n + kTile - 1) / kTile; }
    static __device__ __forceinline__ int upto(int v, int lane)
    {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(v, d);
            if (lane >= d) v += o;
        }
        return v;
    }
    __device__ __forceinline__ Line(const AttendArgs &a, int *s_line, int *s_wave) : s_base(s_line), s_len(s_line + a.T + 1), T(a.T), small(a.T <= 64)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, threads = kTeam * 64;
        if (a.mask) {
            // the first look at the mask and the lengths are asked for together
            const int pairs = T * a.n_units;
            auto alive = [&](int i) {
                const int t = i / a.n_units;
                return unit_alive(a, t, i - t * a.n_units) ? t : -1;
            };
            int hit = tid < pairs ? alive(tid) : -1;
            for (int t = tid; t < T; t += threads) {
                s_base[t] = 0;
                s_len[t] = paged_length(a.lens[t], a.max_len);
            }
            __syncthreads();
            for (int i = tid;;) {
                if (hit >= 0) atomicAdd(&s_base[hit], 1);        // integers: any order gives the same count
                if ((i += threads) >= pairs) break;
                hit = alive(i);
            }
            __syncthreads();
        } else if (!small) {
            for (int t = tid; t < T; t += threads) {
                s_base[t] = a.n_units;
                s_len[t] = paged_length(a.lens[t], a.max_len);
            }
            __syncthreads();
        }
        if (small) {
            const int t = min(lane, T - 1);
            len = a.mask ? s_len[t] : paged_length(a.lens[t], a.max_len);
            const int mine = lane < T ? (a.mask ? s_base[t] : a.n_units) * tiles(len) : 0;
            const int all = upto(mine, lane);
            before = all - mine;
            total = __builtin_amdgcn_readlane(all, 63);
            return;
        }
        const int each = (T + threads - 1) / threads, from = min(tid * each, T), to = min(from + each, T);
        int mine = 0;
        for (int t = from; t < to; ++t) {
            const int n = s_base[t] * tiles(s_len[t]);
            s_base[t] = mine;
            mine += n;
        }
        const int all = upto(mine, lane);
        if (lane == 63) s_wave[wave] = all;
        __syncthreads();
        int others = all - mine;
        for (int w = 0; w < wave; ++w) others += s_wave[w];
        for (int t = from; t < to; ++t) s_base[t] += others;
        if (tid == threads - 1) s_base[T] = others + mine;
        __syncthreads();
        total = same(s_base[T]);
    }
    // all wave-uniform
    __device__ __forceinline__ int base(int t) const
    {
        return !small ? same(s_base[t]) : t < T ? __builtin_amdgcn_readlane(before, t) : total;
    }
    __device__ __forceinline__ int length(int t) const { return small ? __builtin_amdgcn_readlane(len, t) : same(s_len[t]); }
    // the sequence whose tiles hold `at`: base(t) <= at < base(t + 1)
    __device__ __forceinline__ int holds(int at, int lane) const
    {
        if (small) return __popcll(__ballot(lane < T && before <= at)) - 1;
        int lo = 0, hi = T;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (base(mid) <= at) lo = mid; else hi = mid;
        }
        return lo;
    }
};

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
__global__ __launch_bounds__(kTeam * 64, Core::kWaves) void attend_stream(AttendArgs a)
{
    __shared__ __align__(16) char s_own[kTeam * Core::kStage];
    extern __shared__ int s_line[];                  // bases [T + 1], lengths [T]
    constexpr int kMost = Core::QT * kCols;
    __shared__ float2 s_stats[kTeam * kMost];
    __shared__ int s_wave[kTeam];
    __shared__ int4 s_last[kTeam];                   // the pair that a wave's share ends in: first tile (-1: none), tiles, sequence, unit
    float *const s_part = reinterpret_cast<float *>(s_own);
    constexpr int kPart = Core::kStage / 4;
    const Line<Core::kTile> line(a, s_line, s_wave);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int total = line.total, per = tiles_per_worker(total, gridDim.x * kTeam, Core::kLeast);
    if (blockIdx.x == 0) {                           // for the second launch
        for (int t = threadIdx.x; t < a.T; t += kTeam * 64) a.plan[2 + t] = line.small ? line.before : line.s_base[t];
        if (threadIdx.x == 0) a.plan[0] = per, a.plan[1] = total;
    }
    const int worker = blockIdx.x * kTeam + wave;
    int at = (int)min((int64_t)worker * per, (int64_t)total);
    const int end = (int)min((int64_t)at + per, (int64_t)total);
    Core core;
    core.place(a.D, lane, s_own + wave * Core::kStage);
    AliveUnits units;
    int4 last = make_int4(-1, 0, 0, 0);
    for (int t = line.holds(at, lane); at < end; ++t) {
        const int from = line.base(t), size = line.base(t + 1) - from;
        if (size == 0) continue;
        const int len = line.length(t);
        const int tiles = (len + Core::kTile - 1) / Core::kTile;
        int n = (at - from) / tiles;
        units.find(a, t, n, lane);
        for (; at < end && at < from + size; ++n, units.next(a, t, lane)) {
            const Unit unit = Unit::of_wave(a, units.unit());
            const int offset = from + n * tiles, b = at - offset, e = min(tiles, end - offset);
            core.begin(static_cast<const typename Core::Elem *>(a.q) + t * a.q_stride + unit.head * core.D, unit.nq);
            Tiles<Core> mine(a, t, b, 1, lane);
            attend_tiles(a, core, mine, unit.kv, len, e - b);
            at = offset + e;
            float l[Core::QT];
            core.finish(l);
            if (b == 0 && e == tiles) {
                float by[Core::QT];
#pragma unroll
                for (int q = 0; q < Core::QT; ++q) {
                    const int i = q * kCols + core.col();
                    by[q] = i >= unit.nq || !head_alive(a, t, unit.head + i) || core.m[q] == -INFINITY ? 0.0f : 1.0f / l[q];
                }
                store_rows(core, static_cast<typename Core::Elem *>(a.out) + ((int64_t)t * a.n_heads + unit.head) * core.D, unit.nq, by);
            } else if (at < end) {                   // the share goes on: a partial result of its own
                const int64_t slot = 2 * (int64_t)worker;
                store_part(core, a.part + slot * a.rows * core.D, reinterpret_cast<float2 *>(a.stats) + slot * a.rows, unit.nq, l);
            } else {
                last = make_int4(offset, tiles, t, units.unit());
                store_part(core, s_part + wave * kPart, s_stats + wave * kMost, unit.nq, l);
            }
        }
    }
    if (lane == 0) s_last[wave] = last;
    __syncthreads();
    for (int w = 0, waves; w < kTeam; w += waves) {  // the same for every thread
        const int4 pair = s_last[w];
        for (waves = 1; w + waves < kTeam && s_last[w + waves].x == pair.x; ++waves) {}
        if (pair.x < 0) continue;
        const Cut cut(pair.x, pair.y, per, total);
        const Unit unit(a, pair.w);
        const int64_t slot = 2 * (int64_t)(blockIdx.x * kTeam + w) + 1;
        typename Core::Elem *out = static_cast<typename Core::Elem *>(a.out) + ((int64_t)pair.z * a.n_heads + unit.head) * core.D;
        for (int i = threadIdx.x; i < unit.nq * (core.D / 4); i += kTeam * 64) {
            const int n = i / (core.D / 4);
            const Joined j(s_part + w * kPart, kPart, s_stats + w * kMost, kMost, waves, n, i);
            if (cut.in_team) {
                j.store(out + i * 4, head_alive(a, pair.z, unit.head + n));
            } else {
                *reinterpret_cast<float4 *>(a.part + slot * a.rows * core.D + i * 4) = j.o;
                if (i == n * (core.D / 4)) *reinterpret_cast<float2 *>(a.stats + (slot * a.rows + n) * 2) = make_float2(j.m, j.l);
            }
        }
    }
}

// A partial result taken into the running ones (m, l, o).
__device__ __forceinline__ void take_in(float &m, float &l, float4 &o, const float2 &ml, const float4 &p)
{
    const float to = fmaxf(m, ml.x), use = to == -INFINITY ? 0.0f : to;
    const float keep = __builtin_amdgcn_exp2f(m - use), by = __builtin_amdgcn_exp2f(ml.x - use);
    l = l * keep + ml.y * by;
    o.x = o.x * keep + p.x * by;
    o.y = o.y * keep + p.y * by;
    o.z = o.z * keep + p.z * by;
    o.w = o.w * keep + p.w * by;
    m = to;
}

// Joins the pairs that the first launch left in parts, and gives 0 to those that nobody had.  Workgroups stand for pairs (x, z), cut by y; a thread stands
// for four dimensions of one query, kShares threads of a workgroup for the same, each with its share of the parts.
template <typename Elem, int kTile, int kShares>
__global__ __launch_bounds__(256) void attend_join(AttendArgs a)
{
    constexpr int kQuads = 256 / kShares;
    __shared__ float4 s_o[256];
    __shared__ float2 s_ml[256];
    const int lane = threadIdx.x & 63, tid = threadIdx.x, share = tid / kQuads;
    const int t = blockIdx.z, u = blockIdx.x;
    const Unit unit(a, u);
    const int per = a.plan[0], total = a.plan[1], from = a.plan[2 + t];
    const int tiles = (paged_length(a.lens[t], a.max_len) + kTile - 1) / kTile;
    int rank = u;
    bool any = tiles > 0;
    if (a.mask) {
        rank = 0;
        for (int block = 0; block <= u; block += 64) {
            const uint64_t bits = __ballot(block + lane < a.n_units && unit_alive(a, t, block + lane));
            rank += __popcll(u - block < 64 ? bits & ((1ull << (u - block)) - 1) : bits);
            if (u - block < 64) any = any && ((bits >> (u - block)) & 1);
        }
    }
    const Cut cut(any ? from + rank * tiles : 0, any ? tiles : 1, per, total);
    if (any && (cut.whole || cut.in_team)) return;   // written out by the first launch
    const int parts = any ? cut.parts() : 0, quads = unit.nq * (a.D / 4);
    Elem *out = static_cast<Elem *>(a.out) + ((int64_t)t * a.n_heads + unit.head) * a.D;
    for (int block = blockIdx.y * kQuads; block < quads; block += gridDim.y * kQuads) {
        const int i = block + tid % kQuads, n = min(i, quads - 1) / (a.D / 4);
        const bool kept = head_alive(a, t, unit.head + n);
        float m = -INFINITY, l = 0.0f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < quads)
#pragma unroll 4
            for (int k = share; k < parts; k += kShares) {
                const int64_t slot = cut.slot(k);
                take_in(m, l, o, *reinterpret_cast<const float2 *>(a.stats + (slot * a.rows + n) * 2),
                        *reinterpret_cast<const float4 *>(a.part + slot * a.rows * a.D + i * 4));
            }
        if constexpr (kShares > 1) {
            __syncthreads();
            s_o[tid] = o;
            s_ml[tid] = make_float2(m, l);
            __syncthreads();
            if (share == 0)
#pragma unroll
                for (int k = 1; k < kShares; ++k) take_in(m, l, o, s_ml[k * kQuads + tid], s_o[k * kQuads + tid]);
        }
        if (share == 0 && i < quads) {
            const bool none = m == -INFINITY || !kept;
            const float by = 1.0f / l;
            const float v[4] = {none ? 0.0f : o.x * by, none ? 0.0f : o.y * by, none ? 0.0f : o.z * by, none ? 0.0f : o.w * by};
            store_piece(out + i * 4, v);
        }
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
template <typename Core, int kWaves>
int launch_item(const AttendArgs &a, hipStream_t s)
{
    attend_item<Core, kWaves><<<dim3(a.pool.n_kv, a.n_qt, a.T), dim3(kWaves * 64), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}

template <typename Core>
int launch_stream(const AttendArgs &a, hipStream_t s)
{
    typedef typename Core::Elem Elem;
    const int pairs = a.T * a.n_units, tiles = (a.max_len + Core::kTile - 1) / Core::kTile;
    const size_t lds = (2 * (size_t)a.T + 1) * sizeof(int);          // at most 32 KiB and 4 bytes, beside up to 66 KiB that the kernel has of its own (of 160)
    constexpr int grid = kUnits * Core::kWaves;                      // what is resident at once: with rows of 256 half as much
    const int64_t wanted = ((int64_t)pairs * tiles + kTeam * Core::kLeast - 1) / (kTeam * Core::kLeast);
    attend_stream<Core><<<dim3(wanted < grid ? (int)wanted : grid), dim3(kTeam * 64), lds, s>>>(a);
    if (hipGetLastError() != hipSuccess) return HALO_ERR_HIP;
    // few pairs are cut into many parts each, shared by eight threads (one sequence of 32771, 8 cache heads: 37 us by one, 5); many pairs have few
    // parts, and then the shares cost (96 sequences, 8 cache heads: 5 us of the pass, 290 for 285 with eight)
    if (pairs < 256)
        attend_join<Elem, Core::kTile, 8><<<dim3(a.n_units, (a.rows * (a.D / 4) + 31) / 32, a.T), dim3(256), 0, s>>>(a);
    else
        attend_join<Elem, Core::kTile, 1><<<dim3(a.n_units, 1, a.T), dim3(256), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}

// A workgroup a pair, of kWaves waves.
template <template <int, bool, int> class Core, int DP, bool EXACT, int kWaves>
int launch_pairs(const AttendArgs &a, hipStream_t s)
{
    if (a.bytes > (256 << 20)) return launch_item<Core<DP, EXACT, kPassBoth>, kWaves>(a, s);
    if constexpr (Core<DP, EXACT, kKeepAll>::QT == 1) {          // more queries: large caches only
        if (a.bytes <= (64 << 20)) return launch_item<Core<DP, EXACT, kKeepAll>, kWaves>(a, s);
    }
    return launch_item<Core<DP, EXACT, kPassValues>, kWaves>(a, s);
}

// One launch, a workgroup a pair, or even shares and a second launch: the latter costs some 5 us more, the former is as slow as its longest pair on one compute unit.
// One launch up to kSteps steps of a wave (8; 4 and 6 where a step computes longer) at the longest length; from 512 pairs on, two for every unit, up to 8, or 16
// with rows of 256, of which a unit has half as many waves.  us, one launch / two (lengths from half of the longest to the longest):
// bf16 heads of 128, 8 cache heads, 1 sequence of 1024 8.7 / 10.6, 2048 (8 steps) 13.5 / 11.1, 4096 23.4 / 11.7; 16 sequences 2048 21.4 / 25.1, 4096 44.1 / 41.3; 64
// sequences 2048 66.0 / 71.6, 4096 134 / 135, and with lengths from 0 on 102 / 94.  Heads of 64, 1 sequence of 2048 (4 steps) 10.9 / 11.4; 64 of 4000 (8) 69 / 71.
// Heads of 256, 8 sequences of 1024 (8 steps) 16.2 / 21.1, 64 of 2048 (16) 127 / 135.  Float heads of 64, four queries a cache head, 1 sequence of 1024
// 9.2 / 10.9, 2048 (8 steps) 14.7 / 11.2; 8 sequences 2048 15.2 / 17.8; 64 sequences 2048 66.7 / 70.1.
template <template <int, bool, int> class Core, int DP, bool EXACT>
int launch_cut(const AttendArgs &a, hipStream_t s)
{
    typedef Core<DP, EXACT, kKeepAll> C;
    const bool many = a.T * a.n_units >= 512;
    const int steps = !many ? C::kSteps : DP > 128 ? 16 : 8;
    const bool one_launch = a.max_len <= steps * C::kItemWaves * C::kTile;
    // Fewer waves a workgroup where more would have no tile, and where workgroups are many anyway: all of their waves wait for the slowest.
    // us, heads of 128, 8 cache heads, by waves 8 / 4 / 2: 1 sequence of up to 64 (2 tiles) 4.1 / 4.0 / 4.0, of 128 4.3 / 4.2 / 4.7; 128 sequences of 16 12.3 / 7.0 /
    // 4.6, of 256 (8 tiles) 24.2 / 18.5 / 18.2; 192 of 300 (10) 38.0 / 29.8 / 31.2, of 600 (19) 59.2 / 57.4 / 60.1; 32 of 128, 256 pairs, 5.2 / 5.2 / 5.3.  With 20
    // queries a cache head, 8 / 2: 200 sequences of up to 250 54.4 / 40.6, 500 of up to 60 in float 127 / 80; 100 of up to 500, 8 / 4, 38.8 / 39.5.
    const int tiles = (a.max_len + C::kTile - 1) / C::kTile;
    if (tiles <= 2 || (many && tiles <= 8)) return launch_pairs<Core, DP, EXACT, 2>(a, s);
    if constexpr (C::kItemWaves > 4) {
        if (many && tiles <= 16) return launch_pairs<Core, DP, EXACT, 4>(a, s);
    }
    if (one_launch) return launch_pairs<Core, DP, EXACT, C::kItemWaves>(a, s);
    return a.bytes > (256 << 20) ? launch_stream<Core<DP, EXACT, kPassBoth>>(a, s) : launch_stream<Core<DP, EXACT, kPassValues>>(a, s);
}

template <template <int, bool, int> class Core>
int launch_dim_128(const AttendArgs &a, hipStream_t s)
{
    if (a.D == 64) return launch_cut<Core, 64, true>(a, s);
    if (a.D == 128) return launch_cut<Core, 128, true>(a, s);
    if (a.D < 64) return launch_cut<Core, 64, false>(a, s);
    return launch_cut<Core, 128, false>(a, s);
}

template <template <int, bool, int> class Core>
int launch_dim(const AttendArgs &a, hipStream_t s)
{
    if (a.D <= 128) return launch_dim_128<Core>(a, s);
    if (a.D == 256) return launch_cut<Core, 256, true>(a, s);
    return launch_cut<Core, 256, false>(a, s);
}

}  // namespace

// One for each kind of rows and queries, each in a file of its own: bf16 with up to 16 queries a cache head at once and with up to 32 (heads of up to 128),
// float with up to 4, 16 and 32 (heads of up to 128).
int launch_attend_bf16(const AttendArgs &a, hipStream_t s);
int launch_attend_bf16_32(const AttendArgs &a, hipStream_t s);
int launch_attend_f32_4(const AttendArgs &a, hipStream_t s);
int launch_attend_f32(const AttendArgs &a, hipStream_t s);
int launch_attend_f32_32(const AttendArgs &a, hipStream_t s);

}  // namespace halo
