// What stands between two blocks (halo_block_norm): the norm after a block with its gate, the scaled residual and the norm before the next,
//     u = n(y) w_post,  h' = s h + g u,  x = n(h') w_pre,   n(z) = z / sqrt(mean(z^2) + eps)
// in one pass: a row stays in registers between its two sums of squares, so that every element is read and written once.  Bytes bound many
// rows (4099 rows of 5120, bf16: 210 MB in 41 us, 5.1 TB/s, where a copy of 8 GiB reaches 4.8); one row is a launch, a round trip and two exchanges
// between its waves (3 to 4 us).
#include "../../include/halo.h"

#include <algorithm>
#include <cmath>

#include "kernels.hpp"

namespace halo {
namespace {

struct NormArgs {
    const void *h, *y, *w_post, *gate, *w_pre;
    void *h_out, *x;
    int T, d, post, gate_per_token, first;           // first: row of the launch's first workgroup
    float res_scale, eps;
};

// The residual stream comes back only after the block, so that its stores carry the non-temporal hint (us without / with: 8192 rows of 512
// 10.2 / 9.5, 2000 of 2048 9.1 / 8.1, 4096 of 8192 75.7 / 74.7); x is read at once and does not.
__device__ __forceinline__ void store8_pass(float *p, const float (&v)[8])
{
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4 *>(p));
    __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4 *>(p + 4));
}
__device__ __forceinline__ void store8_pass(bf16_t *p, const float (&v)[8])
{
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (uint32_t)f32_to_bf16(v[2 * i]) | ((uint32_t)f32_to_bf16(v[2 * i + 1]) << 16);
    __builtin_nontemporal_store(o, reinterpret_cast<u32x4 *>(p));
}

// Sum over the threads of a row: one wave of several rows' workgroup (WAVE), or the whole workgroup.
template <bool WAVE>
__device__ __forceinline__ float row_sum(float v, float *s_sum)
{
    v = wave_sum(v);
    if constexpr (WAVE) return v;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if (lane == 0) s_sum[wave] = v;
    __syncthreads();
    float total = 0.0f;
    for (int w = 0; w < waves; ++w) total += s_sum[w];
    return total;
}

// C pieces of eight elements a thread: piece c of thread i is c * threads + i.  WAVE: a wave a row, four rows a workgroup.
template <typename T, typename HT, int C, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void block_norm_kernel(NormArgs a)
{
    __shared__ float s_sum[2][16];
    const int threads = WAVE ? 64 : blockDim.x, tid = WAVE ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = a.first + (WAVE ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : (int64_t)blockIdx.x);
    if (WAVE && row >= a.T) return;
    const HT *h = static_cast<const HT *>(a.h) + row * a.d;
    const T *y = static_cast<const T *>(a.y) + row * a.d;
    const T *gate = static_cast<const T *>(a.gate) + (a.gate_per_token ? row * a.d : 0);
    const T *w_post = static_cast<const T *>(a.w_post), *w_pre = static_cast<const T *>(a.w_pre);

    // rows of more than 16384 would need more registers than 1024 threads have: their weights are loaded where they are used
    constexpr bool kAhead = C < 4;
    Piece8<HT> hp[C];
    Piece8<T> yp[C], gp[C], op[C], ep[C];
    auto weights = [&](Piece8<T> &p, const T *w, int c) {
        const int e = (c * threads + tid) * 8;
        p.zero();
        if (w && e < a.d) p.load(w + e);
    };
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = (c * threads + tid) * 8;
        hp[c].zero();
        yp[c].zero();
        if (e < a.d) {
            yp[c].load(y + e);
            hp[c].load(h + e);
        }
        if (kAhead) {
            weights(gp[c], a.gate ? gate : nullptr, c);
            weights(op[c], w_post, c);
            weights(ep[c], w_pre, c);
        }
    }
    float by = 1.0f;
    if (a.post) {
        float sq = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float v[8];
            yp[c].get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sq = __builtin_fmaf(v[i], v[i], sq);
        }
        by = 1.0f / sqrtf(row_sum<WAVE>(sq, s_sum[0]) / (float)a.d + a.eps);
    }
    float z[C][8], sq = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float u[8], g[8];
        yp[c].get(u);
        hp[c].get(z[c]);
        if (a.post) {
            if (!kAhead) weights(op[c], w_post, c);
            op[c].get(g);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] *= a.w_post ? by * g[i] : by;
        }
        if (!kAhead) weights(gp[c], a.gate ? gate : nullptr, c);
        gp[c].get(g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            z[c][i] = a.res_scale * z[c][i] + (a.gate ? g[i] * u[i] : u[i]);
            sq = __builtin_fmaf(z[c][i], z[c][i], sq);
        }
        const int e = (c * threads + tid) * 8;
        if (e < a.d) store8_pass(static_cast<HT *>(a.h_out) + row * a.d + e, z[c]);
    }
    by = 1.0f / sqrtf(row_sum<WAVE>(sq, s_sum[1]) / (float)a.d + a.eps);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float w[8];
        if (!kAhead) weights(ep[c], w_pre, c);
        ep[c].get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[c][i] *= a.w_pre ? by * w[i] : by;
        const int e = (c * threads + tid) * 8;
        if (e < a.d) store8(static_cast<T *>(a.x) + row * a.d + e, z[c]);
    }
}

template <typename T, typename HT>
int launch_norm(const NormArgs &a, hipStream_t s)
{
    const int pieces = a.d / 8;
    // one launch, of rows whose workgroups number less than 2^32 threads; of more rows one after the other
    auto each_run = [&](int rows_a_group, int threads, auto launch) {
        const int64_t run = (int64_t)(0xffffffffu / threads) * rows_a_group;
        for (int64_t first = 0; first < a.T; first += run) {
            NormArgs part = a;
            part.first = (int)first;
            launch(dim3((unsigned)((std::min(run, a.T - first) + rows_a_group - 1) / rows_a_group)), part);
        }
    };
    auto rows_of_waves = [&](auto c) {
        each_run(4, 256, [&](dim3 grid, const NormArgs &p) { block_norm_kernel<T, HT, decltype(c)::value, true><<<grid, dim3(256), 0, s>>>(p); });
    };
    auto row_of_workgroup = [&](auto c) {
        constexpr int C = decltype(c)::value;
        const int threads = ((pieces + C - 1) / C + 63) / 64 * 64;
        each_run(1, threads, [&](dim3 grid, const NormArgs &p) { block_norm_kernel<T, HT, C, false><<<grid, dim3(threads), 0, s>>>(p); });
    };
    // two pieces a thread from 513 on: 4099 rows of 5120 44.3 us with one, 41.6 with two
    if (pieces <= 64) rows_of_waves(std::integral_constant<int, 1>{});
    else if (pieces <= 512) row_of_workgroup(std::integral_constant<int, 1>{});
    else if (pieces <= 2048) row_of_workgroup(std::integral_constant<int, 2>{});
    else row_of_workgroup(std::integral_constant<int, 4>{});
    return hipGetLastError() == hipSuccess ? HALO_OK : HALO_ERR_HIP;
}

}  // namespace
}  // namespace halo

extern "C" int halo_block_norm(const void *h, const void *y, const void *w_post, const void *gate, const void *w_pre, void *h_out,
                               void *x, int32_t T, int32_t d, int32_t dtype, int32_t h_dtype, int32_t post_norm,
                               int32_t gate_per_token, float res_scale, float eps, void *stream)
{
    using namespace halo;
    if (dtype != HALO_F32 && dtype != HALO_BF16) return HALO_ERR_DTYPE;
    if (h_dtype != HALO_F32 && h_dtype != dtype) return HALO_ERR_DTYPE;
    if (T < 0 || d < 8 || d % 8 || d > 32768 || !(eps >= 0.0f) || !std::isfinite(res_scale)) return HALO_ERR_ARG;
    if (T == 0) return HALO_OK;
    if (!h || !y || !h_out || !x) return HALO_ERR_NULL;
    for (const void *p : {h, y, w_post, gate, w_pre, (const void *)h_out, (const void *)x})
        if (reinterpret_cast<uintptr_t>(p) & 15u) return HALO_ERR_ARG;
    const NormArgs a{h, y, w_post, gate, w_pre, h_out, x, T, d, post_norm != 0, gate_per_token != 0, 0, res_scale, eps};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == HALO_F32) return launch_norm<float, float>(a, s);
    return h_dtype == HALO_F32 ? launch_norm<bf16_t, float>(a, s) : launch_norm<bf16_t, bf16_t>(a, s);
}
