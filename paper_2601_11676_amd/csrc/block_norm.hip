// What stands between two blocks (halo_block_norm): the norm after a block with its gate, the scaled residual and the norm before the next,
//     u = n(y) w_post,  h' = s h + g u,  x = n(h') w_pre,   n(z) = z / sqrt(mean(z^2) + eps)
// in one pass: a row stays in registers between its two sums of squares, so that every element is read and written once.  Bytes bound many
// rows; one row is a launch, a round trip and two exchanges between its waves.
#include "../../include/halo.h"

#include <cmath>

#include "kernels.hpp"

namespace halo {
namespace {

struct NormArgs {
    const void *h, *y, *w_post, *gate, *w_pre;
    void *h_out, *x;
    int T, d, post, gate_per_token;
    float res_scale, eps;
};

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
    const int row = WAVE ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (WAVE && row >= a.T) return;
    const HT *h = static_cast<const HT *>(a.h) + (int64_t)row * a.d;
    const T *y = static_cast<const T *>(a.y) + (int64_t)row * a.d;
    const T *gate = static_cast<const T *>(a.gate) + (a.gate_per_token ? (int64_t)row * a.d : 0);
    const T *w_post = static_cast<const T *>(a.w_post), *w_pre = static_cast<const T *>(a.w_pre);

    Piece8<HT> hp[C];
    Piece8<T> yp[C], gp[C], op[C], ep[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = (c * threads + tid) * 8;
        hp[c].zero(); yp[c].zero(); gp[c].zero(); op[c].zero(); ep[c].zero();
        if (e < a.d) {
            yp[c].load(y + e);
            hp[c].load(h + e);
            if (a.gate) gp[c].load(gate + e);
            if (a.w_post) op[c].load(w_post + e);
            if (a.w_pre) ep[c].load(w_pre + e);
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
            op[c].get(g);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] *= a.w_post ? by * g[i] : by;
        }
        gp[c].get(g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            z[c][i] = a.res_scale * z[c][i] + (a.gate ? g[i] * u[i] : u[i]);
            sq = __builtin_fmaf(z[c][i], z[c][i], sq);
        }
        const int e = (c * threads + tid) * 8;
        if (e < a.d) store8(static_cast<HT *>(a.h_out) + (int64_t)row * a.d + e, z[c]);
    }
    by = 1.0f / sqrtf(row_sum<WAVE>(sq, s_sum[1]) / (float)a.d + a.eps);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float w[8];
        ep[c].get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[c][i] *= a.w_pre ? by * w[i] : by;
        const int e = (c * threads + tid) * 8;
        if (e < a.d) store8(static_cast<T *>(a.x) + (int64_t)row * a.d + e, z[c]);
    }
}

template <typename T, typename HT>
int launch_norm(const NormArgs &a, hipStream_t s)
{
    const int pieces = a.d / 8;
    auto rows_of_waves = [&](auto c) {
        block_norm_kernel<T, HT, decltype(c)::value, true><<<dim3((a.T + 3) / 4), dim3(256), 0, s>>>(a);
    };
    auto row_of_workgroup = [&](auto c) {
        constexpr int C = decltype(c)::value;
        const int threads = ((pieces + C - 1) / C + 63) / 64 * 64;
        block_norm_kernel<T, HT, C, false><<<dim3(a.T), dim3(threads), 0, s>>>(a);
    };
    if (pieces <= 64) rows_of_waves(std::integral_constant<int, 1>{});
    else if (pieces <= 1024) row_of_workgroup(std::integral_constant<int, 1>{});
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
    if (!h || !y || !h_out || !x) return HALO_ERR_NULL;
    if (dtype != HALO_F32 && dtype != HALO_BF16) return HALO_ERR_DTYPE;
    if (h_dtype != HALO_F32 && h_dtype != dtype) return HALO_ERR_DTYPE;
    if (T < 0 || d < 8 || d % 8 || d > 32768 || !(eps >= 0.0f) || !std::isfinite(res_scale)) return HALO_ERR_ARG;
    for (const void *p : {h, y, w_post, gate, w_pre, (const void *)h_out, (const void *)x})
        if (reinterpret_cast<uintptr_t>(p) & 15u) return HALO_ERR_ARG;
    if (T == 0) return HALO_OK;
    const NormArgs a{h, y, w_post, gate, w_pre, h_out, x, T, d, post_norm != 0, gate_per_token != 0, res_scale, eps};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == HALO_F32) return launch_norm<float, float>(a, s);
    return h_dtype == HALO_F32 ? launch_norm<bf16_t, float>(a, s) : launch_norm<bf16_t, bf16_t>(a, s);
}
