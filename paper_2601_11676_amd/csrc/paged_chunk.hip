// Attention of chunks of new tokens over a paged cache (halo_paged_chunk_attention, halo_paged_chunk_attention_q8): token i of a sequence, at position p_i, has
//     o_h = sum_j p_j V_j,  p = softmax_j(scale q_h . K_j),  j <= p_i
// one pass over the rows with the running maximum and sum of the softmax.  Products bound it: a cached row meets all the rows of a block, 32, 128 or 256 queries (the heads of
// one cache head, token by token).  512 tokens after 16000, 64 heads over 8 cache heads of 128, bf16: 279 us with the join, 978 TFLOP/s, where a library product of 8192^3 reaches 1230;
// over codes 8192 tokens after as many 2.72 ms, 859 TFLOP/s (medians; from card to card 270 to 291 us, 2.64 to 2.77 ms).  In the attending kernel the matrix cores are busy 51 % of the time and the VALU issues 47 %: two waves of a SIMD,
// each multiplying (1024 cycles a tile of 64 tokens) and taking exponentials (about as long) in turn.
//
// S^T = K Q^T      rows = tokens, columns = queries (matrix instruction of 32 x 32, 16 deep): a lane's results are scores of one query, so that maximum and sum
//                  of a softmax need one exchange between the halves of a wave.
// O^T += V^T P^T   the sum over tokens may take them in any order, so the operand P^T is what the lane already holds; V^T comes from LDS by the loads that
//                  turn 4 x 16 elements on their way, four tokens of a dimension at a time (128 bytes a cycle and unit; 16 bytes a lane of K 210).
//
// How the work is cut: workgroups take blocks of rows; where those are too few for the card, also parts of their tiles, of one size whatever the sequences' lengths, and a second
// launch joins the parts.  Each workgroup finds its own in the lengths: no launch before it, but for a mask with many scores.
//
// What a float is to the matrix cores: three bf16 values, all 24 bits of it, and six products of them (406 TFLOP/s at most where the float instruction has 154; 4 sequences of 4000
// tokens in all, 32 heads of 128, 356 us, 102 TFLOP/s of the formula's).  A bf16 row's probabilities are rounded once, by at most 2^-8 of each, and it is what is
// multiplied that is summed; a second part would leave 2^-16: us, one part / two, 279 / 368 (512 after 16000), 2670 / 3410 (over codes), 80 / 89 (7 sequences of 4099 in all), 23 / 24 (40 drafted
// tokens).  It is the values' own precision: results are off by 0.0022 of their size against 0.0017 that storing them costs.
//
// Tried and left out (us, 512 after 16000, with what was there then): the two waves of a SIMD taking turns by barriers, three tiles in LDS, 315 / 358; the second four waves a product
// behind, 305 / 321; priorities, level; rows two tiles ahead in registers, 315 / 305 for bf16, but codes then spill; four waves a workgroup and two of those a unit, 315 / 367.
#include "paged_chunk.hpp"

namespace halo {

int check_paged_shape(const halo_paged_shape *s);
int launch_chunk_bf16(const ChunkArgs &a, hipStream_t s) { return launch_chunk_dim<KindBf16>(a, s); }

namespace {

inline size_t align256(size_t n) { return (n + 255) / 256 * 256; }
constexpr int kMostSeqs = 4096, kMostTokens = 1 << 21;

// What cut blocks leave, and with a mask the rows that survive.
struct ChunkWorkspace {
    size_t part = 0, kept = 0, n_kept = 0, bytes = 0;
    ChunkWorkspace(const halo_paged_shape &s, int N, int n_seq)
    {
        part = align256((size_t)kPartRows * 2 * sizeof(float));
        kept = part + align256((size_t)kPartRows * s.head_dim * sizeof(float));
        n_kept = kept + align256((size_t)N * s.n_heads * sizeof(int32_t));
        bytes = n_kept + align256((size_t)n_seq * s.n_kv_heads * sizeof(int32_t));
    }
};

int chunk(const halo_paged_shape *shape, int32_t N, const void *q, int64_t q_stride, const void *k, const float *k_scale, const void *v,
          const float *v_scale, bool codes, int32_t n_seq, const int32_t *starts, const int32_t *table, const int32_t *lens, int32_t max_len,
          const uint8_t *mask, float scale, void *out, void *workspace, size_t ws_bytes, void *stream)
{
    if (const int rc = check_paged_shape(shape)) return rc;
    if (N < 0 || N > kMostTokens || n_seq < 0 || n_seq > kMostSeqs) return HALO_ERR_ARG;
    if (N == 0 || n_seq == 0) return HALO_OK;
    if (!q || !k || !v || !starts || !table || !lens || !out || (codes && (!k_scale || !v_scale))) return HALO_ERR_NULL;
    const halo_paged_shape &s = *shape;
    const int size = s.dtype == HALO_F32 ? 4 : 2;
    auto odd = [](const void *p, unsigned by) { return (reinterpret_cast<uintptr_t>(p) & (by - 1)) != 0; };
    if (max_len < 1 || max_len > s.max_pages * s.page_size || !std::isfinite(scale)) return HALO_ERR_ARG;
    if (q_stride < (int64_t)s.n_heads * s.head_dim || q_stride * size % 16 || odd(q, 16) || odd(k, 16) || odd(v, 16) || odd(out, 16) ||
        odd(workspace, 16) || odd(k_scale, 4) || odd(v_scale, 4) || odd(starts, 4) || odd(table, 4) || odd(lens, 4))
        return HALO_ERR_ARG;
    const ChunkWorkspace ws(s, N, n_seq);
    if (!workspace || ws_bytes < ws.bytes) return HALO_ERR_WORKSPACE;

    ChunkArgs a{};
    a.q = q; a.k = k; a.v = v; a.k_scale = k_scale; a.v_scale = v_scale;
    a.starts = starts; a.table = table; a.lens = lens; a.mask = mask; a.out = out;
    a.stats = static_cast<float *>(workspace);
    a.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + ws.part);
    a.kept = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + ws.kept);
    a.n_kept = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + ws.n_kept);
    a.q_stride = q_stride;
    a.pool = PagePool{s.n_pages, s.n_kv_heads, __builtin_ctz((unsigned)s.page_size)};
    a.N = N; a.n_seq = n_seq; a.n_heads = s.n_heads; a.group = s.n_heads / s.n_kv_heads; a.D = s.head_dim;
    a.max_pages = s.max_pages; a.max_len = max_len;
    a.scale2 = scale * 1.44269504088896341f;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (codes) return s.dtype == HALO_F32 ? launch_chunk_q8_f32(a, st) : launch_chunk_q8(a, st);
    return s.dtype == HALO_F32 ? launch_chunk_f32(a, st) : launch_chunk_bf16(a, st);
}

}  // namespace
}  // namespace halo

extern "C" size_t halo_paged_chunk_workspace_bytes(const halo_paged_shape *shape, int32_t N, int32_t n_seq)
{
    using namespace halo;
    if (check_paged_shape(shape) != HALO_OK || N < 0 || N > kMostTokens || n_seq < 0 || n_seq > kMostSeqs) return 0;
    return ChunkWorkspace(*shape, N, n_seq).bytes;
}

extern "C" int halo_paged_chunk_attention(const halo_paged_shape *shape, int32_t N, const void *q, int64_t q_stride, const void *k_pages,
                                          const void *v_pages, int32_t n_seq, const int32_t *starts, const int32_t *page_table,
                                          const int32_t *lens, int32_t max_len, const uint8_t *mask, float scale, void *out, void *workspace,
                                          size_t ws_bytes, void *stream)
{
    return halo::chunk(shape, N, q, q_stride, k_pages, nullptr, v_pages, nullptr, false, n_seq, starts, page_table, lens, max_len, mask, scale, out,
                       workspace, ws_bytes, stream);
}

extern "C" int halo_paged_chunk_attention_q8(const halo_paged_shape *shape, int32_t N, const void *q, int64_t q_stride, const int8_t *k_codes,
                                             const float *k_scales, const int8_t *v_codes, const float *v_scales, int32_t n_seq,
                                             const int32_t *starts, const int32_t *page_table, const int32_t *lens, int32_t max_len,
                                             const uint8_t *mask, float scale, void *out, void *workspace, size_t ws_bytes, void *stream)
{
    return halo::chunk(shape, N, q, q_stride, k_codes, k_scales, v_codes, v_scales, true, n_seq, starts, page_table, lens, max_len, mask, scale, out,
                       workspace, ws_bytes, stream);
}
